// Decode attention over the rows of a paged cache (bf16): one query per sequence, the G query heads of a KV head together.
//   S = K q^T  (16 rows x 8 heads per chain of products),  O^T += V^T P  (16 channels x 8 heads), on warp-level matrix products:
// the work is a stream of K and V past a handful of queries, bound by bandwidth, and these need neither shared memory nor a barrier
// between the two products.  Rows come from memory straight into the operands' registers, 16 bytes per load:
//   - the contraction over channels may run in any order, so the 8 channels that a lane's load brings are the ones that it holds of
//     two products' operands (four lanes read 64 bytes of a row, the q operand is dealt alike);
//   - V^T wants pairs of rows for one channel: a lane loads 8 channels of rows 2t, 2t + 1, 2t + 8, 2t + 9 and interleaves them, and the
//     product of number j takes channel j of every lane's 8 as its 16 channels.
// Work is dealt to warps: the list of all units' blocks of 16 rows, in equal shares, so that neither lengths that differ nor units that are
// short leave any idle (a block of four warps per unit and piece of it took 26 us for 512 units of 292 rows, 76 MB).  Twelve warps to
// an SM, 8 KB in flight for each: the next block's keys are asked for when the keys have been used, and so the values, across the
// ends of units.  16 rows never cross a page (pages are powers of two from 16); page numbers are read a block ahead of the rows.
// A unit's part of a share leaves its state, which another kernel joins (a unit that is whole may go to the output).
// Weights are rounded to bf16 for the second product and divided by the sum of the rounded ones.
#include "serve.cuh"

namespace kvm {
namespace serve {
namespace {

constexpr int WARPS = 4, NT = WARPS * 32, HEADS = 8, PER_SM = 3;
constexpr int MIN_BLOCKS = 2;               // fewest blocks of a warp's share (bounds the number of parts)
constexpr int KEPT = 1024;                  // items whose lengths are kept in shared memory
constexpr float LOWEST = -1e30f, RESCALE_STEP = 8.f;

struct Args {
    const __nv_bfloat16* q;                 // [units, G, D]
    Keys k;
    States st;
    Beside pre;
    __nv_bfloat16* out;                     // null: whole units leave states too
    kvm_stats* stats;
    int G, HG, items;                       // groups of up to 8 heads of a unit; items = units x groups
    float scale2;
};

__device__ __forceinline__ void mma16816(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transpose8x8(uint32_t x) {
    uint32_t r;
    asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(x));
    return r;
}
__device__ __forceinline__ float ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ uint32_t word(const uint4& v, int i) { return i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w; }

// Where a warp stands in the list of blocks.
struct Cursor {
    int item, b, blocks, n;                 // block b of `blocks` of item's unit, which has n rows
    int left;                               // blocks of the share from this one on; 0: past the end
};

template <int D> __global__ void __launch_bounds__(NT, PER_SM) rows_paged_kernel(const Args a) {
    constexpr int KC = D / 32;                      // 16-byte loads per key row and lane
    constexpr int VC = D / 64;                      // ... per value row
    constexpr int MT = D / 16;                      // products of 16 channels
    __shared__ long long sm_all[WARPS];
    __shared__ int sm_sum[WARPS], sm_start, sm_item, sm_rows[KEPT];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, gid = lane >> 2, tig = lane & 3;
    if (!a.pre.units) grid_dependency_wait();       // (beside a prefix: when that kernel lets this one begin, what comes before it is done)
    grid_launch_dependents();                       // (who joins is there when this kernel ends, and waits for that)

    // ---- this block's share, by a prefix sum over the items
    // (in 32 bits: the host has seen to it)
    const bool kept = a.items <= KEPT;
    auto rows_of = [&](int item) { return kept ? sm_rows[item] : a.k.rows_of(item / a.HG); };
    auto blocks_of = [&](int item) { return (a.k.rows_of(item / a.HG) + 15) >> 4; };
    const int E = (a.items + NT - 1) / NT, i0 = min(a.items, (int)threadIdx.x * E), i1 = min(a.items, i0 + E);
    int mine = 0;
    for (int i = i0; i < i1; ++i) {
        const int n = a.k.rows_of(i / a.HG);
        if (kept) sm_rows[i] = n;
        mine += (n + 15) >> 4;
    }
    int inc = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int t = __shfl_up_sync(0xffffffffu, inc, o);
        if (lane >= o) inc += t;
    }
    if (lane == 31) sm_sum[warp] = inc;
    __syncthreads();
    int total = 0, before = inc - mine;
#pragma unroll
    for (int x = 0; x < WARPS; ++x) {
        if (x < warp) before += sm_sum[x];
        total += sm_sum[x];
    }
    // (beside a prefix these blocks have the SMs that it leaves; the other blocks have nothing to do)
    int ctas = gridDim.x;
    if (a.pre.units) ctas = min(ctas, PER_SM * (SMS - prefix_sms(block_sum<NT>(a.pre.part(NT), sm_all), total, D)));
    const int warps = ctas * WARPS, q = max((total + warps - 1) / warps, MIN_BLOCKS);
    const int f0 = (int)min((long long)total, (long long)blockIdx.x * WARPS * q), f1 = (int)min((long long)total, (long long)f0 + WARPS * q);
    const bool busy = (int)blockIdx.x < ctas && f0 < f1;
    if (busy && before <= f0 && f0 < before + mine) {                  // true in exactly one thread
        int st = before, id = i0;
        for (;; ++id) {
            const int n = kept ? (sm_rows[id] + 15) >> 4 : blocks_of(id);
            if (st + n > f0) break;
            st += n;
        }
        sm_start = st;
        sm_item = id;
    }
    __syncthreads();
    if (busy) {
        // ---- this warp's share
        int start = sm_start;                       // blocks before the cursor's item
        Cursor cur;
        const int w0 = min(f1, f0 + warp * q), w1 = min(f1, w0 + q);
        cur.item = sm_item;
        cur.n = rows_of(cur.item);
        cur.blocks = (cur.n + 15) >> 4;
        cur.left = w1 - w0;
        while (cur.left > 0 && start + cur.blocks <= w0) {
            start += cur.blocks;
            cur.n = rows_of(++cur.item);
            cur.blocks = (cur.n + 15) >> 4;
        }
        cur.b = w0 - start;
        auto advance = [&](Cursor c) {
            if (--c.left > 0 && ++c.b == c.blocks) {
                c.b = 0;
                do {
                    c.n = rows_of(++c.item);
                    c.blocks = (c.n + 15) >> 4;
                } while (c.blocks == 0);
            }
            return c;
        };
        const int bshift = a.k.shift - 4, bmask = (1 << bshift) - 1;        // blocks per page
        auto page_of = [&](const Cursor& c) {
            return c.left > 0 ? __ldg(a.k.table + (size_t)(c.item / a.HG) * a.k.max_pages + (c.b >> bshift)) : -1;
        };
        uint4 qf[KC], kf[2][KC], vf[4][VC];
        auto load_q = [&](const Cursor& c) {
            const int u = c.item / a.HG, h = (c.item - u * a.HG) * HEADS + gid;
#pragma unroll
            for (int i = 0; i < KC; ++i)
                qf[i] = h < a.G ? ldg16(a.q + ((size_t)u * a.G + h) * D + i * 32 + tig * 8) : make_uint4(0, 0, 0, 0);
        };
        // (a page that does not exist is not touched: what the registers hold is masked)
        auto load_k = [&](const Cursor& c, int page) {
            if (c.left <= 0 || (unsigned)page >= (unsigned)a.k.n_pages) return;
            const __nv_bfloat16* p = (const __nv_bfloat16*)a.k.K + ((((size_t)page << a.k.shift) + ((c.b & bmask) << 4) + gid) * D + tig * 8);
#pragma unroll
            for (int r = 0; r < 2; ++r)
#pragma unroll
                for (int i = 0; i < KC; ++i) kf[r][i] = ldg16(p + r * 8 * D + i * 32);
        };
        auto load_v = [&](const Cursor& c, int page) {
            if (c.left <= 0 || (unsigned)page >= (unsigned)a.k.n_pages) return;
            const __nv_bfloat16* p = (const __nv_bfloat16*)a.k.V + ((((size_t)page << a.k.shift) + ((c.b & bmask) << 4) + 2 * tig) * D + gid * 8);
#pragma unroll
            for (int r = 0; r < 4; ++r)
#pragma unroll
                for (int i = 0; i < VC; ++i) vf[r][i] = ldg16(p + ((r & 1) + (r >> 1) * 8) * D + i * 64);
        };
#pragma unroll
        for (int r = 0; r < 2; ++r)
#pragma unroll
            for (int i = 0; i < KC; ++i) kf[r][i] = make_uint4(0, 0, 0, 0);
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int i = 0; i < VC; ++i) vf[r][i] = make_uint4(0, 0, 0, 0);

        float o[MT][4];                             // channels of the lane's rows of product j, heads 2 tig, 2 tig + 1
        float m[2], l[2];
        auto reset = [&]() {
#pragma unroll
            for (int j = 0; j < MT; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e) o[j][e] = 0.f;
            m[0] = m[1] = LOWEST;
            l[0] = l[1] = 0.f;
        };
        reset();
        int page = page_of(cur), b_first = cur.b;   // b_first: the part's first block
        Cursor nxt = advance(cur);
        int page_next = page_of(nxt);
        load_k(cur, page);
        load_v(cur, page);
        load_q(cur);
        while (cur.left > 0) {
            const bool there = (unsigned)page < (unsigned)a.k.n_pages;
            const int live = there ? cur.n - cur.b * 16 : 0;       // rows that exist
            if (!there && a.stats) a.stats->status = KVM_E_PAGE;
            const bool last = nxt.left <= 0 || nxt.item != cur.item;
            float c0[4] = {0.f, 0.f, 0.f, 0.f}, c1[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int i = 0; i < KC; ++i) {
                mma16816(c0, kf[0][i].x, kf[1][i].x, kf[0][i].y, kf[1][i].y, qf[i].x, qf[i].y);
                mma16816(c1, kf[0][i].z, kf[1][i].z, kf[0][i].w, kf[1][i].w, qf[i].z, qf[i].w);
            }
            load_k(nxt, page_next);
            if (last && nxt.left > 0) load_q(nxt);
            float x[4];                             // rows gid, gid + 8; heads 2 tig, 2 tig + 1
#pragma unroll
            for (int e = 0; e < 4; ++e) x[e] = gid + (e >> 1) * 8 < live ? (c0[e] + c1[e]) * a.scale2 : -INFINITY;
            const float mx[2] = {fmaxf(x[0], x[2]), fmaxf(x[1], x[3])};
            if (__any_sync(0xffffffffu, mx[0] > m[0] + RESCALE_STEP || mx[1] > m[1] + RESCALE_STEP)) {
                float alpha[2];
#pragma unroll
                for (int y = 0; y < 2; ++y) {
                    float t = mx[y];
#pragma unroll
                    for (int z = 4; z < 32; z <<= 1) t = fmaxf(t, __shfl_xor_sync(0xffffffffu, t, z));
                    const float mn = fmaxf(t, m[y]);
                    alpha[y] = ex2(m[y] - mn);
                    m[y] = mn;
                    l[y] *= alpha[y];
                }
#pragma unroll
                for (int j = 0; j < MT; ++j)
#pragma unroll
                    for (int e = 0; e < 4; ++e) o[j][e] *= alpha[e & 1];
            }
            uint32_t pr[2];
#pragma unroll
            for (int y = 0; y < 2; ++y) {
                pr[y] = Vec<__nv_bfloat16>::pack2(ex2(x[2 * y] - m[0]), ex2(x[2 * y + 1] - m[1]));
                l[0] += __uint_as_float(pr[y] << 16);
                l[1] += __uint_as_float(pr[y] & 0xffff0000u);
                pr[y] = transpose8x8(pr[y]);
            }
            if (live < 16) {                        // rows that do not exist may hold anything: zeros
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    if (2 * tig + (r & 1) + (r >> 1) * 8 >= live)
#pragma unroll
                        for (int i = 0; i < VC; ++i) vf[r][i] = make_uint4(0, 0, 0, 0);
            }
            // product j: channels gid * 8 + j and 64 + gid * 8 + j (D = 64: gid * 8 + j and gid * 8 + 4 + j)
#pragma unroll
            for (int j = 0; j < MT; ++j) {
                const int j1 = D == 128 ? j : j + 4, c1i = D == 128 ? 1 : 0;
                const uint32_t s0 = j & 1 ? 0x7632 : 0x5410;
                mma16816(o[j], __byte_perm(word(vf[0][0], j / 2), word(vf[1][0], j / 2), s0),
                         __byte_perm(word(vf[0][c1i], j1 / 2), word(vf[1][c1i], j1 / 2), s0),
                         __byte_perm(word(vf[2][0], j / 2), word(vf[3][0], j / 2), s0),
                         __byte_perm(word(vf[2][c1i], j1 / 2), word(vf[3][c1i], j1 / 2), s0), pr[0], pr[1]);
            }
            load_v(nxt, page_next);
            if (last) {                             // the part's end: its state, or the output
                const int u = cur.item / a.HG, h0 = (cur.item - u * a.HG) * HEADS;
                const bool whole = b_first == 0 && cur.b == cur.blocks - 1;
#pragma unroll
                for (int y = 0; y < 2; ++y)
#pragma unroll
                    for (int z = 4; z < 32; z <<= 1) l[y] += __shfl_xor_sync(0xffffffffu, l[y], z);
                const int w = blockIdx.x * WARPS + warp;
                if (b_first == 0 && lane == 0) {
                    // parts after the first one begin at the next warps' shares
                    const int begin = w1 - cur.left - cur.b, last_w = (begin + cur.blocks - 1) / q;
                    a.st.pieces[cur.item] = make_int4(last_w - w + 1, cur.item, a.items + w + 1, 0);
                }
                const size_t slot = b_first == 0 ? cur.item : a.items + w;
#pragma unroll
                for (int y = 0; y < 2; ++y) {
                    const int h = 2 * tig + y;
                    if (h0 + h >= a.G) break;
                    if (whole && a.out) {
                        const float f = l[y] == 0.f ? 0.f : 1.f / l[y];
                        __nv_bfloat16* dst = a.out + ((size_t)u * a.G + h0 + h) * D + gid * 8;
                        float z[8];
#pragma unroll
                        for (int s = 0; s < VC; ++s) {
#pragma unroll
                            for (int j = 0; j < 8; ++j) {
                                const float v = D == 128 ? o[j % MT][2 * s + y] : o[j % 4][2 * (j / 4) + y];
                                z[j] = f != 0.f ? v * f : 0.f;
                            }
                            *reinterpret_cast<uint4*>(dst + s * 64) = Vec<__nv_bfloat16>::pack(z);
                        }
                    } else {
                        const size_t r = slot * a.st.rows + h;
                        float* dst = a.st.o + r * D + gid * 8;
#pragma unroll
                        for (int s = 0; s < VC; ++s)
#pragma unroll
                            for (int j = 0; j < 8; j += 4) {
                                float z[4];
#pragma unroll
                                for (int i = 0; i < 4; ++i) z[i] = D == 128 ? o[(j + i) % MT][2 * s + y] : o[i][2 * (j / 4) + y];
                                *reinterpret_cast<float4*>(dst + s * 64 + j) = make_float4(z[0], z[1], z[2], z[3]);
                            }
                        if (gid == 0) a.st.ml[r] = make_float4(m[y], l[y], l[y], 0.f);
                    }
                }
                reset();
                b_first = nxt.b;
            }
            cur = nxt;
            page = page_next;
            nxt = advance(nxt);
            page_next = page_of(nxt);
        }
    }
    if (a.pre.units) grid_dependency_wait();        // (who joins waits for this kernel, and thereby for the prefix's)
}

}  // namespace

// (148 SMs; as many blocks as a share of MIN_BLOCKS per warp needs at most.)
PagedPlan paged_plan(const Shape& s, int rows, bool beside_prefix) {
    PagedPlan p;
    p.hg = (s.G + HEADS - 1) / HEADS;
    p.items = s.U * p.hg;
    const long long most = ((long long)p.items * ((rows + 15) / 16) + MIN_BLOCKS * WARPS - 1) / (MIN_BLOCKS * WARPS);
    const int sms = beside_prefix ? OWN_MOST : SMS;
    p.grid = (int)(most < PER_SM * sms ? most : PER_SM * sms);
    p.slots = p.items + p.grid * WARPS + 1;
    p.slot_rows = s.G < HEADS ? s.G : HEADS;
    return p;
}

cudaError_t launch_rows_paged(const Shape& s, const PagedPlan& plan, const void* q, const Keys& k, const Beside& pre, const States& states, void* out,
                              kvm_stats* stats, cudaStream_t st) {
    const Args a = {(const __nv_bfloat16*)q, k, states, pre, (__nv_bfloat16*)out, stats, s.G, plan.hg, plan.items, s.scale * LOG2E};
    return launch_dependent(s.D == 128 ? rows_paged_kernel<128> : rows_paged_kernel<64>, dim3(plan.grid), dim3(NT), 0, st, a);
}

}  // namespace serve
}  // namespace kvm
