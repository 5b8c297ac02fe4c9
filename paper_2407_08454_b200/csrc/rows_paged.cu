// Decode attention over the rows of a paged cache (bf16): one query per sequence, the G query heads of a KV head together.
//   S = K q^T  (16 rows x 8 heads per chain of products),  O^T += V^T P  (16 channels x 8 heads), on warp-level matrix products:
// the work is a stream of K and V past a handful of queries, bound by bandwidth, and these need neither tensor memory nor a barrier
// between the two products.
// Work is dealt to warps: the list of all units' blocks of 16 rows, in equal shares, so that neither lengths that differ nor units that are
// short leave any idle (a block of four warps per unit and piece of it took 26.5 us for 512 units of 292 rows, 76 MB; this 20.5, of which the
// stream is 12).
// A warp copies its own blocks into a ring of its own (TMA, 128-byte swizzle, so that ldmatrix meets no bank conflict), STAGES ahead
// across the ends of units, and waits for nobody else: 192 KB are in flight per SM.  (Straight from memory into the operands'
// registers, 8 KB in flight for each of twelve warps: as fast on all SMs, but half the rate per SM, which counts beside a prefix.)
// 16 rows never cross a page (pages are powers of two from 16); page numbers are read a block ahead of the copies.
// A prefix may be folded in: its rows are then the first of every unit (read once per sequence, through L2).
// A unit's part of a share leaves its state, which another kernel joins (a unit that is whole may go to the output).  Where units are few or
// short each has a block of its own instead, and no second kernel.
// Weights are rounded to bf16 for the second product and divided by the sum of the rounded ones.  (Error of the output against 64 bits, its own
// rounding to bf16 being 1.66e-3 of it: 1.76e-3 with peaked weights, 2.33e-3 with flat ones.  With what the rounding leaves in a second product it
// is 1.66e-3, and calls take 1 to 5 % longer: 32 units x 512 rows 8.9 -> 9.3 us, 16 x 8 x 16384 180 -> 182.)
#include <float.h>

#include <mutex>

#include "serve.cuh"
#include "tc_common.cuh"

namespace kvm {
namespace serve {
namespace {

using namespace tc;

constexpr int WARPS = 4, NT = WARPS * 32, HEADS = 8, PER_SM = 2;
constexpr int STAGE_ROWS = 16;
template <int D> constexpr int stages() { return D == 128 ? 3 : 6; }      // 24 KB per warp
constexpr int RING_BYTES = 3 * 8192;
constexpr int MIN_BLOCKS = 2;               // fewest blocks of a warp's share (bounds the number of parts)
constexpr int KEPT = 1024;                  // items whose lengths are kept in shared memory
constexpr float LOWEST = -FLT_MAX, RESCALE_STEP = 8.f;      // (LOWEST: the reference before the first row, which any logit outgrows)

struct Args {
    const __nv_bfloat16* q;                 // [units, G, D]
    Keys k;
    Fold fold;
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
__device__ __forceinline__ void ldsm4(uint32_t (&r)[4], uint32_t addr) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ldsm4_t(uint32_t (&r)[4], uint32_t addr) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
// Where a warp stands in the list of blocks.
struct Cursor {
    int item, b, blocks, n, np;             // block b of `blocks` of item's unit, which has n rows of its own, behind np of a folded prefix
    int left;                               // blocks of the share from this one on; 0: past the end
};

// ALONE: a block per item, its warps on a quarter of the unit's blocks each, whose states are joined in shared memory: no second kernel.
template <int D, bool ALONE> __global__ void __launch_bounds__(NT, PER_SM)
rows_paged_kernel(const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v, const __grid_constant__ CUtensorMap map_pk,
                  const __grid_constant__ CUtensorMap map_pv, const __grid_constant__ Args a) {
    constexpr int STAGES = stages<D>(), KCH = D / 64;              // 64-channel (128-byte) column chunks
    constexpr uint32_t CHUNK = STAGE_ROWS * 128, TENSOR = KCH * CHUNK, STAGE = 2 * TENSOR;       // bytes of a chunk, of K or V, of a stage
    constexpr int MT = D / 16;                      // products of 16 channels
    extern __shared__ uint8_t smem_raw[];
    __shared__ __align__(8) uint64_t full[WARPS][STAGES];
    __shared__ volatile int s_bad;
    constexpr int LENGTHS = ALONE ? 1 : KEPT;
    __shared__ long long sm_all[WARPS];
    __shared__ int sm_sum[WARPS], sm_start, sm_item, sm_rows[LENGTHS], sm_pre[LENGTHS];
    __shared__ float sm_ml[WARPS][HEADS][2];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, gid = lane >> 2, tig = lane & 3;
    if (threadIdx.x == 0) {
        for (int w = 0; w < WARPS; ++w)
            for (int i = 0; i < STAGES; ++i) mbar_init(&full[w][i], 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        s_bad = 0;
        asm volatile("prefetch.tensormap [%0];" ::"l"(&map_k) : "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(&map_v) : "memory");
        if (a.fold.rows) {
            asm volatile("prefetch.tensormap [%0];" ::"l"(&map_pk) : "memory");
            asm volatile("prefetch.tensormap [%0];" ::"l"(&map_pv) : "memory");
        }
    }
    if (!a.pre.units) grid_dependency_wait();       // (beside a prefix: when that kernel lets this one begin, what comes before it is done)
    grid_launch_dependents();                       // (who joins is there when this kernel ends, and waits for that)

    // ---- this block's share, by a prefix sum over the items
    // (in 32 bits: the host has seen to it)
    const bool kept = !ALONE && a.items <= KEPT;
    auto unit_of = [&](int item) { return a.HG == 1 ? item : item / a.HG; };
    auto own_of = [&](int item) { return a.k.table ? a.k.rows_of(unit_of(item)) : 0; };
    auto pre_of = [&](int item) { return a.fold.rows ? a.fold.rows_of(unit_of(item) % a.fold.heads) : 0; };
    auto rows_of = [&](int item) { return kept ? sm_rows[item] : own_of(item); };
    auto prefix_of = [&](int item) { return kept ? sm_pre[item] : pre_of(item); };
    auto blocks_of = [&](int item) { return ((rows_of(item) + 15) >> 4) + ((prefix_of(item) + 15) >> 4); };
    bool busy = true;
    int q = 0, f0 = 0, f1 = 0;
    if constexpr (ALONE) {
        __syncthreads();                            // (the barriers are there)
    } else {
        const int E = (a.items + NT - 1) / NT, i0 = min(a.items, (int)threadIdx.x * E), i1 = min(a.items, i0 + E);
        int mine = 0;
        for (int i = i0; i < i1; ++i) {
            const int n = own_of(i), np = pre_of(i);
            if (kept) { sm_rows[i] = n; sm_pre[i] = np; }
            mine += ((n + 15) >> 4) + ((np + 15) >> 4);
            if (blockIdx.x == 0 && n + np == 0) a.st.pieces[i] = make_int4(0, 0, 0, 0);
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
        const int warps = max(ctas, 1) * WARPS;                            // (without own rows the prefix has all SMs)
        q = max((total + warps - 1) / warps, MIN_BLOCKS);
        f0 = (int)min((long long)total, (long long)blockIdx.x * WARPS * q);
        f1 = (int)min((long long)total, (long long)f0 + WARPS * q);
        busy = (int)blockIdx.x < ctas && f0 < f1;
        if (busy && before <= f0 && f0 < before + mine) {                  // true in exactly one thread
            int st = before, id = i0;
            for (;; ++id) {
                const int n = blocks_of(id);
                if (st + n > f0) break;
                st += n;
            }
            sm_start = st;
            sm_item = id;
        }
        __syncthreads();
    }
    if (busy) {
        // ---- this warp's share
        Cursor cur;
        auto settle = [&](Cursor& c) {
            c.n = rows_of(c.item);
            c.np = prefix_of(c.item);
            c.blocks = ((c.n + 15) >> 4) + ((c.np + 15) >> 4);
        };
        int w1;                                     // where this warp's share ends
        if constexpr (ALONE) {
            cur.item = blockIdx.x;
            settle(cur);
            cur.b = cur.blocks * warp / WARPS;
            w1 = cur.blocks * (warp + 1) / WARPS;
            cur.left = w1 - cur.b;
        } else {
            int start = sm_start;                   // blocks before the cursor's item
            const int w0 = min(f1, f0 + warp * q);
            w1 = min(f1, w0 + q);
            cur.item = sm_item;
            settle(cur);
            cur.left = w1 - w0;
            while (cur.left > 0 && start + cur.blocks <= w0) {
                start += cur.blocks;
                ++cur.item;
                settle(cur);
            }
            cur.b = w0 - start;
        }
        [[maybe_unused]] const int share = cur.left;
        auto advance = [&](Cursor c) {
            if (--c.left > 0 && ++c.b == c.blocks) {
                c.b = 0;
                do {
                    ++c.item;
                    settle(c);
                } while (c.blocks == 0);
            }
            return c;
        };
        const int bshift = a.k.shift - 4, bmask = (1 << bshift) - 1;        // blocks per page
        // of a block of own rows its page, of one of the folded prefix its first row in the prefix's tensor
        auto page_of = [&](const Cursor& c) {
            if (c.left <= 0) return -1;
            const int u = unit_of(c.item), b = c.b - ((c.np + 15) >> 4);
            return b < 0 ? u % a.fold.heads * a.fold.rows + c.b * 16 : __ldg(a.k.table + (size_t)u * a.k.max_pages + (b >> bshift));
        };
        auto folded = [&](const Cursor& c) { return c.b < ((c.np + 15) >> 4); };
        auto exists = [&](const Cursor& c, int page) { return folded(c) || (unsigned)page < (unsigned)a.k.n_pages; };
        const uint32_t ring = ((smem_u32(smem_raw) + 1023u) & ~1023u) + warp * RING_BYTES;
        uint8_t* ring_at = smem_raw + (ring - smem_u32(smem_raw));
        uint32_t qf[D / 16][2];                     // q^T as the second operand: channels 2 tig.. (+ 8) of head gid
        auto load_q = [&](const Cursor& c) {
            const int u = unit_of(c.item), h = (c.item - u * a.HG) * HEADS + gid;
            const uint32_t* p = reinterpret_cast<const uint32_t*>(a.q + ((size_t)u * a.G + h) * D) + tig;
#pragma unroll
            for (int ks = 0; ks < D / 16; ++ks) {
                qf[ks][0] = h < a.G ? __ldg(p + ks * 8) : 0u;
                qf[ks][1] = h < a.G ? __ldg(p + ks * 8 + 4) : 0u;
            }
        };
        // (a page that does not exist is not touched: the stage is full at once, and what it holds is masked)
        auto issue = [&](const Cursor& c, int page, int s) {
            if (c.left <= 0 || lane != 0) return;
            uint64_t* bar = &full[warp][s];
#ifdef KVM_TEST_DROP_ATTEND_STAGE
            if (blockIdx.x == KVM_TEST_DROP_CTA && warp == 0 && c.left == share - (KVM_TEST_DROP_ATTEND_STAGE)) return;   // test build only: this block never arrives
#endif
            if (!exists(c, page)) {
                mbar_arrive(bar);
                return;
            }
            mbar_expect_tx(bar, STAGE);
            const bool pre = folded(c);
            const int row = pre ? page : (page << a.k.shift) + (((c.b - ((c.np + 15) >> 4)) & bmask) << 4);
            const CUtensorMap *mk = pre ? &map_pk : &map_k, *mv = pre ? &map_pv : &map_v;
            // (both column chunks in one copy: the thread that issues is one of those that compute)
            tma_load_3d(ring_at + s * STAGE, mk, bar, 0, row, 0);
            tma_load_3d(ring_at + s * STAGE + TENSOR, mv, bar, 0, row, 0);
        };
        float o[MT][4];                             // channels of product j: 16 j + gid (+ 8), heads 2 tig, 2 tig + 1
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
        const int krow = lane & 15, kpc = lane >> 4, vrow = (lane & 7) + ((lane >> 4) << 3), vpc = (lane >> 3) & 1;
        int b_first = cur.b;                        // the part's first block
        Cursor ld = cur;                            // the next block to copy
        int page = page_of(ld);
        uint32_t there_bits = 0, phase = 0;         // of the stages: whether the page exists, the barrier's parity
        auto copy_next = [&](int s) {
            issue(ld, page, s);
            there_bits = (there_bits & ~(1u << s)) | (exists(ld, page) ? 1u << s : 0u);
            ld = advance(ld);
            page = page_of(ld);
        };
#pragma unroll 1
        for (int s = 0; s < STAGES; ++s) copy_next(s);
        load_q(cur);
        int s = 0;
        bool ok = true;
        while (cur.left > 0) {
            const bool there = there_bits >> s & 1;
            const int live = !there ? 0 : folded(cur) ? cur.np - cur.b * 16 : cur.n - (cur.b - ((cur.np + 15) >> 4)) * 16;    // rows that exist
            if (!there && a.stats) a.stats->status = KVM_E_PAGE;
            const Cursor nxt = advance(cur);
            const bool last = nxt.left <= 0 || nxt.item != cur.item;
            // (the warp's own copies always complete; a wait that ran out all the same makes the part NaN)
            ok = ok && __all_sync(0xffffffffu, mbar_wait(&full[warp][s], phase >> s & 1, &s_bad));
            phase ^= 1u << s;
            const uint32_t kb = ring + s * STAGE, vb = kb + TENSOR;
            float c0[4] = {0.f, 0.f, 0.f, 0.f}, c1[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int ks = 0; ks < D / 16; ++ks) {
                uint32_t f[4];
                ldsm4(f, kb + (ks / 4) * CHUNK + krow * 128 + ((((ks % 4) * 2 + kpc) ^ (krow & 7)) << 4));
                mma16816(ks & 1 ? c1 : c0, f[0], f[1], f[2], f[3], qf[ks][0], qf[ks][1]);
            }
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
            // rows that do not exist may hold anything: their V becomes zero (masks of the operand's rows 2 tig.. + 8)
            uint32_t mask[2] = {0xffffffffu, 0xffffffffu};
            if (live < 16)
#pragma unroll
                for (int y = 0; y < 2; ++y)
                    mask[y] = (2 * tig + y * 8 < live ? 0xffffu : 0u) | (2 * tig + 1 + y * 8 < live ? 0xffff0000u : 0u);
#pragma unroll
            for (int j = 0; j < MT; ++j) {
                uint32_t f[4];
                ldsm4_t(f, vb + (j / 4) * CHUNK + vrow * 128 + ((((j % 4) * 2 + vpc) ^ (vrow & 7)) << 4));
                if (live < 16) { f[0] &= mask[0]; f[1] &= mask[0]; f[2] &= mask[1]; f[3] &= mask[1]; }
                mma16816(o[j], f[0], f[1], f[2], f[3], pr[0], pr[1]);
            }
            __syncwarp();                           // (all lanes have read the stage)
            if (ok) copy_next(s);
            if (last) {                             // the part's end: its state, or the output
                const int u = unit_of(cur.item), h0 = (cur.item - u * a.HG) * HEADS;
                const bool whole = b_first == 0 && cur.b == cur.blocks - 1;
#pragma unroll
                for (int y = 0; y < 2; ++y) {
#pragma unroll
                    for (int z = 4; z < 32; z <<= 1) l[y] += __shfl_xor_sync(0xffffffffu, l[y], z);
                    if (!ok) l[y] = NAN;
                }
                if constexpr (ALONE) {                   // (all of the warp's copies have been used: the ring's memory takes the state)
                    float* so = reinterpret_cast<float*>(ring_at);
#pragma unroll
                    for (int y = 0; y < 2; ++y) {
#pragma unroll
                        for (int j = 0; j < MT; ++j)
#pragma unroll
                            for (int e = 0; e < 2; ++e) so[(2 * tig + y) * D + j * 16 + e * 8 + gid] = o[j][2 * e + y];
                        if (gid == 0) { sm_ml[warp][2 * tig + y][0] = m[y]; sm_ml[warp][2 * tig + y][1] = l[y]; }
                    }
                    break;
                }
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
                        __nv_bfloat16* dst = a.out + ((size_t)u * a.G + h0 + h) * D + gid;
#pragma unroll
                        for (int j = 0; j < MT; ++j)
#pragma unroll
                            for (int e = 0; e < 2; ++e) dst[j * 16 + e * 8] = __float2bfloat16_rn(f != 0.f ? o[j][2 * e + y] * f : 0.f);
                    } else {
                        const size_t r = slot * a.st.rows + h;
                        float* dst = a.st.o + r * D + gid;
#pragma unroll
                        for (int j = 0; j < MT; ++j)
#pragma unroll
                            for (int e = 0; e < 2; ++e) dst[j * 16 + e * 8] = o[j][2 * e + y];
                        if (gid == 0) a.st.ml[r] = make_float4(m[y], l[y], l[y], 0.f);
                    }
                }
                reset();
                b_first = nxt.b;
            }
            cur = nxt;
            s = s + 1 == STAGES ? 0 : s + 1;
        }
        if constexpr (ALONE) {
            if (share == 0 && lane < HEADS) { sm_ml[warp][lane][0] = LOWEST; sm_ml[warp][lane][1] = 0.f; }
            __syncthreads();
            const int item = blockIdx.x, u = item / a.HG, h0 = (item - u * a.HG) * HEADS, heads = min(a.G - h0, HEADS);
            const float* all = reinterpret_cast<const float*>(ring_at - warp * RING_BYTES);
            for (int i = threadIdx.x; i < heads * D / 2; i += NT) {
                const int h = i / (D / 2), c = i % (D / 2) * 2;
                float M = LOWEST, L = 0.f, y0 = 0.f, y1 = 0.f;
#pragma unroll
                for (int x = 0; x < WARPS; ++x) M = fmaxf(M, sm_ml[x][h][0]);
#pragma unroll
                for (int x = 0; x < WARPS; ++x) {
                    if (sm_ml[x][h][1] == 0.f) continue;          // (a warp without rows)
                    const float f = ex2(sm_ml[x][h][0] - M);
                    const float2 v = *reinterpret_cast<const float2*>(all + x * (RING_BYTES / 4) + h * D + c);
                    L = fmaf(sm_ml[x][h][1], f, L);
                    y0 = fmaf(v.x, f, y0);
                    y1 = fmaf(v.y, f, y1);
                }
                const float f = L == 0.f ? 0.f : 1.f / L;
                *reinterpret_cast<uint32_t*>(a.out + ((size_t)u * a.G + h0 + h) * D + c) =
                    Vec<__nv_bfloat16>::pack2(f != 0.f ? y0 * f : 0.f, f != 0.f ? y1 * f : 0.f);
            }
        }
        if (!ok) {
            // copies in flight land before shared memory is given back (bounded)
            if (a.stats) a.stats->status = KVM_E_DEVICE_TIMEOUT;
            for (int i = 0; i < STAGES; ++i)
                for (uint32_t it = 0; it < (1u << 12); ++it)
                    if (mbar_try(&full[warp][i], phase >> i & 1)) break;
        }
    }
    if (a.pre.units) grid_dependency_wait();        // (who joins waits for this kernel, and thereby for the prefix's)
}

// Rows (all pages', or a prefix's of all heads) as a tensor [D / 64, rows, 64], boxes of [all, 16 rows, 64 channels]: the column chunks of 16 rows
// one after the other.
bool make_pool_map(CUtensorMap* map, const void* ptr, long long rows, int D) {
    EncodeTiledFn fn = encode_fn();
    if (!fn) return false;
    cuuint64_t dims[3] = {64, (cuuint64_t)rows, (cuuint64_t)(D / 64)};
    cuuint64_t strides[2] = {(cuuint64_t)D * 2, 128};
    cuuint32_t box[3] = {64, STAGE_ROWS, (cuuint32_t)(D / 64)};
    cuuint32_t estr[3] = {1, 1, 1};
    return fn(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(ptr), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
              CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_128B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int D, bool ALONE> cudaError_t launch_t(const PagedPlan& plan, const Args& a, cudaStream_t st) {
    constexpr size_t smem = 1024 + WARPS * RING_BYTES;
    static std::mutex mu;
    static bool ready[KVM_MAX_DEVICES] = {};
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev < 0 || dev >= KVM_MAX_DEVICES) return cudaErrorInvalidDevice;
    {
        std::lock_guard<std::mutex> lock(mu);
        if (!ready[dev]) {
            if ((e = cudaFuncSetAttribute(rows_paged_kernel<D, ALONE>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem)) != cudaSuccess) return e;
            ready[dev] = true;
        }
    }
    CUtensorMap mk, mv, pk, pv;
    const long long pool = (long long)a.k.n_pages << a.k.shift, prefix = (long long)a.fold.heads * a.fold.rows;
    if (a.k.table && (!make_pool_map(&mk, a.k.K, pool, D) || !make_pool_map(&mv, a.k.V, pool, D))) return cudaErrorNotSupported;
    if (prefix && (!make_pool_map(&pk, a.fold.K, prefix, D) || !make_pool_map(&pv, a.fold.V, prefix, D))) return cudaErrorNotSupported;
    if (!a.k.table) { mk = pk; mv = pv; }           // (never read from)
    if (!prefix) { pk = mk; pv = mv; }
    return launch_dependent(rows_paged_kernel<D, ALONE>, dim3(plan.grid), dim3(NT), smem, st, mk, mv, pk, pv, a);
}

}  // namespace

// A block per unit where its four warps are not long at it: nothing is joined by a second kernel.  (The host knows the room, not the lengths; tables
// were as wide as these need.  us, shares / alone, lengths in the upper half of `rows`, 128 channels: 32 units x 256 rows 9.9 / 6.0, x 512 11.2 / 9.0, x 1024 11.0 / 17.3; 128 x 256 11.6 / 5.9, x 1024 19.4 / 18.6, x 2048 26.3 /
// 32.9; 256 x 512 18.5 / 13.7, x 1024 25.7 / 22.3; 512 x 512 27.3 / 24.1; 768 x 256 25.3 / 22.9.  64 channels: 32 x 512 9.7 / 8.6, 128 x 1024 14.1 /
// 15.0, 256 x 1024 20.4 / 17.5.)
static bool alone(int items, int rows) { return items <= 6 * SMS && (rows <= 512 || (items > SMS && rows <= 1024)); }

// (148 SMs; as many blocks as a share of MIN_BLOCKS per warp needs at most.)
PagedPlan paged_plan(const Shape& s, int rows, bool beside_prefix) {
    PagedPlan p;
    p.hg = (s.G + HEADS - 1) / HEADS;
    p.items = s.U * p.hg;
    const long long most = ((long long)p.items * ((rows + 15) / 16) + MIN_BLOCKS * WARPS - 1) / (MIN_BLOCKS * WARPS);
    const int sms = beside_prefix ? OWN_MOST : SMS;
    p.grid = (int)(most < PER_SM * sms ? most : PER_SM * sms);
    p.alone = !beside_prefix && alone(p.items, rows);
    if (p.alone) p.grid = p.items;
    p.slots = p.items + p.grid * WARPS + 1;
    p.slot_rows = s.G < HEADS ? s.G : HEADS;
    return p;
}

cudaError_t launch_rows_paged(const Shape& s, const PagedPlan& plan, const void* q, const Keys& k, const Fold& fold, const Beside& pre, const States& states, void* out,
                              kvm_stats* stats, cudaStream_t st) {
    const Args a = {(const __nv_bfloat16*)q, k, fold, states, pre, (__nv_bfloat16*)out, stats, s.G, plan.hg, plan.items, s.scale * LOG2E};
    return plan.alone ? (s.D == 128 ? launch_t<128, true>(plan, a, st) : launch_t<64, true>(plan, a, st))
                      : (s.D == 128 ? launch_t<128, false>(plan, a, st) : launch_t<64, false>(plan, a, st));
}

}  // namespace serve
}  // namespace kvm
