// Decode attention over the rows of a paged cache (bf16): one query per sequence, the G query heads of a KV head together.
//   S = K q^T  (16 rows x 8 heads per chain of products),  O^T += V^T P  (16 channels x 8 heads), on warp-level matrix products:
// the work is a stream of K and V past a handful of queries, bound by bandwidth, and these need neither shared memory nor a barrier
// between the two products.  Rows come from memory straight into the operands' registers, 16 bytes per load:
//   - the contraction over channels may run in any order, so the 8 channels that a lane's load brings are the ones that it holds of
//     two products' operands (four lanes read 64 bytes of a row, the q operand is dealt alike);
//   - V^T wants pairs of rows for one channel: a lane loads 8 channels of rows 2t, 2t + 1, 2t + 8, 2t + 9 and interleaves them, and the
//     product of number j takes channel j of every lane's 8 as its 16 channels.
// A block is four warps that take 16 rows in turn, three blocks to an SM, 8 KB in flight per warp: the next rows' keys are asked for when
// the keys have been used, and so the values.  16 rows never cross a page (pages are powers of two from 16); page numbers are read
// two rounds ahead.  The rows of a unit are cut into pieces, whose states another kernel joins; shares follow the lengths.
// Weights are rounded to bf16 for the second product and divided by the sum of the rounded ones.
#include "serve.cuh"

namespace kvm {
namespace serve {
namespace {

constexpr int WARPS = 4, NT = WARPS * 32, HEADS = 8;
constexpr float LOWEST = -1e30f, RESCALE_STEP = 8.f;

struct Args {
    const __nv_bfloat16* q;                 // [units, G, D]
    Keys k;
    States st;                              // o null: the output
    __nv_bfloat16* out;
    kvm_stats* stats;
    int G, pieces;
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

template <int D> __global__ void __launch_bounds__(NT, 3) rows_paged_kernel(const Args a) {
    constexpr int KC = D / 32;                      // 16-byte loads per key row and lane
    constexpr int VC = D / 64;                      // ... per value row
    constexpr int MT = D / 16;                      // products of 16 channels
    __shared__ float sm_o[WARPS][HEADS][D], sm_m[WARPS][HEADS], sm_l[WARPS][HEADS];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, gid = lane >> 2, tig = lane & 3;
    const int u = blockIdx.z, h0 = blockIdx.x * HEADS, heads = min(a.G - h0, HEADS);
    grid_dependency_wait();

    // this block's rows: its share of the unit's blocks of 16
    const int n = a.k.rows_of(u), blocks = (n + 15) >> 4;
    const int b0 = (int)((long long)blockIdx.y * blocks / a.pieces), b1 = (int)((long long)(blockIdx.y + 1) * blocks / a.pieces);
    const int32_t* table = a.k.table + (size_t)u * a.k.max_pages;
    const int bshift = a.k.shift - 4, bmask = (1 << bshift) - 1;        // blocks per page
    auto page_of = [&](int b) { return b < b1 ? __ldg(table + (b >> bshift)) : -1; };

    uint4 qf[KC];
#pragma unroll
    for (int c = 0; c < KC; ++c)
        qf[c] = gid < heads ? ldg16(a.q + ((size_t)u * a.G + h0 + gid) * D + c * 32 + tig * 8) : make_uint4(0, 0, 0, 0);

    uint4 kf[2][KC], vf[4][VC];
    // (a page that does not exist is not touched: what the registers hold is masked)
    auto load_k = [&](int b, int page) {
        if (b >= b1 || (unsigned)page >= (unsigned)a.k.n_pages) return;
        const __nv_bfloat16* p = (const __nv_bfloat16*)a.k.K + ((((size_t)page << a.k.shift) + ((b & bmask) << 4) + gid) * D + tig * 8);
#pragma unroll
        for (int r = 0; r < 2; ++r)
#pragma unroll
            for (int c = 0; c < KC; ++c) kf[r][c] = ldg16(p + r * 8 * D + c * 32);
    };
    auto load_v = [&](int b, int page) {
        if (b >= b1 || (unsigned)page >= (unsigned)a.k.n_pages) return;
        const __nv_bfloat16* p = (const __nv_bfloat16*)a.k.V + ((((size_t)page << a.k.shift) + ((b & bmask) << 4) + 2 * tig) * D + gid * 8);
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int c = 0; c < VC; ++c) vf[r][c] = ldg16(p + ((r & 1) + (r >> 1) * 8) * D + c * 64);
    };
#pragma unroll
    for (int r = 0; r < 2; ++r)
#pragma unroll
        for (int c = 0; c < KC; ++c) kf[r][c] = make_uint4(0, 0, 0, 0);
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int c = 0; c < VC; ++c) vf[r][c] = make_uint4(0, 0, 0, 0);

    float o[MT][4];                                 // channels of the lane's rows of product j, heads 2 tig, 2 tig + 1
#pragma unroll
    for (int j = 0; j < MT; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[j][e] = 0.f;
    float m[2] = {LOWEST, LOWEST}, l[2] = {0.f, 0.f};
    int b = b0 + warp, page = page_of(b), page_next = page_of(b + WARPS);
    load_k(b, page);
    load_v(b, page);
    for (; b < b1; b += WARPS) {
        const int page_after = page_of(b + 2 * WARPS);
        const bool there = (unsigned)page < (unsigned)a.k.n_pages;
        const int live = there ? n - b * 16 : 0;    // rows that exist
        if (!there && a.stats) a.stats->status = KVM_E_PAGE;
        float c0[4] = {0.f, 0.f, 0.f, 0.f}, c1[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int c = 0; c < KC; ++c) {
            mma16816(c0, kf[0][c].x, kf[1][c].x, kf[0][c].y, kf[1][c].y, qf[c].x, qf[c].y);
            mma16816(c1, kf[0][c].z, kf[1][c].z, kf[0][c].w, kf[1][c].w, qf[c].z, qf[c].w);
        }
        load_k(b + WARPS, page_next);
        float x[4];                                 // rows gid, gid + 8; heads 2 tig, 2 tig + 1
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
        if (live < 16) {                            // rows that do not exist may hold anything: zeros
#pragma unroll
            for (int r = 0; r < 4; ++r)
                if (2 * tig + (r & 1) + (r >> 1) * 8 >= live)
#pragma unroll
                    for (int c = 0; c < VC; ++c) vf[r][c] = make_uint4(0, 0, 0, 0);
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
        load_v(b + WARPS, page_next);
        page = page_next;
        page_next = page_after;
    }
    // ---- the warps' states, in order
#pragma unroll
    for (int y = 0; y < 2; ++y)
#pragma unroll
        for (int z = 4; z < 32; z <<= 1) l[y] += __shfl_xor_sync(0xffffffffu, l[y], z);
    if (gid == 0)
#pragma unroll
        for (int y = 0; y < 2; ++y) { sm_m[warp][2 * tig + y] = m[y]; sm_l[warp][2 * tig + y] = l[y]; }
#pragma unroll
    for (int j = 0; j < MT; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (2 * tig + (e & 1) < heads) sm_o[warp][2 * tig + (e & 1)][gid * 8 + j + (e >> 1) * (D == 128 ? 64 : 4)] = o[j][e];
    __syncthreads();
    for (int i = threadIdx.x; i < heads * D / 2; i += NT) {
        const int h = i / (D / 2), c = i % (D / 2) * 2;
        float M = LOWEST, L = 0.f, y0 = 0.f, y1 = 0.f;
#pragma unroll
        for (int w = 0; w < WARPS; ++w) M = fmaxf(M, sm_m[w][h]);
#pragma unroll
        for (int w = 0; w < WARPS; ++w) {
            const float f = sm_l[w][h] == 0.f ? 0.f : ex2(sm_m[w][h] - M);      // (a warp without rows weighs nothing)
            L = fmaf(sm_l[w][h], f, L);
            y0 = fmaf(sm_o[w][h][c], f, y0);
            y1 = fmaf(sm_o[w][h][c + 1], f, y1);
        }
        if (a.st.o) {
            const size_t r = ((size_t)u * a.pieces + blockIdx.y) * a.st.rows + h0 + h;
            *reinterpret_cast<float2*>(a.st.o + r * D + c) = make_float2(y0, y1);
            if (c == 0) a.st.ml[r] = make_float4(M, L, L, 0.f);
        } else {
            const float f = L == 0.f ? 0.f : 1.f / L;
            *reinterpret_cast<uint32_t*>(a.out + ((size_t)u * a.G + h0 + h) * D + c) =
                Vec<__nv_bfloat16>::pack2(f != 0.f ? y0 * f : 0.f, f != 0.f ? y1 * f : 0.f);
        }
    }
}

}  // namespace

// Pieces of a unit: four waves of blocks, so that units of different lengths end together, but none with less than 64 rows
// (a round of the block's four warps) where the unit is full.
int paged_pieces(const Shape& s, int rows) {
    const long long blocks = (long long)s.U * ((s.G + HEADS - 1) / HEADS), want = (148ll * 3 * 4 + blocks - 1) / blocks;
    const long long most = (rows + 63) / 64;
    const long long n = want < most ? want : most;
    return n < 1 ? 1 : (int)n;
}

cudaError_t launch_rows_paged(const Shape& s, int pieces, const void* q, const Keys& k, const States& states, void* out, kvm_stats* stats,
                              cudaStream_t st) {
    const Args a = {(const __nv_bfloat16*)q, k, states, (__nv_bfloat16*)out, stats, s.G, pieces, s.scale * LOG2E};
    const dim3 grid((s.G + HEADS - 1) / HEADS, pieces, s.U);
    return launch_dependent(s.D == 128 ? rows_paged_kernel<128> : rows_paged_kernel<64>, grid, dim3(NT), 0, st, a);
}

}  // namespace serve
}  // namespace kvm
