// Joins the states that pieces of a softmax have left, two sets of them if need be (a shared prefix and a sequence's own rows),
// into the rows of the output:  M = max m,  O = sum o 2^(m - M) / sum lr 2^(m - M),  lse = ln sum l 2^(m - M) + M ln 2.
// A warp per row; pieces are taken in order, several at a time so that their loads leave together: results are reproducible.
#include "serve.cuh"

namespace kvm {
namespace serve {
namespace {

constexpr int JOIN_NT = 128;

// A row's pieces in one set of states: `count` of them, in slots first, second, second + stride, ...
struct Pieces {
    int count, first, second, stride;
    const float* o;                             // the row's sums in slot 0, and how far slots lie apart (rows)
    const float4* ml;
    int pitch, half;                            // half: rows to a piece's second state (0: it has one)
    __device__ __forceinline__ long long at(int i) const {
        const int x = half ? i & 1 : 0;
        if (half) i >>= 1;
        return (long long)(i == 0 ? first : second + (i - 1) * stride) * pitch + x * half;
    }
};
template <int D> __device__ __forceinline__ Pieces pieces_of(const States& st, const int32_t* len, int unit, int m) {
    int item, row;
    st.find(m, item, row);
    const int at = unit * st.items + item;
    Pieces p;
    p.stride = st.stride;
    p.pitch = st.rows;
    p.o = st.o + (size_t)row * D;
    p.ml = st.ml + row;
    p.half = st.halves ? st.tile_room : 0;
    if (st.count > 0) {
        p.count = st.count;
        p.first = at * st.count;
        p.second = p.first + 1;
    } else {                                    // (both reads leave together; a unit without keys has no entry in the table)
        const int n = len ? __ldg(len + unit) : 1;
        const int4 pc = __ldcg(st.pieces + at);
        p.count = n > 0 ? pc.x << (st.halves ? 1 : 0) : 0;
        p.first = pc.y;
        p.second = pc.z;
    }
    return p;
}

template <int E> struct Sum {                   // E channels of a row
    float m, l, lr, o[E];
};

// One loop over the pieces of both sets, BATCH at a time so that their loads leave together.  (Short code: a launch of a few warps spends
// most of its time on fetching instructions.  With a copy of the loop for each set, and one for few and one for many pieces, 12.5 us for
// 32 rows of 12 pieces.)
// The warp is number `part` of `parts` that share the row, each taking a batch in turn.
constexpr int BATCH = 8;
template <int D> __device__ __forceinline__ Sum<D / 32> sum_pieces(const Pieces& a, const Pieces& b, int part, int parts) {
    constexpr int E = D / 32;
    const int lane = threadIdx.x & 31, count = a.count + b.count;
    Sum<E> s;
    s.m = -INFINITY;
    s.l = s.lr = 0.f;
#pragma unroll
    for (int e = 0; e < E; ++e) s.o[e] = 0.f;
#pragma unroll 1
    for (int i0 = part * BATCH; i0 < count; i0 += parts * BATCH) {
        float4 z[BATCH];
        float x[BATCH][E], mn = s.m;
#pragma unroll
        for (int i = 0; i < BATCH; ++i) {
            const int k = i0 + i;
            const bool in_a = k < a.count;
            const long long r = in_a ? a.at(k) : b.at(k - a.count);
            z[i] = make_float4(-INFINITY, 0.f, 0.f, 0.f);
#pragma unroll
            for (int e = 0; e < E; ++e) x[i][e] = 0.f;
            if (k < count) {
                z[i] = __ldcg((in_a ? a.ml : b.ml) + r);
                const float* o = (in_a ? a.o : b.o) + r * D;
                if (E == 4) {
                    const float4 v = __ldcg(reinterpret_cast<const float4*>(o) + lane);
                    x[i][0] = v.x; x[i][1] = v.y; x[i][E - 2] = v.z; x[i][E - 1] = v.w;
                } else {
                    const float2 v = __ldcg(reinterpret_cast<const float2*>(o) + lane);
                    x[i][0] = v.x; x[i][1] = v.y;
                }
            }
        }
#pragma unroll
        for (int i = 0; i < BATCH; ++i) mn = fmaxf(mn, z[i].x);
        const float f = rescale2(s.m, mn);
        s.l *= f; s.lr *= f;
#pragma unroll
        for (int e = 0; e < E; ++e) s.o[e] *= f;
#pragma unroll
        for (int i = 0; i < BATCH; ++i) {
            // (an empty state weighs nothing, whatever it holds; one that gave up is NaN whatever its reference says)
            const float w = z[i].y == 0.f ? 0.f : rescale2(z[i].x, mn);
            s.l = fmaf(z[i].y, w, s.l);
            s.lr = fmaf(z[i].z, w, s.lr);
            if (w != 0.f)
#pragma unroll
                for (int e = 0; e < E; ++e) s.o[e] = fmaf(x[i][e], w, s.o[e]);
        }
        s.m = mn;
    }
    return s;
}

// Joins what the warps of a block have of one row (all of them; the first one gets the sums).
template <int D> __device__ __forceinline__ void join_warps(Sum<D / 32>& s) {
    constexpr int E = D / 32, W = JOIN_NT / 32;
    __shared__ float sm[W][3], so[W][D];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (lane == 0) { sm[warp][0] = s.m; sm[warp][1] = s.l; sm[warp][2] = s.lr; }
#pragma unroll
    for (int e = 0; e < E; ++e) so[warp][lane * E + e] = s.o[e];
    __syncthreads();
    if (warp != 0) return;
    float M = -INFINITY;
#pragma unroll
    for (int x = 0; x < W; ++x) M = fmaxf(M, sm[x][0]);
    s.l = s.lr = 0.f;
#pragma unroll
    for (int e = 0; e < E; ++e) s.o[e] = 0.f;
#pragma unroll
    for (int x = 0; x < W; ++x) {
        const float w = sm[x][1] == 0.f ? 0.f : rescale2(sm[x][0], M);
        s.l = fmaf(sm[x][1], w, s.l);
        s.lr = fmaf(sm[x][2], w, s.lr);
        if (w != 0.f)
#pragma unroll
            for (int e = 0; e < E; ++e) s.o[e] = fmaf(so[x][lane * E + e], w, s.o[e]);
    }
    s.m = M;
}

// The row's sums to the output (row w), by a whole warp.
template <typename T, int D> __device__ __forceinline__ void store_row(const Sum<D / 32>& s, const Output& out, long long w) {
    constexpr int E = D / 32;
    const int lane = threadIdx.x & 31;
    const RowEnd end(s.m, s.l, s.lr, out.lse_in, w);
    float y[E], x[E] = {};
    T* orow = (T*)out.O + w * D + lane * E;
    if (out.O_in) {
        const T* irow = (const T*)out.O_in + w * D + lane * E;
#pragma unroll
        for (int e = 0; e < E; ++e) x[e] = (float)irow[e];
    }
#pragma unroll
    for (int e = 0; e < E; ++e) y[e] = end_value(s.o[e], end.f, x[e], end.f_in);
    if (sizeof(T) == 2) {
#pragma unroll
        for (int e = 0; e < E; e += 2) reinterpret_cast<uint32_t*>(orow)[e / 2] = Vec<__nv_bfloat16>::pack2(y[e], y[e + 1]);
    } else {
#pragma unroll
        for (int e = 0; e < E; ++e) orow[e] = (T)y[e];
    }
    __syncwarp();                               // (all lanes have read lse_in, which may be lse)
    if (out.lse && lane == 0) out.lse[w] = end.lse;
}

// Row m of output unit u from one or two sets of states.  b_len: the lengths of b's units, of which those without keys have no entry in the
// table of pieces (a's all have one).
// WIDE: a block per row.  (Of few rows with many pieces each the batches, 0.85 us one after the other, are what takes time: 32 rows of 148
// pieces and all before them 39 us by a warp per row, 23 so.)
template <typename T, int D, bool WIDE> __global__ void __launch_bounds__(JOIN_NT)
join_kernel(const States a, const States b, int has_a, int has_b, const int32_t* __restrict__ b_len,
            int skip_whole, const Output out, int rows, int m_rows, int Hkv, int G) {
    const int warp = threadIdx.x >> 5, w = WIDE ? blockIdx.x : blockIdx.x * (JOIN_NT / 32) + warp;
    grid_dependency_wait();
    grid_launch_dependents();
    if (w >= rows) return;
    const int u = w / m_rows, m = w - u * m_rows;
    Pieces pa = {}, pb = {};
    if (has_a) pa = pieces_of<D>(a, nullptr, u, m);
    if (has_b) pb = pieces_of<D>(b, b_len, u % Hkv, u / Hkv * G + m);
    if (skip_whole && pa.count == 1) return;                       // (by the kernel that had the item whole)
    Sum<D / 32> s = sum_pieces<D>(pa, pb, WIDE ? warp : 0, WIDE ? JOIN_NT / 32 : 1);
    if (WIDE) {
        join_warps<D>(s);
        if (warp != 0) return;
    }
    store_row<T, D>(s, out, w);
}

// Items of which most have gone to the output in one piece: a block per ITEM_ROWS rows of a tile, which looks at its item first.
// (A warp per row of the output took 44 us for 131,072 rows of which three in ten had pieces.)
template <typename T, int D, int ITEM_ROWS> __global__ void __launch_bounds__(JOIN_NT)       // (ITEM_ROWS 1: the block's warps share the row)
join_items_kernel(const States a, const int32_t* __restrict__ len, const Output out, int m_rows) {
    const int per = (a.halves ? a.tile_room : a.rows) / ITEM_ROWS, part = blockIdx.x % per, at = blockIdx.x / per, u = at / a.items;
    const int m0 = (at % a.items) * (per * ITEM_ROWS) + part * ITEM_ROWS;     // (tiles of an item follow one another in the unit)
    grid_dependency_wait();
    grid_launch_dependents();
    if (m0 >= m_rows) return;
    const int n = len ? __ldg(len + u) : 1;
    const int4 pc = __ldcg(a.pieces + at);
    if (n > 0 && pc.x == 1 && !a.halves) return;
    Pieces p = {n > 0 ? pc.x << (a.halves ? 1 : 0) : 0, pc.y, pc.z, a.stride, a.o, a.ml, a.rows, a.halves ? a.tile_room : 0}, none = {};
    if constexpr (ITEM_ROWS == 1) {
        p.o = a.o + (size_t)part * D;
        p.ml = a.ml + part;
        Sum<D / 32> s = sum_pieces<D>(p, none, threadIdx.x >> 5, JOIN_NT / 32);
        join_warps<D>(s);
        if (threadIdx.x < 32) store_row<T, D>(s, out, (long long)u * m_rows + m0);
    } else {
#pragma unroll 1
        for (int r = threadIdx.x >> 5; r < ITEM_ROWS && m0 + r < m_rows; r += JOIN_NT / 32) {
            p.o = a.o + (size_t)(part * ITEM_ROWS + r) * D;
            p.ml = a.ml + part * ITEM_ROWS + r;
            store_row<T, D>(sum_pieces<D>(p, none, 0, 1), out, (long long)u * m_rows + m0 + r);
        }
    }
}

}  // namespace

cudaError_t launch_join(const Shape& s, int units, int m, const States* a, const States* b, const int32_t* b_len,
                        int skip_whole, int pieces_about, const Output& out, cudaStream_t st) {
    const long long rows = (long long)units * m;
    const bool wide = pieces_about > 2 * BATCH && rows <= 2048;
    const long long blocks = wide ? rows : (rows + JOIN_NT / 32 - 1) / (JOIN_NT / 32);
    if (rows > 0x7fffffffll) return cudaErrorInvalidValue;
    auto fn = s.dtype == KVM_BF16 ? (s.D == 128 ? (wide ? join_kernel<__nv_bfloat16, 128, true> : join_kernel<__nv_bfloat16, 128, false>)
                                                : (wide ? join_kernel<__nv_bfloat16, 64, true> : join_kernel<__nv_bfloat16, 64, false>))
                                  : (s.D == 128 ? (wide ? join_kernel<float, 128, true> : join_kernel<float, 128, false>)
                                                : (wide ? join_kernel<float, 64, true> : join_kernel<float, 64, false>));
    return launch_dependent(fn, dim3((unsigned)blocks), dim3(JOIN_NT), 0, st, a ? *a : States{}, b ? *b : States{}, a ? 1 : 0, b ? 1 : 0,
                            b_len, skip_whole, out, (int)rows, m, s.Hkv, s.G);
}

cudaError_t launch_join_items(const Shape& s, int units, int m, const States& a, const int32_t* len, const Output& out, cudaStream_t st) {
    // (few items have many pieces each: a block or a warp per row; of many items few are cut: less blocks that find nothing to do)
    const long long items = (long long)units * a.items;
    const int per_block = items * 2 * BATCH < 148 ? 1 : items <= 148 ? JOIN_NT / 32 : 16;
    const long long blocks = items * ((a.halves ? a.tile_room : a.rows) / per_block);
    if (blocks > 0x7fffffffll) return cudaErrorInvalidValue;
    auto fn = per_block == 1    ? (s.D == 128 ? join_items_kernel<__nv_bfloat16, 128, 1> : join_items_kernel<__nv_bfloat16, 64, 1>)
              : per_block == 16 ? (s.D == 128 ? join_items_kernel<__nv_bfloat16, 128, 16> : join_items_kernel<__nv_bfloat16, 64, 16>)
                                : (s.D == 128 ? join_items_kernel<__nv_bfloat16, 128, JOIN_NT / 32> : join_items_kernel<__nv_bfloat16, 64, JOIN_NT / 32>);
    return launch_dependent(fn, dim3((unsigned)blocks), dim3(JOIN_NT), 0, st, a, len, out, m);
}

}  // namespace serve
}  // namespace kvm
