// Joins the states that pieces of a softmax have left, two sets of them if need be (a shared prefix and a sequence's own rows),
// into the rows of the output:  M = max m,  O = sum o 2^(m - M) / sum lr 2^(m - M),  lse = ln sum l 2^(m - M) + M ln 2.
// A warp per row; pieces are taken in order, several at a time so that their loads leave together: results are reproducible.
#include "serve.cuh"

namespace kvm {
namespace serve {
namespace {

constexpr int JOIN_NT = 128;

template <int E> struct Sum {                   // E channels of a row
    float m = -INFINITY, l = 0.f, lr = 0.f, o[E] = {};
};

template <int D, int BATCH>
__device__ __forceinline__ void add_batches(Sum<D / 32>& s, const States& st, long long first, long long second, int count, int row) {
    constexpr int E = D / 32;
    const int lane = threadIdx.x & 31;
    for (int i0 = 0; i0 < count; i0 += BATCH) {
        float4 z[BATCH];
        float x[BATCH][E], mn = s.m;
#pragma unroll
        for (int i = 0; i < BATCH; ++i) {
            const bool in = i0 + i < count;
            const long long slot = i0 + i == 0 ? first : second + (long long)(i0 + i - 1) * st.stride;
            const long long r = (in ? slot : first) * st.rows + row;
            z[i] = __ldcg(st.ml + r);
            if (E == 4) {
                const float4 v = __ldcg(reinterpret_cast<const float4*>(st.o + r * D) + lane);
                x[i][0] = v.x; x[i][1] = v.y; x[i][E - 2] = v.z; x[i][E - 1] = v.w;
            } else {
                const float2 v = __ldcg(reinterpret_cast<const float2*>(st.o + r * D) + lane);
                x[i][0] = v.x; x[i][1] = v.y;
            }
            if (!in) z[i].x = -INFINITY;
            mn = fmaxf(mn, z[i].x);
        }
        const float a = rescale2(s.m, mn);
        s.l *= a; s.lr *= a;
#pragma unroll
        for (int e = 0; e < E; ++e) s.o[e] *= a;
#pragma unroll
        for (int i = 0; i < BATCH; ++i) {
            if (i0 + i >= count) break;
            // (an empty state weighs nothing; a state that gave up is NaN whatever its reference says)
            const float w = z[i].y == 0.f ? 0.f : rescale2(z[i].x, mn);
            s.l = fmaf(z[i].y, w, s.l);
            s.lr = fmaf(z[i].z, w, s.lr);
            if (w != 0.f)
#pragma unroll
                for (int e = 0; e < E; ++e) s.o[e] = fmaf(x[i][e], w, s.o[e]);
        }
        s.m = mn;
    }
}

// (Two pieces are what most cut items of a large problem have, and the loads of absent ones would not be free; a decode batch
// over one prefix has about twenty.)
template <int D>
__device__ __forceinline__ void add_pieces(Sum<D / 32>& s, const States& st, long long first, long long second, int count, int row) {
    if (count <= 2) add_batches<D, 2>(s, st, first, second, count, row);
    else add_batches<D, 8>(s, st, first, second, count, row);
}

// The row's sums to the output (row w).
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
    if (out.lse && lane == 0) out.lse[w] = end.lse;
}

// Row m of output unit u from one or two sets of states.  len: of the units whose pieces a table tells of (a unit without keys
// has no entry there).
template <typename T, int D> __global__ void __launch_bounds__(JOIN_NT)
join_kernel(const States a, const int32_t* __restrict__ a_len, const States b, int has_a, int has_b, const int32_t* __restrict__ b_len,
            int skip_whole, const Output out, long long rows, int m_rows, int Hkv, int G) {
    const long long w = (long long)blockIdx.x * (JOIN_NT / 32) + (threadIdx.x >> 5);
    grid_dependency_wait();
    if (w >= rows) return;
    const int u = (int)(w / m_rows), m = (int)(w % m_rows);
    Sum<D / 32> s;
    bool done = false;                              // (by the kernel that had the item whole)
    auto add = [&](const States& st, const int32_t* len, int unit, int row_of_unit) {
        int item, row;
        st.find(row_of_unit, item, row);
        const long long at = (long long)unit * st.items + item;
        if (st.count > 0) {
            add_pieces<D>(s, st, at * st.count, at * st.count + 1, st.count, row);
        } else if (!len || __ldg(len + unit) > 0) {
            const int4 pc = __ldcg(st.pieces + at);
            done = skip_whole && pc.x == 1;
            if (!done) add_pieces<D>(s, st, pc.y, pc.z, pc.x, row);
        }
    };
    if (has_b) add(b, b_len, u % Hkv, u / Hkv * G + m);
    if (has_a) add(a, a_len, u, m);
    if (!done) store_row<T, D>(s, out, w);
}

// Items of which most have gone to the output in one piece: a block per 32 rows of a tile, which looks at its item first.
// (A warp per row of the output took 44 us for 131,072 rows of which three in ten had pieces; a block per 32 rows XX.)
template <typename T, int D, int ITEM_ROWS> __global__ void __launch_bounds__(JOIN_NT)
join_items_kernel(const States a, const int32_t* __restrict__ len, const Output out, int m_rows) {
    const int per = a.rows / ITEM_ROWS, part = blockIdx.x % per, at = blockIdx.x / per, u = at / a.items;
    const int m0 = (at % a.items) * a.rows + part * ITEM_ROWS;     // (tiles of an item follow one another in the unit)
    grid_dependency_wait();
    if (m0 >= m_rows) return;
    int4 pc = make_int4(0, 0, 0, 0);
    if (!len || __ldg(len + u) > 0) {
        pc = __ldcg(a.pieces + at);
        if (pc.x == 1) return;
    }
#pragma unroll 1
    for (int r = threadIdx.x >> 5; r < ITEM_ROWS && m0 + r < m_rows; r += JOIN_NT / 32) {
        Sum<D / 32> s;
        add_pieces<D>(s, a, pc.y, pc.z, pc.x, part * ITEM_ROWS + r);
        store_row<T, D>(s, out, (long long)u * m_rows + m0 + r);
    }
}

}  // namespace

cudaError_t launch_join(const Shape& s, int units, int m, const States* a, const int32_t* a_len, const States* b, const int32_t* b_len,
                        int skip_whole, const Output& out, cudaStream_t st) {
    const long long rows = (long long)units * m, blocks = (rows + JOIN_NT / 32 - 1) / (JOIN_NT / 32);
    if (blocks > 0x7fffffffll) return cudaErrorInvalidValue;
    auto fn = s.dtype == KVM_BF16 ? (s.D == 128 ? join_kernel<__nv_bfloat16, 128> : join_kernel<__nv_bfloat16, 64>)
                                  : (s.D == 128 ? join_kernel<float, 128> : join_kernel<float, 64>);
    return launch_dependent(fn, dim3((unsigned)blocks), dim3(JOIN_NT), 0, st, a ? *a : States{}, a_len, b ? *b : States{}, a ? 1 : 0, b ? 1 : 0,
                            b_len, skip_whole, out, rows, m, s.Hkv, s.G);
}

cudaError_t launch_join_items(const Shape& s, int units, int m, const States& a, const int32_t* len, const Output& out, cudaStream_t st) {
    // (few items have many pieces each: a warp per row; of many items few are cut: less blocks that find nothing to do)
    const int per_block = (long long)units * a.items <= 148 ? JOIN_NT / 32 : 16;
    const long long blocks = (long long)units * a.items * (a.rows / per_block);
    if (blocks > 0x7fffffffll) return cudaErrorInvalidValue;
    auto fn = per_block == 16 ? (s.D == 128 ? join_items_kernel<__nv_bfloat16, 128, 16> : join_items_kernel<__nv_bfloat16, 64, 16>)
                              : (s.D == 128 ? join_items_kernel<__nv_bfloat16, 128, JOIN_NT / 32> : join_items_kernel<__nv_bfloat16, 64, JOIN_NT / 32>);
    return launch_dependent(fn, dim3((unsigned)blocks), dim3(JOIN_NT), 0, st, a, len, out, m);
}

}  // namespace serve
}  // namespace kvm
