// What the serving kernels share (paged append, shared-prefix decode, cross attention): where query and key rows lie, the
// states that parts of a softmax leave, and how they are joined.
#pragma once
#include "common.cuh"

namespace kvm {
namespace serve {

constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;

// The shape part of kvm_params, checked.
struct Shape {
    int B, Hq, Hkv, G, D, U, dtype;
    float scale;
};

// A paged cache as the kernels take it.
struct Pages {
    void *K, *V;
    const int32_t *table, *len;
    int n_pages, shift, max_pages;              // rows per page: 1 << shift
    __host__ __device__ __forceinline__ int room() const { return max_pages << shift; }
};

// Query rows of a unit: N blocks of R rows of D channels; unit u's block n starts at row u * su + n * sn of the tensor.  Outputs
// lie alike.
//   cross attention: unit = (b, h), its G heads' n_q rows follow one another: R = G n_q, N = 1
//   a shared prefix: unit = h, block = b: R = G, N = B;  a sequence's own rows: unit = (b, h), R = G, N = 1
struct Queries {
    const void* q;
    long long su, sn;
    int R, N;
    __host__ __device__ __forceinline__ int rows() const { return R * N; }
    __device__ __forceinline__ long long at(int u, int m) const { return u * su + (m / R) * sn + m % R; }
};

// Key rows of a unit: contiguous (K, V [units, rows, D]) or paged.
struct Keys {
    const void *K, *V;
    const int32_t* len;                         // nullable: all `rows`
    int rows;                                   // most rows of a unit
    const int32_t* table;                       // nullable: contiguous
    int n_pages, shift, max_pages;
    __device__ __forceinline__ int rows_of(int u) const { return len ? max(0, min(__ldg(len + u), rows)) : rows; }
    // index of a unit's row in the tensor of all rows, or -1 where its page does not exist
    __device__ __forceinline__ long long row(int u, int r) const {
        if (!table) return (long long)u * rows + r;
        const int page = __ldg(table + (size_t)u * max_pages + (r >> shift));
        return (unsigned)page < (unsigned)n_pages ? ((long long)page << shift) + (r & ((1 << shift) - 1)) : -1;
    }
};

// The states of pieces of a softmax.  A piece covers the query rows of an item (a tile of a unit's query rows, or two) over some of
// the unit's keys; its state, in a slot of its own, is per row the weighted sum of the values o[D] and (m, l, lr): the reference
// (log2 units), the sum of the weights relative to it, and the sum of the weights as they were rounded for the product.
struct States {
    float* o;                                   // [slot][rows][D]
    float4* ml;                                 // [slot][rows]
    int rows;                                   // rows of a slot
    int items;                                  // items of a unit
    int count;                                  // pieces of every item, in slots item * count ..; 0: `pieces` tells
    int4* pieces;                               // per item (count, first slot, second slot, -); the others follow the second by `stride`
    int stride;
    // Which rows an item holds.  Tiles of `tile` consecutive rows of a unit; or (R > 0) each block of R rows in tiles of its own.
    int tile, R, two;                           // two: two tiles to an item, `tile_room` rows apart
    int tile_room, halves;                      // halves: a piece has two states, tile_room rows apart
    __device__ __forceinline__ void find(int m, int& item, int& row) const {
        int t, in;
        if (R > 0) {
            const int n = m / R, r = m % R;
            t = n * ((R + tile - 1) / tile) + r / tile;
            in = r % tile;
        } else {
            t = m / tile;
            in = m % tile;
        }
        item = two ? t >> 1 : t;
        row = two ? (t & 1) * tile_room + in : in;
    }
};
// Where the result goes, and what is joined in.
struct Output {
    void* O;
    float* lse;                                 // nullable
    const void* O_in;                           // nullable
    const float* lse_in;
};

// Weight of a state with reference m under the reference M (an empty state has m = -inf).
__device__ __forceinline__ float rescale2(float m, float M) { return m == -INFINITY ? 0.f : exp2f(m - M); }

// One row's result from its sums, N channels at a time: o / lr, joined with O_in under both log-sum-exps.
// (l = 0: no keys, the row is what is joined in, bit for bit.  NaN sums, and a NaN lse_in, are the mark of a wait that gave up, and stay.)
struct RowEnd {
    float f, f_in, lse;
    __device__ __forceinline__ RowEnd() {}
    __device__ __forceinline__ RowEnd(float m, float l, float lr, const float* lse_in, long long row) {
        const bool none = l == 0.f;
        f = none ? 0.f : 1.f / lr;
        f_in = 0.f;
        lse = none ? -INFINITY : (m + log2f(l)) * LN2;
        if (lse_in) {
            const float z = lse_in[row];
            if (none) {
                f_in = z == -INFINITY ? 0.f : 1.f;
                lse = z;
                return;
            }
            if (z == -INFINITY) return;                          // nothing to join
            const float M = fmaxf(lse, z);
            const float a = expf(lse - M), b = expf(z - M), s = a + b;
            f *= a / s;
            f_in = b / s;
            lse = M + logf(s);
        }
    }
};
// o * f + O_in * f_in; what has no weight counts as nothing, whatever it holds.
__device__ __forceinline__ float end_value(float o, float f, float x, float f_in) {
    const float y = f != 0.f ? o * f : 0.f;
    return f_in != 0.f ? fmaf(x, f_in, y) : y;
}

// A shared prefix's kernel and the one for the sequences' own rows run side by side, each on a part of the SMs: the first is busy
// with products and exponentials while the second waits for memory.  Each finds out from the lengths how much there is for the other.
constexpr int SMS = 148;
struct Beside {
    const int32_t* len;                         // nullable: all `rows`
    int units, rows, per, tile;                 // the other kernel's units (0: it does not run), items of a unit, rows of a step
    // What this thread of `threads` finds of the other's steps (to be summed over the block).
    __device__ __forceinline__ long long part(int threads) const {
        long long n = 0;
        for (int i = threadIdx.x; i < units; i += threads) n += (long long)((len ? max(0, min(__ldg(len + i), rows)) : rows) + tile - 1) / tile * per;
        return n;
    }
};
// SMs for the prefix, such that both parts end at about the same time (by all lanes of a warp).  Measured side by side, us: the prefix 14
// and 2.4 for each of a CTA's steps (128 keys, up to 256 query rows); the own rows 8 and 0.137 for 16 rows of 128 channels on one SM
// (60 GB/s).  (Taken with 128 channels and two query tiles; a step of one tile, or of 64 channels, is shorter.)  64 sequences of 768 rows over 16384 x 8 heads, own rows on 60 / 70 / 80 / 90 SMs: 71.5 / 64.4 / 61.1 / 67.2 us, one after the other 80;
// 16 x 32 of 292 rows over 2048 x 32 heads, on 48 / 60 / 70 / 80 / 90: 39.4 / 34.4 / 35.0 / 36.4 / 39.9, one after the other 43.
constexpr int OWN_MOST = 128;
__device__ __forceinline__ int prefix_sms(long long steps, long long blocks, int D) {
    if (blocks == 0) return SMS;
    const float own = (D == 128 ? 0.137f : 0.09f) * (float)blocks;
    float best = 1e30f;
    int y_best = 1;
#pragma unroll 1
    for (int y = 1 + (threadIdx.x & 31); y <= (steps == 0 ? SMS - 1 : OWN_MOST); y += 32) {
        const float t = fmaxf(14.f + 2.4f * ceilf(__fdividef((float)steps, (float)(SMS - y))), 8.f + __fdividef(own, (float)y));
        if (t < best) { best = t; y_best = y; }
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        const float t = __shfl_xor_sync(0xffffffffu, best, o);
        const int y = __shfl_xor_sync(0xffffffffu, y_best, o);
        if (t < best || (t == best && y < y_best)) { best = t; y_best = y; }
    }
    return SMS - y_best;
}
template <int THREADS> __device__ __forceinline__ long long block_sum(long long v, long long* smem) {       // smem: a long long per warp
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) smem[threadIdx.x >> 5] = v;
    __syncthreads();
    long long t = 0;
#pragma unroll
    for (int i = 0; i < THREADS / 32; ++i) t += smem[i];
    return t;
}

cudaError_t launch_append(const Shape& s, const Pages& c, int32_t* len_out, int n_new, const int32_t* new_len, const int32_t* pos,
                          const uint64_t* turns, int neighbours, const void* q, const void* k, const void* v, const int64_t* strides,
                          void* q_out, kvm_stats* stats, cudaStream_t st);

// Attention of all query rows over all keys of their units, for fp32 tensors: on the fp32 pipes (mt = 8) or on matrix products of three bf16
// planes (mt = 64), see rows_f32.cu.  With one piece per item the result goes to `out`, else the states to `states`.
struct F32Plan {
    int mt, items, pieces;                      // query rows of an item, items of a unit, pieces of an item
};
F32Plan f32_plan(int units, int m, int rows, int D);
cudaError_t launch_rows_f32(const Shape& s, const F32Plan& plan, int units, const Queries& q, const Keys& k, const States& states, const Output& out,
                             kvm_stats* stats, cudaStream_t st);

// The same on the tensor cores (bf16, contiguous keys): equal shares of all items' steps per CTA, see rows_tc.cu.
struct TcPlan {
    int gx, bx;                                 // rows of a query tile: bx blocks of gx rows
    int per_block, tiles, items;                // tiles of a block of more than 128 rows (else 0), tiles and items (pairs of tiles) of a unit
    int direct, grid, slot_rows;                // direct: an item in one piece goes to the output
    int compact, whole, alt;                    // few steps per CTA; items are not cut; both groups on a single tile: two states per piece
    long long slots;
};
TcPlan tc_plan(int units, int R, int N, int rows, bool direct);
cudaError_t launch_rows_tc(const Shape& s, const TcPlan& plan, int units, const Queries& q, const Keys& k, const Beside& own, const States& states,
                           const Output& out, kvm_stats* stats, cudaStream_t st);

// Decode attention over a paged cache (bf16), one query per sequence: rows_paged.cu.
struct PagedPlan {
    int hg, items, grid, slot_rows, alone;      // groups of up to 8 heads per unit; items = units x groups; alone: a block per item, nothing to join
    long long slots;
};
PagedPlan paged_plan(const Shape& s, int rows, bool beside_prefix);
// A prefix whose rows that kernel takes as the first of each unit: K, V [heads, rows, D]; unit u's head is u % heads.  rows 0: none.
struct Fold {
    const void *K, *V;
    const int32_t* len;                         // nullable: all `rows`
    int heads, rows;
    __device__ __forceinline__ int rows_of(int h) const { return len ? max(0, min(__ldg(len + h), rows)) : rows; }
};
cudaError_t launch_rows_paged(const Shape& s, const PagedPlan& plan, const void* q, const Keys& k, const Fold& fold, const Beside& pre, const States& states, void* out,
                              kvm_stats* stats, cudaStream_t st);

// Joins the states: one row of output per row of [units][m].  Two sets of states may be given, over the units of `a` and, with
// unit = h and row = b * G + g, of `b` (a shared prefix).
cudaError_t launch_join(const Shape& s, int units, int m, const States* a, const States* b, const int32_t* b_len,
                        int skip_whole, int pieces_about, const Output& out, cudaStream_t st);
// skip_whole: rows of items in one piece are in the output already.  pieces_about: how many pieces a row may have.
// The same for the tensor-core kernel's items [units][items] of m rows a unit, of which those in one piece are in the output already.
cudaError_t launch_join_items(const Shape& s, int units, int m, const States& a, const int32_t* len, const Output& out, cudaStream_t st);

}  // namespace serve
}  // namespace kvm
