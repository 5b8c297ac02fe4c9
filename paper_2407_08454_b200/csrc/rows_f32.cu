// Attention of a unit's query rows over its keys in fp32 arithmetic, without a mask but the unit's length:
//   o = softmax(c q K^T) V,  lse = ln sum exp(c q.k)
// with one pass over the keys, a running maximum and sum per row, and, where there are few rows, the keys cut into pieces whose
// states are joined by another kernel.
//
// Two forms.  Up to 24 query rows per unit (a decode step): blocks of 8 rows, 32 keys at a time, bound by bandwidth: a pair of
// rows reads a key's channels from shared memory once, 64 KB of shared-memory reads for 32 KB of keys and values and each
// product (about 1,100 clocks against 1,400 that an SM's share of the bandwidth takes).  More rows: blocks of 64 rows by 64 keys
// (32 with 128 channels), four rows per thread, bound by the fp32 pipes and shared memory together.
// (8 heads over 4096 keys, D = 64 / 128, us: 32 rows by eights 38.4 / 54, 48 rows 46.5 / 76, 64 rows together 33.6 / 48.5.)
// The next keys are on their way to registers while the current ones are used.
#include "serve.cuh"
#include "tc_common.cuh"

namespace kvm {
namespace serve {
namespace {

constexpr int NT8 = 256, NT64 = 256;        // threads of a block of 8 and of 64 query rows

struct Args {
    Queries q;
    Keys k;
    States st;
    Output out;
    kvm_stats* stats;
    float scale2;
    int pieces;
};

// A tile of KT keys and values: global memory -> registers -> shared memory as fp32, rows of D + 4 floats (so that 16-byte reads
// of neighbouring rows fall into different banks).  Rows that do not exist become zeros.
template <typename T, int D, int KT, int NT> struct Tile {
    static constexpr int N = Vec<T>::N, LPR = D / N, PER = KT * LPR / NT;       // lanes per row, 16-byte pieces per thread
    static_assert(KT * LPR % NT == 0, "whole rounds");
    uint4 k[PER], v[PER];
    __device__ __forceinline__ void load(const Keys& s, int u, int r0, int r1) {
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int r = r0 + (threadIdx.x + i * NT) / LPR, c = (threadIdx.x + i * NT) % LPR * N;
            k[i] = v[i] = make_uint4(0, 0, 0, 0);
            if (r < r1) {
                const long long at = s.row(u, r);
                if (at >= 0) {
                    k[i] = ldg16((const T*)s.K + at * D + c);
                    v[i] = ldg16((const T*)s.V + at * D + c);
                }
            }
        }
    }
    __device__ __forceinline__ void store(float* sk, float* sv) const {
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            float f[N];
            const int at = (threadIdx.x + i * NT) / LPR * (D + 4) + (threadIdx.x + i * NT) % LPR * N;
            Vec<T>::unpack(k[i], f);
#pragma unroll
            for (int e = 0; e < N; e += 4) *reinterpret_cast<float4*>(sk + at + e) = make_float4(f[e], f[e + 1], f[e + 2], f[e + 3]);
            Vec<T>::unpack(v[i], f);
#pragma unroll
            for (int e = 0; e < N; e += 4) *reinterpret_cast<float4*>(sv + at + e) = make_float4(f[e], f[e + 1], f[e + 2], f[e + 3]);
        }
    }
};

// Does row r of the unit exist, as to its page?  (Its absence is reported.)
__device__ __forceinline__ bool exists(const Args& a, int u, int r) {
    if (!a.k.table) return true;
    const bool ok = a.k.row(u, r) >= 0;
    if (!ok && a.stats) a.stats->status = KVM_E_PAGE;
    return ok;
}

// MT query rows of the unit from row m0, times the scale (log2 units), in shared memory; rows past the last are zeros.
template <typename T, int D, int MT, int NT> __device__ __forceinline__ void load_queries(const Args& a, int u, int m0, float* sq, int pitch) {
    constexpr int N = Vec<T>::N, LPR = D / N;
    for (int i = threadIdx.x; i < MT * LPR; i += NT) {
        const int m = m0 + i / LPR, c = i % LPR * N;
        float f[N] = {};
        if (m < a.q.rows()) Vec<T>::unpack(ldg16((const T*)a.q.q + a.q.at(u, m) * D + c), f);
#pragma unroll
        for (int e = 0; e < N; ++e) sq[(i / LPR) * pitch + c + e] = f[e] * a.scale2;
    }
}

// E neighbouring channels of a finished row from channel c: to the output, or to the piece's state.
template <typename T, int D, int E>
__device__ __forceinline__ void finish(const Args& a, int u, int item, int piece, int row, int m_row, int c, const float* o, float m, float l) {
    if (a.pieces > 1 || a.st.o) {
        const size_t r = (((size_t)u * a.st.items + item) * a.pieces + piece) * a.st.rows + row;
#pragma unroll
        for (int e = 0; e < E; ++e) a.st.o[r * D + c + e] = o[e];
        if (c == 0) a.st.ml[r] = make_float4(m, l, l, 0.f);
        return;
    }
    const long long at = a.q.at(u, m_row);
    const RowEnd end(m, l, l, a.out.lse_in, at);
#pragma unroll
    for (int e = 0; e < E; ++e) {
        const float x = a.out.O_in ? (float)((const T*)a.out.O_in)[at * D + c + e] : 0.f;
        ((T*)a.out.O)[at * D + c + e] = (T)end_value(o[e], end.f, x, end.f_in);
    }
    if (c == 0 && a.out.lse) a.out.lse[at] = end.lse;
}

// This block's keys: the piece's share of the unit's tiles.
template <int KT> __device__ __forceinline__ void share(const Args& a, int u, int& r0, int& r1) {
    const int n = a.k.rows_of(u), tiles = (n + KT - 1) / KT;
    r0 = (int)((long long)blockIdx.y * tiles / a.pieces) * KT;
    r1 = min(n, (int)((long long)(blockIdx.y + 1) * tiles / a.pieces) * KT);
}

// ------------------------------------------------------------------ few rows
template <typename T, int D> __global__ void __launch_bounds__(NT8) rows8_kernel(const Args a) {
    constexpr int MT = 8, KT = 32, P = D + 4, E = D / 32;
    __shared__ __align__(16) float sq[MT * P], sk[KT * P], sv[KT * P];
    __shared__ float sx[2][MT][KT], sp[MT][KT], salpha[MT];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int rp = threadIdx.x >> 6, half = (threadIdx.x >> 5) & 1;      // a pair of rows; half of the channels (S) or keys (O)
    const int u = blockIdx.z, m0 = blockIdx.x * MT;
    grid_dependency_wait();
    int r0, r1;
    share<KT>(a, u, r0, r1);
    load_queries<T, D, MT, NT8>(a, u, m0, sq, P);
    Tile<T, D, KT, NT8> t;
    t.load(a.k, u, r0, r1);
    float m = -INFINITY, l = 0.f, o[2][E] = {};                          // m, l: of row `warp` (l: of this lane's keys)
    for (int r = r0; r < r1; r += KT) {
        __syncthreads();
        t.store(sk, sv);
        __syncthreads();
        if (r + KT < r1) t.load(a.k, u, r + KT, r1);
        float x0 = 0.f, x1 = 0.f;
        const float *qa = sq + 2 * rp * P + half * (D / 2), *ka = sk + lane * P + half * (D / 2);
#pragma unroll 8
        for (int c = 0; c < D / 2; c += 4) {
            const float4 k4 = *reinterpret_cast<const float4*>(ka + c), a4 = *reinterpret_cast<const float4*>(qa + c),
                         b4 = *reinterpret_cast<const float4*>(qa + P + c);
            x0 = fmaf(a4.x, k4.x, x0); x0 = fmaf(a4.y, k4.y, x0); x0 = fmaf(a4.z, k4.z, x0); x0 = fmaf(a4.w, k4.w, x0);
            x1 = fmaf(b4.x, k4.x, x1); x1 = fmaf(b4.y, k4.y, x1); x1 = fmaf(b4.z, k4.z, x1); x1 = fmaf(b4.w, k4.w, x1);
        }
        sx[half][2 * rp][lane] = x0;
        sx[half][2 * rp + 1][lane] = x1;
        __syncthreads();
        {
            const bool live = r + lane < r1 && exists(a, u, r + lane);
            const float s = live ? sx[0][warp][lane] + sx[1][warp][lane] : -INFINITY;
            float mn = s;
#pragma unroll
            for (int z = 16; z > 0; z >>= 1) mn = fmaxf(mn, __shfl_xor_sync(0xffffffffu, mn, z));
            mn = fmaxf(mn, m);
            const float alpha = rescale2(m, mn), p = rescale2(s, mn);
            l = l * alpha + p;
            m = mn;
            sp[warp][lane] = p;
            if (lane == 0) salpha[warp] = alpha;
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int e = 0; e < E; ++e) o[i][e] *= salpha[2 * rp + i];
#pragma unroll 4
        for (int j = half * (KT / 2); j < (half + 1) * (KT / 2); ++j) {
            const float p0 = sp[2 * rp][j], p1 = sp[2 * rp + 1][j];
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const float v = sv[j * P + lane * E + e];
                o[0][e] = fmaf(p0, v, o[0][e]);
                o[1][e] = fmaf(p1, v, o[1][e]);
            }
        }
    }
    // the two halves of the keys, and the rows' sums
#pragma unroll
    for (int z = 16; z > 0; z >>= 1) l += __shfl_xor_sync(0xffffffffu, l, z);
    __syncthreads();
    if (lane == 0) { sp[warp][0] = m; sp[warp][1] = l; }
    if (half == 1)
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int e = 0; e < E; ++e) sk[(2 * rp + i) * P + lane * E + e] = o[i][e];
    __syncthreads();
    if (half == 0)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int row = 2 * rp + i;
            if (m0 + row >= a.q.rows()) break;
#pragma unroll
            for (int e = 0; e < E; ++e) o[i][e] += sk[row * P + lane * E + e];
            finish<T, D, E>(a, u, blockIdx.x, blockIdx.y, row, m0 + row, lane * E, o[i], sp[row][0], sp[row][1]);
        }
}

// ------------------------------------------------------------------ many rows
// A thread takes four rows by KT / 16 keys, then four rows by D / 16 channels, pairs of channels in one instruction.  28.7 TFLOP/s of 72 with
// 64 channels, 30.1 with 128 (16 heads x 1024 queries x 2048 keys); eight rows per thread of half as many, which halves the
// reads per product, is as fast (27.9, 30.0), and so are single products: neither the reads nor the issue slots bound it.
template <int D> constexpr int keys64() { return D == 128 ? 32 : 64; }
template <int D> constexpr size_t rows64_smem() { return ((64 + 2 * keys64<D>()) * (D + 4) + 64 * (keys64<D>() + 4)) * sizeof(float); }
template <typename T, int D> __global__ void __launch_bounds__(NT64) rows64_kernel(const Args a) {
    constexpr int MT = 64, KT = keys64<D>(), P = D + 4, PP = KT + 4, E = D / 16, KJ = KT / 16, R = 4;
    extern __shared__ __align__(16) float smem[];
    float *sq = smem, *sk = sq + MT * P, *sv = sk + KT * P, *sp = sv + KT * P;
    const int rg = threadIdx.x / 16, kg = threadIdx.x % 16;              // four rows; keys kg + 16 j, channels 4 kg + 64 j
    const int u = blockIdx.z, m0 = blockIdx.x * MT;
    grid_dependency_wait();
    int r0, r1;
    share<KT>(a, u, r0, r1);
    load_queries<T, D, MT, NT64>(a, u, m0, sq, P);
    Tile<T, D, KT, NT64> t;
    t.load(a.k, u, r0, r1);
    float m[R], l[R] = {};                                               // l: of this thread's keys
    uint64_t o[R][E / 2] = {};                                           // pairs of channels
#pragma unroll
    for (int i = 0; i < R; ++i) m[i] = -INFINITY;
    for (int r = r0; r < r1; r += KT) {
        __syncthreads();
        t.store(sk, sv);
        __syncthreads();
        if (r + KT < r1) t.load(a.k, u, r + KT, r1);
        uint64_t x2[R][KJ] = {};
#pragma unroll 2
        for (int c = 0; c < D; c += 4) {
            ulonglong2 kv[KJ];
#pragma unroll
            for (int j = 0; j < KJ; ++j) kv[j] = *reinterpret_cast<const ulonglong2*>(sk + (kg + 16 * j) * P + c);
#pragma unroll
            for (int i = 0; i < R; ++i) {
                const ulonglong2 qv = *reinterpret_cast<const ulonglong2*>(sq + (rg * R + i) * P + c);
#pragma unroll
                for (int j = 0; j < KJ; ++j) x2[i][j] = tc::ffma2(qv.y, kv[j].y, tc::ffma2(qv.x, kv[j].x, x2[i][j]));
            }
        }
        float x[R][KJ];
#pragma unroll
        for (int i = 0; i < R; ++i)
#pragma unroll
            for (int j = 0; j < KJ; ++j) {
                float lo, hi;
                tc::unpack2(x2[i][j], lo, hi);
                x[i][j] = lo + hi;
            }
        bool live[KJ];
#pragma unroll
        for (int j = 0; j < KJ; ++j) live[j] = r + kg + 16 * j < r1 && exists(a, u, r + kg + 16 * j);
#pragma unroll
        for (int i = 0; i < R; ++i) {
            float mn = -INFINITY;
#pragma unroll
            for (int j = 0; j < KJ; ++j) {
                if (!live[j]) x[i][j] = -INFINITY;
                mn = fmaxf(mn, x[i][j]);
            }
#pragma unroll
            for (int z = 8; z > 0; z >>= 1) mn = fmaxf(mn, __shfl_xor_sync(0xffffffffu, mn, z));
            mn = fmaxf(mn, m[i]);
            const float alpha = rescale2(m[i], mn);
            m[i] = mn;
            l[i] *= alpha;
#pragma unroll
            for (int j = 0; j < KJ; ++j) {
                const float p = rescale2(x[i][j], mn);
                l[i] += p;
                sp[(rg * R + i) * PP + kg + 16 * j] = p;
            }
#pragma unroll
            for (int e = 0; e < E / 2; ++e) o[i][e] = tc::fmul2(o[i][e], tc::pack2(alpha, alpha));
        }
        __syncwarp();                                                    // (a warp reads the weights of its own rows only)
#pragma unroll 1
        for (int j = 0; j < KT; j += 4) {
            ulonglong2 v[4][E / 4];
#pragma unroll
            for (int jj = 0; jj < 4; ++jj)
#pragma unroll
                for (int x4 = 0; x4 < E / 4; ++x4) v[jj][x4] = *reinterpret_cast<const ulonglong2*>(sv + (j + jj) * P + kg * 4 + x4 * 64);
#pragma unroll
            for (int i = 0; i < R; ++i) {
                const float4 p4 = *reinterpret_cast<const float4*>(sp + (rg * R + i) * PP + j);
#pragma unroll
                for (int jj = 0; jj < 4; ++jj) {
                    const float p = jj == 0 ? p4.x : jj == 1 ? p4.y : jj == 2 ? p4.z : p4.w;
                    const uint64_t p2 = tc::pack2(p, p);
#pragma unroll
                    for (int x4 = 0; x4 < E / 4; ++x4) {
                        o[i][x4 * 2] = tc::ffma2(p2, v[jj][x4].x, o[i][x4 * 2]);
                        o[i][x4 * 2 + 1] = tc::ffma2(p2, v[jj][x4].y, o[i][x4 * 2 + 1]);
                    }
                }
            }
        }
    }
#pragma unroll
    for (int i = 0; i < R; ++i) {
#pragma unroll
        for (int z = 8; z > 0; z >>= 1) l[i] += __shfl_xor_sync(0xffffffffu, l[i], z);
        const int row = rg * R + i;
        if (m0 + row >= a.q.rows()) continue;
#pragma unroll
        for (int x4 = 0; x4 < E / 4; ++x4) {
            float f[4];
            tc::unpack2(o[i][x4 * 2], f[0], f[1]);
            tc::unpack2(o[i][x4 * 2 + 1], f[2], f[3]);
            finish<T, D, 4>(a, u, blockIdx.x, blockIdx.y, row, m0 + row, kg * 4 + x4 * 64, f, m[i], l[i]);
        }
    }
}

template <typename T, int D> cudaError_t launch_t(const Args& a, const SimtPlan& plan, int units, cudaStream_t st) {
    const dim3 grid(plan.items, plan.pieces, units);
    if (plan.mt == 8) return launch_dependent(rows8_kernel<T, D>, grid, dim3(NT8), 0, st, a);
    constexpr size_t smem = rows64_smem<D>();
    // (asked for on every call: the attribute is the current device's, and setting it costs less than keeping track of devices)
    const cudaError_t e = cudaFuncSetAttribute(rows64_kernel<T, D>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
    if (e != cudaSuccess) return e;
    return launch_dependent(rows64_kernel<T, D>, grid, dim3(NT64), smem, st, a);
}

}  // namespace

// Pieces: the number whose blocks fill the SMs best in whole rounds of what is at work at the same time (five blocks of 8 rows to an SM; of
// 64 rows two with 128 channels, three with 64), a few per cent given away for each more, but none with less than 128 keys where all are
// there.  (56 units x 160 rows x 3542 keys x 128: 168 blocks in one piece each, 953 us; by whole rounds 538.)
SimtPlan simt_plan(int units, int m, int rows, int D) {
    SimtPlan p;
    p.mt = m <= 24 ? 8 : 64;
    p.items = (m + p.mt - 1) / p.mt;
    const long long blocks = (long long)units * p.items, room = SMS * (p.mt == 8 ? 5 : D == 128 ? 2 : 3);
    const long long most = ((long long)rows + 127) / 128, least = (room + blocks - 1) / blocks;     // (least: one round, more or less)
    p.pieces = 1;
    double best = 0.0;
    for (long long n = 1; n <= most && n <= 2 * least + 6; ++n) {
        const double fill = (double)(n * blocks) / (double)((n * blocks + room - 1) / room * room) / (1.0 + 0.02 * (double)n / (double)least);
        if (fill > best * 1.0001) { best = fill; p.pieces = (int)n; }
    }
    return p;
}

cudaError_t launch_rows_simt(const Shape& s, const SimtPlan& plan, int units, const Queries& q, const Keys& k, const States& states, const Output& out,
                             kvm_stats* stats, cudaStream_t st) {
    if (units > 65535 || plan.pieces > 65535) return cudaErrorInvalidValue;
    const Args a = {q, k, states, out, stats, s.scale * LOG2E, plan.pieces};
    return s.D == 128 ? launch_t<float, 128>(a, plan, units, st) : launch_t<float, 64>(a, plan, units, st);
}

}  // namespace serve
}  // namespace kvm
