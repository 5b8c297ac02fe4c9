// Attention of a unit's query rows over its keys for fp32 tensors, without a mask but the unit's length:
//   o = softmax(c q K^T) V,  lse = ln sum exp(c q.k)
// with one pass over the keys, a running maximum and sum per row, and, where there are few rows, the keys cut into pieces whose
// states are joined by another kernel.
//
// Two forms.  Up to 16 query rows per unit (a decode step): blocks of 8 rows, 32 keys at a time, bound by bandwidth: a pair of
// rows reads a key's channels from shared memory once, 64 KB of shared-memory reads for 32 KB of keys and values and each
// product (about 1,100 clocks against 1,400 that an SM's share of the bandwidth takes).  More rows: blocks of 64 rows by 32 keys
// on warp-level matrix products of three bf16 planes, bound by those.
// The next keys are on their way to registers while the current ones are used.
#include <mutex>

#include "serve.cuh"
#include "tc_common.cuh"

namespace kvm {
namespace serve {
namespace {

constexpr int NT8 = 256, NT64 = 128;        // threads of a block of 8 and of 64 query rows

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

// A finished row on its way to the output, or to the piece's state.  The lanes that hold its channels each work out the row's end once; then, a
// __syncwarp() later, they put their channels and one of them the sums: lse_in may be lse, so nobody may read it after that.
template <typename T, int D> struct RowTo {
    const Args& a;
    bool state;
    size_t at;                              // row of the states or of the output
    float m, l;
    RowEnd end;
    // (live: a row of the unit; of those past its last one nothing is read)
    __device__ __forceinline__ RowTo(const Args& args, int u, int item, int piece, int row, int m_row, bool live, float m0, float l0)
        : a(args), state(args.pieces > 1 || args.st.o),
          at(state ? (((size_t)u * args.st.items + item) * args.pieces + piece) * args.st.rows + row : (size_t)args.q.at(u, m_row)), m(m0), l(l0) {
        if (!state) end = RowEnd(m0, l0, l0, live ? args.out.lse_in : nullptr, at);
    }
    // E neighbouring channels from channel c
    template <int E> __device__ __forceinline__ void channels(int c, const float* o) const {
#pragma unroll
        for (int e = 0; e < E; ++e) {
            if (state) {
                a.st.o[at * D + c + e] = o[e];
            } else {
                const float x = a.out.O_in ? (float)((const T*)a.out.O_in)[at * D + c + e] : 0.f;
                ((T*)a.out.O)[at * D + c + e] = (T)end_value(o[e], end.f, x, end.f_in);
            }
        }
    }
    __device__ __forceinline__ void sums() const {
        if (state) a.st.ml[at] = make_float4(m, l, l, 0.f);
        else if (a.out.lse) a.out.lse[at] = end.lse;
    }
};

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
            const RowTo<T, D> to(a, u, blockIdx.x, blockIdx.y, row, m0 + row, true, sp[row][0], sp[row][1]);
            __syncwarp();
            to.template channels<E>(lane * E, o[i]);
            if (lane == 0) to.sums();
        }
}

// ------------------------------------------------------------------ many rows
// On warp-level matrix products: an fp32 number is the sum of three bf16 numbers (each rounded to the nearest, what is left after two is below
// 2^-17 of it and after three below 2^-26), and of the nine products of two such sums the six that reach 2^-26 are kept:
//   x y = x1 y1 + (x1 y2 + x2 y1) + (x1 y3 + x2 y2 + x3 y1),
// accumulated in fp32: of the logits the five small ones apart from the large one, and of O each 16 keys by themselves, the small ones first, which
// ordinary additions then join.  (The matrix unit does not round to the nearest: what is added to a long sum again and again loses on one side.
// With one accumulator for all, 30,000 keys of values of one sign came out 3.4e-5 of themselves too small, so 4e-8.)
// A warp has 16 query rows, whose three planes stay in registers; the block's four warps share
// the planes of 32 keys and values, made while they are written to shared memory (16-byte pieces swizzled by the row, so that ldmatrix
// meets no bank conflict).  The weights are split in registers: what a lane holds of the first product is what it needs for the second.
// (By products on the fp32 pipes, 64 x 64 blocks: 28.7 TFLOP/s with 64 channels, 31.9 with 128; this 42.0 and 44.8, which is
// 250 to 270 of bf16 products: 16 heads x 1024 queries x 2048 keys.)
constexpr int KEYS = 32;
// Three planes of two numbers, packed in pairs.  (An infinite number's rest would be NaN: it is none.)
__device__ __forceinline__ void split2(float x, float y, uint32_t (&p)[3]) {
#pragma unroll
    for (int i = 0; i < 3; ++i) {
        p[i] = Vec<__nv_bfloat16>::pack2(x, y);
        if (i == 2) break;
        const float a = __uint_as_float(p[i] << 16), b = __uint_as_float(p[i] & 0xffff0000u);
        x = fabsf(a) == INFINITY ? 0.f : x - a;
        y = fabsf(b) == INFINITY ? 0.f : y - b;
    }
}
__device__ __forceinline__ void ldsm4(uint32_t (&r)[4], uint32_t addr) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ldsm4_t(uint32_t (&r)[4], uint32_t addr) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void mma16816(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

template <int D> __global__ void __launch_bounds__(NT64, D == 128 ? 2 : 3) rows64_kernel(const Args a) {
    constexpr int MT = 64, KS = D / 16, PLANE = KEYS * D * 2;            // a plane of the keys or values, bytes
    constexpr bool AHEAD = D == 64;                                      // (with 128 channels the next keys would not fit beside the rest)
    extern __shared__ __align__(128) uint8_t smem[];                     // [K | V][plane][key][D]
    __shared__ bool slive[KEYS];
    const uint32_t base = tc::smem_u32(smem);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, gid = lane >> 2, tig = lane & 3;
    const int u = blockIdx.z, m0 = blockIdx.x * MT + warp * 16;          // this warp's first row
    grid_dependency_wait();
    int r0, r1;
    share<KEYS>(a, u, r0, r1);
    Tile<float, D, KEYS, NT64> t;
    if (AHEAD) t.load(a.k, u, r0, r1);
    uint32_t q[KS][3][4];                                                // planes of rows gid, gid + 8: the first operand
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int m = m0 + gid + h * 8;
        const float* row = (const float*)a.q.q + a.q.at(u, min(m, a.q.rows() - 1)) * D + 2 * tig;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks)
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                const float2 f = __ldg(reinterpret_cast<const float2*>(row + ks * 16 + x * 8));
                uint32_t pl[3];
                split2(f.x * a.scale2, f.y * a.scale2, pl);
#pragma unroll
                for (int i = 0; i < 3; ++i) q[ks][i][x * 2 + h] = pl[i];
            }
    }
    float m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f}, o[D / 8][4]; // rows gid, gid + 8 (l: of this lane's keys); channels 8 j + 2 tig, + 1
#pragma unroll
    for (int j = 0; j < D / 8; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[j][e] = 0.f;
    // (the planes that a product takes: small ones first)
    constexpr int PA[6] = {2, 1, 0, 1, 0, 0}, PB[6] = {0, 1, 2, 0, 1, 0};
    for (int r = r0; r < r1; r += KEYS) {
        __syncthreads();
        if (!AHEAD) t.load(a.k, u, r, r1);
#pragma unroll
        for (int i = 0; i < t.PER; ++i) {
            const int key = (threadIdx.x + i * NT64) / t.LPR, c = (threadIdx.x + i * NT64) % t.LPR * 4;
            uint8_t* at = smem + key * (D * 2) + ((((c >> 3) ^ (key & 7)) << 4) | ((c & 4) << 1));
#pragma unroll
            for (int kv = 0; kv < 2; ++kv) {
                const uint4 f = kv ? t.v[i] : t.k[i];
                uint32_t lo[3], hi[3];
                split2(__uint_as_float(f.x), __uint_as_float(f.y), lo);
                split2(__uint_as_float(f.z), __uint_as_float(f.w), hi);
#pragma unroll
                for (int pl = 0; pl < 3; ++pl) *reinterpret_cast<uint2*>(at + (kv * 3 + pl) * PLANE) = make_uint2(lo[pl], hi[pl]);
            }
        }
        if (threadIdx.x < KEYS) slive[threadIdx.x] = r + (int)threadIdx.x < r1 && exists(a, u, r + threadIdx.x);
        __syncthreads();
        if (AHEAD && r + KEYS < r1) t.load(a.k, u, r + KEYS, r1);
        // ---- logits: 16 rows x 32 keys
        float x[4][4], small[4][4];                                      // keys 8 n + 2 tig, + 1 of rows gid (first two), gid + 8
#pragma unroll
        for (int n = 0; n < 4; ++n)
#pragma unroll
            for (int e = 0; e < 4; ++e) x[n][e] = small[n][e] = 0.f;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
            uint32_t kf[3][2][4];                                        // plane, 16 keys: channels 0..7, 8..15 of the first 8, of the last 8
#pragma unroll
            for (int pl = 0; pl < 3; ++pl)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const int key = h * 16 + (lane & 7) + ((lane >> 4) << 3), piece = ks * 2 + ((lane >> 3) & 1);
                    ldsm4(kf[pl][h], base + pl * PLANE + key * (D * 2) + ((piece ^ (key & 7)) << 4));
                }
#pragma unroll
            for (int i = 0; i < 6; ++i)
#pragma unroll
                for (int n = 0; n < 4; ++n) mma16816(i < 5 ? small[n] : x[n], q[ks][PA[i]], kf[PB[i]][n >> 1][(n & 1) * 2], kf[PB[i]][n >> 1][(n & 1) * 2 + 1]);
        }
        // ---- weights
        float mn[2] = {m[0], m[1]};
#pragma unroll
        for (int n = 0; n < 4; ++n)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                x[n][e] = slive[n * 8 + 2 * tig + (e & 1)] ? x[n][e] + small[n][e] : -INFINITY;
                mn[e >> 1] = fmaxf(mn[e >> 1], x[n][e]);
            }
        float alpha[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            mn[h] = fmaxf(mn[h], __shfl_xor_sync(0xffffffffu, mn[h], 1));
            mn[h] = fmaxf(mn[h], __shfl_xor_sync(0xffffffffu, mn[h], 2));
            alpha[h] = rescale2(m[h], mn[h]);
            m[h] = mn[h];
            l[h] *= alpha[h];
        }
#pragma unroll
        for (int n = 0; n < 4; ++n)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                x[n][e] = rescale2(x[n][e], m[e >> 1]);
                l[e >> 1] += x[n][e];
            }
        if (__any_sync(0xffffffffu, alpha[0] != 1.f || alpha[1] != 1.f))
#pragma unroll
            for (int j = 0; j < D / 8; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e) o[j][e] *= alpha[e >> 1];
        // ---- the weighted sum, 16 keys at a time
#pragma unroll
        for (int kt = 0; kt < 2; ++kt) {
            uint32_t w[3][4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                uint32_t pl[3];
                split2(x[2 * kt + (e >> 1)][(e & 1) * 2], x[2 * kt + (e >> 1)][(e & 1) * 2 + 1], pl);
#pragma unroll
                for (int i = 0; i < 3; ++i) w[i][e] = pl[i];
            }
#pragma unroll
            for (int j = 0; j < D / 16; ++j) {
                uint32_t vf[3][4];                                       // plane: 16 keys of channels 16 j .. + 8, and of the next 8
#pragma unroll
                for (int pl = 0; pl < 3; ++pl) {
                    const int key = kt * 16 + (lane & 15), piece = j * 2 + (lane >> 4);
                    ldsm4_t(vf[pl], base + (3 + pl) * PLANE + key * (D * 2) + ((piece ^ (key & 7)) << 4));
                }
                float c[2][4] = {};
#pragma unroll
                for (int i = 0; i < 6; ++i)
#pragma unroll
                    for (int z = 0; z < 2; ++z) mma16816(c[z], w[PA[i]], vf[PB[i]][z * 2], vf[PB[i]][z * 2 + 1]);
#pragma unroll
                for (int z = 0; z < 2; ++z)
#pragma unroll
                    for (int e = 0; e < 4; ++e) o[2 * j + z][e] += c[z][e];
            }
        }
    }
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        l[h] += __shfl_xor_sync(0xffffffffu, l[h], 1);
        l[h] += __shfl_xor_sync(0xffffffffu, l[h], 2);
        const int row = warp * 16 + gid + h * 8, mr = blockIdx.x * MT + row;
        const bool live = mr < a.q.rows();
        const RowTo<float, D> to(a, u, blockIdx.x, blockIdx.y, row, mr, live, m[h], l[h]);
        __syncwarp();
        if (!live) continue;
#pragma unroll
        for (int j = 0; j < D / 8; ++j) to.template channels<2>(j * 8 + 2 * tig, &o[j][2 * h]);
        if (tig == 0) to.sums();
    }
}

template <int D> cudaError_t launch_t(const Args& a, const F32Plan& plan, int units, cudaStream_t st) {
    const dim3 grid(plan.items, plan.pieces, units);
    if (plan.mt == 8) return launch_dependent(rows8_kernel<float, D>, grid, dim3(NT8), 0, st, a);
    constexpr size_t smem = 6 * KEYS * D * 2;                            // (48 KB of planes and what is static: an opt-in)
    static std::mutex mu;
    static bool ready[KVM_MAX_DEVICES] = {};
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev < 0 || dev >= KVM_MAX_DEVICES) return cudaErrorInvalidDevice;
    {
        std::lock_guard<std::mutex> lock(mu);
        if (!ready[dev]) {
            if ((e = cudaFuncSetAttribute(rows64_kernel<D>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem)) != cudaSuccess) return e;
            ready[dev] = true;
        }
    }
    return launch_dependent(rows64_kernel<D>, grid, dim3(NT64), smem, st, a);
}

}  // namespace

// Pieces: the number whose blocks fill the SMs best in whole rounds of what is at work at the same time (five blocks of 8 rows to an SM; of
// 64 rows two with 128 channels, three with 64), a few per cent given away for each more, but none with less than 128 keys where all are
// there.  (56 units x 160 rows x 3542 keys x 128: 168 blocks in one piece each, 1.8 times what whole rounds take.)
F32Plan f32_plan(int units, int m, int rows, int D) {
    F32Plan p;
    p.mt = m <= 16 ? 8 : 64;
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

cudaError_t launch_rows_f32(const Shape& s, const F32Plan& plan, int units, const Queries& q, const Keys& k, const States& states, const Output& out,
                             kvm_stats* stats, cudaStream_t st) {
    if (units > 65535 || plan.pieces > 65535) return cudaErrorInvalidValue;
    const Args a = {q, k, states, out, stats, s.scale * LOG2E, plan.pieces};
    return s.D == 128 ? launch_t<128>(a, plan, units, st) : launch_t<64>(a, plan, units, st);
}

}  // namespace serve
}  // namespace kvm
