// Appending to a paged cache, with the position rotation on the way:
//   (x, y) -> (x cos a - y sin a, y cos a + x sin a),  a = 2 pi frac(pos * turn_i)
// for the channel pairs i of every new key and query; values are copied.
//
// Bound by bandwidth (each element read and written once) or, for a decode step, by the launch and three dependent reads (length,
// page, row).  A group of D / 2N lanes (N: elements of 16 bytes) owns a token: it computes the token's cosines and sines once and takes
// the token's heads one after the other, ROUND at a time so that their loads leave together.  The angle is an integer product:
// with the frequency as a 64-bit binary fraction of a turn the product with the position wraps around at whole turns, and
// what is left, rounded to 24 bits, is the argument of sincospi, and eight bits more turn its results by their first order: nothing is lost
// for far positions, and no 64-bit floating-point arithmetic (2 results a clock and SM here) is needed.
#include "serve.cuh"

namespace kvm {
namespace serve {
namespace {

constexpr int APPEND_NT = 256;
constexpr int ROUND = 4;                    // heads (of q; half as many of k and v) whose loads leave together

struct AppendArgs {
    const void *q, *k, *v;
    void* q_out;
    long long sq[3], sk[3], sv[3];          // elements from batch entry, head and token to the next
    const uint64_t* turns;
    const int32_t *pos, *new_len;
    int32_t* len_out;                       // nullable: moved by a kernel of its own
    kvm_stats* stats;
    Pages c;
    int B, Hq, Hkv, T, heads;               // heads: per block; a KV head counts as one
};

__device__ __forceinline__ int start_of(const Pages& c, int u) { return max(0, min(__ldcg(c.len + u), c.room())); }
__device__ __forceinline__ int taken(const AppendArgs& a, int u) { return a.new_len ? max(0, min(__ldg(a.new_len + u), a.T)) : a.T; }

template <typename T, int D, bool NEIGHBOURS>
__global__ void __launch_bounds__(APPEND_NT) append_kernel(const AppendArgs a) {
    constexpr int N = Vec<T>::N, LPT = D / (2 * N), TPB = APPEND_NT / LPT;      // lanes per token, tokens per block
    const int lane = threadIdx.x % LPT;
    const long long tokens = (long long)a.B * a.T, x = (long long)blockIdx.x * TPB + threadIdx.x / LPT;
    const unsigned warp_lanes = __ballot_sync(0xffffffffu, x < tokens);
    if (x >= tokens) return;                    // (leaving early counts as letting the next kernel lie ready)
    const int b = (int)(x / a.T), t = (int)(x % a.T);
    const int o0 = NEIGHBOURS ? lane * 2 * N : lane * N, o1 = NEIGHBOURS ? o0 + N : o0 + D / 2;
    grid_dependency_wait();
    grid_launch_dependents();

    float cs[N], sn[N];
    if (a.turns) {
        const uint64_t p = (uint64_t)((long long)__ldg(a.pos + b) + t);
#pragma unroll
        for (int e = 0; e < N; ++e) {
            const uint64_t turn = p * __ldg(reinterpret_cast<const unsigned long long*>(a.turns) + lane * N + e);
            const int32_t a32 = (int32_t)(turn >> 32);                                            // half turns: 2^-31
            const float a24 = (float)a32, rest = (float)(a32 - __float2int_rn(a24)) * 1.4629180792671596e-9f;      // (pi 2^-31)
            float c, d;
            sincospif(a24 * 4.656612873077393e-10f, &d, &c);
            cs[e] = fmaf(-d, rest, c);
            sn[e] = fmaf(c, rest, d);
        }
    }
    auto rotate = [&](uint4& r0, uint4& r1) {
        if (!a.turns) return;
        float f[2 * N];
        Vec<T>::unpack(r0, f);
        Vec<T>::unpack(r1, f + N);
#pragma unroll
        for (int e = 0; e < N; ++e) {
            float& p = NEIGHBOURS ? f[2 * e] : f[e];
            float& q = NEIGHBOURS ? f[2 * e + 1] : f[N + e];
            const float p0 = p, q0 = q;
            p = fmaf(p0, cs[e], -(q0 * sn[e]));
            q = fmaf(q0, cs[e], p0 * sn[e]);
        }
        r0 = Vec<T>::pack(f);
        r1 = Vec<T>::pack(f + N);
    };

    const int j0 = blockIdx.y * a.heads, j1 = min(j0 + a.heads, a.Hkv + a.Hq);
    // ---- keys and values: entries [0, Hkv) of the list of heads
    const T* kt = (const T*)a.k + b * a.sk[0] + t * a.sk[2];
    const T* vt = (const T*)a.v + b * a.sv[0] + t * a.sv[2];
    for (int h0 = j0; h0 < min(j1, a.Hkv); h0 += ROUND / 2) {
        uint4 r[ROUND / 2][4];
        int start[ROUND / 2];
#pragma unroll
        for (int i = 0; i < ROUND / 2; ++i) {
            const int h = min(h0 + i, min(j1, a.Hkv) - 1);
            const T *kr = kt + h * a.sk[1], *vr = vt + h * a.sv[1];
            start[i] = start_of(a.c, b * a.Hkv + h);
            r[i][0] = ldg16(kr + o0);
            r[i][1] = ldg16(kr + o1);
            r[i][2] = ldg16(vr + o0);
            r[i][3] = ldg16(vr + o1);
        }
#pragma unroll
        for (int i = 0; i < ROUND / 2; ++i) {
            const int h = h0 + i, u = b * a.Hkv + h;
            if (h >= min(j1, a.Hkv)) break;
            const int cnt = taken(a, u), row = start[i] + t;
            if (t < cnt) {
                const int page = row < a.c.room() ? __ldg(a.c.table + (size_t)u * a.c.max_pages + (row >> a.c.shift)) : -1;
                if ((unsigned)page < (unsigned)a.c.n_pages) {
                    const size_t at = (((size_t)page << a.c.shift) + (row & ((1 << a.c.shift) - 1))) * D;
                    rotate(r[i][0], r[i][1]);
                    T *ko = (T*)a.c.K + at, *vo = (T*)a.c.V + at;
                    *reinterpret_cast<uint4*>(ko + o0) = r[i][0];
                    *reinterpret_cast<uint4*>(ko + o1) = r[i][1];
                    *reinterpret_cast<uint4*>(vo + o0) = r[i][2];
                    *reinterpret_cast<uint4*>(vo + o1) = r[i][3];
                } else if (a.stats) {
                    a.stats->status = KVM_E_PAGE;
                }
            }
            // (The token's lanes have all read the length, which may be moved in place.  The whole warp takes the same rounds: gathered at once, where
            // each token's lanes by themselves take it apart, 8 x 2048 tokens 65.1 -> 68.2 us.)
            __syncwarp(warp_lanes);
            if (a.len_out && t == 0 && lane == 0) a.len_out[u] = min(start[i] + cnt, a.c.room());
        }
    }
    // ---- queries: the entries behind
    if (!a.q) return;
    const T* qt = (const T*)a.q + b * a.sq[0] + t * a.sq[2];
    for (int h0 = max(j0 - a.Hkv, 0); h0 < j1 - a.Hkv; h0 += ROUND) {
        uint4 r[ROUND][2];
#pragma unroll
        for (int i = 0; i < ROUND; ++i) {
            const T* qr = qt + min(h0 + i, j1 - a.Hkv - 1) * a.sq[1];
            r[i][0] = *reinterpret_cast<const uint4*>(qr + o0);      // (may be the output's memory)
            r[i][1] = *reinterpret_cast<const uint4*>(qr + o1);
        }
#pragma unroll
        for (int i = 0; i < ROUND; ++i) {
            if (h0 + i >= j1 - a.Hkv) break;
            rotate(r[i][0], r[i][1]);
            T* qo = (T*)a.q_out + (((size_t)b * a.Hq + h0 + i) * a.T + t) * D;
            *reinterpret_cast<uint4*>(qo + o0) = r[i][0];
            *reinterpret_cast<uint4*>(qo + o1) = r[i][1];
        }
    }
}

// Lengths in place, where several blocks have read them.
__global__ void __launch_bounds__(APPEND_NT) advance_kernel(const AppendArgs a, int32_t* len) {
    const int u = blockIdx.x * APPEND_NT + threadIdx.x;
    grid_dependency_wait();
    if (u < a.B * a.Hkv) len[u] = min(start_of(a.c, u) + taken(a, u), a.c.room());
}

template <typename T, int D, bool NEIGHBOURS>
cudaError_t launch_t(AppendArgs a, int32_t* len_out, cudaStream_t st) {
    constexpr int TPB = APPEND_NT / (D / (2 * Vec<T>::N));
    const long long tokens = (long long)a.B * a.T, blocks = (tokens + TPB - 1) / TPB;
    if (blocks > 0x7fffffffll) return cudaErrorInvalidValue;
    const int heads = a.Hkv + (a.q ? a.Hq : 0);
    // few tokens: a head or two per block, so that all loads are in flight at once; many: eight heads share the cosines
    a.heads = blocks * heads < 148 * 16 ? 1 : 8;
    // In place a unit's length may only move when all who read it have: with one token per sequence these are the lanes
    // of one group, otherwise a second kernel moves it.
    const bool apart = len_out != a.c.len || a.T == 1;
    a.len_out = apart ? len_out : nullptr;
    cudaError_t e = launch_dependent(append_kernel<T, D, NEIGHBOURS>, dim3((unsigned)blocks, (heads + a.heads - 1) / a.heads), dim3(APPEND_NT),
                                     0, st, a);
    if (e != cudaSuccess || apart) return e;
    return launch_dependent(advance_kernel, dim3((a.B * a.Hkv + APPEND_NT - 1) / APPEND_NT), dim3(APPEND_NT), 0, st, a, len_out);
}

}  // namespace

cudaError_t launch_append(const Shape& s, const Pages& c, int32_t* len_out, int n_new, const int32_t* new_len, const int32_t* pos,
                          const uint64_t* turns, int neighbours, const void* q, const void* k, const void* v, const int64_t* strides,
                          void* q_out, kvm_stats* stats, cudaStream_t st) {
    AppendArgs a = {};
    a.q = q; a.k = k; a.v = v; a.q_out = q_out;
    for (int i = 0; i < 3; ++i) { a.sq[i] = strides[i]; a.sk[i] = strides[3 + i]; a.sv[i] = strides[6 + i]; }
    a.turns = turns; a.pos = pos; a.new_len = new_len; a.stats = stats;
    a.c = c; a.B = s.B; a.Hq = s.Hq; a.Hkv = s.Hkv; a.T = n_new;
    auto fn = s.dtype == KVM_BF16 ? (s.D == 128 ? (neighbours ? launch_t<__nv_bfloat16, 128, true> : launch_t<__nv_bfloat16, 128, false>)
                                                : (neighbours ? launch_t<__nv_bfloat16, 64, true> : launch_t<__nv_bfloat16, 64, false>))
                                  : (s.D == 128 ? (neighbours ? launch_t<float, 128, true> : launch_t<float, 128, false>)
                                                : (neighbours ? launch_t<float, 64, true> : launch_t<float, 64, false>));
    return fn(a, len_out, st);
}

}  // namespace serve
}  // namespace kvm
