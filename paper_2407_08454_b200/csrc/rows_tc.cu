// Attention of a unit's query rows over its keys on the 5th-generation tensor cores (bf16), without a mask but the unit's length:
//   O = softmax(c Q K^T) V,  lse = ln sum exp(c q.k)
// The query rows that share keys lie together (the query heads of a KV head, all their queries; or the whole batch over a shared
// prefix), so that two tiles of 128 rows take each key and value tile from shared memory once:
//   S_g = Q_g K_j^T  ->  P_g = exp(S_g - reference), written over S_g in tensor memory  ->  O_g += P_g V_j,   g = 0, 1,
// as the two-tile kernel of the prefill attention does, whose pipeline this is: softmax group g owns tile g, one thread's products
// of one tile run while the other tile's exponentials do.  What differs:
//   - The work is a list of items (unit, pair of tiles), each with as many steps as the unit has key tiles, and a CTA takes an
//     equal share of all steps: a decode batch over one prefix has 8 items for 148 CTAs, a chunk of a prompt 512, lengths differ by unit.
//     An item that falls into several shares leaves the states of its pieces (O, reference, sums), which another kernel joins.
//   - Where a unit has one tile of queries only (a few drafted tokens, a small batch over a prefix) both groups work on it, on alternate key
//     tiles, so that one's exponentials run under the other's products here too; their states are joined like those of pieces.
//   - The last key tile is cut where the unit ends: logits beyond are -inf, and what V holds there, which may be anything, is kept out
//     of the product (16 keys at a time; the last ones' rows of V are zeroed in shared memory).
// Weights are rounded to bf16 for the second product and divided by the sum of the rounded ones: their rest as a second product would add half
// as many clocks again to the 2,048 that a pair's step has of products.
// Bound by the exponentials and the softmax around them where there are many rows (see prefill_tc.cu for the clocks), by bandwidth where
// a unit has one tile (64 KB of keys and values per step of about 2,800 clocks at an SM's share).
#include <float.h>

#include <initializer_list>
#include <mutex>
#include <type_traits>

#include "serve.cuh"
#include "tc_common.cuh"

namespace kvm {
namespace serve {
namespace {

using namespace tc;

constexpr int TILE = 128;
constexpr int KCHUNK = 64;
constexpr int NST = 2;                  // iterations in the rings of K and V tiles
constexpr int NSOFT = 8;                // softmax warps: four per tile
constexpr int NTHREADS = (NSOFT + 4) * 32;
// 2 x 128 x 208 + 128 x 88 = 384 x 168, the registers that the block is launched with
constexpr int REGS_SOFTMAX = 208, REGS_OTHER = 88;
constexpr uint32_t CHUNK_BYTES = TILE * 128;            // [128 rows x 64 bf16]
constexpr float RESCALE_STEP = 8.f;     // a row's reference moves when outgrown by this (log2 units): a weight is at most 2^8
constexpr int P_FIRST = 96;             // keys of a step whose P is handed over first
constexpr uint32_t S_COLS = TILE, O_COL0 = 2 * S_COLS;
constexpr int NEAR = 64;
constexpr float LOWEST = -FLT_MAX;      // the reference before the first key, which any logit outgrows (a row of -inf logits keeps it, and weighs nothing)

struct __align__(8) Bars {
    uint64_t q_full[2], q_empty[2], k0_full, k0_done;   // an item's Q tiles; its first K tile, loaded and used
    uint64_t kv_full[NST], kv_empty[NST];               // iteration j: V tile j and K tile j + 1
    uint64_t s_full[2], p_full[2][2], o_full[2];
};
struct Args {
    Output out;
    States st;
    const int32_t* len;
    int rows, units, tiles, alt, whole, direct;      // direct: an item in one piece goes to the output, else to slot 2 * gridDim.x + its number
    int gx, bx, per_block;              // a tile's box, tiles per block of more than 128 rows
    int m;                              // query rows of a unit
    float scale2;
    kvm_stats* stats;
    Beside own;                         // the kernel that runs beside this one
};

// A part of an item: key tiles [k0, k1) of `nk` for query tiles 2 * pair, 2 * pair + 1 of unit u.
struct Piece {
    int u, pair, k0, k1, nk, n;         // n: keys of the unit
    __device__ __forceinline__ int steps() const { return k1 - k0; }
    __device__ __forceinline__ bool whole() const { return k0 == 0 && k1 == nk; }
};
// A CTA's walk over its share of the steps.
struct Walk {
    const int32_t *len, *near;                  // near: the lengths of the first NEAR units of the share, in shared memory
    int rows, units, pairs, u0;
    int u, pair, n, nk, whole;                  // whole: items are not cut: a share is the items that begin in it
    unsigned long long q, f, f_end, start;      // steps per share; what is left of it; steps before the current item
    __device__ __forceinline__ int rows_of(int unit) const { return len ? max(0, min(__ldg(len + unit), rows)) : rows; }
    __device__ __forceinline__ int next_rows(int unit) const { return unit - u0 < NEAR ? near[unit - u0] : rows_of(unit); }
    __device__ __forceinline__ static int tiles_of(int n) { return (n + TILE - 1) / TILE; }
    __device__ __forceinline__ bool next(Piece& p) {
        while (f < f_end) {
            if (f < start + nk) {
                p.u = u; p.pair = pair; p.nk = nk; p.n = n;
                p.k0 = (int)(f - start);
                p.k1 = whole ? nk : (int)(min(start + nk, f_end) - start);
                f += p.k1 - p.k0;
                return true;
            }
            start += nk;
            if (nk == 0 || ++pair == pairs) {
                pair = 0;
                if (++u >= units) return false;
                n = next_rows(u);
                nk = tiles_of(n);
            }
        }
        return false;
    }
    // slot of a piece that is not its whole item: each share has at most one that begins before it and one that ends behind it
    __device__ __forceinline__ static int slot(const Piece& p) { return 2 * blockIdx.x + (p.k0 > 0 ? 0 : 1); }
};

struct alignas(16) Shared {
    Bars bar;
    uint32_t tmem_base;
    int abort_flag;
    long long wsum[NTHREADS / 32];
    unsigned long long start;
    int unit, near[NEAR];
    Walk walk[NSOFT];                   // of the softmax warps, whose registers hold the logits
    Piece piece[NSOFT];
};

// This CTA's share, by a prefix sum over the units (all threads; false: nothing to do).
__device__ __forceinline__ bool take_share(Walk& w, const Beside& own, int D, Shared& sh) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int E = (w.units + NTHREADS - 1) / NTHREADS, i0 = min(w.units, (int)threadIdx.x * E), i1 = min(w.units, i0 + E);
    unsigned long long mine = 0;
    for (int i = i0; i < i1; ++i) mine += (unsigned long long)Walk::tiles_of(w.rows_of(i)) * w.pairs;
    unsigned long long inc = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const unsigned long long t = __shfl_up_sync(0xffffffffu, inc, o);
        if (lane >= o) inc += t;
    }
    if (lane == 31) sh.wsum[warp] = (long long)inc;
    __syncthreads();
    unsigned long long total = 0, before = inc - mine;
#pragma unroll
    for (int x = 0; x < NTHREADS / 32; ++x) {
        if (x < warp) before += (unsigned long long)sh.wsum[x];
        total += (unsigned long long)sh.wsum[x];
    }
    // (beside another kernel the CTAs of the SMs that it gets have nothing to do)
    unsigned ctas = gridDim.x;
    if (own.units) ctas = min(ctas, (unsigned)prefix_sms((long long)total, block_sum<NTHREADS>(own.part(NTHREADS), sh.wsum), D));
    w.q = (total + ctas - 1) / ctas;
    w.f = blockIdx.x < ctas ? min(total, w.q * blockIdx.x) : total;
    w.f_end = min(total, w.f + w.q);
    w.u = w.u0 = w.n = w.nk = w.pair = 0;
    w.start = 0;
    if (w.f == w.f_end) return false;
    if (before <= w.f && w.f < before + mine) {                    // true in exactly one thread
        unsigned long long st = before;
        int id = i0;
        for (;; ++id) {
            const unsigned long long n = (unsigned long long)Walk::tiles_of(w.rows_of(id)) * w.pairs;
            if (st + n > w.f) break;
            st += n;
        }
        sh.start = st;
        sh.unit = id;
    }
    __syncthreads();
    w.u = w.u0 = sh.unit;
    w.near = sh.near;
    if (threadIdx.x < NEAR) sh.near[threadIdx.x] = w.rows_of(min(w.u + (int)threadIdx.x, w.units - 1));
    __syncthreads();
    w.n = sh.near[0];
    w.nk = Walk::tiles_of(w.n);
    w.pair = (int)((w.f - sh.start) / w.nk);
    w.start = sh.start + (unsigned long long)w.pair * w.nk;
    if (w.whole && w.f > w.start) w.f = w.start + w.nk;            // the item that began before belongs to that share
    return true;
}

__device__ __forceinline__ void tma_load_4d(void* dst, const CUtensorMap* map, uint64_t* bar, int x, int y, int z, int w) {
    asm volatile(
        "cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6}], [%2];"
        ::"r"(smem_u32(dst)), "l"(map), "r"(smem_u32(bar)), "r"(x), "r"(y), "r"(z), "r"(w)
        : "memory");
}
__device__ __forceinline__ void tma_store_2d(const CUtensorMap* map, const void* src, int x, int y) {
    asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.bulk_group [%0, {%2, %3}], [%1];" ::"l"(map), "r"(smem_u32(src)), "r"(x), "r"(y)
                 : "memory");
    asm volatile("cp.async.bulk.commit_group;" ::: "memory");
}

template <int KCH, bool COMPACT>
__global__ void __launch_bounds__(NTHREADS, 1)
rows_tc_kernel(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v,
               const __grid_constant__ CUtensorMap map_o, const __grid_constant__ CUtensorMap map_s, const __grid_constant__ Args a) {
    constexpr int D = KCH * KCHUNK;
    constexpr uint32_t TILE_BYTES = KCH * CHUNK_BYTES;
    extern __shared__ uint8_t smem_raw[];
    const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    uint8_t* sQ = smem_raw + (base - smem_u32(smem_raw));  // two Q tiles
    uint8_t* sK = sQ + 2 * TILE_BYTES;
    uint8_t* sV = sK + NST * TILE_BYTES;
    uint8_t* sO = sV + NST * TILE_BYTES;                   // 32 rows of 128 bytes per softmax warp
    Shared& sh = *reinterpret_cast<Shared*>(sO + NSOFT * 4096);
    volatile int* abort_flag = &sh.abort_flag;

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (threadIdx.x == 0) {
        mbar_init(&sh.bar.k0_full, 1); mbar_init(&sh.bar.k0_done, 1);
        for (int i = 0; i < NST; ++i) { mbar_init(&sh.bar.kv_full[i], 1); mbar_init(&sh.bar.kv_empty[i], 1); }
        for (int g = 0; g < 2; ++g) {
            mbar_init(&sh.bar.q_full[g], 1); mbar_init(&sh.bar.q_empty[g], 1);
            mbar_init(&sh.bar.s_full[g], 1); mbar_init(&sh.bar.o_full[g], 1);
            for (int h = 0; h < 2; ++h) mbar_init(&sh.bar.p_full[g][h], 4);
        }
        sh.abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        for (const CUtensorMap* map : {&map_q, &map_k, &map_v, &map_o, &map_s}) asm volatile("prefetch.tensormap [%0];" ::"l"(map) : "memory");
    }
    grid_dependency_wait();
    grid_launch_dependents();                              // (the kernel beside this one begins, or the one that joins lies ready)
    Walk walk;
    walk.len = a.len; walk.rows = a.rows; walk.units = a.units; walk.whole = a.whole; walk.pairs = (a.tiles + 1) / 2;
    if (!take_share(walk, a.own, D, sh) && !(a.whole && a.direct && a.len)) return;
    if (a.gx * a.bx < TILE) {                              // rows of a Q tile that no copy fills: zeros
        for (int i = threadIdx.x; i < (int)(2 * TILE_BYTES / 16); i += NTHREADS) reinterpret_cast<uint4*>(sQ)[i] = make_uint4(0, 0, 0, 0);
        fence_proxy_async();
    }
    if (warp == NSOFT + 1) tmem_alloc(&sh.tmem_base, 512);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem_base = sh.tmem_base;
    if (warp >= NSOFT) {
      Piece p;
      asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(REGS_OTHER));
      if (warp == NSOFT) {
        // ============================== producer ==============================
        if (lane == 0) {
            uint32_t kv = 0;                                  // K tiles (= V tiles = iterations) before this piece
            uint32_t q_ph = 0;                                // bit g: phase of Q tile g
            bool ok = true;
            auto load = [&](uint8_t* dst, const CUtensorMap* map, uint64_t* bar, int t, int u) {
#pragma unroll
                for (int kc = 0; kc < KCH; ++kc) tma_load_3d(dst + kc * CHUNK_BYTES, map, bar, kc * KCHUNK, t * TILE, u);
            };
            for (int i = 0; ok && walk.next(p); ++i) {
                const int len = p.steps();
                if (i > 0) ok = mbar_wait(&sh.bar.k0_done, (i & 1) ^ 1, abort_flag);
                if (!ok) break;
                mbar_expect_tx(&sh.bar.k0_full, TILE_BYTES);
                load(sK + (kv % NST) * TILE_BYTES, &map_k, &sh.bar.k0_full, p.k0, p.u);
                for (int g = 0; ok && g < 2; ++g) {
                    const int t = 2 * p.pair + g;
                    if (t >= a.tiles) continue;
                    ok = mbar_wait(&sh.bar.q_empty[g], ((q_ph >> g) & 1) ^ 1, abort_flag);
                    if (!ok) break;
                    q_ph ^= 1u << g;
                    const int y = a.per_block ? t % a.per_block * TILE : 0, z = a.per_block ? t / a.per_block : t * a.bx;
                    mbar_expect_tx(&sh.bar.q_full[g], (uint32_t)(KCH * 128 * a.gx * a.bx));
#pragma unroll
                    for (int kc = 0; kc < KCH; ++kc)
                        tma_load_4d(sQ + g * TILE_BYTES + kc * CHUNK_BYTES, &map_q, &sh.bar.q_full[g], kc * KCHUNK, y, z, p.u);
                }
                for (int j = 0; ok && j < len; ++j) {
                    const uint32_t x = kv + (uint32_t)j, s = x % NST;
                    ok = mbar_wait(&sh.bar.kv_empty[s], ((x / NST) & 1) ^ 1, abort_flag);
                    if (j == 1) ok = ok && mbar_wait(&sh.bar.k0_done, i & 1, abort_flag);   // K tile 2 takes the first one's place
                    if (!ok) break;
#ifdef KVM_TEST_DROP_B_STAGE
                    if (x == (uint32_t)(KVM_TEST_DROP_B_STAGE)) continue;   // test build only: these tiles never arrive
#endif
                    mbar_expect_tx(&sh.bar.kv_full[s], TILE_BYTES * (1u + (j + 1 < len)));
                    if (j + 1 < len) load(sK + ((x + 1) % NST) * TILE_BYTES, &map_k, &sh.bar.kv_full[s], p.k0 + j + 1, p.u);
                    load(sV + s * TILE_BYTES, &map_v, &sh.bar.kv_full[s], p.k0 + j, p.u);
                }
                kv += (uint32_t)len;
            }
            if (*abort_flag)                                  // copies already issued land (bounded)
                for (uint32_t it = 0; it < (1u << 14); ++it) mbar_try(&sh.bar.k0_full, 0);
        }
      } else if (warp == NSOFT + 1) {
        // ============================== MMA issue ==============================
        constexpr uint32_t IDESC_S = idesc_bf16(TILE), IDESC_O = idesc_bf16(D, true);
        const uint64_t dq = smem_desc(base), dk = smem_desc(base + 2 * TILE_BYTES);
        const uint64_t dv = smem_desc_mn(base + (2 + NST) * TILE_BYTES, CHUNK_BYTES);
        const uint32_t q_lo = (uint32_t)dq, k_lo = (uint32_t)dk, hi = (uint32_t)(dk >> 32), v_lo = (uint32_t)dv, v_hi = (uint32_t)(dv >> 32);
        uint32_t kv = 0, p_ph = 0, q_ph = 0;                 // iterations before this piece; phases of P and Q (bit g)
        bool ok = true;
        auto logits = [&](int g, int qt, uint32_t x, bool last) {         // S_g = Q K^T of Q tile qt with K tile number x; that Q tile's last one
            if (elect_one()) {
#pragma unroll
                for (int kc = 0; kc < KCH; ++kc)
#pragma unroll
                    for (int ks = 0; ks < KCHUNK / 16; ++ks)
                        umma_bf16_lo(tmem_base + g * S_COLS, q_lo + ((qt * TILE_BYTES + kc * CHUNK_BYTES + ks * 32) >> 4), hi,
                                     k_lo + (x % NST) * (TILE_BYTES >> 4) + ((kc * CHUNK_BYTES + ks * 32) >> 4), hi, IDESC_S, (kc | ks) ? 1u : 0u);
                umma_commit(&sh.bar.s_full[g]);
                if (last) umma_commit(&sh.bar.q_empty[qt]);
            }
        };
        // A piece's first logits of a tile come right after the tile's last P V of the piece before (the walk starts with a piece of
        // no steps).  The tiles take turns in a loop, so that the instructions are there once: they are fetched anew by every launch.
        Piece nx;
        bool has_next = walk.next(nx);
        p.u = p.pair = p.k0 = p.k1 = p.nk = p.n = 0;
        auto next_piece_here = [&](int g, int i) {           // its first K and Q tiles are there; false: it has no such tile
            if (2 * nx.pair + g >= a.tiles) return false;
            ok = ok && mbar_wait_warp(&sh.bar.k0_full, i & 1, abort_flag) && mbar_wait_warp(&sh.bar.q_full[g], (q_ph >> g) & 1, abort_flag);
            if (!ok) return false;
            q_ph ^= 1u << g;
            tc_fence_after();
            return true;
        };
        for (int i = 0;; ++i) {                              // (number of the piece after p)
            const int len = p.steps(), both = len > 0 && 2 * p.pair + 1 < a.tiles;
#pragma unroll 1
            for (int j = 0; ok && j < len; ++j) {
                const uint32_t x = kv + (uint32_t)j, s = x % NST;
                ok = mbar_wait_warp(&sh.bar.kv_full[s], (x / NST) & 1, abort_flag);
                // the unit's last tile: 16 keys at a time as far as there are any, zeros in V for those of them that do not exist
                int slices = TILE / 16;
                if (p.k0 + j == p.nk - 1) {
                    const int live = p.n - (p.nk - 1) * TILE;
                    slices = (live + 15) / 16;
                    if (ok && (live & 15)) {
                        for (int r = live + lane / 8; r < slices * 16; r += 4)
#pragma unroll
                            for (int kc = 0; kc < KCH; ++kc)
                                *reinterpret_cast<uint4*>(sV + s * TILE_BYTES + kc * CHUNK_BYTES + r * 128 + (lane % 8) * 16) = make_uint4(0, 0, 0, 0);
                        fence_proxy_async();
                        __syncwarp();
                    }
                }
                // (a single tile: both groups work on it, on alternate key tiles; the next logits are made beside this step's softmax)
                const int g0 = a.alt ? j & 1 : 0, g1 = a.alt ? g0 + 1 : 1 + both;
                if (a.alt && ok && j + 1 < len) logits((j + 1) & 1, 0, x + 1, j + 2 == len);
#pragma unroll 1
                for (int g = g0; g < g1; ++g) {
                    if (!ok) break;
#pragma unroll
                    for (int h = 0; h < 2; ++h) {            // the first keys' products run while the last ones' P is made
                        ok = ok && mbar_wait_warp(&sh.bar.p_full[g][h], (p_ph >> g) & 1, abort_flag);
                        if (!ok) break;
                        tc_fence_after();
                        if (elect_one()) {
#pragma unroll
                            for (int kk = h ? P_FIRST / 16 : 0; kk < (h ? TILE / 16 : P_FIRST / 16); ++kk)   // 16 keys per MMA: 8 columns of P, 2 KB of V
                                if (kk < slices)
                                    umma_bf16_ts(tmem_base + O_COL0 + g * D, tmem_base + g * S_COLS + kk * 8,
                                                 v_lo + s * (TILE_BYTES >> 4) + ((kk * 16 * 128) >> 4), v_hi, IDESC_O, (j > a.alt || kk) ? 1u : 0u);
                            if (h && j >= len - 1 - a.alt) umma_commit(&sh.bar.o_full[g]);
                        }
                    }
                    if (!ok) break;
                    p_ph ^= 1u << g;
                    const bool more = j + 1 < len;
                    const int t = a.alt ? 0 : g;             // (of a single tile the other logits have been issued above)
                    if (more ? !a.alt : has_next && next_piece_here(t, i))
                        logits(t, t, more ? x + 1 : kv + (uint32_t)len, more ? j + 2 == len : nx.steps() == 1);
                }
                if (ok && elect_one()) umma_commit(&sh.bar.kv_empty[s]);
            }
            if (!ok || !has_next) break;
#pragma unroll 1
            for (int g = len > 0 ? 1 + both : 0; g < 2; ++g)
                if (next_piece_here(g, i)) logits(g, g, kv + (uint32_t)len, nx.steps() == 1);
            if (!ok) break;
            if (elect_one()) umma_commit(&sh.bar.k0_done);
            kv += (uint32_t)len;
            p = nx;
            has_next = walk.next(nx);
        }
      } else if (warp == NSOFT + 3) {
        // ============================== units without keys ==============================
        // (where items are cut, the kernel that joins their pieces sees to these)
        if (a.whole && a.direct && a.len)
            for (int u0 = 0; u0 < a.units; u0 += 32) {
                uint32_t empty = __ballot_sync(0xffffffffu, u0 + lane < a.units && walk.rows_of(min(u0 + lane, a.units - 1)) == 0);
                for (; empty; empty &= empty - 1)
                    for (int r = blockIdx.x; r < a.m; r += gridDim.x) {      // every CTA a part of the unit's rows
                        const long long at = (long long)(u0 + __ffs(empty) - 1) * a.m + r;
                        const float z = a.out.lse_in ? a.out.lse_in[at] : -INFINITY;
                        if (lane * 8 < D) {
                            uint4 x = make_uint4(0, 0, 0, 0);
                            if (z != -INFINITY) x = __ldcg(reinterpret_cast<const uint4*>((const __nv_bfloat16*)a.out.O_in + at * D) + lane);
                            reinterpret_cast<uint4*>((__nv_bfloat16*)a.out.O + at * D)[lane] = x;
                        }
                        __syncwarp();
                        if (lane == 0) a.out.lse[at] = z;
                    }
            }
      }
    } else {
        // ============================== softmax of tile g ==============================
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(REGS_SOFTMAX));
        const int g = warp >> 2, lq = warp & 3;
        const int row = lq * 32 + lane;                      // query row of the tile = TMEM lane
        const uint32_t t_lane = tmem_base + ((uint32_t)(lq * 32) << 16);
        const uint32_t t_s = t_lane + g * S_COLS, t_o = t_lane + O_COL0 + g * D;
        const uint64_t sc2 = pack2(a.scale2, a.scale2);
        uint32_t s_ph = 0, o_ph = 0;
        bool ok = true;
        Walk& mine = sh.walk[warp];
        if (lane == 0) mine = walk;
        // (lane 0 walks one piece ahead, so that what the lengths take to arrive is hidden)
        bool ahead = lane == 0 && mine.next(sh.piece[warp]);
        for (;;) {
            const bool more = __any_sync(0xffffffffu, ahead);
            __syncwarp();
            if (!more) break;
            const Piece p = sh.piece[warp];
            const int pairs = mine.pairs, item = p.u * pairs + p.pair;
            __syncwarp();
            if (lane == 0) {
                if (warp == 0 && p.k0 == 0) {                // (also where a wait gave up: whoever joins reads it)
                    const unsigned long long s0 = mine.f - p.steps();
                    const int last = (int)((s0 + p.nk - 1) / mine.q), count = mine.whole ? 1 : last - (int)blockIdx.x + 1;
                    a.st.pieces[item] = make_int4(count, count > 1 ? 2 * blockIdx.x + 1 : 2 * gridDim.x + item, 2 * blockIdx.x + 2, 0);
                }
                ahead = mine.next(sh.piece[warp]);
            }
            const int tile = a.alt ? 0 : 2 * p.pair + g;
            if (tile >= a.tiles) continue;
            const int k0 = a.alt ? p.k0 + g : p.k0, k1 = p.k1, kstep = 1 + a.alt, last_live = p.k1 == p.nk ? p.n - (p.nk - 1) * TILE : TILE;   // keys of the last step
            float m = LOWEST, l = 0.f, lr = 0.f;             // reference (log2 units); sums relative to it: exact, of the rounded weights
#pragma unroll 1
            for (int j = k0; j < k1; j += kstep) {
                ok = ok && mbar_wait(&sh.bar.s_full[g], s_ph, abort_flag);
                ok = __all_sync(0xffffffffu, ok);
                if (!ok) break;
                s_ph ^= 1;
                tc_fence_after();
                // p = 2^(x - m), summed in fp32, rounded to bf16 for the tensor core.
                uint64_t sum[2] = {0ull, 0ull};
                float rsum[4] = {0.f, 0.f, 0.f, 0.f};
                float pk[16];                                // (two bf16 each)
                float alpha = 1.f;
                auto exponentials = [&](const float* v) {    // of 32 keys
                    const uint64_t nm2 = pack2(-m, -m);
#pragma unroll
                    for (int c = 0; c < 32; c += 2) {
                        float x0, x1;
                        unpack2(ffma2(pack2(v[c], v[c + 1]), sc2, nm2), x0, x1);
                        const float e0 = ex2(x0), e1 = ex2(x1);
                        sum[(c >> 1) & 1] = fadd2(sum[(c >> 1) & 1], pack2(e0, e1));
                        const uint32_t r = Vec<__nv_bfloat16>::pack2(e0, e1);
                        add_bf16x2(rsum[c & 2], rsum[(c & 2) + 1], r);
                        pk[c >> 1] = __uint_as_float(r);
                    }
                };
                auto move_reference = [&](float mx) {        // of the rows that have outgrown theirs, and of all O
                    if (mx > m) { alpha = ex2(m - mx); m = mx; }
                    if (j == k0) return;                     // (an S that is there says that the last P V is done)
#pragma unroll 1
                    for (int q = 0; q < D / 16; ++q) {
                        float o[16];
                        tmem_ld16(t_o + q * 16, o);
#pragma unroll
                        for (int c = 0; c < 16; ++c) o[c] *= alpha;
                        tmem_st16(t_o + q * 16, o);
                    }
                };
                auto hand_over = [&](int q) {                // P of quarter q is in tensor memory
                    if (q == P_FIRST / 32 - 1 || q == 3) {   // (96 keys first: their products run while the last ones' P is made)
                        tmem_st_wait();
                        tc_fence_before();
                        __syncwarp();
                        if (lane == 0) mbar_arrive(&sh.bar.p_full[g][q == 3]);
                    }
                };
                const int live = j == k1 - 1 ? last_live : TILE;
                if (COMPACT) {
                    // Short shares: a quarter of the step at a time, read twice from tensor memory.  Three times less instructions to fetch
                    // by a launch that executes them a few times only.
                    auto load = [&](int q, float* v) {
                        uint32_t r[32];
                        tmem_ld32_issue(t_s + q * 32, r);
                        tmem_ld_wait();
                        tmem_ld_fence(r);
#pragma unroll
                        for (int c = 0; c < 32; ++c) v[c] = __uint_as_float(r[c]);
                        const int there = live - q * 32;     // keys that exist
                        if (there < 32)
#pragma unroll
                            for (int c = 0; c < 32; ++c)
                                if (c >= there) v[c] = -INFINITY;
                    };
                    float mx = -INFINITY, v[32];
#pragma unroll 1
                    for (int q = 0; q < 4; ++q) {
                        load(q, v);
#pragma unroll
                        for (int c = 0; c < 32; c += 2) mx = fmax3(mx, v[c], v[c + 1]);
                    }
                    mx *= a.scale2;
                    if (__any_sync(0xffffffffu, mx > m + RESCALE_STEP)) move_reference(mx);
#pragma unroll 1
                    for (int q = 0; q < 4; ++q) {
                        load(q, v);
                        exponentials(v);
                        tmem_st16(t_s + q * 16, pk);
                        hand_over(q);
                    }
                } else {
                    uint32_t vr[TILE];
#pragma unroll
                    for (int q = 0; q < 4; ++q) tmem_ld32_issue(t_s + q * 32, vr + q * 32);
                    tmem_ld_wait();
#pragma unroll
                    for (int q = 0; q < 4; ++q) tmem_ld_fence(vr + q * 32);
                    float v[TILE];
#pragma unroll
                    for (int c = 0; c < TILE; ++c) v[c] = __uint_as_float(vr[c]);
                    if (live < TILE) {                       // keys that do not exist
#pragma unroll
                        for (int q = 0; q < 4; ++q)
                            if (live < q * 32 + 32) {
#pragma unroll
                                for (int c = q * 32; c < q * 32 + 32; ++c)
                                    if (c >= live) v[c] = -INFINITY;
                            }
                    }
                    // The first 32 keys are tried with the reference as it is, beside the search for the step's maximum: the warp's
                    // references move only when a row's maximum has outgrown its own by RESCALE_STEP, seldom after the first step.
                    bool again = false;
#pragma unroll 1
                    for (;;) {                               // (a loop, so that the instructions are there once)
                        exponentials(v);
                        if (again) break;
                        float mx4[4] = {v[0], v[1], v[2], v[3]};
#pragma unroll
                        for (int c = 4; c + 7 < TILE; c += 8)
#pragma unroll
                            for (int e = 0; e < 4; ++e) mx4[e] = fmax3(mx4[e], v[c + e], v[c + 4 + e]);
#pragma unroll
                        for (int e = 0; e < 4; ++e) mx4[e] = fmaxf(mx4[e], v[TILE - 4 + e]);
                        const float mx = fmaxf(fmax3(mx4[0], mx4[1], mx4[2]), mx4[3]) * a.scale2;
                        if (!__any_sync(0xffffffffu, mx > m + RESCALE_STEP)) break;
                        move_reference(mx);
                        sum[0] = sum[1] = 0ull;
                        rsum[0] = rsum[1] = rsum[2] = rsum[3] = 0.f;
                        again = true;
                    }
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        if (q > 0) exponentials(v + q * 32);
                        tmem_st16(t_s + q * 16, pk);
                        hand_over(q);
                    }
                }
                float s0, s1;
                unpack2(fadd2(sum[0], sum[1]), s0, s1);
                l = l * alpha + (s0 + s1);
                lr = lr * alpha + ((rsum[0] + rsum[1]) + (rsum[2] + rsum[3]));
            }
            // ---- the piece's end
            const bool none = k0 >= k1;                      // (a single step is the first group's)
            ok = ok && (none || mbar_wait(&sh.bar.o_full[g], o_ph, abort_flag));
            ok = __all_sync(0xffffffffu, ok);
            const bool direct = a.direct && p.whole();
            const long long slot = p.whole() ? 2ll * gridDim.x + item : Walk::slot(p);
            const long long srow = slot * a.st.rows + g * TILE + row;
            const int in = tile * TILE + row;                // (direct: row of the unit)
            const bool live = direct ? in < a.m : row < a.gx * a.bx;
            const long long orow = (long long)p.u * a.m + in;
            uint8_t* buf = sO + warp * 4096;
            if (!ok) {
                // a wait gave up: what this row, and those of the pieces after it, would have received is marked, not made up
                if (direct && live) {
                    __nv_bfloat16* o = (__nv_bfloat16*)a.out.O + orow * D;
                    for (int c = 0; c < D; c += 8)
                        *reinterpret_cast<uint4*>(o + c) = make_uint4(0x7FC07FC0u, 0x7FC07FC0u, 0x7FC07FC0u, 0x7FC07FC0u);
                    a.out.lse[orow] = NAN;
                } else if (!direct) {
                    a.st.ml[srow] = make_float4(0.f, NAN, NAN, 0.f);
                }
                continue;
            }
            if (none) {
                a.st.ml[srow] = make_float4(LOWEST, 0.f, 0.f, 0.f);
                continue;
            }
            o_ph ^= 1;
            tc_fence_after();
            // Logits enter the exponent by one multiply-add, less a reference that is a rounded product.  From 2^27 on half a step of it is more than
            // exponentials bear: all weights of the row may be 0 or one infinite.  Such a row says so.  (Products rounded first would do, by a branch
            // in every step: 3 % of all calls' time.)
            if (m != LOWEST && !(l > 0.f && l < INFINITY)) l = lr = NAN;
            // 128 bytes of the warp's 32 rows at a time through shared memory to the copy engine, which takes them out beside the next
            // piece (stored by the threads, 64 KB of two tiles hold the softmax up for 2,000 clocks more).
            // (In loops: unrolled, these instructions are fetched anew for every piece.)
            const RowEnd end(m, l, lr, direct && live ? a.out.lse_in : nullptr, orow);
            if (!direct) {
#pragma unroll 1
                for (int q = 0; q < D / 32; ++q) {
                    uint32_t o[32];
                    tmem_ld32_issue(t_o + q * 32, o);
                    tmem_ld_wait();
                    tmem_ld_fence(o);
                    if (lane == 0) bulk_wait_read();
                    __syncwarp();
#pragma unroll
                    for (int c = 0; c < 8; ++c)
                        *reinterpret_cast<uint4*>(buf + lane * 128 + ((c ^ (lane & 7)) << 4)) = make_uint4(o[4 * c], o[4 * c + 1], o[4 * c + 2], o[4 * c + 3]);
                    fence_proxy_async();
                    __syncwarp();
                    if (lane == 0 && lq * 32 < a.gx * a.bx) tma_store_2d(&map_s, buf, q * 32, (int)(srow - lane));
                }
            } else {
                const uint64_t f2 = pack2(end.f, end.f);
#pragma unroll 1
                for (int kc = 0; kc < KCH; ++kc) {
                    uint32_t o[64];
                    tmem_ld32_issue(t_o + kc * 64, o);
                    tmem_ld32_issue(t_o + kc * 64 + 32, o + 32);
                    tmem_ld_wait();
                    tmem_ld_fence(o);
                    tmem_ld_fence(o + 32);
                    if (lane == 0) bulk_wait_read();
                    __syncwarp();
#pragma unroll
                    for (int c = 0; c < 8; ++c) {
                        float y[8];
#pragma unroll
                        for (int e = 0; e < 8; e += 2)
                            unpack2(fmul2(pack2(__uint_as_float(o[c * 8 + e]), __uint_as_float(o[c * 8 + e + 1])), f2), y[e], y[e + 1]);
                        if (end.f_in != 0.f) {               // (only where O_in is given)
                            float x[8];
                            Vec<__nv_bfloat16>::unpack(__ldcg(reinterpret_cast<const uint4*>((const __nv_bfloat16*)a.out.O_in + orow * D + kc * 64) + c), x);
#pragma unroll
                            for (int e = 0; e < 8; ++e) y[e] = fmaf(x[e], end.f_in, y[e]);
                        }
                        *reinterpret_cast<uint4*>(buf + lane * 128 + ((c ^ (lane & 7)) << 4)) = Vec<__nv_bfloat16>::pack(y);
                    }
                    fence_proxy_async();
                    __syncwarp();
                    if (lane == 0 && tile * TILE + lq * 32 < a.m) tma_store_3d(&map_o, buf, kc * KCHUNK, tile * TILE + lq * 32, p.u);
                }
            }
            tc_fence_before();                               // (the next piece's first P says that O has been read)
            if (!direct) a.st.ml[srow] = make_float4(m, l, lr, 0.f);
            else if (live) a.out.lse[orow] = end.lse;
        }
        if (lane == 0) bulk_wait();
    }
    __syncthreads();
    if (threadIdx.x == 0 && sh.abort_flag && a.stats) a.stats->status = KVM_E_DEVICE_TIMEOUT;
    if (warp == NSOFT + 1) {
        tc_fence_after();
        tmem_dealloc(tmem_base, 512);
    }
}

// Query rows as a tensor [units, N, R, D] with boxes of [1, bx, gx, 64 channels].
bool make_rows_map(CUtensorMap* map, const Queries& q, int units, int D, int gx, int bx) {
    EncodeTiledFn fn = encode_fn();
    if (!fn) return false;
    const cuuint64_t pitch = (cuuint64_t)D * 2;
    cuuint64_t dims[4] = {(cuuint64_t)D, (cuuint64_t)q.R, (cuuint64_t)q.N, (cuuint64_t)units};
    cuuint64_t strides[3] = {pitch, pitch * (cuuint64_t)(q.N > 1 ? q.sn : q.R), pitch * (cuuint64_t)q.su};
    cuuint32_t box[4] = {64, (cuuint32_t)gx, (cuuint32_t)bx, 1};
    cuuint32_t estr[4] = {1, 1, 1, 1};
    return fn(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, const_cast<void*>(q.q), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
              CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_128B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}
// The states' sums [rows, D] fp32, boxes of [32 rows, 32 channels].
bool make_states_map(CUtensorMap* map, float* o, size_t rows, int D) {
    EncodeTiledFn fn = encode_fn();
    if (!fn) return false;
    cuuint64_t dims[2] = {(cuuint64_t)D, (cuuint64_t)rows};
    cuuint64_t strides[1] = {(cuuint64_t)D * 4};
    cuuint32_t box[2] = {32, 32};
    cuuint32_t estr[2] = {1, 1};
    return fn(map, CU_TENSOR_MAP_DATA_TYPE_FLOAT32, 2, o, dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
              CU_TENSOR_MAP_L2_PROMOTION_NONE, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int KCH, bool COMPACT>
cudaError_t launch_t(const TcPlan& plan, const CUtensorMap& mq, const CUtensorMap& mk, const CUtensorMap& mv, const CUtensorMap& mo,
                     const CUtensorMap& ms, const Args& a, cudaStream_t st) {
    constexpr size_t smem = 1024 + (size_t)(2 + 2 * NST) * KCH * CHUNK_BYTES + NSOFT * 4096 + sizeof(Shared);
    static std::mutex mu;
    static bool ready[KVM_MAX_DEVICES] = {};
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev < 0 || dev >= KVM_MAX_DEVICES) return cudaErrorInvalidDevice;
    {
        std::lock_guard<std::mutex> lock(mu);
        if (!ready[dev]) {
            if ((e = cudaFuncSetAttribute(rows_tc_kernel<KCH, COMPACT>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem)) != cudaSuccess) return e;
            ready[dev] = true;
        }
    }
    return launch_dependent(rows_tc_kernel<KCH, COMPACT>, dim3((unsigned)plan.grid), dim3(NTHREADS), smem, st, mq, mk, mv, mo, ms, a);
}

}  // namespace

// Steps of a CTA that cut items cost in all.  (128 heads x 1024 queries x 1075-1433 keys, 512 items of up to 12 steps: cut 126 us, whole 109.)
constexpr int WHOLE = 12;

// (Sizes only: the workspace is asked for without a device.  148 SMs, one CTA each.)
TcPlan tc_plan(int units, int R, int N, int rows, bool direct) {
    TcPlan p;
    p.gx = R < TILE ? R : TILE;
    p.bx = N == 1 ? 1 : TILE / p.gx;
    p.per_block = R > TILE ? (R + TILE - 1) / TILE : 0;
    p.tiles = p.per_block ? N * p.per_block : (N + p.bx - 1) / p.bx;
    p.items = (p.tiles + 1) / 2;
    const long long tiles = (rows + TILE - 1) / TILE, all = (long long)units * p.items, steps = all * tiles;
    p.grid = steps < SMS ? (int)steps : SMS;
    // Items stay whole where the fullest CTA then has at most WHOLE steps more than an equal share: what the states of cut items and their
    // joining cost.
    p.whole = (all + p.grid - 1) / p.grid * tiles * p.grid <= steps + WHOLE * p.grid;
    // (148 units x 256 rows, us without / with, by steps: 1 10.2 / 10.0, 4 16.4 / 17.2, 8 25.2 / 27.2, 24 60.8 / 64.7, the instructions being at hand
    // from the last launch; between other kernels, 6 steps, 66.6 / 64.1 and 3 steps 37.1 / 35.2.)
    p.compact = steps <= 12 * p.grid;
    // A single tile per unit: both softmax groups on it, each with a state of its own (which are joined, so nothing goes straight to the output).
    // (us with / without, steps per CTA: 64 units x 20 rows x 14336 keys 48 steps 86.7 / 93.2; 64 x 128 x 3584 12 steps 38.6 / 41.1; 32 x 32 x 3584
    // 6.3 steps 25.8 / 27.3; 2 x 64 x 28672 3 steps 24.4 / 21.4; beside own rows, 8 x 32 x 14336 6 steps 35.4 / 34.4.  all: what the states take.)
    p.alt = p.tiles == 1 && !p.whole && all <= 4 * SMS && steps >= (direct ? 6 : 8) * p.grid;
    p.direct = direct && !p.alt;
    p.slot_rows = p.tiles > 1 || p.alt ? 2 * TILE : TILE;
    p.slots = 2ll * p.grid + (p.direct ? 0 : all);
    return p;
}

cudaError_t launch_rows_tc(const Shape& s, const TcPlan& plan, int units, const Queries& q, const Keys& k, const Beside& own, const States& states,
                           const Output& out, kvm_stats* stats, cudaStream_t st) {
    CUtensorMap mq, mk, mv, mo, ms;
    if (!make_rows_map(&mq, q, units, s.D, plan.gx, plan.bx) || !make_map(&mk, k.K, units, k.rows, s.D) || !make_map(&mv, k.V, units, k.rows, s.D) ||
        !make_states_map(&ms, states.o, (size_t)plan.slots * plan.slot_rows, s.D))
        return cudaErrorNotSupported;
    mo = mq;                                    // (not used where nothing goes to the output)
    if (plan.direct && !make_map(&mo, out.O, units, q.R, s.D, 32)) return cudaErrorNotSupported;
    Args a;
    a.out = out; a.st = states; a.len = k.len; a.rows = k.rows; a.units = units; a.tiles = plan.tiles; a.whole = plan.whole; a.alt = plan.alt; a.direct = plan.direct;
    a.gx = plan.gx; a.bx = plan.bx; a.per_block = plan.per_block; a.m = q.rows(); a.scale2 = s.scale * LOG2E; a.stats = stats; a.own = own;
    auto fn = s.D == 128 ? (plan.compact ? launch_t<2, true> : launch_t<2, false>) : (plan.compact ? launch_t<1, true> : launch_t<1, false>);
    return fn(plan, mq, mk, mv, mo, ms, a, st);
}

}  // namespace serve
}  // namespace kvm
