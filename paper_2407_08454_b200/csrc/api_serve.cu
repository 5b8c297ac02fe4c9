// C ABI of the serving operators: paged append, shared-prefix decode attention, cross attention.  Host-side validation, workspace
// carving, dispatch, in the manner of api.cu: everything is checked before anything is enqueued, nothing is allocated or synchronised.
#include <math.h>

#include "serve.cuh"

namespace kvm {
namespace serve {
namespace {

inline bool misaligned(const void* p, size_t a = 16) { return ((uintptr_t)p & (a - 1)) != 0; }
inline size_t align_up(size_t x) { return (x + 255) / 256 * 256; }

// (These operators take a cache of any length: of the parameters only the heads, the types and the scale matter.)
int derive(const kvm_params* p, Shape& s) {
    if (!p) return KVM_E_NULL;
    if (p->dtype != KVM_BF16 && p->dtype != KVM_F32) return KVM_E_DTYPE;
    if (p->batch < 1 || p->n_q_heads < 1 || p->n_kv_heads < 1 || p->n_q_heads % p->n_kv_heads != 0) return KVM_E_SHAPE;
    if (p->head_dim != 64 && p->head_dim != 128) return KVM_E_SHAPE;
    if ((long long)p->batch * p->n_q_heads > 65535) return KVM_E_SHAPE;
    if (!isfinite(p->softmax_scale)) return KVM_E_PARAM;
    s.B = p->batch; s.Hq = p->n_q_heads; s.Hkv = p->n_kv_heads; s.G = s.Hq / s.Hkv;
    s.D = p->head_dim; s.U = s.B * s.Hkv; s.dtype = p->dtype;
    s.scale = p->softmax_scale > 0.f ? p->softmax_scale : 1.0f / sqrtf((float)s.D);
    return KVM_OK;
}

// sizes_only: as a workspace query needs them (the pointers may be missing).
int derive(const kvm_pages* c, bool sizes_only, Pages& o) {
    if (c->page_rows < 16 || c->page_rows > 4096 || (c->page_rows & (c->page_rows - 1))) return KVM_E_SHAPE;
    if (c->n_pages < 1 || c->max_pages < 1 || (long long)c->max_pages * c->page_rows > KVM_MAX_ROWS) return KVM_E_SHAPE;
    if ((long long)c->n_pages * c->page_rows >= (1ll << 31)) return KVM_E_SHAPE;
    if (c->reserved != 0) return KVM_E_PARAM;
    if (!sizes_only) {
        if (!c->K || !c->V || !c->table || !c->len) return KVM_E_NULL;
        if (misaligned(c->K) || misaligned(c->V) || misaligned(c->table, 4) || misaligned(c->len, 4)) return KVM_E_ALIGN;
    }
    o.K = c->K; o.V = c->V; o.table = c->table; o.len = c->len;
    o.n_pages = c->n_pages; o.max_pages = c->max_pages;
    o.shift = 0;
    while ((1 << o.shift) < c->page_rows) ++o.shift;
    return KVM_OK;
}

// (Blocks of 16 rows are counted in 32 bits.)
bool too_many(const Shape& s, int pre_rows, const Pages* c) {
    return (long long)s.B * s.Hq * ((c ? c->room() / 16 : 0) + (pre_rows + 15) / 16) >= (1ll << 31);
}

struct Carver {
    char* base;
    size_t off = 0;
    void* take(size_t n) {
        void* r = base + off;
        off += align_up(n);
        return r;
    }
};

// States of a fixed number of pieces per item (plan.mt rows each).
States f32_states(const F32Plan& plan, int units, int D, Carver& c) {
    States s = {};
    const size_t slots = (size_t)units * plan.items * plan.pieces;
    s.rows = s.tile = plan.mt;
    s.items = plan.items;
    s.count = plan.pieces;
    s.stride = 1;
    s.o = (float*)c.take(slots * plan.mt * D * sizeof(float));
    s.ml = (float4*)c.take(slots * plan.mt * sizeof(float4));
    return s;
}

// States of the tensor-core kernel's pieces.
States tc_states(const TcPlan& plan, int units, int D, int R, Carver& c) {
    States s = {};
    s.rows = plan.slot_rows;
    s.items = plan.items;
    s.stride = 2;
    s.tile = plan.gx * plan.bx;
    s.R = plan.per_block ? R : 0;
    s.two = 1;
    s.tile_room = 128;
    s.halves = plan.alt;
    s.o = (float*)c.take((size_t)plan.slots * plan.slot_rows * D * sizeof(float));
    s.ml = (float4*)c.take((size_t)plan.slots * plan.slot_rows * sizeof(float4));
    s.pieces = (int4*)c.take((size_t)units * plan.items * sizeof(int4));
    return s;
}

// States of the parts of the paged kernel's items.
States paged_states(const PagedPlan& plan, int D, Carver& c) {
    States s = {};
    s.rows = s.tile = plan.slot_rows;
    s.items = plan.hg;
    s.stride = 1;
    s.o = (float*)c.take((size_t)plan.slots * plan.slot_rows * D * sizeof(float));
    s.ml = (float4*)c.take((size_t)plan.slots * plan.slot_rows * sizeof(float4));
    s.pieces = (int4*)c.take((size_t)plan.items * sizeof(int4));
    return s;
}

constexpr long long FOLD_BYTES = 32ll << 20;

// How a call of the decode attention is dealt, and what it needs of the workspace.
struct SharedWork {
    bool pre, own, fold;                        // fold: the prefix's rows go with each sequence's own
    TcPlan pre_tc;
    PagedPlan own_paged;
    F32Plan pre_plan, own_plan;
    States pre_states, own_states;
    size_t bytes;
};
SharedWork plan_shared(const Shape& s, int pre_rows, const Pages* own, void* ws) {
    SharedWork w = {};
    Carver c{(char*)ws};
    w.pre = pre_rows > 0;
    w.own = own != nullptr;
    if (w.pre && s.dtype == KVM_BF16) {
        // A kernel for the prefix, and joining its states, costs about 10 us that reading a short one again for every sequence, through L2,
        // does not.
        const long long groups = (long long)s.B * ((s.G + 7) / 8) - 1;
        w.fold = groups * s.Hkv * pre_rows * 4 * s.D <= FOLD_BYTES;
        w.pre = !w.fold;
    }
    if (w.fold) {
        w.own_paged = paged_plan(s, pre_rows + 16 + (own ? own->room() : 0), false);
        w.own_states = paged_states(w.own_paged, s.D, c);
        w.bytes = c.off + 256;
        return w;
    }
    if (w.pre && s.dtype == KVM_BF16) {
        w.pre_tc = tc_plan(s.Hkv, s.G, s.B, pre_rows, false);
        w.pre_states = tc_states(w.pre_tc, s.Hkv, s.D, s.G, c);
    } else if (w.pre) {
        w.pre_plan = f32_plan(s.Hkv, s.B * s.G, pre_rows, s.D);
        if (w.own || w.pre_plan.pieces > 1) w.pre_states = f32_states(w.pre_plan, s.Hkv, s.D, c);
    }
    if (w.own && s.dtype == KVM_BF16) {
        w.own_paged = paged_plan(s, own->room(), w.pre);
        w.own_states = paged_states(w.own_paged, s.D, c);
    } else if (w.own) {
        w.own_plan = f32_plan(s.U, s.G, own->room(), s.D);
        if (w.pre || w.own_plan.pieces > 1) w.own_states = f32_states(w.own_plan, s.U, s.D, c);
    }
    w.bytes = c.off + 256;
    return w;
}

struct CrossWork {
    TcPlan tc;
    F32Plan plan;
    States states;
    size_t bytes;
};
CrossWork plan_cross(const Shape& s, int n_q, int rows, void* ws) {
    CrossWork w = {};
    Carver c{(char*)ws};
    if (s.dtype == KVM_BF16) {
        w.tc = tc_plan(s.U, s.G * n_q, 1, rows, true);
        w.states = tc_states(w.tc, s.U, s.D, s.G * n_q, c);
        w.bytes = c.off + 256;
        return w;
    }
    w.plan = f32_plan(s.U, s.G * n_q, rows, s.D);
    if (w.plan.pieces > 1) w.states = f32_states(w.plan, s.U, s.D, c);
    w.bytes = c.off + 256;
    return w;
}

int check_cross(const kvm_params* p, int n_q, int rows, Shape& s) {
    const int rc = derive(p, s);
    if (rc != KVM_OK) return rc;
    if (n_q < 1 || n_q > KVM_MAX_SEQ || rows < 1 || rows > KVM_MAX_ROWS) return KVM_E_SHAPE;
    if ((long long)s.B * s.Hq * n_q >= (1ll << 30)) return KVM_E_SHAPE;
    return KVM_OK;
}

}  // namespace
}  // namespace serve
}  // namespace kvm

using namespace kvm;
using namespace kvm::serve;

extern "C" {

int kvm_rope_turns(int32_t head_dim, double base, uint64_t* turns) {
    if (!turns) return KVM_E_NULL;
    if (head_dim != 64 && head_dim != 128) return KVM_E_SHAPE;
    if (!isfinite(base) || !(base > 1.0)) return KVM_E_PARAM;
    // (a double holds a frequency to 2^-53 of itself: positions up to 2^27 lose less than 2^-28 of a turn)
    for (int i = 0; i < head_dim / 2; ++i)
        turns[i] = (uint64_t)ldexp(pow(base, -2.0 * i / head_dim) / 6.283185307179586476925, 64);
    return KVM_OK;
}

int kvm_paged_append(const kvm_params* p, const kvm_pages* c, int32_t* len_out, int32_t n_new, const int32_t* new_len,
                     const int32_t* pos, const uint64_t* turns, int32_t rope_layout, const void* q, const void* k,
                     const void* v, const int64_t* strides, void* q_out, kvm_stats* stats, void* cuda_stream) {
    Shape s;
    Pages pg;
    int rc = derive(p, s);
    if (rc != KVM_OK) return rc;
    if (!c || !len_out || !k || !v || (turns && !pos) || !q != !q_out) return KVM_E_NULL;
    if ((rc = derive(c, false, pg)) != KVM_OK) return rc;
    if (n_new < 1 || n_new > KVM_MAX_ROWS) return KVM_E_SHAPE;
    if (rope_layout != KVM_ROPE_HALVES && rope_layout != KVM_ROPE_NEIGHBOURS) return KVM_E_PARAM;
    if (misaligned(k) || misaligned(v) || (q && (misaligned(q) || misaligned(q_out))) || (turns && misaligned(turns, 8)) ||
        misaligned(len_out, 4) || misaligned(stats, 4) || (new_len && misaligned(new_len, 4)) || (pos && misaligned(pos, 4)))
        return KVM_E_ALIGN;
    int64_t st[9];
    const int64_t vec = s.dtype == KVM_BF16 ? 8 : 4;
    for (int i = 0; i < 3; ++i) {
        const int64_t heads = i == 0 ? s.Hq : s.Hkv;
        st[3 * i] = strides ? strides[3 * i] : heads * n_new * s.D;
        st[3 * i + 1] = strides ? strides[3 * i + 1] : (int64_t)n_new * s.D;
        st[3 * i + 2] = strides ? strides[3 * i + 2] : s.D;
        if (i == 0 && !q) continue;
        for (int j = 0; j < 3; ++j) {
            if (st[3 * i + j] < 0) return KVM_E_PARAM;
            if (st[3 * i + j] % vec != 0) return KVM_E_ALIGN;
        }
    }
    return launch_append(s, pg, len_out, n_new, new_len, pos, turns, rope_layout == KVM_ROPE_NEIGHBOURS, q, k, v, st, q_out, stats,
                         (cudaStream_t)cuda_stream) == cudaSuccess
               ? KVM_OK
               : KVM_E_CUDA;
}

int kvm_shared_workspace_bytes(const kvm_params* p, int32_t pre_rows, const kvm_pages* own, size_t* bytes) {
    Shape s;
    Pages pg;
    int rc = derive(p, s);
    if (rc != KVM_OK) return rc;
    if (!bytes) return KVM_E_NULL;
    if (pre_rows < 0 || pre_rows > KVM_MAX_ROWS || (pre_rows == 0 && !own)) return KVM_E_SHAPE;
    if (own && (rc = derive(own, true, pg)) != KVM_OK) return rc;
    if (too_many(s, pre_rows, own ? &pg : nullptr)) return KVM_E_SHAPE;
    *bytes = plan_shared(s, pre_rows, own ? &pg : nullptr, nullptr).bytes;
    return KVM_OK;
}

int kvm_shared_attend(const kvm_params* p, const void* q, const void* K_pre, const void* V_pre, int32_t pre_rows,
                      const int32_t* pre_len, const kvm_pages* own, void* out, kvm_stats* stats, void* ws, size_t ws_bytes,
                      void* cuda_stream) {
    Shape s;
    Pages pg = {};
    int rc = derive(p, s);
    if (rc != KVM_OK) return rc;
    if (!q || !out || !K_pre != !V_pre || (!K_pre && !own)) return KVM_E_NULL;
    if (K_pre ? (pre_rows < 1 || pre_rows > KVM_MAX_ROWS) : pre_rows != 0) return KVM_E_SHAPE;
    if (own && (rc = derive(own, false, pg)) != KVM_OK) return rc;
    if (too_many(s, pre_rows, own ? &pg : nullptr)) return KVM_E_SHAPE;
    if (misaligned(q) || misaligned(out) || misaligned(stats, 4) || (K_pre && (misaligned(K_pre) || misaligned(V_pre))) || (pre_len && misaligned(pre_len, 4)))
        return KVM_E_ALIGN;
    const SharedWork w = plan_shared(s, pre_rows, own ? &pg : nullptr, ws);
    if (!ws || ws_bytes < w.bytes) return KVM_E_WORKSPACE;
    if (misaligned(ws)) return KVM_E_ALIGN;
    cudaStream_t st = (cudaStream_t)cuda_stream;
    const Output o = {out, nullptr, nullptr, nullptr};
    const Queries pre_q = {q, s.G, s.Hq, s.G, s.B}, own_q = {q, s.G, 0, s.G, 1};
    const Keys pre_k = {K_pre, V_pre, pre_len, pre_rows, nullptr, 0, 0, 0};
    const Keys own_k = {pg.K, pg.V, pg.len, own ? pg.room() : 0, pg.table, pg.n_pages, own ? pg.shift : 4, pg.max_pages};
    if (w.fold) {
        const Fold f = {K_pre, V_pre, pre_len, s.Hkv, pre_rows};
        if (launch_rows_paged(s, w.own_paged, q, own_k, f, Beside{}, w.own_states, out, stats, st) != cudaSuccess) return KVM_E_CUDA;
        if (w.own_paged.alone) return KVM_OK;
        return launch_join(s, s.U, s.G, &w.own_states, nullptr, nullptr, 1, w.own_paged.grid * 4 / w.own_paged.items, o, st) == cudaSuccess ? KVM_OK : KVM_E_CUDA;
    }
    if (s.dtype == KVM_BF16) {
        const Beside pre = {pre_len, w.pre ? s.Hkv : 0, pre_rows, w.pre_tc.items, 128}, mine = {pg.len, w.own ? s.U : 0, own_k.rows, w.own_paged.hg, 16};
        if (w.pre && launch_rows_tc(s, w.pre_tc, s.Hkv, pre_q, pre_k, mine, w.pre_states, o, stats, st) != cudaSuccess) return KVM_E_CUDA;
        if (w.own && launch_rows_paged(s, w.own_paged, q, own_k, Fold{}, pre, w.own_states, w.pre ? nullptr : out, stats, st) != cudaSuccess) return KVM_E_CUDA;
    } else {
        if (w.pre && launch_rows_f32(s, w.pre_plan, s.Hkv, pre_q, pre_k, w.pre_states, o, stats, st) != cudaSuccess) return KVM_E_CUDA;
        if (w.own && launch_rows_f32(s, w.own_plan, s.U, own_q, own_k, w.own_states, o, stats, st) != cudaSuccess) return KVM_E_CUDA;
    }
    if ((!w.pre_states.o && !w.own_states.o) || w.own_paged.alone) return KVM_OK;
    const int about = s.dtype == KVM_BF16 ? (w.own ? w.own_paged.grid * 4 / w.own_paged.items : 0) + (w.pre ? w.pre_tc.grid / (s.Hkv * w.pre_tc.items) : 0)
                                          : w.own_plan.pieces + w.pre_plan.pieces;
    return launch_join(s, s.U, s.G, w.own ? &w.own_states : nullptr, w.pre ? &w.pre_states : nullptr, pre_len, !w.pre, about, o, st) == cudaSuccess
               ? KVM_OK
               : KVM_E_CUDA;
}

int kvm_cross_workspace_bytes(const kvm_params* p, int32_t n_q, int32_t rows, size_t* bytes) {
    Shape s;
    const int rc = check_cross(p, n_q, rows, s);
    if (rc != KVM_OK) return rc;
    if (!bytes) return KVM_E_NULL;
    *bytes = plan_cross(s, n_q, rows, nullptr).bytes;
    return KVM_OK;
}

int kvm_cross_attend(const kvm_params* p, const void* Q, int32_t n_q, const void* K, const void* V, int32_t rows,
                     const int32_t* len, const void* O_in, const float* lse_in, void* O, float* lse, kvm_stats* stats, void* ws,
                     size_t ws_bytes, void* cuda_stream) {
    Shape s;
    const int rc = check_cross(p, n_q, rows, s);
    if (rc != KVM_OK) return rc;
    if (!Q || !K || !V || !O || !lse || !O_in != !lse_in) return KVM_E_NULL;
    if (misaligned(Q) || misaligned(K) || misaligned(V) || misaligned(O) || misaligned(lse, 4) || misaligned(stats, 4) || (len && misaligned(len, 4)) ||
        (O_in && (misaligned(O_in) || misaligned(lse_in, 4))))
        return KVM_E_ALIGN;
    const CrossWork w = plan_cross(s, n_q, rows, ws);
    if (!ws || ws_bytes < w.bytes) return KVM_E_WORKSPACE;
    if (misaligned(ws)) return KVM_E_ALIGN;
    cudaStream_t st = (cudaStream_t)cuda_stream;
    const int m = s.G * n_q;
    const Queries qs = {Q, m, 0, m, 1};
    const Keys ks = {K, V, len, rows, nullptr, 0, 0, 0};
    const Output o = {O, lse, O_in, lse_in};
    if (s.dtype == KVM_BF16) {
        if (launch_rows_tc(s, w.tc, s.U, qs, ks, Beside{}, w.states, o, stats, st) != cudaSuccess) return KVM_E_CUDA;
        if (w.tc.whole) return KVM_OK;
        return launch_join_items(s, s.U, m, w.states, len, o, st) == cudaSuccess ? KVM_OK : KVM_E_CUDA;
    }
    if (launch_rows_f32(s, w.plan, s.U, qs, ks, w.states, o, stats, st) != cudaSuccess) return KVM_E_CUDA;
    if (!w.states.o) return KVM_OK;
    return launch_join(s, s.U, m, &w.states, nullptr, nullptr, 0, w.plan.pieces, o, st) == cudaSuccess ? KVM_OK : KVM_E_CUDA;
}

}  // extern "C"
