"""The serving operators around the compression, as measurable cases.

Three operators:

  append  a step's new keys and values go behind the rows of a paged cache, keys and queries rotated by their positions on the
          way (kvm_paged_append)
  shared  one decode step for a batch whose sequences share a prefix (a prompt that was prefilled and compressed once) and
          have rows of their own in pages (kvm_shared_attend); either part may be missing
  cross   queries over a cache of another length, no mask but the units' lengths, output and log-sum-exp, on request joined
          with the attention of the same queries over other keys (kvm_cross_attend)

`own` false: elementary torch operations in 32 bits.  `own` true: the package's entry points.
"""
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
BASE = 10000.0                     # of the rotation's frequencies
LOGIT_STD = 4.0                    # of q.k / sqrt(D), as the queries are scaled


def _append(batch, n_q_heads, n_kv_heads, tokens, head_dim, page_rows=16, held=512, dtype="bf16", interleaved=False,
            fused=True, ragged=False, **name):
    """`held`: most rows a unit holds before the call; `fused`: q, k, v are views of one projection's output
    [batch, tokens, heads, head_dim]; `ragged`: units take different numbers of the new rows."""
    return {**name, "op": "append", "batch": batch, "n_q_heads": n_q_heads, "n_kv_heads": n_kv_heads, "tokens": tokens,
            "head_dim": head_dim, "page_rows": page_rows, "held": held, "dtype": dtype, "interleaved": interleaved,
            "fused": fused, "ragged": ragged}


def _shared(batch, n_q_heads, n_kv_heads, prefix, held, head_dim, page_rows=16, dtype="bf16", **name):
    """`prefix`: rows the shared prefix has room for (0: none), `held`: most rows of a sequence's own (0: none)."""
    return {**name, "op": "shared", "batch": batch, "n_q_heads": n_q_heads, "n_kv_heads": n_kv_heads, "prefix": prefix,
            "held": held, "head_dim": head_dim, "page_rows": page_rows, "dtype": dtype}


def _cross(batch, n_q_heads, n_kv_heads, n_q, rows, head_dim, dtype="bf16", join=False, **name):
    """`join`: the attention of the same queries over other keys is joined in."""
    return {**name, "op": "cross", "batch": batch, "n_q_heads": n_q_heads, "n_kv_heads": n_kv_heads, "n_q": n_q,
            "rows": rows, "head_dim": head_dim, "dtype": dtype, "join": join}


def listed():
    return [
        # a decode step's append for a serving batch with grouped queries: launches and dependent loads
        _append(64, 32, 8, 1, 128, name="append-decode-gqa"),
        # a prompt chunk of a batch, straight from the projection's output: bandwidth
        _append(8, 32, 8, 2048, 128, page_rows=64, held=4096, name="append-chunk-gqa"),
        # fp32, neighbouring channels as pairs, units that take different numbers of rows
        _append(3, 8, 4, 389, 64, page_rows=32, dtype="f32", interleaved=True, fused=False, ragged=True,
                name="append-f32-ragged"),
        # the smallest decode step: one Llama2-7B-shaped sequence with a short paged cache and no prefix: latency
        _shared(1, 32, 32, 0, 512, 128, name="paged-7b-latency"),
        # sixteen sequences behind one Llama2-7B-shaped compressed prompt (4096 tokens at the 50 % budget)
        _shared(16, 32, 32, 2048, 389, 128, name="shared-7b-2k"),
        # a serving batch behind one Mistral-7B-shaped compressed prompt (32k tokens at the 50 % budget)
        _shared(64, 32, 8, 16384, 1024, 128, page_rows=64, name="shared-gqa-16k"),
        # long caches of sequences that share nothing: bandwidth
        _shared(16, 32, 8, 0, 16384, 128, page_rows=64, name="paged-gqa-16k"),
        # fp32, head dimension 64, odd sizes
        _shared(5, 8, 4, 999, 461, 64, dtype="f32", name="shared-f32-ragged"),
        # a few drafted tokens per sequence over compressed 32k-token caches: bandwidth
        _cross(8, 32, 8, 5, 16384, 128, name="cross-draft-gqa"),
        # the next chunk of a prompt over its compressed past, joined with the chunk's own causal attention: the largest
        _cross(1, 32, 8, 4096, 16384, 128, join=True, name="cross-chunk-gqa"),
        # decoder queries over four encoded sources of up to 1433 states
        _cross(4, 32, 32, 1024, 1433, 128, name="cross-7b-batch"),
        # fp32, head dimension 64, odd sizes
        _cross(2, 8, 4, 389, 777, 64, dtype="f32", join=True, name="cross-f32-ragged"),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, round(math.exp(rng.uniform(math.log(lo), math.log(hi))))))


def draw(rng):
    op = rng.choices(["append", "shared", "cross"], [3, 5, 4])[0]
    dtype = "f32" if rng.random() < 0.25 else "bf16"
    wide = 2 if dtype == "f32" else 1
    D, page_rows = rng.choice([64, 128, 128]), rng.choice([16, 16, 32, 64, 128])
    while True:
        n_kv_heads, group = _log_int(rng, 1, 40), rng.choice([1, 1, 2, 4, 8])
        if n_kv_heads * group > 64:
            continue
        heads, batch = n_kv_heads * group, _log_int(rng, 1, 64)
        if op == "append":
            tokens = rng.choice([1, 1, _log_int(rng, 1, 4096)])
            held = _log_int(rng, 1, 4096)
            if batch * tokens * (heads + 2 * n_kv_heads) * D * wide <= 8 * 2048 * 48 * 128 and \
                    batch * n_kv_heads * (held + tokens) * D * wide <= 8 * 8 * 6144 * 128:
                return _append(batch, heads, n_kv_heads, tokens, D, page_rows, held, dtype, rng.random() < 0.3,
                               rng.random() < 0.7, rng.random() < 0.5)
        if op == "shared":
            prefix = rng.choice([0, _log_int(rng, 1, 32768), _log_int(rng, 64, 32768)])
            held = rng.choice([0, _log_int(rng, 1, 16384), _log_int(rng, 1, 2048)])
            cells = n_kv_heads * (prefix + batch * held) * D * wide
            pairs = batch * heads * (prefix + held) * D * (16 if dtype == "f32" else 1)
            if prefix + held and cells <= 16 * 8 * 16384 * 128 and pairs <= 64 * 32 * 17408 * 128:
                return _shared(batch, heads, n_kv_heads, prefix, held, D, page_rows, dtype)
        if op == "cross":
            batch, n_q, rows = min(batch, 8), _log_int(rng, 1, 4096), _log_int(rng, 1, 32768)
            pairs = batch * heads * n_q * rows * D * (16 if dtype == "f32" else 1)
            if batch * heads * n_q <= 1 << 18 and batch * n_kv_heads * rows * D * wide <= 8 * 8 * 16384 * 128 and \
                    pairs <= 32 * 4096 * 16384 * 128:
                return _cross(batch, heads, n_kv_heads, n_q, rows, D, dtype, rng.random() < 0.4)


# ------------------------------------------------------------------ inputs
def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _randn(g, *shape):
    return torch.randn(shape, generator=g, device="cuda")


def _scales(g, n_kv_heads, D):
    """Channels of unequal scale with two outliers per head, as keys have them."""
    s = torch.exp(0.5 * _randn(g, n_kv_heads, 1, D))
    out = torch.rand((n_kv_heads, 1, D), generator=g, device="cuda").topk(2).indices
    gain = torch.ones_like(s).scatter_(-1, out, 10.0)
    return s * gain, gain


def _queries(g, case, tokens, sk, gain):
    """[batch, heads, tokens, D] on the same outlier channels, scaled so that the logits have a standard deviation."""
    B, Hq, Hkv, D = (case[k] for k in ("batch", "n_q_heads", "n_kv_heads", "head_dim"))
    G = Hq // Hkv
    sq = torch.exp(0.5 * _randn(g, Hq, 1, D)) * gain.repeat_interleave(G, 0)
    sq = sq * (LOGIT_STD * math.sqrt(D) / (sq * sk.repeat_interleave(G, 0)).square().sum(-1, keepdim=True).sqrt())
    return (_randn(g, B, Hq, tokens, D) * sq).to(DTYPES[case["dtype"]])


def _pool(g, case, rows, sk):
    """A paged cache: `rows` rows of room per unit, pages dealt in random order, table entries past a unit's pages -1.
    Lengths lie in the upper half of `held`."""
    B, Hkv, D, R = (case[k] for k in ("batch", "n_kv_heads", "head_dim", "page_rows"))
    dt, U, P = DTYPES[case["dtype"]], B * Hkv, max(1, -(-rows // R))
    ids = torch.randperm(U * P, generator=g, device="cuda").to(torch.int32).view(U, P)
    K, V = (torch.empty((U * P, R, D), dtype=dt, device="cuda") for _ in range(2))
    for h in range(Hkv):                                   # (a head's pages at a time: its keys' scales)
        mine = ids.view(B, Hkv, P)[:, h].reshape(-1).long()
        K[mine] = (_randn(g, B * P, R, D) * sk[h]).to(dt)
        V[mine] = _randn(g, B * P, R, D).to(dt)
    held = case["held"]
    length = torch.randint(held // 2, held + 1, (B, Hkv), generator=g, device="cuda", dtype=torch.int32)
    new = rows - held
    used = (length.view(U, 1) + new + R - 1) // R
    table = torch.where(torch.arange(P, device="cuda") < used, ids, torch.full_like(ids, -1))
    return {"K": K, "V": V, "table": table.to(torch.int32).contiguous(), "len": length}


def prepare(case, seed):
    g, op, dt = _gen(seed), case["op"], DTYPES[case["dtype"]]
    B, Hq, Hkv, D = (case[k] for k in ("batch", "n_q_heads", "n_kv_heads", "head_dim"))
    sk, gain = _scales(g, Hkv, D)
    st = {"case": case}
    if op == "append":
        T = case["tokens"]
        q = _queries(g, case, T, sk, gain)
        k, v = (_randn(g, B, Hkv, T, D) * sk).to(dt), _randn(g, B, Hkv, T, D).to(dt)
        if case["fused"]:
            qkv = torch.cat([x.transpose(1, 2) for x in (q, k, v)], 2).contiguous()
            q, k, v = (x.transpose(1, 2) for x in qkv.split([Hq, Hkv, Hkv], 2))
        st.update(_pool(g, case, case["held"] + T, sk), q=q, k=k, v=v)
        st["pos"] = torch.randint(0, 131072, (B,), generator=g, device="cuda", dtype=torch.int32)
        st["new"] = (torch.randint(0, T + 1, (B, Hkv), generator=g, device="cuda", dtype=torch.int32)
                     if case["ragged"] else None)
        st["q_out"] = torch.empty((B, Hq, T, D), dtype=dt, device="cuda")
        st["len_out"] = torch.empty_like(st["len"])
    if op == "shared":
        P = case["prefix"]
        st["q"] = _queries(g, case, 1, sk, gain).squeeze(2).contiguous()
        if P:
            st["K_pre"] = (_randn(g, Hkv, P, D) * sk).to(dt)
            sets = torch.randint(1, 4, (Hkv, P, 1), generator=g, device="cuda")     # merged values carry their set's size
            st["V_pre"] = (_randn(g, Hkv, P, D) * sets).to(dt)
            st["pre_len"] = torch.randint((3 * P + 3) // 4, P + 1, (Hkv,), generator=g, device="cuda", dtype=torch.int32)
        if case["held"]:
            st["pages"] = _pool(g, case, case["held"], sk)
        st["out"] = torch.empty((B, Hq, D), dtype=dt, device="cuda")
    if op == "cross":
        n, R = case["n_q"], case["rows"]
        st["Q"] = _queries(g, case, n, sk, gain)
        st["K"], st["V"] = (_randn(g, B, Hkv, R, D) * sk).to(dt), _randn(g, B, Hkv, R, D).to(dt)
        st["len"] = torch.randint((3 * R + 3) // 4, R + 1, (B, Hkv), generator=g, device="cuda", dtype=torch.int32)
        st["O"] = torch.empty((B, Hq, n, D), dtype=dt, device="cuda")
        st["lse"] = torch.empty((B, Hq, n), dtype=torch.float32, device="cuda")
        if case["join"]:                                   # query i has seen i + 1 keys of its own chunk
            seen = torch.arange(1, n + 1, device="cuda", dtype=torch.float32)
            st["lse_in"] = (seen.log() + 0.5 * LOGIT_STD ** 2 + _randn(g, B, Hq, n)).contiguous()
            st["O_in"] = (_randn(g, B, Hq, n, D) / seen.sqrt().clamp(max=4.0).view(n, 1)).to(dt)
    if own:
        import paper_2407_08454_b200 as kvm
        st["kvm"] = kvm
        p = st["p"] = kvm.make_params(B, Hq, Hkv, 1, D, dt)
        if op == "append":
            st["turns"] = kvm.rope_turns(D, BASE)
            st["cache"] = kvm.make_pages(st["K"], st["V"], st["table"], st["len"])
        if op == "shared":
            c = st.get("pages")
            st["cache"] = kvm.make_pages(c["K"], c["V"], c["table"], c["len"]) if c else None
            st["ws"] = torch.empty(kvm.kvm_shared_workspace_bytes(p, case["prefix"], st["cache"]), dtype=torch.uint8, device="cuda")
        if op == "cross":
            st["ws"] = torch.empty(kvm.kvm_cross_workspace_bytes(p, case["n_q"], case["rows"]), dtype=torch.uint8, device="cuda")
    return st


# ------------------------------------------------------------------ plain forms
def _rotated(x, pos, interleaved):
    """x [batch, heads, tokens, D] rotated by its positions pos [batch, tokens]: angles in 64 bits, the rest in 32."""
    D = x.shape[-1]
    freq = BASE ** (-torch.arange(0, D, 2, device=x.device, dtype=torch.float64) / D)
    angle = pos.to(torch.float64)[:, None, :, None] * freq
    c, s = angle.cos().float(), angle.sin().float()
    y = x.float()
    a, b = (y[..., 0::2], y[..., 1::2]) if interleaved else (y[..., :D // 2], y[..., D // 2:])
    ra, rb = a * c - b * s, b * c + a * s
    return (torch.stack([ra, rb], -1).flatten(-2) if interleaved else torch.cat([ra, rb], -1)).to(x.dtype)


def _run_append(st):
    case, q, k, v = st["case"], st["q"], st["k"], st["v"]
    B, Hkv, T, D = k.shape
    R = case["page_rows"]
    t = torch.arange(T, device=k.device, dtype=torch.int32)
    pos = st["pos"][:, None] + t
    st["q_out"].copy_(_rotated(q, pos, case["interleaved"]))
    kr = _rotated(k, pos, case["interleaved"])
    new = torch.full_like(st["len"], T) if st["new"] is None else st["new"]
    row = st["len"][:, :, None] + t                                            # [B, Hkv, T]
    page = st["table"].view(B, Hkv, -1).gather(2, (row // R).clamp(max=st["table"].shape[1] - 1).long())
    at = page.long() * R + row % R
    if st["new"] is None:
        st["K"].view(-1, D)[at.view(-1)] = kr.reshape(-1, D)
        st["V"].view(-1, D)[at.view(-1)] = v.reshape(-1, D)
    else:                                                                      # rows that are not taken go nowhere
        keep = (t < new[:, :, None]).view(-1)
        at = at.view(-1)[keep]
        st["K"].view(-1, D)[at] = kr.reshape(-1, D)[keep]
        st["V"].view(-1, D)[at] = v.reshape(-1, D)[keep]
    torch.add(st["len"], new, out=st["len_out"])
    return {"q": st["q_out"], "K": st["K"], "V": st["V"], "len": st["len_out"]}


def _gathered(c, b0, b1, Hkv, real):
    """Rows of batch entries b0..b1 of a paged cache: K, V [b, Hkv, room, D] (zeros past the lengths) and which exist."""
    R, D = c["K"].shape[1:]
    table = c["table"].view(-1, Hkv, c["table"].shape[1])[b0:b1].clamp(min=0).long()
    room = table.shape[2] * R
    live = torch.arange(room, device=table.device) < c["len"][b0:b1, :, None]
    K, V = (c[x][table].reshape(b1 - b0, Hkv, room, D).to(real).masked_fill(~live[..., None], 0.0) for x in ("K", "V"))
    return K, V, live


def _run_shared(st, real=torch.float32):
    case, q = st["case"], st["q"]
    B, Hq, Hkv, D = (case[k] for k in ("batch", "n_q_heads", "n_kv_heads", "head_dim"))
    G, P, c = Hq // Hkv, case["prefix"], st.get("pages")
    scale = 1.0 / math.sqrt(D)
    room = c["table"].shape[1] * case["page_rows"] if c else 0
    step = max(1, min(B, (1 << 28) // max(1, Hkv * room * D, Hq * P)))
    if P:
        live = torch.arange(P, device=q.device) < st["pre_len"][:, None]
        Kp, Vp = (st[x].to(real).masked_fill(~live[..., None], 0.0) for x in ("K_pre", "V_pre"))
    outs = []
    for b0 in range(0, B, step):
        b1 = min(B, b0 + step)
        qs = q[b0:b1].to(real).view(b1 - b0, Hkv, G, D) * scale
        logits = []
        if P:
            x = torch.matmul(qs.transpose(0, 1).reshape(Hkv, -1, D), Kp.transpose(1, 2)).view(Hkv, b1 - b0, G, P).transpose(0, 1)
            logits.append(x.masked_fill(~live[None, :, None], -math.inf))
        if c:
            Ko, Vo, mine = _gathered(c, b0, b1, Hkv, real)
            logits.append(torch.matmul(qs, Ko.transpose(2, 3)).masked_fill(~mine[:, :, None], -math.inf))
        x = torch.cat(logits, -1)
        m = x.amax(-1, keepdim=True)
        w = torch.exp(x - m.masked_fill(m == -math.inf, 0.0))
        total = w.sum(-1, keepdim=True)
        o = torch.zeros((b1 - b0, Hkv, G, D), dtype=real, device=q.device)
        if P:
            wp = w[..., :P].transpose(0, 1).reshape(Hkv, -1, P)
            o = o + torch.matmul(wp, Vp).view(Hkv, b1 - b0, G, D).transpose(0, 1)
        if c:
            o = o + torch.matmul(w[..., P:], Vo)
        outs.append((o / total.masked_fill(total == 0.0, 1.0)).view(b1 - b0, Hq, D))
    return torch.cat(outs)


def _run_cross(st, O, lse):
    case, Q = st["case"], st["Q"]
    B, Hq, Hkv, n, R, D = (case[k] for k in ("batch", "n_q_heads", "n_kv_heads", "n_q", "rows", "head_dim"))
    G, U = Hq // Hkv, B * Hkv
    real = lse.dtype
    Qu, Ku, Vu = Q.view(U, G * n, D), st["K"].view(U, R, D), st["V"].view(U, R, D)
    live = torch.arange(R, device=Q.device) < st["len"].view(U, 1)
    Ou, lu = O.view(U, G * n, D), lse.view(U, G * n)
    units = max(1, min(U, (1 << 28) // (G * n * R)))
    rows = max(1, min(G * n, (1 << 28) // R))
    for u in range(0, U, units):
        ok = live[u:u + units]
        K, V = (x[u:u + units].to(real).masked_fill(~ok[..., None], 0.0) for x in (Ku, Vu))
        for r in range(0, G * n, rows):
            x = torch.matmul(Qu[u:u + units, r:r + rows].to(real) * (1.0 / math.sqrt(D)), K.transpose(1, 2))
            x = x.masked_fill(~ok[:, None], -math.inf)
            m = x.amax(-1, keepdim=True)
            w = torch.exp(x - m.masked_fill(m == -math.inf, 0.0))
            total = w.sum(-1, keepdim=True)
            o = torch.matmul(w, V) / total.masked_fill(total == 0.0, 1.0)
            z = (m + total.log()).squeeze(-1)
            if case["join"]:
                z_in = st["lse_in"].view(U, G * n)[u:u + units, r:r + rows].to(real)
                both = torch.logaddexp(z, z_in)
                o = o * (z - both).exp()[..., None] + \
                    st["O_in"].view(U, G * n, D)[u:u + units, r:r + rows].to(real) * (z_in - both).exp()[..., None]
                z = both
            Ou[u:u + units, r:r + rows] = o.to(O.dtype)
            lu[u:u + units, r:r + rows] = z
    return {"O": O, "lse": lse}


def run(st):
    case, op = st["case"], st["case"]["op"]
    if not own:
        if op == "append":
            return _run_append(st)
        if op == "shared":
            st["out"].copy_(_run_shared(st))
            return st["out"]
        return _run_cross(st, st["O"], st["lse"])
    kvm = st["kvm"]
    if op == "append":
        kvm.kvm_paged_append(st["p"], st["cache"], st["pos"], st["turns"], st["q"], st["k"], st["v"], st["q_out"], st["len_out"],
                             new_len=st["new"], interleaved=case["interleaved"])
        return {"q": st["q_out"], "K": st["K"], "V": st["V"], "len": st["len_out"]}
    if op == "shared":
        kvm.kvm_shared_attend(st["p"], st["q"], st.get("K_pre"), st.get("V_pre"), st.get("pre_len"), st["cache"], st["out"], st["ws"])
        return st["out"]
    kvm.kvm_cross_attend(st["p"], st["Q"], st["K"], st["V"], st["len"], st["O"], st["lse"], st["ws"],
                         O_in=st.get("O_in"), lse_in=st.get("lse_in"))
    return {"O": st["O"], "lse": st["lse"]}


# ------------------------------------------------------------------ 64 bits, from the definitions
def _softmax_rows(q, K, V, scale):
    """One head's rows: softmax(q K^T scale) V and the log-sum-exp, over exactly the rows given."""
    x = scale * (q @ K.T)
    z = torch.logsumexp(x, -1)
    return torch.exp(x - z[:, None]) @ V, z


def exact(case, seed):
    st, f64 = prepare(case, seed), torch.float64
    B, Hq, Hkv, D = (case[k] for k in ("batch", "n_q_heads", "n_kv_heads", "head_dim"))
    G, scale, op = Hq // Hkv, 1.0 / math.sqrt(D), case["op"]
    if op == "append":
        T, R = case["tokens"], case["page_rows"]
        # the pair (x, y) at frequency i and position n is the complex number x + iy times exp(i n base^(-2i/D))
        power = torch.arange(D // 2, device="cuda", dtype=f64) * (2.0 / D)
        n = st["pos"].to(f64)[:, None] + torch.arange(T, device="cuda", dtype=f64)
        turn = torch.polar(torch.ones((), dtype=f64, device="cuda"), n[:, :, None] / torch.pow(BASE, power))[:, None]

        def spin(x):
            x = x.to(f64)
            if case["interleaved"]:
                return torch.view_as_real(torch.view_as_complex(x.reshape(*x.shape[:-1], D // 2, 2).contiguous()) * turn).flatten(-2)
            z = torch.complex(x[..., :D // 2].contiguous(), x[..., D // 2:].contiguous()) * turn
            return torch.cat([z.real, z.imag], -1)

        q, k, v = spin(st["q"]), spin(st["k"]), st["v"].to(f64)
        K, V, length = st["K"].to(f64), st["V"].to(f64), st["len"].cpu()
        new = torch.full((B, Hkv), T) if st["new"] is None else st["new"].cpu()
        for b in range(B):
            for h in range(Hkv):
                first, count = int(length[b, h]), int(new[b, h])
                rows = torch.arange(first, first + count, device="cuda")
                page = st["table"][b * Hkv + h, rows // R].long()
                K[page, rows % R] = k[b, h, :count]
                V[page, rows % R] = v[b, h, :count]
        return {"q": q, "K": K, "V": V, "len": length.to("cuda") + new.to("cuda")}
    if op == "shared":
        out = torch.zeros((B, Hkv, G, D), dtype=f64, device="cuda")
        c, q = st.get("pages"), st["q"].to(f64).view(B, Hkv, G, D)
        for h in range(Hkv):
            n_pre = int(st["pre_len"][h]) if case["prefix"] else 0
            Kp, Vp = ((st[x][h, :n_pre].to(f64) for x in ("K_pre", "V_pre")) if n_pre else (q.new_zeros(0, D), q.new_zeros(0, D)))
            for b in range(B):
                Ks, Vs = [Kp], [Vp]
                if c:
                    n_own = int(c["len"][b, h])
                    pages = c["table"][b * Hkv + h, :-(-n_own // case["page_rows"])].long()
                    Ks.append(c["K"][pages].reshape(-1, D)[:n_own].to(f64))
                    Vs.append(c["V"][pages].reshape(-1, D)[:n_own].to(f64))
                K, V = torch.cat(Ks), torch.cat(Vs)
                if K.shape[0]:
                    out[b, h] = _softmax_rows(q[b, h], K, V, scale)[0]
        return out.view(B, Hq, D)
    n = case["n_q"]
    O, lse = torch.zeros((B, Hq, n, D), dtype=f64, device="cuda"), torch.full((B, Hq, n), -math.inf, dtype=f64, device="cuda")
    for b in range(B):
        for h in range(Hq):
            m = int(st["len"][b, h // G])
            if m:
                K, V = st["K"][b, h // G, :m].to(f64), st["V"][b, h // G, :m].to(f64)
                O[b, h], lse[b, h] = _softmax_rows(st["Q"][b, h].to(f64), K, V, scale)
    if case["join"]:
        z_in = st["lse_in"].to(f64)
        a, c = torch.sigmoid(lse - z_in), torch.sigmoid(z_in - lse)
        O = O * a[..., None] + st["O_in"].to(f64) * c[..., None]
        lse = torch.maximum(lse, z_in) + torch.log1p(torch.exp(-(lse - z_in).abs()))
    return {"O": O, "lse": lse}


def work(case):
    B, Hq, Hkv, D = (case[k] for k in ("batch", "n_q_heads", "n_kv_heads", "head_dim"))
    e = 2 if case["dtype"] == "bf16" else 4
    if case["op"] == "append":
        T = case["tokens"]
        taken = 0.5 if case["ragged"] else 1.0             # (of the new rows, on average)
        q, kv = B * Hq * T * D, 2 * B * Hkv * T * D * taken
        return {"bytes": 2.0 * e * (q + kv) + 12.0 * B * Hkv, "flops": 3.0 * (q + kv / 2)}
    if case["op"] == "shared":
        pre, mine = 0.875 * case["prefix"], 0.75 * case["held"]        # lengths on average
        rows = Hkv * pre + B * Hkv * mine
        return {"bytes": 2.0 * D * e * rows + 2.0 * B * Hq * D * e, "flops": 4.0 * D * B * Hq * (pre + mine)}
    n, rows = case["n_q"], 0.875 * case["rows"]
    io = B * Hq * n * ((3 if case["join"] else 2) * D * e + (8 if case["join"] else 4))
    return {"bytes": io + 2.0 * B * Hkv * rows * D * e, "flops": 4.0 * D * B * Hq * n * rows}
