"""The serving operators together, as they are used: a prompt is prefilled and compressed, a batch decodes behind it with rows of its
own, the next prompt chunk attends to the compressed rows and to itself; captured into graphs, on other streams, with shared workspaces."""
import math

import pytest
import torch

import paper_2407_08454_b200 as kvm
from serve_ref import F64, Rows, close, make_cache, rotate, turns

pytestmark = pytest.mark.gpu


def layer(g, B, Hq, Hkv, S, D, dtype):
    """Keys whose neighbours are alike, so that the compression merges some."""
    K = torch.randn(B, Hkv, S, D, generator=g)
    for t in range(1, S):
        K[:, :, t] = 0.93 * K[:, :, t - 1] + math.sqrt(1 - 0.93 ** 2) * K[:, :, t]
    Q, V = torch.randn(B, Hq, S, D, generator=g), torch.randn(B, Hkv, S, D, generator=g)
    return [x.to(dtype).cuda() for x in (Q, K, V)]


def compress(Q, K, V, **kw):
    B, Hq, S, D = Q.shape
    p = kvm.make_params(B, Hq, K.shape[1], S, D, Q.dtype, **kw)
    c = kvm.Compressor(p)
    return p, c(Q, K, V)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_a_batch_decodes_behind_a_compressed_prompt(dtype):
    """Prompt -> kvm_compress -> decode steps of a batch: append (rotated, lengths in place) and shared attention, five steps captured
    into one graph and replayed twice; every step's output against 64 bits on the stored caches."""
    g = torch.Generator().manual_seed(11)
    B, Hq, Hkv, S, D, R, steps = 5, 8, 4, 300, 64, 16, 5
    _, c = compress(*layer(g, 1, Hq, Hkv, S, D, dtype))
    p = kvm.make_params(B, Hq, Hkv, 1, D, dtype)
    U, room = B * Hkv, 2
    table = torch.randperm(U * room, generator=g).to(torch.int32).view(U, room)
    pool = [torch.full((U * room, R, D), math.nan, dtype=dtype, device="cuda") for _ in range(2)]
    length = torch.zeros(B, Hkv, dtype=torch.int32, device="cuda")
    cache = kvm.make_pages(pool[0], pool[1], table.cuda(), length)
    tr = kvm.rope_turns(D)
    q, k, v = (torch.randn(steps, B, h, 1, D, generator=g).to(dtype) for h in (Hq, Hkv, Hkv))
    qd, kd, vd = (torch.empty_like(x, device="cuda") for x in (q, k, v))
    pos = torch.empty(B, dtype=torch.int32, device="cuda")
    q_rot = torch.empty(B, Hq, 1, D, dtype=dtype, device="cuda")
    outs = torch.empty(steps, B, Hq, D, dtype=dtype, device="cuda")
    ws = torch.empty(kvm.kvm_shared_workspace_bytes(p, c.cap, cache), dtype=torch.uint8, device="cuda")

    def run():
        for s in range(steps):
            kvm.kvm_paged_append(p, cache, pos, tr, qd[s], kd[s], vd[s], q_rot, length)
            kvm.kvm_shared_attend(p, q_rot.view(B, Hq, D), c.K_out, c.V_out, c.out_len, cache, outs[s], ws)
            pos.add_(1)

    for x, y in ((qd, q), (kd, k), (vd, v)):
        x.copy_(y)
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):                       # (warm up outside the capture, on the stream that captures)
        pos.fill_(S)
        run()
    side.synchronize()
    length.zero_()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        run()
    length.zero_()
    pos.fill_(S)
    for replay in range(2):                             # the second replay continues behind the first one's rows
        graph.replay()
        torch.cuda.synchronize()
        n0 = replay * steps
        assert (length == n0 + steps).all()
        Kc, Vc = pool[0].cpu(), pool[1].cpu()
        n_pre = c.out_len.view(-1).cpu()
        for s in range(steps):
            at = torch.full((B, 1), S + n0 + s)
            want_q = rotate(q[s].to(F64), at[:, None].expand(B, Hq, 1), turns(D), False)
            want_k = rotate(k[s].to(F64), at[:, None].expand(B, Hkv, 1), turns(D), False)
            for b in range(B):
                for h in range(Hkv):
                    rows = torch.arange(n0 + s + 1)
                    page = table[b * Hkv + h][rows // R].long()
                    Ko, Vo = Kc[page, rows % R], Vc[page, rows % R]
                    bound = 1e-5 + 2.0 ** -8 * want_k[b, h].abs() if dtype == torch.bfloat16 else torch.full((1, D), 1e-5)
                    close(Ko[-1:], want_k[b, h], bound, "key")
                    # the rotated queries as they were stored: one rounding
                    qs = want_q[b, h * 2:h * 2 + 2, 0].to(dtype)
                    ref = Rows(qs, torch.cat([c.K_out[0, h, :int(n_pre[h])].cpu(), Ko]), torch.cat([c.V_out[0, h, :int(n_pre[h])].cpu(), Vo]),
                               1.0 / math.sqrt(D))
                    # (a query may round the other way: one step of it moves each logit by 2^-8 (2^-24) of sum |q_i k_i| at most)
                    step = 2.0 ** -8 if dtype == torch.bfloat16 else 2.0 ** -22
                    slack = 2.0 * step * ref.dot[:, None] * ref.vmax * 0.25
                    close(outs[s, b, h * 2:h * 2 + 2], ref.O, ref.O_bound(dtype) + slack, (replay, s, b, h))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_compressed_caches_move_into_pages_and_decode_alike(dtype):
    """Units of a compressed batch hold different numbers of rows: moved into pages they give what kvm_attend gives on the contiguous cache."""
    g = torch.Generator().manual_seed(12)
    B, Hq, Hkv, S, D, R = 3, 4, 2, 260, 128, 32
    p, c = compress(*layer(g, B, Hq, Hkv, S, D, dtype))
    U = B * Hkv
    room = -(-c.cap // R)
    table = torch.randperm(U * room, generator=g).to(torch.int32).view(U, room).cuda()
    pool = [torch.full((U * room, R, D), math.nan, dtype=dtype, device="cuda") for _ in range(2)]
    length = torch.zeros(B, Hkv, dtype=torch.int32, device="cuda")
    cache = kvm.make_pages(pool[0], pool[1], table, length)
    kvm.kvm_paged_append(p, cache, None, None, None, c.K_out, c.V_out, None, length, new_len=c.out_len)
    assert torch.equal(length, c.out_len)
    q = torch.randn(B, Hq, D, generator=g).to(dtype).cuda()
    out = torch.empty(B, Hq, D, dtype=dtype, device="cuda")
    ws = torch.empty(kvm.kvm_shared_workspace_bytes(p, 0, cache), dtype=torch.uint8, device="cuda")
    kvm.kvm_shared_attend(p, q, None, None, None, cache, out, ws)
    want = torch.empty(B, Hq, D, device="cuda")
    kvm.kvm_attend(p, q, c.K_out, c.V_out, c.cap, c.out_len, want, torch.empty(kvm.kvm_workspace_bytes(p), dtype=torch.uint8, device="cuda"))
    for b in range(B):
        for h in range(Hkv):
            n = int(c.out_len[b, h])
            ref = Rows(q[b, 2 * h:2 * h + 2].cpu(), c.K_out[b, h, :n].cpu(), c.V_out[b, h, :n].cpu(), 1.0 / math.sqrt(D))
            close(out[b, 2 * h:2 * h + 2], ref.O, ref.O_bound(dtype), (b, h))
            close(want[b, 2 * h:2 * h + 2], ref.O, ref.O_bound(torch.float32) + 1e-4, (b, h))


@pytest.mark.parametrize("S,n", [(300, 77), (513, 300)])
def test_the_next_chunk_attends_to_its_compressed_past_and_to_itself(S, n):
    """kvm_prefill_attend over the chunk, kvm_cross_attend over the compressed past joined with it: softmax over both."""
    g = torch.Generator().manual_seed(13)
    B, Hq, Hkv, D = 2, 8, 2, 128
    _, c = compress(*layer(g, B, Hq, Hkv, S, D, torch.bfloat16), budget=0.35)
    Q, K, V = layer(g, B, Hq, Hkv, n, D, torch.bfloat16)
    # (softmax_scale and the shape are what the calls share; seq is the chunk's for the causal part)
    p = kvm.make_params(B, Hq, Hkv, n, D, torch.bfloat16)
    O, lse = torch.empty_like(Q), torch.empty(B, Hq, n, device="cuda")
    kvm.kvm_prefill_attend(p, Q, K, V, O, lse)
    O1, lse1 = O.clone(), lse.clone()
    ws = torch.empty(kvm.kvm_cross_workspace_bytes(p, n, c.cap), dtype=torch.uint8, device="cuda")
    kvm.kvm_cross_attend(p, Q, c.K_out, c.V_out, c.out_len, O, lse, ws, O_in=O, lse_in=lse)          # in place
    G, sc = Hq // Hkv, 1.0 / math.sqrt(D)
    for b in range(B):
        for h in range(Hq):
            m = int(c.out_len[b, h // G])
            ref = Rows(Q[b, h].cpu(), c.K_out[b, h // G, :m].cpu(), c.V_out[b, h // G, :m].cpu(), sc).joined(O1[b, h].cpu(), lse1[b, h].cpu())
            close(O[b, h], ref.O, ref.O_bound(torch.bfloat16), (b, h))
            close(lse[b, h], ref.lse, ref.lse_bound(), (b, h))
            # ... and against one softmax over everything
            x = sc * (Q[b, h].cpu().to(F64) @ torch.cat([c.K_out[b, h // G, :m].cpu(), K[b, h // G].cpu()]).to(F64).T)
            x[:, m:] = x[:, m:].masked_fill(torch.ones(n, n, dtype=torch.bool).triu(1), -math.inf)
            want = torch.softmax(x, -1) @ torch.cat([c.V_out[b, h // G, :m].cpu(), V[b, h // G].cpu()]).to(F64)
            # two roundings of O to bf16 and two of the weights, each 2^-8 of at most the largest value
            assert float((O[b, h].cpu().to(F64) - want).abs().max()) <= 4 * 2.0 ** -8 * ref.vmax


def test_two_graphs_that_share_a_workspace():
    """Two captured calls with one workspace, replayed in turn on one stream, give what they give alone."""
    g = torch.Generator().manual_seed(14)
    D = 128
    shapes = [(3, 8, 2, 200, 900), (2, 4, 4, 5, 1500)]
    calls, need = [], 0
    for B, Hq, Hkv, n, rows in shapes:
        p = kvm.make_params(B, Hq, Hkv, 1, D, torch.bfloat16)
        Q = torch.randn(B, Hq, n, D, generator=g).bfloat16().cuda()
        K, V = (torch.randn(B, Hkv, rows, D, generator=g).bfloat16().cuda() for _ in range(2))
        O, lse = torch.empty_like(Q), torch.empty(B, Hq, n, device="cuda")
        calls.append((p, Q, K, V, O, lse))
        need = max(need, kvm.kvm_cross_workspace_bytes(p, n, rows))
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    alone = []
    for p, Q, K, V, O, lse in calls:
        kvm.kvm_cross_attend(p, Q, K, V, None, O, lse, ws)
        alone.append((O.clone(), lse.clone()))
    torch.cuda.synchronize()
    graphs = []
    for p, Q, K, V, O, lse in calls:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            kvm.kvm_cross_attend(p, Q, K, V, None, O, lse, ws)
        graphs.append(graph)
    for _ in range(3):
        for (_, _, _, _, O, lse), graph, (Ow, lw) in zip(calls, graphs, alone):
            O.fill_(7.0)
            graph.replay()
            assert torch.equal(O, Ow) and torch.equal(lse, lw)


def test_calls_on_several_streams_at_once():
    """Independent calls, each with its own workspace, on streams of their own and named by argument."""
    g = torch.Generator().manual_seed(15)
    B, Hq, Hkv, D, P, held = 4, 8, 4, 128, 700, 90
    p = kvm.make_params(B, Hq, Hkv, 1, D, torch.bfloat16)
    lengths = torch.randint(1, held + 1, (B, Hkv), generator=g, dtype=torch.int32)
    K, V, table = make_cache(g, B, Hkv, D, 16, lengths, torch.bfloat16)
    own = kvm.make_pages(K.cuda(), V.cuda(), table.cuda(), lengths.cuda())
    Kp, Vp = (torch.randn(Hkv, P, D, generator=g).bfloat16().cuda() for _ in range(2))
    q = [torch.randn(B, Hq, D, generator=g).bfloat16().cuda() for _ in range(4)]
    n = kvm.kvm_shared_workspace_bytes(p, P, own)
    ws = [torch.empty(n, dtype=torch.uint8, device="cuda") for _ in q]
    want = []
    for x, w in zip(q, ws):
        out = torch.empty_like(x)
        kvm.kvm_shared_attend(p, x, Kp, Vp, None, own, out, w)
        want.append(out)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in q]
    outs = [torch.empty_like(x) for x in q]
    torch.cuda.synchronize()
    for _ in range(20):
        for x, w, o, s in zip(q, ws, outs, streams):
            kvm.kvm_shared_attend(p, x, Kp, Vp, None, own, o, w, stream=s)
    torch.cuda.synchronize()
    for o, w in zip(outs, want):
        assert torch.equal(o, w)


def test_prefix_and_own_rows_side_by_side():
    """A batch large enough for the prefix to have a kernel of its own, which runs beside the one for the sequences' rows: captured and replayed, and
    from two streams at once, it gives the bits of the plain call, which are right."""
    g = torch.Generator().manual_seed(31)
    B, Hq, Hkv, D, P, held, R = 64, 8, 2, 128, 1200, 100, 16
    p = kvm.make_params(B, Hq, Hkv, 1, D, torch.bfloat16)
    lengths = torch.randint(0, held + 1, (B, Hkv), generator=g, dtype=torch.int32)
    K, V, table = make_cache(g, B, Hkv, D, R, lengths, torch.bfloat16)
    own = kvm.make_pages(K.cuda(), V.cuda(), table.cuda(), lengths.cuda())
    Kp, Vp = (torch.randn(Hkv, P, D, generator=g).bfloat16() for _ in range(2))
    n_pre = torch.tensor([P, 900], dtype=torch.int32)
    q = [torch.randn(B, Hq, D, generator=g).bfloat16() for _ in range(2)]
    qd, Kd, Vd, nd = [x.cuda() for x in q], Kp.cuda(), Vp.cuda(), n_pre.cuda()
    n = kvm.kvm_shared_workspace_bytes(p, P, own)
    ws = [torch.full((n,), 255, dtype=torch.uint8, device="cuda") for _ in q]
    want = []
    for x, w in zip(qd, ws):
        out = torch.empty_like(x)
        kvm.kvm_shared_attend(p, x, Kd, Vd, nd, own, out, w)
        want.append(out)
    torch.cuda.synchronize()
    G = Hq // Hkv
    for b in range(0, B, 7):
        for h in range(Hkv):
            rows = torch.arange(int(lengths[b, h]))
            page = table[b * Hkv + h][rows // R].long()
            ref = Rows(q[0][b, h * G:(h + 1) * G], torch.cat([Kp[h, :int(n_pre[h])], K[page, rows % R]]),
                       torch.cat([Vp[h, :int(n_pre[h])], V[page, rows % R]]), 1.0 / math.sqrt(D))
            close(want[0][b, h * G:(h + 1) * G], ref.O, ref.O_bound(torch.bfloat16), (b, h))
    out = torch.empty_like(want[0])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        for _ in range(3):
            kvm.kvm_shared_attend(p, qd[0], Kd, Vd, nd, own, out, ws[0])
    for _ in range(10):
        out.fill_(math.nan)
        graph.replay()
        assert torch.equal(out, want[0])
    streams, outs = [torch.cuda.Stream() for _ in q], [torch.empty_like(x) for x in qd]
    torch.cuda.synchronize()
    for _ in range(30):
        for x, w, o, s in zip(qd, ws, outs, streams):
            kvm.kvm_shared_attend(p, x, Kd, Vd, nd, own, o, w, stream=s)
    torch.cuda.synchronize()
    for o, w in zip(outs, want):
        assert torch.equal(o, w)


def test_rows_behind_the_outputs_are_left_as_they_were():
    """Outputs that lie inside larger buffers: what surrounds them keeps its bits (tiles and boxes end past the last row)."""
    g = torch.Generator().manual_seed(32)
    for dtype in (torch.bfloat16, torch.float32):
        for B, Hq, Hkv, n, rows, D in ((2, 6, 2, 43, 300, 128), (3, 4, 4, 1, 77, 64), (1, 3, 1, 200, 2600, 64)):
            p = kvm.make_params(B, Hq, Hkv, 1, D, dtype)
            Q = torch.randn(B, Hq, n, D, generator=g).to(dtype).cuda()
            K, V = (torch.randn(B, Hkv, rows, D, generator=g).to(dtype).cuda() for _ in range(2))
            size, pad = Q.numel(), 64 * D
            buf, lbuf = torch.full((size + 2 * pad,), 7.0, dtype=dtype, device="cuda"), torch.full((B * Hq * n + 256,), 7.0, device="cuda")
            O, lse = buf[pad:pad + size].view(Q.shape), lbuf[128:128 + B * Hq * n].view(B, Hq, n)
            ws = torch.empty(kvm.kvm_cross_workspace_bytes(p, n, rows) + 256, dtype=torch.uint8, device="cuda")
            need = ws.numel() - 256
            ws[need:] = 99
            kvm.kvm_cross_attend(p, Q, K, V, None, O, lse, ws[:need])
            assert (buf[:pad] == 7).all() and (buf[pad + size:] == 7).all()
            assert (lbuf[:128] == 7).all() and (lbuf[128 + lse.numel():] == 7).all() and (ws[need:] == 99).all()
            if n == 1:                                  # a decode step, the same
                q, ob = Q[:, :, 0].contiguous(), torch.full((B * Hq * D + 2 * pad,), 7.0, dtype=dtype, device="cuda")
                out = ob[pad:pad + B * Hq * D].view(B, Hq, D)
                Kp, Vp = K[0].contiguous(), V[0].contiguous()
                ws = torch.empty(kvm.kvm_shared_workspace_bytes(p, rows, None) + 256, dtype=torch.uint8, device="cuda")
                ws[-256:] = 99
                kvm.kvm_shared_attend(p, q, Kp, Vp, None, None, out, ws[:-256])
                assert (ob[:pad] == 7).all() and (ob[pad + out.numel():] == 7).all() and (ws[-256:] == 99).all()


def test_workspaces_and_stats_on_the_host_are_refused():
    p = kvm.make_params(1, 2, 2, 1, 64, torch.float32)
    q, K, lse = torch.zeros(1, 2, 3, 64, device="cuda"), torch.zeros(1, 2, 5, 64, device="cuda"), torch.zeros(1, 2, 3, device="cuda")
    ws = torch.zeros(kvm.kvm_cross_workspace_bytes(p, 3, 5), dtype=torch.uint8, device="cuda")
    for w, stats in ((ws.cpu(), None), (ws, kvm.new_stats("cpu")), (ws, kvm.new_stats("cuda")[:-8])):
        with pytest.raises(ValueError):
            kvm.kvm_cross_attend(p, q, K, K, None, q.clone(), lse, w, stats=stats)
        with pytest.raises(ValueError):
            kvm.kvm_shared_attend(p, q[:, :, 0].contiguous(), K[0], K[0], None, None, q[:, :, 0].contiguous(), w, stats=stats)
    with pytest.raises(kvm.KvmError):
        kvm.kvm_cross_attend(p, q, K, K, None, q.clone(), lse, None)


def test_a_large_batch_decodes_beside_its_prefix():
    """Append and shared attention step by step where the prefix has a kernel of its own: the paged kernel beside it reads lengths, queries and rows that the
    call before has just written.  Some sequences begin without rows.  Called one after the other, and captured and replayed."""
    g = torch.Generator().manual_seed(33)
    B, Hq, Hkv, D, P, R, steps = 64, 8, 2, 128, 1200, 16, 4
    G, U, room = Hq // Hkv, B * Hkv, 4
    p = kvm.make_params(B, Hq, Hkv, 1, D, torch.bfloat16)
    start = torch.randint(0, 30, (B, Hkv), generator=g, dtype=torch.int32)
    start[::5] = 0
    table = torch.randperm(U * room, generator=g).to(torch.int32).view(U, room)
    first = [torch.randn(U * room, R, D, generator=g).bfloat16() for _ in range(2)]
    pool, length = [x.cuda() for x in first], start.cuda()
    cache = kvm.make_pages(pool[0], pool[1], table.cuda(), length)
    q, k, v = (torch.randn(steps, B, h, 1, D, generator=g).bfloat16().cuda() for h in (Hq, Hkv, Hkv))
    Kp, Vp = (torch.randn(Hkv, P, D, generator=g).bfloat16() for _ in range(2))
    Kd, Vd, n_pre = Kp.cuda(), Vp.cuda(), torch.tensor([P, 900], dtype=torch.int32, device="cuda")
    tr, pos = kvm.rope_turns(D), torch.full((B,), P, dtype=torch.int32, device="cuda")
    q_rot, outs = torch.empty(steps, B, Hq, 1, D, dtype=torch.bfloat16, device="cuda"), torch.zeros(steps, B, Hq, D, dtype=torch.bfloat16, device="cuda")
    ws = torch.full((kvm.kvm_shared_workspace_bytes(p, P, cache),), 255, dtype=torch.uint8, device="cuda")

    def run():
        for s in range(steps):
            kvm.kvm_paged_append(p, cache, pos, tr, q[s], k[s], v[s], q_rot[s], length)
            kvm.kvm_shared_attend(p, q_rot[s].view(B, Hq, D), Kd, Vd, n_pre, cache, outs[s], ws)
            pos.add_(1)

    def reset():
        for x, y in zip(pool, first):
            x.copy_(y)
        length.copy_(start)
        pos.fill_(P)
        outs.zero_()

    torch.cuda.synchronize()
    run()
    torch.cuda.synchronize()
    want = [x.clone() for x in (outs, q_rot, length, *pool)]
    Kc, Vc, qc = pool[0].cpu(), pool[1].cpu(), q_rot.cpu()
    assert torch.equal(length.cpu(), start + steps)
    for s in range(steps):
        for b in (0, 5, 13, 31, 50, 63):
            for h in range(Hkv):
                rows = torch.arange(int(start[b, h]) + s + 1)
                page = table[b * Hkv + h][rows // R].long()
                m = (P, 900)[h]
                ref = Rows(qc[s, b, h * G:(h + 1) * G, 0], torch.cat([Kp[h, :m], Kc[page, rows % R]]), torch.cat([Vp[h, :m], Vc[page, rows % R]]),
                           1.0 / math.sqrt(D))
                close(outs[s, b, h * G:(h + 1) * G], ref.O, ref.O_bound(torch.bfloat16), (s, b, h))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    for _ in range(5):
        reset()
        graph.replay()
        for x, w in zip((outs, q_rot, length, *pool), want):
            assert torch.equal(x, w)
    for _ in range(5):
        reset()
        run()
        for x, w in zip((outs, q_rot, length, *pool), want):
            assert torch.equal(x, w)
