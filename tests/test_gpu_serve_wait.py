"""The give-up path of the serving kernels' bounded waits, on the test-only build whose producers leave out a stage: the kernels come back by
themselves, mark what they could not finish, report it, and the next call of the shipped library is right."""
import ctypes
import math

import pytest
import torch

import paper_2407_08454_b200 as kvm
from paper_2407_08454_b200 import build
from serve_ref import Rows, close, make_cache

pytestmark = pytest.mark.gpu
vp = ctypes.c_void_p


def ptr(t):
    return vp(0 if t is None else t.data_ptr())


def stream():
    return vp(torch.cuda.current_stream().cuda_stream)


def test_cross_attention_gives_up_and_says_so():
    lib = ctypes.CDLL(build.build_waittest())
    g = torch.Generator().manual_seed(21)
    B, H, n, rows, D = 1, 2, 300, 900, 128             # 8 steps per item: the fourth V tile never arrives in CTAs with that many
    p = kvm.make_params(B, H, H, 1, D, torch.bfloat16)
    # few CTAs with many steps: items stay whole
    Q = torch.randn(B, H, n, D, generator=g).bfloat16().cuda()
    K, V = (torch.randn(B, H, rows, D, generator=g).bfloat16().cuda() for _ in range(2))
    O, lse, stats = torch.zeros_like(Q), torch.zeros(B, H, n, device="cuda"), kvm.new_stats("cuda")
    ws = torch.empty(kvm.kvm_cross_workspace_bytes(p, n, rows), dtype=torch.uint8, device="cuda")
    rc = lib.kvm_cross_attend(ctypes.byref(p), ptr(Q), ctypes.c_int32(n), ptr(K), ptr(V), ctypes.c_int32(rows), vp(0), vp(0), vp(0), ptr(O),
                              ptr(lse), ptr(stats), ptr(ws), ctypes.c_size_t(ws.numel()), stream())
    assert rc == 0
    torch.cuda.synchronize()
    assert kvm.read_stats(stats).status == -9
    assert torch.isnan(O).any() and torch.isnan(lse).any()
    kvm.kvm_cross_attend(p, Q, K, V, None, O, lse, ws)
    for h in range(H):
        ref = Rows(Q[0, h].cpu(), K[0, h].cpu(), V[0, h].cpu(), 1.0 / math.sqrt(D))
        close(O[0, h], ref.O, ref.O_bound(torch.bfloat16), h)


def test_decode_attention_gives_up_and_says_so():
    lib = ctypes.CDLL(build.build_waittest())
    g = torch.Generator().manual_seed(22)
    B, H, D, n = 4, 8, 128, 200
    p = kvm.make_params(B, H, H, 1, D, torch.bfloat16)
    lengths = torch.full((B, H), n, dtype=torch.int32)
    K, V, table = make_cache(g, B, H, D, 16, lengths, torch.bfloat16)
    own = kvm.make_pages(K.cuda(), V.cuda(), table.cuda(), lengths.cuda())
    q = torch.randn(B, H, D, generator=g).bfloat16().cuda()
    out, stats = torch.zeros_like(q), kvm.new_stats("cuda")
    ws = torch.empty(kvm.kvm_shared_workspace_bytes(p, 0, own), dtype=torch.uint8, device="cuda")
    rc = lib.kvm_shared_attend(ctypes.byref(p), ptr(q), vp(0), vp(0), ctypes.c_int32(0), vp(0), ctypes.byref(own), ptr(out), ptr(stats), ptr(ws),
                               ctypes.c_size_t(ws.numel()), stream())
    assert rc == 0
    torch.cuda.synchronize()
    assert kvm.read_stats(stats).status == -9
    assert torch.isnan(out).any() and not torch.isnan(out).all()
    kvm.kvm_shared_attend(p, q, None, None, None, own, out, ws)
    for b in range(B):
        for h in range(H):
            rows = [(int(table[b * H + h, r // 16]), r % 16) for r in range(n)]
            Kr, Vr = (torch.stack([x[i, j] for i, j in rows]) for x in (K, V))
            ref = Rows(q[b, h:h + 1].cpu(), Kr, Vr, 1.0 / math.sqrt(D))
            close(out[b, h:h + 1], ref.O, ref.O_bound(torch.bfloat16), (b, h))


def shared_call(lib, p, q, Kp, Vp, pre_rows, pre_len, own, out, stats, ws):
    rc = lib.kvm_shared_attend(ctypes.byref(p), ptr(q), ptr(Kp), ptr(Vp), ctypes.c_int32(pre_rows), ptr(pre_len), ctypes.byref(own), ptr(out),
                               ptr(stats), ptr(ws), ctypes.c_size_t(ws.numel()), stream())
    assert rc == 0
    torch.cuda.synchronize()


def own_rows(K, V, table_row, n, R=16):
    rows = [(int(table_row[r // R]), r % R) for r in range(n)]
    return (torch.stack([x[i, j] for i, j in rows]) for x in (K, V))


@pytest.mark.parametrize("n,room,spoilt", [
    (600, 0, [0]),                # units in parts of several warps: the state of one of them never comes, the join passes its mark on
    (24, 1000, [4, 5, 6, 7]),     # units that a warp has whole, straight to the output (the other warps of the block may see the flag)
])
def test_decode_attention_in_shares_gives_up_and_says_so(n, room, spoilt):
    lib = ctypes.CDLL(build.build_waittest())
    g = torch.Generator().manual_seed(23)
    B, H, D = 4, 8, 128
    p = kvm.make_params(B, H, H, 1, D, torch.bfloat16)
    lengths = torch.full((B, H), n, dtype=torch.int32)
    K, V, table = make_cache(g, B, H, D, 16, lengths, torch.bfloat16, room=room)
    own = kvm.make_pages(K.cuda(), V.cuda(), table.cuda(), lengths.cuda())
    q = torch.randn(B, H, D, generator=g).bfloat16().cuda()
    out, stats = torch.zeros_like(q), kvm.new_stats("cuda")
    ws = torch.empty(kvm.kvm_shared_workspace_bytes(p, 0, own), dtype=torch.uint8, device="cuda")
    shared_call(lib, p, q, None, None, 0, None, own, out, stats, ws)
    assert kvm.read_stats(stats).status == -9
    got = out.view(B * H, D).cpu()
    bad = got.isnan().any(-1)
    assert bool(bad[spoilt[0]]) and not [u for u in range(B * H) if bad[u] and u not in spoilt]
    assert torch.equal(got.isnan().all(-1), bad)
    kvm.kvm_shared_attend(p, q, None, None, None, own, out, ws)
    for u in range(B * H):
        ref = Rows(q.view(B * H, 1, D)[u].cpu(), *own_rows(K, V, table[u], n), 1.0 / math.sqrt(D))
        close(out.view(B * H, 1, D)[u], ref.O, ref.O_bound(torch.bfloat16), u)
        if not bad[u]:
            close(got[u:u + 1], ref.O, ref.O_bound(torch.bfloat16), u)


@pytest.mark.parametrize("n", [200, 100])      # two query tiles, cut items; one tile, two states to a piece
def test_cross_attention_in_pieces_gives_up_and_says_so(n):
    """Every CTA that has four steps leaves out the fourth one's tiles.  Units of 40,000 keys lose some of their pieces, one without keys nothing;
    what is joined in has seen no keys in the first row, which must not hide the mark."""
    lib = ctypes.CDLL(build.build_waittest())
    g = torch.Generator().manual_seed(24)
    B, H, rows, D = 1, 3, 40000, 128
    p = kvm.make_params(B, H, H, 1, D, torch.bfloat16)
    Q = torch.randn(B, H, n, D, generator=g).bfloat16().cuda()
    K, V = (torch.randn(B, H, rows, D, generator=g).bfloat16().cuda() for _ in range(2))
    ln = torch.tensor([[rows, 0, rows]], dtype=torch.int32, device="cuda")
    O_in, lse_in = torch.randn(B, H, n, D, generator=g).bfloat16().cuda(), torch.randn(B, H, n, generator=g).cuda()
    lse_in[:, :, 0] = -math.inf
    O, lse, stats = torch.zeros_like(Q), torch.zeros(B, H, n, device="cuda"), kvm.new_stats("cuda")
    ws = torch.empty(kvm.kvm_cross_workspace_bytes(p, n, rows), dtype=torch.uint8, device="cuda")
    rc = lib.kvm_cross_attend(ctypes.byref(p), ptr(Q), ctypes.c_int32(n), ptr(K), ptr(V), ctypes.c_int32(rows), ptr(ln), ptr(O_in), ptr(lse_in), ptr(O),
                              ptr(lse), ptr(stats), ptr(ws), ctypes.c_size_t(ws.numel()), stream())
    assert rc == 0
    torch.cuda.synchronize()
    assert kvm.read_stats(stats).status == -9
    for h in (0, 2):
        assert O[0, h].isnan().all() and lse[0, h].isnan().all()
    assert torch.equal(lse[0, 1], lse_in[0, 1]) and torch.equal(O[0, 1, 1:], O_in[0, 1, 1:]) and (O[0, 1, 0] == 0).all()
    kvm.kvm_cross_attend(p, Q, K, V, ln, O, lse, ws, O_in=O_in, lse_in=lse_in)
    for h in (0, 2):
        ref = Rows(Q[0, h].cpu(), K[0, h].cpu(), V[0, h].cpu(), 1.0 / math.sqrt(D)).joined(O_in[0, h].cpu(), lse_in[0, h].cpu())
        close(O[0, h], ref.O, ref.O_bound(torch.bfloat16), h)


def test_prefix_beside_own_rows_gives_up_and_says_so():
    """A long prefix of one head loses pieces, which spoils that head; a block of the kernel beside it loses some of the own rows."""
    lib = ctypes.CDLL(build.build_waittest())
    g = torch.Generator().manual_seed(25)
    B, Hq, Hkv, D, P, n = 64, 8, 2, 128, 80000, 100
    G = Hq // Hkv
    p = kvm.make_params(B, Hq, Hkv, 1, D, torch.bfloat16)
    lengths = torch.full((B, Hkv), n, dtype=torch.int32)
    K, V, table = make_cache(g, B, Hkv, D, 16, lengths, torch.bfloat16)
    own = kvm.make_pages(K.cuda(), V.cuda(), table.cuda(), lengths.cuda())
    Kp, Vp = (torch.randn(Hkv, P, D, generator=g).bfloat16().cuda() for _ in range(2))
    pre_len = torch.tensor([P, 0], dtype=torch.int32, device="cuda")
    q = torch.randn(B, Hq, D, generator=g).bfloat16().cuda()
    out, stats = torch.zeros_like(q), kvm.new_stats("cuda")
    ws = torch.empty(kvm.kvm_shared_workspace_bytes(p, P, own), dtype=torch.uint8, device="cuda")
    shared_call(lib, p, q, Kp, Vp, P, pre_len, own, out, stats, ws)
    assert kvm.read_stats(stats).status == -9
    got = out.cpu()
    assert got[:, :G].isnan().all()
    bad = got[:, G:].isnan().any(-1).any(-1)
    assert bool(bad.any()) and int(bad.sum()) <= B // 4
    kvm.kvm_shared_attend(p, q, Kp, Vp, pre_len, own, out, ws)
    for b in range(B):
        ref = Rows(q[b, G:].cpu(), *own_rows(K, V, table[b * Hkv + 1], n), 1.0 / math.sqrt(D))
        close(out[b, G:], ref.O, ref.O_bound(torch.bfloat16), b)
        if not bad[b]:
            close(got[b, G:], ref.O, ref.O_bound(torch.bfloat16), b)
    for b in range(0, B, 16):
        Ko, Vo = own_rows(K, V, table[b * Hkv], n)
        ref = Rows(q[b, :G].cpu(), torch.cat([Kp[0].cpu(), Ko]), torch.cat([Vp[0].cpu(), Vo]), 1.0 / math.sqrt(D))
        close(out[b, :G], ref.O, ref.O_bound(torch.bfloat16), b)
