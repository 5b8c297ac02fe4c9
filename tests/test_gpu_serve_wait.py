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
