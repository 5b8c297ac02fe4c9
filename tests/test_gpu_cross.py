"""kvm_cross_attend against 64 bits: output and log-sum-exp, ragged and empty units, joined with other keys' attention."""
import math

import pytest
import torch

import paper_2407_08454_b200 as kvm
from serve_ref import Rows, close

pytestmark = pytest.mark.gpu


def check(B, Hq, Hkv, n_q, rows, D, dtype, join=False, lengths="ragged", in_place=False, seed=0, scale=0.0):
    g = torch.Generator().manual_seed(seed + B + Hq * 3 + n_q * 5 + rows)
    G, U = Hq // Hkv, B * Hkv
    p = kvm.make_params(B, Hq, Hkv, 1, D, dtype, softmax_scale=scale)
    Q = (2.0 * torch.randn(B, Hq, n_q, D, generator=g)).to(dtype)
    K, V = (torch.randn(B, Hkv, rows, D, generator=g).to(dtype) for _ in range(2))
    ln = torch.full((B, Hkv), rows, dtype=torch.int32)
    if lengths == "ragged":
        ln = torch.randint(0, rows + 1, (B, Hkv), generator=g, dtype=torch.int32)
        ln.view(-1)[-1] = rows
        if U > 1:
            ln.view(-1)[0] = 0
    for u in range(U):
        K.view(U, rows, D)[u, int(ln.view(-1)[u]):] = math.nan
        V.view(U, rows, D)[u, int(ln.view(-1)[u]):] = math.inf
    O_in = lse_in = None
    if join:
        O_in = torch.randn(B, Hq, n_q, D, generator=g).to(dtype)
        lse_in = 3.0 * torch.randn(B, Hq, n_q, generator=g) + math.log(max(rows, 2))
        lse_in[..., 0] = -math.inf                         # a query that has seen no other keys: its O_in may be anything
        O_in[:, :, 0] = math.nan
        lse_in[..., -1] += 200.0                           # ... and one for which the rows here weigh nothing
    O = torch.full((B, Hq, n_q, D), math.nan, dtype=dtype, device="cuda")
    lse = torch.full((B, Hq, n_q), math.nan, device="cuda")
    a = b = None
    if join:
        a, b = O_in.cuda(), lse_in.cuda()
        if in_place:
            O, lse = a, b
    ws = torch.full((kvm.kvm_cross_workspace_bytes(p, n_q, rows),), 255, dtype=torch.uint8, device="cuda")
    stats = kvm.new_stats("cuda")
    args = (p, Q.cuda(), K.cuda(), V.cuda(), None if lengths is None else ln.cuda())
    kvm.kvm_cross_attend(*args, O, lse, ws, O_in=a, lse_in=b, stats=stats)
    assert kvm.read_stats(stats).status == 0
    if not in_place:
        O2, lse2 = torch.empty_like(O), torch.empty_like(lse)
        kvm.kvm_cross_attend(*args, O2, lse2, ws, O_in=a, lse_in=b)
        assert torch.equal(O, O2) and torch.equal(lse, lse2)
    sc = scale if scale > 0 else 1.0 / math.sqrt(D)
    for bi in range(B):
        for h in range(Hq):
            n = int(ln[bi, h // G])
            ref = Rows(Q[bi, h], K[bi, h // G, :n], V[bi, h // G, :n], sc)
            if join:
                ref.joined(O_in[bi, h], lse_in[bi, h])
            close(O[bi, h], ref.O, ref.O_bound(dtype), ("O", bi, h, n))
            close(lse[bi, h], ref.lse, ref.lse_bound(), ("lse", bi, h, n))


SHAPES = [
    # B, Hq, Hkv, n_q, rows, D
    (1, 1, 1, 1, 1, 128),
    (2, 4, 2, 1, 300, 64),
    (2, 4, 4, 1, 128, 128),
    (3, 8, 2, 5, 1000, 128),              # drafted tokens
    (1, 2, 2, 127, 129, 64),
    (1, 2, 1, 128, 127, 128),             # 256 rows a head: two full tiles
    (2, 6, 2, 43, 128, 128),              # 129 rows
    (1, 3, 1, 200, 260, 64),              # 600: three tiles and a bit
    (2, 2, 2, 300, 77, 128),
    (1, 4, 1, 129, 513, 128),
    (5, 5, 5, 64, 65, 64),
    (1, 1, 1, 700, 1500, 128),
    (8, 16, 8, 20, 200, 128),
    (40, 8, 4, 3, 40, 64),                # more units than SMs
    (1, 16, 16, 260, 390, 128),
    (3, 8, 8, 300, 1000, 128),            # more steps than SMs: shares that hold whole items and parts
    (6, 8, 4, 200, 700, 64),
    (1, 2, 1, 7, 4000, 128),              # one tile, keys in many pieces of one step
    (12, 8, 8, 9, 2600, 128),             # ... of several steps
    (30, 4, 4, 100, 2000, 64),
]


@pytest.mark.parametrize("B,Hq,Hkv,n_q,rows,D", SHAPES)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("join", [False, True])
def test_cross_matches_64_bits(B, Hq, Hkv, n_q, rows, D, dtype, join):
    check(B, Hq, Hkv, n_q, rows, D, dtype, join=join)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("n_q", [3, 290])
def test_cross_in_place_without_lengths_and_with_a_scale(dtype, n_q):
    check(2, 8, 4, n_q, 333, 128, dtype, join=True, in_place=True)
    check(2, 8, 4, n_q, 256, 64, dtype, lengths=None, scale=0.05)
    check(1, 2, 2, n_q, 5000, 128, dtype, join=True)       # one unit's keys in many pieces


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_a_maximum_that_keeps_growing(dtype):
    """Keys that outgrow one another by more than any step of a running reference, all through the sequence."""
    B, H, n_q, rows, D = 1, 2, 140, 900, 128
    g = torch.Generator().manual_seed(8)
    u = torch.randn(H, 1, D, generator=g)
    Q = (u / u.norm(dim=-1, keepdim=True) * torch.linspace(1.0, 8.0, n_q)[:, None]).to(dtype).view(B, H, n_q, D)
    K = (u / u.norm(dim=-1, keepdim=True) * torch.linspace(-60.0, 120.0, rows)[:, None] + 0.1 * torch.randn(H, rows, D, generator=g)).to(dtype)
    K = K.view(B, H, rows, D)
    V = torch.randn(B, H, rows, D, generator=g).to(dtype)
    p = kvm.make_params(B, H, H, 1, D, dtype)
    O, lse = torch.empty(B, H, n_q, D, dtype=dtype, device="cuda"), torch.empty(B, H, n_q, device="cuda")
    ws = torch.empty(kvm.kvm_cross_workspace_bytes(p, n_q, rows), dtype=torch.uint8, device="cuda")
    kvm.kvm_cross_attend(p, Q.cuda(), K.cuda(), V.cuda(), None, O, lse, ws)
    for h in range(H):
        ref = Rows(Q[0, h], K[0, h], V[0, h], 1.0 / math.sqrt(D))
        close(O[0, h], ref.O, ref.O_bound(dtype), h)
        close(lse[0, h], ref.lse, ref.lse_bound(), h)


@pytest.mark.parametrize("B,Hq,Hkv,n_q,rows,D", [
    (2, 8, 4, 20, 100, 64),               # the rows of a unit in one tile, its keys in one piece
    (2, 8, 4, 20, 128, 128),
    (1, 2, 1, 45, 1, 128),                # a tile and a bit
    (37, 8, 8, 64, 300, 128),             # as many blocks as run at a time: longer caches stay in one piece
    (37, 12, 12, 40, 260, 64),
    (5, 8, 8, 3, 120, 128),               # few rows
    (3, 8, 2, 4, 90, 64),
])
def test_fp32_in_place_with_the_keys_in_one_piece(B, Hq, Hkv, n_q, rows, D):
    """Nothing is joined by a second kernel: the one that attends reads O_in and lse_in and overwrites them."""
    p = kvm.make_params(B, Hq, Hkv, 1, D, torch.float32)
    assert kvm.kvm_cross_workspace_bytes(p, n_q, rows) <= 256          # no states
    for lengths in ("ragged", None):
        check(B, Hq, Hkv, n_q, rows, D, torch.float32, join=True, in_place=True, lengths=lengths)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("B,Hq,Hkv,n_q,rows,D", [
    (1, 4, 2, 60, 3000, 128),             # few items in many pieces: a block joins a row
    (3, 4, 4, 300, 4000, 64),             # a warp for each of a block's four rows
    (13, 16, 16, 150, 2700, 64),          # many items: sixteen rows a block
])
def test_in_place_joined_by_a_second_kernel(B, Hq, Hkv, n_q, rows, D, dtype):
    check(B, Hq, Hkv, n_q, rows, D, dtype, join=True, in_place=True)


@pytest.mark.parametrize("B,Hq,Hkv,n_q,rows,D,dtype", [
    (1, 4, 2, 40, 300, 128, torch.bfloat16),      # items stay whole
    (1, 4, 2, 150, 6000, 128, torch.bfloat16),    # items are cut
    (1, 5, 5, 9, 24000, 64, torch.bfloat16),      # two states to a piece
    (1, 4, 2, 40, 100, 64, torch.float32),        # one piece, several; few rows the same
    (1, 4, 2, 40, 3000, 128, torch.float32),
    (1, 4, 2, 3, 100, 64, torch.float32),
    (1, 4, 2, 3, 3000, 64, torch.float32),
])
@pytest.mark.parametrize("in_place", [False, True])
def test_a_mark_of_what_gave_up_stays(B, Hq, Hkv, n_q, rows, D, dtype, in_place):
    """lse_in is NaN where the attention that is joined in gave up: so are O and lse then, and a unit without keys passes both on as they are."""
    g = torch.Generator().manual_seed(41)
    G = Hq // Hkv
    p = kvm.make_params(B, Hq, Hkv, 1, D, dtype)
    Q = torch.randn(B, Hq, n_q, D, generator=g).to(dtype)
    K, V = (torch.randn(B, Hkv, rows, D, generator=g).to(dtype) for _ in range(2))
    ln = torch.full((B, Hkv), rows, dtype=torch.int32)
    ln[0, 0] = 0
    O_in, lse_in = torch.randn(B, Hq, n_q, D, generator=g).to(dtype), math.log(rows) + torch.randn(B, Hq, n_q, generator=g)
    lse_in[:, :, :2] = math.nan
    O_in[:, :, 0] = math.nan
    a, b = O_in.cuda(), lse_in.cuda()
    O, lse = (a, b) if in_place else (torch.zeros_like(a), torch.zeros_like(b))
    ws = torch.empty(kvm.kvm_cross_workspace_bytes(p, n_q, rows), dtype=torch.uint8, device="cuda")
    kvm.kvm_cross_attend(p, Q.cuda(), K.cuda(), V.cuda(), ln.cuda(), O, lse, ws, O_in=a, lse_in=b)
    O, lse = O.cpu(), lse.cpu()
    for h in range(Hq):
        if h < G:
            assert torch.equal(O[0, h].nan_to_num(7.0), O_in[0, h].nan_to_num(7.0)) and torch.equal(lse[0, h].nan_to_num(7.0), lse_in[0, h].nan_to_num(7.0))
        else:
            assert O[0, h, :2].isnan().all() and lse[0, h, :2].isnan().all()
            ref = Rows(Q[0, h], K[0, h // G], V[0, h // G], 1.0 / math.sqrt(D)).joined(O_in[0, h], lse_in[0, h])
            close(O[0, h, 2:], ref.O[2:], ref.O_bound(dtype)[2:], h)
            close(lse[0, h, 2:], ref.lse[2:], ref.lse_bound()[2:], h)


@pytest.mark.parametrize("n_q,D", [(512, 128), (768, 64)])
def test_fp32_long_sums_do_not_lose_on_one_side(n_q, D):
    """Many keys in one piece, values of one sign, logits near zero: errors of single additions have to cancel.
    O is a sum of N = rows / 16 terms, rounded after each addition by at most 2^-24 of the running sum.  Rounded to the nearest, these errors
    are independent and uniform: together a standard deviation of 2^-24 sqrt(N) / 3 of the whole; six of them are 2^-23 sqrt(N).
    Beside that 2^-21 for the logits and their exponentials (all below 1), twice (numerator and denominator), 17 roundings of 2^-24 within a term's
    products, the value's planes, the division and the store, 2^-24 each: below 2^-19.  (Losing half a step of 2^-24 at each of six products a term
    instead would be 2^-25 * 6 N / 2 = 1.1e-4 here.)"""
    H, rows = 37, 20000
    g = torch.Generator().manual_seed(51)
    p = kvm.make_params(1, H, H, 1, D, torch.float32)
    assert kvm.kvm_cross_workspace_bytes(p, n_q, rows) <= 256
    Q = 0.05 * torch.randn(1, H, n_q, D, generator=g)
    K, V = (torch.randn(1, H, rows, D, generator=g) for _ in range(2))
    V = V.abs() + 0.5
    O, lse = torch.empty_like(Q, device="cuda"), torch.empty(1, H, n_q, device="cuda")
    ws = torch.empty(kvm.kvm_cross_workspace_bytes(p, n_q, rows), dtype=torch.uint8, device="cuda")
    kvm.kvm_cross_attend(p, Q.cuda(), K.cuda(), V.cuda(), None, O, lse, ws)
    for h in (0, 17, 36):
        ref = Rows(Q[0, h], K[0, h], V[0, h], 1.0 / math.sqrt(D))
        close(O[0, h], ref.O, ref.O * (2.0 ** -19 + 2.0 ** -23 * math.sqrt(rows / 16)), h)
        close(lse[0, h], ref.lse, ref.lse_bound(), h)


@pytest.mark.parametrize("B,Hq,Hkv,n_q,rows,D", [(1, 2, 1, 40, 300, 64), (1, 4, 2, 150, 6000, 128), (1, 5, 5, 9, 24000, 64), (1, 2, 1, 3, 90, 128)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_logits_far_below_zero(B, Hq, Hkv, n_q, rows, D, dtype):
    """Logits of -1e31 and -2e31: numbers like others, of which the larger takes all the weight.  (On the tensor cores, whose multiply-adds bear
    references up to 2^27, a row may be NaN instead, as documented, but nothing else.)"""
    g = torch.Generator().manual_seed(61)
    p = kvm.make_params(B, Hq, Hkv, 1, D, dtype, softmax_scale=0.125)
    Q, K = torch.zeros(B, Hq, n_q, D), torch.zeros(B, Hkv, rows, D)
    Q[..., 5], K[..., 5] = 1e16, -1.6e16
    top = torch.randint(0, rows, (Hkv,), generator=g)
    for h in range(Hkv):
        K[0, h, top[h], 5] = -8e15
    Q, K, V = Q.to(dtype), K.to(dtype), torch.randn(B, Hkv, rows, D, generator=g).to(dtype)
    O, lse = torch.empty(B, Hq, n_q, D, dtype=dtype, device="cuda"), torch.empty(B, Hq, n_q, device="cuda")
    ws = torch.empty(kvm.kvm_cross_workspace_bytes(p, n_q, rows), dtype=torch.uint8, device="cuda")
    kvm.kvm_cross_attend(p, Q.cuda(), K.cuda(), V.cuda(), None, O, lse, ws)
    for h in range(Hq):
        u = h // (Hq // Hkv)
        want = 0.125 * float(Q[0, h, 0, 5].double() * K[0, u, top[u], 5].double())
        if dtype == torch.bfloat16:
            gone = O[0, h].cpu().isnan().all(-1)
            assert torch.equal(gone, lse[0, h].cpu().isnan()) and torch.equal(gone, O[0, h].cpu().isnan().any(-1))
            O[0, h][gone.cuda()], lse[0, h][gone.cuda()] = V[0, u, top[u]].cuda(), want
        # one weight of 1; an fp32 value is the sum of its three planes, off by 2^-26; the logit rounds a handful of times
        assert bool(((O[0, h].cpu().double() - V[0, u, top[u]].double()).abs() <= 2.0 ** -24 * V[0, u, top[u]].double().abs()).all()), h
        assert bool(((lse[0, h].cpu().double() - want).abs() <= 2.0 ** -20 * abs(want)).all()), h


@pytest.mark.parametrize("size", [2.0 ** 10, 2.0 ** 20, 2.0 ** 25])
@pytest.mark.parametrize("sign", [-1.0, 1.0])
def test_logits_of_some_size(size, sign):
    """bf16 on the tensor cores: logits around +-size, one ahead of the others by more than half its size."""
    B, H, n_q, rows, D = 1, 2, 140, 700, 64
    g = torch.Generator().manual_seed(63)
    p = kvm.make_params(B, H, H, 1, D, torch.bfloat16, softmax_scale=0.5)
    Q, K = torch.zeros(B, H, n_q, D), torch.zeros(B, H, rows, D)
    Q[..., 7], K[..., 7] = 2.0 * size, sign if sign < 0 else 0.25
    top = torch.randint(0, rows, (H,), generator=g)
    for h in range(H):
        K[0, h, top[h], 7] = -0.4375 if sign < 0 else 1.0
    Q, K, V = Q.bfloat16(), K.bfloat16(), torch.randn(B, H, rows, D, generator=g).bfloat16()
    O, lse = torch.empty(B, H, n_q, D, dtype=torch.bfloat16, device="cuda"), torch.empty(B, H, n_q, device="cuda")
    ws = torch.empty(kvm.kvm_cross_workspace_bytes(p, n_q, rows), dtype=torch.uint8, device="cuda")
    kvm.kvm_cross_attend(p, Q.cuda(), K.cuda(), V.cuda(), None, O, lse, ws)
    for h in range(H):
        want = size * (-0.4375 if sign < 0 else 1.0)
        # (the reference may be off by half a step of the logit, by at most 2 here: the weight divides by itself)
        assert torch.equal(O[0, h].cpu(), V[0, h, top[h]].expand(n_q, D)), h
        assert bool(((lse[0, h].cpu().double() - want).abs() <= 2.0 ** -21 * abs(want)).all()), h
