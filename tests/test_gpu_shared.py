"""kvm_shared_attend against 64 bits: prefix and own rows, either alone, ragged and empty units, rows past the lengths NaN."""
import math

import pytest
import torch

import paper_2407_08454_b200 as kvm
from serve_ref import Rows, close, make_cache, page_rows_of

pytestmark = pytest.mark.gpu


def ragged(g, shape, top, zero_at=None):
    n = torch.randint(0, top + 1, shape, generator=g, dtype=torch.int32)
    n.view(-1)[-1] = top
    if zero_at is not None:
        n.view(-1)[zero_at] = 0
    return n


def check(B, Hq, Hkv, D, prefix, held, R, dtype, scale=0.0, lengths=None, pre_len=None, full_prefix=False, seed=0):
    g = torch.Generator().manual_seed(seed + B * 31 + Hq * 7 + prefix + held)
    G = Hq // Hkv
    p = kvm.make_params(B, Hq, Hkv, 1, D, dtype, softmax_scale=scale)
    sc = scale if scale > 0 else 1.0 / math.sqrt(D)
    q = (2.0 * torch.randn(B, Hq, D, generator=g)).to(dtype)
    Kp = Vp = own = None
    if prefix:
        Kp, Vp = (torch.randn(Hkv, prefix, D, generator=g).to(dtype) for _ in range(2))
        if full_prefix:
            pre_len = torch.full((Hkv,), prefix, dtype=torch.int32)
        else:
            pre_len = ragged(g, (Hkv,), prefix, 0 if Hkv > 1 else None) if pre_len is None else pre_len
            for h in range(Hkv):
                Kp[h, int(pre_len[h]):] = math.nan
                Vp[h, int(pre_len[h]):] = math.inf
    if held:
        lengths = ragged(g, (B, Hkv), held, 1 % (B * Hkv - 1) if B * Hkv > 1 else None) if lengths is None else lengths
        K, V, table = make_cache(g, B, Hkv, D, R, lengths, dtype, spare=2)
        own = kvm.make_pages(K.cuda(), V.cuda(), table.cuda(), lengths.cuda())
    ws = torch.full((kvm.kvm_shared_workspace_bytes(p, prefix, own),), 255, dtype=torch.uint8, device="cuda")     # (NaN patterns)
    out = torch.full((B, Hq, D), math.nan, dtype=dtype, device="cuda")
    stats = kvm.new_stats("cuda")
    kvm.kvm_shared_attend(p, q.cuda(), None if Kp is None else Kp.cuda(), None if Kp is None else Vp.cuda(),
                          None if Kp is None or full_prefix else pre_len.cuda(), own, out, ws, stats=stats)
    assert kvm.read_stats(stats).status == 0
    again = torch.empty_like(out)
    kvm.kvm_shared_attend(p, q.cuda(), None if Kp is None else Kp.cuda(), None if Kp is None else Vp.cuda(),
                          None if Kp is None or full_prefix else pre_len.cuda(), own, again, ws)
    assert torch.equal(out, again)                         # the same bits every time
    for b in range(B):
        for h in range(Hkv):
            Ks, Vs = [q.new_zeros(0, D)], [q.new_zeros(0, D)]
            if prefix:
                n = int(pre_len[h])
                Ks.append(Kp[h, :n]); Vs.append(Vp[h, :n])
            if held:
                n = int(lengths[b, h])
                Ks.append(page_rows_of(K, table[b * Hkv + h], n)); Vs.append(page_rows_of(V, table[b * Hkv + h], n))
            ref = Rows(q[b, h * G:(h + 1) * G], torch.cat(Ks), torch.cat(Vs), sc)
            close(out[b, h * G:(h + 1) * G], ref.O, ref.O_bound(dtype), (b, h))


SHAPES = [
    # B, Hq, Hkv, D, prefix, held, R
    (1, 1, 1, 128, 0, 1, 16),
    (1, 4, 4, 64, 0, 17, 16),
    (2, 8, 2, 128, 0, 300, 16),
    (3, 6, 2, 64, 0, 129, 32),
    (2, 18, 2, 128, 0, 77, 64),            # nine heads share a row
    (1, 24, 2, 64, 0, 200, 16),            # twelve
    (2, 40, 1, 128, 0, 65, 128),           # forty
    (1, 4, 2, 128, 1, 0, 16),
    (4, 8, 8, 128, 127, 0, 16),
    (2, 8, 4, 64, 128, 0, 16),
    (7, 12, 4, 128, 513, 0, 16),
    (3, 8, 2, 128, 200, 40, 16),
    (16, 16, 2, 128, 300, 33, 16),         # 128 query rows a head
    (17, 16, 2, 64, 300, 33, 32),          # 136
    (33, 32, 4, 128, 140, 5, 16),          # 264
    (5, 40, 2, 64, 260, 50, 16),           # blocks of twenty rows
    (2, 136, 1, 128, 150, 20, 16),         # a block of more than 128 rows
    (9, 3, 3, 128, 1000, 100, 64),
    (2, 4, 4, 128, 0, 1500, 16),           # units in parts
    (40, 8, 8, 64, 0, 700, 32),            # a block per unit, and some
    (50, 18, 18, 64, 0, 20, 16),           # more units than blocks at a time
    (20, 64, 16, 64, 2500, 10, 16),        # more steps over the prefix than SMs
]


# Batches for which the prefix has a kernel of its own (reading it again for every sequence would cost more): tiles of query rows that hold
# whole blocks of heads or a part of one, one tile, a pair, several; with and without own rows beside it.
LARGE = [
    (64, 40, 2, 128, 200, 33, 16),
    (16, 136, 1, 128, 400, 20, 16),
    (70, 32, 4, 128, 300, 17, 32),
    (100, 12, 3, 64, 600, 40, 16),
    (130, 6, 2, 128, 300, 0, 16),
    (40, 4, 4, 128, 1700, 30, 16),         # one tile of 40 rows, pieces of several steps
    (33, 8, 8, 64, 2100, 5, 64),
    (128, 1, 1, 128, 530, 12, 16),         # exactly one tile
]


@pytest.mark.parametrize("B,Hq,Hkv,D,prefix,held,R", SHAPES + LARGE)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_shared_matches_64_bits(B, Hq, Hkv, D, prefix, held, R, dtype):
    check(B, Hq, Hkv, D, prefix, held, R, dtype)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_full_prefix_without_lengths_and_a_scale_of_its_own(dtype):
    check(3, 8, 4, 128, 333, 21, 16, dtype, scale=0.03, full_prefix=True)
    check(2, 8, 4, 64, 4097, 0, 16, dtype, full_prefix=True)                  # many pieces to join


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("prefix", [0, 64])
def test_sequences_without_any_rows_give_zeros(dtype, prefix):
    B, Hkv = 3, 2
    none = torch.zeros(B, Hkv, dtype=torch.int32)
    none[1, 1] = 20
    check(B, 4, Hkv, 128, prefix, 20, 16, dtype, lengths=none, pre_len=torch.tensor([0, 0], dtype=torch.int32))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_logits_far_apart(dtype):
    """A row that outweighs everything before it by far, in each part, and values of large size beside it."""
    g = torch.Generator().manual_seed(1)
    B, H, D, P, n = 2, 2, 128, 700, 90
    p = kvm.make_params(B, H, H, 1, D, dtype)
    q = torch.randn(B, H, D, generator=g).to(dtype)
    Kp, Vp = (torch.randn(H, P, D, generator=g).to(dtype) for _ in range(2))
    lengths = torch.full((B, H), n, dtype=torch.int32)
    K, V, table = make_cache(g, B, H, D, 16, lengths, dtype)
    Kp[0, 650] = (30.0 * q[0, 0].float()).to(dtype)
    K[int(table[3, 5]), 3] = (30.0 * q[1, 1].float()).to(dtype)
    Vp[0, 10] = 1e4
    own = kvm.make_pages(K.cuda(), V.cuda(), table.cuda(), lengths.cuda())
    out = torch.empty(B, H, D, dtype=dtype, device="cuda")
    ws = torch.empty(kvm.kvm_shared_workspace_bytes(p, P, own), dtype=torch.uint8, device="cuda")
    kvm.kvm_shared_attend(p, q.cuda(), Kp.cuda(), Vp.cuda(), None, own, out, ws)
    for b in range(B):
        for h in range(H):
            ref = Rows(q[b, h:h + 1], torch.cat([Kp[h], page_rows_of(K, table[b * H + h], n)]),
                       torch.cat([Vp[h], page_rows_of(V, table[b * H + h], n)]), 1.0 / math.sqrt(D))
            close(out[b, h:h + 1], ref.O, ref.O_bound(dtype), (b, h))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_rows_on_missing_pages_do_not_exist_and_are_reported(dtype):
    g = torch.Generator().manual_seed(2)
    B, H, D, R = 2, 1, 64, 16
    lengths = torch.tensor([[50], [40]], dtype=torch.int32)
    K, V, table = make_cache(g, B, H, D, R, lengths, dtype)
    broken = table.clone()
    broken[0, 1] = K.shape[0]                              # the first number past the pool
    broken[0, 3] = -1
    p = kvm.make_params(B, 4, H, 1, D, dtype)
    q = torch.randn(B, 4, D, generator=g).to(dtype)
    own = kvm.make_pages(K.cuda(), V.cuda(), broken.cuda(), lengths.cuda())
    out, stats = torch.empty(B, 4, D, dtype=dtype, device="cuda"), kvm.new_stats("cuda")
    ws = torch.empty(kvm.kvm_shared_workspace_bytes(p, 0, own), dtype=torch.uint8, device="cuda")
    kvm.kvm_shared_attend(p, q.cuda(), None, None, None, own, out, ws, stats=stats)
    assert kvm.read_stats(stats).status == kvm.KVM_E_PAGE
    for b in range(B):
        rows = [r for r in range(int(lengths[b, 0])) if 0 <= int(broken[b, r // R]) < K.shape[0]]
        Kb, Vb = (x[[int(broken[b, r // R]) for r in rows], [r % R for r in rows]] for x in (K, V))
        ref = Rows(q[b], Kb, Vb, 1.0 / math.sqrt(D))
        close(out[b], ref.O, ref.O_bound(dtype), b)


def test_lengths_outside_the_room_are_clamped():
    g = torch.Generator().manual_seed(4)
    B, H, D, R = 2, 2, 128, 16
    lengths = torch.full((B, H), 32, dtype=torch.int32)
    K, V, table = make_cache(g, B, H, D, R, lengths, torch.bfloat16)
    p = kvm.make_params(B, H, H, 1, D, torch.bfloat16)
    q = torch.randn(B, H, D, generator=g).bfloat16().cuda()
    Kp, Vp = (torch.randn(H, 40, D, generator=g).bfloat16().cuda() for _ in range(2))
    outs = []
    for own_len, pre_len in ((32, [40, 0]), (1 << 30, [1 << 30, -8])):
        own = kvm.make_pages(K.cuda(), V.cuda(), table.cuda(), torch.full((B, H), own_len, dtype=torch.int32, device="cuda"))
        out = torch.empty(B, H, D, dtype=torch.bfloat16, device="cuda")
        ws = torch.empty(kvm.kvm_shared_workspace_bytes(p, 40, own), dtype=torch.uint8, device="cuda")
        kvm.kvm_shared_attend(p, q, Kp, Vp, torch.tensor(pre_len, dtype=torch.int32, device="cuda"), own, out, ws)
        outs.append(out)
    assert torch.equal(*outs)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("B,Hq,Hkv,D,prefix,held,R", [LARGE[0], LARGE[3], LARGE[6]])
def test_a_large_batch_of_which_a_part_is_empty(B, Hq, Hkv, D, prefix, held, R, dtype):
    """The first step behind a prompt has no own rows yet, beside a prefix with a kernel of its own; or nothing is in the prefix, or in either."""
    own, pre = torch.zeros(B, Hkv, dtype=torch.int32), torch.zeros(Hkv, dtype=torch.int32)
    check(B, Hq, Hkv, D, prefix, held, R, dtype, lengths=own)
    check(B, Hq, Hkv, D, prefix, held, R, dtype, pre_len=pre)
    check(B, Hq, Hkv, D, prefix, held, R, dtype, lengths=own, pre_len=pre)
    own[B // 2, Hkv - 1] = 1                               # a single row
    check(B, Hq, Hkv, D, prefix, held, R, dtype, lengths=own)
    check(B, Hq, Hkv, D, prefix, held, R, dtype, lengths=own, pre_len=pre)


@pytest.mark.parametrize("prefix", [0, 30, 200])           # none, one that is folded in, one with a kernel of its own
def test_more_units_than_keep_their_lengths(prefix):
    check(70, 16, 16, 64, prefix, 40, 16, torch.bfloat16)
    check(70, 32, 16, 128, prefix, 600, 32, torch.bfloat16, lengths=torch.randint(0, 4, (70, 16), generator=torch.Generator().manual_seed(6), dtype=torch.int32) ** 3)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("B,Hq,Hkv,D,prefix,held", [(2, 4, 2, 64, 0, 100), (2, 4, 2, 128, 0, 1500), (3, 4, 2, 128, 60, 40), (64, 40, 2, 128, 200, 33)])
def test_logits_far_below_zero(B, Hq, Hkv, D, prefix, held, dtype):
    """Logits of -1e31 and -2e31: numbers like others, of which the larger takes all the weight.  (Where the prefix has a kernel of its own, on the
    tensor cores, a row may be NaN instead, as documented, but nothing else.)"""
    g = torch.Generator().manual_seed(62)
    G, R = Hq // Hkv, 16
    p = kvm.make_params(B, Hq, Hkv, 1, D, dtype, softmax_scale=0.125)
    lengths = torch.full((B, Hkv), held, dtype=torch.int32)
    K, V, table = make_cache(g, B, Hkv, D, R, lengths, dtype)
    K[:] = 0.0
    K[..., 5] = -1.6e16
    q = torch.zeros(B, Hq, D)
    q[..., 5] = 1e16
    q = q.to(dtype)
    Kp = Vp = None
    if prefix:
        Kp, Vp = torch.zeros(Hkv, prefix, D).to(dtype), torch.randn(Hkv, prefix, D, generator=g).to(dtype)
        Kp[..., 5] = -1.6e16
        Kp[0, prefix // 2, 5] = -8e15                      # head 0's is in the prefix, the others' among their own rows
    want = torch.empty(B, Hq, D, dtype=torch.float64)
    for b in range(B):
        for h in range(Hkv):
            if prefix and h == 0:
                top = Vp[0, prefix // 2]
            else:
                r = int(torch.randint(0, held, (1,), generator=g))
                page = int(table[b * Hkv + h, r // R])
                K[page, r % R, 5] = -8e15
                top = V[page, r % R]
            want[b, h * G:(h + 1) * G] = top.double()
    own = kvm.make_pages(K.cuda(), V.cuda(), table.cuda(), lengths.cuda())
    out = torch.empty(B, Hq, D, dtype=dtype, device="cuda")
    ws = torch.empty(kvm.kvm_shared_workspace_bytes(p, prefix, own), dtype=torch.uint8, device="cuda")
    kvm.kvm_shared_attend(p, q.cuda(), None if Kp is None else Kp.cuda(), None if Kp is None else Vp.cuda(), None, own, out, ws)
    got = out.cpu().double()
    if dtype == torch.bfloat16 and B > 8:
        got = torch.where(got.isnan().all(-1, keepdim=True), want, got)
    assert bool(((got - want).abs() <= 2.0 ** -24 * want.abs()).all())                     # (fp32: three planes, off by 2^-26)
