"""kvm_paged_append against 64 bits: every rotated value, every copied one, and that nothing else changes."""
import pytest
import torch

import paper_2407_08454_b200 as kvm
from serve_ref import F64, HALF_STEP, make_cache, rotate, turns

pytestmark = pytest.mark.gpu

# An angle is an integer product rounded to 24 bits of a half turn: off by at most pi 2^-25 + 2^-31 < 1e-7.  sincospi is good to 2
# units in the last place (2^-22 of at most 1); two products, one of them in a fused multiply-add, round twice more (2^-24 each):
# together below 1e-7 + 2.4e-7 + 1.2e-7 < 5e-7 of |x| + |y|.  The store rounds once more.
ROTATION = 5e-7


def build(g, B, Hq, Hkv, D, T, R, dtype, held, spare=3):
    lengths = torch.randint(0, held + 1, (B, Hkv), generator=g, dtype=torch.int32)
    lengths.view(-1)[0] = 0
    lengths.view(-1)[-1] = held
    K, V, table = make_cache(g, B, Hkv, D, R, lengths, dtype, spare=spare, room=T)
    q, k, v = (torch.randn(B, h, T, D, generator=g).to(dtype) for h in (Hq, Hkv, Hkv))
    pos = torch.randint(0, 1 << 20, (B,), generator=g, dtype=torch.int32)
    return lengths, K, V, table, q, k, v, pos


def expect(lengths, K, V, table, q, k, v, pos, new, R, neighbours, rotated=True):
    B, Hkv, T, D = k.shape
    p = pos[:, None, None].to(F64) + torch.arange(T, dtype=F64)
    tr = turns(D)

    def spin(x):
        return rotate(x.to(F64), p.expand(B, x.shape[1], T), tr, neighbours) if rotated else x.to(F64)

    def mass(x):                                           # |x| + |y| of each pair, at both of its channels
        y = x.to(F64).abs()
        m = y[..., 0::2] + y[..., 1::2] if neighbours else y[..., :D // 2] + y[..., D // 2:]
        return m.repeat_interleave(2, -1) if neighbours else torch.cat([m, m], -1)

    qw, kw = spin(q), spin(k)
    half = HALF_STEP[k.dtype]
    Kw, Vw, Kb = K.to(F64).clone(), V.clone(), torch.zeros(K.shape, dtype=F64)
    out = lengths.clone()
    for b in range(B):
        for h in range(Hkv):
            n, start = int(new[b, h]), int(lengths[b, h])
            for t in range(n):
                page, r = int(table[b * Hkv + h, (start + t) // R]), (start + t) % R
                Kw[page, r], Vw[page, r] = kw[b, h, t], v[b, h, t]
                Kb[page, r] = (ROTATION * mass(k)[b, h, t] + half * kw[b, h, t].abs() * 1.01) if rotated else 0.0
            out[b, h] = start + n
    qb = ROTATION * mass(q) + half * qw.abs() * 1.01 if rotated else torch.zeros_like(qw)
    return qw, qb, Kw, Kb, Vw, out


def within(got, want, bound):
    got = got.cpu().to(F64)
    same = (got.isnan() & want.isnan()) | ((got - want).abs() <= bound)
    assert bool(same.all()), float(((got - want).abs() - bound)[~same].max())


def same_bits(a, b):
    view = torch.int16 if a.dtype == torch.bfloat16 else torch.int32
    assert torch.equal(a.cpu().contiguous().view(view), b.contiguous().view(view))


@pytest.mark.parametrize("B,Hq,Hkv,D,T,R,held", [
    (1, 4, 4, 64, 1, 16, 0),            # the first row of empty units
    (3, 8, 2, 128, 1, 16, 40),
    (2, 4, 4, 128, 37, 16, 31),         # over several pages, starting inside one
    (5, 6, 3, 64, 130, 32, 64),
    (64, 32, 8, 128, 1, 64, 70),
    (1, 40, 1, 64, 3, 128, 5),
])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("neighbours", [False, True])
def test_append_matches_64_bits(B, Hq, Hkv, D, T, R, held, dtype, neighbours):
    g = torch.Generator().manual_seed(B * 1000 + T)
    lengths, K, V, table, q, k, v, pos = build(g, B, Hq, Hkv, D, T, R, dtype, held)
    p = kvm.make_params(B, Hq, Hkv, 1, D, dtype)
    tr = kvm.rope_turns(D)
    ragged = torch.randint(0, T + 1, (B, Hkv), generator=g, dtype=torch.int32)
    for case in ("plain", "ragged", "fused", "in place"):
        new = ragged if case == "ragged" else torch.full((B, Hkv), T, dtype=torch.int32)
        want = expect(lengths, K, V, table, q, k, v, pos, new, R, neighbours)
        Kd, Vd, ln = K.cuda(), V.cuda(), lengths.cuda()
        qd, kd, vd = q.cuda(), k.cuda(), v.cuda()
        if case == "fused":                                # views of one projection's output, with a channel block of someone else's
            qkv = torch.cat([x.transpose(1, 2) for x in (qd, kd, vd, vd)], 2).contiguous()
            qd, kd, vd = (x.transpose(1, 2) for x in qkv.split([Hq, Hkv, Hkv, Hkv], 2)[:3])
            q_out = torch.empty((B, Hq, T, D), dtype=dtype, device="cuda")
        else:
            q_out = qd if case == "in place" else torch.empty_like(qd)
        len_out = ln if case == "in place" else torch.full_like(ln, -99)
        stats = kvm.new_stats("cuda")
        cache = kvm.make_pages(Kd, Vd, table.cuda(), ln)
        kvm.kvm_paged_append(p, cache, pos.cuda(), tr, qd, kd, vd, q_out, len_out, new_len=ragged.cuda() if case == "ragged" else None,
                             interleaved=neighbours, stats=stats)
        assert kvm.read_stats(stats).status == 0
        within(q_out, want[0], want[1])
        within(Kd, want[2], want[3])
        same_bits(Vd, want[4])
        assert torch.equal(len_out.cpu(), want[5]), case
        if case != "in place":
            assert torch.equal(ln.cpu(), lengths)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_rows_move_unrotated_bit_for_bit(dtype):
    """A compressed cache moves into pages: lengths per unit, no rotation, no queries."""
    g = torch.Generator().manual_seed(3)
    B, Hq, Hkv, D, T, R = 2, 4, 2, 128, 53, 16
    lengths, K, V, table, q, k, v, pos = build(g, B, Hq, Hkv, D, T, R, dtype, 20)
    new = torch.tensor([[53, 0], [17, 1]], dtype=torch.int32)
    want = expect(lengths, K, V, table, q, k, v, pos, new, R, False, rotated=False)
    Kd, Vd, ln = K.cuda(), V.cuda(), lengths.cuda()
    p = kvm.make_params(B, Hq, Hkv, 1, D, dtype)
    kvm.kvm_paged_append(p, kvm.make_pages(Kd, Vd, table.cuda(), ln), None, None, None, k.cuda(), v.cuda(), None, ln, new_len=new.cuda())
    within(Kd, want[2], want[3])
    same_bits(Vd, want[4])
    assert torch.equal(ln.cpu(), want[5])


def test_positions_far_out_and_negative():
    B, H, D, T = 4, 2, 128, 2
    g = torch.Generator().manual_seed(9)
    pos = torch.tensor([0, (1 << 27) - 1, -5, 1 << 24], dtype=torch.int32)
    q = torch.randn(B, H, T, D, generator=g)
    k = torch.randn(B, H, T, D, generator=g)
    lengths = torch.zeros(B, H, dtype=torch.int32)
    K, V, table = make_cache(g, B, H, D, 16, lengths, torch.float32, room=T)
    p = kvm.make_params(B, H, H, 1, D, torch.float32)
    q_out, ln = torch.empty(B, H, T, D, device="cuda"), lengths.cuda()
    kvm.kvm_paged_append(p, kvm.make_pages(K.cuda(), V.cuda(), table.cuda(), ln), pos.cuda(), kvm.rope_turns(D), q.cuda(), k.cuda(), k.cuda(),
                         q_out, ln)
    where = pos[:, None, None].to(F64) + torch.arange(T, dtype=F64)
    # (the reference's own angle: a product of 53 bits at 2^27 positions is off by 2^-26 of a turn, 1e-7)
    want = rotate(q.to(F64), where.expand(B, H, T), turns(D), False)
    mass = q.abs().to(F64)[..., :64] + q.abs().to(F64)[..., 64:]
    within(q_out, want, (ROTATION + 1e-7) * torch.cat([mass, mass], -1) + 2.0 ** -24 * want.abs() * 1.01)


def test_rows_without_a_page_are_left_out_and_reported():
    """Bad page numbers, and units that run out of pages: nothing is written for them, the rest is, the status says so."""
    g = torch.Generator().manual_seed(5)
    B, Hq, Hkv, D, T, R = 2, 2, 2, 64, 20, 16
    lengths = torch.tensor([[3, 30], [0, 12]], dtype=torch.int32)
    K, V = (torch.full((8, R, D), 7.0) for _ in range(2))
    table = torch.tensor([[0, 1], [2, 3], [4, 1 << 30], [-1, 5]], dtype=torch.int32)       # two pages: room for 32 rows
    k, v = (torch.randn(B, Hkv, T, D, generator=g) for _ in range(2))
    Kw, Vw = K.clone(), V.clone()
    for u in range(4):
        for t in range(T):
            r = int(lengths.view(-1)[u]) + t
            if r < 32 and 0 <= int(table[u, r // R]) < 8:
                Kw[int(table[u, r // R]), r % R], Vw[int(table[u, r // R]), r % R] = k.view(4, T, D)[u, t], v.view(4, T, D)[u, t]
    Kd, Vd, ln, stats = K.cuda(), V.cuda(), lengths.cuda(), kvm.new_stats("cuda")
    p = kvm.make_params(B, Hq, Hkv, 1, D, torch.float32)
    kvm.kvm_paged_append(p, kvm.make_pages(Kd, Vd, table.cuda(), ln), None, None, None, k.cuda(), v.cuda(), None, ln, stats=stats)
    assert torch.equal(Kd.cpu(), Kw) and torch.equal(Vd.cpu(), Vw)
    assert ln.cpu().tolist() == [[23, 32], [20, 32]]
    assert kvm.read_stats(stats).status == kvm.KVM_E_PAGE


def test_offsets_past_32_bits():
    """The last page of a pool of more than 2^31 elements."""
    D, R = 128, 128
    n_pages = (1 << 31) // (R * D) + 3
    K = torch.empty(n_pages, R, D, dtype=torch.bfloat16, device="cuda")
    V = torch.empty_like(K)
    table = torch.tensor([[n_pages - 1, 0]], dtype=torch.int32, device="cuda")
    ln = torch.tensor([5], dtype=torch.int32, device="cuda")
    K[-1, :5], V[-1, :5] = 1.0, 2.0
    k, v = (torch.randn(1, 1, 2, D, device="cuda").bfloat16() for _ in range(2))
    p = kvm.make_params(1, 1, 1, 1, D, torch.bfloat16)
    cache = kvm.make_pages(K, V, table, ln)
    kvm.kvm_paged_append(p, cache, None, None, None, k, v, None, ln)
    assert torch.equal(K[-1, 5:7], k[0, 0]) and torch.equal(V[-1, 5:7], v[0, 0])
    q, out = torch.zeros(1, 1, D, device="cuda").bfloat16(), torch.empty(1, 1, D, dtype=torch.bfloat16, device="cuda")
    ws = torch.empty(kvm.kvm_shared_workspace_bytes(p, 0, cache), dtype=torch.uint8, device="cuda")
    kvm.kvm_shared_attend(p, q, None, None, None, cache, out, ws)                          # equal weights: the mean of the rows
    want = torch.cat([V[-1, :5], v[0, 0]]).double().mean(0)
    # weights of one seventh rounded to bf16 alike (they cancel against the rounded sum), fp32 sums, one rounding
    assert bool(((out[0, 0].double() - want).abs() <= 2.0 ** -8 * want.abs() * 1.01 + 1e-5).all())


@pytest.mark.parametrize("B,Hq,Hkv,D,dtype", [
    (2000, 32, 8, 128, torch.bfloat16), (1000, 32, 8, 128, torch.float32), (1900, 20, 20, 64, torch.bfloat16), (1600, 36, 36, 64, torch.float32),
])
def test_decode_steps_of_a_large_batch_with_lengths_in_place(B, Hq, Hkv, D, dtype):
    """So many sequences that a block takes several heads of a token, a few at a time, and moves each one's length when its lanes have read it."""
    g = torch.Generator(device="cuda").manual_seed(B)
    U, R, room, steps = B * Hkv, 16, 2, 12
    table = torch.randperm(U * room, generator=g, device="cuda").to(torch.int32).view(U, room)
    pool = [torch.full((U * room, R, D), 7.0, dtype=dtype, device="cuda") for _ in range(2)]
    want = [x.clone() for x in pool]
    length = torch.randint(0, R * room - steps + 1, (U,), generator=g, device="cuda", dtype=torch.int32)
    start = length.clone()
    cache = kvm.make_pages(pool[0], pool[1], table, length)
    p = kvm.make_params(B, Hq, Hkv, 1, D, dtype)
    q = torch.randn(B, Hq, 1, D, generator=g, device="cuda").to(dtype)
    q_out, units = torch.empty_like(q), torch.arange(U, device="cuda")
    for s in range(steps):
        k, v = (torch.randn(B, Hkv, 1, D, generator=g, device="cuda").to(dtype) for _ in range(2))
        kvm.kvm_paged_append(p, cache, None, None, q, k, v, q_out, length)
        rows = (start + s).long()
        page = table[units, rows // R].long()
        want[0][page, rows % R], want[1][page, rows % R] = k.view(U, D), v.view(U, D)
        assert torch.equal(length, start + s + 1)
    assert torch.equal(pool[0], want[0]) and torch.equal(pool[1], want[1]) and torch.equal(q_out, q)


def test_angles_have_more_than_24_bits():
    """fp32 pairs (1, 0), which come out as the cosine and the sine themselves.  sincospi is off by at most one unit in the last place, 2^-24 below 1; the
    angle's last bits are added by one multiply-add, 2^-25; what is left of the angle is below 2^-31 half turns, 2^-29.3: together below 1.6 x 2^-24."""
    B, H, D, T = 16, 2, 128, 64
    g = torch.Generator().manual_seed(71)
    pos = torch.randint(0, 1 << 20, (B,), generator=g, dtype=torch.int32)
    q = torch.zeros(B, H, T, D)
    q[..., :D // 2] = 1.0
    lengths = torch.zeros(B, H, dtype=torch.int32)
    K, V, table = make_cache(g, B, H, D, 16, lengths, torch.float32, room=T)
    p = kvm.make_params(B, H, H, 1, D, torch.float32)
    q_out, ln = torch.empty(B, H, T, D, device="cuda"), lengths.cuda()
    kvm.kvm_paged_append(p, kvm.make_pages(K.cuda(), V.cuda(), table.cuda(), ln), pos.cuda(), kvm.rope_turns(D), q.cuda(), q.cuda(), q.cuda(), q_out, ln)
    where = pos[:, None, None].to(F64) + torch.arange(T, dtype=F64)
    # (the reference's own angle: 2^-53 of up to 2^20 / 2 pi turns, 2^-35)
    want = rotate(q.to(F64), where.expand(B, H, T), turns(D), False)
    within(q_out, want, torch.full_like(want, 1.6 * 2.0 ** -24 + 2.0 ** -32))
