"""Host side of the serving operators: refusals before anything is enqueued, workspace sizes, the rotation's frequencies."""
import ctypes
import math

import pytest
import torch

import paper_2407_08454_b200 as kvm
from paper_2407_08454_b200 import binding

NULL, SHAPE, DTYPE, PARAM, ALIGN, WORKSPACE = -1, -2, -3, -4, -5, -6
vp = ctypes.c_void_p
OK, OFF = vp(4096), vp(4097)           # never dereferenced: the checks come first


@pytest.fixture(scope="module")
def lib(kvm_lib):
    return kvm_lib


def params(**kw):
    base = dict(batch=2, n_q_heads=8, n_kv_heads=4, seq=1, head_dim=128, dtype=kvm.KVM_BF16)
    base.update(kw)
    return kvm.make_params(**base)


def pages(**kw):
    base = dict(K=4096, V=4096, table=4096, len=4096, n_pages=64, page_rows=16, max_pages=8, reserved=0)
    base.update(kw)
    return kvm.KvmPages(**base)


def test_frequencies_are_exact_binary_fractions(lib):
    for D in (64, 128):
        for base in (10000.0, 500000.0, 1e6):
            t = kvm.rope_turns(D, base, device="cpu")
            for i in range(D // 2):
                want = base ** (-2.0 * i / D) / (2.0 * math.pi)
                got = (int(t[i]) & (2 ** 64 - 1)) / 2.0 ** 64
                # (units of 2^-64, cut off; pow and the division round a few times to 53 bits)
                assert abs(got - want) <= 2.0 ** -50 * want + 2.0 ** -64
    n = (ctypes.c_uint64 * 64)()
    assert lib.kvm_rope_turns(ctypes.c_int32(96), ctypes.c_double(1e4), n) == SHAPE
    assert lib.kvm_rope_turns(ctypes.c_int32(128), ctypes.c_double(1e4), None) == NULL
    for bad in (1.0, 0.0, -3.0, float("nan"), float("inf")):
        assert lib.kvm_rope_turns(ctypes.c_int32(128), ctypes.c_double(bad), n) == PARAM


def append(lib, p, c, len_out=OK, n_new=3, pos=OK, turns=OK, layout=0, q=OK, k=OK, v=OK, strides=None, q_out=OK):
    s = None if strides is None else (ctypes.c_int64 * 9)(*strides)
    return lib.kvm_paged_append(None if p is None else ctypes.byref(p), None if c is None else ctypes.byref(c), len_out,
                                ctypes.c_int32(n_new), vp(0), pos, turns, ctypes.c_int32(layout), q, k, v, s, q_out, vp(0), vp(0))


@pytest.mark.parametrize("kw,want", [
    (dict(p=None), NULL), (dict(c=None), NULL), (dict(len_out=vp(0)), NULL), (dict(k=vp(0)), NULL), (dict(v=vp(0)), NULL),
    (dict(pos=vp(0)), NULL), (dict(q=vp(0)), NULL), (dict(q_out=vp(0)), NULL),
    (dict(n_new=0), SHAPE), (dict(n_new=(1 << 24) + 1), SHAPE), (dict(layout=2), PARAM),
    (dict(q=OFF), ALIGN), (dict(k=OFF), ALIGN), (dict(v=OFF), ALIGN), (dict(q_out=OFF), ALIGN), (dict(turns=vp(4100)), ALIGN),
    (dict(pos=OFF), ALIGN), (dict(len_out=OFF), ALIGN),
    (dict(strides=[128, 128, 128, 4, 128, 128, 128, 128, 128]), ALIGN), (dict(strides=[128] * 8 + [-128]), PARAM),
    (dict(p=params(dtype=5)), DTYPE), (dict(p=params(head_dim=96)), SHAPE), (dict(p=params(n_q_heads=6)), SHAPE),
    (dict(p=params(batch=0)), SHAPE), (dict(p=params(batch=65536)), SHAPE), (dict(p=params(softmax_scale=float("nan"))), PARAM),
    (dict(c=pages(K=0)), NULL), (dict(c=pages(V=0)), NULL), (dict(c=pages(table=0)), NULL), (dict(c=pages(len=0)), NULL),
    (dict(c=pages(K=4104)), ALIGN), (dict(c=pages(table=4098)), ALIGN),
    (dict(c=pages(page_rows=8)), SHAPE), (dict(c=pages(page_rows=48)), SHAPE), (dict(c=pages(page_rows=8192)), SHAPE),
    (dict(c=pages(n_pages=0)), SHAPE), (dict(c=pages(max_pages=0)), SHAPE), (dict(c=pages(max_pages=(1 << 20) + 1)), SHAPE),
    (dict(c=pages(reserved=1)), PARAM),
])
def test_append_refusals(lib, kw, want):
    args = dict(p=params(), c=pages())
    args.update(kw)
    assert append(lib, args.pop("p"), args.pop("c"), **args) == want


def shared(lib, p, q=OK, K=OK, V=OK, rows=100, ln=vp(0), own=None, out=OK, ws=OK, n=1 << 40):
    return lib.kvm_shared_attend(ctypes.byref(p), q, K, V, ctypes.c_int32(rows), ln, None if own is None else ctypes.byref(own), out,
                                 vp(0), ws, ctypes.c_size_t(n), vp(0))


@pytest.mark.parametrize("kw,want", [
    (dict(q=vp(0)), NULL), (dict(out=vp(0)), NULL), (dict(K=vp(0)), NULL), (dict(V=vp(0)), NULL),
    (dict(K=vp(0), V=vp(0), rows=0), NULL),                                   # neither prefix nor own rows
    (dict(rows=0), SHAPE), (dict(rows=(1 << 24) + 1), SHAPE), (dict(K=vp(0), V=vp(0), rows=5, own=pages()), SHAPE),
    (dict(q=OFF), ALIGN), (dict(out=OFF), ALIGN), (dict(K=OFF), ALIGN), (dict(V=OFF), ALIGN), (dict(ln=OFF), ALIGN),
    (dict(ws=vp(0)), WORKSPACE), (dict(n=100), WORKSPACE), (dict(ws=vp(4104)), ALIGN),
    (dict(own=pages(page_rows=24)), SHAPE), (dict(own=pages(len=0)), NULL), (dict(p=params(head_dim=32)), SHAPE),
])
def test_shared_refusals(lib, kw, want):
    args = dict(p=params(), own=pages())
    if "own" not in kw and kw.get("rows") == 0 and "K" in kw:
        args["own"] = None
    args.update(kw)
    assert shared(lib, args.pop("p"), **args) == want


def cross(lib, p, Q=OK, n_q=7, K=OK, V=OK, rows=100, ln=vp(0), O_in=vp(0), lse_in=vp(0), O=OK, lse=OK, ws=OK, n=1 << 40):
    return lib.kvm_cross_attend(ctypes.byref(p), Q, ctypes.c_int32(n_q), K, V, ctypes.c_int32(rows), ln, O_in, lse_in, O, lse, vp(0), ws,
                                ctypes.c_size_t(n), vp(0))


@pytest.mark.parametrize("kw,want", [
    (dict(Q=vp(0)), NULL), (dict(K=vp(0)), NULL), (dict(V=vp(0)), NULL), (dict(O=vp(0)), NULL), (dict(lse=vp(0)), NULL),
    (dict(O_in=OK), NULL), (dict(lse_in=OK), NULL),
    (dict(n_q=0), SHAPE), (dict(n_q=65537), SHAPE), (dict(rows=0), SHAPE), (dict(rows=(1 << 24) + 1), SHAPE),
    (dict(p=params(batch=1, n_q_heads=32768, n_kv_heads=1), n_q=65536), SHAPE),
    (dict(Q=OFF), ALIGN), (dict(K=OFF), ALIGN), (dict(V=OFF), ALIGN), (dict(O=OFF), ALIGN), (dict(lse=OFF), ALIGN), (dict(ln=OFF), ALIGN),
    (dict(O_in=OFF, lse_in=OK), ALIGN), (dict(O_in=OK, lse_in=OFF), ALIGN),
    (dict(ws=vp(0)), WORKSPACE), (dict(n=100), WORKSPACE), (dict(ws=vp(4104)), ALIGN), (dict(p=params(dtype=-1)), DTYPE),
])
def test_cross_refusals(lib, kw, want):
    args = dict(p=params())
    args.update(kw)
    assert cross(lib, args.pop("p"), **args) == want


def test_workspace_queries(lib):
    p = params()
    assert kvm.kvm_cross_workspace_bytes(p, 7, 100) > 0
    assert kvm.kvm_shared_workspace_bytes(p, 100, None) > 0
    assert kvm.kvm_shared_workspace_bytes(p, 0, pages(K=0, V=0, table=0, len=0)) > 0         # sizes are enough
    n = ctypes.c_size_t()
    assert lib.kvm_shared_workspace_bytes(ctypes.byref(p), ctypes.c_int32(0), None, ctypes.byref(n)) == SHAPE
    assert lib.kvm_cross_workspace_bytes(ctypes.byref(p), ctypes.c_int32(7), ctypes.c_int32(100), None) == NULL
    assert lib.kvm_cross_workspace_bytes(ctypes.byref(p), ctypes.c_int32(0), ctypes.c_int32(100), ctypes.byref(n)) == SHAPE
    # budget, rules and seq do not matter to these operators
    odd = params(seq=0, budget=0.0, causal=0)
    assert kvm.kvm_cross_workspace_bytes(odd, 7, 100) == kvm.kvm_cross_workspace_bytes(p, 7, 100)


def test_the_binding_refuses_tensors_of_another_shape_type_or_device():
    p = params(dtype=torch.float32, head_dim=64)
    x = torch.zeros(2, 8, 7, 64)
    with pytest.raises(ValueError):                  # not a CUDA tensor
        kvm.kvm_cross_attend(p, x, x[:, :4], x[:, :4], None, x, x[..., 0], x)
    with pytest.raises(ValueError):
        kvm.make_pages(torch.zeros(4, 16, 64), torch.zeros(4, 16, 64), torch.zeros(2, 2, dtype=torch.int32), torch.zeros(2, dtype=torch.int32))
    assert "page" in kvm.status_string(kvm.KVM_E_PAGE)
    assert binding.KVM_E_PAGE == -11


class Elsewhere(torch.Tensor):
    """A tensor that says it is on another device than those beside it."""
    def get_device(self):
        return 5


def test_the_binding_refuses_workspaces_and_stats_of_another_device_or_size(monkeypatch):
    """(With CPU tensors taken for ones of the current device, and the library's entry points for a list of what reached them.)"""
    reached = []
    monkeypatch.setattr(binding, "_on", lambda t: t.get_device())
    monkeypatch.setattr(binding, "_call", lambda name, *args: reached.append(name))
    monkeypatch.setattr(binding, "_stream", lambda stream: 0)
    p = params(dtype=torch.float32, head_dim=64)
    Q, K, lse, ws = torch.zeros(2, 8, 7, 64), torch.zeros(2, 4, 9, 64), torch.zeros(2, 8, 7), torch.zeros(4096, dtype=torch.uint8)
    stats = kvm.new_stats("cpu")
    cache = pages()
    cache.of = (-1, 8, 64, torch.float32)
    length = torch.zeros(8, dtype=torch.int32)
    calls = {
        "kvm_cross_attend": lambda ws, stats: kvm.kvm_cross_attend(p, Q, K, K, None, Q, lse, ws, stats=stats),
        "kvm_shared_attend": lambda ws, stats: kvm.kvm_shared_attend(p, Q[:, :, 0].contiguous(), K[0], K[0], None, None, Q[:, :, 0].contiguous(), ws, stats=stats),
        "kvm_paged_append": lambda ws, stats: kvm.kvm_paged_append(p, cache, None, None, None, K, K, None, length, stats=stats),
    }
    for name, call in calls.items():
        call(ws, stats)
        call(ws, None)
        assert reached == [name, name]
        for bad in (stats.as_subclass(Elsewhere), stats[:-1], torch.zeros(64, dtype=torch.uint8)[::2]):
            with pytest.raises(ValueError):
                call(ws, bad)
        if name != "kvm_paged_append":
            for bad in (ws.as_subclass(Elsewhere), ws[::2]):
                with pytest.raises(ValueError):
                    call(bad, None)
            call(None, None)                          # (the library answers that: no workspace)
            reached.pop()
        assert reached == [name, name]
        reached.clear()


def test_misaligned_stats_are_refused(lib):
    """(Without the check a kernel that reports something stores a word at such an address.)"""
    p, c = params(), pages()
    assert lib.kvm_paged_append(ctypes.byref(p), ctypes.byref(c), OK, ctypes.c_int32(1), vp(0), OK, OK, ctypes.c_int32(0), OK, OK, OK, None, OK,
                                vp(4098), vp(0)) == ALIGN
    assert lib.kvm_shared_attend(ctypes.byref(p), OK, OK, OK, ctypes.c_int32(10), vp(0), ctypes.byref(c), OK, vp(4098), vp(0), ctypes.c_size_t(0),
                                 vp(0)) == ALIGN
    assert lib.kvm_cross_attend(ctypes.byref(p), OK, ctypes.c_int32(3), OK, OK, ctypes.c_int32(10), vp(0), vp(0), vp(0), OK, OK, vp(4098), vp(0),
                                ctypes.c_size_t(0), vp(0)) == ALIGN
