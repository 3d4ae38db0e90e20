"""Distillation operators, what needs no GPU: sizes, refusals before the first HIP call, the binding's own checks,
and the plain forms of the tests against each other (the gradient against differences)."""
import ctypes as C
import os
import subprocess

import numpy as np
import pytest
import torch

import distill_ref as ref


@pytest.fixture(scope="module")
def bpc():
    import paper_2105_07829_amd as bpc
    bpc.lib()
    return bpc


def ru4(x):
    return -(-x // 4) * 4


@pytest.mark.parametrize("k", [1, 3, 4, 5, 64, 1023, 1024])
def test_record_sizes(bpc, k):
    assert bpc.logits_stride(bpc.make_distill(bpc.TOPK, 5000, k)) == 16 + 8 * ru4(k)
    assert bpc.logits_stride(bpc.make_distill(bpc.TOPK16, 5000, k)) == 16 + 4 * ru4(k) + 4 * ru4(-(-k // 2))
    d = bpc.make_distill(bpc.TOPK16, 5000, k)
    assert bpc.logits_message_bytes(d, 7) == 7 * bpc.logits_stride(d)
    assert bpc.logits_message_bytes(d, 0) == 0


def test_the_struct_is_the_headers(bpc):
    assert C.sizeof(bpc.Distill) == 32


def bad_descriptions(bpc):
    m = bpc.make_distill
    yield m(bpc.SIGN, 100, 4)
    yield m(9, 100, 4)
    yield m(bpc.TOPK, 0, 4)
    yield m(bpc.TOPK, 100, 0)
    yield m(bpc.TOPK, 100, 4, tail=2)
    for tau in (0.0, -1.0, float("inf"), float("nan"), 1e-38):
        yield m(bpc.TOPK, 100, 4, temperature=tau)
    yield m(bpc.TOPK, 100, 4, soft_weight=float("nan"))
    yield m(bpc.TOPK, 100, 4, hard_weight=float("inf"))


def calls(L, d, who=("topk", "loss", "grad", "step"), dtype=0, stride=100, rows=8, gstride=100, logits=0x10000, messages=0x20000, labels=0x30000, weight=0x40000,
          loss=0x50000, stats=0x60000, grad=0x70000, ws=0x80000, ws_bytes=1 << 40):
    """Status of the calls `who` on fake addresses: each has to return before it touches them."""
    D = C.byref(d) if d is not None else None
    every = {"topk": lambda: L.bpc_logits_topk(D, logits, dtype, stride, rows, weight, messages, ws, ws_bytes, None),
             "loss": lambda: L.bpc_distill_loss(D, logits, dtype, stride, rows, messages, labels, weight, loss, stats, ws, ws_bytes, None),
             "grad": lambda: L.bpc_distill_grad(D, logits, dtype, stride, rows, messages, labels, weight, stats, grad, gstride, None),
             "step": lambda: L.bpc_distill_step(D, logits, dtype, stride, rows, messages, labels, weight, loss, grad, gstride, ws,
                                                ws_bytes, None)}
    return {name: every[name]() for name in who}


def test_bad_descriptions_are_refused(bpc):
    L = bpc.lib()
    for d in [None, *bad_descriptions(bpc)]:
        assert set(calls(L, d).values()) == {bpc.ERR_INVALID_ARG}
        if d is not None:
            assert bpc.logits_stride(d) == 0 and bpc.logits_message_bytes(d, 3) == 0 and bpc.distill_workspace_bytes(d, 3) == 0


def test_argument_errors_come_before_any_device_work(bpc):
    L = bpc.lib()
    d = bpc.make_distill(bpc.TOPK16, 100, 4)
    inv, ali, uns, wsp = bpc.ERR_INVALID_ARG, bpc.ERR_ALIGNMENT, bpc.ERR_UNSUPPORTED, bpc.ERR_WORKSPACE
    everyone = {"topk", "loss", "grad", "step"}

    def refused(status, who, **kw):
        got = calls(L, d, who, **kw)
        assert set(got.values()) == {status}, (kw, got)

    refused(inv, everyone, dtype=3)
    refused(inv, everyone, stride=99)
    refused(inv, everyone, logits=None)
    refused(inv, everyone, messages=None)
    refused(ali, everyone, logits=0x10002)
    refused(ali, everyone, messages=0x20008)
    refused(ali, everyone, weight=0x40004)
    refused(ali, ("loss", "grad", "step"), labels=0x30008)
    refused(inv, ("loss", "step"), loss=None)
    refused(ali, ("loss", "step"), loss=0x50004)
    refused(ali, ("loss", "grad"), stats=0x60008)
    refused(inv, ("grad",), stats=None)
    refused(inv, ("grad", "step"), grad=None)
    refused(inv, ("grad", "step"), gstride=99)
    refused(uns, ("grad", "step"), gstride=1 << 41)
    refused(ali, ("grad", "step"), grad=0x70002)
    refused(wsp, ("topk", "loss", "step"), ws=None)
    refused(wsp, ("topk", "loss", "step"), ws_bytes=bpc.distill_workspace_bytes(d, 8) - 1)
    refused(ali, ("topk", "loss", "step"), ws=0x80004)
    refused(uns, everyone, rows=1 << 22)
    refused(uns, everyone, stride=1 << 41)
    assert set(calls(L, d, rows=0).values()) == {bpc.OK}
    for big in (bpc.make_distill(bpc.TOPK, (1 << 24) + 1, 4), bpc.make_distill(bpc.TOPK, 100, 1025)):
        assert set(calls(L, big, stride=1 << 25, gstride=1 << 25).values()) == {uns}
        assert bpc.logits_stride(big) == 0 and bpc.distill_workspace_bytes(big, 1) == 0


def test_workspace_grows_with_rows(bpc):
    """A workspace for `rows` rows serves every smaller call, of every type."""
    for vocab in (1, 1000, 50257, 131072, 300001, 1 << 24):
        for k in (1, 100, 1024):
            d = bpc.make_distill(bpc.TOPK, vocab, k)
            sizes = [bpc.distill_workspace_bytes(d, r) for r in (1, 2, 3, 7, 8, 15, 61, 64, 100, 255, 256, 257, 511, 512, 513,
                                                                 1000, 1024, 2047, 4096, 10000, 100000)]
            assert sizes[0] >= 256 and sizes == sorted(sizes)
            assert all(s % 256 == 0 for s in sizes)


@pytest.fixture(scope="module")
def geometry(tmp_path_factory):
    """csrc/distill_geometry.hpp compiled for the host."""
    so = str(tmp_path_factory.mktemp("distill") / "host_distill.so")
    here = os.path.dirname(os.path.abspath(__file__))
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-shared", "-fPIC", "-o", so, os.path.join(here, "host_distill.cpp")], check=True)
    L = C.CDLL(so)
    L.dg_needed.argtypes, L.dg_needed.restype = [C.c_uint64, C.c_uint32, C.c_int, C.c_uint64, C.c_int], C.c_uint64
    L.dg_cut.argtypes = [C.c_uint64, C.c_uint32, C.c_int, C.c_uint64, C.c_int] + [C.c_void_p] * 3
    return L


def test_every_call_fits_its_workspace_and_its_rows(bpc, geometry):
    rs = np.random.default_rng(1)
    chunks, vecs, nv = (C.c_uint32() for _ in range(3))
    for _ in range(3000):
        vocab = int(np.exp(rs.uniform(0, np.log(1 << 24))))
        rows = int(np.exp(rs.uniform(0, np.log((1 << 22) - 1))))
        smaller = int(rs.integers(1, rows + 1))
        size = bpc.distill_workspace_bytes(bpc.make_distill(bpc.TOPK, vocab, 8), rows)
        for dtype in range(3):
            for stride in (vocab, vocab + 1, (vocab + 63) // 64 * 64):
                for step in (0, 1):
                    for r in (rows, smaller, 1):
                        assert geometry.dg_needed(r, vocab, dtype, stride, step) <= size
                        geometry.dg_cut(r, vocab, dtype, stride, step, C.addressof(chunks), C.addressof(vecs), C.addressof(nv))
                        assert chunks.value * vecs.value >= nv.value and chunks.value <= 65535
                        if chunks.value > 1:
                            assert vecs.value <= 16384
                        else:   # a bit a logit in 32 KB
                            assert nv.value * (4 if dtype == 0 else 8) <= 1 << 18


def test_binding_refuses_what_the_kernels_cannot_take(bpc, monkeypatch):
    """On CPU tensors that are taken for tensors of the current device: nothing is launched, the library is not called."""
    d = bpc.make_distill(bpc.TOPK, 100, 4)
    x = torch.zeros(3, 100)
    msg = torch.zeros(3 * bpc.logits_stride(d), dtype=torch.uint8)
    loss, stats, ws = torch.zeros(3), torch.zeros(3, 32, dtype=torch.uint8), torch.zeros(256, dtype=torch.uint8)
    for at in (-1, 0):                                          # no GPU, and everything on the CPU
        monkeypatch.setattr(bpc, "_distill_torch", lambda at=at, real=bpc._distill_torch: (real(), at)[1])
        with pytest.raises(ValueError, match="current device"):
            bpc.bpc_logits_topk(d, x, None, msg, ws)
        with pytest.raises(ValueError, match="current device"):
            bpc.bpc_distill_step(d, x, msg, None, None, loss, x, ws)
    with pytest.raises(TypeError):
        bpc.bpc_distill_loss(d, x.double(), msg, None, None, loss, stats, ws)
    for bad in (x[:, :99], torch.zeros(100, 3).t(), x[0], x[None]):
        with pytest.raises(ValueError, match="logits"):
            bpc.bpc_distill_loss(d, bad, msg, None, None, loss, stats, ws)
    u8, f32, i64 = bpc._types
    for bad in (msg[:-1], msg.float(), torch.zeros(2, msg.numel(), dtype=u8)[:, ::2]):
        with pytest.raises(ValueError, match="messages: expected"):
            bpc._flat(bad, u8, 3 * bpc._record_bytes(d), -1, "messages")
    for dtype, per in ((i64, 1), (f32, 1), (u8, 32)):
        for bad in (torch.zeros(3 * per - 1, dtype=dtype), torch.zeros(3 * per, dtype=torch.int32), torch.zeros(3 * per, 2, dtype=dtype)[:, 0]):
            with pytest.raises(ValueError, match="expected a contiguous"):
                bpc._flat(bad, dtype, 3 * per, 0, "it")


def test_binding_knows_the_record(bpc):
    for kind in (bpc.TOPK, bpc.TOPK16):
        for k in (1, 2, 3, 4, 5, 7, 8, 9, 100, 1023, 1024):
            d = bpc.make_distill(kind, 5000, k)
            assert bpc._record_bytes(d) == bpc.logits_stride(d)


@pytest.mark.parametrize("tail_rest", [False, True])
@pytest.mark.parametrize("tau", [1.0, 2.5])
def test_plain_gradient_against_differences(tail_rest, tau):
    rs = np.random.default_rng(5)
    V, n = 23, 6
    s = rs.standard_normal(V) * 2
    idx = np.sort(rs.choice(V, n, replace=False))
    val = -rs.exponential(1.5, n)
    val -= val.max()

    def loss(x):
        return ref.student_row(x, n, idx, val, 0.3, tau, 1.7, 0.4, tail_rest, 4, 0.8)[0]
    g = ref.student_row(s, n, idx, val, 0.3, tau, 1.7, 0.4, tail_rest, 4, 0.8)[1]
    h = 1e-5
    for j in range(V):
        step = np.zeros(V)
        step[j] = h
        # (central differences: h^2 times a third derivative of order 1, and 1e-16 / h)
        assert abs((loss(s + step) - loss(s - step)) / (2 * h) - g[j]) < 1e-8
