"""Distillation operators, what needs no GPU: the plain forms where a row has no term or no softmax, and what the teacher's
forms need of workspace and LDS."""
import ctypes as C
import os
import subprocess

import numpy as np
import pytest

import distill_ref as ref

ANY, DENSE, GROUPS = 0, 1, 2


@pytest.fixture(scope="module")
def bpc():
    import paper_2105_07829_amd as bpc
    bpc.lib()
    return bpc


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    """csrc/distill_geometry.hpp compiled for the host."""
    so = str(tmp_path_factory.mktemp("distill_topk") / "host_distill_topk.so")
    here = os.path.dirname(os.path.abspath(__file__))
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-shared", "-fPIC", "-o", so, os.path.join(here, "host_distill_topk.cpp")], check=True)
    L = C.CDLL(so)
    L.dt_plan.argtypes = [C.c_uint64, C.c_uint32, C.c_uint32, C.c_int, C.c_uint64, C.c_void_p]
    L.dt_plan.restype = None
    out = (C.c_uint64 * 10)()

    def plan(rows, vocab, k, dtype, stride):
        L.dt_plan(rows, vocab, k, dtype, stride, C.addressof(out))
        return dict(zip(("form", "threads", "lds", "lanes", "n_groups", "cap", "region", "few", "ws", "nv"), out))
    return plan


def shapes():
    """Sizes at the borders of the forms, and sizes over their ranges."""
    for vocab in (1, 15360, 15361, 16384, 32767, 32768, 131065, 131072, 131073, 262080, 262136, 262137, 262144, 262145, 1 << 20, 1 << 24):
        for k in (1, 256, 511, 512, 1023, 1024):
            for rows in (1, 32, 33, 511, 512, 4096):
                yield rows, vocab, k
    rs = np.random.default_rng(3)
    for _ in range(4000):
        yield (int(np.exp(rs.uniform(0, np.log((1 << 22) - 1)))), int(np.exp(rs.uniform(0, np.log(1 << 24)))),
               int(np.exp(rs.uniform(0, np.log(1024)))))


def test_every_teacher_call_fits_its_workspace_and_its_lds(bpc, plan):
    seen = set()
    for rows, vocab, k in shapes():
        d = bpc.make_distill(bpc.TOPK, vocab, k)
        size = bpc.distill_workspace_bytes(d, rows)
        for dtype in range(3):
            e = 4 if dtype == 0 else 8
            for stride in (vocab, vocab + 1, (vocab + 63) // 64 * 64):
                for r in {rows, min(rows, 32), 1}:
                    p = plan(r, vocab, k, dtype, stride)
                    case = (r, vocab, k, dtype, stride, p)
                    seen.add((p["form"], p["threads"], p["lanes"], p["few"]))
                    assert p["ws"] <= size, case
                    assert p["threads"] in (64, 256, 1024), case
                    # what the kernel declares beside it: a word a thread, 256 counters, a few words a wave and a dozen
                    assert p["lds"] + 4 * p["threads"] + 1024 + 16 * p["threads"] // 64 + 64 <= 65536, case
                    if p["form"] == DENSE:
                        assert p["lds"] >= 4 * p["nv"] * e, case
                    if p["form"] != GROUPS:
                        assert p["ws"] == 0, case
                        continue
                    n, t, lanes = p["n_groups"], p["threads"], p["lanes"]
                    assert n <= 4096 and n % 4 == 0 and n * lanes >= p["nv"] and n * lanes % (4 * t) == 0, case
                    assert lanes <= 8 or t > 64, case                     # (no kernel of one wave has groups of 16)
                    assert p["region"] >= 8 * n and p["region"] >= 4 * p["cap"] and p["region"] % 16 == 0, case
                    span = -(-p["nv"] * e // (128 * t)) * 4                # words of a bit a logit that a thread looks through
                    assert p["region"] >= 4 * span * t and 32 * span * t >= p["nv"] * e, case
                    assert p["cap"] >= 2 * k and p["lds"] >= p["region"] + 8 * p["cap"] + 2 * n, case
                    if p["few"]:   # keys and sums, written by whole workgroups of 256 threads with four vectors each
                        assert r <= 32 and p["ws"] == 8 * n * r and n * lanes % 1024 == 0 and t == 1024, case
                    else:
                        assert p["ws"] == 0, case
    # the shapes reach every form
    assert {f for f, _, _, _ in seen} == {ANY, DENSE, GROUPS}
    assert {(t, lanes) for f, t, lanes, _ in seen if f == GROUPS} == {(64, l) for l in (1, 2, 4, 8)} | {(t, l) for t in (256, 1024) for l in (1, 2, 4, 8, 16)}
    assert {lanes for f, _, lanes, few in seen if few} == {2, 4, 8, 16}   # (few rows are cut from 4096 vectors on, four for each entry)


@pytest.mark.parametrize("tail_rest", [False, True])
@pytest.mark.parametrize("bad", [0.0, np.nan, np.inf, "masked"])
def test_plain_rows_without_a_term_are_zero(bad, tail_rest):
    s = np.linspace(-1.0, 2.0, 11)
    s[4] = -3.0 if bad == "masked" else s[4] + bad
    if bad == "masked":
        s[:] = -np.inf
    idx, val = np.array([1, 4]), np.array([0.0, -1.0])
    for n, soft, label in ((0, 1.0, -100), (0, 1.0, 11), (0, 1.0, None), (2, 0.0, -100)):
        loss, g, _, _ = ref.student_row(s, n, idx[:n], val[:n], 0.5, 2.0, soft, 0.3, tail_rest, label, 0.7)
        assert loss == 0.0 and np.array_equal(g, np.zeros(11)), (n, soft, label)
