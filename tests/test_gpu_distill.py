"""Distillation operators on the GPU against their plain float64 forms (distill_ref.py): records to the bit, sums,
losses and gradients within the bounds derived there."""
import math

import numpy as np
import pytest

import distill_ref as ref

pytestmark = pytest.mark.gpu

DT = ["f32", "f16", "bf16"]


@pytest.fixture(scope="module")
def bpc():
    import torch
    assert torch.cuda.is_available()
    import paper_2105_07829_amd as bpc
    bpc.lib()
    return bpc


def tdtype(name):
    import torch
    return {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}[name]


def rows_of(x, dtype, pad=0, fill=7.0, lead=0):
    """[rows, vocab] on the GPU in `dtype`, `pad` elements between rows; the buffer too."""
    import torch
    rows, vocab = x.shape
    buf = torch.full((rows, vocab + pad), fill, dtype=tdtype(dtype), device="cuda")
    view = buf[:, :vocab]
    view.copy_(torch.from_numpy(np.ascontiguousarray(x, np.float32)))
    return buf, view


def host(t):
    return t.detach().float().cpu().numpy()


def fields(bpc, d, messages, rows):
    """n, idx, val, rest, top of every record, and the raw words."""
    raw = messages.cpu().numpy()[:rows * bpc.logits_stride(d)].reshape(rows, -1)
    k, at = d.k, 16 + 4 * (-(-d.k // 4) * 4)
    w = raw[:, :16].copy().view(np.uint32)
    f = raw[:, :16].copy().view(np.float32)
    idx = raw[:, 16:16 + 4 * k].copy().view(np.int32)
    val = (raw[:, at:at + 4 * k].copy().view(np.float32) if d.kind == bpc.TOPK else raw[:, at:at + 2 * k].copy().view(np.float16))
    return w[:, 0], idx, val, f[:, 1], f[:, 2]


def make_messages(bpc, d, records):
    """Messages from (n, idx, val, rest, top) of every row."""
    import torch
    raw = np.zeros((len(records), bpc.logits_stride(d)), np.uint8)
    at = 16 + 4 * (-(-d.k // 4) * 4)
    for r, (n, idx, val, rest, top) in enumerate(records):
        raw[r, :4] = np.array([n], np.uint32).view(np.uint8)
        raw[r, 4:12] = np.array([rest, top], np.float32).view(np.uint8)
        i = np.full(d.k, -1, np.int32)
        i[:len(idx)] = idx
        v = np.full(d.k, -np.inf, np.float32 if d.kind == bpc.TOPK else np.float16)
        v[:len(val)] = val
        raw[r, 16:16 + 4 * d.k] = i.view(np.uint8)
        raw[r, at:at + v.nbytes] = v.view(np.uint8)
    return torch.from_numpy(raw).cuda()


def workspace(bpc, d, rows):
    import torch
    return torch.full((bpc.distill_workspace_bytes(d, rows),), 0xA5, dtype=torch.uint8, device="cuda")


def check_topk(bpc, d, x, dtype, pad=0, weight=None, only=None):
    import torch
    rows, vocab = x.shape
    _, view = rows_of(x, dtype, pad)
    size = bpc.logits_message_bytes(d, rows)
    guard = torch.full((size + 64,), 0x5A, dtype=torch.uint8, device="cuda")
    w = None if weight is None else torch.tensor(weight, dtype=torch.float32, device="cuda")
    print("topk", x.shape, dtype, "k", d.k, flush=True)
    bpc.bpc_logits_topk(d, view, w, guard[:size], workspace(bpc, d, rows))
    torch.cuda.synchronize()
    assert bool((guard[size:] == 0x5A).all())
    n, idx, val, rest, top = fields(bpc, d, guard, rows)
    t = host(view)
    for r in (range(rows) if only is None else only):
        row = t[r] if weight is None or weight[r] != 0 else np.full(vocab, -np.inf, np.float32)
        want_idx, want_val, want_top, want_rest, bound = ref.topk_row(row, d.k, d.temperature, d.kind == bpc.TOPK16)
        assert n[r] == len(want_idx), (r, n[r], len(want_idx))
        assert np.array_equal(idx[r, :n[r]], want_idx), r
        assert np.all(idx[r, n[r]:] == -1) and np.all(np.isneginf(val[r, n[r]:].astype(np.float32)))
        assert np.array_equal(val[r, :n[r]], want_val, equal_nan=True), r
        assert np.array_equal([top[r]], [want_top], equal_nan=True)
        if math.isfinite(want_rest):
            assert abs(rest[r] - want_rest) <= bound, (r, rest[r], want_rest, bound)
    return guard[:size]


VOCABS = [1, 2, 7, 8, 9, 63, 64, 65, 511, 1000, 4099, 8191, 30522, 50257]


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("vocab", VOCABS)
def test_topk_sizes(bpc, dtype, vocab):
    rs = np.random.default_rng(vocab)
    x = rs.standard_normal((5, vocab)) * 3
    for k, kind, tau, pad in [(1, bpc.TOPK, 1.0, 0), (10, bpc.TOPK16, 2.0, 3), (64, bpc.TOPK, 0.5, 1), (257, bpc.TOPK16, 1.0, 8)]:
        check_topk(bpc, bpc.make_distill(kind, vocab, k, temperature=tau), x, dtype, pad)


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("vocab,rows", [(131072, 2), (131073, 3), (151936, 1), (262147, 2), (1 << 20, 1)])
def test_topk_long_rows(bpc, dtype, vocab, rows):
    x = np.random.default_rng(vocab).standard_normal((rows, vocab)) * 2
    for k, kind in [(1, bpc.TOPK), (50, bpc.TOPK16), (1024, bpc.TOPK)]:
        check_topk(bpc, bpc.make_distill(kind, vocab, k), x, dtype, pad=5)


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("rows", [1, 2, 31, 300, 1100])
def test_topk_rows(bpc, dtype, rows):
    x = np.random.default_rng(rows).standard_normal((rows, 2050)) * 3
    for k in (3, 500, 1024):
        check_topk(bpc, bpc.make_distill(bpc.TOPK16, 2050, k), x, dtype, pad=1)


def shapes_of_rows(vocab):
    """Rows on which a selection can go wrong."""
    rs = np.random.default_rng(9)
    base = rs.standard_normal(vocab)
    j = np.arange(vocab)
    yield "constant", np.zeros(vocab)
    yield "signed zeros", np.where(j % 2, 0.0, -0.0)
    yield "two levels", (j % 3 == 0) * 1.0
    yield "few levels", np.round(base * 2)
    yield "ascending", j * (60.0 / vocab)
    yield "descending", -j * (60.0 / vocab)
    yield "sawtooth", (j % 256) * 0.125
    yield "one thread's share", np.where(j % 2048 < 8, 5.0 + base, base - 20)
    yield "one stretch", np.where((j >= vocab // 3) & (j < vocab // 3 + 1500), 9.0 + base, base - 9)
    yield "masked all", np.full(vocab, -np.inf)
    yield "masked but three", np.where(j % max(1, vocab // 3) == 1, base, -np.inf)
    yield "masked but the last", np.where(j == vocab - 1, 3.0, -np.inf)
    yield "masked half", np.where(j % 2, base, -np.inf)
    yield "lowest", np.full(vocab, -60000.0)
    yield "far apart", np.where(j % 100 == 7, 100.0, -100.0) + base
    yield "infinite", np.where(j == vocab // 2, np.inf, base)
    yield "nan", np.where((j == vocab // 2) | (j == 1), np.nan, base)
    yield "nan all", np.full(vocab, np.nan)


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("vocab", [40, 2100, 40000, 150001])
def test_topk_hard_rows(bpc, dtype, vocab):
    x = np.stack([row for _, row in shapes_of_rows(vocab)])
    for k, kind in [(1, bpc.TOPK), (33, bpc.TOPK16), (1000, bpc.TOPK)]:
        check_topk(bpc, bpc.make_distill(kind, vocab, k, temperature=1.5), x, dtype, pad=1)
    if vocab == 150001:   # row by row: few rows are cut
        for r in range(len(x)):
            check_topk(bpc, bpc.make_distill(bpc.TOPK, vocab, 300), x[r:r + 1], dtype)


@pytest.mark.parametrize("dtype", DT)
def test_topk_many_rows(bpc, dtype):
    """Enough rows that a smaller workgroup takes each, hard ones among them."""
    vocab = 9001
    hard = np.stack([row for _, row in shapes_of_rows(vocab)])
    x = np.random.default_rng(21).standard_normal((540, vocab)) * 2
    x[7:7 + len(hard)] = hard
    for k, kind in [(5, bpc.TOPK), (100, bpc.TOPK16), (900, bpc.TOPK)]:
        check_topk(bpc, bpc.make_distill(kind, vocab, k, temperature=1.5), x, dtype, pad=3)


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("vocab,k", [(20011, 20), (40001, 300), (140001, 64), (40001, 1024)])
def test_topk_many_long_rows(bpc, dtype, vocab, k):
    """The forms that rows of these lengths take where there are enough of them; some rows are looked at."""
    x = np.random.default_rng(k).standard_normal((530, vocab), dtype=np.float32) * 2
    hard = np.stack([row for _, row in shapes_of_rows(vocab)])
    x[100:100 + len(hard)] = hard
    check_topk(bpc, bpc.make_distill(bpc.TOPK, vocab, k, temperature=1.5), x, dtype, pad=3,
               only=[0, 1, 2, 3, *range(100, 100 + len(hard)), 255, 256, 528, 529])


@pytest.mark.parametrize("dtype", DT)
def test_topk_lowest_of_the_type(bpc, dtype):
    import torch
    low = torch.finfo(tdtype(dtype)).min
    x = np.random.default_rng(1).standard_normal((3, 3000)).astype(np.float32)
    x[0, 10:] = low
    x[1, :] = low
    x[2, 2900:] = low
    check_topk(bpc, bpc.make_distill(bpc.TOPK, 3000, 64, temperature=0.7), x, dtype)
    check_topk(bpc, bpc.make_distill(bpc.TOPK16, 3000, 64, temperature=2.0), x, dtype)


@pytest.mark.parametrize("vocab", [1000, 50257])
def test_topk_idle_rows(bpc, vocab):
    x = np.random.default_rng(4).standard_normal((40, vocab))
    weight = np.where(np.arange(40) % 3 == 1, 0.0, 0.5)
    x[1] = np.nan
    check_topk(bpc, bpc.make_distill(bpc.TOPK, vocab, 8), x, "bf16", weight=weight)


# ---- the student

def make_case(rs, vocab, k, rows, masked=0):
    """Logits and records of `rows` rows; entries among the unmasked words."""
    x = rs.standard_normal((rows, vocab)) * 2.5
    used = vocab - masked
    if masked:
        x[:, used:] = -np.inf
    records = []
    for r in range(rows):
        n = min(k, used)
        idx = np.sort(rs.choice(used, n, replace=False))
        val = -rs.exponential(2.0, n)
        val -= val.max()
        x[r, idx] += 4.0
        rest = float(np.float32(rs.random() * 0.6)) if n < used else 0.0
        records.append((n, idx, val, rest, 3.0))
    return x, records


def check_student(bpc, d, x, records, dtype, pad=0, gpad=None, labels=None, weight=None, in_place=False, want_nan=(), only=None):
    import torch
    rows, vocab = x.shape
    buf, view = rows_of(x, dtype, pad)
    messages = make_messages(bpc, d, records)
    lab = None if labels is None else torch.tensor(labels, dtype=torch.int64, device="cuda")
    w = None if weight is None else torch.tensor(weight, dtype=torch.float32, device="cuda")
    wh = np.ones(rows) if weight is None else np.asarray(weight, np.float32)
    ws = workspace(bpc, d, rows)
    s = host(view)
    gpad = pad if gpad is None else gpad

    def new_grad():
        g = torch.full((rows, vocab + gpad), 7.0, dtype=tdtype(dtype), device="cuda")
        return g, g[:, :vocab]

    def new_loss():
        return torch.full((rows + 4,), 7.0, device="cuda")
    print("student", x.shape, dtype, "k", d.k, flush=True)
    loss1, stats = new_loss(), torch.zeros(rows, 32, dtype=torch.uint8, device="cuda")
    bpc.bpc_distill_loss(d, view, messages, lab, w, loss1[:rows], stats, ws)
    gbuf1, grad1 = new_grad()
    bpc.bpc_distill_grad(d, view, messages, lab, w, stats, grad1)
    loss0 = new_loss()
    bpc.bpc_distill_loss(d, view, messages, lab, w, loss0[:rows], None, ws)
    loss2 = new_loss()
    gbuf2, grad2 = new_grad()
    bpc.bpc_distill_step(d, view, messages, lab, w, loss2[:rows], grad2, ws)
    got = [(loss1, gbuf1, grad1), (loss2, gbuf2, grad2)]
    if in_place:
        buf3, view3 = rows_of(x, dtype, pad)
        bpc.bpc_distill_grad(d, view3, messages, lab, w, stats, view3)
        got.append((loss1, buf3, view3))
        buf4, view4 = rows_of(x, dtype, pad)
        loss4 = new_loss()
        bpc.bpc_distill_step(d, view4, messages, lab, w, loss4[:rows], view4, ws)
        got.append((loss4, buf4, view4))
    torch.cuda.synchronize()
    assert torch.equal(loss0.view(torch.int32), loss1.view(torch.int32))
    assert np.array_equal(host(view), s, equal_nan=True)
    n, idx, val, rest, _ = fields(bpc, d, messages, rows)
    for loss, gbuf, grad in got:
        assert bool((loss[rows:] == 7.0).all()) and bool((gbuf[:, vocab:] == 7.0).all())
        l, g = host(loss), host(grad)
        for r in (range(rows) if only is None else only):
            if r in want_nan and wh[r] != 0.0:
                assert np.isnan(l[r]) and np.isnan(g[r]).all(), r
                continue
            want_l, want_g, le, ge = ref.student_row(s[r], min(int(n[r]), d.k), idx[r], val[r], rest[r], d.temperature, d.soft_weight,
                                                     d.hard_weight, d.tail == bpc.TAIL_REST, None if labels is None else labels[r],
                                                     float(wh[r]), dtype)
            if math.isinf(want_l):
                assert l[r] == want_l
            else:
                assert abs(l[r] - want_l) <= le, (r, l[r], want_l, le)
            bad = ~(np.abs(g[r] - want_g) <= ge)
            assert not bad.any(), (r, np.nonzero(bad)[0][:5], g[r][bad][:5], want_g[bad][:5], ge[bad][:5])


def describe(bpc, vocab, k, kind=None, **kw):
    return bpc.make_distill(bpc.TOPK if kind is None else kind, vocab, k, **kw)


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("vocab", VOCABS)
def test_student_sizes(bpc, dtype, vocab):
    rs = np.random.default_rng(vocab + 1)
    for k, kind, tau, tail, hard, pad, gpad in [(1, bpc.TOPK, 1.0, 0, 0.0, 0, 0), (10, bpc.TOPK16, 2.0, 1, 0.3, 3, 3),
                                                (64, bpc.TOPK, 0.5, 1, 0.0, 1, 6), (257, bpc.TOPK16, 1.0, 0, 0.5, 8, 1)]:
        x, records = make_case(rs, vocab, k, 4)
        labels = [int(records[0][1][0]), vocab - 1, -100, int(rs.integers(vocab))]
        check_student(bpc, describe(bpc, vocab, k, kind, temperature=tau, tail=tail, soft_weight=1.3, hard_weight=hard), x, records,
                      dtype, pad, gpad, labels, in_place=pad == 3)


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("vocab,rows", [(65531, 3), (131072, 2), (131073, 2), (262147, 2), (1 << 20, 1)])
def test_student_long_rows(bpc, dtype, vocab, rows):
    rs = np.random.default_rng(vocab)
    for k, tau, tail, hard in [(50, 1.0, 1, 0.0), (1024, 2.0, 0, 0.3), (300, 2.0, 1, 0.1)]:
        x, records = make_case(rs, vocab, k, rows)
        check_student(bpc, describe(bpc, vocab, k, temperature=tau, tail=tail, hard_weight=hard), x, records, dtype, 5, 5,
                      [int(records[r][1][-1]) if r else vocab - 2 for r in range(rows)], in_place=tail == 1)


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("rows", [1, 2, 31, 300, 1100])
def test_student_rows(bpc, dtype, rows):
    rs = np.random.default_rng(rows)
    x, records = make_case(rs, 1500, 40, rows)
    labels = list(rs.integers(-2, 1502, rows))
    weight = np.where(np.arange(rows) % 4 == 2, 0.0, rs.random(rows) - 0.3).astype(np.float32)
    check_student(bpc, describe(bpc, 1500, 40, tail=1, temperature=3.0, hard_weight=0.2), x, records, dtype, 1, 1, labels, weight)


@pytest.mark.parametrize("dtype,hard,tau,tail", [("bf16", 0.2, 2.0, 1), ("f32", 0.0, 1.0, 0), ("f16", 0.1, 1.7, 1), ("f32", 0.3, 4.0, 1)])
def test_student_many_rows(bpc, dtype, hard, tau, tail):
    """Enough rows that a smaller workgroup takes each, odd ones among them."""
    rs = np.random.default_rng(22)
    vocab = 9001
    x, records = make_case(rs, vocab, 300, 1030)
    x[3] = np.nan
    x[4, 17] = np.inf
    x[5] *= 2e4 if dtype != "f16" else 1e3
    x[6, 4000:] = {"f32": -3.4028234663852886e38, "f16": -65504.0, "bf16": -3.3895313892515355e38}[dtype]
    x[6, 4000 + int(rs.integers(5000))] = 1.0
    weight = np.where(np.arange(1030) % 9 == 8, 0.0, 1.0)
    check_student(bpc, describe(bpc, vocab, 300, tail=tail, temperature=tau, hard_weight=hard), x, records, dtype, 1, 1,
                  list(rs.integers(0, vocab, 1030)), weight, want_nan=(3, 4))


@pytest.mark.parametrize("vocab,dtype,hard,tau,tail", [(20011, "bf16", 0.2, 2.0, 1), (20011, "f16", 0.0, 1.0, 0), (50257, "bf16", 0.1, 1.3, 1),
                                                       (30522, "f32", 0.1, 1.0, 1), (70001, "bf16", 0.3, 4.0, 1), (70001, "f32", 0.0, 0.7, 0)])
def test_student_many_long_rows(bpc, vocab, dtype, hard, tau, tail):
    """The forms that rows of these lengths take where there are enough of them; some rows are looked at."""
    rs = np.random.default_rng(vocab)
    rows, k = 530, 90
    x = rs.standard_normal((rows, vocab), dtype=np.float32) * 2
    idx = [np.sort(rs.choice(vocab, k, replace=False)) for _ in range(rows)]
    records = [(k, i, -np.arange(k) * 0.07, 0.2, 3.0) for i in idx]
    for r in range(rows):
        x[r, idx[r]] += 5.0
    x[20] = np.nan
    x[40] *= 1e4
    x[60, vocab // 2:] = -np.inf
    weight = np.where(np.arange(rows) % 7 == 5, 0.0, 1.5)
    labels = [int(idx[r][3]) if r % 3 else int(rs.integers(vocab)) for r in range(rows)]
    check_student(bpc, describe(bpc, vocab, k, bpc.TOPK16, tail=tail, temperature=tau, hard_weight=hard), x, records, dtype, 1, 1,
                  labels, weight, in_place=True, want_nan=(20,), only=[0, 1, 5, 20, 40, 60, 61, 255, 256, 511, 512, 528, 529])


@pytest.mark.parametrize("tail", [0, 1])
@pytest.mark.parametrize("vocab", [300, 20000, 140000])
def test_student_masks(bpc, vocab, tail):
    """Masked words, rows with nothing in them, words that the teacher wants and the student masks."""
    rs = np.random.default_rng(3)
    for dtype in DT:
        x, records = make_case(rs, vocab, 16, 8, masked=vocab // 5)
        lowest = {"f32": -3.4028234663852886e38, "f16": -65504.0, "bf16": -3.3895313892515355e38}[dtype]
        x[1, vocab - vocab // 5:] = lowest                       # masked by the lowest number
        records[2] = (0, [], [], 0.0, -np.inf)                   # an empty record: no soft term
        records[3] = (0, [], [], 0.5, 1.0)                       # nothing listed, some rest: nothing to compare
        x[4, records[4][1][0]] = -np.inf                         # the student masks a listed word: infinite loss
        all_idx = np.arange(16)
        records[5] = (16, all_idx, -all_idx * 0.5, 0.0, 0.0)     # the student has the listed words only, no rest
        x[5, :] = -np.inf
        x[5, :16] = rs.standard_normal(16)
        records[6] = (16, all_idx, -all_idx * 0.5, 0.0, 0.0)     # rest far below the listed words
        x[6, :] = rs.standard_normal(vocab) - 400.0
        x[6, :16] = 3.0
        records[7] = (16, all_idx, np.where(all_idx == 0, 0.0, -np.inf), 0.0, 0.0)   # one word has everything
        labels = [0, 1, 2, -1, 3, 5, 7, 0]
        for tau, hard in [(1.0, 0.0), (2.0, 0.4)]:
            check_student(bpc, describe(bpc, vocab, 16, tail=tail, temperature=tau, hard_weight=hard), x, records, dtype,
                          3, 3, labels, in_place=True)


def test_student_without_a_soft_term(bpc):
    """soft_weight 0: the hard term alone, whatever the teacher says of words that the student masks."""
    rs = np.random.default_rng(15)
    for vocab in (700, 20000, 140000):
        x, records = make_case(rs, vocab, 9, 3)
        x[1, records[1][1][2]] = -np.inf
        for tail in (0, 1):
            check_student(bpc, describe(bpc, vocab, 9, tail=tail, temperature=3.0, soft_weight=0.0, hard_weight=1.0), x, records, "f32",
                          labels=[3, 4, vocab - 1], in_place=True)


def test_student_rest_far_below(bpc):
    """The teacher's rest is compared with a student's rest of 1e-87: a difference 1 - sum p would be 0."""
    rs = np.random.default_rng(8)
    for vocab in (500, 150000):
        x = rs.standard_normal((2, vocab)) - 200.0
        x[:, :4] = 1.0
        records = [(4, np.arange(4), [0.0, -1.0, -2.0, -0.5], 0.25, 0.0)] * 2
        check_student(bpc, describe(bpc, vocab, 4, tail=1), x, records, "f32", in_place=True)


def test_student_lowest_everywhere(bpc):
    """A row of the type's lowest value is a uniform row."""
    import torch
    for dtype in DT:
        low = torch.finfo(tdtype(dtype)).min
        x = np.full((2, 700), low, np.float32)
        records = [(3, np.array([1, 5, 9]), [0.0, -0.5, -1.0], 0.2, 0.0)] * 2
        for tau in (1.0, 0.5):
            check_student(bpc, describe(bpc, 700, 3, tail=1, temperature=tau, hard_weight=0.1), x, records, dtype, labels=[0, 5])
            check_student(bpc, describe(bpc, 700, 3, tail=0, temperature=tau, hard_weight=0.1), x, records, dtype, labels=[0, 5])


@pytest.mark.parametrize("tail", [0, 1])
@pytest.mark.parametrize("vocab", [200, 30000, 140000])
def test_student_nan_and_infinity(bpc, vocab, tail):
    """NaN and +inf stay in their rows, and rows of weight 0 are not looked at."""
    rs = np.random.default_rng(6)
    x, records = make_case(rs, vocab, 5, 7)
    x[1, vocab - 1] = np.nan
    x[2, int(records[2][1][1])] = np.nan
    x[3, 3] = np.inf
    x[4, :] = np.nan
    x[5, :] = -np.inf
    weight = [1.0, 1.0, 1.0, 1.0, 0.0, 1.0, 0.5]
    for hard in (0.0, 0.5):
        check_student(bpc, describe(bpc, vocab, 5, tail=tail, temperature=2.0, hard_weight=hard), x, records, "f32", 1, 2,
                      [1] * 7, weight, want_nan=(1, 2, 3, 5))


def test_student_reads_no_more_than_a_record_says(bpc):
    """Records that name words outside the vocabulary or more entries than there is room for: those are skipped."""
    import torch
    rs = np.random.default_rng(2)
    for vocab in (90, 140000):
        x, records = make_case(rs, vocab, 6, 3)
        d = describe(bpc, vocab, 6, tail=1)
        n, idx, val, rest, top = records[0]
        bad = [(n, np.where(np.arange(6) < 5, idx, 2 ** 31 - 1), val, rest, top), (n, np.where(np.arange(6) > 0, idx, -5), val, rest, top),
               (2 ** 31, idx, val, rest, top)]
        _, view = rows_of(np.stack([x[0]] * 3), "f32")
        ws = workspace(bpc, d, 3)
        loss, grad = torch.zeros(3, device="cuda"), torch.zeros(3, vocab, device="cuda")
        bpc.bpc_distill_step(d, view, make_messages(bpc, d, bad), None, None, loss, grad, ws)
        for r, keep in enumerate([slice(0, 5), slice(1, 6), slice(0, 6)]):
            i, v = idx[keep], np.asarray(val, np.float32)[keep]
            want_l, want_g, le, ge = ref.student_row(host(view)[r], len(i), i, v, np.float32(rest), 1.0, 1.0, 0.0, True, None, 1.0)
            assert abs(float(loss[r]) - want_l) <= le
            assert (np.abs(host(grad)[r] - want_g) <= ge).all()


def test_offsets_past_32_bits(bpc):
    """Rows more than 2^32 elements (and bytes) apart."""
    import torch
    stride, vocab, k = (1 << 31) + 24, 1000, 12
    rs = np.random.default_rng(11)
    buf = torch.empty(2 * stride + vocab, dtype=torch.bfloat16, device="cuda")
    view = torch.as_strided(buf, (3, vocab), (stride, 1))
    x, records = make_case(rs, vocab, k, 3)
    view.copy_(torch.from_numpy(x))
    d = describe(bpc, vocab, k, tail=1)
    ws = workspace(bpc, d, 3)
    msg = torch.zeros(bpc.logits_message_bytes(d, 3), dtype=torch.uint8, device="cuda")
    bpc.bpc_logits_topk(d, view, None, msg, ws)
    # (the order of a sum goes by where a row starts in its 128-byte line: 24 elements further each, here as there)
    small = torch.empty(3, 1024 + 24, dtype=torch.bfloat16, device="cuda")[:, :vocab]
    small.copy_(view)
    msg2 = torch.zeros_like(msg)
    bpc.bpc_logits_topk(d, small, None, msg2, ws)
    assert torch.equal(msg, msg2)
    m = make_messages(bpc, d, records)
    loss, loss2 = torch.zeros(3, device="cuda"), torch.zeros(3, device="cuda")
    grad = torch.zeros(3, vocab, dtype=torch.bfloat16, device="cuda")
    bpc.bpc_distill_step(d, small, m, None, None, loss2, grad, ws)
    bpc.bpc_distill_step(d, view, m, None, None, loss, view, ws)
    assert torch.equal(loss, loss2) and torch.equal(view, grad)
    del buf, view
    torch.cuda.empty_cache()


@pytest.mark.parametrize("rows,vocab", [(1, 50257), (3, 140001), (64, 1000), (200, 30522)])
def test_teacher_and_student_together(bpc, rows, vocab):
    """A teacher's logits through its message into a student's loss and gradient, against the dense distributions."""
    import torch
    rs = np.random.default_rng(rows)
    k, tau = 48, 2.0
    t = rs.standard_normal((rows, vocab)) * 3
    s = t * 0.5 + rs.standard_normal((rows, vocab))
    _, tv = rows_of(t, "bf16", 1)
    _, sv = rows_of(s, "f32", 3)
    d = describe(bpc, vocab, k, temperature=tau, tail=1, soft_weight=tau * tau * 0.9, hard_weight=0.1)
    ws = workspace(bpc, d, rows)
    msg = torch.zeros(bpc.logits_message_bytes(d, rows), dtype=torch.uint8, device="cuda")
    lab = torch.from_numpy(rs.integers(0, vocab, rows)).cuda()
    loss, grad = torch.zeros(rows, device="cuda"), torch.zeros(rows, vocab, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        bpc.bpc_logits_topk(d, tv, None, msg, ws)
        bpc.bpc_distill_step(d, sv, msg, lab, None, loss, grad, ws)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    th, sh = host(tv), host(sv)
    for r in range(rows):
        idx, val, top, rest, _ = ref.topk_row(th[r], k, tau, False)
        want_l, want_g, le, ge = ref.student_row(sh[r], len(idx), idx, val, np.float32(rest), tau, d.soft_weight, d.hard_weight, True,
                                                 int(lab[r]), 1.0)
        # (the record's rest has an error of its own: `chain` additions and exponentials of arguments up to 40)
        more = ref.chain(vocab) * ref.U + ref.exp_error(40.0)
        assert abs(float(loss[r]) - want_l) <= le + abs(d.soft_weight) * more * (1 + abs(want_l))
        assert (np.abs(host(grad)[r] - want_g) <= ge + abs(d.soft_weight) / tau * more).all()


def test_loss_falls_along_the_gradient(bpc):
    """Differences of the kernel's own loss along its own gradient."""
    import torch
    rs = np.random.default_rng(12)
    x, records = make_case(rs, 800, 20, 4)
    d = describe(bpc, 800, 20, temperature=2.0, tail=1, soft_weight=3.0, hard_weight=0.5)
    _, view = rows_of(x, "f32")
    m, ws = make_messages(bpc, d, records), workspace(bpc, d, 4)
    lab = torch.tensor([1, 5, 9, 700], device="cuda")
    loss, grad = torch.zeros(4, device="cuda"), torch.zeros(4, 800, device="cuda")
    bpc.bpc_distill_step(d, view, m, lab, None, loss, grad, ws)
    h = 2.0 ** -4
    ends = []
    for sign in (1, -1):
        out = torch.zeros(4, device="cuda")
        bpc.bpc_distill_loss(d, view + sign * h * grad, m, lab, None, out, None, ws)
        ends.append(out.double())
    got = (ends[0] - ends[1]) / (2 * h)
    want = (grad.double() ** 2).sum(1)
    # |third derivative along g| <= |g|_1^3 * 6 for a sum of log-sum-exps of total weight 4; |g|_1 <= 4;
    # measured along g its size is that of |g|_2^3, so h^2 / 6 * 6 * 4 * |g|_2^3; roundings: 2^-20 of the loss over 2 h
    bound = h * h * 4 * want ** 1.5 + loss.double().abs() * 2.0 ** -20 / (2 * h)
    assert bool(((got - want).abs() <= bound).all()), (got, want, bound)


def test_same_bits_every_time_and_in_graphs(bpc):
    """Calls recorded into graphs, replayed between eager calls, with workspaces of their own and two graphs on one."""
    import torch
    rs = np.random.default_rng(13)
    for rows, vocab in [(70, 3001), (2, 140003)]:
        k = 30
        d = describe(bpc, vocab, k, temperature=2.0, tail=1, hard_weight=0.2)
        x, _ = make_case(rs, vocab, k, rows)
        _, tv = rows_of(rs.standard_normal((rows, vocab)) * 3, "bf16", 1)
        _, sv = rows_of(x, "bf16", 1)
        lab = torch.from_numpy(rs.integers(0, vocab, rows)).cuda()
        ws = workspace(bpc, d, rows)
        msg = torch.zeros(bpc.logits_message_bytes(d, rows), dtype=torch.uint8, device="cuda")
        stats = torch.zeros(rows, 32, dtype=torch.uint8, device="cuda")
        loss, loss2 = torch.zeros(rows, device="cuda"), torch.zeros(rows, device="cuda")
        grad, grad2 = torch.zeros_like(sv), torch.zeros_like(sv)

        def teacher():
            bpc.bpc_logits_topk(d, tv, None, msg, ws)

        def student():
            bpc.bpc_distill_step(d, sv, msg, lab, None, loss, grad, ws)
            bpc.bpc_distill_loss(d, sv, msg, lab, None, loss2, stats, ws)
            bpc.bpc_distill_grad(d, sv, msg, lab, None, stats, grad2)
        out = (msg, loss, loss2, grad, grad2)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            teacher(), student()
        torch.cuda.current_stream().wait_stream(side)
        torch.cuda.synchronize()
        want = [t.clone() for t in out]
        graphs = []
        for call in (teacher, student):
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g):
                call()
            graphs.append(g)
        for rep in range(4):
            for t in out:
                t.zero_()
            ws.fill_(rep + 1)
            assert torch.rand(1 << 18, device="cuda").sum().item() > 0
            for g in graphs:
                g.replay()
            torch.cuda.synchronize()
            for a, b in zip(out, want):
                assert torch.equal(a, b), rep
            for t in out:
                t.zero_()
            teacher(), student()
            torch.cuda.synchronize()
            for a, b in zip(out, want):
                assert torch.equal(a, b), rep
