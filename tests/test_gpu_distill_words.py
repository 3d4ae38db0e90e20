"""Distillation operators on the GPU: every word of a row counts once.  Logits are chosen so that all exponentials are powers
of two and all sums exact in f32; what is left are the few roundings named at each test, and each test holds its bound against
what one word more or less would change."""
import math

import numpy as np
import pytest

import distill_ref as ref
from test_gpu_distill import bpc, describe, fields, host, make_messages, tdtype, workspace  # noqa: F401  (bpc: the fixture)

pytestmark = pytest.mark.gpu

U = ref.U


def padded(rows, vocab, pad, dtype, fill=0.0):
    import torch
    buf = torch.full((rows, vocab + pad), 7.0, dtype=tdtype(dtype), device="cuda")
    view = buf[:, :vocab]
    view.fill_(fill)
    return view


# vocabulary, rows, entries, type: a wave, 256 and 1024 threads a row, groups of 1 to 16 vectors, in one launch and in two,
# rows in LDS, rows by the radix select
RECORDS = [(1000, 5, 10, "f32"), (4099, 5, 200, "bf16"), (9001, 520, 20, "bf16"), (9001, 520, 900, "f16"), (20011, 520, 20, "f32"),
           (50257, 520, 64, "bf16"), (30522, 40, 300, "f16"), (50257, 1, 32, "f32"), (131073, 3, 50, "f32"), (140001, 520, 64, "bf16"),
           (140001, 40, 1000, "f16"), (151936, 2, 700, "bf16"), (40001, 2, 1000, "bf16"), (262001, 4, 20, "bf16"), (262147, 2, 20, "bf16"), (1 << 20, 1, 20, "f32")]


@pytest.mark.parametrize("pad", [0, 1, 5])
@pytest.mark.parametrize("vocab,rows,k,dtype", RECORDS)
def test_record_counts_every_word(bpc, vocab, rows, k, dtype, pad):  # noqa: F811
    """k logits of 4, all others 0, at the temperature whose exponentials are powers of two: rest = (vocab - k) / 16, to the
    rounding of the temperature and one of the result."""
    import torch
    tau = float(np.float32(1.0 / math.log(2.0)))   # (exp(x / tau) is 2^x to 2^-24 of x)
    assert np.float32(1.44269504088896340736 / tau) == 1.0
    rs = np.random.default_rng(vocab + pad)
    view = padded(rows, vocab, pad, dtype)
    # (one in each of k groups, none beside the groups: the k-th largest of the groups is 4, only k logits reach it)
    ends, apart = min(100, vocab // 9), (vocab - 2 * min(100, vocab // 9)) // k
    words = ends + apart * np.arange(k) + rs.integers(0, max(1, apart // 4), (rows, k))
    view.scatter_(1, torch.from_numpy(words).cuda(), 4.0)
    d = describe(bpc, vocab, k, temperature=tau)
    msg = torch.zeros(bpc.logits_message_bytes(d, rows), dtype=torch.uint8, device="cuda")
    print("words of a record", vocab, rows, k, dtype, pad, flush=True)
    bpc.bpc_logits_topk(d, view, None, msg, workspace(bpc, d, rows))
    n, idx, val, rest, top = fields(bpc, d, msg, rows)
    assert (n == k).all() and np.array_equal(idx, words) and (val == 0.0).all() and (top == 4.0).all()
    want = (vocab - k) / 16
    bound = (4 * math.log(2.0) + 1) * U * want
    assert bound < 1 / 16
    assert (np.abs(rest.astype(np.float64) - want) <= bound).all(), (rest, want)


# vocabulary, rows: held by a wave, by 256 threads (two lengths), by 512; in two passes of 1024 and of 512 threads; in chunks
STEPS = [(1000, 5), (8001, 5), (10011, 520), (30011, 520), (40011, 40), (40011, 520), (150001, 33), (66001, 3), (140001, 2), (280001, 33),
         (1 << 20, 1)]


@pytest.mark.parametrize("tail,tau,hard", [(0, 1.0, 0.0), (1, 1.0, 0.0), (1, 2.0, 1.0), (1, 1.5, 1.0)])
@pytest.mark.parametrize("vocab,rows", STEPS)
def test_sums_count_every_word(bpc, vocab, rows, tail, tau, hard):  # noqa: F811
    """A uniform row, one word listed with half of the teacher's mass (TAIL_DROP: all of it): an unlisted word's gradient is
    c (1 / V - 0.5 / (V - 1)) + hard / V to at most seven roundings: two quotients, their difference, c, its product with
    that, the sum and the product with the hard weight."""
    import torch
    rs = np.random.default_rng(vocab + tail)
    at = rs.integers(0, vocab - 1, rows)
    d = describe(bpc, vocab, 1, tail=tail, temperature=tau, hard_weight=hard)
    msg = make_messages(bpc, d, [(1, [a], [0.0], 1.0, 0.0) for a in at])
    lab = torch.full((rows,), vocab - 1, device="cuda") if hard else None
    view = padded(rows, vocab, 3, "f32")
    ws = workspace(bpc, d, rows)
    loss, stats = torch.zeros(rows, device="cuda"), torch.zeros(rows, 32, dtype=torch.uint8, device="cuda")
    grads = [padded(rows, vocab, 1, "f32", 9.0) for _ in range(2)]
    print("words of a row", vocab, rows, tail, tau, hard, flush=True)
    bpc.bpc_distill_step(d, view, msg, lab, None, loss, grads[0], ws)
    bpc.bpc_distill_loss(d, view, msg, lab, None, loss, stats, ws)
    bpc.bpc_distill_grad(d, view, msg, lab, None, stats, grads[1])
    q, c = (0.5 if tail else 0.0), 1.0 / tau

    def slope(v):
        return c * (1.0 / v - q / (v - 1)) + hard / v
    want, bound = slope(vocab), 7 * U * (c * (1.0 / vocab + q / (vocab - 1)) + hard / vocab)
    assert abs(slope(vocab - 1) - want) > bound or vocab > 300000   # (what one lost word would do; a lost vector: four times that)
    assert abs(slope(vocab - 4) - want) > bound
    spot = torch.from_numpy(at).cuda()[:, None]
    for grad in grads:
        g = grad.double()
        listed = g.gather(1, spot)[:, 0]
        assert bool(((listed - (c * (1.0 / vocab - (1.0 - q)) + hard / vocab)).abs() <= 7 * U * (c + hard)).all())
        if hard:
            assert bool(((g[:, -1] - (want - hard)).abs() <= 7 * U * hard).all())
            g[:, -1] = want
        g.scatter_(1, spot, want)
        off = (g - want).abs() > bound
        assert not bool(off.any()), (torch.nonzero(off)[:5], float(g[off][0]), want)


@pytest.mark.parametrize("tail", [0, 1])
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("vocab,rows", [(1000, 5), (16001, 60), (20011, 520), (50257, 520), (50257, 20), (80011, 40), (80011, 520), (200001, 32),
                                        (280001, 32)])
def test_losses_count_every_word(bpc, vocab, rows, dtype, tail):  # noqa: F811
    """Row r has the words j with j % rows = r at 0 and masks all others, so that each word counts in one row: of its C words
    one is listed with half of the mass (TAIL_DROP: all of it).  The loss adds up to four logarithms of at most two steps
    each and as many additions: 16 u of their sizes."""
    import torch
    rs = np.random.default_rng(vocab + tail)
    view = padded(rows, vocab, 1, dtype, -math.inf)
    first = torch.arange(rows, device="cuda")
    view[torch.arange(vocab, device="cuda") % rows == first[:, None]] = 0.0
    count = np.array([len(range(r, vocab, rows)) for r in range(rows)], np.float64)
    at = np.arange(rows) + rows * rs.integers(0, count)
    d = describe(bpc, vocab, 1, tail=tail)
    msg = make_messages(bpc, d, [(1, [a], [0.0], 1.0, 0.0) for a in at.astype(np.int64)])
    ws = workspace(bpc, d, rows)
    loss, loss2 = torch.zeros(rows, device="cuda"), torch.zeros(rows, device="cuda")
    print("words of a loss", vocab, rows, dtype, tail, flush=True)
    bpc.bpc_distill_loss(d, view, msg, None, None, loss, None, ws)
    bpc.bpc_distill_step(d, view, msg, None, None, loss2, padded(rows, vocab, 2, dtype), ws)

    def kl(c):
        return 0.5 * (math.log(0.5) + np.log(c)) + 0.5 * (math.log(0.5) - np.log((c - 1) / c)) if tail else np.log(c)
    want, bound = kl(count), 16 * U * (np.log(count) + 2)
    assert (np.abs(kl(count - 1) - want) > 2 * bound).all()
    for got in (loss, loss2):
        assert (np.abs(host(got) - want) <= bound).all(), (host(got)[:4], want[:4])
