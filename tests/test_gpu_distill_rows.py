"""Rows of a student's call that one of its two terms, or both, leave out: on the GPU against the plain float64 forms
(distill_ref.py), in every form that a step and a loss with its gradient can take."""
import numpy as np
import pytest

from test_gpu_distill import DT, bpc, check_student, describe, make_case  # noqa: F401  (bpc: the fixture)

pytestmark = pytest.mark.gpu

# vocabulary, rows, entries, type: held by one wave; by 256 threads; by 256 and by 512 where there are rows enough; in two
# passes of 1024 and of 512 threads; in chunks
FORMS = [(900, 40, 20, "f32"), (9001, 40, 300, "bf16"), (20011, 520, 20, "f16"), (20011, 520, 20, "f32"), (40011, 40, 20, "bf16"),
         (33001, 520, 20, "f32"), (66001, 22, 20, "f32")]
BAD = {"nan": lambda x: x.__setitem__(len(x) // 3, np.nan), "nan all": lambda x: x.fill(np.nan), "infinite": lambda x: x.__setitem__(7, np.inf),
       "masked": lambda x: x.fill(-np.inf)}
EMPTY = (0, [], [], 0.5, 1.0)


def case(rs, vocab, rows, k, plan):
    """Logits, records and labels in which row r + 1 is plan[r]: (bad, empty record, hard label)."""
    x = rs.standard_normal((rows, vocab), dtype=np.float32) * 2
    small, record = make_case(rs, min(vocab, 2000), k, 1)
    records = [(record[0][0], record[0][1] * (vocab // min(vocab, 2000)), *record[0][2:])] * rows
    labels = [5] * rows
    for r, (bad, empty, hard) in enumerate(plan, 1):
        if bad:
            BAD[bad](x[r])
        records[r] = EMPTY if empty else records[r]
        labels[r] = vocab - 2 if hard else -100
    return x, records, labels


@pytest.mark.parametrize("tail,tau", [(0, 1.0), (1, 2.0), (1, 1.7)])
@pytest.mark.parametrize("vocab,rows,k,dtype", FORMS)
def test_rows_without_a_term(bpc, vocab, rows, k, dtype, tail, tau):  # noqa: F811
    """A row with an empty record and no hard label has loss 0 and gradient 0 whatever its logits are; one with either term
    and logits that have no softmax is NaN."""
    rs = np.random.default_rng(vocab + tail)
    plan = [(bad, empty, hard) for bad in (None, *BAD) for empty, hard in ((True, False), (True, True), (False, False), (False, True))]
    x, records, labels = case(rs, vocab, rows, k, plan)
    only = range(len(plan) + 2)

    def nan(has_term):
        return [r for r, (bad, empty, hard) in enumerate(plan, 1) if bad and has_term(not empty, hard)]

    def describe_with(soft, hard):
        return describe(bpc, vocab, k, tail=tail, temperature=tau, soft_weight=soft, hard_weight=hard)
    check_student(bpc, describe_with(1.0, 0.3), x, records, dtype, 1, 2, labels, want_nan=nan(lambda full, hard: full or hard), only=only)
    check_student(bpc, describe_with(1.0, 0.3), x, records, dtype, 1, 2, None, want_nan=nan(lambda full, hard: full), only=only)
    check_student(bpc, describe_with(0.0, 0.3), x, records, dtype, 1, 1, labels, want_nan=nan(lambda full, hard: hard), only=only, in_place=True)
    check_student(bpc, describe_with(0.0, 0.0), x, records, dtype, 1, 2, labels, only=only)


@pytest.mark.parametrize("tail", [0, 1])
@pytest.mark.parametrize("vocab,rows,k,dtype", FORMS)
def test_no_soft_term_from_a_record_of_nan(bpc, vocab, rows, k, dtype, tail):  # noqa: F811
    """soft_weight 0: values of a record that are no numbers (a teacher's NaN or +inf) leave the hard term as it is."""
    rs = np.random.default_rng(vocab + 7)
    x, records, labels = case(rs, vocab, rows, k, [])
    n, idx, _, _, _ = records[0]
    records[1] = (n, idx, np.full(n, np.nan), np.nan, np.nan)                           # a NaN in the teacher's row
    records[2] = (n, idx, np.where(np.arange(n) == 1, np.nan, -np.inf), 0.0, np.inf)    # +inf
    labels[1], labels[2], labels[3] = int(idx[0]), int(idx[1]), -100                    # (listed words; no term at all)
    records[3] = records[1]
    d = describe(bpc, vocab, k, tail=tail, temperature=2.0, soft_weight=0.0, hard_weight=0.4)
    check_student(bpc, d, x, records, dtype, 1, 1, labels, only=range(6), in_place=True)


def test_gradient_of_the_hard_term_alone(bpc):  # noqa: F811
    """bpc_distill_grad with soft_weight 0 from statistics of both terms: the hard term's gradient, also where the record's
    values are no numbers."""
    import torch
    import distill_ref as ref
    from test_gpu_distill import fields, host, make_messages, rows_of, workspace
    rs = np.random.default_rng(17)
    vocab, k = 1000, 12
    x, records, labels = case(rs, vocab, 4, k, [])
    n, idx, _, _, _ = records[0]
    records[1] = (n, idx, np.full(n, np.nan), np.nan, np.nan)
    labels[1], labels[3] = int(idx[3]), -100
    _, view = rows_of(x, "f32", 1)
    both = describe(bpc, vocab, k, tail=1, temperature=1.7, soft_weight=1.0, hard_weight=0.4)
    alone = describe(bpc, vocab, k, tail=1, temperature=1.7, soft_weight=0.0, hard_weight=0.4)
    msg, lab, ws = make_messages(bpc, both, records), torch.tensor(labels, device="cuda"), workspace(bpc, both, 4)
    loss, stats = torch.zeros(4, device="cuda"), torch.zeros(4, 32, dtype=torch.uint8, device="cuda")
    grad = torch.full((4, vocab), 7.0, device="cuda")
    bpc.bpc_distill_loss(both, view, msg, lab, None, loss, stats, ws)
    bpc.bpc_distill_grad(alone, view, msg, lab, None, stats, grad)
    count, at, val, rest, _ = fields(bpc, both, msg, 4)
    for r in range(4):
        _, want, _, bound = ref.student_row(host(view)[r], int(count[r]), at[r], val[r], rest[r], 1.7, 0.0, 0.4, True, labels[r], 1.0)
        bad = np.nonzero(~(np.abs(host(grad)[r] - want) <= bound))[0]
        assert not bad.size, (r, bad[:5])
    assert np.isnan(float(loss[1])) and np.isfinite(loss[[0, 2, 3]].cpu().numpy()).all()


@pytest.mark.parametrize("rows,vocab,k,dtype", [(1, 131072, 40, "f32"), (32, 131072, 40, "f32"), (3, 262144, 1024, "bf16"), (32, 32768, 700, "f16"),
                                                (2, 65536, 1000, "f32"), (5, 140001, 300, "f16"), (33, 270001, 20, "f32"), (300, 2000, 16, "bf16")])
def test_nothing_is_written_behind_the_workspace(bpc, rows, vocab, k, dtype):  # noqa: F811
    """Every call on a workspace of exactly the bytes that the sizing call answers, between guards."""
    import torch
    from test_gpu_distill import tdtype
    g = torch.Generator(device="cuda").manual_seed(vocab + rows)
    logits = torch.randn(rows, vocab, generator=g, device="cuda").to(tdtype(dtype))
    d = bpc.make_distill(bpc.TOPK, vocab, k, temperature=2.0, hard_weight=0.2, tail=bpc.TAIL_REST)
    size, edge = bpc.distill_workspace_bytes(d, rows), 4096
    buf = torch.full((size + 2 * edge,), 0x5A, dtype=torch.uint8, device="cuda")
    ws = buf[edge:edge + size]
    msg = torch.zeros(bpc.logits_message_bytes(d, rows), dtype=torch.uint8, device="cuda")
    lab = torch.arange(rows, device="cuda")
    loss, grad = torch.zeros(rows, device="cuda"), torch.empty_like(logits)
    print("guards", rows, vocab, k, dtype, size, flush=True)
    bpc.bpc_logits_topk(d, logits, None, msg, ws)
    bpc.bpc_distill_loss(d, logits, msg, lab, None, loss, None, ws)
    bpc.bpc_distill_step(d, logits, msg, lab, None, loss, grad, ws)
    torch.cuda.synchronize()
    assert bool((buf[:edge] == 0x5A).all()) and bool((buf[edge + size:] == 0x5A).all())
    assert bool(torch.isfinite(loss).all())
