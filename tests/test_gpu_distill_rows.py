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
