"""Plain float64 forms of the distillation operators, row by row from their definition, and how far the
kernels' f32 arithmetic may be from them.

u = 2^-24 is half a step of f32.  An exponential exp2_hw((x - ref) * c2) has an argument with three
roundings (difference, c2, product), each relative to the argument, and one unit in the last place of its
own: its relative error is at most ln2 * 3u * |argument| + 2u.  A sum of positive terms adds n u for a
chain of n additions; `chain` counts the longest (a thread's elements and the reductions over threads)."""
import math

import numpy as np

U = 2.0 ** -24
LN2 = math.log(2.0)
LOG2E = 1.0 / LN2
TINY = 2.0 ** -120          # what exponentials that flush to 0 may lose, scaled freely
HALF_STEP = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}
SUBNORMAL = {"f32": 2.0 ** -126, "f16": 2.0 ** -25, "bf16": 2.0 ** -126}


def chain(vocab):
    """Additions in a row: a thread's share of a row (64 threads at least, 8 elements at a time) and the tree."""
    return min(vocab, vocab // 64 + 16) + 24


def exp_error(args):
    """Relative error of exponentials with these arguments (in powers of two)."""
    return LN2 * 3 * U * np.abs(args) + 2 * U


def topk_row(t, k, tau, half):
    """Fields of a record, the bound of `rest`'s error.  t: float32 values of the row."""
    t = np.asarray(t, np.float32)
    nan = np.isnan(t)
    key = np.where(nan, np.inf, t).astype(np.float64)
    order = np.lexsort((np.arange(t.size), -key, ~nan))       # NaN first, then the largest, then the lowest index
    order = order[(nan | (key > -np.inf))[order]][:k]
    idx = np.sort(order)
    top = np.float32(np.nan) if nan.any() else t.max() if t.size else np.float32(-np.inf)
    ref = np.float32(0.0) if top == -np.inf else top
    with np.errstate(all="ignore"):
        val = (t[idx] - ref).astype(np.float32)
        if half:
            val = val.astype(np.float16)
        others = np.delete(t.astype(np.float64), idx) - np.float64(ref)
        e = np.exp(others / tau)
        rest = e.sum()
        bound = (e * (exp_error(others / tau * LOG2E) + chain(t.size) * U))[others > -np.inf].sum() + TINY
    return idx, val, top, rest, bound


def student_row(s, n, idx, val, rest, tau, soft, hard, tail_rest, label, weight, out="f32"):
    """loss, gradient and the bounds of their errors.  s: values of the row; idx, val: the record's n entries."""
    s = np.asarray(s, np.float64)
    V = s.size
    if weight == 0.0:
        return 0.0, np.zeros(V), 0.0, np.zeros(V)
    c = 1.0 / tau
    with np.errstate(all="ignore"):
        def softmax(x):
            m = x.max() if x.size else -np.inf
            m = 0.0 if m == -np.inf else m
            e = np.exp(x - m)
            return m, e / e.sum(), (x - m) - np.log(e.sum())   # (differences first: m may be the type's lowest value)
        m, p, logp = softmax(s * c)
        lse = np.log(np.exp(s * c - m).sum())                  # relative to m
        use = np.asarray(idx[:n], np.int64)
        v = np.asarray(val[:n], np.float64)
        e = np.exp(v * c)
        r = float(rest) if tail_rest else 0.0
        Q = e.sum() + r
        soft_on = n > 0 and Q != 0.0 and soft != 0.0
        kl, kl_err = 0.0, 0.0
        d_sum = (chain(V) + 4) * U + float((p[p > 0] * exp_error(logp[p > 0] * LOG2E)).sum()) + 2 * U
        g = np.zeros(V)
        g_abs = np.zeros(V)
        if soft_on:
            q = e / Q
            d_q = (n + 24) * U + float((q[q > 0] * exp_error(v[q > 0] * c * LOG2E)).sum()) + 2 * U
            live = ~(q == 0)
            ratio = np.log(q) - logp[use]
            kl = (q * ratio)[live].sum()
            sizes = np.abs(v) * c + np.abs(logp[use]) + abs(math.log(Q)) + np.abs(lse) + 4
            kl_err = float((q * (sizes * (8 * U + exp_error(v * c * LOG2E) + d_q) + d_sum + d_q))[live].sum())
            if tail_rest and r != 0.0:
                out_of = np.ones(V, bool)
                out_of[use] = False
                mr, pr, _ = softmax(s[out_of] * c)
                log_rest = (mr - m) + (np.log(np.exp(s[out_of] * c - mr).sum()) - lse)
                q_r = r / Q
                kl += q_r * (math.log(q_r) - log_rest)
                kl_err += q_r * ((abs(log_rest) + abs(math.log(q_r)) + 4) * (10 * U + d_q) + 3 * d_sum + d_q)
                share = np.zeros(V)
                share[out_of] = np.where(s[out_of] == -np.inf, 0.0, q_r * pr)
                g -= share
                g_abs += share
            g += p
            g_abs += p
            np.subtract.at(g, use, q)
            np.add.at(g_abs, use, q)
            g *= soft * c
            g_abs = g_abs * abs(soft * c)
            g_err = g_abs * (3 * d_sum + d_q + 16 * U)
            arg = np.where(s == -np.inf, 0.0, np.abs(logp)) * LOG2E
            g_err += g_abs * exp_error(2 * arg)
        else:
            g_err = np.zeros(V)
        loss, loss_err = soft * kl, abs(soft) * kl_err
        if hard != 0.0 and label is not None and 0 <= label < V:
            m1, p1, logp1 = softmax(s)
            ce = -logp1[label]
            lse1 = np.log(np.exp(s - m1).sum())
            loss += hard * ce
            d1 = (chain(V) + 4) * U + float((p1[p1 > 0] * exp_error(logp1[p1 > 0] * LOG2E)).sum()) + 2 * U
            loss_err += abs(hard) * (d1 + (abs(ce) + abs(lse1) + 4) * 6 * U)
            g += hard * p1
            arg1 = np.where(s == -np.inf, 0.0, np.abs(logp1)) * LOG2E
            g_err += abs(hard) * p1 * (3 * d1 + 16 * U + exp_error(2 * arg1))
            g[label] -= hard
            g_err[label] += abs(hard) * 4 * U
        loss_err = abs(weight) * (loss_err + 4 * U * abs(loss)) + TINY
        g *= weight
        g_err = abs(weight) * g_err + TINY
        g_err = g_err + (np.abs(g) + g_err) * HALF_STEP[out] * (0 if out == "f32" else 1) + SUBNORMAL[out] + np.abs(g) * 2 * U
    return weight * loss, g, loss_err, g_err
