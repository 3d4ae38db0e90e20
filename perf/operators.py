"""Distillation from a teacher's top logits, as cases that can be timed and compared.

A case is one role of a training job in which teachers send students their top logits as top-k
messages, called through the public entry points of ``paper_2105_07829_amd``:

  topk    a teacher compresses its logits, one record a row: ``bpc_logits_topk``
  loss    a student's loss against the messages (validation): ``bpc_distill_loss``
  train   loss and gradient as two calls, as an autograd engine makes them: ``bpc_distill_loss``,
          ``bpc_distill_grad``
  step    loss and gradient in one call: ``bpc_distill_step``

Where ``own`` is false, the same is computed by elementary torch operations.

With teacher logits t, student logits s, c = 1 / temperature and S the entries of a row's record:

  record   top = max t, val_i = t_i - top for the k largest t_i in index order (ties: lowest index;
           -inf is not listed), rest = sum over j not in S of exp((t_j - top) c)
  loss     w (a KL + b CE), Q = sum_S exp(val_i c) + rest, q_i = exp(val_i c) / Q, q_R = rest / Q,
           p = softmax(s c), KL = sum_S q_i log(q_i / p_i) + q_R log(q_R / p_R), CE = -log softmax(s)[label]
           ("rest" counts only where the case's tail is "rest"; p_R = sum of p outside S)
  gradient w (a c (p_j - q_j) + b (softmax(s)_j - [j = label])) for j in S,
           w (a c p_j (1 - q_R / p_R) + b (softmax(s)_j - [j = label])) for the others

Rows of weight 0 have loss 0 and gradient 0; a label outside the vocabulary has no hard term.
"""
from __future__ import annotations

import math

import torch

own = False

DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
BYTES = {"f32": 4, "f16": 2, "bf16": 2}
DEFAULTS = {"kind": "topk16", "tau": 1.0, "soft": 1.0, "hard": 0.0, "tail": "drop", "pad": 0, "masked": "no", "idle": 0}


def listed():
    return [
        # a teacher that serves one token of an odd vocabulary: latency of a single row
        {"name": "topk_one_row", "role": "topk", "rows": 1, "vocab": 50257, "k": 32, "dtype": "f32", "kind": "topk"},
        # a teacher of image classes (1000 logits): rows that one wave holds
        {"name": "topk_classes", "role": "topk", "rows": 256, "vocab": 1000, "k": 10, "dtype": "f32", "kind": "topk"},
        # a teacher over a batch of tokens, odd vocabulary, so that rows start at any even byte
        {"name": "topk_batch", "role": "topk", "rows": 4096, "vocab": 50257, "k": 64, "dtype": "bf16", "tau": 2.0,
         "masked": "lowest", "idle": 7},
        # a teacher over a large batch and a large vocabulary, many entries a row
        {"name": "topk_large", "role": "topk", "rows": 8192, "vocab": 131072, "k": 256, "dtype": "bf16"},
        # validation loss of a few tokens of a very large vocabulary: few rows, long axis
        {"name": "loss_few_rows", "role": "loss", "rows": 8, "vocab": 151936, "k": 64, "dtype": "bf16", "tail": "rest"},
        # validation loss of a batch with the vocabulary of BERT and padded rows, mass of the rest counted
        {"name": "loss_batch", "role": "loss", "rows": 2047, "vocab": 30522, "k": 20, "dtype": "f16", "kind": "topk",
         "tau": 2.0, "tail": "rest", "pad": 6, "idle": 5},
        # forward and backward as two calls, f32 logits
        {"name": "train_f32", "role": "train", "rows": 1024, "vocab": 32000, "k": 50, "dtype": "f32", "kind": "topk",
         "tail": "rest"},
        # forward and backward as two calls on a batch of tokens: odd vocabulary, temperature, hard labels, padding
        {"name": "train_batch", "role": "train", "rows": 4096, "vocab": 50257, "k": 64, "dtype": "bf16", "tau": 2.0,
         "soft": 3.6, "hard": 0.1, "masked": "lowest", "idle": 7},
        # image classes in one call, hard labels, one wave a row
        {"name": "step_classes", "role": "step", "rows": 256, "vocab": 1000, "k": 10, "dtype": "f32", "kind": "topk",
         "tau": 4.0, "soft": 14.4, "hard": 0.1},
        # a short micro-batch: fewer rows than compute units
        {"name": "step_short", "role": "step", "rows": 61, "vocab": 128000, "k": 128, "dtype": "bf16", "tail": "rest"},
        # the vocabulary of BERT in f16 with rows padded to a multiple of 16 bytes, hard labels, mass of the rest
        {"name": "step_batch", "role": "step", "rows": 2048, "vocab": 30522, "k": 20, "dtype": "f16", "tau": 2.0,
         "soft": 3.2, "hard": 0.2, "tail": "rest", "pad": 6, "idle": 5},
        # the largest: a large batch of tokens over a large vocabulary in one call
        {"name": "step_large", "role": "step", "rows": 8192, "vocab": 131072, "k": 256, "dtype": "bf16", "tail": "rest"},
    ]


LARGEST = 8192 * 131072


def _log_between(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    role = rng.choice(("topk", "loss", "train", "step"))
    dtype = rng.choice(("f32", "f16", "bf16", "bf16"))
    vocab = _log_between(rng, 100, 262144)
    k = min(_log_between(rng, 1, 1024), vocab)
    rows = _log_between(rng, 1, 16384)
    # (train passes over the logits twice, f32 moves twice the bytes: at most the largest listed case's cost)
    rows = max(1, min(rows, LARGEST // (vocab * (BYTES[dtype] // 2) * (2 if role == "train" else 1))))
    hard = role != "topk" and rng.random() < 0.5
    return {"role": role, "rows": rows, "vocab": vocab, "k": k, "dtype": dtype,
            "kind": rng.choice(("topk", "topk16")), "tau": rng.choice((1.0, 1.0, 0.7, 2.0, 4.0)),
            "soft": rng.choice((1.0, 0.9, 3.6)), "hard": rng.choice((0.1, 0.5)) if hard else 0.0,
            "tail": rng.choice(("drop", "rest")), "pad": rng.choice((0, 0, 1, rng.randrange(2, 64))),
            "masked": rng.choice(("no", "lowest", "inf")), "idle": rng.choice((0, rng.randrange(2, 17)))}


def _full(case):
    return {**DEFAULTS, **case}


def _ru4(x):
    return -(-x // 4) * 4


def _stride(kind, k):
    return 16 + 4 * _ru4(k) + (4 * _ru4(k) if kind == "topk" else 4 * _ru4(-(-k // 2)))


def _fields(messages, kind, k):
    """The fields of the records of ``messages`` (uint8 [rows, stride]) as views."""
    words = messages.view(torch.int32)
    at = 4 + _ru4(k)
    val = words.view(torch.float32)[:, at:at + k] if kind == "topk" else messages.view(torch.float16)[:, 2 * at:2 * at + k]
    return {"count": words[:, 0], "rest": words.view(torch.float32)[:, 1], "top": words.view(torch.float32)[:, 2],
            "idx": words[:, 4:4 + k], "val": val}


def prepare(case, seed):
    c = _full(case)
    rows, vocab, k, dt = c["rows"], c["vocab"], c["k"], DTYPES[c["dtype"]]
    gen = torch.Generator(device="cuda").manual_seed(seed)
    rand = lambda *shape: torch.rand(shape, generator=gen, device="cuda")  # noqa: E731
    # logits: a frequency a word, noise a row, a spread that differs between rows
    buf = torch.empty(rows, vocab + c["pad"], dtype=dt, device="cuda")
    logits = buf[:, :vocab]
    spread = 1.0 + 1.5 * rand(rows, 1)
    logits.copy_(torch.randn(rows, vocab, generator=gen, device="cuda").mul_(spread).add_(-1.5 * rand(vocab).add_(1e-3).log_().neg_()))
    used = vocab if c["masked"] == "no" else max(1, vocab - max(1, vocab // 50))  # the rest pads the vocabulary
    if used < vocab:
        logits[:, used:] = -math.inf if c["masked"] == "inf" else torch.finfo(dt).min
    weight = None
    if c["idle"]:  # padding tokens
        weight = 0.5 + rand(rows)
        weight[c["idle"] - 1::c["idle"]] = 0.0
    state = {"case": c, "logits": logits, "weight": weight}
    if c["role"] == "topk":
        if c["masked"] == "inf":  # a few rows restricted to a few words
            logits[3::64, 5:] = -math.inf
        state["messages"] = torch.zeros(rows, _stride(c["kind"], k), dtype=torch.uint8, device="cuda")
    else:
        n = min(k, used)
        messages = torch.zeros(rows, _stride(c["kind"], k), dtype=torch.uint8, device="cuda")
        f = _fields(messages, c["kind"], k)
        f["idx"][:] = -1
        f["val"][:] = -math.inf
        # distinct words in ascending order, one of each of n stretches; the student knows them in part
        first = torch.arange(n + 1, device="cuda") * used // n
        at = first[:-1] + torch.minimum((rand(rows, n) * first.diff()).long(), first.diff() - 1)
        val = rand(rows, n).clamp_(min=1e-6).log_().mul_(2.0)
        val -= val.amax(1, keepdim=True)
        f["count"][:] = n
        f["idx"][:, :n] = at.int()
        f["val"][:, :n] = val.to(f["val"].dtype)
        f["top"][:] = 4.0 + 8.0 * rand(rows)
        f["rest"][:] = rand(rows) * (0.5 if n < used else 0.0)
        near = 9.0 + 0.8 * val + torch.randn(rows, n, generator=gen, device="cuda")
        logits.scatter_(1, at, near.to(dt))
        state["messages"] = messages
        state["labels"] = None
        if c["hard"]:
            lab = (rand(rows).double() * used).long().clamp_(max=used - 1)
            lab[::2] = at[::2, 0]
            lab[15::16] = -100
            state["labels"] = lab
        state["loss"] = torch.zeros(rows, device="cuda")
        if c["role"] != "loss":
            state["grad"] = torch.zeros_like(buf)[:, :vocab]
        if c["role"] == "train":
            state["stats"] = torch.zeros(rows, 32, dtype=torch.uint8, device="cuda")
    if own:  # the description and the workspace that a program keeps from call to call
        import paper_2105_07829_amd as bpc

        d = bpc.make_distill(bpc.TOPK if c["kind"] == "topk" else bpc.TOPK16, vocab, k, temperature=c["tau"],
                             soft_weight=c["soft"], hard_weight=c["hard"],
                             tail=bpc.TAIL_REST if c["tail"] == "rest" else bpc.TAIL_DROP)
        state["plan"] = bpc, d, torch.empty(bpc.distill_workspace_bytes(d, rows), dtype=torch.uint8, device="cuda")
    return state


def run(state):
    c = state["case"]
    if own:
        bpc, d, ws = state["plan"]
        if c["role"] == "topk":
            bpc.bpc_logits_topk(d, state["logits"], state["weight"], state["messages"], ws)
            return _fields(state["messages"], c["kind"], c["k"])
        args = (d, state["logits"], state["messages"], state["labels"], state["weight"])
        if c["role"] == "loss":
            bpc.bpc_distill_loss(*args, state["loss"], None, ws)
            return {"loss": state["loss"]}
        if c["role"] == "train":
            bpc.bpc_distill_loss(*args, state["loss"], state["stats"], ws)
            bpc.bpc_distill_grad(*args, state["stats"], state["grad"])
        else:
            bpc.bpc_distill_step(*args, state["loss"], state["grad"], ws)
        return {"loss": state["loss"], "grad": state["grad"]}
    if c["role"] == "topk":
        return _topk_plain(c, state["logits"].float(), state["weight"])
    return _distill_plain(c, state)


def _topk_plain(c, t, weight):
    rows, vocab, k = c["rows"], c["vocab"], c["k"]
    if weight is not None:
        t = torch.where(weight[:, None] == 0, -math.inf, t)
    kth = torch.topk(t, min(k, vocab), dim=1).values[:, -1:]
    above, level = t > kth, (t == kth) & (t > -math.inf)
    # of the words level with the k-th, the first ones
    left = min(k, vocab) - above.sum(1, keepdim=True)
    keep = above | (level & (torch.cumsum(level, 1, dtype=torch.int32) <= left))
    place = torch.cumsum(keep, 1, dtype=torch.int32) - 1
    row, word = torch.nonzero(keep, as_tuple=True)
    at = row * k + place[row, word]
    top = t.amax(1, keepdim=True)
    diff = t - torch.where(top > -math.inf, top, 0.0)
    idx = torch.full((rows * k,), -1, dtype=torch.int32, device=t.device)
    val = torch.full((rows * k,), -math.inf, device=t.device)
    idx[at] = word.int()
    val[at] = diff[row, word]
    rest = torch.where(keep, 0.0, torch.exp(diff * (1.0 / c["tau"]))).sum(1)
    return {"count": keep.sum(1, dtype=torch.int32), "rest": rest, "top": top[:, 0], "idx": idx.view(rows, k),
            "val": val.view(rows, k).to(torch.float32 if c["kind"] == "topk" else torch.float16)}


def _softmax_parts(s, over):
    """Largest value, exponentials relative to it and their sum, over the words that ``over`` marks."""
    if over is not None:
        s = torch.where(over, s, -math.inf)
    m = s.amax(1, keepdim=True)
    m = torch.where(m > -math.inf, m, 0.0)
    e = torch.exp(s - m)
    return m, e, e.sum(1, keepdim=True)


def _distill_plain(c, state):
    inv = 1.0 / c["tau"]
    s, f = state["logits"].float(), _fields(state["messages"], c["kind"], c["k"])
    rows, vocab = s.shape
    used = torch.arange(c["k"], device=s.device)[None] < f["count"][:, None]
    at = torch.where(used, f["idx"], 0).long()
    e = torch.where(used, torch.exp(f["val"].float() * inv), 0.0)
    rest = f["rest"][:, None] if c["tail"] == "rest" else torch.zeros(rows, 1, device=s.device)
    total = e.sum(1, keepdim=True) + rest
    q, q_rest = e / total, rest / total
    m, es, z = _softmax_parts(s * inv, None)
    log_p = s.gather(1, at) * inv - m - torch.log(z)
    log_q = f["val"].float() * inv - torch.log(total)
    kl = torch.where(q > 0, q * (log_q - log_p), 0.0).sum(1, keepdim=True)
    p = es / z
    if c["tail"] == "rest":
        outside = torch.ones(rows, vocab + 1, dtype=torch.bool, device=s.device)
        outside.scatter_(1, torch.where(used, f["idx"], vocab).long(), False)
        outside = outside[:, :vocab]
        mr, er, zr = _softmax_parts(s * inv, outside)
        some = q_rest > 0
        log_p_rest = mr + torch.log(zr) - m - torch.log(z)
        kl = kl + torch.where(some, q_rest * (torch.log(q_rest) - log_p_rest), 0.0)
    loss = c["soft"] * kl
    if state["labels"] is not None:
        m1, e1, z1 = _softmax_parts(s, None)
        lab = state["labels"][:, None]
        given = (lab >= 0) & (lab < vocab)
        lab = torch.where(given, lab, 0)
        ce = m1 + torch.log(z1) - s.gather(1, lab)
        loss = loss + c["hard"] * torch.where(given, ce, 0.0)
    w = state["weight"][:, None] if state["weight"] is not None else torch.ones(rows, 1, device=s.device)
    loss = torch.where(w == 0, 0.0, w * loss)[:, 0]
    if c["role"] == "loss":
        return {"loss": loss}
    g = p.scatter_add(1, at, -q)
    if c["tail"] == "rest":
        g = g - torch.where(some & outside, q_rest * er / zr, 0.0)
    g = g * (c["soft"] * inv)
    if state["labels"] is not None:
        hard = (e1 / z1).scatter_add(1, lab, torch.full_like(z1, -1.0))
        g = g + c["hard"] * torch.where(given, hard, 0.0)
    return {"loss": loss, "grad": torch.where(w == 0, 0.0, w * g).to(state["logits"].dtype)}


def work(case):
    c = _full(case)
    rows = c["rows"] - (c["rows"] // c["idle"] if c["idle"] else 0)  # rows of weight 0 are not read
    size, message = BYTES[c["dtype"]], _stride(c["kind"], c["k"])
    if c["role"] == "topk":
        return {"bytes": rows * c["vocab"] * size + c["rows"] * (message + (4 if c["idle"] else 0)), "flops": 5 * rows * c["vocab"]}
    some = c["rows"] * (4 + (4 if c["idle"] else 0) + (8 if c["hard"] else 0)) + rows * message
    exps = 2 if c["hard"] and c["tau"] != 1.0 else 1
    if c["role"] == "loss":
        return {"bytes": rows * c["vocab"] * size + some, "flops": (2 + 3 * exps) * rows * c["vocab"]}
    return {"bytes": (rows + c["rows"]) * c["vocab"] * size + some, "flops": (2 + 7 * exps) * rows * c["vocab"]}


def exact(case, seed):
    """What ``run`` returns, row block by row block from the definition in float64."""
    state = prepare(case, seed)
    c, logits, weight = state["case"], state["logits"], state["weight"]
    block = max(1, (1 << 26) // c["vocab"])
    parts = []
    for r in range(0, c["rows"], block):
        x = logits[r:r + block].double()
        w = None if weight is None else weight[r:r + block].double()
        if c["role"] == "topk":
            parts.append(_topk_exact(c, x, w))
        else:
            lab = None if state["labels"] is None else state["labels"][r:r + block]
            parts.append(_distill_exact(c, x, state["messages"][r:r + block], lab, w))
    return {name: torch.cat([part[name] for part in parts]) for name in parts[0]}


def _topk_exact(c, t, w):
    k = c["k"]
    if w is not None:
        t[w == 0] = -math.inf
    value, word = torch.sort(t, dim=1, descending=True, stable=True)
    value, word = value[:, :k], word[:, :k]
    count = (value > -math.inf).sum(1)
    word = torch.where(value > -math.inf, word, 1 << 30).sort(1).values  # (index order, unused places last)
    some = word < (1 << 30)
    top = t.max(1).values
    ref = torch.where(count > 0, top, 0.0)[:, None]
    listed_ = torch.zeros(t.shape[0], c["vocab"] + 1, dtype=torch.bool, device=t.device)  # (a column for unused places)
    listed_.scatter_(1, torch.where(some, word, c["vocab"]), True)
    weigh = torch.exp((t - ref) / c["tau"]).masked_fill(listed_[:, :-1], 0.0)
    val = torch.where(some, t.gather(1, torch.where(some, word, 0)) - ref, -math.inf)
    idx = torch.where(some, word, -1).int()
    return {"count": count.int(), "rest": weigh.sum(1), "top": top, "idx": idx, "val": val}


def _distill_exact(c, s, messages, labels, w):
    f = _fields(messages, c["kind"], c["k"])
    rows, vocab = s.shape
    # the teacher's distribution, dense, one more column for the padding of the records
    dense = torch.zeros(rows, vocab + 1, dtype=torch.float64, device=s.device)
    listed_ = torch.zeros(rows, vocab + 1, dtype=torch.bool, device=s.device)
    at = torch.where(f["idx"] >= 0, f["idx"], vocab).long()
    dense.scatter_(1, at, torch.exp(f["val"].double() / c["tau"]))
    listed_.scatter_(1, at, True)
    dense, listed_ = dense[:, :vocab], listed_[:, :vocab]
    rest = f["rest"].double() if c["tail"] == "rest" else torch.zeros(rows, dtype=torch.float64, device=s.device)
    total = dense.sum(1) + rest
    q, q_rest = dense / total[:, None], rest / total
    lsm = torch.log_softmax(s / c["tau"], 1)
    kl = torch.where(q > 0, q * (q.log() - lsm), 0.0).sum(1)
    g = lsm.exp() - q
    if c["tail"] == "rest":
        away = lsm.masked_fill(listed_, -math.inf)
        log_rest = torch.logsumexp(away, 1)
        kl = kl + torch.where(q_rest > 0, q_rest * (q_rest.log() - log_rest), 0.0)
        g = g - torch.where(q_rest > 0, q_rest, 0.0)[:, None] * torch.nan_to_num(torch.exp(away - log_rest[:, None]), nan=0.0)
    loss, g = c["soft"] * kl, g * (c["soft"] / c["tau"])
    if labels is not None:
        given = labels >= 0
        lab = labels.clamp(min=0)[:, None]
        hard = torch.log_softmax(s, 1)
        loss = loss - c["hard"] * torch.where(given, hard.gather(1, lab)[:, 0], 0.0)
        hard = hard.exp()
        hard.scatter_add_(1, lab, torch.full((rows, 1), -1.0, dtype=torch.float64, device=s.device))
        g = g + c["hard"] * torch.where(given[:, None], hard, 0.0)
    if w is not None:
        loss = torch.where(w == 0, 0.0, w * loss)
        g = torch.where((w == 0)[:, None], 0.0, w[:, None] * g)
    return {"loss": loss} if c["role"] == "loss" else {"loss": loss, "grad": g}
