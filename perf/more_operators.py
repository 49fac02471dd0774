"""What the operators around experts, 8-bit integers and distillation are measured on: the matrix product
in 8-bit integers with a scale per row of either operand, the products of rows grouped by expert (forward
and both gradients in bf16, forward in 8-bit integers), and the loss of a student against a teacher's top
logits with its gradient.

``run`` makes one pass through one operator.  With ``own`` false it is written out in elementary torch
operations in fp32, rounded once at the end; with ``own`` true it makes the calls a user of the library
makes.  ``exact`` evaluates the same definitions in fp64.

Definitions
  int8      y = X W^T in 8-bit integers.  A row of X (quantised in the call) or W (kept quantised) with the
            largest magnitude a (2^-110 if that is larger) has the scale a / 127 and the codes x (127 / a),
            rounded to nearest even, both quotients in fp32; y is the sum of products of codes times both scales.
  experts   Rows are sorted by expert, expert e has rows offsets[e] to offsets[e + 1] and the matrix W_e
            (n x k): Y = X W_e^T.  Some experts have no rows.
  gradient  dX = dY W_e, and dW_e = dY^T X over the rows of e (zeros for an expert without rows).
  distill   Student logits s, teacher's logits z at up to ``top`` places id of each row (others are -1 and
            absent), temperature T, weight a of the teacher's part:
              p = softmax(z / T) over the places present,  q = softmax(s / T),  q1 = softmax(s)
              loss = a T^2 sum p (log p - log q[id]) + (1 - a) (-log q1[label])
            without the first part where no place is present, without the second where the label is -1;
            dlogits = w (a T (q - p at id) + (1 - a) (q1 - 1 at label)) for a weight w of each row.
"""
import math

import numpy as np
import torch

own = False

_DT = {"f32": torch.float32, "bf16": torch.bfloat16}
_TINY = 2.0 ** -110


# ----------------------------------------------------------------------------------- the cases
def listed():
    return [
        # Generation: four sequences advance by one token through one layer kept in 8-bit integers.
        dict(name="int8_tokens", op="int8", tokens=4, k=4096, n=4096, x="bf16", out="bf16"),
        # A prompt of odd length through a layer of odd widths.
        dict(name="int8_odd_prompt", op="int8", tokens=777, k=1003, n=2505, x="f32", out="f32"),
        # The forward pass of a large layer over a long batch.
        dict(name="int8_forward", op="int8", tokens=8192, k=4096, n=8192, x="bf16", out="bf16"),
        # Generation: 16 tokens with two experts each out of 16; the weights of the experts met are all there is.
        dict(name="experts_tokens", op="experts", rows=32, experts=16, k=2048, n=4096, out="bf16"),
        # A prompt through experts kept in 8-bit integers.
        dict(name="experts_int8", op="experts8", rows=4096, experts=16, k=2048, n=4096, x="bf16", out="bf16"),
        # A ragged batch over many small experts, widths that are no multiples of a tile.
        dict(name="experts_ragged", op="experts", rows=5003, experts=60, k=1000, n=1448, out="f32"),
        # The forward pass of a large layer in training.
        dict(name="experts_forward", op="experts", rows=32768, experts=8, k=4096, n=8192, out="bf16"),
        # Both gradients of small experts over a short ragged batch.
        dict(name="gradient_ragged", op="gradient", rows=3001, experts=12, k=1000, n=648, out="bf16"),
        # Both gradients of a large layer.
        dict(name="gradient_large", op="gradient", rows=32768, experts=8, k=4096, n=4096, out="bf16"),
        # A short batch against a teacher: loss and gradient in fp32, where latency counts.
        dict(name="distill_tokens", op="distill", tokens=32, vocab=32000, top=32, logits="f32", teacher="f32", ids="i64",
             temperature=1.0, alpha=1.0, grad=True),
        # Evaluation: the loss alone, a vocabulary of odd size, labels beside the teacher.
        dict(name="distill_evaluate", op="distill", tokens=4096, vocab=50021, top=100, logits="bf16", teacher="bf16", ids="i32",
             temperature=1.0, alpha=0.5, grad=False),
        # A training step on a large vocabulary: loss and gradient, labels and a raised temperature.
        dict(name="distill_large", op="distill", tokens=4096, vocab=131072, top=64, logits="bf16", teacher="f32", ids="i64",
             temperature=2.0, alpha=0.5, grad=True),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _width(rng, lo, hi):
    """A layer's width: a multiple of 128, of 8, or anything."""
    m = rng.choice([1, 8, 128])
    return max(lo, _log_int(rng, lo, hi) // m * m)


def draw(rng):
    op = rng.choice(["int8", "experts", "experts8", "gradient", "distill", "distill"])
    if op == "distill":
        while True:
            case = dict(op=op, tokens=_log_int(rng, 1, 8192), vocab=_log_int(rng, 1000, 151000), top=_log_int(rng, 1, 256),
                        logits=rng.choice(["bf16", "f32"]), teacher=rng.choice(["bf16", "f32"]), ids=rng.choice(["i32", "i64"]),
                        temperature=rng.choice([1.0, round(rng.uniform(0.5, 4.0), 2)]), alpha=rng.choice([1.0, 0.5, round(rng.uniform(0.1, 0.9), 2)]),
                        grad=rng.random() < 0.7)
            if case["tokens"] * case["vocab"] * (2 if case["logits"] == "f32" else 1) <= 4096 * 131072:
                return case
    while True:
        rows, k, n = _log_int(rng, 1, 32768), _width(rng, 96, 8192), _width(rng, 96, 8192)
        experts = 1 if op == "int8" else _log_int(rng, 2, 128)
        if rows * k * n <= 32768 * 4096 * 4096 and experts * k * n <= 8 * 4096 * 8192 and rows * k * n >= 1 << 18:
            break
    if op == "int8":
        return dict(op=op, tokens=rows, k=k, n=n, x=rng.choice(["bf16", "f32"]), out=rng.choice(["bf16", "f32"]))
    case = dict(op=op, rows=rows, experts=experts, k=k, n=n, out=rng.choice(["bf16", "f32"]))
    if op == "experts8":
        case["x"] = rng.choice(["bf16", "f32"])
    return case


def _shares(experts):
    """How often the experts are chosen: the favourite eight times as often as the rarest."""
    p = 8.0 ** -(np.arange(experts) / max(1, experts - 1))
    return p / p.sum()


def _met(rows, experts):
    """Expected number of experts with rows."""
    return float((1.0 - (1.0 - _shares(experts)) ** rows).sum())


def work(case):
    op = case["op"]
    size = {"f32": 4, "bf16": 2, "i32": 4, "i64": 8}
    if op == "distill":
        t, v, top = case["tokens"], case["vocab"], case["top"]
        labels = size[case["ids"]] if case["alpha"] < 1.0 else 0
        return {"bytes": t * v * size[case["logits"]] * (2 if case["grad"] else 1) + t * (top * (size[case["teacher"]] + size[case["ids"]]) + labels + 4),
                "flops": t * v * (6 if case["grad"] else 3)}
    k, n = case["k"], case["n"]
    if op == "int8":
        t = case["tokens"]
        return {"bytes": t * k * size[case["x"]] + n * (k + 4) + t * n * size[case["out"]], "flops": 2 * t * k * n}
    rows = case["rows"]
    met = _met(rows, case["experts"])
    if op == "experts8":
        return {"bytes": rows * k * size[case["x"]] + met * n * (k + 4) + rows * n * size[case["out"]], "flops": 2 * rows * k * n}
    if op == "experts":
        return {"bytes": 2 * (rows * k + met * n * k) + rows * n * size[case["out"]], "flops": 2 * rows * k * n}
    return {"bytes": 2 * (rows * (k + n) + met * n * k) + rows * k * size[case["out"]] + 4 * case["experts"] * n * k, "flops": 4 * rows * k * n}


# ----------------------------------------------------------------------------------- the inputs
def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) * 1000003 + 29)
    return g


def _activations(rows, cols, g, dtype):
    """Normal values; one column in 64 is larger by a factor of 16, as layer outputs have them."""
    x = torch.randn(rows, cols, generator=g, device="cuda")
    x *= torch.where(torch.rand(cols, generator=g, device="cuda") < 1 / 64, 16.0, 1.0)
    return x.to(dtype)


def _neural_gradient(rows, cols, g):
    """Lognormal magnitudes with random signs, two in five exactly zero."""
    x = torch.exp(-12.0 + 2.0 * torch.randn(rows, cols, generator=g, device="cuda"))
    u = torch.rand(rows, cols, generator=g, device="cuda")
    return torch.where(u < 0.3, x, torch.where(u < 0.6, -x, torch.zeros_like(x))).to(torch.bfloat16)


def _inputs(case, seed):
    """The tensors of a case, from the seed alone."""
    g, op = _gen(seed), case["op"]
    if op == "distill":
        t, v, top = case["tokens"], case["vocab"], case["top"]
        it = torch.int64 if case["ids"] == "i64" else torch.int32
        # different places in a row: steps of at least 1 that add up to less than the vocabulary
        step = 1 + (torch.rand(t, top, generator=g, device="cuda") * (v // top - 1)).long()
        ids = (torch.cumsum(step, 1) + torch.randint(0, v, (t, 1), generator=g, device="cuda")) % v
        z = 14.0 - 6.0 * torch.rand(t, 1, generator=g, device="cuda") * torch.linspace(0.0, 1.0, top, device="cuda") - torch.rand(t, top, generator=g, device="cuda")
        s = 2.0 * torch.randn(t, v, generator=g, device="cuda")
        s.scatter_(1, ids, z + torch.randn(t, top, generator=g, device="cuda"))
        # one row in eight has a shorter list, one of 32 none at all
        u, short = torch.rand(t, 1, generator=g, device="cuda"), torch.randint(0, top + 1, (t, 1), generator=g, device="cuda")
        count = torch.where(u < 1 / 32, 0, torch.where(u < 5 / 32, short, top))
        labels = torch.where(torch.rand(t, generator=g, device="cuda") < 0.6, ids[:, 0], torch.randint(0, v, (t,), generator=g, device="cuda"))
        labels = torch.where(torch.rand(t, generator=g, device="cuda") < 0.1, -1, labels)
        ids = torch.where(torch.arange(top, device="cuda") < count, ids, -1)
        return {"logits": s.to(_DT[case["logits"]]), "ids": ids.to(it), "teacher": z.to(_DT[case["teacher"]]),
                "labels": labels.to(it) if case["alpha"] < 1.0 else None,
                "weight": torch.rand(t, generator=g, device="cuda") / t if case["grad"] else None}
    k, n = case["k"], case["n"]
    if op == "int8":
        return {"x": _activations(case["tokens"], k, g, _DT[case["x"]]), "w": (torch.randn(n, k, generator=g, device="cuda") / math.sqrt(k)).to(torch.bfloat16)}
    e, rows = case["experts"], case["rows"]
    host = np.random.RandomState((int(seed) * 7919 + 11) % (1 << 31))
    sizes = [int(c) for c in host.multinomial(rows, host.permutation(_shares(e)))]
    d = {"sizes": sizes, "offsets": torch.tensor([0] + sizes, dtype=torch.int64).cumsum(0).to(torch.int32).cuda(),
         "x": _activations(rows, k, g, _DT[case["x"]] if op == "experts8" else torch.bfloat16),
         "w": (torch.randn(e, n, k, generator=g, device="cuda") / math.sqrt(k)).to(torch.bfloat16)}
    if op == "gradient":
        d["dy"] = _neural_gradient(rows, n, g)
    return d


def _codes(x):
    """(codes, scales) of the rows of a matrix; the product that is rounded to a code is formed in fp64, next to
    a border fp32 would round it twice."""
    a = x.float().abs().amax(dim=1, keepdim=True).clamp(min=_TINY)
    top = torch.full_like(a, 127.0)         # with a number in its place torch multiplies by a rounded reciprocal
    return torch.round(x.double() * (top / a).double()).float(), a / top


def prepare(case, seed):
    st, op = _inputs(case, seed), case["op"]
    st["case"] = case
    if own:
        from paper_2006_08173_b200 import binding as lgn
        st["lgn"] = lgn
    if op in ("int8", "experts8"):
        # the weights as a program keeps them: codes and scales, the experts' one below the other
        w = st.pop("w").reshape(-1, case["k"])
        st["w"] = st["lgn"].lgn_int8_quantize(w) if own else _codes(w)
    return st


# ----------------------------------------------------------------------------------- one pass
def run(st):
    return _own(st) if own else _plain(st)


def _own(st):
    case, lgn = st["case"], st["lgn"]
    op = case["op"]
    if op == "int8":
        return lgn.lgn_int8_matmul(lgn.lgn_int8_quantize(st["x"]), st["w"], out_dtype=_DT[case["out"]])
    if op == "experts8":
        return lgn.lgn_int8_matmul(lgn.lgn_int8_quantize(st["x"]), st["w"], offsets=st["offsets"], out_dtype=_DT[case["out"]])
    if op == "experts":
        return lgn.lgn_grouped_matmul(st["x"], st["w"], st["offsets"], out_dtype=_DT[case["out"]])
    if op == "gradient":
        dx = lgn.lgn_grouped_matmul(st["dy"], st["w"], st["offsets"], transposed=True, out_dtype=_DT[case["out"]])
        return dx, lgn.lgn_grouped_weight_grad(st["dy"], st["x"], st["offsets"], out_dtype=torch.float32)
    loss, dlogits = lgn.lgn_distill_loss(st["logits"], st["ids"], st["teacher"], labels=st["labels"], temperature=case["temperature"],
                                         alpha=case["alpha"], weight=st["weight"], grad=case["grad"])
    return (loss, dlogits) if case["grad"] else loss


def _by_expert(sizes, parts):
    """The rows' parts, expert by expert: one slice of each tensor."""
    at = 0
    for e, size in enumerate(sizes):
        yield (e,) + tuple(p[at:at + size] for p in parts)
        at += size


def _plain(st):
    case = st["case"]
    op = case["op"]
    if op == "distill":
        return _plain_distill(st)
    if op in ("int8", "experts8"):
        (q, s), (wq, ws) = _codes(st["x"]), st["w"]
        if op == "int8":
            return ((q @ wq.t()) * s * ws.t()).to(_DT[case["out"]])
        n = case["n"]
        return torch.cat([((qe @ wq[e * n:(e + 1) * n].t()) * se * ws[e * n:(e + 1) * n].t()).to(_DT[case["out"]])
                          for e, qe, se in _by_expert(st["sizes"], (q, s))])
    w = st["w"].float()
    if op == "experts":
        return torch.cat([(xe @ w[e].t()).to(_DT[case["out"]]) for e, xe in _by_expert(st["sizes"], (st["x"].float(),))])
    dx, dw = [], []
    for e, xe, de in _by_expert(st["sizes"], (st["x"].float(), st["dy"].float())):
        dx.append((de @ w[e]).to(_DT[case["out"]]))
        dw.append(de.t() @ xe)
    return torch.cat(dx), torch.stack(dw)


def _plain_distill(st):
    case, s = st["case"], st["logits"].float()
    temp, alpha = case["temperature"], case["alpha"]
    zero = torch.zeros((), device="cuda")
    ids = st["ids"].long()
    there = ids >= 0
    at = torch.where(there, ids, 0)
    z = torch.where(there, st["teacher"].float() / temp, -math.inf)
    some = there.any(dim=1, keepdim=True)
    top = torch.where(some, z.amax(dim=1, keepdim=True), zero)
    p = torch.exp(z - top)
    total = torch.where(some, p.sum(dim=1, keepdim=True), torch.ones_like(top))
    p, logp = p / total, z - top - torch.log(total)

    def softmax(u):
        m = u.amax(dim=1, keepdim=True)
        e = torch.exp(u - m)
        t = e.sum(dim=1, keepdim=True)
        return e / t, m + torch.log(t)

    u = s / temp
    q, lse = softmax(u)
    loss = alpha * temp * temp * torch.where(there, p * (logp - (u.gather(1, at) - lse)), zero).sum(dim=1)
    if case["grad"]:
        d = q * torch.where(some, alpha * temp, zero)
        d.scatter_add_(1, at, torch.where(there, -alpha * temp * p, zero))
    if st["labels"] is not None:
        labels = st["labels"].long()[:, None]
        q1, lse1 = softmax(s) if temp != 1.0 else (q, lse)
        known = labels >= 0
        lab = torch.where(known, labels, 0)
        loss = loss + (1.0 - alpha) * torch.where(known, lse1 - s.gather(1, lab), zero)[:, 0]
        if case["grad"]:
            c = torch.where(known, 1.0 - alpha, zero)
            d = d + q1 * c
            d.scatter_add_(1, lab, -c)
    if not case["grad"]:
        return loss
    return loss, (d * st["weight"][:, None]).to(st["logits"].dtype)


# ----------------------------------------------------------------------------------- in 64 bits
def _levels(x):
    """What the 8-bit codes of the rows of x stand for."""
    x = x.double()
    a = x.abs().max(dim=1, keepdim=True).values
    a = torch.where(a < _TINY, torch.full_like(a, _TINY), a)
    top = torch.full_like(a, 127.0)
    per, scale = (top / a).to(torch.float32).double(), (a / top).to(torch.float32).double()
    y = x * per
    lower = torch.floor(y)
    rest = y - lower
    up = (rest > 0.5) | ((rest == 0.5) & (torch.remainder(lower, 2.0) == 1.0))
    return (lower + up.double()) * scale


def exact(case, seed):
    st, op = _inputs(case, seed), case["op"]
    if op == "distill":
        return _exact_distill(case, st)
    if op == "int8":
        return _levels(st["x"]) @ _levels(st["w"]).t()
    ends = np.cumsum(st["sizes"])
    spans = [slice(int(b - c), int(b)) for b, c in zip(ends, st["sizes"])]
    if op in ("experts", "experts8"):
        x = _levels(st["x"]) if op == "experts8" else st["x"].double()
        out = torch.zeros(case["rows"], case["n"], dtype=torch.float64, device="cuda")
        for e, span in enumerate(spans):
            w = _levels(st["w"][e]) if op == "experts8" else st["w"][e].double()
            out[span] = x[span] @ w.t()
        return out
    dx = torch.zeros(case["rows"], case["k"], dtype=torch.float64, device="cuda")
    dw = torch.zeros(case["experts"], case["n"], case["k"], dtype=torch.float64, device="cuda")
    for e, span in enumerate(spans):
        dy = st["dy"][span].double()
        dx[span] = dy @ st["w"][e].double()
        dw[e] = dy.t() @ st["x"][span].double()
    return dx, dw


def _exact_distill(case, st):
    temp, alpha = case["temperature"], case["alpha"]
    losses, grads = [], []
    for rows in torch.arange(case["tokens"], device="cuda").split(256):
        s, ids, z = st["logits"][rows].double(), st["ids"][rows].long(), st["teacher"][rows].double() / temp
        absent = ids < 0
        z = z.masked_fill(absent, -math.inf)
        empty = absent.all(dim=1)
        logp = (z - torch.logsumexp(z, 1, keepdim=True)).masked_fill(absent, 0.0)
        p = torch.exp(logp).masked_fill(absent, 0.0)
        logq = s / temp - torch.logsumexp(s / temp, 1, keepdim=True)
        picked = logq.gather(1, ids.clamp(min=0))
        loss = alpha * temp ** 2 * (p * (logp - picked)).sum(1)
        d = torch.exp(logq).masked_fill(empty[:, None], 0.0).scatter_add(1, ids.clamp(min=0), -p) * (alpha * temp)
        if st["labels"] is not None:
            lab = st["labels"][rows].long()
            known = (lab >= 0).double()[:, None]
            log1 = s - torch.logsumexp(s, 1, keepdim=True)
            loss = loss - (1.0 - alpha) * (known * log1.gather(1, lab.clamp(min=0)[:, None]))[:, 0]
            d += (1.0 - alpha) * known * torch.exp(log1)
            d.scatter_add_(1, lab.clamp(min=0)[:, None], -(1.0 - alpha) * known)
        losses.append(loss)
        if case["grad"]:
            grads.append(d * st["weight"][rows].double()[:, None])
    return (torch.cat(losses), torch.cat(grads)) if case["grad"] else torch.cat(losses)
