"""What is timed of the language-model operators beside the optimizer step.

Three operators, each as a training loop around the step calls it: the word
table's lookup and its gradient, the vocabulary head's cross entropy (the loss
alone, and with both gradients), and the orthogonalised (Muon) update of
matrices (the direction alone, and the whole step).  Every case has two forms on
the same inputs: the plain one of elementary torch operations in 32 bits, and
the library's calls; `exact` gives the same from the definitions in 64 bits.

Word ids follow a Zipf-like law as in text, with one id (the mask token) more
frequent than all others in masked-language batches and -1 where a batch is
padded.  Hidden rows are of a normalised layer's size and lean towards their
label's row by different amounts, as in a model half trained: the label's
probability is anywhere between that of a blind guess and nearly one.
"""
from __future__ import annotations

import math

import torch

own = False

DEV = "cuda:0"
VOCAB = 30522              # of the BERT layouts
NS = (3.4445, -4.7750, 2.0315)
NS_STEPS = 5
BETA, DECAY, LR, EPS = 0.95, 0.01, 2e-4, 1e-7

LAYER_BASE = "4*768x768,1*3072x768,1*768x3072"
LAYER_LARGE = "4*1024x1024,1*4096x1024,1*1024x4096"


def listed():
    return [
        # one sequence of a mixed-precision model: the call's latency
        dict(name="lookup_sequence", op="lookup", tokens=512, vocab=VOCAB,
             width=1024, table="bf16", out="bf16", masked=0.12, padded=0.0),
        # a batch of 128 sequences of 512, from the fp32 master table
        dict(name="lookup_batch", op="lookup", tokens=65536, vocab=VOCAB,
             width=768, table="f32", out="bf16", masked=0.12, padded=0.1),
        # a tied table's micro-batch: added to the head's gradient, fp32
        dict(name="lookup_grad_tied", op="lookup_grad", tokens=4095,
             vocab=VOCAB, width=768, grad="f32", table="f32",
             accumulate=True, masked=0.12, padded=0.05),
        # the whole batch's gradient of a table of its own
        dict(name="lookup_grad_batch", op="lookup_grad", tokens=65536,
             vocab=VOCAB, width=1024, grad="bf16", table="bf16",
             accumulate=False, masked=0.12, padded=0.1),
        # one token's log-probability, as in scoring word by word
        dict(name="head_score_token", op="head", tokens=1, vocab=VOCAB,
             width=768, train=False, ignored=0.0),
        # validation loss over a padded batch
        dict(name="head_eval_batch", op="head", tokens=8192, vocab=VOCAB,
             width=768, train=False, ignored=0.15),
        # the masked positions of one sequence
        dict(name="head_train_sequence", op="head", tokens=77, vocab=VOCAB,
             width=1024, train=True, ignored=0.0),
        # the masked positions of 32 sequences, BERT-base
        dict(name="head_train_base", op="head", tokens=2458, vocab=VOCAB,
             width=768, train=True, ignored=0.0),
        # the masked positions of 128 sequences, BERT-large
        dict(name="head_train_large", op="head", tokens=9830, vocab=VOCAB,
             width=1024, train=True, ignored=0.02),
        # the tiny MLP's two matrices: latency of a chain of small products
        dict(name="muon_direction_mlp", op="direction",
             shapes="1*64x32,1*32x10"),
        # the matrices of one BERT-large layer
        dict(name="muon_direction_layer", op="direction",
             shapes=LAYER_LARGE),
        # all matrices of BERT-base's twelve layers: a whole step
        dict(name="muon_step_base", op="step",
             shapes="48*768x768,12*3072x768,12*768x3072,1*768x768"),
    ]


def draw(rng):
    def logint(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    op = rng.choice(["lookup", "lookup_grad", "head", "head", "direction",
                     "step"])
    if op in ("direction", "step"):
        shapes = []
        for _ in range(rng.randint(1, 3)):
            short = logint(10, 1536)
            shape = [short, logint(short, 4096)]
            rng.shuffle(shape)
            shapes.append("%d*%dx%d" % (rng.randint(1, 3), *shape))
        return dict(op=op, shapes=",".join(shapes))
    width = logint(32, 1024)
    if rng.random() < 0.6:
        width = max(64, width // 64 * 64)
    vocab = logint(500, VOCAB)
    if op == "head":
        return dict(op=op, tokens=logint(1, 9830), vocab=vocab, width=width,
                    train=rng.random() < 0.6,
                    ignored=rng.choice([0.0, 0.02, 0.5]))
    case = dict(op=op, tokens=logint(1, 65536), vocab=vocab, width=width,
                table=rng.choice(["f32", "bf16"]),
                masked=rng.choice([0.0, 0.12]), padded=rng.choice([0.0, 0.1]))
    other = rng.choice(["f32", "bf16"])
    if op == "lookup":
        return dict(case, out=other)
    return dict(case, grad=other, accumulate=rng.random() < 0.5)


# ---------------------------------------------------------------------------
# Inputs
# ---------------------------------------------------------------------------
_DTYPE = {"f32": torch.float32, "bf16": torch.bfloat16}


def _shapes(case):
    out = []
    for part in case["shapes"].split(","):
        count, shape = part.split("*")
        r, c = shape.split("x")
        out += [(int(r), int(c))] * int(count)
    return out


def _weights_of_ids(vocab):
    return 1.0 / (torch.arange(vocab, dtype=torch.float64) + 2.7)


def _ids(n, vocab, gen, masked=0.0):
    """Zipf-like word ids, ranks spread over the table."""
    p = _weights_of_ids(vocab).to(DEV)
    cum = torch.cumsum(p, 0)
    u = torch.rand(n, generator=gen, device=DEV, dtype=torch.float64)
    rank = torch.searchsorted(cum, u * cum[-1]).clamp(max=vocab - 1)
    ids = torch.randperm(vocab, generator=gen, device=DEV)[rank]
    if masked:
        at = torch.rand(n, generator=gen, device=DEV) < masked
        ids = torch.where(at, min(103, vocab - 1), ids)
    return ids


def _normal(shape, gen, std=1.0, dtype=torch.float32):
    x = torch.randn(shape, generator=gen, device=DEV)
    return x.mul_(std).to(dtype)


class _State:
    """What a program has in hand: the tensors, and the plan if it is used."""


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    s = _State()
    s.case, s.plan = case, None
    op = case["op"]
    if op in ("direction", "step"):
        s.shapes = _shapes(case)
        sizes = [r * c for r, c in s.shapes]
        # tensors of one flat buffer each, on 256-byte boundaries
        s.offsets, cur = [], 0
        for n in sizes:
            s.offsets.append(cur)
            cur += (n + 63) // 64 * 64

        def flat(dtype):
            return torch.zeros(cur, device=DEV, dtype=dtype)

        def views(buf):
            return [buf[o:o + r * c].view(r, c)
                    for o, (r, c) in zip(s.offsets, s.shapes)]

        def gradient(r, c, std):
            """A few strong directions over noise, as gradients have."""
            k = min(8, r, c)
            a = _normal((r, k), gen) @ _normal((k, c), gen)
            return (a * 0.3 + _normal((r, c), gen)) * std

        s.g = flat(torch.bfloat16)
        for x, (r, c) in zip(views(s.g), s.shapes):
            x.copy_(gradient(r, c, 1e-3))
        if op == "direction":
            s.out = flat(torch.bfloat16)
        else:
            s.w, s.m, s.copy = (flat(torch.float32), flat(torch.float32),
                                flat(torch.bfloat16))
            for w, m, (r, c) in zip(views(s.w), views(s.m), s.shapes):
                w.copy_(_normal((r, c), gen, 0.04))
                m.copy_(gradient(r, c, 3e-4))
            s.lr = torch.full((1,), LR, device=DEV)
        s.views = views
        if own:
            from paper_1904_00962_gb300 import binding as B
            from paper_1904_00962_gb300.muon import MuonPlan
            s.hyper = B.make_muon_hyper(momentum=BETA, weight_decay=DECAY,
                                        scale="rms")
            s.plan = MuonPlan(s.shapes, grad_dtype="bf16",
                              copy_dtype="bf16" if op == "step" else None)
            if op == "direction":
                s.plan.bind_direction(views(s.g), views(s.out))
            else:
                s.plan.bind(views(s.w), views(s.g), views(s.m),
                            views(s.copy))
        return s

    T, V, D = case["tokens"], case["vocab"], case["width"]
    if op == "head":
        s.weight = _normal((V, D), gen, 0.04, torch.bfloat16)
        s.labels = _ids(T, V, gen)
        lean = torch.rand((T, 1), generator=gen, device=DEV) * 12.0
        rows = s.weight[s.labels].float()
        rows = rows / rows.square().sum(1, keepdim=True).sqrt()
        s.hidden = (_normal((T, D), gen) + lean * rows).to(torch.bfloat16)
        drop = torch.rand(T, generator=gen, device=DEV) < case["ignored"]
        s.labels = torch.where(drop, -100, s.labels)
        s.loss = torch.zeros(1, device=DEV)
        s.token_loss = torch.zeros(T, device=DEV)
        if case["train"]:
            s.grad_hidden = torch.zeros_like(s.hidden)
            s.grad_weight = torch.zeros_like(s.weight)
    else:
        s.ids = _ids(T, V, gen, case["masked"])
        if case["padded"]:
            at = torch.rand(T, generator=gen, device=DEV) < case["padded"]
            s.ids = torch.where(at, -1, s.ids)
        s.scale = math.sqrt(D)
        if op == "lookup":
            s.table = _normal((V, D), gen, 0.02, _DTYPE[case["table"]])
            s.out = torch.zeros((T, D), device=DEV,
                                dtype=_DTYPE[case["out"]])
        else:
            s.grad_out = _normal((T, D), gen, 1e-3, _DTYPE[case["grad"]])
            s.table_grad = torch.zeros((V, D), device=DEV,
                                       dtype=_DTYPE[case["table"]])
            if case["accumulate"]:
                s.table_grad.copy_(_normal((V, D), gen, 1e-3))
    if own:
        from paper_1904_00962_gb300.vocab import VocabPlan
        s.plan = VocabPlan(V, D, max_tokens=T)
    return s


# ---------------------------------------------------------------------------
# One pass
# ---------------------------------------------------------------------------
def run(s):
    return (_own if own else _plain)(s)


def _own(s):
    case, op = s.case, s.case["op"]
    if op == "lookup":
        return s.plan.embed(s.table, s.ids, scale=s.scale, out=s.out)
    if op == "lookup_grad":
        return s.plan.embed_grad(s.grad_out, s.ids, s.table_grad,
                                 scale=s.scale,
                                 accumulate=case["accumulate"])
    if op == "head":
        if not case["train"]:
            s.plan.loss(s.hidden, s.weight, s.labels, loss=s.loss,
                        token_loss=s.token_loss)
            return {"loss": s.loss, "token_loss": s.token_loss}
        s.plan.loss_grad(s.hidden, s.weight, s.labels, s.grad_hidden,
                         s.grad_weight, loss=s.loss,
                         token_loss=s.token_loss)
        return {"loss": s.loss, "token_loss": s.token_loss,
                "grad_hidden": s.grad_hidden, "grad_weight": s.grad_weight}
    if op == "direction":
        s.plan.direction(s.hyper)
        return s.out
    s.plan.step(s.hyper, s.lr)
    return {"w": s.w, "m": s.m, "copy": s.copy}


def _plain(s):
    case, op = s.case, s.case["op"]
    if op == "lookup":
        rows = s.table[s.ids.clamp(min=0)].float() * s.scale
        rows = torch.where((s.ids >= 0)[:, None], rows, 0.0)
        return rows.to(s.out.dtype)
    if op == "lookup_grad":
        rows = s.grad_out.float() * s.scale
        rows = torch.where((s.ids >= 0)[:, None], rows, 0.0)
        total = (s.table_grad.float() if case["accumulate"] else
                 torch.zeros(s.table_grad.shape, device=DEV))
        total.index_add_(0, s.ids.clamp(min=0), rows)
        s.table_grad.copy_(total)
        return s.table_grad
    if op == "head":
        return _plain_head(s)
    if op == "direction":
        for u, o in zip(s.views(s.g), s.views(s.out)):
            o.copy_(_plain_direction(u.float()))
        return s.out
    for w, g, m, c in zip(s.views(s.w), s.views(s.g), s.views(s.m),
                          s.views(s.copy)):
        g = g.float()
        m.mul_(BETA).add_(g, alpha=1.0 - BETA)
        x = _plain_direction((1.0 - BETA) * g + BETA * m)
        size = 0.2 * math.sqrt(max(w.shape))
        w.copy_(w * (1.0 - s.lr * DECAY) - (s.lr * size) * x)
        c.copy_(w)
    return {"w": s.w, "m": s.m, "copy": s.copy}


def _plain_direction(u):
    a, b, c = NS
    x = u.T if u.shape[0] > u.shape[1] else u
    x = x / (x.square().sum().sqrt() + EPS)
    for _ in range(NS_STEPS):
        gram = x @ x.T
        x = a * x + (b * gram + c * (gram @ gram)) @ x
    return x.T if u.shape[0] > u.shape[1] else x


def _plain_head(s):
    h, w = s.hidden.float(), s.weight.float()
    valid = s.labels >= 0
    at = s.labels.clamp(min=0)[:, None]
    count = valid.sum().clamp(min=1).float()
    logits = h @ w.T
    top = logits.amax(1, keepdim=True)
    label = torch.gather(logits, 1, at)
    p = (logits - top).exp()
    total = p.sum(1, keepdim=True)
    token_loss = torch.where(valid, (top + total.log() - label)[:, 0], 0.0)
    out = {"loss": (token_loss.sum() / count)[None], "token_loss": token_loss}
    if s.case["train"]:
        p = p / total
        p.scatter_add_(1, at, -torch.ones_like(label))
        p = p * (valid / count)[:, None]
        out["grad_hidden"] = (p @ w).to(s.hidden.dtype)
        out["grad_weight"] = (p.T @ h).to(s.weight.dtype)
    return out


# ---------------------------------------------------------------------------
# The definitions in 64 bits
# ---------------------------------------------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "lookup":
        table = torch.cat([s.table.double(),
                           torch.zeros((1, case["width"]), device=DEV,
                                       dtype=torch.float64)])
        return table[s.ids] * s.scale          # -1: the row of zeros
    if op == "lookup_grad":
        keep = s.ids >= 0
        ids, order = torch.sort(s.ids[keep])
        rows = s.grad_out[keep].double()[order]
        ends = torch.cumsum(rows, 0)
        ends = torch.cat([torch.zeros_like(ends[:1]), ends]) \
            if len(ids) else torch.zeros((1, case["width"]), device=DEV,
                                         dtype=torch.float64)
        v = torch.arange(case["vocab"], device=DEV)
        sums = ends[torch.searchsorted(ids, v, right=True)] - \
            ends[torch.searchsorted(ids, v)]
        out = sums * s.scale
        return out + s.table_grad.double() if case["accumulate"] else out
    if op == "head":
        return _exact_head(s)
    if op == "direction":
        out = torch.zeros(s.g.shape, device=DEV, dtype=torch.float64)
        for u, o in zip(s.views(s.g), s.views(out)):
            o.copy_(_exact_direction(u.double()))
        return out
    g, m, w = s.g.double(), s.m.double(), s.w.double()
    m = BETA * m + (1.0 - BETA) * g
    u = (1.0 - BETA) * g + BETA * m
    lr = s.lr.double()
    new = w * (1.0 - lr * DECAY)
    for x, o in zip(s.views(u), s.views(new)):
        o.sub_(lr * 0.2 * math.sqrt(max(x.shape)) * _exact_direction(x))
    return {"w": new, "m": m, "copy": new}


def _exact_direction(u):
    """Each step as x <- (a I + G (b I + c G)) x, G of the shorter side."""
    a, b, c = NS
    wide = u.shape[0] <= u.shape[1]
    x = u / (torch.linalg.matrix_norm(u) + EPS)
    for _ in range(NS_STEPS):
        if wide:
            gram = torch.einsum("ik,jk->ij", x, x)
            poly = gram @ (c * gram).add_(torch.eye(
                len(gram), device=DEV, dtype=x.dtype), alpha=b)
            x = torch.addmm(x, poly, x, beta=a)
        else:
            gram = torch.einsum("ki,kj->ij", x, x)
            poly = (c * gram).add_(torch.eye(
                len(gram), device=DEV, dtype=x.dtype), alpha=b) @ gram
            x = torch.addmm(x, x, poly, beta=a)
    return x


def _exact_head(s):
    h, w = s.hidden.double(), s.weight.double()
    keep = torch.nonzero(s.labels >= 0)[:, 0]
    n = max(1, len(keep))
    token_loss = torch.zeros(len(h), device=DEV, dtype=torch.float64)
    out = {"token_loss": token_loss}
    grad_h, grad_w = torch.zeros_like(h), torch.zeros_like(w)
    for rows in torch.split(keep, 2048):      # a part of the tokens at a time
        logp = torch.log_softmax(h[rows] @ w.T, dim=1)
        y = s.labels[rows]
        token_loss[rows] = -logp[torch.arange(len(rows), device=DEV), y]
        if s.case["train"]:
            d = torch.softmax(logp, dim=1)
            d[torch.arange(len(rows), device=DEV), y] -= 1.0
            d /= n
            grad_h[rows] = d @ w
            grad_w += d.T @ h[rows]
    out["loss"] = (token_loss.sum() / n)[None]
    if s.case["train"]:
        out.update(grad_hidden=grad_h, grad_weight=grad_w)
    return out


# ---------------------------------------------------------------------------
# What a pass cannot do without
# ---------------------------------------------------------------------------
def work(case):
    op = case["op"]
    if op in ("direction", "step"):
        n = flops = 0
        for r, c in _shapes(case):
            lo, hi = min(r, c), max(r, c)
            n += r * c
            # two symmetric products (half of each) and a full one
            flops += NS_STEPS * (3 * lo * lo * hi + lo ** 3)
        per = 4 if op == "direction" else 2 + 8 + 8 + 2
        return {"bytes": per * n, "flops": flops}
    T, V, D = case["tokens"], case["vocab"], case["width"]
    if op == "head":
        # the loss: one product; the gradients: two more (products that only
        # replace kept logits are not counted)
        both = 2 if case["train"] else 1
        return {"bytes": both * 2 * (T + V) * D + 12 * T,
                "flops": (6 if case["train"] else 2) * T * V * D}
    size = {"f32": 4, "bf16": 2}
    p = _weights_of_ids(V)
    p = p / p.sum() * (1.0 - case["masked"])
    real = round(T * (1.0 - case["padded"]))
    touched = min(real, round(float((1.0 - (1.0 - p) ** real).sum())))
    if op == "lookup":
        return {"bytes": 8 * T + touched * D * size[case["table"]] +
                T * D * size[case["out"]], "flops": T * D}
    rows = 2 * touched if case["accumulate"] else V
    return {"bytes": 8 * T + real * D * size[case["grad"]] +
            rows * D * size[case["table"]], "flops": real * D}
