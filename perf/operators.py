"""Learning the dense rows and holding them in 8 bits, as cases that can be timed.

Three operators: dense rows out of token lists (``embed``) with their gradients, the softmax loss of queries over all
documents (``softmax_loss``) with its gradients, and scores out of 8-bit rows with a scale for each query and document
(``quantize_rows``, ``scores_int8``).  ``own`` chooses between the library's calls and plain torch operations in 32 bits.

The shapes are those of the named workloads: ``tiny``; 768 columns of f32 on 100,000 documents, vocabulary 30,522; 1,024
columns of bf16, vocabulary 250,002.  Tokens are Zipf(1.1), dense rows unit Gaussian, texts of log-normal length.
"""
from __future__ import annotations

import math

import torch

own = False
DEVICE = "cuda:0"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}

# n: rows of the table, or documents; rows: token lists, or queries; mean: tokens a list (0: one token a row, no lists);
# uneven: every query's loss counts with a weight of its own instead of 1 / rows
EMBED = dict(kind="embed", weighted=True)
GRAD = dict(kind="embed gradient", weighted=True)
LOSS = dict(kind="loss", grad=False, uneven=False)
STEP = dict(kind="loss", grad=True, uneven=False)
INT8 = dict(kind="int8")


def listed():
    return [
        # one user's query: its 8 tokens become a dense row, nothing but latency
        dict(EMBED, name="embed one query", type="f32", n=30_522, dim=768, rows=1, mean=8),
        # a shard's texts of about 60 tokens, weighted by their importance
        dict(EMBED, name="embed texts", type="bf16", n=250_002, dim=1024, rows=20_000, mean=60),
        # gradient of a training batch of short queries: nearly all of it is a table of zeros
        dict(GRAD, name="embed gradient of queries", type="f32", n=30_522, dim=768, rows=64, mean=8),
        # gradient of a batch of texts, a few tokens of which are in nearly every one
        dict(GRAD, name="embed gradient of texts", type="bf16", n=250_002, dim=1024, rows=20_000, mean=60),
        # the loss of one query over the benchmark's f32 corpus: one pass over its documents
        dict(LOSS, name="loss of one query", type="f32", n=100_000, dim=768, rows=1),
        # how well the rows are learned, over a batch of queries: the loss without its gradient
        dict(LOSS, name="loss of an evaluation", type="bf16", n=120_011, dim=1024, rows=1_000),
        # a training step on a small collection: launches count
        dict(STEP, name="step tiny", type="f32", n=2_000, dim=128, rows=100),
        # a step whose classes are the learned-sparse vocabulary, with an odd number of rows of uneven weight
        dict(STEP, name="step over terms", type="bf16", n=30_522, dim=768, rows=1_003, uneven=True),
        # a step over the benchmark's f32 corpus
        dict(STEP, name="step f32", type="f32", n=100_000, dim=768, rows=2_048),
        # the largest: a large batch over the large vocabulary
        dict(STEP, name="step large", type="bf16", n=250_002, dim=1024, rows=4_096),
        # one query against a million documents in 8 bits: their bytes, once
        dict(INT8, name="int8 one query", type="bf16", n=1_000_000, dim=1024, rows=1),
        # the benchmark's batch against its documents, held in 8 bits
        dict(INT8, name="int8 batch", type="f32", n=100_000, dim=768, rows=10_000),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind, of = rng.choice(["embed", "embed gradient", "loss", "step", "int8"]), rng.choice(["f32", "bf16"])
    # a row is a multiple of 4 (f32) or 8 (bf16) columns
    case = dict(type=of, dim=rng.choice([128, 264, 384, 520, 768, 1000, 1024] if of == "bf16" else [96, 128, 260, 384, 500, 768, 1024]))
    if kind.startswith("embed"):
        mean = rng.choice([0, 0, 8, 30, 60])
        rows = _log(rng, 1, 20_000 if mean else 500_000)
        return dict(kind=kind, weighted=rng.random() < 0.6, **case, n=_log(rng, 1_000, 250_002), rows=rows, mean=mean)
    if kind == "int8":
        rows = _log(rng, 1, 10_000)
        return dict(INT8, **case, n=_log(rng, 1_000, min(1_000_000, 1_000_000_000 // rows)), rows=rows)
    rows = _log(rng, 1, 4_096)
    most = 250_002 if of == "bf16" else 100_000
    return dict(STEP if kind == "step" else LOSS, **case, n=_log(rng, 1_000, min(most, 500_000_000 // rows)), rows=rows) | {"uneven": rng.random() < 0.5}


def _cdf(n, device):
    p = torch.arange(1, n + 1, dtype=torch.float64, device=device).pow(-1.1)
    return torch.cumsum(p / p.sum(), 0)


def _unit(g, n, dim, dtype):
    x = torch.randn((n, dim), generator=g, device=DEVICE)
    return (x / x.norm(dim=1, keepdim=True)).to(dtype)


def prepare(case, seed):
    g = torch.Generator(device=DEVICE).manual_seed(int(seed))
    n, rows, dim, dtype = case["n"], case["rows"], case["dim"], TYPES[case["type"]]
    s = dict(case=case)
    if case["kind"].startswith("embed"):
        if case["mean"]:
            sigma = 0.5   # of the logarithm of a list's length, as in the workloads' texts
            ends = torch.exp(torch.randn(rows, generator=g, device=DEVICE, dtype=torch.float64) * sigma).cumsum(0)
            count = rows * case["mean"]   # a batch holds this many tokens, the lists as they fall
            s["indptr"] = torch.cat([ends.new_zeros(1), ends * (count / ends[-1])]).round().long()
        else:
            s["indptr"], count = None, rows
        ranks = torch.searchsorted(_cdf(n, DEVICE), torch.rand(count, generator=g, device=DEVICE, dtype=torch.float64)).clamp(max=n - 1)
        s["tokens"] = torch.randperm(n, generator=g, device=DEVICE)[ranks].int()
        s["tokens"][torch.rand(count, generator=g, device=DEVICE) < 0.01] = -1   # unused slots
        s["weights"] = torch.randn(count, generator=g, device=DEVICE).abs() if case["weighted"] else None
        s["table"] = torch.randn((n, dim), generator=g, device=DEVICE).mul_(dim ** -0.5).to(dtype)
        s["scale"] = 1.0 / max(1, case["mean"])
        if case["kind"] == "embed gradient":
            s["grad_out"] = torch.randn((rows, dim), generator=g, device=DEVICE).mul_(1.0 / rows).to(dtype)
    elif case["kind"] == "loss":
        s["docs"] = _unit(g, n, dim, dtype)
        s["labels"] = torch.randint(0, n, (rows,), generator=g, device=DEVICE, dtype=torch.int32)
        # a query lies between its document and anywhere: cosine about 0.4, as half-way through training
        x = s["docs"][s["labels"].long()].float() * 0.45 + _unit(g, rows, dim, torch.float32)
        s["x"] = (x / x.norm(dim=1, keepdim=True)).to(dtype)
        if rows > 1:
            s["labels"][torch.rand(rows, generator=g, device=DEVICE) < 0.02] = -1   # queries whose document is not known
        s["scale"] = 20.0   # one over the temperature
        s["row_grad"] = torch.rand(rows, generator=g, device=DEVICE) * (2.0 / rows) if case["uneven"] else torch.full((rows,), 1.0 / rows, device=DEVICE)
    else:
        s["x"] = _unit(g, rows, dim, dtype)
        s["q"], s["q_scale"] = _quantized(_unit(g, n, dim, torch.float32))
    return s


def _quantized(x):
    """Rows in 8 bits: the largest magnitude of a row becomes 127; zeros fill the last group of 16 columns."""
    x = torch.nn.functional.pad(x.float(), (0, -x.shape[1] % 16))
    scale = x.abs().amax(1)
    scale = scale / torch.full_like(scale, 127.0)
    return torch.where(scale[:, None] > 0, x / scale[:, None], 0.0).round().to(torch.int8), scale


def _row_of(indptr, count):
    if indptr is None:
        return torch.arange(count, device=DEVICE)
    return torch.repeat_interleave(torch.arange(len(indptr) - 1, device=DEVICE), indptr.diff(), output_size=count)


def _plain_embed(s):
    tokens, table = s["tokens"].long(), s["table"]
    w = s["scale"] * (1.0 if s["weights"] is None else s["weights"]) * (tokens >= 0)
    e = table[tokens.clamp(min=0)].float() * w[:, None]
    if s["indptr"] is None:
        return e.to(table.dtype)
    out = torch.zeros((len(s["indptr"]) - 1, table.shape[1]), device=DEVICE)
    return out.index_add_(0, _row_of(s["indptr"], len(tokens)), e).to(table.dtype)


def _plain_embed_grad(s):
    tokens, table = s["tokens"].long(), s["table"]
    used = tokens >= 0
    g = s["grad_out"][_row_of(s["indptr"], len(tokens))].float() * (s["scale"] * used)[:, None]
    out = torch.zeros(table.shape, device=DEVICE).index_add_(0, tokens.clamp(min=0), g if s["weights"] is None else g * s["weights"][:, None]).to(table.dtype)
    if s["weights"] is None:
        return dict(table=out)
    return dict(table=out, weights=(g * table[tokens.clamp(min=0)].float()).sum(1))


def _plain_loss(s):
    x, docs, labels = s["x"].float(), s["docs"].float(), s["labels"].long()
    known = labels >= 0
    at = labels.clamp(min=0)[:, None]
    logits = (x @ docs.T).mul_(s["scale"])
    most = logits.amax(1, keepdim=True)
    true = logits.gather(1, at)[:, 0]
    p = logits.sub_(most).exp_()
    total = p.sum(1, keepdim=True)
    lse = (most + total.log())[:, 0]
    out = dict(loss=torch.where(known, lse - true, 0.0), lse=lse)
    if not s["case"]["grad"]:
        return out
    c = p.div_(total).scatter_add_(1, at, torch.full_like(total, -1.0)).mul_((s["row_grad"] * known * s["scale"])[:, None])
    return dict(out, x=(c @ docs).to(s["x"].dtype), docs=(c.T @ x).to(s["docs"].dtype))


def _plain_int8(s):
    x, x_scale = _quantized(s["x"])
    return (x.float() @ s["q"].float().T).mul_(x_scale[:, None]).mul_(s["q_scale"])


def run(state):
    s, kind = state, state["case"]["kind"]
    if not own:
        return {"embed": _plain_embed, "embed gradient": _plain_embed_grad, "loss": _plain_loss, "int8": _plain_int8}[kind](s)
    from paper_2511_00855_amd import binding as B
    if kind == "embed":
        return B.embed(s["table"], s["tokens"], s["weights"], s["indptr"], scale=s["scale"])
    if kind == "embed gradient":
        table = B.embed_grad(s["grad_out"], s["tokens"], s["table"].shape[0], s["weights"], s["indptr"], scale=s["scale"])
        if s["weights"] is None:
            return dict(table=table)
        return dict(table=table, weights=B.embed_grad_weights(s["grad_out"], s["table"], s["tokens"], s["indptr"], scale=s["scale"]))
    if kind == "loss":
        loss, lse = B.softmax_loss(s["x"], s["docs"], s["labels"], scale=s["scale"])
        if not s["case"]["grad"]:
            return dict(loss=loss, lse=lse)
        x, docs = B.softmax_loss_grad(s["x"], s["docs"], s["labels"], lse, s["row_grad"], scale=s["scale"])
        return dict(loss=loss, lse=lse, x=x, docs=docs)
    return B.scores_int8(s["x"], s["q"], s["q_scale"])


def work(case):
    n, rows, dim, size = case["n"], case["rows"], case["dim"], 2 if case["type"] == "bf16" else 4
    if case["kind"].startswith("embed"):
        count = rows * max(1, case["mean"])
        ids = count * (8 if case["weighted"] else 4) + (8 * (rows + 1) if case["mean"] else 0)
        p = _cdf(n, "cpu").diff(prepend=torch.zeros(1, dtype=torch.float64))
        named = float((1 - (1 - p) ** count).sum())   # rows of the table that some token names
        if case["kind"] == "embed":
            return dict(bytes=ids + (named + rows) * dim * size, flops=2.0 * count * dim)
        more = named * dim * size + 4 * count if case["weighted"] else 0
        return dict(bytes=ids + more + (rows + n) * dim * size, flops=(4.0 if case["weighted"] else 2.0) * count * dim)
    if case["kind"] == "loss":
        passes = 3 if case["grad"] else 1   # the logits; both gradients
        return dict(bytes=(rows + n) * dim * size * (2 if case["grad"] else 1) + rows * (16 if case["grad"] else 12), flops=2.0 * passes * rows * n * dim)
    return dict(bytes=rows * dim * size + n * (dim + 4) + 4.0 * rows * n, flops=2.0 * rows * n * dim)


def _exact_embed(s):
    tokens, table = s["tokens"].long(), s["table"].double()
    w = torch.ones(len(tokens), device=DEVICE, dtype=torch.float64) if s["weights"] is None else s["weights"].double()
    w = torch.where(tokens < 0, 0.0, w) * s["scale"]
    if s["indptr"] is None:
        return w[:, None] * table[tokens.clamp(min=0)]
    first, lengths = s["indptr"][:-1], s["indptr"].diff()
    out = torch.zeros((len(lengths), table.shape[1]), device=DEVICE, dtype=torch.float64)
    for j in range(int(lengths.max())):   # the j-th token of every list that has one
        has = torch.nonzero(lengths > j)[:, 0]
        at = first[has] + j
        out[has] += w[at][:, None] * table[tokens[at].clamp(min=0)]
    return out


def _exact_embed_grad(s):
    tokens, table, grad = s["tokens"].long(), s["table"].double(), s["grad_out"].double()
    count = len(tokens)
    places = torch.arange(count, device=DEVICE)
    row = places if s["indptr"] is None else torch.searchsorted(s["indptr"], places, right=True) - 1
    w = torch.ones(count, device=DEVICE, dtype=torch.float64) if s["weights"] is None else s["weights"].double()
    order = torch.argsort(tokens, stable=True)
    order = order[tokens[order] >= 0]
    out = torch.zeros_like(table)
    ids, lengths = torch.unique_consecutive(tokens[order], return_counts=True)
    first = lengths.cumsum(0) - lengths
    for j in range(0, int(lengths.max()) if len(lengths) else 0):   # the j-th place that names each token, until few have one
        has = torch.nonzero(lengths > j)[:, 0]
        if len(has) <= 64:
            break
        at = order[first[has] + j]
        out[ids[has]] += w[at][:, None] * grad[row[at]]
    else:
        j = int(lengths.max()) if len(lengths) else 0
    for k in torch.nonzero(lengths > j)[:, 0].tolist():   # the frequent ones, each by itself
        at = order[int(first[k]) + j:int(first[k] + lengths[k])]
        out[ids[k]] += w[at] @ grad[row[at]]
    out *= s["scale"]
    if s["weights"] is None:
        return dict(table=out)
    step = 1 << 18
    dots = [torch.where(tokens[b:b + step] < 0, 0.0, (table[tokens[b:b + step].clamp(min=0)] * grad[row[b:b + step]]).sum(1)) for b in range(0, count, step)]
    return dict(table=out, weights=torch.cat(dots) * s["scale"])


def _exact_loss(s):
    x, docs, labels = s["x"].double(), s["docs"].double(), s["labels"].long()
    step = max(1, (1 << 29) // docs.shape[0])   # queries at a time
    out = dict(loss=[], lse=[])
    if s["case"]["grad"]:
        out |= dict(x=[], docs=torch.zeros_like(docs))
    for b in range(0, len(x), step):
        known = labels[b:b + step] >= 0
        logits = s["scale"] * (x[b:b + step] @ docs.T)
        lse = torch.logsumexp(logits, 1)
        rows = torch.arange(len(lse), device=DEVICE)
        at = torch.where(known, labels[b:b + step], 0)
        out["lse"].append(lse)
        out["loss"].append(torch.where(known, lse - logits[rows, at], 0.0))
        if s["case"]["grad"]:
            c = torch.exp(logits - lse[:, None])
            c[rows, at] -= 1.0
            c *= torch.where(known, s["row_grad"][b:b + step].double(), 0.0)[:, None]
            out["x"].append(s["scale"] * (c @ docs))
            out["docs"] += s["scale"] * (c.T.contiguous() @ x[b:b + step])
    return {k: torch.cat(v) if isinstance(v, list) else v for k, v in out.items()}


def _exact_int8(s):
    x = s["x"].double()
    scale = (x.abs().amax(1, keepdim=True) / 127).float()   # what a row is divided by is an f32 number, and so is the quotient
    q = torch.where(scale > 0, torch.round((x / scale.double()).float()), 0.0).double()
    return (q * scale.double()) @ (s["q"][:, :x.shape[1]].double() * s["q_scale"].double()[:, None]).T


def exact(case, seed):
    if case["kind"] in ("loss", "int8") and case["rows"] * case["n"] > 1_100_000_000:
        return None
    s = prepare(case, seed)
    return {"embed": _exact_embed, "embed gradient": _exact_embed_grad, "loss": _exact_loss, "int8": _exact_int8}[case["kind"]](s)
