"""What the operators beside the decoder are measured on: the output layer that makes log-likelihoods out of an
encoder's hidden states, and the log-probabilities of given tokens with their gradient.

  linear                    residual + scale * act(x w^T + bias)
  loglikes                  log-softmax of the same product, minus the classes' log priors: the decoder's input
  token_logprobs            log-probabilities of given tokens, log of the sum, entropy and the top alternatives of a row of scores
  token_logprobs_backward   its gradient with respect to the scores

Sizes follow workloads/configs.py (batches of 1 to 256 utterances of 50 to 875 frames, 512 streams of 16 frames, 29 or 129
classes, up to the decoder's 2,048) and, for the scores of a language model over n best paths, vocabularies of up to 128,001."""
from __future__ import annotations

import math

import torch

own = False

DTYPES = {"float32": torch.float32, "float16": torch.float16, "bfloat16": torch.bfloat16}
SIZE = {"float32": 4, "float16": 2, "bfloat16": 2}
ACTS = ("none", "relu", "silu", "gelu")

LINEAR = dict(op="linear", dtype="bfloat16", out="bfloat16", act="none", bias=True, residual=False, scale=1.0, pad=0)
LOGLIKES = dict(op="loglikes", dtype="bfloat16", out="float32", bias=True, prior=False)
# given: tokens per row; top: alternatives per row; masked: share of the rows in which most of the vocabulary is ruled out
LOGPROBS = dict(op="logprobs", dtype="float32", given=1, top=4, masked=0.0, pad=0)
BACKWARD = dict(op="backward", dtype="bfloat16", given=1, top=0, entropy=True, masked=0.0, pad=0)


def listed():
    return [
        # one frame of one stream through a feed-forward layer: the smallest call
        dict(LINEAR, name="linear: one frame", m=1, k=512, n=2048, act="silu"),
        # a chunk of 16 frames of 64 streams, back to the model's width, added to what came in (a half-step layer)
        dict(LINEAR, name="linear: 64 streams", m=64 * 16, k=2048, n=512, residual=True, scale=0.5, dtype="float16", out="float16"),
        # a batch of 256 utterances: every frame of 2 to 35 s of audio each
        dict(LINEAR, name="linear: batch of 256", m=118417, k=512, n=2048, act="silu"),
        # a model that is kept in 32 bits, with sizes that are no multiple of anything, out of a wider buffer
        dict(LINEAR, name="linear: odd sizes in 32 bits", m=14803, k=177, n=333, act="gelu", dtype="float32", out="float32", pad=7),
        # live captions: a chunk of 16 frames of one stream
        dict(LOGLIKES, name="loglikes: one stream", b=1, t=16, d=512, v=129, lo=16, hi=16),
        # the throughput configuration: a padded batch of 256 utterances, with label priors
        dict(LOGLIKES, name="loglikes: batch of 256", b=256, t=875, d=512, v=129, lo=50, hi=875, prior=True),
        # 1,024 word pieces and the blank, half-precision scores
        dict(LOGLIKES, name="loglikes: word pieces", b=32, t=875, d=512, v=1025, lo=50, hi=875, dtype="float16", out="float16"),
        # confidence of decoded paths: the label of every frame of a batch of 256, with the entropy and the nearest labels
        dict(LOGPROBS, name="logprobs: frames of 256", rows=118417, v=129, given=1, top=4),
        # rescoring of n best paths under a language model: every token of the paths
        dict(LOGPROBS, name="logprobs: n best paths", rows=2048, v=64001, given=1, top=8, dtype="bfloat16", masked=0.1),
        # the next token of a few hypotheses
        dict(LOGPROBS, name="logprobs: next token", rows=4, v=128000, given=1, top=16, dtype="bfloat16"),
        # training on n best paths: the gradient at the language model's scores
        dict(BACKWARD, name="backward: n best paths", rows=2048, v=64001, given=1, top=0, entropy=True, masked=0.1),
        # ... and at the frames' scores, the labels of eight paths each
        dict(BACKWARD, name="backward: frames of 32", rows=14803, v=129, given=8, top=2, entropy=True, dtype="float32"),
    ]


def _size(rng, lo, hi):
    """A whole number of lo..hi, even over the logarithm; a third of them multiples of 64, a third of 8."""
    x = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    step = rng.choice((1, 8, 64))
    return max(lo, min(hi, (x + step - 1) // step * step))


def draw(rng):
    op = rng.choice(("linear", "loglikes", "logprobs", "backward"))
    dtype = rng.choice(tuple(DTYPES))
    if op == "linear":
        k, n = _size(rng, 32, 2048), _size(rng, 16, 2048)
        most = min(118417, 118417 * 512 * 2048 // (k * n) // (8 if dtype == "float32" else 1))
        return dict(LINEAR, m=_size(rng, 1, most), k=k, n=n, dtype=dtype, out=rng.choice((dtype, dtype, "float32")), act=rng.choice(ACTS),
                    bias=rng.random() < 0.8, residual=rng.random() < 0.4, scale=rng.choice((1.0, 0.5)), pad=rng.choice((0, 0, 8, 5)))
    if op == "loglikes":
        d, v = _size(rng, 64, 1024), rng.choice((29, 129, _size(rng, 16, 2048)))
        t = rng.choice((1, 16, _size(rng, 17, 875)))
        lo = rng.choice((t, max(1, t // 17), 0))
        most = 256 * 875 * 512 * 256 // (t * d * v) // (8 if dtype == "float32" else 1)
        return dict(LOGLIKES, b=_size(rng, 1, max(1, min(512 if t <= 16 else 256, most))), t=t, d=d, v=v, lo=lo, hi=t, dtype=dtype,
                    out=rng.choice((dtype, "float32")), bias=rng.random() < 0.8, prior=rng.random() < 0.4)
    v = rng.choice((29, 129, _size(rng, 16, 2048), _size(rng, 2049, 128001)))
    rows = _size(rng, 1, max(1, min(118417, 2048 * 64001 // v // (2 if dtype == "float32" else 1))))
    common = dict(rows=rows, v=v, dtype=dtype, given=rng.choice((1, 1, 8, rng.randint(2, 16))), masked=rng.choice((0.0, 0.2)),
                  pad=rng.choice((0, 0, 8, 3)))
    if op == "logprobs":
        return dict(LOGPROBS, top=rng.choice((0, 1, 4, 8, 16)), **common)
    return dict(BACKWARD, top=rng.choice((0, 0, 4)), entropy=rng.random() < 0.6, **common)


def work(case):
    e = SIZE[case["dtype"]]
    if case["op"] == "linear":
        m, k, n, o = case["m"], case["k"], case["n"], SIZE[case["out"]]
        return {"bytes": (m * k + n * k + n * case["bias"]) * e + m * n * o * (2 if case["residual"] else 1), "flops": 2 * m * n * k}
    if case["op"] == "loglikes":
        frames, d, v = case["b"] * (case["lo"] + case["hi"]) / 2, case["d"], case["v"]
        return {"bytes": (frames * d + v * d + v * case["bias"]) * e + 4 * v * case["prior"] + frames * v * SIZE[case["out"]],
                "flops": 2 * frames * v * d}
    rows, v, g, k = case["rows"], case["v"], case["given"], case["top"]
    if case["op"] == "logprobs":
        return {"bytes": rows * v * e + rows * (8 * g + 8 + 8 * k), "flops": 5 * rows * v}
    return {"bytes": 2 * rows * v * e + rows * (8 * g + 8 + 8 * k + 4 + 4 * case["entropy"]), "flops": 6 * rows * v}


def _rows(gen, shape, pad, dtype, sd=1.0):
    """A [rows, n] matrix, with `pad` > 0 the left part of one that is `pad` wider (whose rest is NaN and no one's)."""
    x = torch.randn(shape, generator=gen, device="cuda") * sd
    if not pad:
        return x.to(DTYPES[dtype])
    wide = torch.full((shape[0], shape[1] + pad), math.nan, dtype=DTYPES[dtype], device="cuda")
    wide[:, :shape[1]] = x
    return wide[:, :shape[1]]


def _scores(case, gen):
    """Scores of a model that is sure of some rows and not of others: normal ones, one of them raised; and its tokens:
    the raised one mostly, any at times, none (-1) at others."""
    rows, v, g = case["rows"], case["v"], case["given"]
    x = _rows(gen, (rows, v), case["pad"], case["dtype"], 2.0)
    best = torch.randint(0, v, (rows, 1), generator=gen, device="cuda")
    if case["masked"]:                                   # a grammar that allows one token in eight, and the raised one
        for rule in range(0, rows, 64):
            part = x[rule:rule + 64]
            if torch.rand(1, generator=gen, device="cuda").item() < case["masked"]:
                part.masked_fill_(torch.rand(part.shape, generator=gen, device="cuda") < 0.875, -math.inf)
    raised = torch.rand((rows, 1), generator=gen, device="cuda") * 12
    x.scatter_(1, best, raised.to(x.dtype))
    tokens = torch.where(torch.rand((rows, g), generator=gen, device="cuda") < 0.6, best,
                         torch.randint(0, v, (rows, g), generator=gen, device="cuda"))
    tokens = torch.where(torch.rand((rows, g), generator=gen, device="cuda") < 0.05, -1, tokens)
    return x, tokens.to(torch.int32)


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    s = dict(case)
    dt = DTYPES[case["dtype"]]
    if case["op"] == "linear":
        m, k, n = case["m"], case["k"], case["n"]
        s["x"] = _rows(gen, (m, k), case["pad"], case["dtype"])
        s["w"] = (torch.randn((n, k), generator=gen, device="cuda") / math.sqrt(k)).to(dt)
        s["b"] = torch.randn(n, generator=gen, device="cuda").mul_(0.2).to(dt) if case["bias"] else None
        s["r"] = _rows(gen, (m, n), 0, case["out"]) if case["residual"] else None
    elif case["op"] == "loglikes":
        b, t, d, v = case["b"], case["t"], case["d"], case["v"]
        s["lengths"] = torch.randint(case["lo"], case["hi"] + 1, (b,), generator=gen, device="cuda", dtype=torch.int32)
        s["x"] = torch.randn((b, t, d), generator=gen, device="cuda").to(dt)
        s["x"][torch.arange(t, device="cuda")[None, :] >= s["lengths"][:, None]] = math.nan      # padding: anything
        s["w"] = (torch.randn((v, d), generator=gen, device="cuda") * (2.0 / math.sqrt(d))).to(dt)
        s["b"] = torch.randn(v, generator=gen, device="cuda").mul_(0.2).to(dt) if case["bias"] else None
        if s["b"] is not None:
            s["b"][0] += 4.0                             # most frames are blank
        s["prior"] = torch.log_softmax(torch.randn(v, generator=gen, device="cuda"), 0) if case["prior"] else None
        s["out_buffer"] = torch.zeros((b, t, v), dtype=DTYPES[case["out"]], device="cuda")
    else:
        s["x"], s["tokens"] = _scores(case, gen)
        if case["op"] == "backward":
            rows, g, k = case["rows"], case["given"], case["top"]
            s["g_lp"] = torch.randn((rows, g), generator=gen, device="cuda") / rows
            s["g_h"] = torch.randn(rows, generator=gen, device="cuda") * (0.1 / rows) if case["entropy"] else None
            s["g_top"] = torch.randn((rows, k), generator=gen, device="cuda") / rows if k else None
            if own:
                from paper_2311_04996_amd import token_logprobs
                s["saved"] = token_logprobs(s["x"], s["tokens"], top=k)      # what the training program's forward pass left
            else:
                s["saved"] = _logprobs_plain(s["x"], s["tokens"], k)
    return s


# ---- the operators in elementary operations, 32 bits
def _act(z, act):
    if act == "relu":
        return torch.where(z > 0, z, torch.zeros_like(z))
    if act == "silu":
        return z / (1 + torch.exp(-z))
    if act == "gelu":
        return 0.5 * z * (1 + torch.erf(z * math.sqrt(0.5)))
    return z


def _linear_plain(s):
    z = s["x"].float() @ s["w"].float().t()
    if s["b"] is not None:
        z += s["b"].float()
    y = _act(z, s["act"])
    if s["scale"] != 1.0:
        y = y * s["scale"]
    if s["r"] is not None:
        y = y + s["r"].float()
    return y.to(DTYPES[s["out"]])


def _loglikes_plain(s):
    valid = torch.arange(s["t"], device="cuda")[None, :] < s["lengths"][:, None]
    z = s["x"][valid].float() @ s["w"].float().t()
    if s["b"] is not None:
        z += s["b"].float()
    z = z - z.max(-1, keepdim=True).values
    z = z - torch.log(torch.exp(z).sum(-1, keepdim=True))
    if s["prior"] is not None:
        z = z - s["prior"]
    s["out_buffer"][valid] = z.to(DTYPES[s["out"]])
    return s["out_buffer"]


def _top(x, k):
    """Indices of the k largest, equal ones by the lowest index: by whole numbers that order (value, -index)."""
    bits = (x + 0.0).view(torch.int32)
    order = torch.where(bits < 0, bits ^ 0x7fffffff, bits).long()
    order = (order << 32) + torch.arange(x.shape[-1] - 1, -1, -1, device="cuda")
    return torch.topk(order, k, dim=-1).indices


def _logprobs_plain(x, tokens, k):
    x = x.float()
    m = x.max(-1, keepdim=True).values
    d = x - m
    e = torch.exp(d)
    total = e.sum(-1, keepdim=True)
    log_total = torch.log(total)
    lse = (m + log_total)[:, 0]
    entropy = (log_total - torch.where(e > 0, e * d, 0.0).sum(-1, keepdim=True) / total)[:, 0]
    tok = tokens.long()
    lp = torch.gather(d, 1, tok.clamp(min=0)) - log_total
    lp = torch.where(tok < 0, 0.0, lp)
    out = dict(logprobs=lp, lse=lse, entropy=entropy)
    if k:
        ids = _top(x, k)
        out["top_ids"] = ids.to(torch.int32)
        out["top_logprobs"] = torch.gather(d, 1, ids) - log_total
    return out


def _backward_plain(s):
    x, f = s["x"].float(), s["saved"]
    lp = x - f["lse"][:, None]
    p = torch.exp(lp)
    tok = s["tokens"].long()
    g = torch.where(tok < 0, 0.0, s["g_lp"])
    c = -g.sum(-1, keepdim=True)
    if s["g_top"] is not None:
        c = c - s["g_top"].sum(-1, keepdim=True)
    if s["g_h"] is not None:
        dx = torch.where(p > 0, p * (c - s["g_h"][:, None] * (lp + f["entropy"][:, None])), 0.0)
    else:
        dx = p * c
    dx.scatter_add_(1, tok.clamp(min=0), g)
    if s["g_top"] is not None:
        dx.scatter_add_(1, f["top_ids"].long(), s["g_top"])
    return dx.to(s["x"].dtype)


def run(state):
    s = state
    if not own:
        if s["op"] == "linear":
            return _linear_plain(s)
        if s["op"] == "loglikes":
            return _loglikes_plain(s)
        if s["op"] == "logprobs":
            return _logprobs_plain(s["x"], s["tokens"], s["top"])
        return _backward_plain(s)
    from paper_2311_04996_amd import linear, loglikes, token_logprobs, token_logprobs_backward
    if s["op"] == "linear":
        return linear(s["x"], s["w"], s["b"], activation=s["act"], residual=s["r"], scale=s["scale"], out_dtype=DTYPES[s["out"]])
    if s["op"] == "loglikes":
        return loglikes(s["x"], s["w"], s["b"], log_prior=s["prior"], lengths=s["lengths"], out=s["out_buffer"])
    if s["op"] == "logprobs":
        r = token_logprobs(s["x"], s["tokens"], top=s["top"])
        out = dict(logprobs=r.logprobs, lse=r.lse, entropy=r.entropy)
        if s["top"]:
            out.update(top_ids=r.top_ids, top_logprobs=r.top_logprobs)
        return out
    return token_logprobs_backward(s["x"], s["saved"], s["tokens"], grad_logprobs=s["g_lp"], grad_entropy=s["g_h"], grad_top=s["g_top"])


# ---- the definitions in 64 bits
def exact(case, seed):
    s = prepare(dict(case), seed)
    if case["op"] == "linear":
        out = torch.empty((case["m"], case["n"]), dtype=torch.float64, device="cuda")
        w = s["w"].double().t().contiguous()
        for lo in range(0, case["m"], 8192):
            z = torch.matmul(s["x"][lo:lo + 8192].double(), w)
            if case["bias"]:
                z = z + s["b"].double()
            a = case["act"]
            z = z if a == "none" else z.clamp(min=0) if a == "relu" else z * torch.sigmoid(z) if a == "silu" else \
                z * 0.5 * torch.special.erfc(-z / math.sqrt(2.0))
            z = z * case["scale"]
            out[lo:lo + 8192] = z + s["r"][lo:lo + 8192].double() if case["residual"] else z
        return out
    if case["op"] == "loglikes":
        out = torch.zeros((case["b"], case["t"], case["v"]), dtype=torch.float64, device="cuda")
        w = s["w"].double().t().contiguous()
        for i, n in enumerate(s["lengths"].tolist()):
            z = torch.matmul(s["x"][i, :n].double(), w)
            if case["bias"]:
                z = z + s["b"].double()
            z = z - torch.logsumexp(z, dim=1, keepdim=True)
            out[i, :n] = z - s["prior"].double() if case["prior"] else z
        return out
    tok = s["tokens"].long()
    parts = []
    for lo in range(0, case["rows"], 512):
        x, t = s["x"][lo:lo + 512].double(), tok[lo:lo + 512]
        lse = torch.logsumexp(x, dim=1, keepdim=True)
        lp = x - lse
        p = lp.exp()
        ent = -torch.xlogy(p, p).sum(1)
        if case["op"] == "logprobs":
            given = torch.where(t < 0, 0.0, lp.gather(1, t.clamp(min=0)))
            part = dict(logprobs=given, lse=lse[:, 0], entropy=ent)
            if case["top"]:
                ids = torch.sort(x, dim=1, descending=True, stable=True).indices[:, :case["top"]]
                part.update(top_ids=ids.to(torch.int32), top_logprobs=lp.gather(1, ids))
            parts.append(part)
            continue
        dx = torch.zeros_like(p)
        weight = torch.zeros_like(p)                     # d(loss)/d(log-probability of each class)
        for j in range(case["given"]):
            col = t[:, j:j + 1]
            weight.scatter_add_(1, col.clamp(min=0), torch.where(col < 0, 0.0, s["g_lp"][lo:lo + 512, j:j + 1].double()))
        if case["top"]:
            ids = torch.sort(x, dim=1, descending=True, stable=True).indices[:, :case["top"]]
            weight.scatter_add_(1, ids, s["g_top"][lo:lo + 512].double())
        dx = weight - p * weight.sum(1, keepdim=True)
        if case["entropy"]:
            dx = dx - s["g_h"][lo:lo + 512, None].double() * torch.where(p > 0, p * (lp + ent[:, None]), 0.0)
        parts.append(dx)
    if case["op"] == "backward":
        return torch.cat(parts)
    return {k: torch.cat([q[k] for q in parts]) for k in parts[0]}
