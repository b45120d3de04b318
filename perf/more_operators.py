"""Timed cases of what a policy's training and a tokens' scoring take beside the loss: log probabilities with the
entropy and the top alternatives, their gradients, and updates orthogonalised by Newton-Schulz products.

``listed`` holds sizes that a program meets in practice, ``draw`` picks others of the same ranges,
``prepare`` makes what a program holds before a call, ``run`` is one pass (in elementary torch
operations, or through the framework's entry points where ``own`` is set), ``work`` the bytes and
operations a pass cannot do without, and ``exact`` the same outputs in 64 bits.

Kinds of pass:
  probe   of every row: the log probability of its token y (-1: none, 0), the entropy, log sum exp, and the ``top``
          likeliest classes (ties: the lowest index) with their log probabilities
  policy  log probabilities and entropies, then the gradients of sum(g logprob + h entropy) for x, w (and b)
  ortho   every matrix of a model: X = G / (|G| + eps), five times X <- a X + (b X X' + c (X X')^2) X, times its scale
"""
import math

import torch

own = False
DEV = "cuda"
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
STEPS, COEFFICIENTS, EPS = 5, (3.4445, -4.7750, 2.0315), 1e-7


def _rows(name, kind, N, D, V, dtype, tokens, top=0, bias=True, padded=0.0):
    return {"name": name, "kind": kind, "N": N, "D": D, "V": V, "dtype": dtype, "tokens": tokens, "top": top, "bias": bias,
            "padded": padded}


def _ortho(name, layers, width, dtype, rank):
    return {"name": name, "kind": "ortho", "layers": layers, "width": width, "dtype": dtype, "rank": rank}


def listed():
    return [
        # serving: one token's distribution, with the alternatives that an interface shows
        _rows("probe_one_bf16", "probe", 1, 2048, 32000, "bf16", "text", top=5, bias=False),
        # serving: a step's tokens of a few requests, odd sizes in full precision
        _rows("probe_few_f32", "probe", 37, 777, 50021, "f32", "text", top=20),
        # one second of speech through the paper's head (256 mu-law classes)
        _rows("probe_voice_f32", "probe", 16000, 256, 256, "f32", "voice", top=3),
        # the log probabilities of prompts, their ends padded
        _rows("probe_text_bf16", "probe", 4096, 1024, 65536, "bf16", "text", top=8, bias=False, padded=0.05),
        # one short answer
        _rows("policy_few_bf16", "policy", 61, 1024, 32000, "bf16", "text", bias=False),
        # a voice's output layer
        _rows("policy_voice_f32", "policy", 16000, 256, 256, "f32", "voice", padded=0.12),
        # odd sizes in full precision, a third of the rows prompt
        _rows("policy_odd_f32", "policy", 1021, 515, 9973, "f32", "text", padded=0.3),
        # an ordinary step over text, the largest
        _rows("policy_text_bf16", "policy", 8192, 2048, 65536, "bf16", "text", bias=False, padded=0.1),
        # the smallest model's two matrices of a layer and its head
        _ortho("ortho_small_f32", 1, 32, "f32", 4),
        # all matrices of a 20-layer voice
        _ortho("ortho_voice_f32", 20, 64, "f32", 8),
        # odd sizes
        _ortho("ortho_odd_bf16", 3, 333, "bf16", 16),
        # the matrices of a large model
        _ortho("ortho_large_bf16", 6, 2048, "bf16", 32),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(("probe", "probe", "policy", "policy", "ortho", "ortho"))
    dtype = rng.choice(("f32", "bf16"))
    if kind == "ortho":
        layers, width = _log_int(rng, 1, 20), _log_int(rng, 16, 2048)
        # at most the products of the largest listed case, those in 32 bits counting for eight
        while layers * width ** 3 * (8 if dtype == "f32" else 1) > 6 * 2048 ** 3:
            layers, width = max(1, layers * 3 // 4), width * 7 // 8
        c = _ortho("", layers, width, dtype, rng.choice((1, 4, 32)))
    else:
        tokens = rng.choice(("text", "text", "voice"))
        N, D, V = _log_int(rng, 1, 16000), _log_int(rng, 32, 4096), _log_int(rng, 64, 131072)
        # at most the products and the tables of the largest listed case, products in 32 bits counting for four
        while N * D * V * (4 if dtype == "f32" else 1) > 8192 * 2048 * 65536 or D * V > 2048 * 65536:
            N, D, V = max(1, N * 3 // 4), max(32, D * 7 // 8), max(64, V * 3 // 4)
        c = _rows("", kind, N, D, V, dtype, tokens, top=rng.choice((0, 1, 5, 20)) if kind == "probe" else 0,
                  bias=rng.random() < 0.5, padded=rng.choice((0.0, 0.1, 0.5)))
    del c["name"]
    return c


# ------------------------------------------------------------------------------------------------
# inputs
# ------------------------------------------------------------------------------------------------
def _gen(seed, k):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed) * 16 + k)
    return g


def _tokens(c, seed):
    """Codes of speech (around the middle of the range) or of text (the n-th commonest token 1 / n as likely as the
    first), with rows that are padding."""
    N, V = c["N"], c["V"]
    u = torch.rand(N, generator=_gen(seed, 0), device=DEV, dtype=torch.float64)
    if c["tokens"] == "voice":
        s = (u - 0.5).clamp(-0.499999, 0.499999)
        t = V / 2 + V / 16 * torch.sign(s) * -torch.log(1 - 2 * s.abs())
    else:
        t = torch.exp(u * math.log(V + 1.0)) - 1
    t = t.floor().clamp(0, V - 1).to(torch.int32)
    if c["padded"]:
        # sequences of 64 rows, the ends of some of them empty
        row = torch.arange(N, device=DEV)
        left = torch.rand(N // 64 + 1, generator=_gen(seed, 1), device=DEV)
        t[(row % 64) >= 64 * (1 - 2 * c["padded"] * left[row // 64])] = -1
    return t


def _shapes(c):
    """A model of ``layers`` layers: per layer two gate matrices, the residual and the skip projection; the head's
    two matrices."""
    r = c["width"]
    return [(2 * r, r), (2 * r, r), (r, r), (4 * r, r)] * c["layers"] + [(256, 4 * r), (256, 256)]


def prepare(case, seed):
    c = dict(case)
    dtype = DTYPES[c["dtype"]]

    def randn(shape, k, std=1.0):
        return torch.randn(shape, generator=_gen(seed, k), device=DEV) * std

    if c["kind"] == "ortho":
        # a momentum: a few directions that the batches agree on, above the noise of each
        g, grads = _gen(seed, 2), []
        for i, (m, n) in enumerate(_shapes(c)):
            k = min(c["rank"], m, n)
            strength = 2.0 / (1.0 + torch.arange(k, device=DEV))
            u, v = torch.randn((m, k), generator=g, device=DEV), torch.randn((k, n), generator=g, device=DEV)
            t = torch.randn((m, n), generator=g, device=DEV) + (u * strength) @ v
            grads.append((t * (1e-3 * 0.97 ** (i // 4))).to(dtype))
        # the updates go into an optimizer's flat buffer; tall matrices move further, so that their outputs do
        flat, outs, at = torch.zeros(sum(t.numel() for t in grads), dtype=dtype, device=DEV), [], 0
        for t in grads:
            outs.append(flat[at:at + t.numel()].view(t.shape))
            at += t.numel()
        return {"c": c, "grads": grads, "flat": flat, "outs": outs,
                "scales": [0.02 * math.sqrt(max(1.0, t.shape[0] / t.shape[1])) for t in grads]}
    N, D, V = c["N"], c["D"], c["V"]
    s = {"c": c, "y": _tokens(c, seed)}
    # hidden values after a relu, as the framework's head has them, or of any sign
    x = randn((N, D), 2)
    s["x"] = (x.clamp(min=0) if c["tokens"] == "voice" else x).to(dtype)
    s["w"] = randn((V, D), 3, 1.5 / math.sqrt(D)).to(dtype)
    s["b"] = None
    if c["bias"]:
        # common classes are likelier
        v = torch.arange(V, device=DEV, dtype=torch.float32)
        s["b"] = (-8 * ((v - V / 2) / (V / 2)).abs() if c["tokens"] == "voice" else -torch.log1p(v)) + randn((V,), 4, 0.1)
    if c["kind"] == "policy":
        # advantages of either sign, and a bonus on the entropy
        n = (s["y"] >= 0).sum().clamp(min=1)
        s["g"] = randn((N,), 5) / n
        s["h"] = torch.full((N,), 0.05, device=DEV) / n
    return s


# ------------------------------------------------------------------------------------------------
# the operators
# ------------------------------------------------------------------------------------------------
def run(state):
    return _own(state) if own else _plain(state)


def _own(s):
    import paper_1702_07825_amd as wn

    c = s["c"]
    if c["kind"] == "ortho":
        wn.orthogonalize(s["grads"], scales=s["scales"], coefficients=[COEFFICIENTS] * STEPS, eps=EPS, outs=s["outs"])
        return {"updates": s["flat"]}
    logprob, entropy, lse, ids, alternatives = wn.head_logprobs(s["x"], s["w"], s["y"], b=s["b"], top=c["top"])
    out = {"logprob": logprob, "entropy": entropy}
    if c["kind"] == "probe":
        out["lse"] = lse
        if c["top"]:
            out["ids"], out["alternatives"] = ids, alternatives
        return out
    need = ("dx", "dw") if s["b"] is None else ("dx", "dw", "db")
    out["dx"], out["dw"], db = wn.head_logprobs_backward(s["x"], s["w"], s["y"], lse, entropy, s["g"], s["h"], b=s["b"], need=need)
    if db is not None:
        out["db"] = db
    return out


def _plain_ortho(g, scale):
    a, b, c = COEFFICIENTS
    x = g.float()
    tall = x.shape[0] > x.shape[1]
    if tall:
        x = x.t()
    x = x / (x.square().sum().sqrt() + EPS)
    for _ in range(STEPS):
        gram = x @ x.t()
        x = a * x + (b * gram + c * (gram @ gram)) @ x
    return (x.t() if tall else x) * scale


def _plain_top(s, logits, lse):
    """The likeliest classes: some more than wanted in 32 bits, then these in 64, where classes next to each other
    keep their order."""
    c = s["c"]
    ids = logits.topk(min(c["V"], c["top"] + 8), dim=1).indices.sort(dim=1).values
    at = torch.empty(ids.shape, dtype=torch.float64, device=DEV)
    rows = max(1, (1 << 27) // (ids.shape[1] * c["D"]))
    for n in range(0, c["N"], rows):
        at[n:n + rows] = (s["w"][ids[n:n + rows]].double() * s["x"][n:n + rows, None].double()).sum(dim=2)
    if s["b"] is not None:
        at += s["b"].double()[ids]
    at, order = at.sort(dim=1, descending=True, stable=True)
    ids = ids.gather(1, order)[:, :c["top"]]
    return ids.to(torch.int32), (at[:, :c["top"]] - lse.double()).float()


def _plain(s):
    c = s["c"]
    if c["kind"] == "ortho":
        for g, scale, out in zip(s["grads"], s["scales"], s["outs"]):
            out.copy_(_plain_ortho(g, scale))
        return {"updates": s["flat"]}
    y = s["y"].long()
    ok = y >= 0
    x, w = s["x"].float(), s["w"].float()
    logits = x @ w.t()
    if s["b"] is not None:
        logits += s["b"]
    largest = logits.max(dim=1, keepdim=True).values
    lse = (logits - largest).exp().sum(dim=1, keepdim=True).log() + largest
    out = {}
    if c["kind"] == "probe":
        out["lse"] = lse[:, 0]
        if c["top"]:
            out["ids"], out["alternatives"] = _plain_top(s, logits, lse)
    logp = logits.sub_(lse)
    at = torch.where(ok, y, 0)[:, None]
    out["logprob"] = torch.where(ok, logp.gather(1, at)[:, 0], 0.0)
    p = logp.exp()
    out["entropy"] = -(p * logp).sum(dim=1)
    if c["kind"] == "probe":
        return out
    g, h = torch.where(ok, s["g"], 0.0)[:, None], torch.where(ok, s["h"], 0.0)[:, None]
    q = logp.add_(out["entropy"][:, None]).mul_(h).add_(g).mul_(p).neg_()
    q.scatter_add_(1, at, g)
    out["dx"] = (q @ w).to(s["x"].dtype)
    out["dw"] = (q.t() @ x).to(s["w"].dtype)
    if s["b"] is not None:
        out["db"] = q.sum(dim=0)
    return out


def work(case):
    c = case
    e = 4 if c["dtype"] == "f32" else 2
    if c["kind"] == "ortho":
        flops = 0.0
        for s in _shapes(c):
            m, n = min(s), max(s)
            # the two products that give symmetric matrices need half of their sums
            flops += STEPS * (1.0 * m * m * n + 1.0 * m * m * m + 2.0 * m * m * n)
        return {"bytes": 2.0 * e * sum(m * n for m, n in _shapes(c)), "flops": flops}
    N, D, V = c["N"], c["D"], c["V"]
    read = e * D * (N + V) + 4.0 * N + (4.0 * V if c["bias"] else 0.0)
    if c["kind"] == "probe":
        return {"bytes": read + 12.0 * N + 8.0 * N * c["top"], "flops": 2.0 * N * D * V}
    # the values and the gradients share one read of the inputs; the logits, dx and dw are a product each
    write = 8.0 * N + e * D * (V + N) + (4.0 * V if c["bias"] else 0.0)
    return {"bytes": read + 8.0 * N + write, "flops": 6.0 * N * D * V}


# ------------------------------------------------------------------------------------------------
# the definitions in 64 bits
# ------------------------------------------------------------------------------------------------
def exact(case, seed):
    c = dict(case)
    s = prepare(c, seed)
    if c["kind"] == "ortho":
        # an odd polynomial of the singular values, from the side of the shorter rows: X (a + b S + c S^2), S = X' X
        found = []
        for t, scale in zip(s["grads"], s["scales"]):
            z = t.double()
            wide = z.shape[1] > z.shape[0]
            if wide:
                z = z.t().contiguous()
            z = z / (torch.linalg.matrix_norm(z) + EPS)
            unit = torch.eye(z.shape[1], dtype=torch.float64, device=DEV)
            for _ in range(STEPS):
                square = torch.mm(z.t().contiguous(), z)
                z = torch.mm(z, COEFFICIENTS[0] * unit + torch.mm(square, COEFFICIENTS[1] * unit + COEFFICIENTS[2] * square))
            found.append(scale * (z.t() if wide else z).flatten())
        return {"updates": torch.cat(found)}
    N, V = c["N"], c["V"]
    keep = (s["y"] >= 0).nonzero()[:, 0]
    token = s["y"][keep].long()
    x, w = s["x"].double(), s["w"].double()
    z = torch.mm(x, w.t().contiguous())
    if s["b"] is not None:
        z += s["b"].double()
    lse = torch.logsumexp(z, dim=1)
    out = {"logprob": torch.zeros(N, dtype=torch.float64, device=DEV)}
    out["logprob"][keep] = z[keep, token] - lse[keep]
    if c["kind"] == "probe":
        out["lse"] = lse
        if c["top"]:
            ids = torch.sort(torch.topk(z, min(V, c["top"] + 8), dim=1).indices, dim=1).values
            best, order = torch.sort(torch.gather(z, 1, ids), dim=1, descending=True, stable=True)
            out["ids"] = torch.gather(ids, 1, order)[:, :c["top"]].to(torch.int32)
            out["alternatives"] = best[:, :c["top"]] - lse[:, None]
    z -= lse[:, None]
    q = torch.exp(z)
    entropy = torch.stack([-torch.dot(a, b) for a, b in zip(q, z)]) if N < 64 else -torch.einsum("nv,nv->n", q, z)
    out["entropy"] = entropy
    if c["kind"] == "probe":
        return out
    g, h = torch.zeros_like(lse), torch.zeros_like(lse)
    g[keep], h[keep] = s["g"].double()[keep], s["h"].double()[keep]
    z += entropy[:, None]
    z *= h[:, None]
    z += g[:, None]
    q *= z
    q.neg_()
    del z
    q[keep, token] += g[keep]
    out["dx"] = torch.mm(q, w)
    out["dw"] = torch.mm(q.t().contiguous(), x)
    if s["b"] is not None:
        out["db"] = q.sum(dim=0)
    return out
