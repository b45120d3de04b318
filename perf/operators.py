"""Timed cases of the operators at the ends of a training step: the head's loss and its gradients, the
embedding and its gradient, and the clip of all gradients.

``listed`` holds sizes that a program meets in practice, ``draw`` picks others of the same ranges,
``prepare`` makes what a program holds before a call, ``run`` is one pass (in elementary torch
operations, or through the framework's entry points where ``own`` is set), ``work`` the bytes and
operations a pass cannot do without, and ``exact`` the same outputs in 64 bits.

Kinds of pass:
  score   the loss of every row: x [N, D], w [V, D], b [V], targets y [N] (-1: no target, no loss)
  train   the loss and its gradients for upstream gradients g [N]; ``frozen``: for w and b alone
  embed   lookup of N tokens, out = scale table[token] (-1: a row of zeros)
  tables  lookup, then the table's gradient for the rows' upstream gradients
  clip    the norm over all tensors and the tensors scaled to at most ``max_norm``
"""
import math

import torch

own = False
DEV = "cuda"
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def _loss(name, kind, N, D, V, dtype, targets, bias=True, padded=0.0, frozen=False):
    return {"name": name, "kind": kind, "N": N, "D": D, "V": V, "dtype": dtype, "targets": targets, "bias": bias,
            "padded": padded, "frozen": frozen}


def _embed(name, kind, N, D, V, dtype, targets, padded=0.0):
    return {"name": name, "kind": kind, "N": N, "D": D, "V": V, "dtype": dtype, "targets": targets, "padded": padded}


def _clip(name, layers, width, dtype, share):
    return {"name": name, "kind": "clip", "layers": layers, "width": width, "dtype": dtype, "share": share}


def listed():
    return [
        # serving: how likely one token is after its prompt
        _loss("score_one_bf16", "score", 1, 2048, 32000, "bf16", "text", bias=False),
        # scoring one second of speech with the paper's head (256 mu-law classes)
        _loss("score_voice_f32", "score", 16000, 256, 256, "f32", "voice"),
        # adapting a voice's output layer to clips of unequal lengths, the layers below frozen
        _loss("train_voice_f32", "train", 16000, 256, 256, "f32", "voice", padded=0.12, frozen=True),
        # a few short sequences of odd sizes
        _loss("train_few_bf16", "train", 37, 777, 50021, "bf16", "text", bias=False),
        # odd sizes in full precision
        _loss("train_odd_f32", "train", 1531, 513, 10007, "f32", "text", padded=0.3),
        # an ordinary step over text
        _loss("train_text_bf16", "train", 4096, 1024, 32000, "bf16", "text", bias=False, padded=0.05),
        # a class for each 16-bit sample, the largest step
        _loss("train_wide_bf16", "train", 8192, 2048, 65536, "bf16", "voice"),
        # serving: the rows of one step's tokens
        _embed("embed_step_bf16", "embed", 48, 2048, 32000, "bf16", "text"),
        # a batch of utterances through the paper's input embedding
        _embed("tables_voice_f32", "tables", 512000, 64, 256, "f32", "voice", padded=0.1),
        # a step over text
        _embed("tables_text_bf16", "tables", 8191, 2048, 65536, "bf16", "text"),
        # the gradients of a 20-layer voice
        _clip("clip_voice_f32", 20, 64, "f32", 0.3),
        # the gradients of a large model, matrices in 16 bits and vectors in 32
        _clip("clip_large_bf16", 48, 1024, "bf16", 0.3),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(("score", "score", "train", "train", "train", "embed", "tables", "tables", "clip", "clip"))
    if kind == "clip":
        layers, width = _log_int(rng, 1, 48), _log_int(rng, 16, 1024)
        return {k: v for k, v in _clip("", layers, width, rng.choice(("f32", "bf16")), rng.choice((0.3, 3.0))).items()
                if k != "name"}
    dtype = rng.choice(("f32", "bf16"))
    targets = rng.choice(("text", "text", "voice"))
    if kind in ("score", "train"):
        N, D, V = _log_int(rng, 1, 16000), _log_int(rng, 32, 4096), _log_int(rng, 64, 131072)
        # at most the products and the tables of the largest listed case, products in 32 bits counting for four
        while N * D * V * (4 if dtype == "f32" else 1) > 8192 * 2048 * 65536 or D * V > 2048 * 65536:
            N, D, V = max(1, N * 3 // 4), max(32, D * 7 // 8), max(64, V * 3 // 4)
        c = _loss("", kind, N, D, V, dtype, targets, bias=rng.random() < 0.5, padded=rng.choice((0.0, 0.1, 0.5)),
                  frozen=kind == "train" and rng.random() < 0.25)
    else:
        N, D, V = _log_int(rng, 1, 512000), _log_int(rng, 16, 4096), _log_int(rng, 64, 131072)
        while N * D > 512000 * 64 or V * D > 2048 * 65536:
            N, D, V = max(1, N * 3 // 4), max(16, D * 7 // 8), max(64, V * 3 // 4)
        c = _embed("", kind, N, D, V, dtype, targets, padded=rng.choice((0.0, 0.1)))
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
    """Codes of speech (around the middle of the range, silence the commonest) or of text (the n-th
    commonest token 1 / n as likely as the first), with rows that are padding."""
    N, V = c["N"], c["V"]
    u = torch.rand(N, generator=_gen(seed, 0), device=DEV, dtype=torch.float64)
    if c["targets"] == "voice":
        s = (u - 0.5).clamp(-0.499999, 0.499999)
        t = V / 2 + V / 16 * torch.sign(s) * -torch.log(1 - 2 * s.abs()) * (s.abs() > 0.1)
    else:
        t = torch.exp(u * math.log(V + 1.0)) - 1
    t = t.floor().clamp(0, V - 1).to(torch.int32)
    if c["padded"]:
        # sequences of 64 rows, the ends of some of them empty
        row = torch.arange(N, device=DEV)
        left = torch.rand(N // 64 + 1, generator=_gen(seed, 1), device=DEV)
        empty = (row % 64) >= 64 * (1 - 2 * c["padded"] * left[row // 64])
        t[empty] = -1
    return t


def _clip_shapes(c):
    """A model of ``layers`` layers: per layer two gate matrices, the residual, the skip projection and
    their biases; an embedding, and a head of two matrices."""
    l, r = c["layers"], c["width"]
    shapes = [(256, r), (r,)]
    for _ in range(l):
        shapes += [(2 * r, r), (2 * r, r), (2 * r,), (r, r), (r,), (4 * r, r)]
    return shapes + [(4 * r,), (256, 4 * r), (256,), (256, 256), (256,)]


def prepare(case, seed):
    c = dict(case)
    dtype = DTYPES[c["dtype"]]

    def randn(shape, k, std=1.0):
        return torch.randn(shape, generator=_gen(seed, k), device=DEV) * std

    if c["kind"] == "clip":
        # a layer's gradients are smaller the deeper it lies
        grads, g = [], _gen(seed, 2)
        for i, shape in enumerate(_clip_shapes(c)):
            t = torch.randn(shape, generator=g, device=DEV) * (1e-3 * 0.97 ** (i // 6))
            grads.append(t.to(dtype if len(shape) == 2 else torch.float32))
        norm = math.sqrt(sum(t.numel() * (1e-3 * 0.97 ** (i // 6)) ** 2 for i, t in enumerate(grads)))
        # the clipped gradients go into an optimizer's flat buffers, one for each type
        s = {"c": c, "grads": grads, "max_norm": c["share"] * norm, "outs": [], "flat": {}}
        at = {}
        for t in grads:
            at[t.dtype] = at.get(t.dtype, 0) + t.numel()
        s["flat"] = {str(k): torch.zeros(n, dtype=k, device=DEV) for k, n in at.items()}
        at = {}
        for t in grads:
            n = at.get(t.dtype, 0)
            s["outs"].append(s["flat"][str(t.dtype)][n:n + t.numel()].view(t.shape))
            at[t.dtype] = n + t.numel()
        return s
    N, D, V = c["N"], c["D"], c["V"]
    s = {"c": c, "y": _tokens(c, seed)}
    if c["kind"] in ("embed", "tables"):
        s["scale"] = math.sqrt(D)
        s["table"] = randn((V, D), 2, 1 / math.sqrt(D)).to(dtype)
        if c["kind"] == "tables":
            s["dout"] = randn((N, D), 3, 1e-2).to(dtype)
        return s
    # hidden values after a relu, as the framework's head has them, or of any sign
    x = randn((N, D), 2)
    s["x"] = (x.clamp(min=0) if c["targets"] == "voice" else x).to(dtype)
    s["w"] = randn((V, D), 3, 1.5 / math.sqrt(D)).to(dtype)
    s["b"] = None
    if c["bias"]:
        # common classes are likelier
        v = torch.arange(V, device=DEV, dtype=torch.float32)
        b = -8 * ((v - V / 2) / (V / 2)).abs() if c["targets"] == "voice" else -torch.log1p(v)
        s["b"] = b + randn((V,), 4, 0.1)
    if c["kind"] == "train":
        ok = s["y"] >= 0
        s["g"] = ok.float() / ok.sum().clamp(min=1)
    return s


# ------------------------------------------------------------------------------------------------
# the operators
# ------------------------------------------------------------------------------------------------
def run(state):
    return _own(state) if own else _plain(state)


def _own(s):
    import paper_1702_07825_amd as wn

    c = s["c"]
    if c["kind"] == "clip":
        norm = wn.clip_gradients(s["grads"], s["max_norm"], outs=s["outs"])
        return {"norm": norm, "grads": s["flat"]}
    if c["kind"] in ("embed", "tables"):
        out = wn.embed(s["table"], s["y"], scale=s["scale"])
        if c["kind"] == "embed":
            return {"out": out}
        return {"out": out, "dtable": wn.embed_backward(s["dout"], s["y"], c["V"], scale=s["scale"])}
    loss, lse = wn.head_loss(s["x"], s["w"], s["y"], b=s["b"])
    if c["kind"] == "score":
        return {"loss": loss, "lse": lse}
    need = (() if c["frozen"] else ("dx",)) + ("dw",) + (() if s["b"] is None else ("db",))
    dx, dw, db = wn.head_loss_backward(s["x"], s["w"], s["y"], lse, s["g"], b=s["b"], need=need)
    return {"loss": loss, "dx": dx, "dw": dw, "db": db}


def _plain(s):
    c = s["c"]
    if c["kind"] == "clip":
        squares = [t.float().square().sum(dtype=torch.float64) for t in s["grads"]]
        norm = torch.stack(squares).sum().sqrt().float()
        scale = (s["max_norm"] / norm).clamp(max=1.0)
        [o.copy_(t.float() * scale) for t, o in zip(s["grads"], s["outs"])]
        return {"norm": norm, "grads": s["flat"]}
    y = s["y"].long()
    ok = y >= 0
    if c["kind"] in ("embed", "tables"):
        out = s["table"][y.clamp(min=0)].float() * s["scale"]
        out = torch.where(ok[:, None], out, 0.0).to(s["table"].dtype)
        if c["kind"] == "embed":
            return {"out": out}
        # running sums over the rows in the tokens' order, taken at each token's last row and at the one
        # before its first: in 64 bits, since they pass over all rows
        y, order = torch.sort(y, stable=True)
        total = torch.zeros((c["N"] + 1, c["D"]), device=DEV, dtype=torch.float64)
        torch.cumsum(s["dout"][order].double(), dim=0, out=total[1:])
        v = torch.arange(c["V"], device=DEV)
        d = total[torch.searchsorted(y, v, right=True)] - total[torch.searchsorted(y, v)]
        return {"out": out, "dtable": (d * s["scale"]).to(s["dout"].dtype)}
    x, w = s["x"].float(), s["w"].float()
    logits = x @ w.t()
    if s["b"] is not None:
        logits += s["b"]
    top = logits.max(dim=1, keepdim=True).values
    lse = (logits - top).exp().sum(dim=1, keepdim=True).log() + top
    at = torch.where(ok, y, 0)[:, None]
    loss = torch.where(ok, (lse - logits.gather(1, at))[:, 0], 0.0)
    if c["kind"] == "score":
        return {"loss": loss, "lse": lse[:, 0]}
    q = (logits - lse).exp()
    q.scatter_add_(1, at, torch.full_like(lse, -1.0))
    q *= torch.where(ok, s["g"], 0.0)[:, None]
    out = {"loss": loss}
    if not c["frozen"]:
        out["dx"] = (q @ w).to(s["x"].dtype)
    out["dw"] = (q.t() @ x).to(s["w"].dtype)
    if s["b"] is not None:
        out["db"] = q.sum(dim=0)
    return out


def work(case):
    c = case
    e = 4 if c["dtype"] == "f32" else 2
    if c["kind"] == "clip":
        shapes = _clip_shapes(c)
        n = [math.prod(s) * (e if len(s) == 2 else 4) for s in shapes]
        return {"bytes": 2.0 * sum(n) + 4, "flops": 3.0 * sum(math.prod(s) for s in shapes)}
    N, D, V = c["N"], c["D"], c["V"]
    if c["kind"] in ("embed", "tables"):
        rows = min(N, V)
        look = 4.0 * N + e * D * (rows + N)
        if c["kind"] == "embed":
            return {"bytes": look, "flops": 1.0 * N * D}
        return {"bytes": look + 4.0 * N + e * D * (N + V), "flops": 2.0 * N * D + V * D}
    read = e * D * (N + V) + 4.0 * N + (4.0 * V if c["bias"] else 0.0)
    if c["kind"] == "score":
        return {"bytes": read + 8.0 * N, "flops": 2.0 * N * D * V}
    # the loss and the gradients share one read of the inputs; the logits, dx and dw are a product each
    write = 4.0 * N + e * D * (V + (0 if c["frozen"] else N)) + (4.0 * V if c["bias"] else 0.0)
    return {"bytes": read + 4.0 * N + write, "flops": (4.0 if c["frozen"] else 6.0) * N * D * V}


# ------------------------------------------------------------------------------------------------
# the definitions in 64 bits
# ------------------------------------------------------------------------------------------------
def exact(case, seed):
    c = dict(case)
    s = prepare(c, seed)
    if c["kind"] == "clip":
        total = sum(float(t.double().pow(2).sum()) for t in s["grads"])
        norm = math.sqrt(total)
        factor = min(1.0, s["max_norm"] / norm)
        flat = {k: torch.cat([t.double().flatten() * factor for t in s["grads"] if str(t.dtype) == k]) for k in s["flat"]}
        return {"norm": torch.tensor(norm, dtype=torch.float64), "grads": flat}
    tokens = s["y"]
    keep = (tokens >= 0).nonzero()[:, 0]
    ids = tokens[keep].long()
    if c["kind"] in ("embed", "tables"):
        out = torch.zeros((c["N"], c["D"]), dtype=torch.float64, device=DEV)
        out[keep] = s["scale"] * s["table"].double()[ids]
        if c["kind"] == "embed":
            return {"out": out}
        grad = torch.zeros((c["V"], c["D"]), dtype=torch.float64, device=DEV)
        grad.index_put_((ids,), s["scale"] * s["dout"].double()[keep], accumulate=True)
        return {"out": out, "dtable": grad}
    x, w = s["x"].double(), s["w"].double()
    z = torch.mm(x, w.t().contiguous())
    if s["b"] is not None:
        z = z + s["b"].double()
    lse = torch.logsumexp(z, dim=1)
    loss = torch.zeros(c["N"], dtype=torch.float64, device=DEV)
    loss[keep] = lse[keep] - z[keep, ids]
    if c["kind"] == "score":
        return {"loss": loss, "lse": lse}
    p = torch.exp(z.sub_(lse[:, None]))
    del z
    r = p[keep]
    r[torch.arange(len(keep), device=DEV), ids] -= 1
    r *= s["g"].double()[keep, None]
    out = {"loss": loss}
    if not c["frozen"]:
        out["dx"] = torch.zeros((c["N"], c["D"]), dtype=torch.float64, device=DEV)
        out["dx"][keep] = torch.mm(r, w)
    out["dw"] = torch.mm(r.t().contiguous(), x[keep])
    if s["b"] is not None:
        out["db"] = r.sum(dim=0)
    return out
