"""The loss of an output layer and its gradients (wn_loss, wn_loss_backward) against the formulas in 64 bits.

Tolerances.  u = 2^-24 is fp32's half step.  A logit is a sum of D products x w and a bias; with
S = sum |x w| its error is at most
  bf16: D u S (products are exact in fp32)
  fp32: 3 * 2^-22 S (each value is held to 2^-22 of itself or 2^-39 of its row's largest, and the product of the
        two low parts, at most 2^-22 of the product, is left out) + 3 D u S + 2^-38 D max|x| max|w|
plus u (|l| + |b|) for the bias: E.  exp(l - m) is off by a relative 2 E + 2^-23 (1 + |l - m|) (its argument's
rounding twice, exp2's own last place) and the sum of V of them by (V / 2048 + 128) u (the lengths of the
chains: 32 a lane, 16 the joins, then a tile of 128 in 16 parts), so
  loss: 2 E + (V / 2048 + 128) u + 2^-22 (1 + |lse| + |l_y|)
  p:    a relative d = 2 E + tol(lse) + 2^-22 (1 + |l - lse|)
With A = sum |q w| (or over rows |q x|) over K terms, the gradients' products are off by
  bf16: (2^-8 + K u) A for q's rounding and the sum, and 2^-8 of the result
  fp32: (3 * 2^-22 + 3 K u) A + 2^-38 K max max, and 4 u of the result
and by sum d |p| g |w| for q.  Probabilities and products below 2^-126, fp32's smallest normal value, may vanish:
another 2^-126 (1 + max|w|) for each term.
"""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
U = 2.0 ** -24


def _inputs(N, D, V, dtype, seed, bias=True, ignored=0.2, std=1.0):
    g = torch.Generator().manual_seed(seed)
    x = (torch.randn((N, D), generator=g) * std).to(dtype)
    w = (torch.randn((V, D), generator=g) * 1.5 / D ** 0.5 / std).to(dtype)
    b = torch.randn((V,), generator=g) if bias else None
    y = torch.randint(0, V, (N,), generator=g, dtype=torch.int32)
    off = torch.rand((N,), generator=g) < ignored
    y[off] = torch.where(torch.arange(int(off.sum())) % 2 == 0, -1, V).to(torch.int32)
    grad = torch.rand((N,), generator=g) / N - 0.2 / N
    return x, w, b, y, grad


def _formulas(x, w, b, y, grad):
    """Results in 64 bits and the tolerances of each."""
    f32 = x.dtype == torch.float32
    N, D = x.shape
    V = w.shape[0]
    X, W = x.double(), w.double()
    ok = (y >= 0) & (y < V)
    B = torch.zeros(V, dtype=torch.float64, device=x.device) if b is None else b.double()
    l = X @ W.t().contiguous() + B
    S = X.abs() @ W.abs().t().contiguous()
    far = 2.0 ** -38 * float(X.abs().max()) * float(W.abs().max())
    fin = torch.where(torch.isfinite(l), l, torch.zeros_like(l))
    E = ((3 * 2.0 ** -22 + 3 * D * U) * S + D * far if f32 else D * U * S) + U * (fin.abs() + torch.where(torch.isfinite(B), B, 0.0).abs())
    lse = torch.logsumexp(l, dim=1)
    yc = torch.where(ok, y, 0).long()[:, None]
    ly = l.gather(1, yc)[:, 0]
    loss = torch.where(ok, lse - ly, 0.0)
    Em = E.max(dim=1).values
    t_lse = Em + (V / 2048 + 128) * U + 2.0 ** -22 * (1 + lse.abs())
    t_loss = 2 * Em + (V / 2048 + 128) * U + 2.0 ** -22 * (1 + lse.abs() + ly.abs())
    p = (l - lse[:, None]).exp()
    d = 2 * E + t_lse[:, None] + 2.0 ** -22 * (1 + (fin - lse[:, None]).abs())
    gr = torch.where(ok, grad.double(), 0.0)[:, None]
    q = p.clone()
    q.scatter_add_(1, yc, -torch.ones_like(lse)[:, None])
    q *= gr
    dq = d * p * gr.abs()
    out = {"loss": (loss, t_loss), "lse": (lse, t_lse)}
    for name, a, c, qq, e in (("dx", q, W, q.abs(), dq), ("dw", q.t().contiguous(), X, q.abs().t().contiguous(), dq.t().contiguous())):
        K = a.shape[1]
        v, A = a @ c, qq @ c.abs()
        if f32:
            m = float(qq.max()) if name == "dw" else float(gr.abs().max())
            t = (3 * 2.0 ** -22 + 3 * K * U) * A + 2.0 ** -38 * K * float(gr.abs().max()) * float(c.abs().max()) + 4 * U * v.abs()
        else:
            t = (2.0 ** -8 + K * U) * A + 2.0 ** -8 * v.abs()
        out[name] = (v, t + e @ c.abs() + K * 2.0 ** -126 * (1 + float(c.abs().max())))
    out["db"] = (q.sum(dim=0), dq.sum(dim=0) + N * U * q.abs().sum(dim=0) + N * 2.0 ** -126)
    return out


def _near(got, want, name):
    v, t = want
    got = got.double()
    assert got.shape == v.shape, name
    bad = ~((got - v).abs() <= t)
    if bool(bad.any()):
        at = tuple(int(i) for i in bad.nonzero()[0])
        raise AssertionError("%s%s: %r, not %r within %.3g (%d of %d off)" % (name, at, float(got[at]), float(v[at]),
                                                                        float(t[at]), int(bad.sum()), bad.numel()))


def _check(x, w, b, y, grad, need=("dx", "dw", "db"), device="cuda"):
    import paper_1702_07825_amd as wn
    print("loss", tuple(x.shape), tuple(w.shape), x.dtype, flush=True)
    want = _formulas(*(None if t is None else t.to(device) for t in (x, w, b, y, grad)))
    X, W, B, Y, G = (None if t is None else t.cuda() for t in (x, w, b, y, grad))
    loss, lse = wn.head_loss(X, W, Y, b=B)
    got = wn.head_loss_backward(X, W, Y, lse, G, b=B, need=need)
    _near(loss.to(device), want["loss"], "loss")
    _near(lse.to(device), want["lse"], "lse")
    for name, t in zip(("dx", "dw", "db"), got):
        assert (t is None) == (name not in need)
        if t is not None:
            _near(t.to(device), want[name], name)
    return loss, lse, got


SIZES = [(1, 1, 1), (1, 64, 256), (1, 1000, 777), (2, 7, 5), (15, 64, 100), (16, 64, 256), (17, 65, 129), (33, 8, 2000),
         (64, 32, 1000), (64, 1025, 65), (31, 300, 4000), (5, 1100, 300), (4, 100, 17000), (5, 100, 17000), (16, 520, 16400), (16, 2500, 70), (30, 1030, 100), (64, 1999, 33), (1, 5000, 1), (48, 513, 2049), (65, 64, 70), (100, 100, 127), (127, 72, 128), (128, 128, 128), (129, 256, 257), (200, 100, 3001), (256, 256, 256),
         (300, 513, 777), (1000, 64, 300), (2111, 40, 64)]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("N,D,V", SIZES)
def test_sizes(N, D, V, dtype):
    _check(*_inputs(N, D, V, dtype, seed=N + D + V))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("N,D,V", [(4100, 300, 8200), (5, 2048, 20000), (16000, 32, 9000), (20000, 256, 256)])
def test_large(N, D, V, dtype):
    """Tiles that fill the chip; several pieces of the vocabulary forwards (5 rows) and backwards (16000); sums
    over the rows in parts (20000)."""
    _check(*_inputs(N, D, V, dtype, seed=3), device="cuda")


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
def test_without_a_bias_and_each_gradient_alone(dtype):
    args = _inputs(70, 48, 300, dtype, seed=5, bias=False)
    _, _, all_ = _check(*args)
    for i, k in enumerate(("dx", "dw", "db")):
        _, _, got = _check(*args, need=(k,))
        assert torch.equal(got[i], all_[i])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("N", [3, 16, 40, 150])
def test_padding_holds_anything(N, dtype):
    """NaN and infinities in rows without a target, in their upstream gradients and in their lse: the other rows'
    results are those of the call with zeros there."""
    import paper_1702_07825_amd as wn
    x, w, b, y, grad = _inputs(N, 72, 260, dtype, seed=6, ignored=0.4)
    y[1] = -1
    off = (y < 0) | (y >= 260)
    clean = x.clone()
    clean[off] = 0
    bad = x.clone()
    bad[off] = float("nan")
    bad[off.nonzero()[0]] = float("inf")
    grad_bad = grad.clone()
    grad_bad[off] = float("nan")
    _, _, want = _check(clean, w, b, y, grad)
    X, W, B, Y = bad.cuda(), w.cuda(), b.cuda(), y.cuda()
    loss, lse = wn.head_loss(X, W, Y, b=B)
    assert not bool(loss[off.cuda()].any())
    got = wn.head_loss_backward(X, W, Y, lse, grad_bad.cuda(), b=B)
    assert not bool(got[0][off.cuda()].any())
    for a, c in zip(got, want):
        assert torch.equal(a, c)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("N", [1, 40, 140])
def test_no_row_has_a_target(N, dtype):
    import paper_1702_07825_amd as wn
    x, w, b, y, grad = _inputs(N, 24, 90, dtype, seed=7)
    y[:] = -5
    X, W, B, Y, G = (t.cuda() for t in (x, w, b, y, grad))
    loss, lse = wn.head_loss(X, W, Y, b=B)
    assert not bool(loss.any())
    for t in wn.head_loss_backward(X, W, Y, lse, G, b=B):
        assert not bool(t.any())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("mask", [-float("inf"), torch.finfo(torch.float32).min], ids=["inf", "lowest"])
@pytest.mark.parametrize("N", [1, 30, 90])
def test_masked_classes(N, dtype, mask):
    """Classes that a bias masks, whole tiles of them among them."""
    x, w, b, y, grad = _inputs(N, 40, 700, dtype, seed=8, ignored=0)
    b[100:600] = mask
    b[0] = mask
    y = torch.where((y >= 100) & (y < 600) | (y == 0), 650, y).to(torch.int32)
    _check(x, w, b, y, grad)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
def test_every_class_masked_by_the_lowest_value(dtype):
    """The logits' differences are lost beside the mask, so the classes are alike: loss log V, q = g (1 / V - [v = y])."""
    import paper_1702_07825_amd as wn
    x, w, b, y, grad = _inputs(90, 40, 700, dtype, seed=8, ignored=0)
    b[:] = torch.finfo(torch.float32).min
    loss, lse = wn.head_loss(x.cuda(), w.cuda(), y.cuda(), b=b.cuda())
    assert bool(((loss.cpu().double() - np.log(700)).abs() <= 1e-5).all())
    db = wn.head_loss_backward(x.cuda(), w.cuda(), y.cuda(), lse, grad.cuda(), b=b.cuda(), need=("db",))[2]
    # (lse itself is the mask: log 700 is lost in it, and exp(l - lse) is 1)
    q = torch.ones((90, 700), dtype=torch.float64)
    q[torch.arange(90), y.long()] -= 1
    assert bool(((db.cpu().double() - (q * grad.double()[:, None]).sum(dim=0)).abs() <= 1e-6).all())


def test_a_masked_target_has_an_infinite_loss():
    import paper_1702_07825_amd as wn
    x, w, b, y, grad = _inputs(20, 40, 300, torch.float32, seed=9, ignored=0)
    b[7] = -float("inf")
    y[3] = 7
    loss, lse = wn.head_loss(x.cuda(), w.cuda(), y.cuda(), b=b.cuda())
    assert float(loss[3]) == float("inf") and bool(torch.isfinite(loss[:3]).all()) and bool(torch.isfinite(loss[4:]).all())
    for t in wn.head_loss_backward(x.cuda(), w.cuda(), y.cuda(), lse, grad.cuda(), b=b.cuda()):
        assert bool(torch.isfinite(t).all())


def test_not_finite_values_show():
    """A NaN in a row with a target reaches its loss and dw; an infinity in w every loss whose logit it raises (where x is
    negative the logit is -inf, and the class has probability 0)."""
    import paper_1702_07825_amd as wn
    x, w, b, y, grad = _inputs(20, 40, 300, torch.float32, seed=10, ignored=0)
    x[4, 5] = float("nan")
    loss, lse = wn.head_loss(x.cuda(), w.cuda(), y.cuda(), b=b.cuda())
    assert bool(torch.isnan(loss[4])) and int(torch.isnan(loss).sum()) == 1
    assert bool(torch.isnan(wn.head_loss_backward(x.cuda(), w.cuda(), y.cuda(), lse, grad.cuda(), b=b.cuda())[1]).any())
    w[9, 0] = float("inf")
    assert not bool(torch.isfinite(wn.head_loss(x.cuda(), w.cuda(), y.cuda(), b=b.cuda())[0].cpu()[x[:, 0] > 0]).any())


@pytest.mark.parametrize("std", [2.0 ** -100, 2.0 ** -30, 2.0 ** 30, 2.0 ** 100])
def test_fp32_values_far_from_one(std):
    """x of any size (w the other way): the fp16 parts are scaled row by row."""
    _check(*_inputs(70, 48, 200, torch.float32, seed=11, std=std))


def test_fp32_rows_of_unlike_sizes():
    """Rows of x and w, and upstream gradients, that differ by powers of ten."""
    x, w, b, y, grad = _inputs(64, 48, 200, torch.float32, seed=12)
    x *= 10.0 ** torch.linspace(-8, 0, 64)[:, None]
    w *= 10.0 ** torch.linspace(-8, 0, 200)[:, None]
    grad *= 10.0 ** torch.linspace(-6, 6, 64)
    _check(x, w, b, y, grad)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
def test_large_logits(dtype):
    """Logits of some hundreds: the largest is taken off before the exponentials."""
    x, w, b, y, grad = _inputs(80, 64, 500, dtype, seed=13)
    _check((x.float() * 100).to(dtype), w, b, y, grad)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("N,D,V", [(37, 64, 300), (20, 33, 150)])
def test_arrays_that_start_anywhere(dtype, N, D, V):
    """Inputs and outputs one element into their allocations; what lies around the outputs stays."""
    import paper_1702_07825_amd as wn
    x, w, b, y, grad = _inputs(N, D, V, dtype, seed=14)
    loss, lse, want = _check(x, w, b, y, grad)

    def at1(t):
        s = torch.full((t.numel() + 2,), 7, dtype=t.dtype, device="cuda")
        v = s[1:-1].view(t.shape)
        v.copy_(t)
        return s, v

    (_, X), (_, W), (_, B), (_, Y), (_, G) = (at1(t) for t in (x, w, b, y, grad))
    outs = [at1(torch.zeros_like(t)) for t in (loss, lse, *want)]
    wn.head_loss(X, W, Y, b=B, loss=outs[0][1], lse=outs[1][1])
    wn.head_loss_backward(X, W, Y, outs[1][1], G, b=B, dx=outs[2][1], dw=outs[3][1], db=outs[4][1])
    for (s, v), t in zip(outs, (loss, lse, *want)):
        assert torch.equal(v, t)
        assert float(s[0]) == 7 and float(s[-1]) == 7


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("N", [20, 100])
def test_runs_on_another_stream_and_in_a_graph(N, dtype):
    """Captured, replayed on new inputs with other work between, and on a stream of its own: the eager results."""
    import paper_1702_07825_amd as wn
    sets = [[None if t is None else t.cuda() for t in _inputs(N, 72, 400, dtype, seed=20 + k)] for k in range(3)]

    def both(x, w, b, y, g):
        loss, lse = wn.head_loss(x, w, y, b=b)
        return [loss, lse, *wn.head_loss_backward(x, w, y, lse, g, b=b)]

    want = [[t.clone() for t in both(*s)] for s in sets]
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    x, w, b, y, g = sets[1]
    loss, lse = wn.head_loss(x, w, y, b=b, stream=stream)
    got = [loss, lse, *wn.head_loss_backward(x, w, y, lse, g, b=b, stream=stream)]
    torch.cuda.current_stream().wait_stream(stream)
    assert all(torch.equal(a, c) for a, c in zip(got, want[1]))
    held = [t.clone() for t in sets[0]]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = both(*held)
    for k in (0, 1, 2, 1):
        for h, t in zip(held, sets[k]):
            h.copy_(t)
        graph.replay()
        torch.cuda.synchronize()
        both(*sets[(k + 1) % 3])  # eager work between the replays
        assert all(torch.equal(a, c) for a, c in zip(outs, want[k])), k


@pytest.mark.parametrize("N", [40, 200])
def test_targets_at_the_ends_of_int32(N):
    """Any value outside the classes is padding, the types' ends among them."""
    import paper_1702_07825_amd as wn
    x, w, b, y, grad = _inputs(N, 24, 90, torch.float32, seed=19, ignored=0)
    y[0], y[1], y[2], y[3] = -2 ** 31, 2 ** 31 - 1, 90, -1
    _check(x, w, b, y, grad)


def test_two_calls_at_once():
    """On two streams, each with a workspace of its own: the results of one after the other."""
    import paper_1702_07825_amd as wn
    sets = [[t.cuda() for t in _inputs(700, 96, 3000, torch.bfloat16, seed=30 + k)] for k in range(2)]

    def both(s, stream=None):
        x, w, b, y, g = s
        loss, lse = wn.head_loss(x, w, y, b=b, stream=stream)
        return [loss, lse, *wn.head_loss_backward(x, w, y, lse, g, b=b, stream=stream)]

    want = [both(s) for s in sets]
    streams = [torch.cuda.Stream() for _ in sets]
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    got = [[both(s, st) for s, st in zip(sets, streams)] for _ in range(5)]
    torch.cuda.synchronize()
    for r in got:
        for a, c in zip(r, want):
            assert all(torch.equal(p, q) for p, q in zip(a, c))


def test_gradient_against_differences():
    """sum g loss along a direction in x, w and b, from the losses themselves.  The function's third derivative
    along it is at most 8 max|dl|^3 sum|g| with |dl| the logits' change per unit, so the central difference is off by
    h^2 / 6 of that, and by the losses' rounding over h."""
    import paper_1702_07825_amd as wn
    x, w, b, y, grad = _inputs(40, 32, 120, torch.float32, seed=15)
    g = torch.Generator().manual_seed(16)
    dirs = [torch.randn(t.shape, generator=g) / t.numel() ** 0.5 for t in (x, w, b)]
    X, W, B, Y, G = (t.cuda() for t in (x, w, b, y, grad))
    loss, lse = wn.head_loss(X, W, Y, b=B)
    dx, dw, db = wn.head_loss_backward(X, W, Y, lse, G, b=B)
    for k, (t, d, got) in enumerate(zip((X, W, B), dirs, (dx, dw, db))):
        d, h = d.cuda(), 2.0 ** -6
        f = []
        for s in (h, -h):
            a = [X, W, B]
            a[k] = t + s * d
            f.append(float((G.double() * wn.head_loss(a[0], a[1], Y, b=a[2])[0].double()).sum()))
        dl = float((d @ W.t() if k == 0 else X @ d.t() if k == 1 else d).abs().max())
        weight = float(G.abs().sum())
        tol = h * h / 6 * 8 * dl ** 3 * weight + 2e-5 * weight / h + 1e-6
        assert abs((f[0] - f[1]) / (2 * h) - float((got.double() * d.double()).sum())) <= tol


def test_the_same_call_twice_gives_the_same_bits():
    import paper_1702_07825_amd as wn
    x, w, b, y, grad = (t.cuda() for t in _inputs(3000, 96, 5000, torch.bfloat16, seed=17))
    got = []
    for _ in range(3):
        loss, lse = wn.head_loss(x, w, y, b=b)
        got.append([loss, lse, *wn.head_loss_backward(x, w, y, lse, grad, b=b)])
    for g in got[1:]:
        assert all(torch.equal(a, c) for a, c in zip(g, got[0]))


@pytest.mark.parametrize("N", [3, 70])
def test_offsets_beyond_32_bits(N):
    """w of 4.6 GB: classes on both sides of 2^32 bytes, against pieces of it.  Each piece's results are the same sums."""
    import paper_1702_07825_amd as wn
    D, V = 2048, (1 << 20) + 70000
    g = torch.Generator(device="cuda").manual_seed(21)
    w = torch.empty((V, D), dtype=torch.bfloat16, device="cuda")
    for a in range(0, V, 1 << 18):
        w[a:a + (1 << 18)] = (torch.randn((min(V - a, 1 << 18), D), generator=g, device="cuda") * 0.03).bfloat16()
    x = torch.randn((N, D), generator=g, device="cuda").bfloat16()
    y = torch.randint(0, V, (N,), generator=g, device="cuda", dtype=torch.int32)
    y[0], y[1] = V - 1, 5
    loss, lse = wn.head_loss(x, w, y)
    parts, at = [], torch.zeros(N, dtype=torch.float64, device="cuda")
    for a in range(0, V, 1 << 18):
        l = x.float() @ w[a:a + (1 << 18)].float().t()
        parts.append(torch.logsumexp(l.double(), dim=1))
        here = (y >= a) & (y < a + l.shape[1])
        at += torch.where(here, l.gather(1, (y.long() - a).clamp(0, l.shape[1] - 1)[:, None])[:, 0].double(), 0.0)
    want = torch.logsumexp(torch.stack(parts), dim=0)
    # (logits of size 1 to 8: their sums of 2048 products and the exponentials' to 1e-4)
    assert bool(((lse.double() - want).abs() <= 1e-4).all()) and bool(((loss.double() - want + at).abs() <= 2e-4).all())
    grad = torch.full((N,), 1.0 / N, device="cuda")
    dx, dw, db = wn.head_loss_backward(x, w, y, lse, grad)
    rows = torch.tensor([0, 5, (1 << 20) - 1, 1 << 20, (1 << 20) + 1, V - 1], device="cuda")
    l = x.double() @ w[rows].double().t().contiguous()
    q = ((l - want[:, None]).exp() - (rows[None] == y[:, None]).double()) / N
    ref = q.t().contiguous() @ x.double()
    tol = (2.0 ** -7 + 1e-3) * (q.abs().t().contiguous() @ x.double().abs())
    assert bool(((dw[rows].double() - ref).abs() <= tol).all())
    assert bool(((db[rows].double() - q.sum(dim=0)).abs() <= 1e-3 * q.abs().sum(dim=0)).all())
    assert bool(torch.isfinite(dx).all()) and float(db.double().sum().abs()) <= 1e-3


def test_no_rows():
    import paper_1702_07825_amd as wn
    x, y = torch.empty((0, 16), device="cuda"), torch.empty((0,), dtype=torch.int32, device="cuda")
    w, g = torch.ones((30, 16), device="cuda"), torch.empty((0,), device="cuda")
    loss, lse = wn.head_loss(x, w, y)
    assert loss.shape == (0,) and lse.shape == (0,)
    dx, dw, db = wn.head_loss_backward(x, w, y, lse, g)
    assert dx.shape == (0, 16) and not bool(dw.any()) and not bool(db.any())


def test_refusals():
    import paper_1702_07825_amd as wn
    x, w, b, y, grad = (t.cuda() for t in _inputs(8, 16, 30, torch.float32, seed=18))
    lse = torch.zeros(8, device="cuda")
    for kw in (dict(x=x.t()), dict(x=x.half()), dict(w=w.bfloat16()), dict(w=w[:, :8]), dict(y=y.long()), dict(y=y[:4]),
               dict(b=b[:4]), dict(b=b.bfloat16()), dict(x=x.cpu()), dict(y=y.cpu()), dict(w=w[0])):
        a = {**dict(x=x, w=w, y=y, b=b), **kw}
        with pytest.raises((ValueError, TypeError)):
            wn.head_loss(a["x"], a["w"], a["y"], b=a["b"])
    for kw in (dict(need=()), dict(need=("dz",)), dict(dx=torch.zeros(3, device="cuda")), dict(grad=grad[:3]), dict(lse=lse[:3])):
        a = {**dict(lse=lse, grad=grad, need=("dx",), dx=None), **kw}
        with pytest.raises((ValueError, TypeError)):
            wn.head_loss_backward(x, w, y, a["lse"], a["grad"], b=b, need=a["need"], dx=a["dx"])
    with pytest.raises(wn.WnError):
        wn.head_loss(x, w, y, workspace=torch.empty(256, dtype=torch.uint8, device="cuda"))
    for ws in (torch.empty(1 << 26, dtype=torch.uint8), torch.empty((1 << 26, 2), dtype=torch.uint8, device="cuda")[:, 0]):
        with pytest.raises(ValueError):
            wn.head_loss(x, w, y, workspace=ws)


def _whole(N, D, V, dtype, seed):
    """Inputs whose products are whole numbers of at most D, so a logit is rounded once, where the bias is added."""
    g = torch.Generator().manual_seed(seed)
    x, w = (torch.randint(-1, 2, s, generator=g).to(dtype).cuda() for s in ((N, D), (V, D)))
    y = torch.randint(0, V, (N,), generator=g, dtype=torch.int32).cuda()
    grad = ((torch.rand((N,), generator=g) - 0.2) / N).cuda()
    return x, w, y, grad


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("offset", [100.0, -1e4, 1e6, -1e6, -1e9, 1e9, -1e30, 1e30, torch.finfo(torch.float32).min])
@pytest.mark.parametrize("N", [1, 30, 65, 300])
def test_all_logits_far_from_zero(N, offset, dtype):
    """A bias of one value on every class: logits are rounded beside it (from 1e9 on all to the bias itself), and the
    loss is that of the rounded ones, whose differences are exact.  Each exponential is off by a relative
    2^-22 (1 + |l - m|), their sum also by (V / 2048 + 128) u.  The gradients take the lse that the loss returned."""
    import paper_1702_07825_amd as wn
    D, V = 24, 700
    x, w, y, grad = _whole(N, D, V, dtype, seed=31)
    b = torch.full((V,), offset, device="cuda")
    print("far", N, offset, dtype, flush=True)
    l = ((x.double() @ w.double().t().contiguous()) + b.double()).float().double()
    at = y.long()[:, None]
    m = l.max(dim=1, keepdim=True).values
    spread = float((l - m).abs().max())
    want = (l - m).exp().sum(dim=1).log() + (m - l.gather(1, at))[:, 0]
    loss, lse = wn.head_loss(x, w, y, b=b)
    tol = (V / 2048 + 128) * U + 2.0 ** -22 * (1 + spread) + U * want
    assert bool(((loss.double() - want).abs() <= tol).all())
    assert bool(((lse.double() - torch.logsumexp(l - m, dim=1) - m[:, 0]).abs() <= tol + U * lse.double().abs()).all())
    p = (l - lse.double()[:, None]).exp()
    e = 2.0 ** -22 * (1 + (l - lse.double()[:, None]).abs()) * p
    hot = torch.zeros_like(p).scatter_(1, at, 1.0)
    G = grad.double()[:, None]
    got = wn.head_loss_backward(x, w, y, lse, grad, b=b)
    q, e = (p - hot) * G, (e + U * hot) * G.abs()
    for t, a, ea, c in ((got[0], q, e, w), (got[1], q.t().contiguous(), e.t().contiguous(), x)):
        c, K = c.double(), a.shape[1]
        v, A = a @ c, a.abs() @ c.abs()
        if dtype == torch.float32:
            err = (3 * 2.0 ** -22 + 3 * K * U) * A + 2.0 ** -38 * K * float(G.abs().max()) + 4 * U * v.abs()
        else:
            err = (2.0 ** -8 + K * U) * A + 2.0 ** -8 * v.abs()
        assert bool(((t.double() - v).abs() <= err + ea @ c.abs() + K * 2.0 ** -126).all())
    assert bool(((got[2].double() - q.sum(dim=0)).abs() <= e.sum(dim=0) + N * U * q.abs().sum(dim=0) + N * 2.0 ** -126).all())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("N", [1, 40, 65, 300])
@pytest.mark.parametrize("size", [1.0, 20.0, 300.0, 1e4])
def test_losses_are_not_negative(N, size, dtype):
    """Rows whose target has the largest logit, by enough that the others hardly count: the sum of exponentials holds a 1,
    so its log is never below 0, and nor is the loss; above it by the others' 2^-24 and less at most."""
    import paper_1702_07825_amd as wn
    x, w, b, y, grad = (t.cuda() for t in _inputs(N, 64, 500, dtype, seed=32, ignored=0))
    x = (x.float() * size).to(dtype)
    l = x.double() @ w.double().t().contiguous() + b.double()
    top = l.topk(2, dim=1)
    y = top.indices[:, 0].to(torch.int32).contiguous()
    loss = wn.head_loss(x, w, y, b=b)[0]
    assert bool((loss >= 0).all())
    sure = top.values[:, 0] - top.values[:, 1] > 30 + 1e-2 * size  # (beyond the logits' own rounding)
    assert not bool((loss[sure] > 500 * 2.0 ** -40).any())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("N", [1, 40, 100])
@pytest.mark.parametrize("rest", ["nan", "zero", "some"])
def test_upstream_gradients_that_are_nan_show(N, rest, dtype):
    """NaN in every row's g, in one row's beside zeros, or beside others: dw and db hold it throughout (each entry adds
    up a q of that row that is not 0), and dx in those rows alone."""
    import paper_1702_07825_amd as wn
    x, w, b, y, grad = (t.cuda() for t in _inputs(N, 40, 90, dtype, seed=33, ignored=0))
    bad = torch.ones(N, dtype=torch.bool, device="cuda")
    if rest != "nan":
        bad[1:] = False
        grad = grad * (rest == "some")
    grad[bad] = float("nan")
    loss, lse = wn.head_loss(x, w, y, b=b)
    dx, dw, db = wn.head_loss_backward(x, w, y, lse, grad, b=b)
    assert bool(torch.isnan(dw).all()) and bool(torch.isnan(db).all())
    assert bool(torch.isnan(dx[bad]).all()) and bool(torch.isfinite(dx[~bad]).all())


def test_gradient_of_more_values_than_a_launch_takes_threads():
    """dx of 2^32 values, summed over two pieces of the vocabulary."""
    import paper_1702_07825_amd as wn
    N, D, V = 1 << 20, 4096, 300
    g = torch.Generator(device="cuda").manual_seed(34)
    x = torch.empty((N, D), dtype=torch.bfloat16, device="cuda")
    for a in range(0, N, 1 << 17):
        x[a:a + (1 << 17)] = torch.randn((1 << 17, D), generator=g, device="cuda").bfloat16()
    w = (torch.randn((V, D), generator=g, device="cuda") / D ** 0.5).bfloat16()
    y = torch.randint(0, V, (N,), generator=g, device="cuda", dtype=torch.int32)
    y[1::7] = -1
    grad = torch.rand((N,), generator=g, device="cuda")
    loss, lse = wn.head_loss(x, w, y)
    dx = wn.head_loss_backward(x, w, y, lse, grad, need=("dx",))[0]
    rows = torch.cat([torch.arange(300), torch.randint(0, N, (500,), generator=torch.Generator().manual_seed(35)),
                      torch.arange(N - 300, N)]).cuda()
    want = _formulas(x[rows], w, None, y[rows], grad[rows])
    _near(loss[rows], want["loss"], "loss")
    _near(dx[rows], want["dx"], "dx")
    assert not bool(dx[1::7].any())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
def test_logits_of_more_tiles_than_a_launch_takes(dtype):
    """2^20 rows of 8 values under 2^19 classes and some: beyond 2^32 threads for all tiles."""
    import paper_1702_07825_amd as wn
    N, D, V = 1 << 20, 8, (1 << 19) + 77
    x, w, b, y, grad = (t.cuda() for t in _inputs(N, D, V, dtype, seed=36))
    print("tiles", N, V, dtype, flush=True)
    loss, lse = wn.head_loss(x, w, y, b=b)
    rows = torch.cat([torch.arange(40), torch.randint(0, N, (80,), generator=torch.Generator().manual_seed(37)),
                      torch.arange(N - 40, N)]).cuda()
    want = _formulas(x[rows], w, b, y[rows], grad[rows])
    _near(loss[rows], want["loss"], "loss")
    _near(lse[rows], want["lse"], "lse")


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("N,D,V", [(40, 30, 300), (70, 30, 300), (300, 40, 700), (1100, 33, 257), (2000, 64, 9000), (20000, 40, 130)])
def test_gradients_of_classes_that_no_row_targets(N, D, V, dtype):
    """Each row of dw relative to itself, for classes of probabilities down to 1e-26: evenly so, and likely in some
    runs of rows but not in others.  In fp32 q is held to 2^-22 of itself, 2^-39 of the class's largest or 2^-105."""
    import paper_1702_07825_amd as wn
    x, w, b, y, grad = _inputs(N, D, V, dtype, seed=38)
    rare = torch.arange(V) % 3 == 1
    b[rare] -= torch.linspace(5, 30, int(rare.sum()))
    # one feature turns a class's logit by 50 from run to run of 100 rows
    x[:, 0] = torch.where(torch.arange(N) // 100 % 2 == 0, 1.0, -1.0).to(dtype)
    w[:, 0] = 0
    w[5::7, 0], w[6::7, 0] = 25, -25
    y = torch.where((y >= 0) & (y < V), y // 3 * 3, y).to(torch.int32)  # (0, 3, ..: none of the rare ones)
    x, w, b, y, grad = (t.cuda() for t in (x, w, b, y, grad))
    print("classes", N, D, V, dtype, flush=True)
    loss, lse = wn.head_loss(x, w, y, b=b)
    dw = wn.head_loss_backward(x, w, y, lse, grad, b=b, need=("dw",))[1].double()
    ok = (y >= 0) & (y < V)
    X, W = x.double(), w.double()
    l = X @ W.t().contiguous() + b.double()
    S = X.abs() @ W.abs().t().contiguous()
    f32 = dtype == torch.float32
    E = (3 * 2.0 ** -22 + 3 * D * U if f32 else D * U) * S + U * (l.abs() + b.double().abs())
    if f32:
        E += D * 2.0 ** -38 * X.abs().amax(dim=1)[:, None] * W.abs().amax(dim=1)
    far = (l - lse.double()[:, None])
    p = torch.where(ok[:, None], far.exp(), 0.0)
    e = (2 * E + 2.0 ** -22 * (1 + far.abs())) * p
    hot = torch.zeros_like(p).scatter_(1, torch.where(ok, y, 0).long()[:, None], ok.double()[:, None])
    q = (p - hot).t().contiguous()
    gx = torch.where(ok, grad.double(), 0.0)[:, None] * X
    v, A = q @ gx, q.abs() @ gx.abs()
    err = (e + U * hot).t().contiguous() @ gx.abs() + N * 2.0 ** -126
    if f32:
        low = 2.0 ** -38 * q.abs().amax(dim=1) + 2.0 ** -104
        err += (3 * 2.0 ** -22 + 3 * N * U) * A + N * low[:, None] * gx.abs().amax(dim=0) + 4 * U * v.abs()
    else:
        err += (2.0 ** -8 + N * U) * A + 2.0 ** -8 * v.abs()
    _near(dw, (v, err), "dw")
    assert bool((dw != 0).any(dim=1)[q.abs().amax(dim=1) > 2.0 ** -100].all())


# Calls of up to 64 rows have kernels of their own: the same questions on the other side.
@pytest.mark.parametrize("N,D,V,dtype", [(70, 2048, 20000, torch.float32), (300, 1023, 40000, torch.float32),
                                         (70, 2047, 40000, torch.bfloat16), (300, 1999, 33000, torch.bfloat16)])
def test_several_pieces_of_the_vocabulary_forwards(N, D, V, dtype):
    """Packed classes of more than 64 MB: three pieces, which share their place, with targets and biases in each."""
    _check(*_inputs(N, D, V, dtype, seed=40), device="cuda")


@pytest.mark.parametrize("N", [65, 130, 600])
def test_fp32_rows_of_unlike_sizes_from_65_rows_on(N):
    x, w, b, y, grad = _inputs(N, 48, 200, torch.float32, seed=41)
    x *= 10.0 ** torch.linspace(-8, 0, N)[:, None]
    w *= 10.0 ** torch.linspace(-8, 0, 200)[:, None]
    grad *= 10.0 ** torch.linspace(-6, 6, N)
    _check(x, w, b, y, grad)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("N,D,V", [(100, 64, 300), (100, 33, 150), (300, 72, 1001), (1000, 7, 65)])
def test_arrays_that_start_anywhere_from_65_rows_on(dtype, N, D, V):
    """One element into their allocations, rows of whole 16-byte pieces among them; what lies around the outputs stays."""
    import paper_1702_07825_amd as wn
    x, w, b, y, grad = _inputs(N, D, V, dtype, seed=42)
    loss, lse, want = _check(x, w, b, y, grad)

    def at1(t):
        s = torch.full((t.numel() + 2,), 7, dtype=t.dtype, device="cuda")
        v = s[1:-1].view(t.shape)
        v.copy_(t)
        return s, v

    (_, X), (_, W), (_, B), (_, Y), (_, G) = (at1(t) for t in (x, w, b, y, grad))
    outs = [at1(torch.zeros_like(t)) for t in (loss, lse, *want)]
    wn.head_loss(X, W, Y, b=B, loss=outs[0][1], lse=outs[1][1])
    wn.head_loss_backward(X, W, Y, outs[1][1], G, b=B, dx=outs[2][1], dw=outs[3][1], db=outs[4][1])
    for (s, v), t in zip(outs, (loss, lse, *want)):
        assert torch.equal(v, t)
        assert float(s[0]) == 7 and float(s[-1]) == 7


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("N", [20, 100])
def test_masked_targets_and_values_that_are_not_finite(N, dtype):
    """A masked target's loss is infinite, its gradients finite; a NaN in x shows in its row's loss alone and in dw; an
    infinity in w in every loss whose logit it raises."""
    import paper_1702_07825_amd as wn
    x, w, b, y, grad = (t.cuda() for t in _inputs(N, 40, 300, dtype, seed=43, ignored=0))
    masked = b.clone()
    masked[7] = -float("inf")
    y = torch.where(y == 7, 8, y).to(torch.int32)
    y[3] = 7
    loss, lse = wn.head_loss(x, w, y, b=masked)
    assert float(loss[3]) == float("inf") and int(torch.isfinite(loss).sum()) == N - 1
    for t in wn.head_loss_backward(x, w, y, lse, grad, b=masked):
        assert bool(torch.isfinite(t).all())
    x[4, 5] = float("nan")
    loss, lse = wn.head_loss(x, w, y, b=b)
    assert bool(torch.isnan(loss[4])) and int(torch.isnan(loss).sum()) == 1
    assert bool(torch.isnan(wn.head_loss_backward(x, w, y, lse, grad, b=b)[1]).any())
    w[9, 0] = float("inf")
    assert not bool(torch.isfinite(wn.head_loss(x, w, y, b=b)[0][x[:, 0] > 0]).any())


def test_gradient_against_differences_from_65_rows_on():
    """As for few rows: the central difference is off by h^2 / 6 of the third derivative, at most 8 max|dl|^3 sum|g|, and by
    the losses' tolerance over h; the gradient along the direction by its entries' tolerances."""
    import paper_1702_07825_amd as wn
    args = _inputs(150, 32, 120, torch.float32, seed=44)
    g = torch.Generator().manual_seed(45)
    dirs = [torch.randn(t.shape, generator=g) / t.numel() ** 0.5 for t in args[:3]]
    X, W, B, Y, G = (t.cuda() for t in args)
    tols = _formulas(X, W, B, Y, G)
    loss, lse = wn.head_loss(X, W, Y, b=B)
    grads = wn.head_loss_backward(X, W, Y, lse, G, b=B)
    for k, (t, d, got, name) in enumerate(zip((X, W, B), dirs, grads, ("dx", "dw", "db"))):
        d, h = d.cuda(), 2.0 ** -6
        f = []
        for s in (h, -h):
            a = [X, W, B]
            a[k] = t + s * d
            f.append(float((G.double() * wn.head_loss(a[0], a[1], Y, b=a[2])[0].double()).sum()))
        dl = float((d @ W.t().contiguous() if k == 0 else X @ d.t().contiguous() if k == 1 else d).abs().max())
        weight = float(G.abs().sum())
        # (the moved arrays are rounded to fp32 once more: 2^-24 of the logits' terms, within the losses' own tolerance)
        tol = h * h / 6 * 8 * dl ** 3 * weight + 2 * float(tols["loss"][1].max()) * weight / h
        tol += float((tols[name][1] * d.double().abs()).sum())
        assert abs((f[0] - f[1]) / (2 * h) - float((got.double() * d.double()).sum())) <= tol, name


def _late(call, make):
    """call(stream, *tensors) on a stream that is busy; its inputs are dropped and their memory asked for again meanwhile."""
    tensors = make()
    sizes = [(t.shape, t.dtype) for t in tensors]
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        torch.cuda._sleep(100_000_000)
    got = call(stream, *tensors)
    del tensors
    others = [torch.ones(s, dtype=d, device="cuda") for s, d in sizes for _ in range(2)]
    torch.cuda.synchronize()
    del others
    return got


def test_inputs_dropped_before_another_stream_has_run():
    """Memory of inputs (and of workspaces given) that a call on another stream still has to read is not handed out."""
    import paper_1702_07825_amd as wn
    g = torch.Generator(device="cuda").manual_seed(46)

    def make():
        g.manual_seed(46)
        x, w = (torch.randn(s, generator=g, device="cuda") for s in ((300, 64), (500, 64)))
        y = torch.randint(0, 500, (300,), generator=g, device="cuda", dtype=torch.int32)
        return x, w, y, torch.rand((300,), generator=g, device="cuda")

    def loss(stream, x, w, y, grad):
        l, lse = wn.head_loss(x, w, y, stream=stream)
        return [l, lse, *wn.head_loss_backward(x, w, y, lse, grad, stream=stream)]

    def tables(stream, x, w, y, grad):
        return [wn.embed(w, y, stream=stream), wn.embed_backward(x, y, 500, stream=stream)]

    def clip(stream, x, w, y, grad):
        outs = [torch.empty_like(x), torch.empty_like(w)]
        return [wn.clip_gradients([x, w], 1.0, outs=outs, stream=stream), *outs]

    for call in (loss, tables, clip):
        want = call(None, *make())
        torch.cuda.synchronize()
        got = _late(call, make)
        assert all(torch.equal(a, b) for a, b in zip(got, want)), call.__name__


@pytest.mark.parametrize("N,D,V,dtype", [(64, 200, 16384, torch.float32), (64, 200, 16385, torch.float32), (17, 199, 900, torch.float32),
                                         (9, 201, 1003, torch.float32), (33, 400, 8192, torch.bfloat16), (33, 400, 8193, torch.bfloat16),
                                         (32, 401, 9000, torch.bfloat16), (20, 399, 500, torch.bfloat16), (1, 403, 257, torch.bfloat16)])
def test_few_rows_where_waves_begin_to_share_classes(N, D, V, dtype):
    _check(*_inputs(N, D, V, dtype, seed=47), device="cuda")
