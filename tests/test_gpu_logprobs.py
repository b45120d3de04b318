"""Log probabilities with entropies and alternatives, and their gradients (wn_logprobs, wn_logprobs_backward) against the
formulas in 64 bits.

Tolerances.  u = 2^-24 is fp32's half step.  A logit is off by at most E, as derived in the loss's tests:
  bf16: D u S + u (|l| + |b|);  fp32: (3 2^-22 + 3 D u) S + 2^-38 D max|x| max|w| + u (|l| + |b|),  S = sum |x w|
With d = l - largest, s = sum exp d and t = sum exp(d) d all terms of a sum have one sign.  exp d is off by a relative
2^-22 (1 + |d|), sums of V of them by c = (V / 2048 + 128) u (the chains' lengths), those of t by 4 c, so
  lse:     max E + c + 2^-22 (1 + |lse|)
  logprob: 2 max E + c + 2^-22 (1 + |lse| + |l_y|)
  entropy = log s - t / s:  (2 H + 1) max E (its derivative by a logit is -p (log p + H)) + 5 c (1 + T)
           + 2^-22 sum p (1 + |d|)^2 + 2^-21 (|log s| + T),  T = -t / s
  alternatives: the logits are exact but for fp64's rounding, so their order is that of 64 bits; a log probability is the
           logit less the largest one less log s, whose terms are off by the two logits' E: 2 max E + c + 2^-22 (1 + |lse|),
           and 2^-23 of itself
Gradients: c = max(|g|, |h|), a = g / c, e = h / c, q = a [v = y] - p (a + e (log p + H)).  p is off by a relative
r = 2 E + tol(lse) + 2^-22 (1 + |log p|), log p by E + tol(lse) + 2^-22 (|l| + |lse|), the rest by 4 roundings:
  dq = r p |a + e (log p + H)| + p |e| (tol(log p) + tol(H)) + 8 u (|a| [v = y] + p (|a| + |e| (|log p| + H)))
With A = sum c |q w| (or over rows c |q x|) over K terms, the products are off by
  bf16: (2^-8 + K u) A and 2^-8 of the result;  fp32: (3 2^-22 + 3 K u) A + 2^-37 K max c max and 4 u of the result
and by sum c dq |w|.  Products below 2^-126 may vanish: 2^-126 (1 + max|w|) for each term.
"""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
U = 2.0 ** -24
DTYPES = pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])


def _inputs(N, D, V, dtype, seed, bias=True, ignored=0.2, std=1.0):
    g = torch.Generator().manual_seed(seed)
    x = (torch.randn((N, D), generator=g) * std).to(dtype)
    w = (torch.randn((V, D), generator=g) * 1.5 / D ** 0.5 / std).to(dtype)
    b = torch.randn((V,), generator=g) if bias else None
    y = torch.randint(0, V, (N,), generator=g, dtype=torch.int32)
    off = torch.rand((N,), generator=g) < ignored
    y[off] = torch.where(torch.arange(int(off.sum())) % 2 == 0, -1, V).to(torch.int32)
    grad = torch.randn((N,), generator=g) / N
    grad_entropy = 0.3 * torch.randn((N,), generator=g) / N
    return x, w, b, y, grad, grad_entropy


def _top(l, top):
    """The classes of the largest logits, of equal ones the lowest first."""
    values, ids = torch.sort(l, dim=1, descending=True, stable=True)
    return ids[:, :top].to(torch.int32), values[:, :top]


def _rows(x, w, b, y, top):
    """Values and tolerances of wn_logprobs, and what the gradients' formulas need."""
    f32 = x.dtype == torch.float32
    N, D = x.shape
    V = w.shape[0]
    X, W = x.double(), w.double()
    ok = (y >= 0) & (y < V)
    B = torch.zeros(V, dtype=torch.float64, device=x.device) if b is None else b.double()
    l = X @ W.t().contiguous() + B
    S = X.abs() @ W.abs().t().contiguous()
    far = 2.0 ** -38 * float(X.abs().max()) * float(W.abs().max())
    fin = torch.where(torch.isfinite(l), l, 0.0)
    E = ((3 * 2.0 ** -22 + 3 * D * U) * S + D * far if f32 else D * U * S) + U * (fin.abs() + torch.where(torch.isfinite(B), B, 0.0).abs())
    lse = torch.logsumexp(l, dim=1)
    yc = torch.where(ok, y, 0).long()[:, None]
    ly = l.gather(1, yc)[:, 0]
    lp = l - lse[:, None]
    p = lp.exp()
    plp = torch.where(p > 0, p * lp, 0.0)
    H = -plp.sum(dim=1)
    d = torch.where(p > 0, l - l.max(dim=1, keepdim=True).values, 0.0)
    T = -(p * d).sum(dim=1)
    Em = torch.where(p > 0, E, 0.0).max(dim=1).values
    c = (V / 2048 + 128) * U
    t_lse = Em + c + 2.0 ** -22 * (1 + lse.abs())
    t_H = (2 * H + 1) * Em + 5 * c * (1 + T) + 2.0 ** -22 * (p * (1 + d.abs()) ** 2).sum(dim=1) + 2.0 ** -21 * ((H - T).abs() + T)
    fly = torch.where(torch.isfinite(ly), ly, 0.0)
    out = {"logprob": (torch.where(ok, ly - lse, 0.0), 2 * Em + c + 2.0 ** -22 * (1 + lse.abs() + fly.abs())),
           "entropy": (H, t_H), "lse": (lse, t_lse)}
    if top:
        ids, values = _top(l, top)
        v = values - lse[:, None]
        out["top_ids"] = ids
        out["top_logprobs"] = (v, (t_lse + Em)[:, None] + 2.0 ** -23 * torch.where(torch.isfinite(v), v, 0.0).abs())
    return out, dict(E=E, lse=lse, t_lse=t_lse, lp=lp, p=p, H=H, t_H=t_H, yc=yc, ok=ok, X=X, W=W, fin=fin)


def _gradients(k, f32, g, h):
    ok, p, H = k["ok"][:, None], k["p"], k["H"][:, None]
    zero = torch.zeros_like(k["lse"])
    g, h = (torch.where(k["ok"], zero if t is None else t.double(), 0.0)[:, None] for t in (g, h))
    c = torch.maximum(g.abs(), h.abs())
    lp = torch.where(p > 0, k["lp"], 0.0)
    part = g + h * (lp + H)
    q = torch.where(ok, -p * part, 0.0)
    one = torch.zeros_like(p)
    one.scatter_(1, k["yc"], ok.double())
    q += g * one
    t_lp = k["E"] + k["t_lse"][:, None] + 2.0 ** -22 * (k["fin"].abs() + k["lse"].abs()[:, None])
    r = 2 * k["E"] + k["t_lse"][:, None] + 2.0 ** -22 * (1 + lp.abs())
    dq = r * p * part.abs() + p * h.abs() * (t_lp + k["t_H"][:, None]) + 8 * U * (g.abs() * one + p * (g.abs() + h.abs() * (lp.abs() + H)))
    dq = torch.where(ok, dq, 0.0)
    out = {}
    for name, a, m, e in (("dx", q, k["W"], dq), ("dw", q.t().contiguous(), k["X"], dq.t().contiguous())):
        K = a.shape[1]
        v, A = a @ m, a.abs() @ m.abs()
        top = float(m.abs().max())
        if f32:
            t = (3 * 2.0 ** -22 + 3 * K * U) * A + 2.0 ** -37 * K * float(c.max()) * top + 4 * U * v.abs()
        else:
            t = (2.0 ** -8 + K * U) * A + 2.0 ** -8 * v.abs()
        out[name] = (v, t + e @ m.abs() + K * 2.0 ** -126 * (1 + top))
    N = q.shape[0]
    out["db"] = (q.sum(dim=0), dq.sum(dim=0) + N * U * q.abs().sum(dim=0) + N * 2.0 ** -126)
    return out


def _near(got, want, name):
    v, t = want
    got = got.double()
    assert got.shape == v.shape, name
    bad = ~((got - v).abs() <= t) & ~(got == v)
    if bool(bad.any()):
        at = tuple(int(i) for i in bad.nonzero()[0])
        raise AssertionError("%s%s: %r, not %r within %.3g (%d of %d off)" % (name, at, float(got[at]), float(v[at]),
                                                                        float(t[at]), int(bad.sum()), bad.numel()))


NAMES = ("logprob", "entropy", "lse", "top_ids", "top_logprobs")


def _probe(x, w, b, y, top):
    """The call's outputs, checked."""
    import paper_1702_07825_amd as wn
    want, k = _rows(x, w, b, y, top)
    got = wn.head_logprobs(x, w, y, b=b, top=top)
    for name, t in zip(NAMES, got):
        if t is None:
            assert not top and name.startswith("top")
        elif name == "top_ids":
            assert t.dtype == torch.int32
            assert torch.equal(t, want[name]), (name, (t != want[name]).nonzero()[:4].tolist())
        else:
            _near(t, want[name], name)
    return got, k


def _check(x, w, b, y, grad, grad_entropy, top=0, need=("dx", "dw", "db")):
    import paper_1702_07825_amd as wn
    print("logprobs", tuple(x.shape), tuple(w.shape), x.dtype, "top", top, flush=True)
    x, w, b, y, grad, grad_entropy = (None if t is None else t.cuda() for t in (x, w, b, y, grad, grad_entropy))
    rows, k = _probe(x, w, b, y, top)
    want = _gradients(k, x.dtype == torch.float32, grad, grad_entropy)
    got = wn.head_logprobs_backward(x, w, y, rows[2], rows[1], grad, grad_entropy, b=b, need=need)
    for name, t in zip(("dx", "dw", "db"), got):
        assert (t is None) == (name not in need)
        if t is not None:
            _near(t, want[name], name)
    return rows, got


SIZES = [(1, 1, 1), (1, 64, 256), (1, 1000, 777), (2, 7, 5), (16, 64, 256), (17, 65, 129), (33, 8, 2000), (64, 32, 1000),
         (64, 1025, 65), (5, 1100, 300), (4, 100, 17000), (16, 520, 16400), (30, 1030, 100), (1, 5000, 1), (48, 513, 2049),
         (65, 64, 70), (100, 100, 127), (127, 72, 128), (129, 256, 257), (200, 100, 3001), (256, 256, 256), (300, 513, 777),
         (1000, 64, 300), (2111, 40, 64)]


@DTYPES
@pytest.mark.parametrize("N,D,V", SIZES)
def test_sizes(N, D, V, dtype):
    _check(*_inputs(N, D, V, dtype, seed=N + D + V), top=min(V, (N + V) % 33))


@DTYPES
@pytest.mark.parametrize("N,D,V", [(4100, 300, 8200), (5, 2048, 40000), (20000, 256, 256), (3, 64, 200000)])
def test_large(N, D, V, dtype):
    """Tiles that fill the chip; more groups than a wave, and than a block, looks at at a time; sums over the rows in parts."""
    _check(*_inputs(N, D, V, dtype, seed=3), top=20)


@DTYPES
@pytest.mark.parametrize("top", [1, 2, 7, 8, 9, 16, 31, 32])
@pytest.mark.parametrize("N,V", [(1, 32), (7, 100), (150, 40), (90, 2000)])
def test_alternatives_of_any_number(N, V, top, dtype):
    x, w, b, y, _, _ = (t.cuda() for t in _inputs(N, 56, V, dtype, seed=top))
    got, _ = _probe(x, w, b, y, top)
    _, _ = _probe(x, w, None, y, top)
    assert got[3].shape == (N, top)


@DTYPES
@pytest.mark.parametrize("N,V", [(3, 70), (40, 3000), (100, 3000), (70, 20000)])
def test_equal_classes_come_in_order(N, V, dtype):
    """Rows of w that are copies of each other, in other groups and tiles, and rows of x that make all classes alike."""
    x, w, b, y, _, _ = (t.cuda() for t in _inputs(N, 40, V, dtype, seed=41))
    g = torch.Generator().manual_seed(5)
    w = w[torch.randint(0, V // 9, (V,), generator=g).cuda()].contiguous()
    x[1] = 0
    b[:] = 0.25
    for top in (1, 3, 12, 32):
        got, _ = _probe(x, w, b, y, top)
        assert got[3][1].tolist() == list(range(top))


@DTYPES
@pytest.mark.parametrize("N", [9, 128, 129, 2050])
def test_equal_classes_of_several_segments(N, dtype):
    """Copies all over a vocabulary whose groups several waves search, for each number of waves."""
    x, w, b, y, _, _ = (t.cuda() for t in _inputs(N, 16, 20000, dtype, seed=47))
    w = w[:300].repeat(67, 1)[:20000].contiguous()
    b[:] = -1.5
    for top in (1, 2, 8, 32):
        _probe(x, w, b, y, top)


@DTYPES
@pytest.mark.parametrize("rising", [True, False])
@pytest.mark.parametrize("N,V", [(2, 40000), (80, 40000)])
def test_classes_in_order_of_their_logits(N, V, rising, dtype):
    """The likeliest classes beside each other, at one end."""
    x, w, b, y, _, _ = (t.cuda() for t in _inputs(N, 24, V, dtype, seed=42))
    b = torch.linspace(-20, 20, V, device="cuda") * (1 if rising else -1)
    _probe(x, (w.float() * 1e-3).to(dtype), b, y, 32)


@DTYPES
def test_several_pieces_of_the_vocabulary(dtype):
    """More rows than groups of all classes are kept for: the alternatives go from piece to piece."""
    import paper_1702_07825_amd as wn
    N, D, V, top = 70000, 16, 9000, 5
    x, w, b, y, _, _ = (t.cuda() for t in _inputs(N, D, V, dtype, seed=43))
    print("pieces", dtype, flush=True)
    got = wn.head_logprobs(x, w, y, b=b, top=top)
    for n in range(0, N, 14000):
        want, _ = _rows(x[n:n + 14000], w, b, y[n:n + 14000], top)
        for name, t in zip(NAMES, got):
            t = t[n:n + 14000]
            if name == "top_ids":
                assert torch.equal(t, want[name])
            else:
                _near(t, want[name], name)
        del want


@DTYPES
@pytest.mark.parametrize("N", [64, 65, 1100, 2049])
@pytest.mark.parametrize("V", [6, 33, 255, 1023, 1024, 1025])
def test_alternatives_of_few_classes(N, V, dtype):
    """On both sides of where a row's logits are searched themselves; masked classes, copies and alike ones among them."""
    x, w, b, y, _, _ = (t.cuda() for t in _inputs(N, 30, V, dtype, seed=44))
    g = torch.Generator().manual_seed(6)
    w[V // 2:] = w[torch.randint(0, max(1, V // 4), (V - V // 2,), generator=g).cuda()]
    b[V // 2:] = b[0]
    b[::3] = -float("inf")
    x[2] = 0
    print("few classes", N, V, dtype, flush=True)
    for top in {1, min(5, V), min(20, V), min(32, V)}:
        _probe(x, w, b, y, top)


@DTYPES
@pytest.mark.parametrize("V", [300, 8000])
@pytest.mark.parametrize("N", [1536, 1537])
def test_alternatives_where_a_row_takes_one_wave(N, V, dtype):
    x, w, b, y, _, _ = (t.cuda() for t in _inputs(N, 40, V, dtype, seed=48))
    for top in (1, 32):
        _probe(x, w, b, y, top)


@DTYPES
@pytest.mark.parametrize("N,V", [(1, 3000), (64, 300), (65, 1030), (200, 3000), (1600, 3000)])
def test_classes_of_a_group_closer_than_fp32_rounds(N, V, dtype):
    """Eight classes beside each other, far above the others, whose rows differ where x is tiny: their logits of about 16, whose
    sums in 32 bits are off by some 2^-20, lie 2^-22 apart."""
    x, w, b, y, _, _ = (t.cuda() for t in _inputs(N, 2048, V, dtype, seed=49))
    at = 8 * (V // 16)
    w[at:at + 8] = w[at]
    x.copy_((x.float() + 7 * w[at].float()).to(dtype))
    b[at:at + 8] = 1.0
    x[:, 5::400] = (x[:, 5::400].float() * 2.0 ** -21).to(dtype)
    w[at:at + 8, 5::400] = torch.randn(w[at:at + 8, 5::400].shape, generator=torch.Generator().manual_seed(3)).to(dtype).cuda()
    l = x.double() @ w[at:at + 8].double().t().contiguous()
    l = l.sort(dim=1).values
    gap = l[:, 1:] - l[:, :-1]
    assert float(gap.min()) > 1e-12 and float(gap.median()) < 2.0 ** -20 and float(l.min()) > 8
    for top in (1, 5, 8, 12):
        got, _ = _probe(x, w, b, y, top)
        n = min(top, 8)
        assert bool(((got[3][:, :n] >= at) & (got[3][:, :n] < at + 8)).all())


@DTYPES
@pytest.mark.parametrize("N,V", [(20, 300), (64, 2000), (100, 2000), (300, 2000), (1600, 2000)])
def test_candidates_by_the_hundred(N, V, dtype):
    """Terms of 2^17 that cancel exactly, in 32 columns of their own: the logits are as exact as without, but no bound of
    their rounding can tell so, and most of the groups' classes are candidates."""
    x, w, b, y, _, _ = (t.cuda() for t in _inputs(N, 160, V, dtype, seed=53))
    x[:, :32] = 0
    w[:, :32] = 0
    x[:, :2] = 2.0 ** 17
    w[:, 0] = 1
    w[:, 1] = -1
    for top in (1, 5, 32):
        _probe(x, w, b, y, top)


@DTYPES
@pytest.mark.parametrize("N,V,mask", [(20, 300, m) for m in (-1e9, -1e17, -1e30, -3e38, 1e30)] +
                         [(N, 2000, m) for N in (90, 1600) for m in (-1e30, -3e38, 1e30)])
def test_fewer_classes_left_than_alternatives(N, V, mask, dtype):
    """Alternatives among classes that a finite value masks: by their numbers where 64 bits hold nothing beside it, and by their
    logits at -1e9 (at -1e17 where one reaches 8, half of the step there).  32 bits hold nothing there, so all groups' largest
    logits are alike, which lets classes be missed unless all groups are searched: 38 groups of 8 with 32 alternatives."""
    x, w, b, y, _, _ = (t.cuda() for t in _inputs(N, 100, V, dtype, seed=54))
    x[1] = 0
    b[:] = mask
    b[[7, V // 2, V - 1]] = torch.tensor([0.5, -0.5, 1.5], device="cuda") if mask < 0 else 2 * mask
    for top in (1, 3, 32) if -1e18 < mask < 0 else (1, 3, 4, 20, 32):
        _probe(x, w, b, y, top)


def test_few_classes_in_several_pieces():
    """fp32 rows so long that a piece of the packed vocabulary holds a part of the classes only."""
    x, w, b, y, _, _ = (t.cuda() for t in _inputs(66, 50000, 800, torch.float32, seed=45))
    print("few classes in pieces", flush=True)
    _probe(x, w, b, y, 32)


@pytest.mark.parametrize("N", [223696, 223697])
def test_few_classes_of_many_rows(N):
    """On both sides of where the logits of 300 classes would take more than their part of the workspace."""
    import paper_1702_07825_amd as wn
    x, w, b, y, _, _ = (t.cuda() for t in _inputs(N, 8, 300, torch.float32, seed=46))
    print("few classes of many rows", N, flush=True)
    got = wn.head_logprobs(x, w, y, b=b, top=4)
    for n in range(0, N, 60000):
        want, _ = _rows(x[n:n + 60000], w, b, y[n:n + 60000], 4)
        assert torch.equal(got[3][n:n + 60000], want["top_ids"])
        _near(got[4][n:n + 60000], want["top_logprobs"], "top_logprobs")


@DTYPES
def test_each_gradient_and_each_upstream_alone(dtype):
    args = _inputs(70, 48, 300, dtype, seed=5, bias=False)
    _, all_ = _check(*args)
    for i, k in enumerate(("dx", "dw", "db")):
        _, got = _check(*args, need=(k,))
        assert torch.equal(got[i], all_[i])
    for N in (20, 70):
        x, w, b, y, g, h = _inputs(N, 48, 300, dtype, seed=6)
        _check(x, w, b, y, g, None)
        _check(x, w, b, y, None, h)
        _check(x, w, b, y, g, torch.zeros_like(h))
        _check(x, w, b, y, g * 1e-6, h)
        g[::2] = 0
        h[::3] = 0
        _check(x, w, b, y, g, h)


@DTYPES
@pytest.mark.parametrize("N", [30, 200])
def test_without_entropies_it_is_the_loss(N, dtype):
    """logprob = -loss; the gradients of both lie within the two's tolerances of each other."""
    import paper_1702_07825_amd as wn
    x, w, b, y, g, _ = (t.cuda() for t in _inputs(N, 96, 1000, dtype, seed=44))
    loss, lse = wn.head_loss(x, w, y, b=b)
    rows, k = _probe(x, w, b, y, 0)
    assert torch.equal(rows[2], lse)
    assert torch.equal(rows[0], -loss)
    want = _gradients(k, dtype == torch.float32, g, None)
    for name, p, q in zip(("dx", "dw", "db"), wn.head_logprobs_backward(x, w, y, lse, rows[1], g, b=b),
                          wn.head_loss_backward(x, w, y, lse, -g, b=b)):
        _near(p, (q.double(), 2 * want[name][1]), name)


@DTYPES
@pytest.mark.parametrize("N", [3, 16, 40, 150])
def test_padding_holds_anything(N, dtype):
    """NaN and infinities in rows without a token, in their upstream gradients, lse and entropy: the other rows'
    results are those of the call with zeros there."""
    import paper_1702_07825_amd as wn
    x, w, b, y, g, h = (t.cuda() for t in _inputs(N, 72, 260, dtype, seed=6, ignored=0.4))
    y[1] = -1
    off = (y < 0) | (y >= 260)
    clean = x.clone()
    clean[off] = 0
    bad = x.clone()
    bad[off] = float("nan")
    bad[off.nonzero()[0]] = float("inf")
    rows, want = _check(clean, w, b, y, g, h, top=4)
    got = wn.head_logprobs(bad, w, y, b=b, top=4)
    assert not bool(got[0][off].any())
    for p, q in zip(got, rows):
        assert torch.equal(p[~off], q[~off])
    assert bool(((got[3] >= 0) & (got[3] < 260)).all())
    lse, entropy = got[2].clone(), got[1].clone()
    for t in (g, h, lse, entropy):
        t[off] = float("nan")
    got = wn.head_logprobs_backward(bad, w, y, lse, entropy, g, h, b=b)
    assert not bool(got[0][off].any())
    for p, q in zip(got, want):
        assert torch.equal(p, q)


@DTYPES
@pytest.mark.parametrize("N", [1, 40, 140])
def test_no_row_has_a_token(N, dtype):
    import paper_1702_07825_amd as wn
    x, w, b, y, g, h = (t.cuda() for t in _inputs(N, 24, 90, dtype, seed=7))
    y[:] = -5
    y[0] = 2 ** 31 - 1
    rows, _ = _probe(x, w, b, y, 3)
    assert not bool(rows[0].any())
    for t in wn.head_logprobs_backward(x, w, y, rows[2], rows[1], g, h, b=b):
        assert not bool(t.any())


@DTYPES
@pytest.mark.parametrize("mask", [-float("inf"), torch.finfo(torch.float32).min], ids=["inf", "lowest"])
@pytest.mark.parametrize("N", [1, 30, 90])
def test_masked_classes(N, dtype, mask):
    """Classes that a bias masks, whole tiles of them among them, and fewer left than alternatives."""
    x, w, b, y, g, h = _inputs(N, 40, 700, dtype, seed=8, ignored=0)
    b[100:600] = mask
    b[0] = mask
    y = torch.where((y >= 100) & (y < 600) | (y == 0), 650, y).to(torch.int32)
    _check(x, w, b, y, g, h, top=32)
    if mask == -float("inf"):
        b[:] = mask
        b[[3, 300, 650]] = 1.0
        y[:] = 300
        _check(x, w, b, y, g, h, top=9)


@DTYPES
@pytest.mark.parametrize("N", [20, 90])
def test_nothing_left_or_not_finite(N, dtype):
    """All classes masked: nothing finite, and alternatives that are classes.  A NaN shows in its row alone, and in dw; one
    class left has all of the probability."""
    import paper_1702_07825_amd as wn
    x, w, b, y, g, h = (t.cuda() for t in _inputs(N, 40, 300, dtype, seed=9, ignored=0))
    got = wn.head_logprobs(x, w, y, b=torch.full_like(b, -float("inf")), top=5)
    for t in (got[0], got[1], got[2], got[4]):
        assert not bool(torch.isfinite(t).any())
    assert bool(((got[3] >= 0) & (got[3] < 300)).all())
    x[4, 5] = float("nan")
    got = wn.head_logprobs(x, w, y, b=b, top=5)
    for t in (got[0], got[1], got[2]):
        assert bool(torch.isnan(t[4])) and int(torch.isnan(t).sum()) == 1
    assert bool(torch.isnan(got[4][4]).all()) and int(torch.isnan(got[4]).sum()) == 5
    assert bool(((got[3] >= 0) & (got[3] < 300)).all())
    assert bool(torch.isnan(wn.head_logprobs_backward(x, w, y, got[2], got[1], g, h, b=b)[1]).any())
    x[4, 5] = 0
    one = torch.full_like(b, -float("inf"))
    one[77] = 2.0
    y[:] = 77
    y[2] = 5
    got = wn.head_logprobs(x, w, y, b=one, top=1)
    assert bool((got[3] == 77).all()) and not bool(got[1].any()) and not bool(got[4].any())
    assert float(got[0][2]) == -float("inf") and int((got[0] == 0).sum()) == N - 1
    for t in wn.head_logprobs_backward(x, w, y, got[2], got[1], g, h, b=one):
        assert bool(torch.isfinite(t).all())


@DTYPES
@pytest.mark.parametrize("N", [20, 100])
def test_upstream_gradients_that_are_nan_show(N, dtype):
    import paper_1702_07825_amd as wn
    x, w, b, y, g, h = (t.cuda() for t in _inputs(N, 40, 300, dtype, seed=10, ignored=0))
    rows = wn.head_logprobs(x, w, y, b=b)
    for which in (0, 1):
        up = [g.clone(), h.clone()]
        up[which][3] = float("nan")
        dx, dw, db = wn.head_logprobs_backward(x, w, y, rows[2], rows[1], *up, b=b)
        assert bool(torch.isnan(dx[3]).all()) and int(torch.isnan(dx).sum()) == 40
        assert bool(torch.isnan(dw).all()) and bool(torch.isnan(db).all())


@DTYPES
@pytest.mark.parametrize("N", [20, 90])
@pytest.mark.parametrize("offset", [-1e4, 20.0, 1e4])
def test_all_logits_far_from_zero(N, offset, dtype):
    """A bias that all classes share changes no probability: entropies and log probabilities stay as exact as without."""
    x, w, b, y, g, h = _inputs(N, 40, 700, dtype, seed=45)
    _check(x, w, torch.round(b * 64) / 64 + offset, y, g, h, top=6)


@pytest.mark.parametrize("std", [2.0 ** -100, 2.0 ** -30, 2.0 ** 30, 2.0 ** 100])
@pytest.mark.parametrize("N", [20, 70])
def test_fp32_values_far_from_one(N, std):
    _check(*_inputs(N, 48, 200, torch.float32, seed=11, std=std), top=5)


@DTYPES
@pytest.mark.parametrize("N", [40, 80])
def test_certain_and_even_rows(N, dtype):
    """Logits of some hundreds, one class holding nearly all of the probability, and rows whose classes are alike."""
    import paper_1702_07825_amd as wn
    x, w, b, y, g, h = _inputs(N, 64, 500, dtype, seed=13)
    scale = torch.logspace(-3, 2, N)[:, None]
    x = (x.float() * scale).to(dtype)
    x[5] = 0
    rows, _ = _check(x, w, None, y, g, h, top=3)
    assert bool((rows[1] >= 0).all()) and bool((rows[0] <= 0).all()) and bool((rows[4] <= 1e-5).all())
    assert abs(float(rows[1][5]) - 6.2146080984) <= 1e-5  # log 500


@DTYPES
@pytest.mark.parametrize("N,V", [(6, 50), (70, 50)])
def test_an_entropys_gradient_at_its_largest(N, V, dtype):
    """Half of the probability on one class and the rest even: where |q| is largest, beside upstream gradients that differ by
    powers of ten."""
    x, w, b, y, g, h = _inputs(N, 24, V * 64, dtype, seed=46, ignored=0.1)
    b = torch.zeros(V * 64)
    b[17] = float(torch.log(torch.tensor(V * 64.0 - 1)))
    x = (x.float() * 1e-3).to(dtype)
    h = torch.ones(N) * 10.0 ** torch.linspace(-6, 6, N)
    y[::2] = 17
    _check(x, w, b, y, h * 0.01, h)


@DTYPES
@pytest.mark.parametrize("N,D,V", [(37, 64, 300), (100, 33, 150)])
def test_arrays_that_start_anywhere(dtype, N, D, V):
    """Inputs and outputs one element into their allocations; what lies around the outputs stays."""
    import paper_1702_07825_amd as wn
    args = [t.cuda() for t in _inputs(N, D, V, dtype, seed=14)]
    rows, grads = _check(*args, top=6)

    def at1(t):
        s = torch.full((t.numel() + 2,), 7, dtype=t.dtype, device="cuda")
        v = s[1:-1].view(t.shape)
        v.copy_(t)
        return s, v

    x, w, b, y, g, h = (at1(t)[1] for t in args)
    outs = [at1(torch.zeros_like(t)) for t in (*rows, *grads)]
    o = [v for _, v in outs]
    wn.head_logprobs(x, w, y, b=b, top=6, **dict(zip(NAMES, o)))
    wn.head_logprobs_backward(x, w, y, o[2], o[1], g, h, b=b, dx=o[5], dw=o[6], db=o[7])
    for (s, v), t in zip(outs, (*rows, *grads)):
        assert torch.equal(v, t)
        assert float(s[0]) == 7 and float(s[-1]) == 7


def _all(wn, s, stream=None):
    x, w, b, y, g, h = s
    rows = wn.head_logprobs(x, w, y, b=b, top=7, stream=stream)
    return [*rows, *wn.head_logprobs_backward(x, w, y, rows[2], rows[1], g, h, b=b, stream=stream)]


@DTYPES
@pytest.mark.parametrize("N", [20, 100])
def test_runs_on_another_stream_and_in_a_graph(N, dtype):
    """Captured, replayed on new inputs with other work between, and on a stream of its own: the eager results."""
    import paper_1702_07825_amd as wn
    sets = [[t.cuda() for t in _inputs(N, 72, 400, dtype, seed=20 + k)] for k in range(3)]
    want = [[t.clone() for t in _all(wn, s)] for s in sets]
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    got = _all(wn, sets[1], stream)
    torch.cuda.current_stream().wait_stream(stream)
    assert all(torch.equal(a, c) for a, c in zip(got, want[1]))
    held = [t.clone() for t in sets[0]]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = _all(wn, held)
    for k in (0, 1, 2, 1):
        for t, s in zip(held, sets[k]):
            t.copy_(s)
        graph.replay()
        torch.cuda.synchronize()
        _all(wn, sets[(k + 1) % 3])  # eager work between the replays
        assert all(torch.equal(a, c) for a, c in zip(outs, want[k])), k


def test_two_calls_at_once():
    """On two streams, each with a workspace of its own: the results of one after the other."""
    import paper_1702_07825_amd as wn
    sets = [[t.cuda() for t in _inputs(700, 96, 3000, torch.bfloat16, seed=30 + k)] for k in range(2)]
    want = [_all(wn, s) for s in sets]
    streams = [torch.cuda.Stream() for _ in sets]
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    got = [[_all(wn, s, st) for s, st in zip(sets, streams)] for _ in range(5)]
    torch.cuda.synchronize()
    for r in got:
        for a, c in zip(r, want):
            assert all(torch.equal(p, q) for p, q in zip(a, c))


@DTYPES
@pytest.mark.parametrize("N,D,V", [(6, 5, 11), (70, 9, 33)])
def test_gradient_against_differences(N, D, V, dtype):
    """The objective in 64 bits, moved along random directions of x, w and b by +-s: (f(s) - f(-s)) / 2 s is the
    gradient's product with the direction but for s^2 of its third derivative.  The gradients' own tolerances are
    added up along the direction."""
    import paper_1702_07825_amd as wn
    x, w, b, y, g, h = (t.cuda() for t in _inputs(N, D, V, dtype, seed=50))
    rows, k = _probe(x, w, b, y, 0)
    grads = wn.head_logprobs_backward(x, w, y, rows[2], rows[1], g, h, b=b)
    tol = _gradients(k, dtype == torch.float32, g, h)
    ok = ((y >= 0) & (y < V)).nonzero()[:, 0]

    def f(X, W, B):
        lp = torch.log_softmax(X @ W.t().contiguous() + B, dim=1)[ok]
        at = lp.gather(1, y[ok].long()[:, None])[:, 0]
        return float((g.double()[ok] * at).sum() - (h.double()[ok] * (lp.exp() * lp).sum(dim=1)).sum())

    gen = torch.Generator().manual_seed(51)
    s = 1e-4
    for i, name in enumerate(("dx", "dw", "db")):
        for _ in range(4):
            base = [x.double(), w.double(), b.double()]
            d = torch.randn(base[i].shape, generator=gen, dtype=torch.float64).cuda()
            ends = []
            for sign in (1, -1):
                p = list(base)
                p[i] = p[i] + sign * s * d
                ends.append(f(*p))
            diff = (ends[0] - ends[1]) / (2 * s)
            inner = float((grads[i].double() * d).sum())
            bound = float((tol[name][1] * d.abs()).sum()) + 1e-6
            assert abs(inner - diff) <= bound, (name, inner, diff, bound)


@DTYPES
def test_the_same_call_twice_gives_the_same_bits(dtype):
    import paper_1702_07825_amd as wn
    for N in (50, 3000):
        s = [t.cuda() for t in _inputs(N, 120, 5000, dtype, seed=52)]
        a, c = _all(wn, s), _all(wn, s)
        assert all(torch.equal(p, q) for p, q in zip(a, c))


def test_offsets_beyond_32_bits():
    """A table of more than 2^32 bytes whose last rows are the likeliest, and more logits than 2^32."""
    import paper_1702_07825_amd as wn
    V, D = 1100000, 2048
    w = torch.zeros((V, D), dtype=torch.bfloat16, device="cuda")
    w[-5:] = 0.01 * torch.arange(1, 6, device="cuda")[:, None]
    for N in (3, 4000):
        print("rows", N, flush=True)
        x = torch.ones((N, D), dtype=torch.bfloat16, device="cuda")
        y = torch.full((N,), V - 1, dtype=torch.int32, device="cuda")
        logprob, entropy, lse, ids, lps = wn.head_logprobs(x, w, y, top=6)
        assert ids[0].tolist() == [V - 1, V - 2, V - 3, V - 4, V - 5, 0] and bool((ids == ids[0]).all())
        l = torch.zeros(V, dtype=torch.float64, device="cuda")
        l[-5:] = w[-5:].double().sum(dim=1)
        lp = torch.log_softmax(l, dim=0)
        H = float(-(lp.exp() * lp).sum())
        assert bool(((logprob.double() - lp[-1]).abs() <= 1e-4).all())
        assert bool(((entropy.double() - H).abs() <= 1e-4 * (1 + H)).all())
        assert bool(((lps[:, 5].double() - lp[0]).abs() <= 1e-4 * float(-lp[0])).all())


def test_no_rows():
    import paper_1702_07825_amd as wn
    x, w, b, y, g, h = (t.cuda() for t in _inputs(4, 8, 30, torch.float32, seed=1))
    rows = wn.head_logprobs(x[:0], w, y[:0], b=b, top=2)
    assert [tuple(t.shape) for t in rows] == [(0,), (0,), (0,), (0, 2), (0, 2)]
    dx, dw, db = wn.head_logprobs_backward(x[:0], w, y[:0], rows[2], rows[1], g[:0], h[:0], b=b)
    assert dx.shape == (0, 8) and not bool(dw.any()) and not bool(db.any())


def test_refusals():
    import paper_1702_07825_amd as wn
    x, w, b, y, g, h = (t.cuda() for t in _inputs(4, 8, 30, torch.float32, seed=1))
    rows = wn.head_logprobs(x, w, y, b=b, top=2)
    i32 = torch.zeros((4, 2), dtype=torch.int32, device="cuda")
    bad = [lambda: wn.head_logprobs(x.half(), w, y), lambda: wn.head_logprobs(x, w.bfloat16(), y),
           lambda: wn.head_logprobs(x, w[:, :7], y), lambda: wn.head_logprobs(x, w, y.long()),
           lambda: wn.head_logprobs(x, w, y, top=31), lambda: wn.head_logprobs(x, w, y, top=-1),
           lambda: wn.head_logprobs(x, w, y, top_ids=i32), lambda: wn.head_logprobs(x, w, y, top=3, top_ids=i32),
           lambda: wn.head_logprobs(x, w, y, b=b[:-1]), lambda: wn.head_logprobs(x.cpu(), w, y),
           lambda: wn.head_logprobs(x, w, y, logprob=torch.zeros(4)), lambda: wn.head_logprobs(x[:, ::2], w[:, ::2], y),
           lambda: wn.head_logprobs(x, w, y, b=b, workspace=torch.zeros(64, dtype=torch.uint8, device="cuda")),
           lambda: wn.head_logprobs_backward(x, w, y, rows[2], rows[1], b=b),
           lambda: wn.head_logprobs_backward(x, w, y, rows[2], rows[1], g, h, need=()),
           lambda: wn.head_logprobs_backward(x, w, y, rows[2], rows[1], g, h, need=("dy",)),
           lambda: wn.head_logprobs_backward(x, w, y, rows[2], rows[1][:2], g, h),
           lambda: wn.head_logprobs_backward(x, w, y, rows[2], rows[1], g.double(), h)]
    for k, f in enumerate(bad):
        with pytest.raises((ValueError, TypeError, wn.WnError)):
            f()
            raise AssertionError(k)
