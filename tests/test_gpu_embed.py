"""The embedding and its gradient by sorted tokens (wn_embed, wn_embed_backward).

The lookup is one fp32 product, rounded once: it has to be equal.  The gradient of integer-valued rows is exact in
fp32 whatever the order of its sums, and has to be equal too; that of arbitrary rows is within
(n + 2) 2^-24 sum |dout| of the sum over the token's n rows, and rounded to the table's type.
"""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

DTYPES = [torch.float32, torch.bfloat16]
IDS = ["f32", "bf16"]


def _tokens(kind, N, V, seed=1):
    g = torch.Generator().manual_seed(seed)
    if kind == "one":
        t = torch.full((N,), min(V - 1, 3))
    elif kind == "distinct":
        t = torch.randperm(max(N, V), generator=g)[:N] % V
    elif kind == "sorted":
        t = torch.arange(N) * V // max(N, 1)
    elif kind == "down":
        t = V - 1 - torch.arange(N) * V // max(N, 1)
    elif kind == "text":
        t = (torch.exp(torch.rand(N, generator=g, dtype=torch.float64) * torch.log(torch.tensor(V + 1.0))) - 1).long().clamp(0, V - 1)
    elif kind == "none":
        t = torch.where(torch.arange(N) % 2 == 0, -1, V)
    else:  # padded
        t = torch.randint(0, V, (N,), generator=g)
        t[torch.rand(N, generator=g) < 0.3] = -1
        t[torch.rand(N, generator=g) < 0.1] = V + 7
    return t.to(torch.int32)


def _backward(N, D, V, kind, dtype, whole=True, scale=0.5, seed=2):
    import paper_1702_07825_amd as wn
    print("embed", N, D, V, kind, dtype, flush=True)
    t = _tokens(kind, N, V)
    g = torch.Generator().manual_seed(seed)
    # bf16 holds integers up to 256, and the sums are rounded to it once
    d = (torch.randint(-4, 5, (N, D), generator=g).float() if whole else torch.randn((N, D), generator=g)).to(dtype)
    got = wn.embed_backward(d.cuda(), t.cuda(), V, scale=scale)
    ok = (t >= 0) & (t < V)
    ids, rows = t[ok].long(), d[ok].double()
    want = torch.zeros((V, D), dtype=torch.float64).index_add_(0, ids, rows) * scale
    if whole:
        assert torch.equal(got.cpu(), want.float().to(dtype))
        return
    n = torch.bincount(ids, minlength=V)[:, None].double()
    tol = (n + 2) * 2.0 ** -24 * torch.zeros((V, D), dtype=torch.float64).index_add_(0, ids, rows.abs()) * scale
    tol += (2.0 ** -8 if dtype == torch.bfloat16 else 2.0 ** -24) * want.abs()
    assert bool(((got.cpu().double() - want).abs() <= tol).all())


@pytest.mark.parametrize("dtype", DTYPES, ids=IDS)
@pytest.mark.parametrize("N,D,V", [(1, 1, 1), (1, 2048, 300), (7, 3, 2), (64, 64, 256), (65, 100, 511), (300, 777, 512), (1000, 8, 70000)])
def test_lookup(N, D, V, dtype):
    import paper_1702_07825_amd as wn
    table = torch.randn((V, D), generator=torch.Generator().manual_seed(V)).to(dtype).cuda()
    t = _tokens("padded", N, V).cuda()
    want = torch.where(((t >= 0) & (t < V))[:, None], table[t.clamp(0, V - 1).long()].float() * 1.7, 0.0).to(dtype)
    assert torch.equal(wn.embed(table, t, scale=1.7), want)


def test_lookup_of_a_batch_and_the_lookup_in_the_framework_s_own_layout():
    """Tokens [B, T] as generation returns them give [B, T, r]."""
    import paper_1702_07825_amd as wn
    table = torch.randn((256, 64), device="cuda")
    y = torch.randint(0, 256, (3, 50), dtype=torch.int32, device="cuda")
    x = wn.embed(table, y)
    assert torch.equal(x, table[y.long()])
    d = torch.randint(-3, 4, (3, 50, 64), device="cuda").float()
    want = torch.zeros_like(table).index_add_(0, y.flatten().long(), d.view(-1, 64))
    assert torch.equal(wn.embed_backward(d, y, 256), want)


@pytest.mark.parametrize("dtype", DTYPES, ids=IDS)
@pytest.mark.parametrize("kind", ["one", "distinct", "sorted", "down", "text", "none", "padded"])
@pytest.mark.parametrize("N,D,V", [(1, 5, 4), (63, 8, 256), (64, 64, 1), (65, 100, 511), (1000, 33, 513), (5000, 16, 256), (3000, 264, 70000)])
def test_gradient(N, D, V, kind, dtype):
    _backward(N, D, V, kind, dtype)


@pytest.mark.parametrize("kind", ["one", "text", "padded", "sorted"])
@pytest.mark.parametrize("N,D,V", [(16384, 8, 300), (16385, 8, 300), (40000, 16, 300000), (300000, 4, 256)])
def test_gradient_of_many_rows(N, D, V, kind):
    """One block's sort and many blocks', one to three passes, runs over hundreds of chunks."""
    _backward(N, D, V, kind, torch.float32)


@pytest.mark.parametrize("dtype", DTYPES, ids=IDS)
@pytest.mark.parametrize("N,D,V", [(500, 96, 40), (20000, 24, 256), (400, 2055, 100)])
def test_gradient_of_arbitrary_rows(N, D, V, dtype):
    _backward(N, D, V, "padded", dtype, whole=False, scale=3.3)


@pytest.mark.parametrize("dtype", DTYPES, ids=IDS)
def test_padding_holds_anything_and_arrays_start_anywhere(dtype):
    import paper_1702_07825_amd as wn
    N, D, V = 300, 40, 50
    t = _tokens("padded", N, V)
    d = torch.randint(-4, 5, (N, D), generator=torch.Generator().manual_seed(4)).to(dtype)
    want = wn.embed_backward(d.cuda(), t.cuda(), V)
    off = (t < 0) | (t >= V)
    d[off] = float("nan")
    s = torch.zeros(N * D + 1, dtype=dtype, device="cuda")
    s[1:] = d.flatten().cuda()
    out = torch.full((V * D + 2,), 9, dtype=dtype, device="cuda")
    got = wn.embed_backward(s[1:].view(N, D), t.cuda(), V, dtable=out[1:-1].view(V, D))
    assert torch.equal(got, want) and float(out[0]) == 9 and float(out[-1]) == 9


def test_runs_on_another_stream_and_in_a_graph():
    import paper_1702_07825_amd as wn
    for N in (2000, 30000):
        V, D = 300, 24
        sets = [(_tokens(k, N, V, seed=N).cuda(), torch.randn((N, D), device="cuda")) for k in ("text", "padded", "one")]
        table = torch.randn((V, D), device="cuda")
        want = [(wn.embed(table, t, 2.0), wn.embed_backward(d, t, V, 2.0)) for t, d in sets]
        stream = torch.cuda.Stream()
        stream.wait_stream(torch.cuda.current_stream())
        got = (wn.embed(table, sets[1][0], 2.0, stream=stream), wn.embed_backward(sets[1][1], sets[1][0], V, 2.0, stream=stream))
        torch.cuda.current_stream().wait_stream(stream)
        assert all(torch.equal(a, c) for a, c in zip(got, want[1]))
        t, d = sets[0][0].clone(), sets[0][1].clone()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs = (wn.embed(table, t, 2.0), wn.embed_backward(d, t, V, 2.0))
        for k in (0, 1, 2, 0):
            t.copy_(sets[k][0])
            d.copy_(sets[k][1])
            graph.replay()
            torch.cuda.synchronize()
            wn.embed_backward(sets[(k + 1) % 3][1], sets[(k + 1) % 3][0], V)
            assert all(torch.equal(a, c) for a, c in zip(outs, want[k]))


def test_gradient_against_differences():
    """The lookup is linear: (embed(table + d) - embed(table)) . g = d . embed_backward(g), exactly for small integers."""
    import paper_1702_07825_amd as wn
    t = _tokens("padded", 200, 30).cuda()
    table, d = (torch.randint(-8, 9, (30, 16), device="cuda").float() for _ in range(2))
    g = torch.randint(-8, 9, (200, 16), device="cuda").float()
    diff = wn.embed(table + d, t, 2.0) - wn.embed(table, t, 2.0)
    assert float((diff * g).double().sum()) == float((d * wn.embed_backward(g, t, 30, 2.0)).double().sum())


def test_offsets_beyond_32_bits():
    """A table of 4.6 GB: rows on both sides of 2^32 bytes."""
    import paper_1702_07825_amd as wn
    V, D = (1 << 20) + 70000, 2048
    table = torch.zeros((V, D), dtype=torch.bfloat16, device="cuda")
    rows = torch.tensor([0, 5, (1 << 20) - 1, 1 << 20, (1 << 20) + 1, V - 1], device="cuda")
    table[rows] = torch.randn((6, D), device="cuda").bfloat16()
    t = rows.to(torch.int32).repeat(3)
    assert torch.equal(wn.embed(table, t), table[rows].repeat(3, 1))
    d = torch.randint(-4, 5, (18, D), device="cuda").bfloat16()
    got = wn.embed_backward(d, t, V)
    assert torch.equal(got[rows], d.view(3, 6, D).float().sum(dim=0).bfloat16())
    got[rows] = 0
    assert not bool(got.any())


def test_no_rows_and_refusals():
    import paper_1702_07825_amd as wn
    none = torch.empty((0,), dtype=torch.int32, device="cuda")
    table, t = torch.ones((5, 4), device="cuda"), torch.zeros(3, dtype=torch.int32, device="cuda")
    assert wn.embed(table, none).shape == (0, 4)
    assert not bool(wn.embed_backward(torch.empty((0, 4), device="cuda"), none, 5).any())
    for f in (lambda: wn.embed(table.half(), t), lambda: wn.embed(table, t.long()), lambda: wn.embed(table.t(), t),
              lambda: wn.embed_backward(torch.ones((3, 4), device="cuda"), t, (1 << 32) + 5), lambda: wn.embed(table, t.cpu()), lambda: wn.embed(table[0], t),
              lambda: wn.embed_backward(torch.ones((2, 4), device="cuda"), t, 5),
              lambda: wn.embed_backward(torch.ones((3, 4), device="cuda"), t, 5, dtable=torch.ones((4, 4), device="cuda"))):
        with pytest.raises((ValueError, TypeError)):
            f()
    for f in (lambda: wn.embed(table, t, scale=float("inf")), lambda: wn.embed_backward(torch.ones((3, 4), device="cuda"), t, 0),
              lambda: wn.embed_backward(torch.ones((3, 4), device="cuda"), t, 5, workspace=torch.empty(256, dtype=torch.uint8, device="cuda"))):
        with pytest.raises(wn.WnError):
            f()


def test_lookup_of_more_threads_than_a_launch_takes():
    """2^24 rows by a block each (34 GB): beyond 2^32 threads in all."""
    import paper_1702_07825_amd as wn
    N, V, D = (1 << 24) + 5, 300, 1032
    table = torch.randn((V, D), generator=torch.Generator().manual_seed(9)).bfloat16().cuda()
    t = torch.randint(0, V, (N,), generator=torch.Generator(device="cuda").manual_seed(9), device="cuda", dtype=torch.int32)
    out = wn.embed(table, t)
    for a in range(0, N, 1 << 20):
        assert torch.equal(out[a:a + (1 << 20)], table[t[a:a + (1 << 20)].long()]), a
