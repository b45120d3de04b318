"""The norm over many gradients and their clip (wn_clip).

The squares are summed in 64 bits, so the norm is the exact one rounded to fp32 once (2^-24, and 2^-40 for the sum).
max_norm is an fp32 argument; the factor is rounded to fp32 and so is each product: a clipped element is within 2 2^-24 of itself (bf16: and
2^-8 for its rounding).
"""
import math

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def _grads(sizes, dtypes, seed=1, std=1.0):
    g = torch.Generator().manual_seed(seed)
    return [(torch.randn(n, generator=g) * std).to(dtypes[i % len(dtypes)]).cuda() for i, n in enumerate(sizes)]


def _check(grads, max_norm, outs=None):
    import paper_1702_07825_amd as wn
    print("clip", len(grads), "arrays", sum(t.numel() for t in grads), "elements", flush=True)
    before = [t.clone() for t in grads]
    want = math.sqrt(sum(float(t.double().square().sum()) for t in grads))
    norm = wn.clip_gradients(grads, max_norm, outs=outs)
    got = float(norm)
    assert abs(got - want) <= want * (2.0 ** -24 + 2.0 ** -40)
    f = min(1.0, float(torch.tensor(max_norm, dtype=torch.float32)) / want) if want else 1.0  # (as the call takes it)
    for b, g, o in zip(before, grads, grads if outs is None else outs):
        w = b.double() * f
        if f == 1.0:
            assert torch.equal(o, b)
        else:
            tol = w.abs() * (2 * 2.0 ** -24 + 2.0 ** -40 + (2.0 ** -8 if b.dtype == torch.bfloat16 else 0)) + 1e-40
            assert bool(((o.double() - w).abs() <= tol).all())
        if outs is not None:
            assert torch.equal(g, b)
    return norm


F, H = torch.float32, torch.bfloat16


@pytest.mark.parametrize("dtypes", [(F,), (H,), (F, H)], ids=["f32", "bf16", "both"])
@pytest.mark.parametrize("sizes", [(1,), (3, 0, 5), (8191, 8192, 8193), tuple(range(0, 300)), (100000, 1, 77777), (3000001,)],
                         ids=["one", "empty", "chunk", "many", "mixed", "long"])
def test_sizes(sizes, dtypes):
    grads = _grads(sizes, dtypes)
    n = math.sqrt(max(1, sum(sizes)))
    _check([t.clone() for t in grads], 0.3 * n)          # in place
    _check(grads, 0.3 * n, outs=[torch.empty_like(t) for t in grads])
    _check(grads, 3.0 * n, outs=[torch.empty_like(t) for t in grads])  # nothing to clip: a copy
    _check(grads, 3.0 * n)


def test_more_arrays_than_a_launch_takes_and_blocks_than_a_launch_has():
    _check(_grads([97 * k % 1000 for k in range(500)] + [20_000_000, 5], (F, H)), 2.0)


def test_arrays_that_start_anywhere():
    """Views into flat buffers, the outputs' alignment unlike the inputs'; what lies around them stays."""
    flat = {d: _grads([40000], (d,))[0] for d in (F, H)}
    grads, outs, holds, at = [], [], [], 1
    for k, n in enumerate((5, 333, 8200, 1, 16391)):
        d = (F, H)[k % 2]
        grads.append(flat[d][at:at + n])
        hold = torch.full((n + 4,), 5, dtype=d, device="cuda")
        outs.append(hold[k % 3 + 1:k % 3 + 1 + n])
        holds.append((hold, k % 3 + 1, n))
        at += n
    _check(grads, 10.0, outs=outs)
    for h, b, n in holds:
        assert bool((h[:b] == 5).all()) and bool((h[b + n:] == 5).all())


@pytest.mark.parametrize("std", [1e-30, 1e-20, 1e18])
def test_squares_beyond_fp32(std):
    grads = _grads((5000, 77), (F,), std=std)
    _check(grads, std)


@pytest.mark.parametrize("bad", [float("inf"), -float("inf"), float("nan")])
@pytest.mark.parametrize("place", [True, False])
def test_not_finite_gradients_stay_as_they_are(bad, place):
    import paper_1702_07825_amd as wn
    grads = _grads((500, 9000), (F, H))
    grads[1][8999] = bad
    before = [t.clone() for t in grads]
    outs = None if place else [torch.zeros_like(t) for t in grads]
    norm = wn.clip_gradients(grads, 1.0, outs=outs)
    assert not math.isfinite(float(norm))
    for b, o in zip(before, outs or grads):
        assert torch.equal(b.view(torch.int32 if b.dtype == F else torch.int16), o.view(torch.int32 if b.dtype == F else torch.int16))


def test_a_norm_beyond_fp32_is_infinite():
    import paper_1702_07825_amd as wn
    g = torch.full((100,), 3e38, device="cuda")
    assert float(wn.clip_gradients([g], 1.0)) == float("inf") and bool((g == 3e38).all())


def test_zero_norms():
    import paper_1702_07825_amd as wn
    z = torch.zeros(100, device="cuda")
    assert float(wn.clip_gradients([z], 1.0)) == 0 and not bool(z.any())
    assert float(wn.clip_gradients([z], 0.0)) == 0 and not bool(z.any())
    g = torch.ones(100, device="cuda")
    assert float(wn.clip_gradients([g], 0.0)) == 10 and not bool(g.any())
    g = torch.ones(100, device="cuda")
    assert float(wn.clip_gradients([g], float("inf"))) == 10 and bool((g == 1).all())
    e = torch.empty(0, device="cuda")
    assert float(wn.clip_gradients([e], 1.0)) == 0


def test_runs_on_another_stream_and_in_a_graph():
    import paper_1702_07825_amd as wn
    sizes = [33 * k for k in range(150)]
    sets = [_grads(sizes, (F, H), seed=s) for s in (5, 6, 7)]
    want = []
    for s in sets:
        outs = [torch.empty_like(t) for t in s]
        want.append([wn.clip_gradients(s, 1.5, outs=outs), *outs])
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    outs = [torch.empty_like(t) for t in sets[1]]
    norm = wn.clip_gradients(sets[1], 1.5, outs=outs, stream=stream)
    torch.cuda.current_stream().wait_stream(stream)
    assert all(torch.equal(a, c) for a, c in zip([norm, *outs], want[1]))
    held = [t.clone() for t in sets[0]]
    outs = [torch.empty_like(t) for t in held]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        norm = wn.clip_gradients(held, 1.5, outs=outs)
    for k in (0, 1, 2, 1):
        for h, t in zip(held, sets[k]):
            h.copy_(t)
        graph.replay()
        torch.cuda.synchronize()
        wn.clip_gradients([t.clone() for t in sets[0]], 1.0)
        assert all(torch.equal(a, c) for a, c in zip([norm, *outs], want[k]))


def test_refusals():
    import paper_1702_07825_amd as wn
    g = torch.ones(8, device="cuda")
    for f in (lambda: wn.clip_gradients([], 1.0), lambda: wn.clip_gradients([g.half()], 1.0), lambda: wn.clip_gradients([g.cpu()], 1.0),
              lambda: wn.clip_gradients([g[::2]], 1.0), lambda: wn.clip_gradients([g], 1.0, outs=[g[:4]]),
              lambda: wn.clip_gradients([g], 1.0, outs=[]), lambda: wn.clip_gradients([g], 1.0, outs=[g.bfloat16()])):
        with pytest.raises((ValueError, TypeError)):
            f()
    for m in (-1.0, float("nan")):
        with pytest.raises(wn.WnError):
            wn.clip_gradients([g], m)


@pytest.mark.parametrize("max_norm", [1e-3, 1e-7, 1e-20, 1e-30])
@pytest.mark.parametrize("place", [True, False])
def test_factors_below_fp32(max_norm, place):
    """Norms near fp32's largest: max_norm / norm is subnormal in fp32 or 0 there, the clipped gradients are not."""
    grads = _grads((3000, 77, 40000), (F, H), std=5e35)
    _check(grads, max_norm, outs=None if place else [torch.empty_like(t) for t in grads])


@pytest.mark.parametrize("extra", [0, 1, 5])
def test_on_both_sides_of_the_chunks_lengths(extra):
    sizes = (1 << 20, 12345, 0, (1 << 20) - 12345 - 7, 7 + extra)  # 2^21 elements and some
    for dtypes in ((F,), (H,), (F, H)):
        _check(_grads(sizes, dtypes), 300.0)


def test_gradients_that_share_memory_are_refused():
    import paper_1702_07825_amd as wn
    g = torch.ones(100, device="cuda")
    for grads, outs in (([g, g], None), ([g[:60], g[50:]], None), ([g[:50], g[50:]], [g[50:], g[:50]])):
        with pytest.raises(wn.WnError) as e:
            wn.clip_gradients(grads, 1.0, outs=outs)
        assert e.value.code == wn.WN_EINVAL and "overlap" in str(e.value)
    assert bool((g == 1).all())
    outs = [torch.empty_like(g) for _ in range(2)]
    assert float(wn.clip_gradients([g, g], 1e9, outs=outs)) == float(torch.tensor(200.0).sqrt())
