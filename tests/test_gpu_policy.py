"""A policy's step on a model's output layer, as a program takes it: features of recorded speech, log probabilities with
entropies and alternatives, the gradients of advantages and an entropy bonus, their clip, and the orthogonalised update.

Each operator is held to its formula in 64 bits at the inputs that the one before gave it, with the tolerances that the
operators' own tests derive; the clip's outputs to two roundings in fp32 and of bf16 one more, 2^-22 and 2^-8 of a value, and the norm to 2^-23.
"""
import pytest

from tests import test_gpu_logprobs as logprobs
from tests import test_gpu_ortho as ortho
from tests import test_gpu_score as score

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
DTYPES = logprobs.DTYPES


def _step(x, w, b, y, g, h, max_norm=0.05, stream=None):
    """What the step gives: the rows' values, the clipped gradients with their norm, and the layer's update."""
    import paper_1702_07825_amd as wn
    rows = wn.head_logprobs(x, w, y, b=b, top=3, stream=stream)
    _, dw, db = wn.head_logprobs_backward(x, w, y, rows[2], rows[1], g, h, b=b, need=("dw", "db"), stream=stream)
    clipped = [torch.empty_like(dw), torch.empty_like(db)]
    norm = wn.clip_gradients([dw, db], max_norm, outs=clipped, stream=stream)
    update = wn.orthogonalize(clipped[:1], scales=0.02, stream=stream)[0]
    return [*rows, dw, db, norm, *clipped, update]


def _upstream(y, seed):
    """Advantages and an entropy bonus, means over the rows with a token."""
    gen = torch.Generator().manual_seed(seed)
    n = int((y >= 0).sum())
    return (torch.randn(y.shape, generator=gen) / n).cuda(), torch.full(y.shape, 0.05 / n, device="cuda")


def _layer(dtype, T, B=2, seed=4):
    w, net = score._model(8, 64, 256)
    cond, y = score._inputs(8, 64, B, T, seed=seed)
    y[B - 1, T - T // 5:] = -1  # the last sequence's end is padding
    x = net.teacher_features(cond, y).view(-1, 256).to(dtype)
    net.close()
    return x, torch.tensor(w["w_out"]).cuda().to(dtype), torch.tensor(w["b_out"]).cuda(), y.view(-1)


@DTYPES
@pytest.mark.parametrize("T", [17, 301])
def test_each_operator_on_what_the_one_before_gives(T, dtype):
    x, w, b, y = _layer(dtype, T)
    g, h = _upstream(y, 5)
    got = _step(x, w, b, y, g, h)
    want, k = logprobs._rows(x, w, b, y, 3)
    for name, t in zip(logprobs.NAMES, got):
        if name == "top_ids":
            assert torch.equal(t, want[name])
        else:
            logprobs._near(t, want[name], name)
    grads = logprobs._gradients(k, dtype == torch.float32, g, h)
    dw, db, norm, cw, cb, update = got[5:]
    logprobs._near(dw, grads["dw"], "dw")
    logprobs._near(db, grads["db"], "db")
    n = float((dw.double().square().sum() + db.double().square().sum()).sqrt())
    assert abs(float(norm) - n) <= 2.0 ** -23 * n
    f = min(1.0, float(torch.tensor(0.05)) / n)  # (as the call takes it)
    for t, c in ((dw, cw), (db, cb)):
        d = t.double() * f
        assert bool(((c.double() - d).abs() <= (2.0 ** -22 + (2.0 ** -8 if c.dtype == torch.bfloat16 else 0)) * d.abs() + 1e-38).all())
    ortho._near(update, cw, scale=0.02)


@DTYPES
@pytest.mark.parametrize("T", [17, 301])
def test_a_step_in_a_graph(T, dtype):
    """Captured once, replayed on other speech with eager steps between: the eager results, each time."""
    layers = [_layer(dtype, T, seed=10 + k) for k in range(3)]
    w, b = layers[0][1:3]
    sets = [(x, y, *_upstream(y, 20 + k)) for k, (x, _, _, y) in enumerate(layers)]

    def step(x, y, g, h):
        return _step(x, w, b, y, g, h)

    want = [[t.clone() for t in step(*s)] for s in sets]
    held = [t.clone() for t in sets[0]]
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = step(*held)
    for k in (0, 1, 2, 1, 0):
        for a, c in zip(held, sets[k]):
            a.copy_(c)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, c) for a, c in zip(outs, want[k])), k
        other = (k + 1) % 3
        assert all(torch.equal(a, c) for a, c in zip(step(*sets[other]), want[other])), other


@DTYPES
def test_a_step_on_a_busy_stream(dtype):
    """The step's inputs may be dropped when its calls return, on a stream that has yet to reach them."""
    def make():
        x, w, b, y = _layer(dtype, 60)
        return (x, w, b, y, *_upstream(y, 6))

    want = _step(*make())
    given = make()
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        torch.cuda._sleep(100_000_000)
    got = _step(*given, stream=stream)
    sizes = [(t.shape, t.dtype) for t in given]
    del given
    others = [torch.ones(s, dtype=d, device="cuda") for s, d in sizes for _ in range(2)]
    torch.cuda.synchronize()
    del others
    assert all(torch.equal(a, c) for a, c in zip(got, want))
