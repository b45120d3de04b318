"""Scoring of recorded speech (wn_score), the features it goes by (wn_teacher_features), and the training
operators together on a model's two ends.

The features and teacher forcing's logits come from the same sums, so W_out features + b_out in 64 bits is off from
the logits by an fp32 sum of 256 products (256 2^-24 sum |w z| and 2^-24 for the bias), and the scores by what
wn_loss's fp16 parts may add: 3 2^-22 and 3 256 2^-24 of sum |w z|, twice (lse and target), and 2^-20 for
the exponentials' sum.
"""
import numpy as np
import pytest

import synth

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def _model(l, r, s, seed=3, dtype="f32", taps=1, approx=False):
    import paper_1702_07825_amd as wn
    w = synth.make_weights(l, r, s, seed=seed, bias_scale=0.2)
    if taps == 2:
        w["embed"] = np.stack([w["embed"], w["embed"][::-1]]).copy()
    return w, wn.WaveNet(w, [1 << (i % 5) for i in range(l)], weight_dtype=dtype, approx_nonlin=approx)


def _inputs(l, r, B, T, seed=4):
    g = torch.Generator().manual_seed(seed)
    return torch.randn((B, T, l, 2 * r), generator=g).cuda(), torch.randint(0, 256, (B, T), generator=g, dtype=torch.int32).cuda()


def _w_out(w, dtype):
    t = torch.tensor(w["w_out"])
    if dtype == "bf16":
        t = t.bfloat16().float()
    elif dtype == "i8":
        s = (t.double().abs().amax(dim=1) / 127).float()
        t = torch.round(t.double() / s.double()[:, None]).clamp(-127, 127).float() * s[:, None]
    return t.cuda()


@pytest.mark.parametrize("dtype", ["f32", "bf16", "i8"])
@pytest.mark.parametrize("l,r,s,B,T", [(4, 16, 32, 1, 1), (4, 16, 32, 3, 16), (4, 16, 32, 2, 300), (20, 64, 256, 1, 7), (20, 64, 256, 2, 500),
                                       (6, 32, 128, 5, 64), (8, 128, 256, 1, 1000), (5, 64, 128, 70, 9)])
def test_scores_and_features(l, r, s, B, T, dtype):
    w, net = _model(l, r, s, dtype=dtype)
    cond, y = _inputs(l, r, B, T)
    if T > 4:
        y[0, T // 2] = -1  # padding: no score, and 0 to the next step, as teacher forcing clamps it
    print("score", l, r, s, B, T, dtype, flush=True)
    ws = net.new_workspace(B)
    logits = net.teacher_force(cond, y, workspace=ws)
    z = net.teacher_features(cond, y)
    nll = net.score(cond, y, workspace=ws)
    assert net.status(ws) == 0
    wo, b = _w_out(w, dtype).double(), torch.tensor(w["b_out"]).cuda().double()
    zd = z.double()
    S = zd.abs() @ wo.abs().t().contiguous()
    l64 = zd @ wo.t().contiguous() + b
    assert bool((z >= 0).all())
    assert bool(((logits.double() - l64).abs() <= 256 * 2.0 ** -24 * S + 2.0 ** -23 * (l64.abs() + b.abs())).all())
    ok = (y >= 0)
    want = torch.where(ok, torch.logsumexp(l64, dim=2) - l64.gather(2, y.clamp(min=0).long()[..., None])[..., 0], 0.0)
    tol = 2 * (3 * 2.0 ** -22 + 3 * 256 * 2.0 ** -24) * S.amax(dim=2) + 2.0 ** -20 * (1 + want.abs() + l64.abs().amax(dim=2))
    assert bool(((nll.double() - want).abs() <= tol).all())
    net.close()


@pytest.mark.parametrize("l,r,s,B,T", [(4, 16, 32, 2, 40), (20, 64, 256, 1, 600)])
def test_scoring_in_pieces_continues_the_state(l, r, s, B, T):
    """Cut anywhere it gives the scores of one call, and generation goes on as after teacher forcing.  (Calls of up to 64
    rows take the loss's kernel for few rows, whose sums differ in their last places; longer ones agree bit for bit.)"""
    w, net = _model(l, r, s)
    cond, y = _inputs(l, r, B, T)
    ws = net.new_workspace(B)
    whole = net.score(cond, y, workspace=ws)
    u = torch.rand((B, 20), generator=torch.Generator().manual_seed(5)).cuda()
    more = _inputs(l, r, B, 20, seed=6)[0]
    after = net.generate(more, u, workspace=ws, reset=False).clone()
    at, parts = 0, []
    for n in (1, 7, 16, T - 24):
        parts.append(net.score(cond[:, at:at + n].contiguous(), y[:, at:at + n].contiguous(), workspace=ws, reset=at == 0))
        at += n
    z = torch.cat(parts, dim=1)
    assert bool(((z - whole).abs() <= 1e-5).all())
    if B * (T - 24) > 64:
        assert torch.equal(z[:, 24:], whole[:, 24:])
    assert torch.equal(net.generate(more, u, workspace=ws, reset=False), after)
    ws2 = net.new_workspace(B)
    net.teacher_force(cond, y, workspace=ws2)
    assert torch.equal(net.generate(more, u, workspace=ws2, reset=False), after)
    net.close()


def test_two_taps_and_the_approximate_gate():
    for kw in (dict(taps=2), dict(approx=True)):
        w, net = _model(6, 32, 128, **kw)
        cond, y = _inputs(6, 32, 2, 100)
        z, logits = net.teacher_features(cond, y), net.teacher_force(cond, y)
        nll = net.score(cond, y)
        want = torch.nn.functional.cross_entropy(logits.double().flatten(0, 1), y.long().flatten(), reduction="none").view(2, 100)
        assert bool(((nll.double() - want).abs() <= 2e-5).all()) and z.shape == (2, 100, 256)
        net.close()


def test_on_another_stream():
    w, net = _model(20, 64, 256)
    cond, y = _inputs(20, 64, 1, 200)
    want = net.score(cond, y)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    got = net.score(cond, y, stream=s)
    torch.cuda.current_stream().wait_stream(s)
    assert torch.equal(got, want)
    net.close()


def test_refusals(monkeypatch):
    import paper_1702_07825_amd as wn
    w, net = _model(4, 16, 32)
    cond, y = _inputs(4, 16, 1, 20)
    small = torch.empty(256, dtype=torch.uint8, device="cuda")
    for kw in (dict(workspace=small), dict(scratch=small)):
        with pytest.raises(wn.WnError) as e:
            net.score(cond, y, **kw)
        assert e.value.code == wn.WN_EINVAL
    for bad in (lambda: net.score(cond, y.long()), lambda: net.score(cond, y[:, :5]), lambda: net.score(cond.cpu(), y),
                lambda: net.teacher_features(cond, y, features=torch.empty((1, 20, 255), device="cuda"))):
        with pytest.raises((ValueError, TypeError)):
            bad()
    net.close()
    monkeypatch.setenv("WN_KERNEL", "stream_l2")  # goes step by step
    w, net = _model(4, 16, 32)
    for f in (net.score, net.teacher_features):
        with pytest.raises(wn.WnError) as e:
            f(cond, y)
        assert e.value.code == wn.WN_EUNSUPPORTED
    net.close()


def test_gradients_of_an_adapted_output_layer():
    """Features of recorded speech, the loss's gradients for W_out and b_out, their clip: against 64 bits; and the score of
    the model with the layer moved against the gradient is lower."""
    import paper_1702_07825_amd as wn
    w, net = _model(8, 64, 256)
    cond, y = _inputs(8, 64, 2, 300)
    y[1, 250:] = -1
    z = net.teacher_features(cond, y).view(-1, 256)
    t = y.view(-1)
    W, b = torch.tensor(w["w_out"]).cuda(), torch.tensor(w["b_out"]).cuda()
    ok = t >= 0
    g = ok.float() / ok.sum()
    loss, lse = wn.head_loss(z, W, t, b=b)
    assert torch.equal(loss.view_as(y), net.score(cond, y))
    _, dw, db = wn.head_loss_backward(z, W, t, lse, g, b=b, need=("dw", "db"))
    zd = z.double()
    p = torch.softmax(zd @ W.double().t().contiguous() + b.double(), dim=1)
    p[torch.arange(600, device="cuda")[ok], t[ok].long()] -= 1
    q = p * g.double()[:, None]
    want_w, want_b = q.t().contiguous() @ zd, q.sum(dim=0)
    # (each element to 1e-5 of the largest: some 600 fp32 sums of products of at most that size)
    assert float((dw.double() - want_w).abs().max()) <= 1e-5 * float(want_w.abs().max())
    assert float((db.double() - want_b).abs().max()) <= 1e-5 * float(want_b.abs().max())
    norm = wn.clip_gradients([dw, db], 0.1)
    want = float((want_w.square().sum() + want_b.square().sum()).sqrt())
    assert abs(float(norm) - want) <= 1e-5 * want
    f = min(1.0, 0.1 / want)
    assert float((dw.double() - want_w * f).abs().max()) <= 1e-5 * float((want_w * f).abs().max())
    net.close()


def test_a_training_step_of_the_two_ends():
    """Embedding, loss, both gradients and their clip, as a step takes them, against torch's in 64 bits; captured in one
    graph and replayed on other tokens."""
    import paper_1702_07825_amd as wn
    V, D, N = 256, 64, 700
    g = torch.Generator().manual_seed(8)
    table, w, b = ((torch.randn(s, generator=g) * 0.3).cuda() for s in ((V, D), (V, D), (V,)))
    sets = [torch.randint(-1, V, (N + 1,), generator=g, dtype=torch.int32).cuda() for _ in range(3)]
    grad = torch.full((N,), 1.0 / N, device="cuda")

    def step(tokens, targets):
        x = wn.embed(table, tokens, scale=8.0)
        loss, lse = wn.head_loss(x, w, targets, b=b)
        dx, dw, db = wn.head_loss_backward(x, w, targets, lse, grad, b=b)
        dt = wn.embed_backward(dx, tokens, V, scale=8.0)
        norm = wn.clip_gradients([dt, dw, db], 0.05)
        return loss, dt, dw, db, norm

    def exact(tokens, targets):
        p = [t.double().requires_grad_() for t in (table, w, b)]
        x = torch.where((tokens >= 0)[:, None], p[0][tokens.clamp(min=0).long()] * 8.0, 0.0)
        loss = torch.nn.functional.cross_entropy(x @ p[1].t().contiguous() + p[2], targets.long(), ignore_index=-1, reduction="none")
        grads = torch.autograd.grad((loss * grad.double()).sum(), p)
        norm = torch.stack([t.square().sum() for t in grads]).sum().sqrt()
        f = min(1.0, 0.05 / float(norm))
        return [loss.detach(), *(t * f for t in grads), norm]

    def near(got, want):
        for a, c in zip(got, want):
            assert float((a.double() - c).abs().max()) <= 1e-5 * float(c.abs().max())

    want = [exact(s[:-1], s[1:].contiguous()) for s in sets]
    for s, c in zip(sets, want):
        near(step(s[:-1].contiguous(), s[1:].contiguous()), c)
    tokens, targets = sets[0][:-1].clone(), sets[0][1:].clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = step(tokens, targets)
    for k in (0, 1, 2, 0):
        tokens.copy_(sets[k][:-1])
        targets.copy_(sets[k][1:])
        graph.replay()
        torch.cuda.synchronize()
        near(outs, want[k])
        step(sets[(k + 1) % 3][:-1].contiguous(), sets[(k + 1) % 3][1:].contiguous())


def test_scores_of_more_rows_than_the_loss_takes_at_a_time():
    """2^18 rows a call of the loss: three streams of 87500 steps take two.  The scores are those of the loss on both parts,
    and on both sides of the cut and at the ends those of 64 bits, within the tolerance above."""
    import paper_1702_07825_amd as wn
    B, T = 3, 87500
    w, net = _model(4, 16, 32)
    cond, y = _inputs(4, 16, B, T)
    y[2, -3:] = -1
    z = net.teacher_features(cond, y).view(-1, 256)
    nll = net.score(cond, y).view(-1)
    wo, b, t = torch.tensor(w["w_out"]).cuda(), torch.tensor(w["b_out"]).cuda(), y.view(-1)
    for a, e in ((0, 1 << 18), (1 << 18, B * T)):
        assert torch.equal(nll[a:e], wn.head_loss(z[a:e], wo, t[a:e], b=b)[0])
    for a in (0, (1 << 18) - 40, B * T - 80):
        zd, ta = z[a:a + 80].double(), t[a:a + 80]
        S = zd.abs() @ wo.double().abs().t().contiguous()
        l = zd @ wo.double().t().contiguous() + b.double()
        want = torch.where(ta >= 0, torch.logsumexp(l, dim=1) - l.gather(1, ta.clamp(min=0).long()[:, None])[:, 0], 0.0)
        tol = 2 * (3 * 2.0 ** -22 + 3 * 256 * 2.0 ** -24) * S.amax(dim=1) + 2.0 ** -20 * (1 + want.abs() + l.abs().amax(dim=1))
        assert bool(((nll[a:a + 80].double() - want).abs() <= tol).all())
    net.close()


@pytest.mark.parametrize("what", ["y", "nll"])
def test_refused_memory_leaves_the_state(what):
    """y or nll in host memory is refused before anything runs: the call after it gives what it would have given."""
    import paper_1702_07825_amd as wn
    w, net = _model(4, 16, 32)
    cond, y = _inputs(4, 16, 2, 60)
    ws = net.new_workspace(2)
    first, rest = [(cond[:, a:b].contiguous(), y[:, a:b].contiguous()) for a, b in ((0, 30), (30, 60))]
    net.score(*first, workspace=ws)
    want = net.score(*rest, workspace=ws, reset=False)
    net.score(*first, workspace=ws)
    scratch = torch.empty(int(net._lib.wn_score_scratch_bytes(net._h, 2, 30)), dtype=torch.uint8, device="cuda")
    host = torch.zeros((2, 30), dtype=torch.int32 if what == "y" else torch.float32, pin_memory=True)
    nll = torch.empty((2, 30), device="cuda")
    args = {"y": rest[1].data_ptr(), "nll": nll.data_ptr(), what: host.data_ptr()}
    rc = net._lib.wn_score(net._h, 2, 30, rest[0].data_ptr(), args["y"], args["nll"], ws.data_ptr(), ws.numel(), scratch.data_ptr(),
                           scratch.numel(), 0, torch.cuda.current_stream().cuda_stream)
    assert rc == wn.WN_EINVAL and what in net._lib.wn_last_error().decode()
    assert torch.equal(net.score(*rest, workspace=ws, reset=False), want)
    net.close()


def test_generation_on_a_busy_stream_keeps_its_memory():
    """Generation, teacher forcing, scoring and conditioning on a stream that is busy, with workspaces of their own: what they
    need is not handed out when the call returns."""
    import paper_1702_07825_amd as wn
    w, net = _model(4, 16, 32)
    g = np.random.default_rng(9)
    cw = {k: (g.standard_normal(s) * 0.1).astype(np.float32) for k, s in
          (("w1", (2, 96, 2, 20)), ("b1", (2, 96)), ("w2", (2, 192, 2, 64)), ("b2", (2, 192)))}
    conditioner = wn.Conditioner(cw, 4, 16, 1, 60)

    def inputs():
        cond, y = _inputs(4, 16, 2, 100)
        u = torch.rand((2, 100), generator=torch.Generator().manual_seed(10)).cuda()
        return cond, y, u, torch.randn((2, 5, 20), generator=torch.Generator().manual_seed(11)).cuda()

    calls = [lambda s, c, y, u, f: net.generate(c, u, stream=s), lambda s, c, y, u, f: net.teacher_force(c, y, stream=s),
             lambda s, c, y, u, f: net.score(c, y, stream=s), lambda s, c, y, u, f: conditioner(f, 300, stream=s)]
    for call in calls:
        want = call(None, *inputs())
        torch.cuda.synchronize()
        tensors = inputs()
        sizes = [t.shape for t in tensors]
        stream = torch.cuda.Stream()
        stream.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(stream):
            torch.cuda._sleep(100_000_000)
        got = call(stream, *tensors)
        del tensors
        # (small numbers and zeros: harmless as a state, if they were to lie in one)
        others = [torch.zeros(s, device="cuda") for s in sizes] + [torch.zeros(net.workspace_bytes(2), dtype=torch.uint8, device="cuda")]
        torch.cuda.synchronize()
        assert torch.equal(got, want)
        del others
    net.close()
