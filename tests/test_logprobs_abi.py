"""Refusals of wn_logprobs and wn_logprobs_backward (include/wn_train.h) that need no GPU: every argument check comes
before the first device call, so they run here with made-up pointers that nothing reads."""
import os

import pytest

P = 1 << 20  # a non-null, 256-byte aligned pointer that is never read


@pytest.fixture(scope="module")
def lib():
    import paper_1702_07825_amd as wn
    if not os.path.exists(wn.LIB_PATH):
        import __graft_entry__
        __graft_entry__.build()
    return wn.load_library()


def _probe(lib, dtype=0, N=4, D=8, V=16, top=3, x=P, w=P, b=None, y=P, logprob=P, entropy=P, lse=P, ids=P, lps=P, ws=P, n=1 << 40):
    return lib.wn_logprobs(dtype, N, D, V, top, x, w, b, y, logprob, entropy, lse, ids, lps, ws, n, None)


def _backward(lib, dtype=0, N=4, D=8, V=16, x=P, w=P, b=None, y=P, lse=P, entropy=P, g=P, h=P, dx=P, dw=P, db=P, ws=P, n=1 << 40):
    return lib.wn_logprobs_backward(dtype, N, D, V, x, w, b, y, lse, entropy, g, h, dx, dw, db, ws, n, None)


SIZES = [dict(N=-1), dict(N=(1 << 20) + 1), dict(D=0), dict(D=(1 << 16) + 1), dict(V=0), dict(V=(1 << 24) + 1)]


@pytest.mark.parametrize("kw,code", [(dict(dtype=2), -2), (dict(dtype=3), -1), (dict(dtype=-1), -1)]
                         + [(k, -1) for k in SIZES]
                         + [({k: None}, -1) for k in ("x", "w", "y", "logprob", "entropy", "lse", "ids", "lps", "ws")]
                         + [(dict(top=-1), -1), (dict(top=33, V=100), -1), (dict(top=17), -1), (dict(ws=P + 128), -1), (dict(n=100), -1)])
def test_logprobs_refuses(lib, kw, code):
    assert _probe(lib, **kw) == code
    assert lib.wn_last_error().decode()


@pytest.mark.parametrize("kw,code", [(dict(dtype=2), -2), (dict(dtype=3), -1)]
                         + [(k, -1) for k in SIZES]
                         + [({k: None}, -1) for k in ("x", "w", "y", "lse", "entropy", "ws")]
                         + [(dict(g=None, h=None), -1), (dict(dx=None, dw=None, db=None), -1), (dict(ws=P + 8), -1), (dict(n=100), -1)])
def test_logprobs_backward_refuses(lib, kw, code):
    assert _backward(lib, **kw) == code
    assert lib.wn_last_error().decode()


def test_no_rows(lib):
    assert _probe(lib, N=0, x=None, w=None, y=None, logprob=None, entropy=None, lse=None, ids=None, lps=None, ws=None, n=0) == 0
    assert _backward(lib, N=0, x=None, w=None, y=None, lse=None, entropy=None, g=None, h=None, dw=None, db=None, ws=None, n=0) == 0


def test_workspace_sizes(lib):
    for dtype in (0, 1):
        for N in (1, 64, 65, 5000):
            sizes = [lib.wn_logprobs_workspace_bytes(dtype, N, 100, 3000, top) for top in (0, 1, 32)]
            assert 0 < sizes[0] < sizes[1] < sizes[2]
            assert lib.wn_logprobs_backward_workspace_bytes(dtype, N, 100, 3000) > lib.wn_loss_backward_workspace_bytes(dtype, N, 100, 3000)
        # the groups' largest logits are bounded by taking the classes in pieces
        assert lib.wn_logprobs_workspace_bytes(dtype, 1 << 20, 64, 1 << 20, 32) - lib.wn_logprobs_workspace_bytes(dtype, 1 << 20, 64, 1 << 20, 0) < 1 << 30
        for bad in ((-1, 8, 16, 0), (4, 0, 16, 0), (4, 8, 0, 0), (4, 8, 16, -1), (4, 8, 16, 17), (4, 8, 100, 33), (0, 8, 16, 1)):
            assert lib.wn_logprobs_workspace_bytes(dtype, *bad) == 0
        assert lib.wn_logprobs_backward_workspace_bytes(dtype, 0, 8, 16) == 0
    assert lib.wn_logprobs_workspace_bytes(2, 4, 8, 16, 0) == 0
