"""Refusals of the training operators (include/wn_train.h) that need no GPU: every argument check comes
before the first device call, so they run here with made-up pointers that nothing reads."""
import ctypes
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


def _loss(lib, dtype=0, N=4, D=8, V=16, x=P, w=P, b=None, y=P, loss=P, lse=P, ws=P, n=1 << 40):
    return lib.wn_loss(dtype, N, D, V, x, w, b, y, loss, lse, ws, n, None)


def _backward(lib, dtype=0, N=4, D=8, V=16, x=P, w=P, b=None, y=P, lse=P, g=P, dx=P, dw=P, db=P, ws=P, n=1 << 40):
    return lib.wn_loss_backward(dtype, N, D, V, x, w, b, y, lse, g, dx, dw, db, ws, n, None)


def _embed(lib, dtype=0, N=4, D=8, V=16, table=P, t=P, scale=1.0, out=P):
    return lib.wn_embed(dtype, N, D, V, table, t, scale, out, None)


def _embed_backward(lib, dtype=0, N=4, D=8, V=16, dout=P, t=P, scale=1.0, dtable=P, ws=P, n=1 << 40):
    return lib.wn_embed_backward(dtype, N, D, V, dout, t, scale, dtable, ws, n, None)


def _clip(lib, n_arrays=1, g=P, out=P, n=4, dtype=0, max_norm=1.0, norm=P, ws=P, bytes_=1 << 40, arrays=True):
    import paper_1702_07825_amd as wn
    a = (wn.ClipArray * 1)()
    a[0].g, a[0].out, a[0].n, a[0].dtype = g, out, n, dtype
    return lib.wn_clip(n_arrays, a if arrays else None, max_norm, norm, ws, bytes_, None)


SIZES = [dict(N=-1), dict(D=0), dict(D=(1 << 16) + 1), dict(V=0), dict(V=(1 << 24) + 1)]


@pytest.mark.parametrize("kw,code", [(dict(dtype=2), -2), (dict(dtype=3), -1), (dict(dtype=-1), -1)]
                         + [(k, -1) for k in SIZES + [dict(N=(1 << 20) + 1)]]
                         + [({k: None}, -1) for k in ("x", "w", "y", "loss", "lse", "ws")]
                         + [(dict(ws=P + 128), -1), (dict(n=100), -1)])
def test_loss_refuses(lib, kw, code):
    assert _loss(lib, **kw) == code
    assert lib.wn_last_error().decode()


@pytest.mark.parametrize("kw,code", [(dict(dtype=2), -2), (dict(dtype=3), -1)]
                         + [(k, -1) for k in SIZES + [dict(N=(1 << 20) + 1)]]
                         + [({k: None}, -1) for k in ("x", "w", "y", "lse", "g", "ws")]
                         + [(dict(dx=None, dw=None, db=None), -1), (dict(ws=P + 8), -1), (dict(n=100), -1)])
def test_loss_backward_refuses(lib, kw, code):
    assert _backward(lib, **kw) == code
    assert lib.wn_last_error().decode()


@pytest.mark.parametrize("kw,code", [(dict(dtype=2), -2), (dict(dtype=9), -1), (dict(scale=float("nan")), -1),
                                     (dict(scale=float("inf")), -1)]
                         + [(k, -1) for k in SIZES + [dict(N=(1 << 27) + 1)]]
                         + [({k: None}, -1) for k in ("table", "t", "out")])
def test_embed_refuses(lib, kw, code):
    assert _embed(lib, **kw) == code
    assert lib.wn_last_error().decode()


@pytest.mark.parametrize("kw,code", [(dict(dtype=2), -2), (dict(dtype=9), -1), (dict(scale=float("nan")), -1)]
                         + [(k, -1) for k in SIZES + [dict(N=(1 << 27) + 1)]]
                         + [({k: None}, -1) for k in ("dout", "t", "dtable", "ws")]
                         + [(dict(ws=P + 64), -1), (dict(n=100), -1)])
def test_embed_backward_refuses(lib, kw, code):
    assert _embed_backward(lib, **kw) == code
    assert lib.wn_last_error().decode()


@pytest.mark.parametrize("kw,code", [(dict(n_arrays=-1), -1), (dict(n_arrays=(1 << 20) + 1), -1), (dict(arrays=False), -1),
                                     (dict(norm=None), -1), (dict(max_norm=-1.0), -1), (dict(max_norm=float("nan")), -1),
                                     (dict(dtype=2), -2), (dict(dtype=5), -1), (dict(n=-1), -1), (dict(n=(1 << 40) + 1), -1),
                                     (dict(g=None), -1), (dict(out=None), -1), (dict(g=P + 2), -1),
                                     (dict(dtype=1, out=P + 1), -1), (dict(ws=None), -1), (dict(ws=P + 8), -1),
                                     (dict(bytes_=8), -1)])
def test_clip_refuses(lib, kw, code):
    assert _clip(lib, **kw) == code
    assert lib.wn_last_error().decode()


def test_memory_that_is_not_on_a_device_is_refused(lib):
    host = ctypes.create_string_buffer(1 << 16)
    p = (ctypes.addressof(host) + 255) // 256 * 256
    for rc in (_loss(lib, x=p, w=p, y=p, loss=p, lse=p, ws=p), _embed(lib, table=p, t=p, out=p),
               _embed_backward(lib, dout=p, t=p, dtable=p, ws=p), _clip(lib, g=p, out=p, norm=p, ws=p),
               _backward(lib, x=p, w=p, y=p, lse=p, g=p, dx=p, dw=p, db=p, ws=p)):
        assert rc == -1
        assert "device memory" in lib.wn_last_error().decode()


def test_no_rows_are_no_work(lib):
    assert _loss(lib, N=0, x=None, w=None, y=None, loss=None, lse=None, ws=None, n=0) == 0
    assert _backward(lib, N=0, x=None, w=None, y=None, lse=None, g=None, dw=None, db=None, ws=None, n=0) == 0
    assert _embed(lib, N=0, table=None, t=None, out=None) == 0


def test_workspace_sizes(lib):
    for f, args in ((lib.wn_loss_workspace_bytes, (0,)), (lib.wn_loss_backward_workspace_bytes, (0,)),
                    (lib.wn_embed_backward_workspace_bytes, ())):
        assert f(*args, 4, 8, 16) > 0
        for bad in ((0, 8, 16), (-1, 8, 16), (4, 0, 16), (4, 8, 0), (4, 1 << 17, 16), (4, 8, 1 << 25)):
            assert f(*args, *bad) == 0
    assert lib.wn_loss_workspace_bytes(2, 4, 8, 16) == 0
    # a fixed multiple of the pieces' budget, whatever the vocabulary: the logits are not kept
    assert lib.wn_loss_backward_workspace_bytes(1, 8192, 2048, 1 << 20) < 4 << 30
    assert lib.wn_clip_workspace_bytes() > 0


def test_clip_refuses_arrays_that_overlap(lib):
    """Found before any device call; arrays that only touch, outputs that are the inputs, and inputs listed twice with
    outputs of their own go on to the check of the memory."""
    import paper_1702_07825_amd as wn

    def clip(*arrays):
        a = (wn.ClipArray * len(arrays))()
        for k, (g, out, n, dtype) in enumerate(arrays):
            a[k].g, a[k].out, a[k].n, a[k].dtype = P + g, P + out, n, dtype
        assert lib.wn_clip(len(arrays), a, 1.0, P, P, 1 << 40, None) == -1
        return lib.wn_last_error().decode()

    for bad in (((0, 0, 4, 0), (0, 0, 4, 0)), ((0, 0, 4, 0), (12, 12, 4, 0)), ((64, 64, 8, 1), (32, 32, 9, 0)),
                ((0, 64, 4, 0), (32, 64, 4, 0)), ((0, 8, 4, 0),), ((0, 64, 4, 0), (64, 128, 4, 0)),
                ((16, 64, 4, 0), (0, 16, 1, 0)), ((0, 256, 4, 0), (64, 512, 4, 0), (128, 264, 4, 1))):
        assert "overlap" in clip(*bad), bad
    for good in (((0, 0, 4, 0), (16, 16, 4, 0)), ((32, 32, 8, 1), (0, 0, 8, 0)), ((0, 64, 4, 0), (0, 128, 4, 0)),
                 ((0, 16, 4, 0),), ((16, 0, 4, 0),), ((0, 0, 4, 0), (4, 4, 0, 0)), ((0, 256, 4, 0), (16, 64, 4, 0), (32, 128, 4, 1))):
        assert "device memory" in clip(*good), good
