"""Refusals of wn_orthogonalize (include/wn_train.h) that need no GPU: every argument check comes before the first device
call, so they run here with made-up pointers that nothing reads."""
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


def _array(spans):
    import paper_1702_07825_amd as wn
    a = (wn.OrthoArray * len(spans))()
    for k, s in enumerate(spans):
        a[k].g, a[k].out, a[k].rows, a[k].cols, a[k].dtype, a[k].scale = s
    return a


def _call(lib, n_arrays=1, g=P, out=P, rows=4, cols=6, dtype=0, scale=1.0, steps=2, coefficients=(1.0,) * 6, eps=0.0, ws=P, n=1 << 40,
          arrays=True):
    a = _array([(g, out, rows, cols, dtype, scale)])
    c = None if coefficients is None else (ctypes.c_float * len(coefficients))(*coefficients)
    return lib.wn_orthogonalize(n_arrays, a if arrays else None, steps, c, eps, ws, n, None)


@pytest.mark.parametrize("kw,code", [
    (dict(n_arrays=-1), -1), (dict(n_arrays=(1 << 16) + 1), -1), (dict(arrays=False), -1), (dict(dtype=2), -2), (dict(dtype=7), -1),
    (dict(rows=-1), -1), (dict(cols=-1), -1), (dict(rows=(1 << 18) + 1), -1), (dict(cols=(1 << 18) + 1), -1),
    (dict(rows=1 << 17, cols=(1 << 15) + 1), -1), (dict(g=None), -1), (dict(out=None), -1), (dict(g=P + 2), -1),
    (dict(out=P + 1, dtype=1), -1), (dict(scale=float("nan")), -1), (dict(scale=float("inf")), -1), (dict(steps=0), -1),
    (dict(steps=65, coefficients=(1.0,) * 195), -1), (dict(coefficients=None), -1), (dict(coefficients=(1.0,) * 5 + (float("nan"),)), -1),
    (dict(eps=-1.0), -1), (dict(eps=float("nan")), -1), (dict(eps=float("inf")), -1), (dict(ws=None), -1), (dict(ws=P + 8), -1),
    (dict(n=100), -1), (dict(out=P + 4), -1)])
def test_refuses(lib, kw, code):
    assert _call(lib, **kw) == code
    assert lib.wn_last_error().decode()


def test_nothing_to_do(lib):
    assert _call(lib, n_arrays=0, ws=None, n=0) == 0
    assert _call(lib, n_arrays=0, arrays=False, ws=None, n=0) == 0
    assert _call(lib, g=None, out=None, rows=0, ws=None, n=0) == 0
    assert _call(lib, g=None, out=None, cols=0, ws=None, n=0) == 0


@pytest.mark.parametrize("spans", [((P, P), (P, P)), ((P, 2 * P), (3 * P, 2 * P + 92)), ((P, 2 * P), (2 * P + 92, 3 * P)),
                                   ((P, P + 4), (3 * P, 3 * P))])
def test_overlaps_are_refused(lib, spans):
    """4 x 6 fp32 matrices, 96 bytes: the same one twice, outputs that overlap, an output over another's input or askew over
    its own."""
    a = _array([(g, out, 4, 6, 0, 1.0) for g, out in spans])
    c = (ctypes.c_float * 3)(1.0, 0.0, 0.0)
    assert lib.wn_orthogonalize(2, a, 1, c, 0.0, P, 1 << 40, None) == -1
    assert "overlap" in lib.wn_last_error().decode()


def test_workspace_sizes(lib):
    def need(*shapes):
        return lib.wn_orthogonalize_workspace_bytes(len(shapes), _array([(0, 0, r, c, d, 1.0) for r, c, d in shapes]))

    assert need((0, 5, 0)) == 0 and need((4, -1, 0)) == 0 and need((4, 4, 2)) == 0
    assert 0 < need((64, 64, 1)) < need((64, 64, 0)) < need((64, 64, 0), (64, 64, 0))
    assert need((640, 64, 1)) == need((64, 640, 1))
    # groups of about 4 GiB share it
    one = need((4096, 4096, 1))
    assert 5 * 4096 * 4096 * 2 < one < 6 * 4096 * 4096 * 2
    assert need(*[(4096, 4096, 1)] * 60) < 4.1 * (1 << 30)
