"""The dense operators' entry points without a GPU: arguments are refused on the host
before any HIP call (addresses are stand-ins that validation never follows)."""
import ctypes
import math
import random

import pytest

from paper_2608_09388_amd import binding as shc
from tests.test_row_ops_abi_cpu import caller, check, err

A, ODD = 0x10000, 0x10002     # aligned; aligned to bf16 but not to fp32
NAN, INF = float("nan"), float("inf")


@pytest.fixture(scope="module")
def lib():
    return shc.load()


SIZES = [(dict(n=-1), -1, "n_rows"), (dict(n=1 << 27), -4, "2^27"), (dict(dtype=3), -4, "dtype")]
LINEAR = SIZES + [
    (dict(Cin=0), -1, "Cin"), (dict(Cin=65537), -4, "Cin"), (dict(Cout=-1), -1, "Cout"),
    (dict(Cout=65537), -4, "Cout"), (dict(act=-1), -4, "activation"), (dict(act=4), -4, "activation"),
    (dict(x=None), -1, "x is NULL"), (dict(x=ODD), -3, "x"), (dict(x_ld=63), -1, "x"),
    (dict(x_ld=1 << 38), -4, "2^40"), (dict(W=None), -1, "W is NULL"), (dict(W_ld=31), -1, "W"),
    (dict(W=ODD), -3, "W"), (dict(ws=None), -1, "ws"), (dict(ws=A + 8), -3, "ws"),
    (dict(ws_bytes=15), -2, "workspace"),
]


def test_linear(lib):
    need = lib.shc_linear_workspace(10, 64, 32, 0, 0)
    assert need > 0
    call = caller(lib, "shc_linear", dict(
        x=A, x_ld=64, n=10, Cin=64, W=A, W_ld=32, Cout=32, bias=A, act=2, res=A, res_ld=32,
        dtype=0, pre=A, pre_ld=32, out=A * 2, out_ld=32, ws=A, ws_bytes=need, stream=None))
    check(lib, call, LINEAR + [
        (dict(bias=ODD), -3, "bias"), (dict(res=ODD), -3, "residual"), (dict(res_ld=5), -1, "residual"),
        (dict(pre=ODD), -3, "pre"), (dict(pre_ld=5), -1, "pre"), (dict(out=None), -1, "out"),
        (dict(out_ld=31), -1, "out"), (dict(res=A * 2, res_ld=33), -1, "another stride"),
        (dict(n=(1 << 27) - 1, Cin=65536, x_ld=65536), -4, "2^40"),
        (dict(n=1 << 20, Cin=65536, Cout=65536, x_ld=65536, W_ld=65536, pre_ld=65536, res_ld=65536),
         -4, "2^22 tiles"),
    ])
    assert call(n=0, x=None, W=None, res=None, pre=None, out=None, ws=None) == 0


def test_linear_backward(lib):
    need = lib.shc_linear_backward_workspace(10, 64, 32, 0, 2, 0)
    call = caller(lib, "shc_linear_backward", dict(
        dout=A, dout_ld=32, x=A, x_ld=64, n=10, Cin=64, W=A, W_ld=32, Cout=32, pre=A, pre_ld=32,
        act=2, dtype=0, acc=0, dx=A, dx_ld=64, dW=A, dW_ld=32, db=A, ws=A, ws_bytes=need,
        stream=None))
    check(lib, call, LINEAR + [
        (dict(acc=2), -1, "accumulate"), (dict(dout=None), -1, "dout"), (dict(dout_ld=1), -1, "dout"),
        (dict(pre=None), -1, "pre is NULL"), (dict(pre_ld=1), -1, "pre"), (dict(dx=ODD), -3, "dx"),
        (dict(dx_ld=63), -1, "dx"), (dict(dW=ODD), -3, "dW"), (dict(dW_ld=3), -1, "dW"),
        (dict(db=ODD), -3, "db"),
    ])
    assert call(n=0, dout=None, x=None, W=None, pre=None, dx=None, dW=None, db=None, ws=None) == 0


XENT = SIZES + [
    (dict(C=0), -1, "C"), (dict(C=65537), -4, "C"), (dict(V=0), -1, "V"),
    (dict(V=(1 << 24) + 1), -4, "V"), (dict(x=None), -1, "x"), (dict(x_ld=1), -1, "x"),
    (dict(W=None), -1, "W"), (dict(W=ODD), -3, "W"), (dict(W_ld=63), -1, "W"),
    (dict(bias=ODD), -3, "bias"), (dict(labels=None), -1, "labels"),
    (dict(labels=A + 4, id_type=1), -3, "labels"), (dict(id_type=2), -4, "id type"),
    (dict(label_ld=-1), -1, "label_stride"), (dict(label_ld=1 << 40), -1, "label_stride"),
    (dict(ws=None), -1, "ws"), (dict(ws=A + 8), -3, "ws"), (dict(ws_bytes=15), -2, "workspace"),
    (dict(n=1 << 22, V=1 << 24), -4, "2^22 tiles"),
]
GRADS = [(dict(acc=7), -1, "accumulate"), (dict(w=ODD), -3, "row_weight"), (dict(dx=ODD), -3, "dx"),
         (dict(dx_ld=2), -1, "dx"), (dict(dW=ODD), -3, "dW"), (dict(dW_ld=2), -1, "dW"),
         (dict(db=ODD), -3, "db")]


def xent(more):
    return dict(x=A, x_ld=64, n=10, C=64, W=A, W_ld=64, V=100, bias=A, labels=A, id_type=0,
                label_ld=2, **more)


def test_linear_cross_entropy(lib):
    need = lib.shc_linear_cross_entropy_workspace(10, 64, 100, 0, 0, 0)
    call = caller(lib, "shc_linear_cross_entropy", xent(dict(
        dtype=0, loss=A, lse=A, ws=A, ws_bytes=need, stream=None)))
    check(lib, call, XENT + [(dict(loss=None), -1, "loss"), (dict(lse=ODD), -3, "lse")])
    assert call(n=0, x=None, W=None, labels=None, loss=None, ws=None) == 0


def test_linear_cross_entropy_backward(lib):
    need = lib.shc_linear_cross_entropy_workspace(10, 64, 100, 0, 1, 0)
    call = caller(lib, "shc_linear_cross_entropy_backward", xent(dict(
        lse=A, w=A, dtype=0, acc=0, dx=A, dx_ld=64, dW=A, dW_ld=64, db=A, ws=A, ws_bytes=need,
        stream=None)))
    check(lib, call, XENT + GRADS + [(dict(lse=None), -1, "lse")])
    assert call(n=0, x=None, W=None, labels=None, lse=None, dx=None, dW=None, db=None, ws=None) == 0


def test_linear_cross_entropy_step(lib):
    need = lib.shc_linear_cross_entropy_workspace(10, 64, 100, 0, 2, 0)
    call = caller(lib, "shc_linear_cross_entropy_step", xent(dict(
        w=A, dtype=0, acc=0, loss=A, dx=A, dx_ld=64, dW=A, dW_ld=64, db=A, ws=A, ws_bytes=need,
        stream=None)))
    check(lib, call, XENT + GRADS + [(dict(loss=None), -1, "loss")])


def test_workspace_queries_refuse(lib):
    for bad in ((-1, 8, 8, 0, 0), (1 << 27, 8, 8, 0, 0), (8, 0, 8, 0, 0), (8, 8, 65537, 0, 0),
                (8, 8, 8, 2, 0)):
        assert lib.shc_linear_workspace(*bad) == 0
        assert lib.shc_linear_backward_workspace(*bad[:4], 0, bad[4]) == 0
    assert lib.shc_linear_backward_workspace(8, 8, 8, 0, 9, 0) == 0
    assert lib.shc_linear_cross_entropy_workspace(8, 8, 8, 0, 3, 0) == 0
    assert lib.shc_linear_cross_entropy_workspace(8, 8, (1 << 24) + 1, 0, 0, 0) == 0


def test_workspaces_grow_with_the_rows(lib):
    """A workspace for n rows serves every smaller count, and one for any alignment the
    aligned ones."""
    rng = random.Random(7)
    for _ in range(400):
        a, b = (int(math.exp(rng.uniform(0, math.log(65536)))) for _ in range(2))
        V = int(math.exp(rng.uniform(0, math.log(1 << 20))))
        n = int(math.exp(rng.uniform(0, math.log(1 << 21))))
        ns = sorted({1, n // 3 + 1, n - n // 7, n, n + 1, n + 255, 2 * n})
        for dtype in (0, 1):
            for al in (0, 1):
                for f in (lambda m, al=al: lib.shc_linear_workspace(m, a, b, dtype, al),
                          lambda m, al=al: lib.shc_linear_backward_workspace(m, a, b, dtype, 2, al),
                          *(lambda m, p=p, al=al: lib.shc_linear_cross_entropy_workspace(
                              m, a, V, dtype, p, al) for p in range(3))):
                    sizes = [f(m) for m in ns]
                    assert sizes == sorted(sizes), (a, b, V, n, dtype)
            assert (lib.shc_linear_workspace(n, a, b, dtype, 1)
                    <= lib.shc_linear_workspace(n, a, b, dtype, 0))


def grads(*items):
    t = (shc.Grad * max(1, len(items)))()
    for i, g in enumerate(items):
        t[i] = shc.Grad(*g)
    return t, len(items)


def test_clip(lib):
    ok = (A, A, 100, 0)
    for items, code, text in (
            ([(None, A, 5, 0)], -1, "data is NULL"), ([ok, (ODD, A, 5, 0)], -3, "grads[1]"),
            ([(A, A, -1, 0)], -1, "numel"), ([(A, A, 1 << 40, 0)], -1, "numel"),
            ([(A, A, 5, 2)], -4, "dtype")):
        t, n = grads(*items)
        assert lib.shc_grad_norm(t, n, A, A, 1 << 20, None) == code and text in err(lib)
        assert lib.shc_clip_grads(t, n, A, 1.0, None) == code and text in err(lib)
        assert lib.shc_grad_norm_workspace(t, n) == 0
    t, n = grads(ok)
    need = lib.shc_grad_norm_workspace(t, n)
    assert need > 0
    for args, code, text in (((t, n, None, A, need, None), -1, "norm"),
                             ((t, n, ODD, A, need, None), -3, "norm"),
                             ((t, n, A, None, need, None), -1, "ws"),
                             ((t, n, A, A, need - 1, None), -2, "workspace"),
                             ((t, -1, A, A, need, None), -1, "count"),
                             ((t, 65537, A, A, need, None), -1, "count"),
                             ((None, 1, A, A, need, None), -1, "grads")):
        assert lib.shc_grad_norm(*args) == code and text in err(lib)
    for most in (-1.0, NAN):
        assert lib.shc_clip_grads(t, n, A, most, None) == -1 and "max_norm" in err(lib)
    for items in ([(A, None, 5, 0)], [ok, ok], [(A, A + 4, 100, 0)], [ok, (A + 396, A + 396, 2, 0)],
                  [(A, 2 * A, 8, 0), (3 * A, 2 * A + 28, 1, 0)], [(A, 2 * A, 8, 0), (2 * A, 3 * A, 8, 0)]):
        t, n = grads(*items)
        assert lib.shc_clip_grads(t, n, A, 1.0, None) == -1
        assert "NULL" in err(lib) or "overlaps" in err(lib)


def test_struct_layout():
    assert ctypes.sizeof(shc.Grad) == 32


@pytest.mark.parametrize("out,off", [(2 * A, 0), (2 * A, 396), (A, 396), (A, 0)])
def test_clip_refuses_an_output_over_the_norm(lib, out, off):
    t, n = grads((A, out, 100, 0))
    norm = out + off
    assert lib.shc_clip_grads(t, n, norm, 1.0, None) == -1
    assert "norm" in err(lib)
