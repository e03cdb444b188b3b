"""The row operators' entry points without a GPU: arguments are refused on the
host before any HIP call (as in test_abi_cpu.py, addresses are stand-ins that
validation never follows)."""
import math
import random

import pytest

from paper_2608_09388_amd import binding as shc

A, ODD = 0x10000, 0x10002     # aligned; aligned to bf16 but not to fp32


@pytest.fixture(scope="module")
def lib():
    return shc.load()


def err(lib):
    return lib.shc_last_error().decode()


NAN, INF = float("nan"), float("inf")


def caller(lib, name, defaults):
    fn = getattr(lib, name)

    def call(**kw):
        unknown = set(kw) - set(defaults)
        assert not unknown, unknown
        return fn(*dict(defaults, **kw).values())
    return call


def check(lib, call, cases):
    for kw, code, text in cases:
        assert call(**kw) == code, (kw, err(lib))
        assert text in err(lib), (kw, err(lib))


def test_embed_rows(lib):
    call = caller(lib, "shc_embed_rows", dict(
        E=A, E_stride=64, R=100, ids=A, id_type=0, id_stride=2, n=10, C=64, scale=1.0, add=None,
        add_stride=0, dtype=0, out=A, out_stride=64, stream=None))
    check(lib, call, [
        (dict(n=-1), -1, "n_rows"), (dict(C=0), -1, "C = 0"), (dict(C=65537), -4, "C"),
        (dict(dtype=7), -4, "dtype"), (dict(R=0), -1, "n_entries"), (dict(R=1 << 23), -4, "2^22"),
        (dict(scale=NAN), -1, "scale"), (dict(scale=INF), -1, "scale"),
        (dict(id_type=2), -4, "id type"), (dict(id_stride=-1), -1, "id_stride"),
        (dict(id_stride=1 << 50), -1, "id_stride"), (dict(ids=None), -1, "ids"),
        (dict(ids=ODD), -3, "ids"), (dict(ids=A + 4, id_type=1), -3, "ids"),
        (dict(E=None), -1, "E is NULL"), (dict(E=ODD), -3, "E"), (dict(E_stride=63), -1, "E"),
        (dict(E_stride=1 << 40), -4, "2^40"), (dict(out=None), -1, "out"),
        (dict(out_stride=1), -1, "out"), (dict(add=A, add_stride=3), -1, "add"),
        (dict(add=ODD, add_stride=64), -3, "add"), (dict(out=A + 1, dtype=1, E=ODD), -3, "out"),
    ])
    assert call(n=0, ids=None, E=None, out=None) == 0


def test_embed_rows_backward(lib):
    ws = lib.shc_embed_rows_backward_workspace(10, 100, 64)
    assert ws > 0
    assert lib.shc_embed_rows_backward_workspace(-1, 100, 64) == 0
    assert lib.shc_embed_rows_backward_workspace(10, 0, 64) == 0
    assert lib.shc_embed_rows_backward_workspace(10, 100, 0) == 0
    call = caller(lib, "shc_embed_rows_backward", dict(
        dY=A, dY_stride=64, ids=A, id_type=0, id_stride=1, n=10, R=100, C=64, scale=1.0, pad=-1,
        dtype=0, acc=0, dE=A, dE_stride=64, ws=A, ws_bytes=ws, stream=None))
    check(lib, call, [
        (dict(n=-1), -1, "n_rows"), (dict(n=(1 << 28) + 1), -4, "2^28"), (dict(R=-4), -1, "n_entries"),
        (dict(acc=2), -1, "accumulate"), (dict(dY=None), -1, "dY"), (dict(dY_stride=5), -1, "dY"),
        (dict(dE=None), -1, "dE"), (dict(dE=ODD), -3, "dE"), (dict(dE_stride=63), -1, "dE"),
        (dict(ws=None), -1, "ws"), (dict(ws=A + 4), -3, "ws"), (dict(ws_bytes=ws - 1), -2, "workspace"),
        (dict(ids=None), -1, "ids"), (dict(scale=NAN), -1, "scale"),
    ])


def test_workspaces_grow_with_the_rows(lib):
    """A workspace for n rows serves every smaller count."""
    for C in (1, 64, 5000):
        last = 0
        for n in (0, 1, 31, 32, 33, 1000, 4096, 70000, 300000):
            b = lib.shc_embed_rows_backward_workspace(n, 1000, C)
            assert b >= last
            last = b
        last = 0
        for n in (0, 1, 2, 255, 256, 511, 512, 513, 5000, 1 << 20):
            b = lib.shc_layer_norm_backward_workspace(n, C)
            assert b >= last
            last = b
    for V in (1, 4000, 9000, 140001):
        last = 0
        for n in (1, 2, 5, 100, 255, 256, 1023, 1024, 5000):
            b = lib.shc_distill_top_workspace(n, V)
            assert b >= last
            last = b


def test_workspaces_grow_across_the_rules(lib):
    """The counts at which a call changes its cutting need no more than larger ones."""
    rng = random.Random(5)
    for _ in range(300):
        C = int(math.exp(rng.uniform(0, math.log(65536))))
        n = int(math.exp(rng.uniform(0, math.log(1 << 22))))
        sizes = [lib.shc_embed_rows_backward_workspace(m, 1000, C)
                 for m in sorted({max(0, n - n // 3), n - 1, n, n + 1, n + n // 7})]
        assert sizes == sorted(sizes), (n, C)
    for C in (1, 64, 100, 4096):
        for w in (32768, 131072):
            edge = (w << 9) // C
            sizes = [lib.shc_embed_rows_backward_workspace(m, 1000, C)
                     for m in (edge // 2, edge - 1, edge, edge + 1, edge + 4096)]
            assert sizes == sorted(sizes), C
    for edge in (2048, 4096, 524288):
        sizes = [lib.shc_embed_rows_backward_workspace(m, 1000, 16)
                 for m in (edge - 1, edge, edge + 1, edge + 4096)]
        assert sizes == sorted(sizes)


def test_layer_norm(lib):
    call = caller(lib, "shc_layer_norm", dict(
        x=A, x_stride=64, n=10, C=64, gamma=A, beta=A, eps=1e-5, dtype=0, y=A, y_stride=64, mean=A,
        rstd=A, stream=None))
    check(lib, call, [
        (dict(n=-1), -1, "n_rows"), (dict(C=-2), -1, "C"), (dict(C=16385), -4, "C"),
        (dict(dtype=2), -4, "dtype"), (dict(eps=0.0), -1, "eps"), (dict(eps=NAN), -1, "eps"),
        (dict(eps=INF), -1, "eps"), (dict(x=None), -1, "x"), (dict(x=ODD), -3, "x"),
        (dict(x_stride=1), -1, "x"), (dict(y=None), -1, "y"), (dict(gamma=ODD), -3, "gamma"),
        (dict(beta=ODD), -3, "beta"), (dict(mean=ODD), -3, "mean"), (dict(rstd=ODD), -3, "rstd"),
    ])
    assert call(n=0, x=None, y=None) == 0


def test_layer_norm_backward(lib):
    ws = lib.shc_layer_norm_backward_workspace(10, 64)
    assert lib.shc_layer_norm_backward_workspace(-1, 64) == 0
    assert lib.shc_layer_norm_backward_workspace(10, 16385) == 0
    call = caller(lib, "shc_layer_norm_backward", dict(
        dy=A, dy_stride=64, x=A, x_stride=64, n=10, C=64, gamma=None, mean=A, rstd=A, dtype=0,
        acc=0, dx=A, dx_stride=64, dg=A, db=A, ws=A, ws_bytes=ws, stream=None))
    check(lib, call, [
        (dict(n=-1), -1, "n_rows"), (dict(C=20000), -4, "C"), (dict(acc=-1), -1, "accumulate"),
        (dict(dy=None), -1, "dy"), (dict(x=None), -1, "x"), (dict(dx_stride=63), -1, "dx"),
        (dict(dx=ODD), -3, "dx"), (dict(mean=None), -1, "mean"), (dict(rstd=None), -1, "rstd"),
        (dict(dg=ODD), -3, "dgamma"), (dict(db=ODD), -3, "dbeta"), (dict(ws=None), -1, "ws"),
        (dict(ws_bytes=ws - 1), -2, "workspace"),
    ])
    assert call(n=0, dy=None, x=None, mean=None, rstd=None, dx=None, dg=None, db=None, ws=None) == 0


def distill(extra):
    return dict(z=A, stride=64, n=10, V=64, ids=A, top=A, k=8, T=1.0, **extra)


COMMON = [
    (dict(n=-1), -1, "n_rows"), (dict(V=0), -1, "V"), (dict(V=(1 << 24) + 1), -4, "V"),
    (dict(k=0), -1, "k"), (dict(k=257), -4, "k"), (dict(T=0.0), -1, "temperature"),
    (dict(T=1e-40), -1, "temperature"), (dict(T=NAN), -1, "temperature"), (dict(T=INF), -1, "temperature"), (dict(dtype=5), -4, "dtype"),
    (dict(z=None), -1, "logits"), (dict(z=ODD), -3, "logits"), (dict(stride=63), -1, "logits"),
    (dict(ids=None), -1, "top_ids"), (dict(top=None), -1, "top_logits"), (dict(top=ODD), -3, "top"),
]


def test_distill_top(lib):
    call = caller(lib, "shc_distill_top", distill(dict(dtype=0, loss=A, lse=None, ws=None,
                                                       ws_bytes=0, stream=None)))
    check(lib, call, COMMON + [(dict(loss=None), -1, "loss"), (dict(lse=ODD), -3, "lse")])
    need = lib.shc_distill_top_workspace(10, 100000)
    assert need > 0
    check(lib, call, [(dict(V=100000, stride=100000), -1, "ws"),
                      (dict(V=100000, stride=100000, ws=A, ws_bytes=need - 1), -2, "workspace")])
    assert call(n=0, z=None, ids=None, top=None, loss=None) == 0
    assert lib.shc_distill_top_workspace(0, 100) == 0 == lib.shc_distill_top_workspace(5, 0)


def test_distill_top_backward(lib):
    call = caller(lib, "shc_distill_top_backward", distill(dict(
        lse=A, w=None, dtype=0, dz=A, dz_stride=64, stream=None)))
    check(lib, call, COMMON + [(dict(lse=None), -1, "lse"), (dict(w=ODD), -3, "row_weight"),
                               (dict(dz=None), -1, "dlogits"), (dict(dz_stride=2), -1, "dlogits")])
    assert call(n=0, z=None, ids=None, top=None, lse=None, dz=None) == 0


def test_distill_top_step(lib):
    call = caller(lib, "shc_distill_top_step", distill(dict(
        w=None, dtype=0, loss=A, dz=A, dz_stride=64, ws=None, ws_bytes=0, stream=None)))
    check(lib, call, COMMON + [(dict(loss=None), -1, "loss"), (dict(w=ODD), -3, "row_weight"),
                               (dict(dz=ODD), -3, "dlogits")])
    assert call(n=0, z=None, ids=None, top=None, loss=None, dz=None) == 0
