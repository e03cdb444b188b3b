"""Embedding rows and their gradient against the 64-bit oracle."""
import numpy as np
import pytest
import torch

from oracle import row_oracle as O
from paper_2608_09388_amd import binding as shc
from tests.gpu_util import Compaction, require_gpu
from tests.row_util import Rows, close, rounded, stored, u

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def dev():
    return require_gpu()


def ids_tensor(ids, kind, stride=1):
    t = torch.full((max(len(ids), 1), stride), -5, dtype=kind, device="cuda")
    t = t[:len(ids)]
    t[:, stride - 1] = torch.as_tensor(np.asarray(ids))
    return t[:, stride - 1]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,R,C,extra,off", [
    (1, 1, 1, 0, 0), (2, 3, 7, 0, 1), (65, 10, 16, 0, 0), (33, 100, 100, 3, 2),
    (1000, 37, 128, 64, 0), (5, 50, 511, 0, 3), (300, 655, 520, 8, 8), (17, 9, 1024, 0, 0),
    (3, 4, 4099, 1, 1), (2, 2, 16384, 0, 0), (1, 3, 65536, 0, 0),
])
@pytest.mark.parametrize("with_add", [False, True])
def test_rows(dtype, n, R, C, extra, off, with_add):
    r = np.random.default_rng(n * 7 + C)
    E = Rows(R, C, dtype, extra, off, r.standard_normal((R, C)))
    add = Rows(n, C, dtype, extra + 1, off, r.standard_normal((n, C))) if with_add else None
    ids = r.integers(-1, R + 1, n)          # some have no row
    out = Rows(n, C, dtype, 2 * extra, off)
    kind, stride = (torch.int64, 1) if n % 2 else (torch.int32, 2)
    shc.embed_rows(E.t, ids_tensor(ids, kind, stride), out.t, scale=1.7,
                   add=None if add is None else add.t)
    ref = O.embed(E.get(), ids, float(np.float32(1.7)), None if add is None else add.get())
    close(out.get(), ref, rounded(u * np.abs(ref), ref, dtype), "rows")
    out.check_guard("rows")


def test_ids_are_the_compaction_s_vertices():
    r = np.random.default_rng(3)
    mask = (r.random((6, 655)) < 0.1).astype(np.uint8)
    c = Compaction(mask)
    n = c.run()
    E = Rows(655, 64, "bf16", values=r.standard_normal((655, 64)))
    out = shc.embed_rows(E.t, c.coords[:n, 1])
    ref = O.embed(E.get(), np.nonzero(mask)[1])
    assert np.array_equal(out.double().cpu().numpy(), ref)


def test_ids_far_outside_and_one_id_for_all():
    E = Rows(4, 24, "f32", values=np.arange(96).reshape(4, 24))
    big = torch.tensor([2 ** 40 + 1, -2 ** 40, 3, 2 ** 32 + 1], device="cuda")
    out = shc.embed_rows(E.t, big).cpu().numpy()
    assert not out[[0, 1, 3]].any() and np.array_equal(out[2], E.get()[3])
    one = torch.tensor([2], device="cuda").expand(9)          # stride 0
    assert np.array_equal(shc.embed_rows(E.t, one).cpu().numpy(), np.tile(E.get()[2], (9, 1)))
    dE = torch.empty((4, 24), device="cuda")
    shc.embed_rows_backward(torch.ones((4, 24), device="cuda"), big, dE)
    assert dE.sum(1).tolist() == [0, 0, 0, 24]


def test_offsets_past_32_bits():
    """A table and rows whose last element lies past 2^32 bytes and 2^31 elements."""
    R, ld = 600_000, 4096                    # 4.9 GB of bf16, 2.4e9 elements
    buf = torch.zeros((R, ld), dtype=torch.bfloat16, device="cuda")
    E = buf[:, :40]
    E[-1] = 3.0
    E[-2] = 2.0
    ids = torch.tensor([R - 1, 0, R - 2], device="cuda")
    out = shc.embed_rows(E, ids, scale=2.0)
    assert out.float().mean(1).tolist() == [6.0, 0.0, 4.0]
    # the gradient reads rows and writes a table of the same kind
    dY = buf[:, 64:104]
    dY[-1] = 1.0
    every = torch.full((R,), -1, dtype=torch.int32, device="cuda")
    every[-1] = 5
    dE = torch.empty((8, 40), device="cuda")
    shc.embed_rows_backward(dY, every, dE)
    assert dE.sum(1).tolist() == [0, 0, 0, 0, 0, 40, 0, 0]


def grad_case(r, n, R, kind):
    if kind == "uniform":
        return r.integers(0, R, n)
    if kind == "zipf":
        return np.minimum((R + 1.0) ** r.random(n) - 1, R - 1).astype(np.int64)
    if kind == "one":
        return np.full(n, R // 2)
    if kind == "runs":                       # ascending runs, as vertices come
        return np.sort(r.integers(0, R, n)) if n < 8 else np.concatenate(
            [np.sort(a) for a in np.array_split(r.integers(0, R, n), 4)])
    return r.integers(-3, R + 3, n)          # "outside"


@pytest.mark.parametrize("kind", ["uniform", "zipf", "one", "runs", "outside"])
@pytest.mark.parametrize("n", [63, 64, 65, 200, 511, 512, 513, 1024, 1025, 2047, 2048, 2049])
@pytest.mark.parametrize("C,R,dtype", [(8, 600, "f32"), (521, 3, "bf16"), (300, 70, "f32"),
                                       (1300, 900, "f32")])
def test_gradient_of_few_positions(kind, n, C, R, dtype):
    """At the border between one launch and several; rows of ids that do not count
    hold NaN."""
    r = np.random.default_rng(n + C)
    ids = grad_case(r, n, R, kind)
    pad = int(ids[0]) if kind == "zipf" else -1
    rows = r.standard_normal((n, C))
    rows[(ids < 0) | (ids >= R) | (ids == pad)] = np.nan
    dY, dE = Rows(n, C, dtype, 1, 1, rows), Rows(R, C, "f32", 2, 0)
    shc.embed_rows_backward(dY.t, ids_tensor(ids, torch.int64, 1), dE.t, pad_id=pad)
    clean = np.nan_to_num(dY.get())
    ref = O.embed_backward(clean, ids, R, 1.0, pad)
    size = O.embed_backward(np.abs(clean), ids, R, 1.0, pad)
    count = O.embed_backward(np.ones((n, 1)), ids, R, 1.0, pad)
    close(dE.get(), ref, 2 * ((count + 2) * u * size + u * np.abs(ref)), "dE")
    assert np.all(dE.get()[count[:, 0] == 0] == 0)
    dE.check_guard()


@pytest.mark.parametrize("n,R", [(400, 60), (5000, 60), (40000, 300)])
def test_gradient_in_a_graph_and_on_another_stream(n, R):
    """Each replay has ids of its own, with other ids long enough to be cut."""
    r = np.random.default_rng(n)
    C = 40
    dY = Rows(n, C, "bf16", values=r.standard_normal((n, C)))
    ids = torch.zeros(n, dtype=torch.int32, device="cuda")
    dE, want = (torch.empty((R, C), device="cuda") for _ in range(2))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        shc.embed_rows_backward(dY.t, ids, dE)
    torch.cuda.current_stream().wait_stream(side)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        shc.embed_rows_backward(dY.t, ids, dE)
    for k in range(4):
        new = grad_case(r, n, R, ("zipf", "one", "uniform", "runs")[k])
        ids.copy_(torch.as_tensor(new, dtype=torch.int32))
        shc.embed_rows_backward(dY.t, ids, want)
        torch.cuda.synchronize()
        dE.fill_(7.0)
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(dE, want), k
        ref = O.embed_backward(dY.get(), new, R, 1.0, -1)
        size = O.embed_backward(np.abs(dY.get()), new, R, 1.0, -1)
        count = O.embed_backward(np.ones((n, 1)), new, R, 1.0, -1)
        close(want.double().cpu().numpy(), ref, 2 * (count + 2) * u * size, "dE")


@pytest.mark.parametrize("n,R,C,kind", [
    (32767, 40, 12, "zipf"), (32768, 40, 12, "zipf"), (50000, 300, 20, "one"),
    (40001, 1 << 20, 3, "uniform"), (40001, (1 << 20) + 1, 3, "zipf"), (33000, 2, 131, "zipf"),
    (60000, 1500, 20, "uniform"), (60001, 1500, 70, "runs"),
])
def test_gradient_of_many_positions(n, R, C, kind):
    """Where the ordering takes more threads a bucket, and ids of thousands of
    positions."""
    r = np.random.default_rng(n + R)
    ids = grad_case(r, n, R, kind)
    dY, dE = Rows(n, C, "f32", 0, 0, r.standard_normal((n, C))), Rows(R, C, "f32", 1, 0)
    shc.embed_rows_backward(dY.t, ids_tensor(ids, torch.int32, 2), dE.t)
    first = dE.get().copy()
    ref = O.embed_backward(dY.get(), ids, R, 1.0, -1)
    size = O.embed_backward(np.abs(dY.get()), ids, R, 1.0, -1)
    count = O.embed_backward(np.ones((n, 1)), ids, R, 1.0, -1)
    close(first, ref, 2 * ((count + 2) * u * size + u * np.abs(ref)), "dE")
    shc.embed_rows_backward(dY.t, ids_tensor(ids, torch.int32, 2), dE.t)
    assert np.array_equal(dE.get(), first)      # bit for bit
    dE.check_guard()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,R,C,kind,extra,off", [
    (0, 5, 8, "uniform", 0, 0), (1, 1, 1, "uniform", 0, 0), (2, 3, 7, "outside", 1, 1),
    (31, 4, 16, "one", 0, 0), (32, 4, 17, "one", 0, 0), (33, 4, 100, "one", 3, 0),
    (1000, 37, 128, "runs", 0, 0), (4097, 10475, 64, "runs", 64, 0),
    (5000, 3, 40, "zipf", 0, 0), (9000, 100003, 24, "zipf", 0, 3),
    (700, 300, 520, "uniform", 0, 0), (513, 50, 4099, "zipf", 5, 1),
    (20000, 257, 33, "outside", 0, 0), (70000, 655, 16, "runs", 0, 0),
    (300, 1000, 16384, "zipf", 0, 0), (4000, 2000003, 4, "uniform", 0, 0),
    (530000, 700, 8, "zipf", 0, 0), (530001, 5, 3, "uniform", 0, 0),
])
@pytest.mark.parametrize("accumulate", [False, True])
def test_gradient(dtype, n, R, C, kind, extra, off, accumulate):
    r = np.random.default_rng(n + C)
    ids = grad_case(r, n, R, kind)
    pad = -1 if n % 2 else R // 3
    dY = Rows(n, C, dtype, extra, off, r.standard_normal((n, C)))
    dE = Rows(R, C, "f32", extra, off)
    prior = 0.0
    if accumulate:
        prior = stored(r.standard_normal((R, C)), "f32")
        dE.t.copy_(torch.as_tensor(prior, dtype=torch.float32))
    idt = ids_tensor(ids, torch.int32 if n % 3 else torch.int64, 2 if n % 5 == 0 else 1)
    shc.embed_rows_backward(dY.t, idt, dE.t, scale=0.3, pad_id=pad, accumulate=accumulate)
    s = float(np.float32(0.3))
    ref = O.embed_backward(dY.get(), ids, R, s, pad)
    size = O.embed_backward(np.abs(dY.get()), ids, R, s, pad)
    count = O.embed_backward(np.ones((n, 1)), ids, R, 1.0, pad)
    # any order of the sum, the factor and the addition to what was there
    bound = (count + 2) * u * size + u * np.abs(ref + prior)
    close(dE.get(), ref + prior, 2 * bound, "dE")
    # rows without an id: zero, or untouched
    left = count[:, 0] == 0
    assert np.array_equal(dE.get()[left], np.broadcast_to(prior, ref.shape)[left])
    dE.check_guard("dE")


def test_gradient_repeats_and_takes_fewer_rows():
    r = np.random.default_rng(11)
    n, R, C = 30000, 500, 96
    ids = torch.as_tensor(grad_case(r, n, R, "zipf"), device="cuda")
    dY = torch.as_tensor(r.standard_normal((n, C)), dtype=torch.float32, device="cuda")
    a, b = (torch.empty((R, C), device="cuda") for _ in range(2))
    call = shc.prepare_embed_rows_backward(dY, ids, a)
    call(n)
    first = a.clone()
    call(1234)                               # a prepared call takes any smaller count
    shc.embed_rows_backward(dY[:1234], ids[:1234], b)
    assert torch.equal(a, b)
    call(n)
    assert torch.equal(a, first)


def test_gradient_of_fewer_rows_than_prepared():
    """A prepared call's workspace serves smaller counts, also those that are cut
    into shorter jobs (262,144 rows of 64 channels) or narrower chunks (524,288)."""
    r = np.random.default_rng(2)
    n, R, C = 530000, 300, 64
    ids = torch.as_tensor(r.integers(0, R, n), dtype=torch.int32, device="cuda")
    dY = torch.as_tensor(r.integers(-3, 4, (n, C)), dtype=torch.float32, device="cuda")
    dE = torch.empty((R, C), device="cuda")
    call = shc.prepare_embed_rows_backward(dY, ids, dE)
    for m in (n, 524287, 262143, 3000, 17, 1):
        call(m)
        want = torch.zeros((R, C), device="cuda").index_add_(0, ids[:m].long(), dY[:m])
        assert torch.equal(dE, want)         # whole numbers below 2^24: exact


def test_gradient_of_a_table_past_32_bit_offsets():
    R, ld = 270_000, 16000                   # 4.3e9 fp32 elements, 17 GB
    buf = torch.full((R, ld), 1.0, dtype=torch.float32, device="cuda")
    dE = buf[:, :20]
    ids = torch.tensor([R - 1, 7, R - 1], dtype=torch.int32, device="cuda")
    shc.embed_rows_backward(torch.ones((3, 20), device="cuda"), ids, dE)
    assert dE[-1].tolist() == [2.0] * 20 and dE[7].tolist() == [1.0] * 20
    assert float(dE.sum()) == 60.0 and float(buf[-1, 20]) == 1.0


def test_gradient_matches_differences():
    """The gradient against differences of the forward, both by the kernels: the
    forward is linear in E, so a whole step is exact up to rounding."""
    r = np.random.default_rng(5)
    E = torch.as_tensor(r.integers(-8, 8, (6, 4)), dtype=torch.float32, device="cuda")
    dY = torch.as_tensor(r.integers(-8, 8, (40, 4)), dtype=torch.float32, device="cuda")
    ids = torch.as_tensor(r.integers(0, 6, 40), device="cuda")
    dE = torch.empty_like(E)
    shc.embed_rows_backward(dY, ids, dE, scale=2.0)
    base = float((shc.embed_rows(E, ids, scale=2.0) * dY).sum())
    for i in range(6):
        for c in range(4):
            E[i, c] += 1
            up = float((shc.embed_rows(E, ids, scale=2.0) * dY).sum())
            E[i, c] -= 1
            assert up - base == float(dE[i, c])
