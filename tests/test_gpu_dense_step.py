"""The dense operators run together as a training step does: streams, captured graphs
(two that share a workspace among them), padded batches."""
import pytest
import torch

from paper_2608_09388_amd import binding as shc
from tests.gpu_util import require_gpu

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def dev():
    return require_gpu()


class Step:
    """x -> GELU layer -> layer with residual -> cross entropy, all gradients, their norm and
    clipping, every buffer made once."""

    def __init__(self, seed=0, dtype=torch.bfloat16, n=260, C=136, H=272, V=1000, ws=None):
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)

        def rnd(*s, dt=dtype, scale=1.0):
            return (torch.randn(s, generator=g, device="cuda") * scale).to(dt)

        def new(*s, dt=dtype):
            return torch.zeros(s, dtype=dt, device="cuda")

        f32 = torch.float32
        self.n, self.x = n, rnd(n, C)
        self.W1, self.b1 = rnd(C, H, scale=C ** -0.5), rnd(H, dt=f32, scale=0.1)
        self.W2, self.b2 = rnd(H, C, scale=H ** -0.5), rnd(C, dt=f32, scale=0.1)
        self.E = rnd(V, C, scale=C ** -0.5)
        self.labels = torch.randint(-V // 3, V, (n,), generator=g, device="cuda")
        self.w = torch.rand(n, generator=g, device="cuda") / n
        self.pre, self.h, self.y = new(n, H), new(n, H), new(n, C)
        self.dy, self.dh, self.dx = new(n, C), new(n, H), new(n, C)
        self.loss = new(n, dt=f32)
        self.g = dict(W1=new(C, H), b1=new(H, dt=f32), W2=new(H, C), b2=new(C, dt=f32),
                      E=new(V, C))
        self.norm = new(1, dt=f32)
        self.ws = ws if ws is not None else torch.empty(64 << 20, dtype=torch.uint8, device="cuda")

    def run(self, stream=None):
        k, g = dict(ws=self.ws, stream=stream), self.g
        shc.linear(self.x, self.W1, self.b1, self.h, shc.SHC_ACT_GELU, None, self.pre, **k)
        shc.linear(self.h, self.W2, self.b2, self.y, shc.SHC_ACT_NONE, self.x, **k)
        shc.linear_cross_entropy_step(self.y, self.E, self.labels, self.w, None, self.loss, self.dy,
                                      g["E"], **k)
        shc.linear_backward(self.dy, self.h, self.W2, None, self.dh, g["W2"], g["b2"], **k)
        shc.linear_backward(self.dh, self.x, self.W1, self.pre, self.dx, g["W1"], g["b1"],
                            shc.SHC_ACT_GELU, **k)
        shc.grad_norm(g.values(), self.norm, **k)
        shc.clip_grads(g.values(), self.norm, 0.01, stream=stream)

    def outs(self):
        return [self.h, self.y, self.loss, self.dy, self.dh, self.dx, self.norm, *self.g.values()]

    def inputs(self):
        return [self.x, self.W1, self.b1, self.W2, self.b2, self.E, self.labels, self.w]


def check_against_autograd(st):
    """Norms of the differences against autograd in 64 bits: roundings to the type of the
    tensors between the operators (h, y, dy, dh, about ten of them in a chain) and of dz."""
    F = torch.nn.functional
    p = {k: getattr(st, k).double().requires_grad_() for k in ("x", "W1", "b1", "W2", "b2", "E")}
    y = F.gelu(p["x"] @ p["W1"] + p["b1"]) @ p["W2"] + p["b2"] + p["x"]
    labels = torch.where(st.labels < 0, -100, st.labels)
    loss = F.cross_entropy(y @ p["E"].t(), labels, reduction="none")
    (loss * st.w).sum().backward()
    tol = 16 * (2.0 ** -8 if st.x.dtype == torch.bfloat16 else 2.0 ** -20)
    norm = torch.sqrt(sum((p[k].grad ** 2).sum() for k in st.g))
    assert abs(float(st.norm) / float(norm) - 1.0) < tol
    factor = min(1.0, 0.01 / float(norm))
    for k, got in st.g.items():
        ref = p[k].grad * factor
        assert float((got - ref).norm() / ref.norm()) < tol, k
    live = st.labels >= 0
    loss = loss.detach()
    assert float((st.loss - loss)[live].norm() / loss[live].norm()) < tol
    assert not bool(st.loss[~live].any()) and not bool(st.dy[~live].any())


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_step(dtype):
    st = Step(1, dtype)
    st.run()
    check_against_autograd(st)


def test_streams():
    a, b = Step(), Step()
    a.run()
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    b.run(stream=s)
    torch.cuda.current_stream().wait_stream(s)
    assert all(torch.equal(x, y) for x, y in zip(a.outs(), b.outs()))
    for t in b.outs():
        t.zero_()
    s.wait_stream(torch.cuda.current_stream())
    b.run(stream=s.cuda_stream)
    s.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(a.outs(), b.outs()))


def test_workspaces_made_by_the_calls():
    a, b = Step(4), Step(4)
    a.run()
    b.ws = None
    b.run()
    assert all(torch.equal(x, y) for x, y in zip(a.outs(), b.outs()))


def capture(st):
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        st.run()
    torch.cuda.current_stream().wait_stream(s)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        st.run()
    return g


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_graph_replays(dtype):
    """Replays with other inputs, other labels of padding among them, eager work between."""
    st = Step(3, dtype)
    st.run()
    torch.cuda.synchronize()
    g = capture(st)
    for k in range(4):
        other = Step(10 + k, dtype)
        if k == 2:
            other.labels.fill_(-1)        # nothing but padding
        if k == 3:
            other.labels.abs_()           # no padding
        for a, b in zip(st.inputs(), other.inputs()):
            a.copy_(b)
        other.run()
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        for x, y in zip(st.outs(), other.outs()):
            assert torch.equal(x, y) or (k == 2 and bool(torch.isnan(x).all()))


def test_two_graphs_share_a_workspace():
    a = Step(5)
    b = Step(6, n=77, C=72, H=40, V=333, ws=a.ws)
    a.run(), b.run()
    torch.cuda.synchronize()
    want = [[t.clone() for t in st.outs()] for st in (a, b)]
    ga, gb = capture(a), capture(b)
    for order in ((ga, gb), (gb, ga), (ga, ga, gb)):
        for st in (a, b):
            for t in st.outs():
                t.zero_()
        for g in order:
            g.replay()
        torch.cuda.synchronize()
        for st, ref in zip((a, b), want):
            assert all(torch.equal(x, y) for x, y in zip(st.outs(), ref))


def test_refusals_of_the_binding():
    f = dict(device="cuda")
    x, W = torch.zeros((4, 32), **f), torch.zeros((32, 8), **f)
    E = torch.zeros((10, 32), **f)
    ids = torch.zeros(4, dtype=torch.int64, **f)
    with pytest.raises(ValueError, match="W has 10 rows"):
        shc.linear(x, E)
    with pytest.raises(TypeError, match="W must be"):
        shc.linear(x, W.bfloat16())
    with pytest.raises(ValueError, match="residual has rows of 32"):
        shc.linear(x, W, residual=x)
    with pytest.raises(ValueError, match="n_rows = 4"):
        shc.linear(x, W, out=torch.zeros((3, 8), **f))
    with pytest.raises(ValueError, match="bias holds 4"):
        shc.linear(x, W, bias=torch.zeros(4, **f))
    with pytest.raises(ValueError, match="adjacent"):
        shc.linear(x, torch.zeros((8, 32), **f).t())
    with pytest.raises(shc.ShcError, match="activation"):
        shc.linear(x, W, act=7)
    with pytest.raises(shc.ShcError, match="pre is NULL"):
        shc.linear_backward(x[:, :8].contiguous(), x, W, act=shc.SHC_ACT_GELU, dx=x)
    with pytest.raises(ValueError, match="dW has 10 rows"):
        shc.linear_backward(torch.zeros((4, 8), **f), x, W, dW=torch.zeros((10, 8), **f))
    with pytest.raises(ValueError, match="ws holds"):
        shc.linear(x, W, ws=torch.zeros(16, dtype=torch.uint8, **f))
    with pytest.raises(ValueError, match="W has rows of 8"):
        shc.linear_cross_entropy(x, W, ids)
    with pytest.raises(TypeError, match="labels must be int32 or int64"):
        shc.linear_cross_entropy(x, E, ids.float())
    with pytest.raises(ValueError, match="n_rows = 4"):
        shc.linear_cross_entropy(x, E, ids[:3])
    with pytest.raises(ValueError, match="loss holds 3"):
        shc.linear_cross_entropy(x, E, ids, loss=torch.zeros(3, **f))
    with pytest.raises(ValueError, match="db holds 9"):
        shc.linear_cross_entropy_step(x, E, ids, db=torch.zeros(9, **f))
    with pytest.raises(ValueError, match="on the GPU"):
        shc.linear_cross_entropy(x, E, ids.cpu())
    # the sparse layers know no more than they did
    S = torch.zeros((4, 16), **f)
    with pytest.raises(shc.ShcError, match="act"):
        shc.sparse_linear(S, 4, torch.zeros((16, 16), **f), None, torch.zeros((4, 16), **f),
                          shc.SHC_ACT_GELU)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_rows_beyond_four_gigabytes(dtype):
    """Every row tensor with its rows so far apart that offsets pass 32 bits gives what adjacent
    rows give, bit for bit."""
    t = {"f32": torch.float32, "bf16": torch.bfloat16}[dtype]
    n, C, N, far = 2300, 72, 88, (1 << 20) - 8
    g = torch.Generator(device="cuda")
    g.manual_seed(5)

    def near(rows, width):
        return torch.randn((rows, width), generator=g, device="cuda").to(t)

    buf = torch.empty(n * far, dtype=t, device="cuda")
    used = [0]

    def apart(values):
        """The values in columns of the buffer that no other tensor has."""
        rows, width = values.shape
        view = torch.as_strided(buf, (rows, width), (far, 1), used[0])
        used[0] += 256
        view.copy_(values)
        return view

    x, W, dout, pre = near(n, C), near(C, N), near(n, N), near(n, N)
    table, labels = near(n, C), torch.randint(-3, n, (n,), generator=g, device="cuda")

    def run(place):
        X, T = place(x), place(table)
        out, kept = place(torch.zeros_like(dout)), place(torch.zeros_like(dout))
        dx, dW = place(torch.zeros_like(x)), place(torch.zeros_like(W))
        res = place(dout)
        shc.linear(X, place(W), out=out, act=shc.SHC_ACT_GELU, residual=res, pre=kept)
        shc.linear_backward(res, X, place(W), place(pre), dx, dW, act=shc.SHC_ACT_SILU)
        ex, eT = place(torch.zeros_like(x)), place(torch.zeros_like(table))
        loss = shc.linear_cross_entropy_step(X, T, labels, dx=ex, dW=eT)
        return [r.clone() for r in (out, kept, dx, dW, loss, ex, eT)]

    for a, b in zip(run(lambda v: v.clone()), run(apart)):
        assert torch.equal(a, b)
