"""The row operators together: other streams, graph replays, refusals of the
binding."""
import numpy as np
import pytest
import torch

from paper_2608_09388_amd import binding as shc
from tests.gpu_util import require_gpu

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def dev():
    return require_gpu()


class Step:
    """Embedding, norm and distillation with their gradients on fixed buffers."""

    def __init__(self, n=2000, R=700, C=96, V=5000, k=6, seed=0):
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)

        def rand(*s, dtype=torch.bfloat16):
            return torch.randn(s, generator=g, device="cuda").to(dtype)

        f32 = torch.float32
        self.n = n
        self.E, self.ids = rand(R, C), torch.randint(0, R, (n,), generator=g, device="cuda")
        self.gamma, self.beta = rand(C, dtype=f32), rand(C, dtype=f32)
        self.z, self.dyn = rand(n, V), rand(n, C)
        self.top_ids = torch.randint(0, V, (n, k), generator=g, device="cuda", dtype=torch.int32)
        self.top = rand(n, k, dtype=f32)
        e = torch.empty
        kw = dict(device="cuda")
        self.h, self.y, self.dx = (e((n, C), dtype=torch.bfloat16, **kw) for _ in range(3))
        self.mean, self.rstd, self.loss, self.lse, self.loss2 = (e(n, **kw) for _ in range(5))
        self.dg, self.db, self.dE = e(C, **kw), e(C, **kw), e((R, C), **kw)
        self.dz, self.dz2 = (e((n, V), dtype=torch.bfloat16, **kw) for _ in range(2))

    def run(self, stream=None):
        s = self
        shc.embed_rows(s.E, s.ids, s.h, scale=2.0, stream=stream)
        shc.layer_norm(s.h, s.gamma, s.beta, s.y, s.mean, s.rstd, stream=stream)
        shc.distill_top_step(s.z, s.top_ids, s.top, None, s.loss, s.dz, stream=stream)
        shc.distill_top(s.z[:20], s.top_ids, s.top, s.loss2[:20], s.lse[:20], stream=stream)
        shc.distill_top_backward(s.z[:20], s.top_ids, s.top, s.lse[:20], None, s.dz2[:20],
                                 stream=stream)
        shc.layer_norm_backward(s.dyn, s.h, s.gamma, s.mean, s.rstd, s.dx, s.dg, s.db,
                                stream=stream)
        shc.embed_rows_backward(s.dx, s.ids, s.dE, scale=2.0, stream=stream)

    def outs(self):
        return (self.h, self.y, self.mean, self.rstd, self.loss, self.dz, self.loss2[:20],
                self.lse[:20], self.dz2[:20], self.dx, self.dg, self.db, self.dE)


def test_another_stream():
    a, b = Step(), Step()
    a.run()
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    b.run(stream=s)
    torch.cuda.current_stream().wait_stream(s)
    for x, y in zip(a.outs(), b.outs()):
        assert torch.equal(x, y)
    # a raw handle, and the stream made current
    b.dE.zero_()
    s.wait_stream(torch.cuda.current_stream())
    b.run(stream=s.cuda_stream)
    s.synchronize()
    assert torch.equal(a.dE, b.dE)
    with torch.cuda.stream(s):
        b.run()
    s.synchronize()
    assert torch.equal(a.dE, b.dE)


def test_graph_replays():
    st = Step(seed=3)
    st.run()
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        st.run()
    torch.cuda.current_stream().wait_stream(s)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        st.run()
    for k in range(4):
        other = Step(seed=10 + k)
        for name in ("E", "ids", "z", "top_ids", "top", "dyn", "gamma", "beta"):
            getattr(st, name).copy_(getattr(other, name))
        other.run()
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        for x, y in zip(st.outs(), other.outs()):
            assert torch.equal(x, y)


def test_refusals_of_the_binding():
    f = dict(device="cuda")
    E, x = torch.zeros((8, 32), **f), torch.zeros((4, 32), **f)
    ids = torch.zeros(4, dtype=torch.int64, **f)
    ok = shc.embed_rows(E, ids)
    assert ok.shape == (4, 32)
    with pytest.raises(TypeError, match="ids must be int32 or int64"):
        shc.embed_rows(E, ids.float())
    with pytest.raises(ValueError, match="on the GPU"):
        shc.embed_rows(E.cpu(), ids)
    with pytest.raises(TypeError, match="float32 or bfloat16"):
        shc.embed_rows(E.half(), ids)
    with pytest.raises(TypeError, match="out must be"):
        shc.embed_rows(E, ids, out=torch.zeros((4, 32), dtype=torch.bfloat16, **f))
    with pytest.raises(ValueError, match="rows of 16"):
        shc.embed_rows(E, ids, out=torch.zeros((4, 16), **f))
    with pytest.raises(ValueError, match="n_rows = 4"):
        shc.embed_rows(E, ids, out=torch.zeros((3, 32), **f))
    with pytest.raises(ValueError, match="adjacent"):
        shc.layer_norm(torch.zeros((32, 4), **f).t())
    with pytest.raises(ValueError, match="overlap"):
        shc.layer_norm(torch.zeros(1, 32, **f).expand(4, 32), y=x)
    with pytest.raises(ValueError, match="gamma holds 16"):
        shc.layer_norm(x, torch.ones(16, **f))
    with pytest.raises(TypeError, match="gamma must be"):
        shc.layer_norm(x, torch.ones(32, dtype=torch.bfloat16, **f))
    with pytest.raises(ValueError, match="n_rows = 4"):
        shc.layer_norm_backward(x, x[:2], None, ids[:2].float(), ids[:2].float(), dx=x)
    with pytest.raises(shc.ShcError, match="exceeds 16384"):
        shc.layer_norm(torch.zeros((1, 16400), **f))
    with pytest.raises(shc.ShcError, match="eps"):
        shc.layer_norm(x, eps=0.0)
    with pytest.raises(ValueError, match="ws holds"):
        shc.embed_rows_backward(x, ids, E, ws=torch.zeros(16, dtype=torch.uint8, **f))
    ti, tl = torch.zeros((4, 3), dtype=torch.int32, **f), torch.zeros((4, 3), **f)
    with pytest.raises(ValueError, match="alike"):
        shc.distill_top(x, ti, tl[:, :2])
    with pytest.raises(TypeError, match="top_ids must be"):
        shc.distill_top(x, ti.long(), tl)
    with pytest.raises(shc.ShcError, match="temperature"):
        shc.distill_top(x, ti, tl, temperature=0.0)
    with pytest.raises(shc.ShcError, match="k = 300 exceeds 256"):
        shc.distill_top(x, torch.zeros((4, 300), dtype=torch.int32, **f), torch.zeros((4, 300), **f))
    with pytest.raises(ValueError, match="loss holds 3"):
        shc.distill_top(x, ti, tl, loss=torch.zeros(3, **f))
