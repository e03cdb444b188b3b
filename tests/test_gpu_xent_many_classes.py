"""The cross entropy's gradients over so many classes that dz's rows are gigabytes from a tile's
first to its last, against sums over chunks of classes in 64 bits."""
import pytest
import torch

from paper_2608_09388_amd import binding as shc
from tests.gpu_util import require_gpu

pytestmark = pytest.mark.gpu

CHUNK = 1 << 17


@pytest.fixture(scope="module", autouse=True)
def dev():
    yield require_gpu()
    torch.cuda.empty_cache()


def reference(x, W, labels):
    """dict of loss, dx, what the norms of dx's terms add up to, and the largest error of an
    fp32 logit: a chunk of classes at a time."""
    n, C = x.shape
    V = W.shape[0]
    x = x.double()
    top, total = torch.full((n,), -1e300, dtype=torch.float64, device="cuda"), 0.0
    at, off = torch.zeros(n, dtype=torch.float64, device="cuda"), 0.0
    rows = torch.arange(n, device="cuda")

    def chunks():
        for v in range(0, V, CHUNK):
            w = W[v:v + CHUNK].double()
            yield v, w, x @ w.t().contiguous()

    for v, w, z in chunks():
        m = torch.maximum(top, z.amax(1))
        total = total * torch.exp(top - m) + torch.exp(z - m[:, None]).sum(1)
        top = m
        mine = (labels >= v) & (labels < v + len(w))
        at[mine] = z[rows[mine], labels[mine] - v]
        off = max(off, float((x.abs() @ w.abs().t().contiguous()).max()))
    lse = top + torch.log(total)
    dx, size = torch.zeros_like(x), torch.zeros(n, dtype=torch.float64, device="cuda")
    for v, w, z in chunks():
        dz = torch.exp(z - lse[:, None])
        mine = (labels >= v) & (labels < v + len(w))
        dz[rows[mine], labels[mine] - v] -= 1.0
        dx += dz @ w
        size += dz.abs() @ w.norm(dim=1)
        if v + len(w) == V:
            tail = dz.t().contiguous() @ x, dz.abs().t().contiguous() @ x.norm(dim=1)
    return dict(loss=lse - at, dx=dx, size=size, off=(C + 16) * 2.0 ** -24 * off + 2.0 ** -18,
                tail=tail)


@pytest.mark.parametrize("n,C,V,dtype", [
    (256, 1024, 4500008, "bf16"),   # past what a tile of 256 rows reaches
    (64, 1024, 8500000, "bf16"),    # two terms: 128 rows
    (200, 256, 8500003, "f32"),
    (64, 72, 1 << 24, "bf16"),      # the most classes
    (300, 40, (1 << 24) - 1, "bf16"),
])
def test_gradients(n, C, V, dtype):
    """In the 2-norm of a row.  h is half a step of the type (bf16 2^-8; fp32's is in `sums`): a
    gradient is off by h of itself, by h of its terms for dz's rounding, by 2^-11 for exponentials
    kept in fp16, by twice a logit's error for its probabilities, and by its sums: a matrix
    instruction adds 16 products, so that V / 16 and some more additions of 2^-24 follow each
    other, in fp32 six times as many."""
    g = torch.Generator(device="cuda")
    g.manual_seed(n)
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    x = torch.randn((n, C), generator=g, device="cuda").to(dt)
    W = torch.empty((V, C), dtype=dt, device="cuda")
    W.normal_(generator=g).mul_(2.0 * C ** -0.5)
    labels = torch.randint(0, V, (n,), generator=g, device="cuda")
    labels[-2:] = V - 1
    ref = reference(x, W, labels)
    h = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -24
    terms = h + 2.0 ** -11 + 2 * ref["off"]
    sums = (6 if dtype == "f32" else 1) * (V / 16 + 100) * 2.0 ** -24
    ws = torch.empty(shc.linear_cross_entropy_workspace(
        n, C, V, shc.SHC_BF16 if dtype == "bf16" else shc.SHC_F32), dtype=torch.uint8,
        device="cuda")
    lse = torch.empty(n, device="cuda")
    for step in (True, False):
        dx, dW = torch.full_like(x, 7.0), torch.empty_like(W)
        if step:
            loss = shc.linear_cross_entropy_step(x, W, labels, dx=dx, dW=dW, ws=ws)
        else:
            loss = shc.linear_cross_entropy(x, W, labels, lse=lse, ws=ws)
            shc.linear_cross_entropy_backward(x, W, labels, lse, dx=dx, dW=dW, ws=ws)
        assert float((loss - ref["loss"]).abs().max()) <= 4 * ref["off"] + 1e-4
        err = (dx.double() - ref["dx"]).norm(dim=1)
        bound = h * ref["dx"].norm(dim=1) + (terms + sums) * ref["size"]
        assert bool((bound < 0.5 * ref["dx"].norm(dim=1)).all())  # a row that is lost is seen
        assert bool((err <= bound).all()), (step, torch.nonzero(err > bound)[:, 0].tolist())
        rW, size = ref["tail"]
        err = (dW[V - len(rW):].double() - rW).norm(dim=1)
        assert bool((err <= h * rW.norm(dim=1) + (terms + 2.0 ** -14) * size + 1e-12).all()), step
