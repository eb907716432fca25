"""Layer norm and its gradients against the definition in 64 bits.

Tolerances.  u = 2^-24 is fp32's half step.  A sum over a row is made of at most 16 (20 beyond 16384 columns) additions per lane, 6 exchanges and 16
wavefronts' parts, so it is off by at most 48 u times the sum of magnitudes; with the roundings around it, K = 64 covers each of mean, variance,
mean(g) and mean(g h).  With E = rstd (mean |x| + |x|) + |h| a normalised element is off by at most K u E, which goes on into everything made of it.
Outputs are rounded once: half a step of their type, or of its subnormals."""
import numpy as np
import pytest
import torch

import paper_2403_14853_amd as isp
from paper_2403_14853_amd import autograd as ag

pytestmark = pytest.mark.gpu

K = 64 * 2.0 ** -24
TYPES = [torch.float32, torch.bfloat16, torch.float16]
WIDTHS = [1, 2, 3, 4, 5, 7, 8, 9, 16, 31, 32, 47, 64, 100, 128, 250, 256, 257, 500, 512, 602, 1000, 1024, 1025, 2047, 2048, 4096, 4097, 8192, 8200, 16384,
          16385, 20000]


def half_step(ref, dtype):
    info = torch.finfo(dtype)
    return ref.abs() * (info.eps / 2) + info.smallest_normal * info.eps / 2


def reference(x, w, b, dy, eps=1e-5):
    """Values in 64 bits and the bounds above, as (name: (value, bound before the last rounding))."""
    x, w, b, dy = (t.detach().double().cpu() for t in (x, w, b, dy))
    mean = x.mean(1, keepdim=True)
    rstd = ((x - mean).square().mean(1, keepdim=True) + eps).rsqrt()
    h = (x - mean) * rstd
    E = rstd * (x.abs().mean(1, keepdim=True) + x.abs()) + h.abs()
    g = dy * w
    s1, s2 = g.mean(1, keepdim=True), (g * h).mean(1, keepdim=True)
    a1, a2 = g.abs().mean(1, keepdim=True), (g * h).abs().mean(1, keepdim=True)
    dx = rstd * (g - s1 - h * s2)
    dx_err = rstd * (g.abs() + a1 + h.abs() * (a2 + (g.abs() * E).mean(1, keepdim=True)) + E * a2) + dx.abs()
    return {"y": (h * w + b, K * (E * w.abs() + b.abs())), "mean": (mean[:, 0], K * x.abs().mean(1)),
            "rstd": (rstd[:, 0], K * rstd[:, 0] * (1 + (E * h.abs()).mean(1))), "dx": (dx, K * dx_err),
            "dw": ((dy * h).sum(0), K * (dy.abs() * E).sum(0)), "db": (dy.sum(0), K * dy.abs().sum(0))}


def check(got, ref, name):
    value, bound = ref[name]
    g = got.detach().double().cpu()
    assert g.shape == value.shape and torch.isfinite(g).all(), name
    over = ((g - value).abs() / (bound + half_step(value, got.dtype) * 1.001)).max() if g.numel() else torch.tensor(0.0)
    assert over <= 1, "%s: %.3g of the tolerance" % (name, over)


def make(n, d, dtype, ptype, seed=0, ld=None, offset=0):
    gen = torch.Generator().manual_seed(1000 * d + n + seed)
    ld = ld or d
    def rows(std, off):
        full = torch.empty(offset + n * ld, dtype=dtype, device="cuda")
        t = full[offset:].view(n, ld)[:, :d] if n else full[:0].view(0, d)
        t.copy_((torch.randn(n, d, generator=gen) * std + off).to(dtype))
        return t
    x = rows(1.5, 0.7)
    dy = rows(1.0, 0.0)
    w = (1 + 0.3 * torch.randn(d, generator=gen)).to(ptype).cuda()
    b = (0.2 * torch.randn(d, generator=gen)).to(ptype).cuda()
    return x, w, b, dy


def run(x, w, b, dy, y=None, dx=None):
    n, d = x.shape
    y = torch.empty(n, d, dtype=x.dtype, device="cuda") if y is None else y
    dx = torch.empty(n, d, dtype=x.dtype, device="cuda") if dx is None else dx
    mean, rstd = (torch.empty(n, device="cuda") for _ in range(2))
    dw, db = torch.empty_like(w), torch.empty_like(b)
    isp.layer_norm(x, y, w, b, mean=mean, rstd=rstd)
    isp.layer_norm_backward(x, dy, dx, mean, rstd, w, dw, db)
    return {"y": y, "mean": mean, "rstd": rstd, "dx": dx, "dw": dw, "db": db}


@pytest.mark.parametrize("dtype", TYPES, ids=lambda t: str(t)[6:])
@pytest.mark.parametrize("d", WIDTHS)
def test_every_width(d, dtype):
    for n, ptype in ((1, torch.float32), (37, dtype), (300 if d < 5000 else 70, torch.float32)):
        x, w, b, dy = make(n, d, dtype, ptype)
        got, ref = run(x, w, b, dy), reference(x, w, b, dy)
        for name, t in got.items():
            check(t, ref, name)


@pytest.mark.parametrize("dtype", TYPES, ids=lambda t: str(t)[6:])
@pytest.mark.parametrize("d,n", [(6, 70_003), (47, 40_001), (128, 20_011), (1100, 3_001), (5000, 700)])
def test_more_rows_than_one_round(d, n, dtype):
    """Workgroups that pass over several rows, and sums of several rounds."""
    x, w, b, dy = make(n, d, dtype, torch.float32)
    got, ref = run(x, w, b, dy), reference(x, w, b, dy)
    for name, t in got.items():
        check(t, ref, name)


@pytest.mark.parametrize("dtype", TYPES, ids=lambda t: str(t)[6:])
@pytest.mark.parametrize("d", [3, 8, 47, 128, 602, 1500])
def test_leading_dimensions_and_odd_addresses(d, dtype):
    """Operands with gaps between rows that start at any element; what lies in the gaps stays."""
    n = 29
    x, w, b, dy = make(n, d, dtype, torch.float32, ld=d + 5, offset=3)
    full = torch.full((2, 1 + n * (d + 3)), 7.0, dtype=dtype, device="cuda")
    y, dx = (f[1:].view(n, d + 3)[:, :d] for f in full)
    got, ref = run(x, w, b, dy, y, dx), reference(x, w, b, dy)
    for name, t in got.items():
        check(t, ref, name)
    assert (full[:, 0] == 7).all() and all((f[1:].view(n, d + 3)[:, d:] == 7).all() for f in full)


def test_large_offsets_and_scales():
    """Rows far from zero (the centred squares, not a difference of sums), and constant rows (eps alone is left)."""
    x, w, b, dy = make(50, 300, torch.float32, torch.float32)
    x[:10] += 1000
    x[10:20] *= 1e-4
    x[20:25] = 3.0
    x[25] = 0
    got, ref = run(x, w, b, dy), reference(x, w, b, dy)
    for name, t in got.items():
        check(t, ref, name)


def test_optional_operands():
    x, w, b, dy = make(33, 96, torch.float32, torch.float32)
    one, zero = torch.ones_like(w), torch.zeros_like(b)
    ref = reference(x, one, zero, dy)
    y = isp.layer_norm(x, torch.empty_like(x))
    check(y, ref, "y")
    assert torch.equal(isp.layer_norm(x, torch.empty_like(x), one, zero), y)
    mean, rstd = (torch.empty(33, device="cuda") for _ in range(2))
    isp.layer_norm(x, y, mean=mean, rstd=rstd)
    dx, dw, db = torch.empty_like(x), torch.empty_like(w), torch.empty_like(b)
    isp.layer_norm_backward(x, dy, dx, mean, rstd)
    check(dx, ref, "dx")
    assert isp.layer_norm_backward(x, dy, None, mean, rstd, None, dw) is None
    check(dw, ref, "dw")
    isp.layer_norm_backward(x, dy, None, mean, rstd, None, None, db)
    check(db, ref, "db")


@pytest.mark.parametrize("d", [40, 2000, 17000])
def test_no_rows(d):
    x = torch.empty(0, d, device="cuda")
    none = torch.empty(0, device="cuda")
    dw, db = torch.full((d,), 3.0, device="cuda"), torch.full((d,), 3.0, device="cuda")
    isp.layer_norm(x, torch.empty_like(x), dw, db, mean=none, rstd=none)
    isp.layer_norm_backward(x, x, torch.empty_like(x), none, none, dw.clone(), dw, db)
    assert (dw == 0).all() and (db == 0).all()


def test_nan_stays_in_its_row():
    x, w, b, dy = make(64, 100, torch.float32, torch.float32)
    x[7, 3], x[9, 99] = float("nan"), float("inf")
    y = isp.layer_norm(x, torch.empty_like(x), w, b)
    bad = torch.isnan(y).any(1).cpu()
    assert bad[7] and bad[9] and int(bad.sum()) == 2


def test_repeats_bit_for_bit():
    x, w, b, dy = make(30_000, 120, torch.bfloat16, torch.float32)
    first = run(x, w, b, dy)
    for _ in range(3):
        for name, t in run(x, w, b, dy).items():
            assert torch.equal(t, first[name]), name


@pytest.mark.parametrize("dtype", TYPES, ids=lambda t: str(t)[6:])
def test_autograd(dtype):
    for d, ptype in ((48, torch.float32), (1300, dtype)):
        x, w, b, dy = make(211, d, dtype, ptype)
        ref = reference(x, w, b, dy)
        leaves = [t.clone().requires_grad_(True) for t in (x, w, b)]
        y = ag.layer_norm(*leaves)
        check(y, ref, "y")
        for name, t in zip(("dx", "dw", "db"), torch.autograd.grad(y, leaves, dy, retain_graph=True)):
            check(t, ref, name)
        for i, name in enumerate(("dx", "dw", "db")):  # one gradient wanted alone
            only = [t.detach().requires_grad_(i == j) for j, t in enumerate(leaves)]
            check(torch.autograd.grad(ag.layer_norm(*only), only[i], dy)[0], ref, name)
        y.sum().backward()  # (an upstream gradient of stride 0)
        check(leaves[2].grad, reference(x, w, b, torch.ones_like(dy)), "db")
        strided = x.t().contiguous().t().detach().requires_grad_(True)
        y = ag.layer_norm(strided, w, b)
        check(torch.autograd.grad(y, strided, dy)[0], ref, "dx")
    with pytest.raises(RuntimeError):
        y.backward(dy)  # (what the node kept is gone)


def test_gradient_against_differences():
    """Central differences of the forward's definition in 64 bits, in random directions."""
    x, w, b, dy = make(5, 24, torch.float32, torch.float32)
    got = run(x, w, b, dy)
    X, W, B, G = (t.double().cpu() for t in (x, w, b, dy))
    f = lambda X, W, B: (torch.nn.functional.layer_norm(X, (24,), W, B, 1e-5) * G).sum()
    gen = torch.Generator().manual_seed(5)
    for i, name in enumerate(("dx", "dw", "db")):
        args = [X, W, B]
        v = torch.randn(args[i].shape, generator=gen, dtype=torch.float64)
        up, down = list(args), list(args)
        up[i], down[i] = args[i] + 1e-5 * v, args[i] - 1e-5 * v
        num = (f(*up) - f(*down)) / 2e-5
        assert abs(num - (got[name].double().cpu() * v).sum()) < 1e-4 * (1 + abs(num))


def test_captured_and_replayed():
    x, w, b, dy = make(900, 70, torch.bfloat16, torch.float32)
    y, dx = torch.empty_like(x), torch.empty_like(x)
    mean, rstd = (torch.empty(900, device="cuda") for _ in range(2))
    dw, db = torch.empty_like(w), torch.empty_like(b)
    ws = torch.empty(isp.layer_norm_backward_workspace(900, 70), dtype=torch.uint8, device="cuda")

    def step():
        isp.layer_norm(x, y, w, b, mean=mean, rstd=rstd)
        isp.layer_norm_backward(x, dy, dx, mean, rstd, w, dw, db, workspace=ws)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for seed in range(3):
        nx, _, _, ndy = make(900, 70, torch.bfloat16, torch.float32, seed=seed)
        x.copy_(nx)
        dy.copy_(ndy)
        graph.replay()
        torch.cuda.synchronize()
        want = run(nx, w, b, ndy)
        for t, name in ((y, "y"), (dx, "dx"), (dw, "dw"), (db, "db")):
            assert torch.equal(t, want[name]), name


def test_on_another_stream():
    x, w, b, dy = make(5000, 256, torch.float32, torch.float32)
    want = run(x, w, b, dy)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    outs = [torch.empty_like(x), torch.empty_like(x), torch.empty(5000, device="cuda"), torch.empty(5000, device="cuda"), torch.empty_like(w), torch.empty_like(b)]
    torch.cuda.synchronize()
    isp.layer_norm(x, outs[0], w, b, mean=outs[2], rstd=outs[3], stream=side)
    isp.layer_norm_backward(x, dy, outs[1], outs[2], outs[3], w, outs[4], outs[5], stream=side)
    side.synchronize()
    for t, name in zip(outs, ("y", "dx", "mean", "rstd", "dw", "db")):
        assert torch.equal(t, want[name]), name


def test_recorded_by_jit_trace():
    """With weights that are parameters of the traced module (a recording takes no other tensors that require gradients)."""
    x, w, b, dy = make(40, 64, torch.float32, torch.float32)

    class Layer(torch.nn.Module):
        def __init__(self):
            super().__init__()
            self.w, self.b = torch.nn.Parameter(w), torch.nn.Parameter(b)

        def forward(self, x):
            return ag.layer_norm(2 * x, self.w, self.b) + 1

    layer = Layer()
    traced = torch.jit.trace(layer, x, check_trace=False)
    results = []
    for run_ in (layer, traced):
        leaf = dy.clone().requires_grad_(True)
        out = run_(leaf)
        results.append((out.detach(), *torch.autograd.grad(out, (leaf, layer.w, layer.b), x)))
    for one, other in zip(*results):
        assert torch.equal(one, other)


def test_gradients_of_more_columns_than_a_launch_has_threads_for():
    """2^25 columns and more: the sums over the rows have 64 threads to each of twice as many columns.  dw is made of h, off by at most what the row's mean and
    rstd of the forward are off by (both are handed over here), so two products and a sum: 4 half steps of the magnitudes."""
    n, d = 2, (1 << 25) + 37
    gen = torch.Generator(device="cuda").manual_seed(0)
    x, dy = (torch.randn(n, d, device="cuda", generator=gen) for _ in range(2))
    mean, rstd = torch.tensor([0.25, -0.5], device="cuda"), torch.tensor([1.5, 0.75], device="cuda")
    dw, db = torch.full((d,), 7.0, device="cuda"), torch.full((d,), 7.0, device="cuda")
    isp.layer_norm_backward(x, dy, None, mean, rstd, None, dw, db)
    h = (x.double() - mean.double()[:, None]) * rstd.double()[:, None]
    u = 2.0 ** -24
    terms = dy.double() * h
    assert ((dw.double() - terms.sum(0)).abs() <= 4 * u * ((dy.double() * rstd.double()[:, None]).abs() * (x.double().abs() + mean.double().abs()[:, None])).sum(0)).all()
    assert ((db.double() - dy.double().sum(0)).abs() <= 2 * u * dy.double().abs().sum(0)).all()
    isp.layer_norm_backward(x[:0], dy[:0], None, mean[:0], rstd[:0], None, dw, db)
    assert not dw.any() and not db.any()


def test_parameters_of_any_shape():
    """Weight and bias are d elements in any shape; their gradients have it, too."""
    x, w, b, dy = make(40, 24, torch.float32, torch.float32)
    leaves = [w.clone().requires_grad_(True), b.clone().requires_grad_(True)]
    want = torch.autograd.grad(ag.layer_norm(x, *leaves), leaves, dy)
    for ws, bs in (((1, 24), (24, 1)), ((2, 12), (24,)), ((24,), (4, 3, 2))):
        leaves = [w.view(ws).clone().requires_grad_(True), b.view(bs).clone().requires_grad_(True)]
        got = torch.autograd.grad(ag.layer_norm(x, *leaves), leaves, dy)
        for g, t, leaf in zip(got, want, leaves):
            assert g.shape == leaf.shape and torch.equal(g.flatten(), t)
    only = b.view(2, 12).clone().requires_grad_(True)
    assert torch.equal(torch.autograd.grad(ag.layer_norm(x, None, only), only, dy)[0].flatten(), want[1])
