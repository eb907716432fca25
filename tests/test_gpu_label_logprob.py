"""Log probabilities of labels, entropy, top alternatives and the gradient, against the definition in 64 bits.

Tolerances.  u = 2^-24.  With g = z - max every exponential is off by at most (|g| + 3) u of itself; a sum of them is made of at most 4 + 3 additions
per tile of 16, one per tile of the row and lane (`tiles`), 6 exchanges, 8 wavefronts' and 16 workgroups' parts.  As the mean of |g| under the
distribution is at most log C < 16, T and U are off by at most N u, N = 64 + tiles, of their sums of magnitudes.  Differences and the logarithm add
their own half steps.  The gradient's exponent is off by N u + 3 u (|g| + log T), which goes on into p."""
import numpy as np
import pytest
import torch

import paper_2403_14853_amd as isp
from paper_2403_14853_amd import autograd as ag

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
TYPES = [torch.float32, torch.bfloat16, torch.float16]
CLASSES = [1, 2, 3, 4, 5, 7, 8, 9, 16, 33, 47, 64, 100, 128, 349, 512, 1000, 1024, 1025, 2048, 2049, 5000, 8193, 20001]


def half_step(ref, dtype):
    info = torch.finfo(dtype)
    return ref.abs() * (info.eps / 2) + info.smallest_normal * info.eps / 2


def reference(z, labels, top, a=None, e=None):
    z, labels = z.detach().double().cpu(), labels.cpu()
    n, c = z.shape
    N = 64 + c / 1024
    m = z.max(1, keepdim=True).values
    left = m > -np.inf
    g = torch.where(left, z - torch.where(left, m, 0.0), -np.inf)
    t = g.exp().sum(1, keepdim=True)
    logt = t.log()
    lp = g - logt if bool(left.all()) else torch.where(left, g - logt, -np.inf)
    p = lp.exp()
    plp = torch.where(p > 0, p * lp, 0.0)
    ent = -plp.sum(1)
    has = (labels >= 0) & (labels < c)
    at = labels.clamp(0, c - 1)[:, None]
    lt = torch.where(left, logt, 0.0)
    scale = torch.where(left & torch.isfinite(g), g.abs(), 0.0) + lt
    lp_err = U * (N + 2 * scale)
    out = {"logprob": (torch.where(has, lp.gather(1, at)[:, 0], 0.0), torch.where(has, lp_err.gather(1, at)[:, 0], 0.0)),
           "entropy": (ent, U * (N + 4) * (1 + ent + lt[:, 0]))}
    if top:
        order = torch.sort(z, dim=1, descending=True, stable=True).indices[:, :top]
        out["top_index"] = order
        out["top_logprob"] = (lp.gather(1, order), lp_err.gather(1, order))
    if a is not None:
        a, e = a.double().cpu(), e.double().cpu()
        a = torch.where(has, a, 0.0)[:, None]
        hot = torch.zeros_like(z).scatter_(1, at, has.double()[:, None])
        dz = a * (hot - p) - e[:, None] * (plp + p * ent[:, None])
        dz = torch.where(left, dz, 0.0)
        p_err = U * (N + 6 * scale)
        err = p * p_err * (a.abs() + e[:, None].abs() * (scale + ent[:, None] + 1)) + 4 * U * (a.abs() * (hot + p) + e[:, None].abs() * p * (scale + ent[:, None]))
        out["dz"] = (dz, err + 1e-37)
    return out


def check(got, ref, name, rows=None):
    value, bound = ref[name]
    g = got.detach().double().cpu()
    assert g.shape == value.shape, name
    same = g == value.to(got.dtype).double()  # (infinities too, and what is beyond the type's range)
    err = torch.where(same, 0.0, (g - value).abs())
    over = (err / (bound + half_step(torch.where(same, 0.0, value), got.dtype) * 1.001)).max() if g.numel() else torch.tensor(0.0)
    assert over <= 1, "%s: %.3g of the tolerance" % (name, over)


def make(n, c, dtype, seed=0, std=2.0, ld=None, offset=0):
    gen = torch.Generator().manual_seed(100 * c + n + seed)
    ld = ld or c
    full = torch.empty(offset + n * ld, dtype=dtype, device="cuda")
    z = full[offset:].view(n, ld)[:, :c]
    z.copy_((torch.randn(n, c, generator=gen) * std).to(dtype))
    labels = torch.randint(c, (n,), generator=gen)
    labels[torch.rand(n, generator=gen) < 0.2] = -1
    a, e = torch.randn(n, generator=gen), torch.randn(n, generator=gen)
    return z, labels.cuda(), a.cuda(), e.cuda()


def run(z, labels, top, a, e, dz=None):
    n, c = z.shape
    f = lambda *s: torch.full(s, 99.0, device="cuda")
    out = {"logprob": f(n), "entropy": f(n), "stats": f(n, 2)}
    tv, ti = (f(n, top), torch.full((n, top), -9, dtype=torch.int32, device="cuda")) if top else (None, None)
    isp.label_logprob(z, labels, out["logprob"], out["entropy"], stats=out["stats"], top_logprob=tv, top_index=ti)
    out["dz"] = torch.empty(n, c, dtype=z.dtype, device="cuda") if dz is None else dz
    isp.label_logprob_backward(z, labels, out["stats"], a, out["dz"], entropy=out["entropy"], d_entropy=e)
    if top:
        out["top_logprob"], out["top_index"] = tv, ti
    return out


def check_all(got, ref):
    for name in ("logprob", "entropy", "top_logprob", "dz"):
        if name in ref:
            check(got[name], ref, name)
    if "top_index" in ref:
        assert torch.equal(got["top_index"].cpu().long(), ref["top_index"])


@pytest.mark.parametrize("dtype", TYPES, ids=lambda t: str(t)[6:])
@pytest.mark.parametrize("c", CLASSES)
def test_every_width(c, dtype):
    for n, top in ((1, min(c, 1)), (37, min(c, 5)), (130, 0), (23, min(c, 64))):
        z, labels, a, e = make(n, c, dtype)
        check_all(run(z, labels, top, a, e), reference(z, labels, top, a, e))


@pytest.mark.parametrize("dtype", TYPES, ids=lambda t: str(t)[6:])
@pytest.mark.parametrize("n,c,top", [(1, 131_071, 8), (3, 70_000, 16), (600, 9_000, 3), (5_000, 1_030, 4), (4_100, 3_000, 0), (70_001, 13, 2), (30_000, 47, 0)])
def test_ways_to_share_the_rows_out(n, c, top, dtype):
    """Several workgroups to a row, one, a wavefront, lane groups; more rows than one round has."""
    z, labels, a, e = make(n, c, dtype)
    check_all(run(z, labels, top, a, e), reference(z, labels, top, a, e))


@pytest.mark.parametrize("dtype", TYPES, ids=lambda t: str(t)[6:])
@pytest.mark.parametrize("c", [3, 7, 47, 600, 1030, 9001])
def test_leading_dimensions_and_odd_addresses(c, dtype):
    z, labels, a, e = make(19, c, dtype, ld=c + 5, offset=3)
    full = torch.full((1 + 19 * (c + 3),), 7.0, dtype=dtype, device="cuda")
    dz = full[1:].view(19, c + 3)[:, :c]
    check_all(run(z, labels, min(c, 4), a, e, dz), reference(z, labels, min(c, 4), a, e))
    assert full[0] == 7 and (full[1:].view(19, c + 3)[:, c:] == 7).all()


@pytest.mark.parametrize("c", [6, 47, 700, 1500, 40_000])
@pytest.mark.parametrize("dtype", TYPES, ids=lambda t: str(t)[6:])
def test_masked_scores(c, dtype):
    """Classes left out by -inf, rows with one class and with none left, the type's lowest value as a mask, ties."""
    z, labels, a, e = make(40, c, dtype)
    z[:20][torch.rand(20, c, device="cuda") < 0.7] = -np.inf
    z[3] = -np.inf
    z[3, c - 1] = 1.5
    z[4] = -np.inf
    labels[4] = 1
    z[5] = -np.inf
    labels[5] = -1
    low = torch.finfo(dtype).min
    z[6] = low
    z[7, : c // 2] = low
    z[8] = 0
    z[8, ::2] = -0.0
    z[9] = 3
    z[20:30] = z[20:30].round()
    z[30] = torch.finfo(dtype).max
    z[31] = low
    z[31, 0] = torch.finfo(dtype).max
    top = min(c, 9)
    got = run(z, labels, top, a, e)
    ref = reference(z, labels, top, a, e)
    check_all(got, ref)
    assert got["logprob"][4] == -np.inf and got["logprob"][5] == 0 and (got["entropy"][4:6] == 0).all() and (got["dz"][4:6] == 0).all()
    assert (got["top_logprob"][4:6] == -np.inf).all()


@pytest.mark.parametrize("c", [5, 47, 900, 1500, 30_000])
def test_nan_and_infinity(c):
    z, labels, a, e = make(30, c, torch.float32)
    labels.clamp_(min=0)
    z[2, c - 2] = np.nan
    z[3, 1] = np.inf
    z[4] = np.nan
    z[5, 1], z[5, 3] = np.nan, np.nan
    z[6, 2], z[6, 0] = np.inf, np.nan
    got = run(z, labels, 3, a, e)
    bad = torch.zeros(30, dtype=torch.bool)
    bad[2:7] = True
    for name in ("logprob", "entropy"):
        assert torch.equal(torch.isnan(got[name]).cpu(), bad), name
    assert torch.equal(torch.isnan(got["top_logprob"]).any(1).cpu(), bad)
    assert torch.equal(torch.isnan(got["dz"]).any(1).cpu(), bad)
    index = got["top_index"].cpu()
    assert index[2, 0] == c - 2 and index[3, 0] == 1 and index[4].tolist() == [0, 1, 2] and index[5, :2].tolist() == [1, 3]
    assert index[6, :2].tolist() == [0, 2]
    good = ~bad
    ref = reference(z[good.cuda()], labels[good.cuda()], 3, a[good.cuda()], e[good.cuda()])
    check_all({k: v[good.cuda()] for k, v in got.items()}, ref)


def test_labels_outside_and_optional_outputs():
    z, labels, a, e = make(50, 40, torch.float32)
    labels[:6] = torch.tensor([-100, 40, 2 ** 40, -(2 ** 62), 39, 0])
    got, ref = run(z, labels, 0, a, e), reference(z, labels, 0, a, e)
    check_all(got, ref)
    f = lambda *s: torch.full(s, 5.0, device="cuda")
    only = f(50)
    isp.label_logprob(z, labels, only)
    assert torch.equal(only, got["logprob"])
    index = torch.empty(50, 2, dtype=torch.int32, device="cuda")
    ent = f(50)
    isp.label_logprob(z, None, None, ent, top_index=index)
    assert torch.equal(ent, got["entropy"]) and torch.equal(index.cpu().long(), reference(z, labels, 2)["top_index"])
    zero = torch.zeros_like(a)
    for da, de in ((a, None), (None, e), (None, None)):
        dz = torch.empty_like(z)
        isp.label_logprob_backward(z, labels if da is not None else None, got["stats"], da, dz, entropy=got["entropy"] if de is not None else None, d_entropy=de)
        check(dz, reference(z, labels, 0, zero if da is None else da, zero if de is None else de), "dz")
    none = torch.empty(0, 40, device="cuda")
    isp.label_logprob(none, labels[:0], f(0), f(0))
    isp.label_logprob_backward(none, labels[:0], f(0, 2), f(0), torch.empty_like(none))


def test_repeats_bit_for_bit():
    for n, c in ((2000, 47), (4, 60_000)):
        z, labels, a, e = make(n, c, torch.bfloat16)
        first = run(z, labels, 6, a, e)
        for _ in range(3):
            for name, t in run(z, labels, 6, a, e).items():
                assert torch.equal(t, first[name]), name


@pytest.mark.parametrize("dtype", TYPES, ids=lambda t: str(t)[6:])
@pytest.mark.parametrize("n,c", [(200, 47), (9, 3_500), (2, 50_000)])
def test_autograd(n, c, dtype):
    z, labels, a, e = make(n, c, dtype)
    ref = reference(z, labels, 3, a, e)
    leaf = z.clone().requires_grad_(True)
    lp, en, tv, ti = ag.label_logprob(leaf, labels, top=3)
    check_all({"logprob": lp, "entropy": en, "top_logprob": tv, "top_index": ti, "dz": torch.autograd.grad((lp, en), leaf, (a, e), retain_graph=True)[0]}, ref)
    assert not tv.requires_grad and not ti.requires_grad
    zero = torch.zeros_like(a)
    check(torch.autograd.grad(lp, leaf, a, retain_graph=True)[0], reference(z, labels, 0, a, zero), "dz")
    check(torch.autograd.grad(en.sum(), leaf, retain_graph=True)[0], reference(z, labels, 0, zero, torch.ones_like(e)), "dz")
    with torch.no_grad():
        en.zero_()  # (the backward needs it)
    with pytest.raises(RuntimeError):
        torch.autograd.grad(lp, leaf, a)
    pair = ag.label_logprob(z, labels)
    assert len(pair) == 2 and not pair[0].requires_grad
    strided = z.t().contiguous().t().detach().requires_grad_(True)
    check(torch.autograd.grad(ag.label_logprob(strided, labels)[0], strided, a)[0], reference(z, labels, 0, a, zero), "dz")


def test_gradient_against_differences():
    z, labels, a, e = make(6, 11, torch.float32)
    labels.clamp_(min=0)
    dz = run(z, labels, 0, a, e)["dz"].double().cpu()
    Z, A, E = (t.double().cpu() for t in (z, a, e))

    def f(Z):
        lp = torch.log_softmax(Z, 1)
        return (A * lp.gather(1, labels.cpu()[:, None])[:, 0]).sum() - (E * (lp.exp() * lp).sum(1)).sum()

    gen = torch.Generator().manual_seed(1)
    for _ in range(5):
        v = torch.randn(Z.shape, generator=gen, dtype=torch.float64)
        num = (f(Z + 1e-5 * v) - f(Z - 1e-5 * v)) / 2e-5
        assert abs(num - (dz * v).sum()) < 1e-4 * (1 + abs(num))


@pytest.mark.parametrize("n,c", [(300, 47), (3, 40_000)])
def test_captured_and_replayed(n, c):
    z, labels, a, e = make(n, c, torch.float16)
    f = lambda *s: torch.empty(*s, device="cuda")
    lp, en, st, tv, ti, dz = f(n), f(n), f(n, 2), f(n, 4), torch.empty(n, 4, dtype=torch.int32, device="cuda"), torch.empty_like(z)
    ws = torch.empty(isp.label_logprob_workspace(n, c, 4), dtype=torch.uint8, device="cuda")

    def step():
        isp.label_logprob(z, labels, lp, en, stats=st, top_logprob=tv, top_index=ti, workspace=ws)
        isp.label_logprob_backward(z, labels, st, a, dz, entropy=en, d_entropy=e)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for seed in range(3):
        nz, nl, na, ne = make(n, c, torch.float16, seed=seed)
        for t, s in ((z, nz), (labels, nl), (a, na), (e, ne)):
            t.copy_(s)
        graph.replay()
        torch.cuda.synchronize()
        want = run(nz, nl, 4, na, ne)
        for t, name in ((lp, "logprob"), (en, "entropy"), (tv, "top_logprob"), (ti, "top_index"), (dz, "dz")):
            assert torch.equal(t, want[name]), name


def test_on_another_stream():
    z, labels, a, e = make(4, 100_000, torch.float32)
    want = run(z, labels, 5, a, e)
    side = torch.cuda.Stream()
    lp, tv = torch.empty(4, device="cuda"), torch.empty(4, 5, device="cuda")
    torch.cuda.synchronize()
    isp.label_logprob(z, labels, lp, top_logprob=tv, stream=side)
    side.synchronize()
    assert torch.equal(lp, want["logprob"]) and torch.equal(tv, want["top_logprob"])


def test_recorded_by_jit_trace():
    z, labels, a, e = make(40, 20, torch.float32)
    f = lambda z: ag.label_logprob(2 * z, labels, top=2)
    traced = torch.jit.trace(f, z, check_trace=False)
    other = make(40, 20, torch.float32, seed=3)[0]
    results = []
    for run_ in (f, traced):
        leaf = other.clone().requires_grad_(True)
        out = run_(leaf)
        results.append([*(t.detach() for t in out), torch.autograd.grad(out[:2], leaf, (a, e))[0]])
    for x, y in zip(*results):
        assert torch.equal(x, y)
