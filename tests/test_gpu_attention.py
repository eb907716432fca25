"""Attention over the stored entries of a CSR matrix and its gradients, against the definition in 64 bits.

Tolerances.  u = 2^-24.  A score is a sum of products over the head's columns (4 in a lane, up to 6 exchanges, scale and bias): off by at most 16 u A,
A = scale sum |q k| + |bias|.  An exponential of a difference to the row's reference is off by the differences' and 2 |s - m| + 3 half steps, |s - m| at
most 2 A; the row's sums are made of at most 800 additions in a row (a work item's entries) and their joins.  So each P is off by at
most e u of itself, e = 40 + min(L, 800) + 40 max A over the entries that count.  What is made of P (and of t = <dy, v>, off by 16 u T, T = sum |dy v|)
takes that on, and its sums over L entries the same number of half steps again.  Outputs are rounded once.  An exponential below 2^-126 is
zero, and a row's sum is 1 or more (its reference is one of its scores): beside e u P every P may be off by 2^-126, which matters where a gradient is made
of such entries alone (with scores of +-300: P = 5e-39 times t = 4 times q = 200 is 4e-36)."""
import ctypes

import numpy as np
import pytest
import torch

import paper_2403_14853_amd as isp
from paper_2403_14853_amd import autograd as ag

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
FLUSH = 2.0 ** -126
TYPES = [torch.float32, torch.bfloat16, torch.float16]
HEADS = [(1, 1, 1), (2, 1, 2), (3, 3, 3), (5, 5, 4), (1, 1, 5), (4, 4, 8), (8, 2, 16), (6, 2, 7), (3, 3, 20), (2, 2, 50), (1, 1, 256), (2, 1, 130), (5, 1, 12),
         (16, 16, 4), (8, 1, 64), (70, 70, 3), (9, 3, 33), (32, 8, 16), (4, 2, 128), (16, 2, 6)]


def half_step(ref, dtype):
    info = torch.finfo(dtype)
    return ref.abs() * (info.eps / 2) + info.smallest_normal * info.eps / 2


def graph(n, m, seed, hubs=((5, 1500), (17, 300), (40, 90)), longest=30):
    """Rows of 0 to `longest` entries and a few long ones, columns unsorted and repeated."""
    gen = np.random.default_rng(seed)
    lengths = gen.integers(0, longest + 1, n)
    lengths[gen.random(n) < 0.2] = 0
    for row, length in hubs:
        if row < n:
            lengths[row] = length
    indptr = np.zeros(n + 1, np.int64)
    np.cumsum(lengths, out=indptr[1:])
    cols = gen.integers(0, m, int(indptr[-1])).astype(np.int32)
    few = gen.random(cols.shape[0]) < 0.2  # a popular column: a long row of the transpose
    cols[few] = m // 3
    return torch.from_numpy(indptr), torch.from_numpy(cols)


def reference(indptr, cols, q, k, v, dy, heads, kv, scale, bias=None):
    """{name: (value, bound before the last rounding)} in 64 bits."""
    q, k, v, dy = (t.detach().double().cpu() for t in (q, k, v, dy))
    n, m, c = q.shape[0], k.shape[0], q.shape[1] // heads
    lengths = torch.diff(indptr)
    rows = torch.repeat_interleave(torch.arange(n), lengths)
    cols = cols.long()
    per_row = lambda x: torch.zeros(n, *x.shape[1:], dtype=torch.float64).index_add_(0, rows, x)
    per_col = lambda x: torch.zeros(m, *x.shape[1:], dtype=torch.float64).index_add_(0, cols, x)
    long_row = lengths.clamp(max=800).double()
    long_col = torch.bincount(cols, minlength=m).clamp(max=800).double() * (heads // kv)
    out = {x: (torch.zeros(s, dtype=torch.float64), torch.zeros(s, dtype=torch.float64)) for x, s in
           (("y", q.shape), ("dq", q.shape), ("dk", k.shape), ("dv", v.shape))}
    b = torch.zeros(len(cols), dtype=torch.float64) if bias is None else bias.double().cpu()
    live = b > -np.inf
    for h in range(heads):
        a, g = slice(h * c, h * c + c), slice(h // (heads // kv) * c, h // (heads // kv) * c + c)
        clean = lambda x: torch.where(live[:, None], x, 0.0)
        Q, K, V, G = clean(q[rows, a]), clean(k[cols, g]), clean(v[cols, g]), clean(dy[rows, a])
        s = torch.where(live, scale * (Q * K).sum(1) + b, -np.inf)
        A = torch.where(live, scale * (Q * K).abs().sum(1) + b.abs(), 0.0)
        top = torch.full((n,), -np.inf, dtype=torch.float64).scatter_reduce(0, rows, s, "amax")
        e = torch.where(live, (s - torch.where(torch.isfinite(top), top, 0.0)[rows]).exp(), 0.0)
        z = per_row(e)
        p = e / torch.where(z > 0, z, 1.0)[rows]
        worst = torch.zeros(n, dtype=torch.float64).scatter_reduce(0, rows, torch.where(p > 0, A, 0.0), "amax")
        er = U * (40 + long_row + 40 * worst)
        pm = p + FLUSH / er[rows]  # (er pm = er p + FLUSH)
        t, T = (G * V).sum(1), (G * V).abs().sum(1)
        D, Dm = per_row(p * t), per_row(pm * T)
        ds, dsm = p * (t - D[rows]), pm * (T + Dm[rows])
        out["y"][0][:, a] = per_row(p[:, None] * V)
        out["y"][1][:, a] = 2 * er[:, None] * per_row(pm[:, None] * V.abs())
        out["dq"][0][:, a] = scale * per_row(ds[:, None] * K)
        out["dq"][1][:, a] = 3 * er[:, None] * scale * (per_row((pm * T)[:, None] * K.abs()) + Dm[:, None] * per_row(pm[:, None] * K.abs()))
        ec = (3 * er[rows] + U * long_col[cols])[:, None]
        out["dk"][0][:, g] += scale * per_col(ds[:, None] * Q)
        out["dk"][1][:, g] += scale * per_col(ec * dsm[:, None] * Q.abs())
        out["dv"][0][:, g] += per_col(p[:, None] * G)
        out["dv"][1][:, g] += per_col(ec * pm[:, None] * G.abs())
    return out


def check(got, ref, name):
    value, bound = ref[name]
    g = got.detach().double().cpu()
    assert g.shape == value.shape and torch.isfinite(g).all(), name
    over = ((g - value).abs() / (bound + half_step(value, got.dtype) * 1.001 + 1e-37)).max() if g.numel() else torch.tensor(0.0)
    assert over <= 1, "%s: %.3g of the tolerance" % (name, over)


def operands(n, m, heads, kv, c, dtype, seed=0, gap=0, offset=0):
    gen = torch.Generator().manual_seed(seed + 31 * n + c)
    def rows(r, w):
        full = torch.full((offset + r * (w + gap),), 7.0, dtype=dtype, device="cuda")
        t = full[offset:].view(r, w + gap)[:, :w]
        t.copy_(torch.randn(r, w, generator=gen).to(dtype))
        return t
    return rows(n, heads * c), rows(m, kv * c), rows(m, kv * c), rows(n, heads * c)


def build(indptr, cols, m, bias=None):
    A = isp.csr_build(indptr.cuda(), cols.cuda(), None if bias is None else bias.cuda(), n_cols=m)
    isp.csr_transpose_cached(A)
    return A


def run(A, q, k, v, dy, heads, kv, scale=None, bias=False, outs=None, **kw):
    like = lambda t: torch.full(t.shape, 99.0, dtype=t.dtype, device="cuda")
    y, dq, dk, dv = outs or (like(q), like(q), like(k), like(v))
    stats = torch.empty(q.shape[0], heads, 2, device="cuda")
    isp.attention(A, q, k, v, y, heads, kv, scale=scale, bias=bias, stats=stats, **kw)
    isp.attention_backward(A, q, k, v, stats, dy, dq, dk, dv, heads, kv, scale=scale, bias=bias, **kw)
    return {"y": y, "dq": dq, "dk": dk, "dv": dv}


def check_all(got, ref):
    for name in ("y", "dq", "dk", "dv"):
        check(got[name], ref, name)


@pytest.mark.parametrize("dtype", TYPES, ids=lambda t: str(t)[6:])
@pytest.mark.parametrize("heads,kv,c", HEADS)
def test_every_shape_of_heads(heads, kv, c, dtype):
    n, m = 230, 190
    indptr, cols = graph(n, m, heads * 100 + c)
    q, k, v, dy = operands(n, m, heads, kv, c, dtype)
    A = build(indptr, cols, m)
    assert A.info()["n_segments"] > 0
    check_all(run(A, q, k, v, dy, heads, kv), reference(indptr, cols, q, k, v, dy, heads, kv, c ** -0.5))


@pytest.mark.parametrize("dtype", TYPES, ids=lambda t: str(t)[6:])
@pytest.mark.parametrize("n,m,hubs,longest", [(1, 1, (), 1), (1, 50, ((0, 700),), 3), (7, 3, (), 4), (4000, 3500, ((100, 5000), (200, 900)), 12), (3000, 4000, (), 2)])
def test_sizes(n, m, hubs, longest, dtype):
    indptr, cols = graph(n, m, n, hubs, longest)
    if n == 1 and m == 1:
        indptr, cols = torch.tensor([0, 1]), torch.tensor([0], dtype=torch.int32)
    for heads, kv, c in ((4, 2, 16), (1, 1, 24)):
        q, k, v, dy = operands(n, m, heads, kv, c, dtype)
        check_all(run(build(indptr, cols, m), q, k, v, dy, heads, kv), reference(indptr, cols, q, k, v, dy, heads, kv, c ** -0.5))


@pytest.mark.parametrize("dtype", TYPES, ids=lambda t: str(t)[6:])
@pytest.mark.parametrize("heads,kv,c", [(2, 1, 2), (6, 2, 7), (4, 4, 16), (2, 2, 50), (8, 1, 20)])
def test_leading_dimensions_and_odd_addresses(heads, kv, c, dtype):
    n, m = 120, 110
    indptr, cols = graph(n, m, 3)
    q, k, v, dy = operands(n, m, heads, kv, c, dtype, gap=3, offset=5)
    outs = operands(n, m, heads, kv, c, dtype, gap=5, offset=1)
    outs = (outs[0], outs[3], outs[1], outs[2])
    check_all(run(build(indptr, cols, m), q, k, v, dy, heads, kv, outs=outs), reference(indptr, cols, q, k, v, dy, heads, kv, c ** -0.5))
    for t in outs:
        full = torch.as_strided(t, (t.shape[0], t.stride(0)), (t.stride(0), 1), t.storage_offset())
        assert (full[:, t.shape[1]:] == 7).all()


@pytest.mark.parametrize("dtype", TYPES, ids=lambda t: str(t)[6:])
@pytest.mark.parametrize("heads,kv,c", [(4, 4, 8), (8, 2, 16), (3, 3, 20), (2, 1, 3), (6, 1, 64)])
def test_bias_and_masks(heads, kv, c, dtype):
    """An edge bias; entries masked by -inf, rows with one entry left and with none, biases of fp32's lowest value alone in a row and beside others."""
    n, m = 150, 140
    indptr, cols = graph(n, m, 8)
    gen = torch.Generator().manual_seed(2)
    bias = torch.randn(len(cols), generator=gen)
    bias[torch.rand(len(cols), generator=gen) < 0.3] = -np.inf
    low = torch.finfo(torch.float32).min
    full = [i for i in range(n) if indptr[i + 1] - indptr[i] >= 3]
    at = lambda i: slice(int(indptr[full[i]]), int(indptr[full[i] + 1]))
    bias[at(0)] = -np.inf
    bias[at(1)] = -np.inf
    bias[at(1)][1:2] = 0.5
    bias[at(2)] = low
    bias[at(3)] = low
    bias[at(3)][2:3] = 1.0
    bias[at(4)][:1] = low
    hub = slice(int(indptr[5]), int(indptr[6]))  # (the longest row: whole segments masked)
    bias[hub][: 900] = -np.inf
    masked_hub = slice(int(indptr[17]), int(indptr[18]))
    bias[masked_hub] = -np.inf
    q, k, v, dy = operands(n, m, heads, kv, c, dtype)
    A = build(indptr, cols, m, bias)
    got = run(A, q, k, v, dy, heads, kv, scale=0.37, bias=True)
    check_all(got, reference(indptr, cols, q, k, v, dy, heads, kv, 0.37, bias))
    for i in (full[0], 17):
        assert (got["y"][i] == 0).all() and (got["dq"][i] == 0).all()
    # the values are not looked at unless they are asked for
    check_all(run(A, q, k, v, dy, heads, kv), reference(indptr, cols, q, k, v, dy, heads, kv, c ** -0.5))


def test_masked_entries_may_hold_anything():
    n, m, heads, kv, c = 60, 50, 4, 2, 12
    indptr, cols = graph(n, m, 4)
    bias = torch.zeros(len(cols))
    bias[(cols == 7) | (cols == 9)] = -np.inf
    rows = torch.repeat_interleave(torch.arange(n), torch.diff(indptr))
    bias[rows == 11] = -np.inf
    q, k, v, dy = operands(n, m, heads, kv, c, torch.float32)
    clean = reference(indptr, cols, q, k, v, dy, heads, kv, c ** -0.5, bias)
    k[7], v[7], k[9], v[9] = np.nan, np.inf, np.inf, np.nan
    q[11], dy[11] = np.inf, np.nan
    got = run(build(indptr, cols, m, bias), q, k, v, dy, heads, kv, bias=True)
    check_all(got, clean)


def test_large_scores():
    """Scores in the hundreds, whose exponentials overflow without a reference, in any order within a row."""
    n, m, heads, c = 100, 90, 4, 16
    indptr, cols = graph(n, m, 6)
    q, k, v, dy = operands(n, m, heads, heads, c, torch.float32)
    q *= 60
    check_all(run(build(indptr, cols, m), q, k, v, dy, heads, heads), reference(indptr, cols, q, k, v, dy, heads, heads, c ** -0.5))


def test_nan_stays_in_its_row():
    n, m, heads, c = 100, 90, 2, 8
    indptr, cols = graph(n, m, 7, hubs=())
    q, k, v, dy = operands(n, m, heads, heads, c, torch.float32)
    q[33] = np.nan
    y = run(build(indptr, cols, m), q, k, v, dy, heads, heads)["y"]
    bad = torch.isnan(y).any(1).cpu()
    assert int(bad.sum()) == int(indptr[34] > indptr[33]) and bool(bad[33]) == bool(indptr[34] > indptr[33])


def test_no_entries_and_no_rows():
    heads, c = 2, 12
    for n, m in ((5, 4), (0, 4), (5, 0)):
        A = build(torch.zeros(n + 1, dtype=torch.int64), torch.zeros(0, dtype=torch.int32), m)
        q, k, v, dy = operands(n, m, heads, heads, c, torch.float32)
        for t in run(A, q, k, v, dy, heads, heads).values():
            assert (t == 0).all()


def test_block_diagonal_batch_and_causal_rows():
    """Graphs of different sizes packed into one matrix give what each gives alone; a causal pattern is a lower triangle."""
    sizes, heads, kv, c = [1, 40, 7, 130], 4, 2, 16
    parts = [(torch.arange(s + 1) * torch.arange(1, s + 2) // 2, torch.cat([torch.arange(i + 1) for i in range(s)]).int()) for s in sizes]  # lower triangles
    q, k, v, dy = operands(sum(sizes), sum(sizes), heads, kv, c, torch.float32)
    indptr, cols, at, entries = [torch.zeros(1, dtype=torch.int64)], [], 0, 0
    for (p, x), s in zip(parts, sizes):
        indptr.append(p[1:] + entries)
        cols.append(x + at)
        at, entries = at + s, entries + len(x)
    got = run(build(torch.cat(indptr), torch.cat(cols), at), q, k, v, dy, heads, kv)
    check_all(got, reference(torch.cat(indptr), torch.cat(cols), q, k, v, dy, heads, kv, c ** -0.5))
    at = 0
    for (p, x), s in zip(parts, sizes):
        r = slice(at, at + s)
        check_all({name: t[r] for name, t in got.items()}, reference(p, x, q[r], k[r], v[r], dy[r], heads, kv, c ** -0.5))
        dense = torch.softmax((q[r, :c].double() @ k[r, :c].double().t() * c ** -0.5).masked_fill(torch.ones(s, s, device="cuda").triu(1) > 0, -np.inf), 1) @ v[r, :c].double()
        assert torch.allclose(got["y"][r, :c].double(), dense, rtol=1e-4, atol=1e-5)
        at += s


def test_gradients_wanted_in_part():
    n, m, heads, kv, c = 80, 70, 4, 2, 8
    indptr, cols = graph(n, m, 9)
    q, k, v, dy = operands(n, m, heads, kv, c, torch.float32)
    A = build(indptr, cols, m)
    want = run(A, q, k, v, dy, heads, kv)
    stats = torch.empty(n, heads, 2, device="cuda")
    y = isp.attention(A, q, k, v, torch.empty_like(q), heads, kv, stats=stats)
    assert torch.equal(y, want["y"])
    dq, dk, dv = torch.empty_like(q), torch.empty_like(k), torch.empty_like(v)
    assert isp.attention_backward(A, q, k, v, stats, dy, dq, None, None, heads, kv) == (dq, None, None)
    isp.attention_backward(A, q, k, v, stats, dy, None, dk, dv, heads, kv)
    for t, name in ((dq, "dq"), (dk, "dk"), (dv, "dv")):
        assert torch.equal(t, want[name])
    B = isp.csr_build(indptr.cuda(), cols.cuda(), None, n_cols=m)  # (without a transpose)
    dq.zero_()
    isp.attention_backward(B, q, k, v, stats, dy, dq, None, None, heads, kv)
    assert torch.equal(dq, want["dq"])
    with pytest.raises(isp.IspError):
        isp.attention_backward(B, q, k, v, stats, dy, dq, dk, dv, heads, kv)
    assert torch.equal(isp.attention(A, q, k, v, torch.empty_like(q), heads, kv), want["y"])


def test_the_transpose_as_the_matrix():
    n, m, c = 60, 80, 16
    indptr, cols = graph(n, m, 10)
    A = build(indptr, cols, m)
    At, _ = isp.csr_transpose_cached(A)
    ti, tj, _, _ = At.export()
    q, k, v, dy = operands(m, n, 2, 2, c, torch.float32)
    y = isp.attention(At, q, k, v, torch.empty_like(q), 2)
    check(y, reference(ti.cpu(), tj.cpu(), q, k, v, dy, 2, 2, c ** -0.5), "y")
    with pytest.raises(isp.IspError):
        isp.attention_backward(At, q, k, v, torch.empty(m, 2, 2, device="cuda"), dy, y, k, v, 2)


def test_refusals():
    n, m, heads, kv, c = 30, 20, 4, 2, 8
    indptr, cols = graph(n, m, 1, hubs=((3, 400),))
    A = build(indptr, cols, m)
    q, k, v, dy = operands(n, m, heads, kv, c, torch.float32)
    y, stats = torch.empty_like(q), torch.empty(n, heads, 2, device="cuda")
    ok = dict(A=A, Q=q, K=k, V=v, Y=y, heads=heads, kv_heads=kv)
    for bad in (dict(Q=q[:-1]), dict(K=k[:-1]), dict(V=v[:, :-1]), dict(Y=y[:, 1:]), dict(Q=q.cpu()), dict(K=k.half()), dict(Y=y.bfloat16()), dict(Q=q.double()),
                dict(heads=5), dict(kv_heads=4), dict(kv_heads=0), dict(heads=0), dict(stats=stats[1:]), dict(stats=stats.half()), dict(Q=q.t()),
                dict(workspace=torch.empty(8, device="cuda")), dict(Q=q[0])):
        with pytest.raises(AssertionError):
            isp.attention(**{**ok, **bad})
    need = isp.attention_workspace(A, heads, c)
    assert need > 0
    for bad in (dict(workspace=torch.empty(need - 1, dtype=torch.uint8, device="cuda")), dict(workspace=torch.empty(need + 8, dtype=torch.uint8, device="cuda")[8:]),
                dict(bias=True)):
        with pytest.raises(isp.IspError):
            isp.attention(**{**ok, **bad})
    wide = torch.empty(n, 514, device="cuda"), torch.empty(m, 514, device="cuda")
    with pytest.raises(isp.IspError) as e:
        isp.attention(A, wide[0], wide[1], wide[1], torch.empty_like(wide[0]), 2)
    assert e.value.status_name == "ISP_EUNSUPPORTED"
    three = torch.empty(n, 3 * c, device="cuda")
    with pytest.raises(isp.IspError):  # (three query heads on two key heads)
        isp.attention(A, three, k, v, torch.empty_like(three), 3, 2, workspace=torch.empty(1 << 20, dtype=torch.uint8, device="cuda"))
    back = dict(A=A, Q=q, K=k, V=v, stats=stats, dY=dy, dQ=torch.empty_like(q), dK=torch.empty_like(k), dV=torch.empty_like(v), heads=heads, kv_heads=kv)
    for bad in (dict(dY=dy[:-1]), dict(dQ=y[:, 1:]), dict(dK=q), dict(dV=v.half()), dict(stats=stats.view(-1)[1:])):
        with pytest.raises(AssertionError):
            isp.attention_backward(**{**back, **bad})
    with pytest.raises(TypeError):
        isp.attention_backward(**{**back, "stats": None})
    for bad in (dict(dK=None), dict(bias=True), dict(workspace=torch.empty(64, dtype=torch.uint8, device="cuda"))):
        with pytest.raises(isp.IspError):
            isp.attention_backward(**{**back, **bad})


def test_repeats_bit_for_bit_and_calls_overlap():
    """Two streams on one handle, each with a workspace of its own."""
    n, m, heads, kv, c = 3000, 2500, 8, 4, 16
    indptr, cols = graph(n, m, 12, hubs=((100, 6000), (900, 2000)))
    A = build(indptr, cols, m)
    sets = [operands(n, m, heads, kv, c, torch.bfloat16, seed=s) for s in range(2)]
    want = [run(A, *s, heads, kv) for s in sets]
    for _ in range(3):
        streams = [torch.cuda.Stream() for _ in sets]
        torch.cuda.synchronize()
        got = []
        for s, ops in zip(streams, sets):
            with torch.cuda.stream(s):
                got.append(run(A, *ops, heads, kv))
        torch.cuda.synchronize()
        for g, w in zip(got, want):
            for name in w:
                assert torch.equal(g[name], w[name]), name
    B = isp.csr_alias(A)
    for name, t in run(B, *sets[0], heads, kv).items():
        assert torch.equal(t, want[0][name])
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    got = run(A, *sets[1], heads, kv, stream=side)
    side.synchronize()
    for name, t in got.items():
        assert torch.equal(t, want[1][name])


def test_captured_and_replayed():
    n, m, heads, kv, c = 500, 400, 4, 2, 16
    indptr, cols = graph(n, m, 13)
    A = build(indptr, cols, m)
    ops = operands(n, m, heads, kv, c, torch.float16)
    outs = [torch.empty_like(ops[i]) for i in (0, 0, 1, 2)]
    stats = torch.empty(n, heads, 2, device="cuda")
    ws = torch.empty(max(isp.attention_workspace(A, heads, c), isp.attention_backward_workspace(A, heads, kv, c)), dtype=torch.uint8, device="cuda")

    def step():
        isp.attention(A, *ops[:3], outs[0], heads, kv, stats=stats, workspace=ws)
        isp.attention_backward(A, *ops[:3], stats, ops[3], *outs[1:], heads, kv, workspace=ws)

    step()
    torch.cuda.synchronize()
    captured = torch.cuda.CUDAGraph()
    with torch.cuda.graph(captured):
        step()
    for seed in range(3):
        new = operands(n, m, heads, kv, c, torch.float16, seed=seed)
        for t, s in zip(ops, new):
            t.copy_(s)
        captured.replay()
        torch.cuda.synchronize()
        want = run(A, *new, heads, kv)
        for t, name in zip(outs, ("y", "dq", "dk", "dv")):
            assert torch.equal(t, want[name]), name


@pytest.mark.parametrize("dtype", TYPES, ids=lambda t: str(t)[6:])
def test_autograd(dtype):
    n, m, heads, kv, c = 200, 180, 8, 2, 12
    indptr, cols = graph(n, m, 14)
    bias = torch.randn(len(cols), generator=torch.Generator().manual_seed(0))
    q, k, v, dy = operands(n, m, heads, kv, c, dtype)
    g = ag.SparseGraph(indptr.cuda(), cols.cuda(), bias.cuda(), n_cols=m)
    for use in (False, True):
        ref = reference(indptr, cols, q, k, v, dy, heads, kv, c ** -0.5, bias if use else None)
        leaves = [t.clone().requires_grad_(True) for t in (q, k, v)]
        y = ag.attention(g, *leaves, heads, kv, bias=use)
        check(y, ref, "y")
        grads = torch.autograd.grad(y, leaves, dy, retain_graph=True)
        for t, name in zip(grads, ("dq", "dk", "dv")):
            check(t, ref, name)
        for i, name in enumerate(("dq", "dk", "dv")):
            only = [t.detach().requires_grad_(i == j) for j, t in enumerate(leaves)]
            check(torch.autograd.grad(ag.attention(g, *only, heads, kv, bias=use), only[i], dy)[0], ref, name)
        y.sum().backward()  # (an upstream gradient of stride 0)
        ones = reference(indptr, cols, q, k, v, torch.ones_like(dy), heads, kv, c ** -0.5, bias if use else None)
        check(leaves[2].grad, ones, "dv")
        with pytest.raises(RuntimeError):
            y.backward(dy)
    # values rewritten in place reach both passes
    with torch.no_grad():
        g.values.mul_(2)
    y = ag.attention(g, *leaves, heads, kv, bias=True)
    for t, name in zip(torch.autograd.grad(y, leaves, dy), ("dq", "dk", "dv")):
        check(t, reference(indptr, cols, q, k, v, dy, heads, kv, c ** -0.5, 2 * bias), name)
    y, plain = ag.attention(g, *leaves, heads, kv, bias=True), ag.attention(g, *leaves, heads, kv)
    with torch.no_grad():
        g.values.mul_(2)
    with pytest.raises(RuntimeError):  # (the backward needs the bias of the forward)
        y.backward(dy)
    check(torch.autograd.grad(plain, leaves, dy)[0], reference(indptr, cols, q, k, v, dy, heads, kv, c ** -0.5), "dq")
    x = q.clone().requires_grad_(True)
    w = x * 1
    y = ag.attention(g, w, k, v, heads, kv)
    with torch.no_grad():
        w.zero_()
    with pytest.raises(RuntimeError):  # (the backward needs Q)
        y.backward(dy)
    trained = ag.SparseGraph(indptr.cuda(), cols.cuda(), bias.cuda().requires_grad_(True), n_cols=m)
    with pytest.raises(NotImplementedError):
        ag.attention(trained, q, k, v, heads, kv, bias=True)
    check(ag.attention(trained, q, k, v, heads, kv), reference(indptr, cols, q, k, v, dy, heads, kv, c ** -0.5), "y")


def test_gradient_against_differences():
    n, m, heads, kv, c = 12, 10, 2, 1, 6
    indptr, cols = graph(n, m, 15, hubs=(), longest=5)
    q, k, v, dy = operands(n, m, heads, kv, c, torch.float32)
    got = run(build(indptr, cols, m), q, k, v, dy, heads, kv)
    Q, K, V, G = (t.double().cpu() for t in (q, k, v, dy))
    f = lambda *x: (reference(indptr, cols, *x, G, heads, kv, c ** -0.5)["y"][0] * G).sum()
    gen = torch.Generator().manual_seed(3)
    for i, name in enumerate(("dq", "dk", "dv")):
        args = [Q, K, V]
        d = torch.randn(args[i].shape, generator=gen, dtype=torch.float64)
        up, down = list(args), list(args)
        up[i], down[i] = args[i] + 1e-5 * d, args[i] - 1e-5 * d
        num = (f(*up) - f(*down)) / 2e-5
        assert abs(num - (got[name].double().cpu() * d).sum()) < 1e-4 * (1 + abs(num)), name


def test_recorded_by_jit_trace():
    n, heads, c = 50, 2, 8
    indptr, cols = graph(n, n, 16, hubs=())
    g = ag.SparseGraph(indptr.cuda(), cols.cuda())
    q, k, v, dy = operands(n, n, heads, heads, c, torch.float32)
    f = lambda q, k, v: torch.relu(ag.attention(g, 2 * q, k, v, heads)) + 1
    traced = torch.jit.trace(f, (dy, k, v), check_trace=False)
    results = []
    for run_ in (f, traced):
        leaves = [t.clone().requires_grad_(True) for t in (q, k, v)]
        y = run_(*leaves)
        results.append((y.detach(), *torch.autograd.grad(y, leaves, dy)))
    for one, other in zip(*results):
        assert torch.equal(one, other)


@pytest.mark.parametrize("heads,kv,c,dtype,wide", [(4, 2, 12, torch.float32, False), (8, 2, 16, torch.bfloat16, False), (2, 1, 3, torch.float16, False), (3, 3, 20, torch.float16, True),
                                                   (8, 8, 16, torch.bfloat16, True), (6, 1, 8, torch.float32, False)])
@pytest.mark.parametrize("where", ["q", "dy", "v"])
def test_masked_entries_of_rows_that_are_not_finite(where, heads, kv, c, dtype, wide):
    """Rows with masked entries and with others that make their sums infinite or NaN: the keys that such a row only reaches through masked entries have
    the gradients of the row left out.  wide: rows of 16 entries and more on average, which 16-bit passes over one query head per key head take with eight
    columns to a lane."""
    n, m, bad = 90, 150, torch.tensor([11, 30, 55])
    gen = np.random.default_rng(c)
    lengths = gen.integers(20, 60, n) if wide else gen.integers(3, 9, n)
    lengths[30] = 700  # (segments of a split row)
    indptr = torch.zeros(n + 1, dtype=torch.int64)
    indptr[1:] = torch.from_numpy(lengths).cumsum(0)
    cols = torch.from_numpy(gen.integers(3, m, int(indptr[-1])).astype(np.int32))
    rows = torch.repeat_interleave(torch.arange(n), torch.diff(indptr))
    bias = torch.randn(len(cols), generator=torch.Generator().manual_seed(1))
    mine = torch.isin(rows, bad)
    bias[mine & (cols >= 30)] = -np.inf
    for j, i in enumerate(bad.tolist()):  # the row's first entry counts, in a column that is its alone; the next one does not
        at = int(indptr[i])
        cols[at], bias[at] = j, 0.5
        cols[at + 1], bias[at + 1] = 100 + j, -np.inf
    q, k, v, dy = operands(n, m, heads, kv, c, dtype)
    without = torch.where(mine, -np.inf, bias)
    clean = reference(indptr, cols, q, k, v, dy, heads, kv, c ** -0.5, without)
    values = torch.tensor([np.nan, np.inf, -np.inf], dtype=dtype, device="cuda")[:, None]
    if where == "v":
        v[:3] = values
    else:
        (q if where == "q" else dy)[bad.cuda()] = values
    got = run(build(indptr, cols, m, bias), q, k, v, dy, heads, kv, bias=True)
    outside, far = torch.ones(n, dtype=torch.bool), torch.arange(m) >= 30  # (columns below 30 may hold anything)
    outside[bad] = False
    for name, keep in (("y", outside), ("dq", outside), ("dk", far), ("dv", far)):
        check(got[name][keep.cuda()], {name: tuple(t[keep] for t in clean[name])}, name)


def test_workspace_without_split_rows():
    """No row is split, so no partial rows are wanted; a workspace with room for the copy of K and V takes it, and has to be one."""
    n, m, heads, c = 40_000, 600, 3, 20
    indptr = torch.arange(n + 1) * 60
    gen = torch.Generator().manual_seed(1)
    cols = torch.randint(m, (60 * n,), generator=gen, dtype=torch.int32)
    q, k, v, _ = operands(n, m, heads, heads, c, torch.float16)
    A = isp.csr_build(indptr.cuda(), cols.cuda(), None, n_cols=m)
    assert A.info()["n_segments"] == 0
    need = isp.attention_workspace(A, heads, c, heads, torch.float16)
    assert need == m * 256  # (two rows of 120 bytes in two lines)
    y = torch.full_like(q, 7.0)
    ws = torch.empty(need + 256, dtype=torch.uint8, device="cuda")
    p = lambda t: ctypes.c_void_p(t.data_ptr())
    call = lambda ws, size: isp.load_library().isp_attention(A.handle, p(q), heads * c, p(k), heads * c, p(v), heads * c, heads, heads, c, ctypes.c_float(c ** -0.5), 0, 2,
                                                             p(y), heads * c, None, ctypes.c_void_p(ws), size, None)
    for bad in ((None, need), (None, 1 << 40), (ws.data_ptr() + 8, need), (ws.data_ptr() + 128, need)):
        assert call(*bad) == 1  # ISP_EINVAL
        torch.cuda.synchronize()
        assert (y == 7).all()
    results = []
    for good in ((None, 0), (None, need - 1), (ws.data_ptr(), need), (ws.data_ptr() + 8, need - 1)):  # (with less than the copy takes nothing of it is used)
        y.fill_(7)
        torch.cuda.synchronize()
        assert call(*good) == 0
        torch.cuda.synchronize()
        results.append(y.clone())
    for r in results:
        assert torch.equal(r, results[0])
    assert (results[0] != 7).any(1).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["float32", "bfloat16"])
@pytest.mark.parametrize("heads,kv,c", [(1, 1, 4), (4, 2, 12), (3, 3, 20)])
def test_keys_of_large_magnitude(heads, kv, c, dtype):
    """Keys of 2^117 and rows of up to 1,500 entries: dq is of the keys' size, and so has every sum on the way to be."""
    n, m = 300, 250
    indptr, cols = graph(n, m, 41)
    q, k, v, dy = (t.float() for t in operands(n, m, heads, kv, c, dtype))
    q, k = (q * 2.0 ** -114).to(dtype), (k * 2.0 ** 115).to(dtype)
    scale = 1.5 / c ** 0.5
    check_all(run(build(indptr, cols, m), q, k, v.to(dtype), dy.to(dtype), heads, kv, scale=scale), reference(indptr, cols, q, k, v, dy, heads, kv, scale))


@pytest.mark.parametrize("heads,kv,c", [(4, 2, 12), (3, 3, 20), (1, 1, 3)])
@pytest.mark.parametrize("dtype,large,small", [(torch.bfloat16, 2.0 ** 124, 2.0 ** -128), (torch.float16, 2.0 ** 12, 2.0 ** -16)], ids=["bfloat16", "float16"])
def test_subnormal_operands(dtype, large, small, heads, kv, c):
    """Keys that are mostly subnormal in their type, and queries that are too.  A sum of two products and a third term is off by at most 3 u of the terms, in which a subnormal operand counts as
    the smallest normal number; up to 4 of those, 5 exchanges and the scale make 20 u A' of a score, A' = scale sum max(|q|, tiny) max(|k|, tiny), so
    e = 40 + min(L, 800) + 44 max A' in place of the file's (its two differences of scores, and their rounding)."""
    n, m = 300, 250
    indptr, cols = graph(n, m, 31, longest=50)
    tiny = torch.finfo(dtype).smallest_normal
    for swap in (False, True):
        q, k, v, dy = (t.float() for t in operands(n, m, heads, kv, c, dtype))
        q, k = ((q * small, k * large) if swap else (q * large, k * small))
        q, k, v, dy = (t.to(dtype) for t in (q, k, v, dy * 2.0 ** -6))
        sub = q if swap else k
        assert ((sub != 0) & (sub.abs() < tiny)).float().mean() > 0.8
        scale = 1 / (small * large * c ** 0.5)
        ref = reference(indptr, cols, q, k, v, dy, heads, kv, scale)
        rows = torch.repeat_interleave(torch.arange(n), torch.diff(indptr))
        long_row = torch.diff(indptr).clamp(max=800).double()
        more = 1.0
        for h in range(heads):
            a, g = slice(h * c, h * c + c), slice(h // (heads // kv) * c, h // (heads // kv) * c + c)
            Q, Kk = q[:, a].double().abs().cpu()[rows], k[:, g].double().abs().cpu()[cols.long()]
            A, Am = scale * (Q * Kk).sum(1), scale * (Q.clamp(min=tiny) * Kk.clamp(min=tiny)).sum(1)
            top = lambda x: torch.zeros(n, dtype=torch.float64).scatter_reduce(0, rows, x, "amax")
            more = max(more, ((40 + long_row + 44 * top(Am)) / (40 + long_row + 40 * top(A))).max().item())
        got = run(build(indptr, cols, m), q, k, v, dy, heads, kv, scale=scale)
        checked = 0
        for name in ("y", "dq", "dk", "dv"):
            value, bound = ref[name]
            if value.abs().max() < torch.finfo(dtype).max * 0.9:  # (fp16's gradients of the small operand are large)
                check(got[name], {name: (value, bound * more)}, name)
                checked += 1
        assert checked >= 3


@pytest.mark.parametrize("longest", [10, 100, 700])
@pytest.mark.parametrize("keys", [0.0, 30.0])
def test_values_with_a_common_part(keys, longest):
    """Values (and keys) that are nearly the same in all columns: t = <dy, v> is nearly D in every entry, and dq = scale sum P (t - D) k is a small difference of
    large numbers, whichever way it is formed.  In 32 bits the sum over the entries rounds t and D, numbers of the size of T = |dy| |v|; the kernel's
    sum e t k - D sum e k rounds, per entry, products and sums of the size of T |k| some three times as often: no more than 3 times the error."""
    heads, c = 2, 16
    n = max(60, 30_000 // longest)
    m = max(n, 400)
    gen = torch.Generator().manual_seed(longest)
    indptr = torch.arange(n + 1) * longest
    cols = torch.randint(m, (n * longest,), generator=gen, dtype=torch.int32)
    r = lambda *s: torch.randn(*s, generator=gen).cuda()
    q, k, dy, v = r(n, heads * c) / (1 + keys), r(m, heads * c) + keys, r(n, heads * c), r(m, heads * c) + 300 * r(1, heads * c)
    got = run(build(indptr, cols, m), q, k, v, dy, heads, heads)["dq"].double()

    def by_entries(t):
        Q, Kk, V, G = (x.to(t).view(-1, heads, c) for x in (q, k, v, dy))
        j = cols.long().cuda().view(n, longest)
        s = (Q[:, None] * Kk[j]).sum(3) * c ** -0.5
        p = torch.softmax(s, 1)
        x = (G[:, None] * V[j]).sum(3)
        ds = p * (x - (p * x).sum(1, keepdim=True)) * c ** -0.5
        return (ds[..., None] * Kk[j]).sum(1).reshape(n, heads * c)

    want, other = by_entries(torch.float64), by_entries(torch.float32).double()
    assert (got - want).norm() <= 3 * (other - want).norm()


def test_on_another_stream():
    """Both passes on a stream of the caller's, with workspaces of their own; outputs and statistics are there, filled, before the calls."""
    n, m, heads, kv, c = 3000, 2500, 8, 4, 16
    indptr, cols = graph(n, m, 12, hubs=((100, 6000), (900, 2000)))
    A = build(indptr, cols, m)
    q, k, v, dy = operands(n, m, heads, kv, c, torch.bfloat16, seed=1)
    want = run(A, q, k, v, dy, heads, kv)
    side = torch.cuda.Stream()
    for _ in range(3):
        outs = [torch.full_like(t, 99.0) for t in (q, q, k, v)]
        stats = torch.full((n, heads, 2), 99.0, device="cuda")
        torch.cuda.synchronize()
        isp.attention(A, q, k, v, outs[0], heads, kv, stats=stats, stream=side)
        isp.attention_backward(A, q, k, v, stats, dy, *outs[1:], heads, kv, stream=side)
        side.synchronize()
        for t, name in zip(outs, ("y", "dq", "dk", "dv")):
            assert torch.equal(t, want[name]), name
