"""Calls of the attention and the row-wise operators that their own files' sizes do not reach: operands beyond 4 GB, offsets beyond 32 bits, forced small
work partitions, shared transposes, aliasing-free slices of one buffer, parameters left out."""
import os

import numpy as np
import pytest
import torch

import graphgen
import paper_2403_14853_amd as isp
from paper_2403_14853_amd import autograd as ag
import test_gpu_attention as att
import test_gpu_label_logprob as lab
import test_gpu_layer_norm as norm

pytestmark = pytest.mark.gpu


def with_env(env, f):
    old = {k: os.environ.get(k) for k in env}
    os.environ.update(env)
    try:
        return f()
    finally:
        for k, v in old.items():
            if v is None:
                os.environ.pop(k, None)
            else:
                os.environ[k] = v


@pytest.mark.parametrize("env", [dict(ISP_HUB_THRESHOLD="8", ISP_SEGMENT_LEN="8", ISP_BLOCK_COST="16"), dict(ISP_HUB_THRESHOLD="512", ISP_SEGMENT_LEN="768", ISP_BLOCK_COST="256"),
                                 dict(ISP_HUB_THRESHOLD="64", ISP_SEGMENT_LEN="100", ISP_BLOCK_COST="256", ISP_BANDS="4"), dict(ISP_NO_GROUPED="1")],
                         ids=["tiny", "largest", "bands", "general"])
@pytest.mark.parametrize("heads,kv,c,dtype", [(4, 4, 16, torch.float32), (8, 2, 12, torch.bfloat16), (3, 3, 20, torch.float16), (2, 1, 3, torch.float32), (1, 1, 256, torch.float16)])
def test_forced_partitions(env, heads, kv, c, dtype):
    n, m = 260, 240
    indptr, cols = att.graph(n, m, 21)
    bias = torch.randn(len(cols), generator=torch.Generator().manual_seed(1))
    bias[::7] = -np.inf
    q, k, v, dy = att.operands(n, m, heads, kv, c, dtype)
    A = with_env(env, lambda: att.build(indptr, cols, m, bias))
    att.check_all(att.run(A, q, k, v, dy, heads, kv, bias=True), att.reference(indptr, cols, q, k, v, dy, heads, kv, c ** -0.5, bias))


def test_shared_transpose_of_a_large_symmetric_pattern():
    """(More than 4 Mi entries: the transpose shares the matrix's partitions; the values differ between an entry and its mirror.)"""
    n = 40_000
    gen = np.random.default_rng(0)
    u, v = gen.integers(0, n, 2_400_000), gen.integers(0, n, 2_400_000)
    u[:300_000] = 17  # a long row and column
    keys = np.unique(np.concatenate([u * n + v, v * n + u]))
    indptr = torch.from_numpy(np.searchsorted(keys // n, np.arange(n + 1)).astype(np.int64))
    cols = torch.from_numpy((keys % n).astype(np.int32))
    assert len(cols) > 4 << 20
    bias = torch.randn(len(cols), generator=torch.Generator().manual_seed(2))
    heads, kv, c = 2, 1, 4
    q, k, v, dy = att.operands(n, n, heads, kv, c, torch.float32)
    A = att.build(indptr, cols, n, bias)
    assert A.info()["symmetric_pattern"] == 1
    att.check_all(att.run(A, q, k, v, dy, heads, kv, bias=True), att.reference(indptr, cols, q, k, v, dy, heads, kv, c ** -0.5, bias))


@pytest.mark.parametrize("heads,kv,c,dtype", [(3, 3, 20, torch.float16), (1, 1, 7, torch.bfloat16), (2, 1, 50, torch.float32), (4, 2, 3, torch.float32)])
def test_copy_of_keys_and_values(heads, kv, c, dtype):
    """Many entries per column: K and V are copied side by side where the workspace has room, with the same bits as without."""
    n, m = 8000, 600
    gen = np.random.default_rng(c)
    lengths = gen.integers(0, 700, n)
    indptr = torch.zeros(n + 1, dtype=torch.int64)
    indptr[1:] = torch.from_numpy(lengths).cumsum(0)
    cols = torch.from_numpy(gen.integers(0, m, int(indptr[-1])).astype(np.int32))
    q, k, v, dy = att.operands(n, m, heads, kv, c, dtype, gap=1, offset=1)
    A = isp.csr_build(indptr.cuda(), cols.cuda(), None, n_cols=m)
    full = isp.attention_workspace(A, heads, c, kv, dtype)
    least = (A.info()["n_segments"] * heads * (c + 2) * 4 + 255) // 256 * 256
    row = kv * c * (4 if dtype == torch.float32 else 2)
    assert full - least == m * ((2 * row + 127) // 128 * 128) and isp.attention_workspace(A, heads, c) >= full
    results = []
    for size in (full, least, full - 1):
        ws = torch.full((size,), 255, dtype=torch.uint8, device="cuda")
        results.append(isp.attention(A, q, k, v, torch.empty_like(q), heads, kv, workspace=ws))
    assert torch.equal(results[0], results[1]) and torch.equal(results[0], results[2])
    att.check(results[0], att.reference(indptr, cols, q, k, v, dy, heads, kv, c ** -0.5), "y")


def test_keys_and_values_beyond_4_gb():
    """1.2 M rows of K and V, 4 KB each (4.9 GB an operand), of which the matrix reads the first, the last and some between."""
    n, m, heads, c = 9, 1_200_000, 4, 256
    gen = torch.Generator().manual_seed(0)
    few = torch.cat([torch.arange(40), m // 2 + torch.arange(40), m - 40 + torch.arange(40)])
    lengths = torch.tensor([0, 3, 700, 20, 1, 0, 90, 400, 2])
    indptr = torch.zeros(n + 1, dtype=torch.int64)
    indptr[1:] = lengths.cumsum(0)
    pick = torch.randint(len(few), (int(indptr[-1]),), generator=gen)
    r = lambda *s: torch.randn(*s, generator=gen)
    q, dy, ks, vs = r(n, heads * c), r(n, heads * c), r(len(few), heads * c), r(len(few), heads * c)
    k, v = (torch.empty(m, heads * c, device="cuda") for _ in range(2))
    k[few.cuda()], v[few.cuda()] = ks.cuda(), vs.cuda()
    A = att.build(indptr, few[pick].int(), m)
    got = att.run(A, q.cuda(), k, v, dy.cuda(), heads, heads)
    ref = att.reference(indptr, pick.int(), q, ks, vs, dy, heads, heads, c ** -0.5)
    for name in ("dk", "dv"):
        untouched = torch.ones(m, dtype=torch.bool, device="cuda")
        untouched[few.cuda()] = False
        assert not got[name].abs().amax(1)[untouched].any()
        got[name] = got[name][few.cuda()]
    att.check_all(got, ref)


@pytest.mark.parametrize("dtype,pitch", [(torch.bfloat16, 1_500_000_001), (torch.float32, 1_100_000_003)], ids=["bfloat16", "float32"])
def test_rows_far_apart(dtype, pitch):
    """Rows whose offsets pass 2^32 bytes and 2^31 elements."""
    n, d = 3, 700
    def far(t):
        full = torch.empty(2 * pitch + d, dtype=dtype, device="cuda")
        out = torch.as_strided(full, (n, d), (pitch, 1))
        if t is not None:
            out.copy_(t)
        return out
    x, w, b, dy = norm.make(n, d, dtype, torch.float32)
    got = norm.run(far(x), w, b, dy, dx=far(None))
    ref = norm.reference(x, w, b, dy)
    for name, t in got.items():
        norm.check(t, ref, name)
    z, labels, a, e = lab.make(n, d, dtype)
    lab.check_all(lab.run(far(z), labels, 5, a, e, dz=far(None)), lab.reference(z, labels, 5, a, e))


def test_slices_of_one_buffer():
    """Queries, keys and values as column ranges of one projection's output, their gradients written into ranges of another."""
    n, heads, c = 200, 4, 12
    indptr, cols = att.graph(n, n, 5)
    for dtype in (torch.float32, torch.bfloat16):
        q, k, v, dy = att.operands(n, n, heads, heads, c, dtype)
        w = heads * c
        packed, grads = torch.cat([q, k, v], 1), torch.empty(n, 3 * w, dtype=dtype, device="cuda")
        parts, outs = packed.split(w, 1), grads.split(w, 1)
        A = att.build(indptr, cols, n)
        got = att.run(A, *parts, dy, heads, heads, outs=(torch.empty_like(q), *outs))
        att.check_all(got, att.reference(indptr, cols, q, k, v, dy, heads, heads, c ** -0.5))
        g = ag.SparseGraph(indptr.cuda(), cols.cuda())
        leaf = packed.clone().requires_grad_(True)
        y = ag.attention(g, *leaf.split(w, 1), heads)
        assert torch.equal(y, got["y"]) and torch.equal(torch.autograd.grad(y, leaf, dy)[0], grads)


def test_norm_without_parameters_through_autograd():
    x, w, b, dy = norm.make(50, 90, torch.float32, torch.float32)
    one, zero = torch.ones_like(w), torch.zeros_like(b)
    ref = norm.reference(x, one, zero, dy)
    leaf = x.clone().requires_grad_(True)
    norm.check(torch.autograd.grad(ag.layer_norm(leaf), leaf, dy)[0], ref, "dx")
    bias = b.clone().requires_grad_(True)
    y = ag.layer_norm(x, None, bias)
    norm.check(torch.autograd.grad(y, bias, dy)[0], ref, "db")
    half = norm.make(50, 90, torch.bfloat16, torch.bfloat16)
    only = half[2].clone().requires_grad_(True)
    got = torch.autograd.grad(ag.layer_norm(half[0], None, only), only, half[3])[0]
    assert got.dtype == torch.bfloat16
    norm.check(got, norm.reference(half[0], torch.ones(90), torch.zeros(90), half[3]), "db")


def test_refusals_of_the_rowwise_calls():
    x = torch.randn(6, 20, device="cuda")
    w, f = torch.ones(20, device="cuda"), torch.empty(6, device="cuda")
    y, dx = torch.empty_like(x), torch.empty_like(x)
    labels = torch.zeros(6, dtype=torch.int64, device="cuda")
    bad = [lambda: isp.layer_norm(x, y[:, 1:]), lambda: isp.layer_norm(x, y.half()), lambda: isp.layer_norm(x, y, w[1:]), lambda: isp.layer_norm(x, y, w.half()),
           lambda: isp.layer_norm(x, y, w, torch.ones(40, device="cuda")[::2]), lambda: isp.layer_norm(x, y, w, mean=f[1:]), lambda: isp.layer_norm(x.double(), y.double()),
           lambda: isp.layer_norm(x.t(), y.t()), lambda: isp.layer_norm(x[0], y[0]), lambda: isp.layer_norm(x, y, w, w.half()),
           lambda: isp.layer_norm_backward(x, x, dx, None, f), lambda: isp.layer_norm_backward(x, x[1:], dx, f, f), lambda: isp.layer_norm_backward(x, x, dx[:, 1:], f, f),
           lambda: isp.layer_norm_backward(x, x, dx, f, f, w, w.half()), lambda: isp.layer_norm_backward(x, x, dx, f, f, w, w, w, workspace=torch.empty(8, device="cuda")),
           lambda: isp.label_logprob(x, labels[1:], f), lambda: isp.label_logprob(x, labels.int(), f), lambda: isp.label_logprob(x, labels, f.double()),
           lambda: isp.label_logprob(x, labels, f, f[1:]), lambda: isp.label_logprob(x, labels, f, stats=f), lambda: isp.label_logprob(x, labels, f, top_logprob=torch.empty(6, 21, device="cuda")),
           lambda: isp.label_logprob(x, labels, f, top_index=torch.empty(6, 2, device="cuda")), lambda: isp.label_logprob(x, labels, f, top_logprob=f),
           lambda: isp.label_logprob_backward(x, labels, f, f, dx), lambda: isp.label_logprob_backward(x, labels, torch.empty(6, 2, device="cuda"), f, dx[:5]),
           lambda: ag.label_logprob(x, labels, 21), lambda: ag.label_logprob(x, labels, -1), lambda: ag.label_logprob(x, labels.int()), lambda: ag.layer_norm(x, w[1:])]
    for i, call in enumerate(bad):
        with pytest.raises(AssertionError):
            call()
            print("call %d was taken" % i)
    stats = torch.empty(6, 2, device="cuda")
    for call in (lambda: isp.layer_norm(x, y, eps=-1.0), lambda: isp.layer_norm_backward(x, x, dx, f, f, w, w, w, workspace=torch.empty(16, dtype=torch.uint8, device="cuda")),
                 lambda: isp.label_logprob(x, None, f), lambda: isp.label_logprob_backward(x, None, stats, f, dx), lambda: isp.label_logprob_backward(x, labels, stats, f, dx, d_entropy=f),
                 lambda: isp.layer_norm(x[:, :0], y[:, :0])):
        with pytest.raises(isp.IspError):
            call()
    wide = torch.randn(3, 100, device="cuda")
    with pytest.raises(isp.IspError) as err:
        isp.label_logprob(wide, labels[:3], f[:3], top_logprob=torch.empty(3, 65, device="cuda"))
    assert err.value.status_name == "ISP_EUNSUPPORTED"


def test_more_long_rows_than_a_launch_has_threads_for():
    """Rows of 1030 scores, more than 2^25 of them, whose backward has more than 2^24 workgroups' chunks: 2 x 70 GB in bf16."""
    n, c = (1 << 25) + 13, 1030
    if torch.cuda.mem_get_info()[0] < 150e9:
        pytest.skip("needs 150 GB of device memory")
    z = torch.zeros(n, c, dtype=torch.bfloat16, device="cuda")
    picks = torch.tensor([0, 1, 7, 8, (1 << 24) - 1, 1 << 24, (1 << 25) - 1, 1 << 25, (1 << 25) + 1, n - 1], device="cuda")
    gen = torch.Generator().manual_seed(0)
    rows = torch.randn(len(picks), c, generator=gen).bfloat16()
    z[picks] = rows.cuda()
    labels = torch.arange(n, device="cuda") % c
    lp, en, stats = torch.empty(n, device="cuda"), torch.empty(n, device="cuda"), torch.empty(n, 2, device="cuda")
    tv, ti = torch.empty(n, 2, device="cuda"), torch.empty(n, 2, dtype=torch.int32, device="cuda")
    isp.label_logprob(z, labels, lp, en, stats=stats, top_logprob=tv, top_index=ti)
    p = rows.double().log_softmax(1)
    at = labels[picks].cpu()
    # (two roundings of the maximum's difference and the logarithm, and a sum of 1030 terms in 32 bits: under 2^-18 of numbers below 16)
    tol = 16 * 2.0 ** -18
    assert (lp[picks].cpu().double() - p[torch.arange(len(picks)), at]).abs().max() < tol
    assert (en[picks].cpu().double() + (p.exp() * p).sum(1)).abs().max() < tol
    assert (tv[picks].cpu().double() - p.topk(2).values).abs().max() < tol
    other = torch.ones(n, dtype=torch.bool, device="cuda")
    other[picks] = False
    log_c = float(np.log(c))
    assert (lp + log_c)[other].abs().max() < tol and (en - log_c)[other].abs().max() < tol and (tv + log_c)[other].abs().max() < tol
    assert torch.equal(ti[other], torch.tensor([[0, 1]], dtype=torch.int32, device="cuda").expand(n - len(picks), 2))
    del tv, ti, other
    dz = torch.full_like(z, 7.0)
    isp.label_logprob_backward(z, labels, stats, torch.ones(n, device="cuda"), dz)
    want = torch.nn.functional.one_hot(at, c).double() - p.exp()
    assert ((dz[picks].cpu().double() - want).abs() <= 2.0 ** -8 * want.abs() + 2.0 ** -15).all()
    # every other row: 1 - 1/c at its label, -1/c elsewhere, rounded to bf16
    there, elsewhere = (torch.tensor(x).bfloat16().item() for x in (1 - 1 / c, -1 / c))
    for r0 in range(0, n, 1 << 22):
        part = dz[r0:r0 + (1 << 22)]
        skip = picks[(picks >= r0) & (picks < r0 + (1 << 22))] - r0
        got = part.gather(1, labels[r0:r0 + (1 << 22), None])[:, 0]
        got[skip] = there
        assert (got == there).all()
        part.scatter_(1, labels[r0:r0 + (1 << 22), None], elsewhere)
        part[skip] = elsewhere
        assert part.min().item() == elsewhere and part.max().item() == elsewhere


@pytest.mark.parametrize("heads,kv,c,dtype", [(4, 2, 12, torch.float32), (1, 1, 64, torch.bfloat16), (3, 3, 5, torch.float16), (8, 1, 3, torch.float32)])
def test_infinite_scores_and_values(heads, kv, c, dtype):
    """Columns of K that make scores of +inf and NaN, columns of V with an infinity and a NaN, in short rows and in split ones."""
    n, m = 300, 200
    gen = torch.Generator().manual_seed(3)
    lengths = torch.randint(1, 6, (n,), generator=gen)
    lengths[[5, 50, 150, 222]] = 3000
    indptr = torch.zeros(n + 1, dtype=torch.int64)
    indptr[1:] = lengths.cumsum(0)
    cols = torch.randint(10, m, (int(indptr[-1]),), generator=gen).int()
    r = lambda rows, heads: torch.randn(rows, heads * c, generator=gen).to(dtype).cuda()
    q, k, v = r(n, heads), r(m, kv), r(m, kv)
    q[:, ::c] = q[:, ::c].abs() + 0.5  # (the first column of each head: the sign of what K holds there is the score's)
    highest, none, inf_v, nan_v = range(4)
    seen = ({30, 5}, {40, 50}, {60, 150, 222}, {70, 222})
    for col in range(4):
        for row in seen[col]:
            cols[indptr[row] + (0 if row % 10 == 0 and lengths[row] < 10 else 800 + 700 * col)] = col
    k[highest, ::c], k[none, ::c] = np.inf, np.nan
    v[inf_v, 0::c], v[nan_v, 1::c] = np.inf, np.nan
    y = isp.attention(att.build(indptr, cols, m), q, k, v, torch.empty_like(q), heads, kv)
    kc, vc = k.clone(), v.clone()
    kc[:10], vc[:10] = 0, 0
    value, bound = att.reference(indptr, cols, q, kc, vc, q, heads, kv, c ** -0.5)["y"]
    room = bound + att.half_step(value, dtype) * 1.001 + 1e-37
    y = y.double().cpu().view(n, heads, c)
    right = ((y - value.view(n, heads, c)).abs() <= room.view(n, heads, c)).flatten(1).all(1)
    for row in range(n):
        if row in seen[highest] | seen[none]:
            assert torch.isnan(y[row]).all(), row
        elif row in seen[inf_v] | seen[nan_v]:
            bad = torch.zeros(c, dtype=torch.bool)
            bad[0], bad[1] = row in seen[inf_v], row in seen[nan_v]
            assert not torch.isfinite(y[row][:, bad]).any() and torch.isfinite(y[row][:, ~bad]).all(), row
        else:
            assert right[row], row


def test_attention_on_an_alias():
    """A second handle on the matrix, with its own copy of the cached transpose: the same bits, also beside calls on the first one; refused once stale."""
    n, m, heads, kv, c = 400, 300, 4, 2, 20
    indptr, cols = att.graph(n, m, 9)
    bias = torch.randn(len(cols), generator=torch.Generator().manual_seed(1))
    A = att.build(indptr, cols, m, bias)
    B = isp.csr_alias(A)
    q, k, v, dy = att.operands(n, m, heads, kv, c, torch.bfloat16)
    want = att.run(A, q, k, v, dy, heads, kv, bias=True)
    other = torch.cuda.Stream()
    other.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(other):
        got = att.run(B, q, k, v, dy, heads, kv, bias=True)
    again = att.run(A, q, k, v, dy, heads, kv, bias=True)
    torch.cuda.synchronize()
    for name in want:
        assert torch.equal(got[name], want[name]) and torch.equal(again[name], want[name]), name
    att.check_all(want, att.reference(indptr, cols, q, k, v, dy, heads, kv, c ** -0.5, bias))
    isp.csr_values_changed(A)
    with pytest.raises(isp.IspError):
        isp.attention(B, q, k, v, torch.empty_like(q), heads, kv)


@pytest.mark.parametrize("heads,kv,c,dtype", [(4096, 4096, 2, torch.float32), (4096, 512, 3, torch.bfloat16), (192, 3, 4, torch.float16), (64, 1, 256, torch.float32)])
def test_many_heads(heads, kv, c, dtype):
    n, m = 12, 9
    indptr, cols = att.graph(n, m, 2, hubs=((3, 1300),), longest=5)
    q, k, v, dy = att.operands(n, m, heads, kv, c, dtype)
    att.check_all(att.run(att.build(indptr, cols, m), q, k, v, dy, heads, kv), att.reference(indptr, cols, q, k, v, dy, heads, kv, c ** -0.5))
    with pytest.raises(isp.IspError):
        isp.attention(att.build(indptr, cols, m), *(torch.zeros(r, 4097 * 2, device="cuda") for r in (n, m, m, n)), 4097)


@pytest.mark.parametrize("heads,kv,c", [(4, 2, 12), (3, 3, 20), (2, 1, 64), (1, 1, 3)])
@pytest.mark.parametrize("small,large", [(2.0 ** -20, 2.0 ** 12), (2.0 ** 12, 2.0 ** -20), (2.0 ** 13, 2.0 ** 13)])
def test_fp16_at_the_ends_of_its_range(heads, kv, c, small, large):
    """Queries, or keys and values, that are subnormal in fp16, and products that fp16 could not hold: what the sums take of them is exact."""
    n, m = 300, 250
    indptr, cols = att.graph(n, m, 12)
    q, k, v, dy = (t.float() for t in att.operands(n, m, heads, kv, c, torch.float16))
    scale = 1 / (small * large * c ** 0.5)
    both = small == large  # (then the gradients of values of 2^13 each would not fit: the small ones of V and dY)
    q, k, v, dy = (t.half() for t in (q * small, k * large, v * (1 if both else large * 2.0 ** -4), dy * (2.0 ** -4 if both else small * 2.0 ** -2)))
    if not both:
        sub = q if small < large else k
        assert ((sub != 0) & (sub.abs() < 2.0 ** -14)).float().mean() > 0.95  # (one in 40 is below half the smallest number, 2^-25)
    got = att.run(att.build(indptr, cols, m), q, k, v, dy, heads, kv, scale=scale)
    ref = att.reference(indptr, cols, q, k, v, dy, heads, kv, scale)
    for name in ("y", "dq", "dk", "dv"):
        if ref[name][0].abs().max() < 6e4:  # (fp16's largest number is 65504)
            att.check(got[name], ref, name)
    assert ref["y"][0].abs().max() < 6e4 and ref["dv"][0].abs().max() < 6e4


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16], ids=["bfloat16", "float16"])
@pytest.mark.parametrize("heads,c", [(8, 8), (3, 20), (2, 50), (1, 64), (1, 256), (16, 16), (5, 9), (70, 8)])
def test_long_rows_in_16_bits(heads, c, dtype):
    """Rows and columns of 30 entries on average: eight columns to a lane in every pass; with a bias that masks entries and whole rows, and without."""
    n, m = 220, 200
    indptr, cols = att.graph(n, m, 21, longest=60)
    q, k, v, dy = att.operands(n, m, heads, heads, c, dtype)
    att.check_all(att.run(att.build(indptr, cols, m), q, k, v, dy, heads, heads), att.reference(indptr, cols, q, k, v, dy, heads, heads, c ** -0.5))
    bias = torch.randn(len(cols), generator=torch.Generator().manual_seed(2))
    bias[::3] = -np.inf
    bias[int(indptr[100]):int(indptr[104])] = -np.inf
    got = att.run(att.build(indptr, cols, m, bias), q, k, v, dy, heads, heads, bias=True)
    att.check_all(got, att.reference(indptr, cols, q, k, v, dy, heads, heads, c ** -0.5, bias))
