"""The row-wise and attention operators around the sparse products, as measurable cases.

A training step on a graph normalises the nodes' features, lets every node attend to its neighbours, and scores the nodes
against their labels.  `op` says which operator a case has:

  norm       layer norm of n rows of d columns
  labels     log probabilities of given labels, their entropy and the top alternatives, n rows of `classes` scores
  attention  softmax attention over the stored entries of a CSR matrix, `heads` query heads on `kv_heads` key heads of `dh` columns

`train` adds the gradients.  `through` says how a program calls it: the calls of the binding, with its own buffers, or the autograd
wrappers.  With `own` false everything is computed in plain torch operations.
"""
import math

import torch

own = False

DTYPE = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BYTES = {"f32": 4, "bf16": 2, "f16": 2}


def _norm(name, n, d, dtype, params, train, through="calls"):
    return {"name": name, "op": "norm", "n": n, "d": d, "dtype": dtype, "params": params, "train": train, "through": through}


def _labels(name, n, classes, dtype, train, top=0, masked=False, entropy=False, through="autograd"):
    return {"name": name, "op": "labels", "n": n, "classes": classes, "dtype": dtype, "train": train, "top": top, "masked": masked,
            "entropy": entropy, "through": through if train else "calls"}


def _attention(name, graph, n, nnz, heads, kv_heads, dh, dtype, train, bias=False, n_cols=0):
    return {"name": name, "op": "attention", "graph": graph, "n": n, "n_cols": n_cols or n, "nnz": nnz, "heads": heads,
            "kv_heads": kv_heads, "dh": dh, "dtype": dtype, "train": train, "bias": bias, "through": "autograd" if train else "calls"}


def listed():
    return [
        # hidden features of a small graph: launches and latency are all there is
        _norm("small-norm-train", 4_096, 32, "f32", "f32", True),
        # hidden features of the largest power-law graph, half-precision activations with fp32 weights
        _norm("products-norm-train-bf16", 2_449_029, 128, "bf16", "f32", True, "autograd"),
        # raw node features, 602 wide, inference
        _norm("features-norm-f16", 232_965, 602, "f16", "f16", False),
        # few wide rows: the normalisation of a wide dense block
        _norm("wide-norm-train", 4_099, 8_192, "f32", "f32", True, "autograd"),
        # node classification with 47 classes, a mid-sized graph of which a part is labelled: one training step's loss
        _labels("arxiv-labels-train", 169_343, 47, "f32", True),
        # the same on the largest graph in half precision, with an entropy term in the loss
        _labels("products-labels-train-bf16", 2_449_029, 47, "bf16", True, entropy=True),
        # scores against many candidates, some of them masked out
        _labels("candidates-labels-train-bf16", 2_053, 65_521, "bf16", True, masked=True),
        # a handful of rows scored against every candidate while serving: the best eight and the given one's log probability
        _labels("serving-top", 5, 131_071, "f32", False, top=8),
        # one attention layer of a small graph
        _attention("small-attention-train", "er", 4_096, 36_864, 4, 4, 8, "f32", True),
        # a hidden layer on a mid-sized citation graph, 8 heads of 16 columns
        _attention("arxiv-attention-train", "rmat", 169_343, 2_404_585, 8, 8, 16, "f32", True),
        # the same in half precision on a directed graph of a million nodes, half of the rows empty: grouped heads, an edge bias that masks some edges
        _attention("embed-attention-train-bf16", "rmat", 1_048_576, 16_851_165, 8, 2, 16, "bf16", True, bias=True),
        # inference over many entries, heads of a width that is no power of two
        _attention("dense-attention-f16", "rmat", 232_965, 40_000_003, 3, 3, 20, "f16", False),
    ]


MAX_NORM, MAX_SCORES, MAX_ATT = 2_449_029 * 128, 2_053 * 65_521, 16_851_165 * 128


def _log_uniform(rng, lo, hi):
    return lo if hi <= lo else int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))


def draw(rng):
    op = rng.choice(["norm", "labels", "attention"])
    dtype = rng.choice(["f32", "bf16", "f16"])
    train = rng.random() < 0.6
    through = rng.choice(["calls", "autograd"])
    if op == "norm":
        d = _log_uniform(rng, 8, 16_384)
        if rng.random() < 0.6:
            d = (d + 7) // 8 * 8
        n = _log_uniform(rng, 1, min(2_449_029, MAX_NORM // d))
        case = _norm("", n, d, dtype, rng.choice(["f32", dtype]), train, through)
    elif op == "labels":
        classes = _log_uniform(rng, 2, 131_071)
        n = _log_uniform(rng, 1, min(2_449_029, MAX_SCORES // classes))
        top = 0 if rng.random() < 0.5 else min(classes, rng.choice([1, 3, 5, 8, 16]))
        case = _labels("", n, classes, dtype, train, top, rng.random() < 0.3, rng.random() < 0.4, through)
    else:
        kv_heads = rng.choice([1, 2, 3, 4, 8])
        heads = kv_heads * rng.choice([1, 1, 1, 2, 4])
        dh = rng.choice([4, 7, 8, 12, 16, 16, 20, 32, 32, 50, 64, 64, 128])
        n = _log_uniform(rng, 500, 1_048_576)
        n_cols = n if rng.random() < 0.7 else _log_uniform(rng, max(500, n // 8), min(1_048_576, n * 8))
        nnz = n * math.exp(rng.uniform(math.log(3), math.log(min(200, math.sqrt(min(n, n_cols))))))
        nnz = int(min(nnz, 16_851_165, MAX_ATT / (heads * dh)))
        if nnz < 2 * n:
            n, n_cols = max(500, nnz // 3), max(500, min(n_cols, nnz // 3))
        case = _attention("", rng.choice(["er", "rmat", "rmat"]), n, nnz, heads, kv_heads, dh, dtype, train, rng.random() < 0.3, n_cols)
    del case["name"]
    return case


# ---- inputs ---------------------------------------------------------------------------------------------------
def _graph(n, n_cols, nnz, kind, g):
    """(indptr, indices): nnz distinct entries, uniform or R-MAT (.57 / .19 / .19 / .05, vertices relabelled), rows sorted by column."""
    keys = torch.empty(0, dtype=torch.int64, device="cuda")
    levels = max(1, math.ceil(math.log2(max(n, n_cols))))
    for turn in range(40):
        missing = nnz - keys.numel()
        if missing <= 0:
            break
        m = int(missing * (2.5 if kind == "rmat" and turn < 6 else 1.25)) + 1024
        if kind == "rmat" and turn < 6:
            u = torch.zeros(m, dtype=torch.int32, device="cuda")
            v = torch.zeros(m, dtype=torch.int32, device="cuda")
            for _ in range(levels):
                r = torch.rand(m, device="cuda", generator=g)
                u.mul_(2).add_(r >= 0.76)
                v.mul_(2).add_(((r >= 0.57) & (r < 0.76)) | (r >= 0.95))
            u, v = u % n, v % n_cols
        else:
            u = torch.randint(n, (m,), device="cuda", generator=g)
            v = torch.randint(n_cols, (m,), device="cuda", generator=g)
        keys = torch.unique(torch.cat([keys, u.long() * n_cols + v.long()]))
    if keys.numel() > nnz:
        drop = torch.randperm(keys.numel(), device="cuda", generator=g)[: keys.numel() - nnz]
        keep = torch.ones(keys.numel(), dtype=torch.bool, device="cuda")
        keep[drop] = False
        keys = keys[keep]
    u, v = keys // n_cols, keys % n_cols
    if kind == "rmat":  # popular vertices do not sit next to each other
        u = torch.randperm(n, device="cuda", generator=g)[u]
        v = torch.randperm(n_cols, device="cuda", generator=g)[v]
    keys = torch.sort(u * n_cols + v).values
    u = keys // n_cols
    indptr = torch.zeros(n + 1, dtype=torch.int64, device="cuda")
    indptr[1:] = torch.cumsum(torch.bincount(u, minlength=n), 0)
    return indptr, (keys - u * n_cols).to(torch.int32)


def _inputs(case, seed):
    """The tensors that a program has before the call."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    t = DTYPE[case["dtype"]]
    randn = lambda *shape: torch.randn(*shape, device="cuda", generator=g)
    n = case["n"]
    if case["op"] == "norm":
        d, tp = case["d"], DTYPE[case["params"]]
        # features of different scales with an offset of their own in each row, as aggregation leaves them
        s = {"x": ((0.3 + torch.rand(n, 1, device="cuda", generator=g)) * randn(n, d) + 0.5 * randn(n, 1)).to(t),
             "w": (1 + 0.2 * randn(d)).to(tp), "b": (0.1 * randn(d)).to(tp)}
        if case["train"]:
            s["dy"] = randn(n, d).to(t)
        return s
    if case["op"] == "labels":
        c = case["classes"]
        z = (2.0 * randn(n, c)).to(t)
        labels = torch.randint(c, (n,), device="cuda", generator=g)
        if case["masked"]:
            out = torch.rand(n, c, device="cuda", generator=g) < 0.1
            out.scatter_(1, labels[:, None], False)
            z.masked_fill_(out, float("-inf"))
            del out
        labels[torch.rand(n, device="cuda", generator=g) < 0.2] = -1  # unlabelled
        s = {"z": z, "labels": labels}
        if case["train"]:
            s["da"] = -torch.ones(n, device="cuda") / n + 0.1 * randn(n) / n
            s["de"] = 0.05 * randn(n) / n if case["entropy"] else None
        return s
    indptr, indices = _graph(n, case["n_cols"], case["nnz"], case["graph"], g)
    h, k, dh = case["heads"], case["kv_heads"], case["dh"]
    s = {"indptr": indptr, "indices": indices, "q": randn(n, h * dh).to(t), "k": randn(case["n_cols"], k * dh).to(t),
         "v": randn(case["n_cols"], k * dh).to(t), "bias": None}
    if case["bias"]:
        s["bias"] = randn(case["nnz"])
        s["bias"][torch.rand(case["nnz"], device="cuda", generator=g) < 0.05] = float("-inf")
    if case["train"]:
        s["dy"] = randn(n, h * dh).to(t)
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = dict(case)
    n, train, calls = case["n"], case["train"], case["through"] == "calls"
    if case["op"] == "attention" and not own:
        s["rows"] = torch.repeat_interleave(torch.arange(n, device="cuda"), s["indptr"][1:] - s["indptr"][:-1])
        s["cols"] = s["indices"].long()
    if not own:
        return s
    import paper_2403_14853_amd as isp
    from paper_2403_14853_amd import autograd as ag
    s["isp"], s["ag"] = isp, ag
    if case["op"] == "norm":
        if calls:
            s["y"], s["mean"], s["rstd"] = torch.empty_like(s["x"]), torch.empty(n, device="cuda"), torch.empty(n, device="cuda")
            if train:
                s["dx"], s["dw"], s["db"] = torch.empty_like(s["x"]), torch.empty_like(s["w"]), torch.empty_like(s["b"])
                s["ws"] = torch.empty(isp.layer_norm_backward_workspace(n, case["d"]), dtype=torch.uint8, device="cuda")
        elif train:
            for key in ("x", "w", "b"):
                s[key].requires_grad_(True)
    elif case["op"] == "labels":
        if calls:
            f = lambda *shape: torch.empty(*shape, device="cuda")
            s["a"], s["e"], s["stats"] = f(n), f(n), f(n, 2)
            s["tv"] = f(n, case["top"]) if case["top"] else None
            s["ti"] = torch.empty(n, case["top"], dtype=torch.int32, device="cuda") if case["top"] else None
            s["ws"] = torch.empty(isp.label_logprob_workspace(n, case["classes"], case["top"]), dtype=torch.uint8, device="cuda")
            s["dz"] = torch.empty_like(s["z"]) if train else None
        elif train:
            s["z"].requires_grad_(True)
    else:
        s["graph"] = ag.SparseGraph(s["indptr"], s["indices"], s["bias"], n_cols=case["n_cols"])
        if train:
            s["graph"].transpose()
            for key in ("q", "k", "v"):
                s[key].requires_grad_(True)
        else:
            s["y"] = torch.empty_like(s["q"])
            s["ws"] = torch.empty(isp.attention_workspace(s["graph"].handle, case["heads"], case["dh"]), dtype=torch.uint8, device="cuda")
    return s


# ---- the operators ----------------------------------------------------------------------------------------------
def run(s):
    case = s["case"]
    if own:
        return {"norm": _own_norm, "labels": _own_labels, "attention": _own_attention}[case["op"]](s, case)
    return {"norm": _plain_norm, "labels": _plain_labels, "attention": _plain_attention}[case["op"]](s, case)


def _own_norm(s, case):
    if case["through"] == "autograd":
        y = s["ag"].layer_norm(s["x"], s["w"], s["b"])
        if not case["train"]:
            return y
        return (y.detach(), *torch.autograd.grad(y, (s["x"], s["w"], s["b"]), s["dy"]))
    isp = s["isp"]
    if not case["train"]:
        return isp.layer_norm(s["x"], s["y"], s["w"], s["b"])
    isp.layer_norm(s["x"], s["y"], s["w"], s["b"], mean=s["mean"], rstd=s["rstd"])
    isp.layer_norm_backward(s["x"], s["dy"], s["dx"], s["mean"], s["rstd"], s["w"], s["dw"], s["db"], workspace=s["ws"])
    return s["y"], s["dx"], s["dw"], s["db"]


def _own_labels(s, case):
    if case["through"] == "autograd":
        a, e, *top = s["ag"].label_logprob(s["z"], s["labels"], top=case["top"])
        if not case["train"]:
            return (a, e, *top)
        outs, grads = ((a, e), (s["da"], s["de"])) if s["de"] is not None else ((a,), (s["da"],))
        return (a.detach(), e.detach(), *top, torch.autograd.grad(outs, s["z"], grads)[0])
    isp = s["isp"]
    isp.label_logprob(s["z"], s["labels"], s["a"], s["e"], stats=s["stats"], top_logprob=s["tv"], top_index=s["ti"], workspace=s["ws"])
    out = (s["a"], s["e"]) if s["tv"] is None else (s["a"], s["e"], s["tv"], s["ti"])
    if not case["train"]:
        return out
    isp.label_logprob_backward(s["z"], s["labels"], s["stats"], s["da"], s["dz"], entropy=s["e"], d_entropy=s["de"])
    return (*out, s["dz"])


def _own_attention(s, case):
    if case["train"]:
        y = s["ag"].attention(s["graph"], s["q"], s["k"], s["v"], case["heads"], case["kv_heads"], bias=case["bias"])
        return (y.detach(), *torch.autograd.grad(y, (s["q"], s["k"], s["v"]), s["dy"]))
    return s["isp"].attention(s["graph"].handle, s["q"], s["k"], s["v"], s["y"], case["heads"], case["kv_heads"], bias=case["bias"],
                              workspace=s["ws"])


def _plain_norm(s, case):
    x, w, b = s["x"].float(), s["w"].float(), s["b"].float()
    xc = x - x.mean(1, keepdim=True)
    rstd = ((xc * xc).mean(1, keepdim=True) + 1e-5).rsqrt()
    h = xc * rstd
    y = (h * w + b).to(s["x"].dtype)
    if not case["train"]:
        return y
    dy = s["dy"].float()
    g = dy * w
    dx = (g - g.mean(1, keepdim=True) - h * (g * h).mean(1, keepdim=True)) * rstd
    dw = (dy * h).sum(0, dtype=torch.float64)
    db = dy.sum(0, dtype=torch.float64)
    return y, dx.to(s["x"].dtype), dw.to(s["w"].dtype), db.to(s["b"].dtype)


def _plain_labels(s, case):
    z, labels = s["z"].float(), s["labels"]
    m = z.max(1, keepdim=True).values
    e = (z - m).exp()
    total = e.sum(1, keepdim=True)
    lp = z - (m + total.log())
    p = e / total
    plp = torch.where(p > 0, p * lp, torch.zeros_like(p))
    entropy = -plp.sum(1)
    has = (labels >= 0) & (labels < case["classes"])
    at = labels.clamp(0, case["classes"] - 1)[:, None]
    logprob = torch.where(has, lp.gather(1, at)[:, 0], torch.zeros_like(entropy))
    out = [logprob, entropy]
    if case["top"]:
        left = z.clone()
        values, picks = [], []
        for _ in range(case["top"]):  # the largest that is left, of equal ones the first
            best = left.max(1, keepdim=True).values
            pick = (left == best).to(torch.uint8).argmax(1, keepdim=True)
            values.append(lp.gather(1, pick))
            picks.append(pick)
            left.scatter_(1, pick, float("-inf"))
        out += [torch.cat(values, 1), torch.cat(picks, 1).to(torch.int32)]
    if case["train"]:
        da = torch.where(has, s["da"], torch.zeros_like(s["da"]))
        dz = p * -da[:, None]
        dz.scatter_add_(1, at, da[:, None])
        if s["de"] is not None:
            dz -= s["de"][:, None] * (plp + p * entropy[:, None])
        out.append(dz.to(s["z"].dtype))
    return tuple(out)


def _plain_attention(s, case):
    h, k, dh, n = case["heads"], case["kv_heads"], case["dh"], case["n"]
    rows, cols, t = s["rows"], s["cols"], s["q"].dtype
    scale = dh ** -0.5
    y = torch.zeros(n, h * dh, device="cuda")
    train = case["train"]
    if train:
        dq = torch.zeros_like(y)
        dk, dv = (torch.zeros(case["n_cols"], k * dh, device="cuda") for _ in range(2))
    for i in range(h):
        a, b = slice(i * dh, (i + 1) * dh), slice(i // (h // k) * dh, (i // (h // k) + 1) * dh)
        q, kk, v = s["q"][:, a].float(), s["k"][:, b].float(), s["v"][:, b].float()
        z = (q[rows] * kk[cols]).sum(1) * scale
        if s["bias"] is not None:
            z = z + s["bias"]
        m = torch.full((n,), float("-inf"), device="cuda").scatter_reduce(0, rows, z, "amax")
        m = torch.where(m == float("-inf"), torch.zeros_like(m), m)
        e = (z - m[rows]).exp()
        total = torch.zeros(n, device="cuda").index_add_(0, rows, e)
        p = e / torch.where(total > 0, total, torch.ones_like(total))[rows]
        o = torch.zeros(n, dh, device="cuda").index_add_(0, rows, p[:, None] * v[cols])
        y[:, a] = o
        if train:
            dy = s["dy"][:, a].float()
            ds = p * ((dy[rows] * v[cols]).sum(1) - (dy * o).sum(1)[rows]) * scale
            dq[:, a] = torch.zeros(n, dh, device="cuda").index_add_(0, rows, ds[:, None] * kk[cols])
            dk[:, b] += torch.zeros(case["n_cols"], dh, device="cuda").index_add_(0, cols, ds[:, None] * q[rows])
            dv[:, b] += torch.zeros(case["n_cols"], dh, device="cuda").index_add_(0, cols, p[:, None] * dy[rows])
    return (y.to(t), dq.to(t), dk.to(t), dv.to(t)) if train else y.to(t)


# ---- what one pass cannot do without -----------------------------------------------------------------------------
def work(case):
    b, n = BYTES[case["dtype"]], case["n"]
    if case["op"] == "norm":
        d, bp = case["d"], BYTES[case["params"]]
        if not case["train"]:
            return {"bytes": 2 * n * d * b + 2 * d * bp, "flops": 8 * n * d}
        return {"bytes": 4 * n * d * b + 4 * d * bp, "flops": 24 * n * d}  # x, dy in; y, dx out
    if case["op"] == "labels":
        c = case["classes"]
        out = 8 * n + 8 * n + 8 * n * case["top"]
        if not case["train"]:
            return {"bytes": n * c * b + out, "flops": 6 * n * c}
        return {"bytes": 2 * n * c * b + out + 4 * n, "flops": 12 * n * c}
    h, k, dh, m, e = case["heads"], case["kv_heads"], case["dh"], case["n_cols"], case["nnz"]
    entry = 8 if case["bias"] else 4
    csr = 8 * (n + 1) + entry * e
    rows, cols = n * h * dh * b, m * k * dh * b
    if not case["train"]:
        return {"bytes": csr + 2 * rows + 2 * cols, "flops": 4 * e * h * dh}
    return {"bytes": 2 * csr + 4 * rows + 4 * cols, "flops": 14 * e * h * dh}  # q, dy, k, v in; y, dq, dk, dv out


# ---- the definitions in 64 bits ----------------------------------------------------------------------------------
def exact(case, seed):
    s = _inputs(case, seed)
    return {"norm": _exact_norm, "labels": _exact_labels, "attention": _exact_attention}[case["op"]](s, case)


def _slabs(n, width):
    step = max(1, (1 << 26) // max(width, 1))
    return [slice(i, min(i + step, n)) for i in range(0, n, step)]


def _exact_norm(s, case):
    n, d = s["x"].shape
    w, b = s["w"].double(), s["b"].double()
    y = torch.empty(n, d, dtype=torch.float64, device="cuda")
    dx = torch.empty_like(y) if case["train"] else None
    dw, db = torch.zeros_like(w), torch.zeros_like(b)
    for r in _slabs(n, d):
        x = s["x"][r].double()
        var, mean = torch.var_mean(x, 1, correction=0, keepdim=True)
        sigma = torch.sqrt(var + 1e-5)
        hat = (x - mean) / sigma
        y[r] = torch.addcmul(b, hat, w)
        if case["train"]:
            up = s["dy"][r].double()
            dw += torch.einsum("ij,ij->j", up, hat)
            db += up.sum(0)
            up = up * w
            # the projection of the upstream gradient off the constant and off the normalised row
            along = (up * hat).sum(1, keepdim=True) / d
            dx[r] = (up - up.sum(1, keepdim=True) / d - along * hat) / sigma
    return (y, dx, dw, db) if case["train"] else y


def _exact_labels(s, case):
    n, c = s["z"].shape
    top = case["top"]
    logprob, entropy = (torch.empty(n, dtype=torch.float64, device="cuda") for _ in range(2))
    tv = torch.empty(n, top, dtype=torch.float64, device="cuda")
    ti = torch.empty(n, top, dtype=torch.int32, device="cuda")
    dz = torch.empty(n, c, dtype=torch.float64, device="cuda") if case["train"] else None
    for r in _slabs(n, c):
        z, y = s["z"][r].double(), s["labels"][r]
        lp = torch.log_softmax(z, 1)
        p = lp.exp()
        entropy[r] = torch.special.entr(p).sum(1)
        known = torch.logical_and(y >= 0, y < c)
        hot = torch.zeros_like(z)
        hot[known.nonzero()[:, 0], y[known]] = 1
        logprob[r] = torch.where(hot > 0, lp, 0.0).sum(1)
        if top:
            order = torch.sort(z, dim=1, descending=True, stable=True).indices[:, :top]
            ti[r] = order.to(torch.int32)
            tv[r] = torch.take_along_dim(lp, order, 1)
        if case["train"]:
            a = torch.where(known, s["da"][r].double(), 0.0)[:, None]
            grad = a * (hot - p)
            if s["de"] is not None:  # dS / dz_j = -p_j (log p_j + S)
                grad = grad + s["de"][r].double()[:, None] * (torch.special.entr(p) - p * entropy[r][:, None])
            dz[r] = grad
    out = (logprob, entropy) + ((tv, ti) if top else ())
    return out + ((dz,) if case["train"] else ())


def _exact_attention(s, case):
    n, m, h, k, dh = case["n"], case["n_cols"], case["heads"], case["kv_heads"], case["dh"]
    indptr, cols = s["indptr"], s["indices"].long()
    lengths = torch.diff(indptr)
    rows = torch.repeat_interleave(torch.arange(n, device="cuda"), lengths)
    heads = lambda x, c: x.double().reshape(x.shape[0], c, dh)
    q, kk, v = heads(s["q"], h), heads(s["k"], k), heads(s["v"], k)
    y = torch.zeros_like(q)
    train = case["train"]
    grads = [torch.zeros_like(t) for t in (q, kk, v)] if train else None
    dy = heads(s["dy"], h) if train else None
    spans = _slabs(case["nnz"], 4 * dh)
    for i in range(h):
        j = i * k // h
        z = torch.cat([torch.linalg.vecdot(q[rows[e], i], kk[cols[e], j]) for e in spans]) / math.sqrt(dh)
        if s["bias"] is not None:
            z = z + s["bias"].double()
        peak = torch.segment_reduce(z, "max", offsets=indptr, initial=-1e300).clamp(min=-1e300)
        z = torch.exp(z - peak[rows])
        norm = torch.segment_reduce(z, "sum", offsets=indptr, initial=0)
        p = torch.where(z > 0, z / norm[rows], 0.0)
        for e in spans:
            y[:, i].index_add_(0, rows[e], p[e, None] * v[cols[e], j])
        if not train:
            continue
        flat = torch.linalg.vecdot(dy[:, i], y[:, i])
        for e in spans:
            r, c = rows[e], cols[e]
            ds = (p[e] * (torch.linalg.vecdot(dy[r, i], v[c, j]) - flat[r]) / math.sqrt(dh))[:, None]
            grads[0][:, i].index_add_(0, r, ds * kk[c, j])
            grads[1][:, j].index_add_(0, c, ds * q[r, i])
            grads[2][:, j].index_add_(0, c, p[e, None] * dy[r, i])
    y = y.reshape(n, h * dh)
    return (y, *(t.reshape(t.shape[0], -1) for t in grads)) if train else y
