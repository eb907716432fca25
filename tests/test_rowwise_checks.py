"""What the row-wise operators and the attention refuse, on the CPU: arguments are looked at before any device work."""
import ctypes

import numpy as np
import pytest
import torch

import paper_2403_14853_amd as isp
from paper_2403_14853_amd import autograd as ag
from paper_2403_14853_amd import binding

P = 0x1000  # (an address that nothing reads)
EINVAL, EUNSUPPORTED = 1, 5


@pytest.fixture(scope="module")
def lib():
    return isp.load_library()


def test_layer_norm_at_the_c_boundary(lib):
    f = lambda X=P, ldx=8, n=4, d=8, t=0, w=P, b=P, pt=0, eps=1e-5, Y=P, ldy=8: lib.isp_layer_norm(X, ldx, n, d, t, w, b, pt, eps, Y, ldy, None, None, None)
    for bad in (dict(X=None), dict(Y=None), dict(ldx=7), dict(ldy=7), dict(d=0), dict(n=-1), dict(eps=-1.0), dict(eps=float("nan"))):
        assert f(**bad) == EINVAL, bad
    for bad in (dict(t=3), dict(t=-1), dict(pt=1), dict(t=1, pt=2), dict(d=2 ** 31 - 1, ldx=2 ** 31, ldy=2 ** 31)):
        assert f(**bad) == EUNSUPPORTED, bad
    assert f(n=0, X=None, Y=None) == 0
    need = ctypes.c_size_t()
    assert lib.isp_layer_norm_backward_workspace(4, 8, None) == EINVAL
    assert lib.isp_layer_norm_backward_workspace(-1, 8, ctypes.byref(need)) == EINVAL
    assert lib.isp_layer_norm_backward_workspace(4, 8, ctypes.byref(need)) == 0 and need.value > 0
    g = lambda X=P, dY=P, ldg=8, mean=P, rstd=P, dX=P, lddx=8, ws=P, bytes_=need.value, d=8, t=0: lib.isp_layer_norm_backward(
        X, 8, dY, ldg, 4, d, t, P, 0, mean, rstd, dX, lddx, P, P, ws, bytes_, None)
    for bad in (dict(X=None), dict(dY=None), dict(ldg=7), dict(mean=None), dict(rstd=None), dict(lddx=7), dict(ws=None), dict(ws=P + 8),
                dict(bytes_=need.value - 1), dict(d=0)):
        assert g(**bad) == EINVAL, bad
    assert g(t=9) == EUNSUPPORTED


def test_label_logprob_at_the_c_boundary(lib):
    need = ctypes.c_size_t()
    assert lib.isp_label_logprob_workspace(4, 8, 0, None) == EINVAL
    assert lib.isp_label_logprob_workspace(4, 8, 9, ctypes.byref(need)) == EINVAL
    assert lib.isp_label_logprob_workspace(4, 8, -1, ctypes.byref(need)) == EINVAL
    assert lib.isp_label_logprob_workspace(4, 100, 65, ctypes.byref(need)) == EUNSUPPORTED
    assert lib.isp_label_logprob_workspace(4000, 100, 64, ctypes.byref(need)) == 0 and need.value == 0
    assert lib.isp_label_logprob_workspace(2, 100_000, 8, ctypes.byref(need)) == 0 and need.value > 0
    f = lambda Z=P, ldz=8, n=4, c=8, t=0, labels=P, lp=P, top=0, ws=None, bytes_=0: lib.isp_label_logprob(
        Z, ldz, n, c, t, labels, lp, P, P, top, P, P, ws, bytes_, None)
    for bad in (dict(Z=None), dict(ldz=7), dict(n=-1), dict(c=0), dict(labels=None), dict(top=9), dict(top=-1), dict(n=2, c=100_000, ldz=100_000, top=8),
                dict(n=2, c=100_000, ldz=100_000, top=8, ws=P + 8, bytes_=1 << 30), dict(n=2, c=100_000, ldz=100_000, top=8, ws=P, bytes_=need.value - 1)):
        assert f(**bad) == EINVAL, bad
    assert f(t=7) == EUNSUPPORTED and f(c=100, ldz=100, top=65) == EUNSUPPORTED
    assert f(n=0, Z=None, labels=None) == 0
    g = lambda Z=P, ldz=8, labels=P, stats=P, ent=P, da=P, de=P, dZ=P, lddz=8, n=4: lib.isp_label_logprob_backward(
        Z, ldz, n, 8, 0, labels, stats, ent, da, de, dZ, lddz, None)
    for bad in (dict(Z=None), dict(ldz=7), dict(labels=None), dict(stats=None), dict(ent=None), dict(dZ=None), dict(lddz=7), dict(n=-1)):
        assert g(**bad) == EINVAL, bad


def test_attention_at_the_c_boundary(lib):
    need = ctypes.c_size_t()
    assert lib.isp_attention_workspace(None, 2, 2, 8, 0, ctypes.byref(need)) == EINVAL and lib.isp_attention_workspace(None, 2, 2, 8, 0, None) == EINVAL
    assert lib.isp_attention_backward_workspace(None, 2, 2, 8, ctypes.byref(need)) == EINVAL
    assert lib.isp_attention(None, P, 16, P, 16, P, 16, 2, 2, 8, 1.0, 0, 0, P, 16, None, None, 0, None) == EINVAL
    assert lib.isp_attention_backward(None, P, 16, P, 16, P, 16, 2, 2, 8, 1.0, 0, 0, P, P, 16, P, 16, P, 16, P, 16, None, 0, None) == EINVAL


NOT_TENSORS = [np.zeros((4, 8), np.float32), [[1.0, 2.0]], "x", 3.0]


def cell(nat):
    return nat.cell(0, 4, 4, 6)  # a NULL handle of a 4 x 4 matrix


@pytest.mark.parametrize("x", NOT_TENSORS, ids=lambda x: type(x).__name__)
def test_operands_must_be_tensors(x):
    nat, t = binding._native(), torch.zeros(4, 8)
    for call in (lambda: nat.layer_norm(x, t, None, None, None, None, 1e-5, 0), lambda: nat.layer_norm(t, x, None, None, None, None, 1e-5, 0),
                 lambda: nat.layer_norm(t, t, x, None, None, None, 1e-5, 0), lambda: nat.layer_norm_backward(t, x, t, t, t, None, None, None, None, 0),
                 lambda: nat.label_logprob(x, t, t, None, None, None, None, None, 0), lambda: nat.label_logprob(t, x, t, None, None, None, None, None, 0),
                 lambda: nat.label_logprob_backward(x, t, t, t, t, t, t, 0), lambda: ag.layer_norm(x), lambda: ag.layer_norm(t, x),
                 lambda: ag.label_logprob(x, t), lambda: ag.label_logprob(t, x), lambda: nat.attention(cell(nat), x, t, t, t, None, None, 1, 1, 1.0, 0, 0),
                 lambda: nat.attention(cell(nat), t, t, t, x, None, None, 1, 1, 1.0, 0, 0), lambda: nat.attention(cell(nat), t, t, t, t, x, None, 1, 1, 1.0, 0, 0),
                 lambda: nat.attention_backward(cell(nat), t, t, t, x, t, None, None, None, None, 1, 1, 1.0, 0, 0),
                 lambda: nat.ag_attention(nat.graph(cell(nat), object(), None), t, x, t, 1, 1, None, 0)):
        with pytest.raises(TypeError):
            call()


def test_cpu_tensors_are_refused():
    t, y = torch.zeros(4, 8), torch.zeros(4, dtype=torch.int64)
    for call in (lambda: isp.layer_norm(t, t), lambda: isp.layer_norm_backward(t, t, t, t[:, 0], t[:, 0], workspace=t), lambda: ag.layer_norm(t),
                 lambda: isp.label_logprob(t, y, t[:, 0]), lambda: isp.label_logprob_backward(t, y, t, t[:, 0], t), lambda: ag.label_logprob(t, y),
                 lambda: binding._native().attention(cell(binding._native()), t, t, t, t, None, None, 1, 1, 1.0, 0, 0),
                 lambda: binding._native().ag_attention(binding._native().graph(cell(binding._native()), object(), None), t, t, t, 1, 1, None, 0)):
        with pytest.raises(AssertionError):
            call()


def test_forward_mode_is_refused():
    import torch.autograd.forward_ad as fw
    t, y = torch.zeros(4, 8), torch.zeros(4, dtype=torch.int64)
    with fw.dual_level():
        x = fw.make_dual(t, torch.ones(4, 8))
        w = fw.make_dual(t[0], torch.ones(8))
        for call in (lambda: ag.layer_norm(x), lambda: ag.layer_norm(t, w), lambda: ag.layer_norm(t, None, w), lambda: ag.label_logprob(x, y),
                     lambda: binding._native().ag_attention(binding._native().graph(cell(binding._native()), object(), None), t, x, t, 1, 1, None, 0)):
            with pytest.raises(NotImplementedError):
                call()


def test_tensors_without_storage_raise():
    from torch._subclasses.fake_tensor import FakeTensorMode
    nat = binding._native()
    with FakeTensorMode():
        X = torch.empty(3, 4, 8, device="cuda")
        for call in (lambda x: nat.layer_norm(x, x, None, None, None, None, 1e-5, 0), lambda x: nat.label_logprob(x, None, None, None, None, None, None, None, 0),
                     lambda x: ag.layer_norm(x), lambda x: ag.label_logprob(x, x)):
            with pytest.raises((RuntimeError, AssertionError)):
                torch.func.vmap(call)(X)
