"""The operators' refusals, on the CPU: every bad argument is found on the
host, before anything reaches a GPU."""
import ctypes

import pytest

from paper_2607_01455_gb300 import ember as E
from paper_2607_01455_gb300.build import build_library

P = 1 << 20  # an address that is never used
OK, BAD, ALIGN, DTYPE, WS, UNSUP = (E.EMBER_OK, E.EMBER_ERR_INVALID_ARG, E.EMBER_ERR_ALIGNMENT, E.EMBER_ERR_DTYPE,
                                    E.EMBER_ERR_WORKSPACE, E.EMBER_ERR_UNSUPPORTED)
F32, BF = E.EMBER_F32, E.EMBER_BF16


@pytest.fixture(scope="module", autouse=True)
def lib():
    build_library()
    return E.lib()


NORM = dict(x=P, ldx=64, xtype=BF, residual=P, ldr=64, rtype=F32, gain=P, gtype=F32, T=4, D=64, eps=1e-6, h=P, ldh=64,
            y=P, ldy=64, stream=None)
QUANT = dict(x=P, ldx=64, xtype=BF, residual=P, ldr=64, rtype=F32, gain=P, gtype=F32, T=4, D=64, eps=1e-6, h=P, ldh=64,
             q=P, ldq=64, scales=P, stream=None)
ROWS = dict(x=P, ldx=64, xtype=BF, T=4, D=64, q=P, ldq=64, scales=P, stream=None)
DEQ = dict(q=P, ldq=64, scales=P, T=4, D=64, y=P, ldy=64, ytype=BF, stream=None)
BACK = dict(dy=P, lddy=64, h=P, ldh=64, dres=P, lddres=64, type=BF, gain=P, gtype=F32, T=4, D=64, eps=1e-6, dx=P,
            lddx=64, dgain=P, workspace=P, bytes=1 << 30, stream=None)
MM = dict(xq=P, ldx=64, xs=P, wq=P, ldw=64, ws=P, T=4, V=100, K=64, out=P, ldo=100, otype=BF, workspace=P,
          bytes=1 << 30, status=P, stream=None)
LOSS = dict(logits=P, ldz=100, ztype=BF, targets=P, idtype=E.EMBER_I64, weights=P, ignore=-100, mean=1, T=4, V=100,
            loss=P, nll=P, dlogits=P, ldd=100, dtype=BF, workspace=P, bytes=1 << 20, status=P, stream=None)

CASES = [("ember_rmsnorm", NORM, kw, st) for kw, st in [
    (dict(x=None), BAD), (dict(y=None), BAD), (dict(h=None), BAD), (dict(residual=None), BAD), (dict(T=-1), BAD),
    (dict(D=0), BAD), (dict(ldx=63), BAD), (dict(ldy=63), BAD), (dict(ldr=63), BAD), (dict(ldh=63), BAD),
    (dict(eps=-1.0), BAD), (dict(eps=float("nan")), BAD), (dict(eps=float("inf")), BAD), (dict(xtype=2), DTYPE),
    (dict(rtype=-1), DTYPE), (dict(gtype=9), DTYPE), (dict(x=P + 1), ALIGN), (dict(residual=P + 2), ALIGN),
    (dict(gain=P + 2), ALIGN), (dict(y=P + 1), ALIGN), (dict(ldx=1 << 60), BAD),
    (dict(D=32769, ldx=32769, ldr=32769, ldh=32769, ldy=32769), UNSUP), (dict(T=1 << 31), UNSUP), (dict(T=0), OK)]]
CASES += [("ember_rmsnorm_quant", QUANT, kw, st) for kw, st in [
    (dict(q=None), BAD), (dict(scales=None), BAD), (dict(ldq=63), BAD), (dict(scales=P + 2), ALIGN),
    (dict(xtype=5), DTYPE), (dict(x=None), BAD), (dict(T=0), OK)]]
CASES += [("ember_quantize_rows", ROWS, kw, st) for kw, st in [
    (dict(x=None), BAD), (dict(q=None), BAD), (dict(scales=None), BAD), (dict(ldq=8), BAD), (dict(xtype=3), DTYPE),
    (dict(D=40000, ldx=40000, ldq=40000), UNSUP), (dict(scales=P + 1), ALIGN), (dict(T=0), OK)]]
CASES += [("ember_dequantize_rows", DEQ, kw, st) for kw, st in [
    (dict(y=None), BAD), (dict(q=None), BAD), (dict(scales=None), BAD), (dict(ldq=8), BAD), (dict(ldy=8), BAD),
    (dict(ytype=3), DTYPE), (dict(y=P + 1), ALIGN), (dict(T=0), OK)]]
CASES += [("ember_rmsnorm_backward", BACK, kw, st) for kw, st in [
    (dict(dy=None), BAD), (dict(h=None), BAD), (dict(dx=None), BAD), (dict(dgain=None), BAD), (dict(lddy=63), BAD),
    (dict(lddres=63), BAD), (dict(type=2), DTYPE), (dict(gtype=2), DTYPE), (dict(workspace=None), WS),
    (dict(bytes=16), WS), (dict(workspace=P + 8), ALIGN), (dict(dgain=P + 2), ALIGN), (dict(eps=-1e-9), BAD),
    (dict(D=32769, lddy=32769, ldh=32769, lddres=32769, lddx=32769), UNSUP)]]
CASES += [("ember_matmul_quant", MM, kw, st) for kw, st in [
    (dict(xq=None), BAD), (dict(xs=None), BAD), (dict(wq=None), BAD), (dict(ws=None), BAD), (dict(out=None), BAD),
    (dict(status=None), BAD), (dict(ldx=63), BAD), (dict(ldw=63), BAD), (dict(ldo=99), BAD), (dict(V=0), BAD),
    (dict(K=0), BAD), (dict(T=-1), BAD), (dict(otype=2), DTYPE), (dict(out=P + 1), ALIGN), (dict(xs=P + 2), ALIGN),
    (dict(workspace=None), WS), (dict(T=1 << 31), UNSUP), (dict(K=32769, ldx=32769, ldw=32769), UNSUP),
    (dict(T=0), OK)]]
CASES += [("ember_softmax_loss", LOSS, kw, st) for kw, st in [
    (dict(logits=None), BAD), (dict(targets=None), BAD), (dict(loss=None), BAD), (dict(nll=None), BAD),
    (dict(status=None), BAD), (dict(ldz=99), BAD), (dict(ldd=99), BAD), (dict(mean=2), BAD), (dict(V=0), BAD),
    (dict(T=-1), BAD), (dict(ztype=2), DTYPE), (dict(dtype=2), DTYPE), (dict(idtype=2), DTYPE),
    (dict(targets=P + 4), ALIGN), (dict(logits=P + 1), ALIGN), (dict(weights=P + 2), ALIGN),
    (dict(dlogits=P + 1), ALIGN), (dict(workspace=None), WS), (dict(bytes=0), WS), (dict(T=1 << 31), UNSUP),
    (dict(V=1 << 31, ldz=1 << 31, ldd=1 << 31), UNSUP)]]


@pytest.mark.parametrize("name,base,kw,status", CASES, ids=lambda v: v if isinstance(v, str) else None)
def test_refusals(lib, name, base, kw, status):
    assert getattr(lib, name)(*{**base, **kw}.values()) == status, kw


def lists(ptrs, numel, types):
    n = len(ptrs)
    return ((ctypes.c_void_p * n)(*ptrs), (ctypes.c_int64 * n)(*numel), (ctypes.c_int * n)(*types))


@pytest.mark.parametrize("ptrs,numel,types,status", [
    ([P, P], [4, -1], [F32, F32], BAD), ([P, None], [4, 4], [F32, F32], BAD), ([P, P], [4, 4], [F32, 2], DTYPE),
    ([P, P + 2], [4, 4], [F32, F32], ALIGN), ([P, P + 1], [4, 4], [F32, BF], ALIGN),
    ([P, P], [1 << 43, 4], [F32, F32], UNSUP), ([P, P], [1 << 42, 1], [F32, F32], UNSUP)])
def test_clip_refuses_bad_lists(lib, ptrs, numel, types, status):
    p, n, t = lists(ptrs, numel, types)
    assert lib.ember_grad_norm(2, p, n, t, P, P, 1 << 20, None) == status
    assert lib.ember_clip_grads(2, p, p, n, t, 1.0, 1e-6, P, P, 1 << 20, None) == status


def test_clip_refusals(lib):
    p, n, t = lists([P], [4], [F32])
    call = lambda n_=1, out=p, max_norm=1.0, eps=1e-6, norm=P, ws=P, nb=1 << 20: \
        lib.ember_clip_grads(n_, p, out, n, t, max_norm, eps, norm, ws, nb, None)  # noqa: E731
    assert call(n_=-1) == BAD and call(out=None) == BAD and call(max_norm=-1.0) == BAD
    assert call(max_norm=float("nan")) == BAD and call(eps=-1.0) == BAD and call(norm=None) == BAD
    assert call(norm=P + 2) == ALIGN and call(ws=P + 8) == ALIGN and call(ws=None) == WS and call(nb=8) == WS
    assert lib.ember_grad_norm(1, None, n, t, P, P, 1 << 20, None) == BAD


def test_status_word_refusals(lib):
    assert lib.ember_status_init(None, None) == BAD and lib.ember_status_read(None, None) == BAD
    assert lib.ember_status_init(P + 2, None) == ALIGN and lib.ember_status_read(P + 1, None) == ALIGN


def test_workspace_sizes(lib):
    assert lib.ember_rmsnorm_backward_workspace_bytes(4096, 4096) >= 4 * 4096 * 152
    assert lib.ember_rmsnorm_backward_workspace_bytes(-1, 4) == 0
    assert lib.ember_rmsnorm_backward_workspace_bytes(4, 40000) == 0
    assert lib.ember_softmax_loss_workspace_bytes(-1) == 0 and lib.ember_softmax_loss_workspace_bytes(5) > 0
    assert lib.ember_matmul_quant_workspace_bytes(4, 0, 4) == 0 and lib.ember_matmul_quant_workspace_bytes(4, 4, 4) > 0
    assert lib.ember_clip_workspace_bytes(-1) == 0
    assert lib.ember_clip_workspace_bytes(5000) > lib.ember_clip_workspace_bytes(5) > 0


def test_the_python_layer_names_what_it_refuses():
    torch = pytest.importorskip("torch")
    from paper_2607_01455_gb300 import Ops
    with pytest.raises(E.EmberError, match="CUDA device"):
        Ops("cpu")
    o = Ops.__new__(Ops)  # the checks themselves touch no GPU
    o.device, o._index = torch.device("cpu"), -1  # what a CPU tensor's get_device() gives
    z = torch.zeros(4, 8)
    assert o._matrix("f", "x", z, (torch.float32,))[1] == 8
    assert o._matrix("f", "x", z[:, 2:5], (torch.float32,))[1] == 8
    for bad in (z.T, z[:, ::2], z[0], z[:1].expand(4, 8), z[:, :0]):
        with pytest.raises(ValueError, match="x has"):
            o._matrix("f", "x", bad, (torch.float32,))
    with pytest.raises(E.EmberError) as ex:
        o._matrix("f", "x", z, (torch.bfloat16,))
    assert ex.value.status == DTYPE
    with pytest.raises(ValueError, match="shape"):
        o._matrix("f", "x", z, (torch.float32,), (8, 4))
    with pytest.raises(ValueError, match="not 3 in a row"):
        o._vector("f", "w", z[0], 3, (torch.float32,))
    with pytest.raises(ValueError, match="contiguous"):
        o._list("f", [z.T], None)
    with pytest.raises(ValueError, match="outputs"):
        o._list("f", [z], [])
    with pytest.raises(ValueError, match="output of shape"):
        o._list("f", [z], [z[:2]])
    with pytest.raises(E.EmberError) as ex:
        o._list("f", [z.double()], None)
    assert ex.value.status == DTYPE


def test_binding_passes_on_what_is_not_on_its_device():
    """Arguments that are no CUDA tensors are left to the module, which names what is wrong."""
    import torch

    from paper_2607_01455_gb300 import ember
    b = ember.ops_binding()
    x, n = torch.zeros(2, 8), torch.zeros(8)
    q, s, y = torch.zeros(2, 8, dtype=torch.int8), torch.zeros(2), torch.zeros(2, dtype=torch.int64)
    big = 1 << 30
    assert b.rmsnorm(0, x, n, None, 1e-6, None, None) is None
    assert b.rmsnorm(0, None, n, None, 1e-6, None, None) is None
    assert b.rmsnorm_quant(0, x, n, None, 1e-6, None) is None
    assert b.rmsnorm_backward(0, 0, big, x, x, n, 1e-6, None, None) is None
    assert b.dequantize_rows(0, q, s, 0, None) is None
    assert b.matmul_quant(0, 0, big, 0, q, s, q, s, 0, None) is None
    assert b.softmax_loss(0, 0, big, 0, x, y, None, -100, True, 0, None) is None
    assert b.grad_norm(0, 0, big, [x]) is None
    assert b.clip_grads(0, 0, big, [x], 1.0, 1e-6, None) is None
    assert b.clip_grads(0, 0, big, [x], 1.0, 1e-6, [x, x]) is None
    with pytest.raises(TypeError):
        b.rmsnorm(0, x)
    with pytest.raises(TypeError):
        b.bind(1)
