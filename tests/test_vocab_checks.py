"""Refusals of the embedding lookup, the softmax cross entropy and the distillation over a vocabulary, on the host
before anything is launched: the C ABI's codes, and the binding's sizes and types (no GPU: only calls that are
refused, or that have nothing to do)."""
import ctypes
import os

import pytest
import torch

import paper_2103_00959_amd as cg

OK, INVALID, DTYPE, TOO_LARGE = 0, 1, 2, 6
FAKE, ODD = ctypes.c_void_p(0x1000), ctypes.c_void_p(0x1010)
F32, BF16, F16 = 0, 1, 2
INF = float("inf")


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(cg.LIB_PATH):
        from paper_2103_00959_amd import build
        build.build(verbose=False)
    return cg.lib()


def test_embedding_validation(L):
    def E(n=4, V=10, k=8, table=FAKE, dt=F32, index=FAKE, Y=FAKE, ydt=BF16):
        return L.cogdl_embedding(n, V, k, table, dt, index, 1.0, Y, ydt, None)

    assert E(n=-1) == INVALID and E(V=0) == INVALID and E(k=-1) == INVALID
    assert E(dt=3) == DTYPE and E(ydt=-1) == DTYPE
    assert E(n=cg.MAX_NNZ + 1) == TOO_LARGE and E(k=2 ** 22 + 1) == TOO_LARGE and E(V=2 ** 31 - 1) == TOO_LARGE
    assert E(table=None) == INVALID and E(index=None) == INVALID and E(Y=None) == INVALID
    assert E(n=0, table=None, index=None, Y=None) == OK and E(k=0, table=None, Y=None) == OK


def test_embedding_backward_validation(L):
    size = ctypes.c_size_t()
    S = L.cogdl_embedding_backward_workspace
    assert S(1000, 50, 16, ctypes.byref(size)) == OK and size.value > 0
    need = size.value
    assert S(1000, 50, 16, None) == INVALID and S(-1, 50, 16, ctypes.byref(size)) == INVALID
    assert S(1000, 0, 16, ctypes.byref(size)) == INVALID and S(1000, 50, 2 ** 23, ctypes.byref(size)) == TOO_LARGE
    assert S(0, 50, 16, ctypes.byref(size)) == OK and size.value == 0

    def B(n=1000, V=50, k=16, dY=FAKE, dt=BF16, index=FAKE, out=FAKE, odt=F32, add=0, ws=FAKE, wsb=need):
        return L.cogdl_embedding_backward(n, V, k, dY, dt, index, 1.0, out, odt, add, ws, wsb, None)

    assert B(n=-1) == INVALID and B(V=0) == INVALID and B(k=-1) == INVALID
    assert B(dt=5) == DTYPE and B(odt=3) == DTYPE and B(n=cg.MAX_NNZ + 1) == TOO_LARGE
    assert B(dY=None) == INVALID and B(index=None) == INVALID and B(out=None) == INVALID
    assert B(ws=None) == INVALID and B(ws=ODD) == INVALID and B(wsb=need - 1) == INVALID
    assert B(k=0, dY=None, index=None, out=None, ws=None, wsb=0) == OK
    assert B(n=0, dY=None, index=None, add=1, ws=None, wsb=0) == OK


def forward(L, K):
    def f(n=8, V=100, k=16, X=FAKE, W=FAKE, dt=BF16, bias=None, index=FAKE, teacher=FAKE, T=1.0, loss=FAKE, lse=FAKE,
          logp=FAKE, ws=FAKE, wsb=1 << 40, K=K):
        if K == 0:
            return L.cogdl_linear_cross_entropy(n, V, k, X, W, dt, bias, index, loss, lse, ws, wsb, None)
        return L.cogdl_linear_distill(n, V, k, K, X, W, dt, bias, index, teacher, T, loss, lse, logp, ws, wsb, None)
    return f


def backward(L, K):
    def f(n=8, V=100, k=16, dloss=FAKE, X=FAKE, W=FAKE, dt=BF16, bias=None, index=FAKE, teacher=FAKE, T=1.0, loss=FAKE,
          lse=FAKE, logp=FAKE, dX=FAKE, dW=FAKE, db=FAKE, ws=FAKE, wsb=1 << 40, K=K):
        if K == 0:
            return L.cogdl_linear_cross_entropy_backward(n, V, k, dloss, X, W, dt, bias, index, loss, lse, dX, dW, db, ws,
                                                         wsb, None)
        return L.cogdl_linear_distill_backward(n, V, k, K, dloss, X, W, dt, bias, index, teacher, T, lse, logp, dX, dW,
                                               db, ws, wsb, None)
    return f


@pytest.mark.parametrize("K", [0, 5])
@pytest.mark.parametrize("way", ["forward", "backward"])
def test_loss_validation(L, way, K):
    f = (forward if way == "forward" else backward)(L, K)
    size = ctypes.c_size_t()
    S = L.cogdl_linear_loss_workspace if way == "forward" else L.cogdl_linear_loss_backward_workspace
    assert S(8, 100, 16, K, ctypes.byref(size)) == OK and size.value > 0
    need = size.value
    for bad in ((-1, 100, 16, K), (8, 0, 16, K), (8, 100, -1, K), (8, 100, 16, -1)):
        assert S(*bad, ctypes.byref(size)) == INVALID
    assert S(8, 100, 16, K, None) == INVALID
    large = ((2 ** 24 + 1, 100, 16), (8, 100, 2 ** 22 + 1), (2 ** 24, 2 ** 31 - 1, 16), (2 ** 24, 100, 2 ** 22),
             (8, 2 ** 31 - 1, 2 ** 22))
    for bad in large:
        assert S(*bad, K, ctypes.byref(size)) == TOO_LARGE and f(*bad) == TOO_LARGE
    assert S(8, 100, 16, 1025, ctypes.byref(size)) == TOO_LARGE
    # near the limits, a size is given
    assert S(2, 2 ** 31 - 1, 16, K, ctypes.byref(size)) == OK and size.value > 0
    assert f(n=-1) == INVALID and f(V=0) == INVALID and f(k=-1) == INVALID
    assert f(dt=F32) == DTYPE and f(dt=9) == DTYPE
    for name in ("X", "W", "index", "lse", "ws") + (("loss",) if way == "forward" or K == 0 else ()):
        assert f(**{name: None}) == INVALID, name
    assert f(ws=ODD) == INVALID and f(wsb=need - 1) == INVALID
    if way == "backward":
        assert f(dloss=None) == INVALID
        assert f(dX=None, dW=None, db=None) == OK
        assert f(n=0, dloss=None, X=None, dX=None, dW=None, db=None) == OK
    else:
        assert f(n=0, X=None, index=None, loss=None, lse=None, ws=None, wsb=0) == OK
    if K:
        assert f(teacher=None) == INVALID and f(logp=None) == INVALID
        assert f(K=0 - 1) == INVALID and f(K=1025) == TOO_LARGE
        for T in (0.0, -1.0, INF, float("nan"), 2.0 ** -21, 2.0 ** 21):
            assert f(T=T) == INVALID


bf16, f16, f32, i32 = torch.bfloat16, torch.float16, torch.float32, torch.int32


def refused(fn, pattern):
    with pytest.raises(cg.CogdlError, match=pattern):
        fn()


def reaches_device_check(fn):
    refused(fn, r"must be a CUDA \(HIP\) tensor")


def test_embedding_sizes():
    T, index, dY = torch.zeros(10, 6), torch.zeros(4, dtype=i32), torch.zeros(4, 6)
    reaches_device_check(lambda: cg.embedding(T, index))
    refused(lambda: cg.embedding(T[0], index), "table must have 2 dimensions")
    refused(lambda: cg.embedding(T[:0], index), "at least one row")
    refused(lambda: cg.embedding(T, index.view(2, 2)), "index must have 1 dimensions")
    refused(lambda: cg.embedding(T, index, out=torch.zeros(4, 5)), "out has 20 elements, expected 24")
    reaches_device_check(lambda: cg.embedding_backward(dY, index, 10))
    refused(lambda: cg.embedding_backward(dY, index[:3], 10), "index has 3 elements, expected 4")
    refused(lambda: cg.embedding_backward(dY, index, 0), "at least one row")
    refused(lambda: cg.embedding_backward(dY, index, 10, out=T[:9]), "out has 54 elements, expected 60")
    refused(lambda: cg.embedding_backward(dY, index, 10, accumulate=True), "accumulate needs out")
    refused(lambda: cg.embedding_backward(dY[0], index, 10), "dY must have 2 dimensions")


def test_loss_sizes():
    X, W, t, v = torch.zeros(4, 8, dtype=bf16), torch.zeros(20, 8, dtype=bf16), torch.zeros(4, dtype=i32), torch.zeros(4)
    f, b = cg.linear_cross_entropy, cg.linear_cross_entropy_backward
    reaches_device_check(lambda: f(X, W, t))
    refused(lambda: f(X, W[:, :7], t), "same dtype")
    refused(lambda: f(X.half(), W, t), "same dtype")
    refused(lambda: f(X[0], W, t), "X must have 2 dimensions")
    refused(lambda: f(X, W[:0], t), "at least one row")
    refused(lambda: f(X, W, t[:3]), "target has 3 elements, expected 4")
    refused(lambda: f(X, W, t, torch.zeros(19)), "bias has 19 elements, expected 20")
    refused(lambda: f(X, W, t, loss=v[:3]), "loss has 3 elements, expected 4")
    refused(lambda: f(X, W, t, lse=torch.zeros(5)), "lse has 5 elements, expected 4")
    reaches_device_check(lambda: b(v, X, W, t, v, v))
    refused(lambda: b(v[:3], X, W, t, v, v), "dloss has 3 elements, expected 4")
    refused(lambda: b(None, X, W, t, v, v), "dloss must be a torch tensor")
    refused(lambda: b(v, X, W, t[:3], v, v), "target has 3 elements, expected 4")
    refused(lambda: b(v, X, W, t, v[:3], v), "loss has 3 elements, expected 4")
    refused(lambda: b(v, X, W, t, v, v[:3]), "lse has 3 elements, expected 4")


def test_distill_sizes():
    X, W, v = torch.zeros(4, 8, dtype=f16), torch.zeros(20, 8, dtype=f16), torch.zeros(4)
    index, teacher = torch.zeros(4, 3, dtype=i32), torch.zeros(4, 3)
    f, b = cg.linear_distill, cg.linear_distill_backward
    reaches_device_check(lambda: f(X, W, index, teacher))
    refused(lambda: f(X, W, index[:3], teacher), r"must both be \[4, K\]")
    refused(lambda: f(X, W, index, teacher[:, :2]), r"must both be \[4, K\]")
    refused(lambda: f(X, W, index[:, :0], teacher[:, :0]), "0 entries")
    refused(lambda: f(X, W, torch.zeros(4, 1025, dtype=i32), torch.zeros(4, 1025)), "1025 entries")
    for T in (0.0, -2.0, INF, float("nan"), 2.0 ** -21, 2.0 ** 21):
        refused(lambda: f(X, W, index, teacher, temperature=T), "temperature must be positive")
    refused(lambda: f(X, W, index, teacher, logp=torch.zeros(4, 2)), "logp has 8 elements, expected 12")
    reaches_device_check(lambda: b(v, X, W, index, teacher, v, teacher))
    refused(lambda: b(v, X, W, index, teacher, v, teacher[:, :2]), "logp has 8 elements, expected 12")
    refused(lambda: b(v, X, W, index, teacher, v[:2], teacher), "lse has 2 elements, expected 4")
    refused(lambda: b(v, X, W, index, teacher, v, teacher, temperature=0.0), "temperature must be positive")


def test_sizes_past_32_bits():
    far = 2 ** 32 + 5
    index, t = torch.zeros(3, dtype=i32), torch.zeros(3, dtype=i32)
    refused(lambda: cg.embedding(torch.zeros(far, 0), index), "past 32 bits")
    refused(lambda: cg.embedding_backward(torch.zeros(3, 8), index, far), "past 32 bits")
    refused(lambda: cg.embedding_backward(torch.zeros(0, far), index[:0], 9), "past 32 bits")
    refused(lambda: cg.linear_cross_entropy(torch.zeros(3, 0, dtype=bf16), torch.zeros(far, 0, dtype=bf16), t), "past 32 bits")
    refused(lambda: cg.linear_distill(torch.zeros(3, 0, dtype=bf16), torch.zeros(far, 0, dtype=bf16), index.view(3, 1),
                                      torch.zeros(3, 1)), "past 32 bits")
    with pytest.raises(TypeError):
        cg.embedding_backward(torch.zeros(3, 8), index, 9.0)
