"""Refusals of the grouped products and the 8-bit checkpoints, on the host before anything is launched: the C ABI's
codes, and the binding's sizes and types (no GPU: only calls that are refused, or that have nothing to do)."""
import ctypes
import os

import pytest
import torch

import paper_2103_00959_amd as cg

OK, INVALID, DTYPE, TOO_LARGE = 0, 1, 2, 6
FAKE = ctypes.c_void_p(0x1000)
F32, BF16, F16 = 0, 1, 2


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(cg.LIB_PATH):
        from paper_2103_00959_amd import build
        build.build(verbose=False)
    return cg.lib()


def test_checkpoint_validation(L):
    def C(n=4, F=64, A=FAKE, dt=BF16, codes=FAKE, exps=FAKE):
        return L.cogdl_act_checkpoint(n, F, A, dt, codes, exps, None)

    assert C(n=-1) == INVALID and C(F=0) == INVALID
    assert C(dt=3) == DTYPE and C(dt=-1) == DTYPE
    assert C(A=None) == INVALID and C(codes=None) == INVALID and C(exps=None) == INVALID
    assert C(n=0, A=None, codes=None, exps=None) == OK

    def R(n=4, F=64, codes=FAKE, exps=FAKE, out=FAKE, dt=BF16):
        return L.cogdl_act_restore(n, F, codes, exps, out, dt, None)

    assert R(n=-1) == INVALID and R(F=0) == INVALID and R(dt=7) == DTYPE
    assert R(codes=None) == INVALID and R(exps=None) == INVALID and R(out=None) == INVALID
    assert R(n=0, codes=None, exps=None, out=None) == OK


def test_grouped_linear_validation(L):
    def G(n=8, E=2, k=4, m=4, off=FAKE, X=FAKE, W=FAKE, dt=BF16, bias=None, act=0, Y=FAKE, ydt=BF16, codes=None,
          exps=None):
        return L.cogdl_grouped_linear(n, E, k, m, off, X, W, dt, bias, act, Y, ydt, codes, exps, None)

    assert G(n=-1) == INVALID and G(E=0) == INVALID and G(k=-1) == INVALID and G(m=-1) == INVALID
    assert G(dt=F32) == DTYPE and G(dt=5) == DTYPE and G(ydt=7) == DTYPE
    assert G(E=4097) == TOO_LARGE and G(n=2 ** 31) == TOO_LARGE
    assert G(n=2 ** 31 - 1, m=2 ** 31 - 1) == TOO_LARGE          # more tiles than a launch has
    assert G(off=None) == INVALID and G(X=None) == INVALID and G(W=None) == INVALID and G(Y=None) == INVALID
    assert G(act=3) == INVALID and G(act=-1) == INVALID
    assert G(codes=FAKE) == INVALID and G(exps=FAKE) == INVALID
    assert G(n=0, X=None, W=None, Y=None) == OK
    assert G(m=0, W=None, Y=None) == OK


def test_grouped_backward_validation(L):
    size = ctypes.c_size_t()

    def S(n=8, E=2, k=4, m=4, out=ctypes.byref(size)):
        return L.cogdl_grouped_linear_backward_workspace(n, E, k, m, out)

    assert S() == OK and size.value == 0                          # few rows: no partial sums
    assert S(n=1_000_000, k=64, m=48) == OK and size.value > 0
    assert S(n=-1) == INVALID and S(E=0) == INVALID and S(k=-1) == INVALID and S(m=-1) == INVALID
    assert S(out=None) == INVALID and S(E=4097) == TOO_LARGE and S(n=2 ** 31) == TOO_LARGE

    def B(n=8, E=2, k=4, m=4, off=FAKE, dY=FAKE, W=FAKE, X=FAKE, codes=None, exps=None, dt=BF16, Y=None, act=0,
          dX=FAKE, dW=FAKE, dwdt=BF16, db=FAKE, ws=None, wsb=0):
        return L.cogdl_grouped_linear_backward(n, E, k, m, off, dY, W, X, codes, exps, dt, Y, act, dX, dW, dwdt, db,
                                               ws, wsb, None)

    assert B(n=-1) == INVALID and B(E=0) == INVALID and B(k=-1) == INVALID and B(m=-1) == INVALID
    assert B(dt=F32) == DTYPE and B(dwdt=F16) == DTYPE and B(dwdt=9) == DTYPE
    assert B(E=4097) == TOO_LARGE and B(n=2 ** 31) == TOO_LARGE
    assert B(off=None) == INVALID and B(dY=None) == INVALID and B(W=None) == INVALID
    assert B(act=4) == INVALID and B(act=1, Y=None) == INVALID
    assert B(X=None) == INVALID                                   # neither the input nor its checkpoint
    assert B(codes=FAKE, exps=FAKE) == INVALID                    # both
    assert B(X=None, codes=FAKE) == INVALID and B(X=None, exps=FAKE) == INVALID
    many = dict(n=1_000_000, k=64, m=48)
    S(**many)
    need = size.value
    assert B(**many) == INVALID                                   # no workspace
    assert B(ws=FAKE, wsb=need - 1, **many) == INVALID
    assert B(ws=ctypes.c_void_p(0x1008), wsb=need, **many) == INVALID
    assert B(dX=None, dW=None, db=None, dY=None, W=None, X=None) == OK
    assert B(m=0, dY=None, W=None, X=None, dX=None) == OK


bf16, f16, f32, i32 = torch.bfloat16, torch.float16, torch.float32, torch.int32


def refused(fn, pattern):
    with pytest.raises(cg.CogdlError, match=pattern):
        fn()


def reaches_device_check(fn):
    refused(fn, r"must be a CUDA \(HIP\) tensor")


def test_checkpoint_sizes():
    A = torch.zeros(4, 70, dtype=bf16)
    codes, exps = torch.zeros(4, 70, dtype=torch.int8), torch.zeros(4, 3, dtype=torch.uint8)
    reaches_device_check(lambda: cg.act_checkpoint(A))
    refused(lambda: cg.act_checkpoint(A[0]), "A must have 2 dimensions")
    refused(lambda: cg.act_checkpoint(torch.zeros(4, 0)), "at least one feature")
    refused(lambda: cg.act_checkpoint(A, codes=codes[:3]), "codes has 210 elements, expected 280")
    refused(lambda: cg.act_checkpoint(A, exps=exps[:, :2]), "exps has 8 elements, expected 12")
    reaches_device_check(lambda: cg.act_restore(codes, exps))
    refused(lambda: cg.act_restore(codes, exps[:, :2]), "exps has 8 elements, expected 12")
    refused(lambda: cg.act_restore(codes, exps, out=torch.zeros(4, 69)), "out has 276 elements, expected 280")
    refused(lambda: cg.act_restore(codes.view(-1), exps), "codes must have 2 dimensions")


def test_grouped_sizes():
    X, W, off = torch.zeros(6, 40, dtype=bf16), torch.zeros(3, 16, 40, dtype=bf16), torch.zeros(4, dtype=i32)
    reaches_device_check(lambda: cg.grouped_linear(X, W, off))
    refused(lambda: cg.grouped_linear(X, W[0], off), "W must have 3 dimensions")
    refused(lambda: cg.grouped_linear(X, W[:, :, :39], off), "same dtype")
    refused(lambda: cg.grouped_linear(X.half(), W, off), "same dtype")
    refused(lambda: cg.grouped_linear(X, W, off[:3]), "offsets has 3 elements, expected 4")
    refused(lambda: cg.grouped_linear(X, W, off.view(2, 2)), "offsets must have 1 dimensions")
    refused(lambda: cg.grouped_linear(X, W[:0], off[:1]), "W has 0 groups")
    refused(lambda: cg.grouped_linear(X, torch.zeros(4097, 1, 40, dtype=bf16), off), "W has 4097 groups")
    refused(lambda: cg.grouped_linear(X, W, off, bias=torch.zeros(16)), "bias has 16 elements, expected 48")
    refused(lambda: cg.grouped_linear(X, W, off, out=torch.zeros(6, 15)), "out has 90 elements, expected 96")
    refused(lambda: cg.grouped_linear(X, W, off, codes=torch.zeros(6, 40, dtype=torch.int8)), "together")
    refused(lambda: cg.grouped_linear(X, W, off, codes=torch.zeros(6, 40, dtype=torch.int8),
                                      exps=torch.zeros(6, 1, dtype=torch.uint8)), "exps has 6 elements, expected 12")
    refused(lambda: cg.grouped_linear(X[:, :0], W[:, :, :0], off, save=True), "at least one feature")
    with pytest.raises(ValueError):
        cg.grouped_linear(X, W, off, act="gelu")


def test_grouped_backward_sizes():
    X, W, off = torch.zeros(6, 40, dtype=bf16), torch.zeros(3, 16, 40, dtype=bf16), torch.zeros(4, dtype=i32)
    dY, codes, exps = torch.zeros(6, 16, dtype=bf16), torch.zeros(6, 40, dtype=torch.int8), torch.zeros(6, 2, dtype=torch.uint8)
    B = cg.grouped_linear_backward
    reaches_device_check(lambda: B(dY, W, off, X=X))
    reaches_device_check(lambda: B(dY, W, off, codes=codes, exps=exps))
    reaches_device_check(lambda: B(dY, W, off, out={"dW": None}))
    refused(lambda: B(dY[:, :15], W, off, X=X), "same dtype")
    refused(lambda: B(dY, W, off), "dW needs X or its checkpoint")
    refused(lambda: B(dY, W, off, X=X, codes=codes, exps=exps), "not both")
    refused(lambda: B(dY, W, off, codes=codes), "together")
    refused(lambda: B(dY, W, off, X=X[:5]), r"X must be \[6, 40\]")
    refused(lambda: B(dY, W, off, X=X.half()), "dY's dtype")
    refused(lambda: B(dY, W, off, codes=codes[:5], exps=exps), r"codes must be \[6, 40\]")
    refused(lambda: B(dY, W, off, codes=codes, exps=exps[:, :1]), "exps has 6 elements, expected 12")
    refused(lambda: B(dY, W, off, X=X, act="relu"), "needs Y")
    refused(lambda: B(dY, W, off, X=X, act="relu", Y=torch.zeros(6, 16)), "dY's dtype")
    refused(lambda: B(dY, W, off, X=X, act="relu", Y=dY[:5]), r"Y must be \[6, 16\]")
    refused(lambda: B(dY, W, off, X=X, out={"dx": None}), "unknown output 'dx'")
    refused(lambda: B(dY, W, off, X=X, out={"dW": torch.zeros(3, 16, 39)}), "dW has 1872 elements, expected 1920")
    big = torch.zeros(100000, 16, dtype=bf16)
    need = cg.grouped_linear_backward_workspace(100000, 3, 40, 16)
    assert need > 0
    refused(lambda: B(big, W, off, X=torch.zeros(100000, 40, dtype=bf16),
                      workspace=torch.zeros(need - 1, dtype=torch.uint8)), "workspace has")
    with pytest.raises(ValueError):
        B(dY, W, off, X=X, act="gelu")


def test_widths_past_the_largest(L):
    wide, size = 2 ** 22 + 1, ctypes.c_size_t()
    for k, m in ((wide, 8), (8, wide)):
        assert L.cogdl_grouped_linear(8, 2, k, m, FAKE, FAKE, FAKE, BF16, None, 0, FAKE, BF16, None, None,
                                      None) == TOO_LARGE
        assert L.cogdl_grouped_linear_backward_workspace(8, 2, k, m, ctypes.byref(size)) == TOO_LARGE
        assert L.cogdl_grouped_linear_backward(8, 2, k, m, FAKE, FAKE, FAKE, FAKE, None, None, BF16, None, 0, FAKE,
                                               FAKE, BF16, FAKE, None, 0, None) == TOO_LARGE
