"""Refusals of the experts' products and quantisers, on the host (no GPU needed): the C entry points
reject bad sizes, types and pointers before touching a device, the Python ones tensors that the kernels
must not address."""
import ctypes

import pytest
import torch

import paper_2609_01024_amd as pcm
from paper_2609_01024_amd import binding

OK, ARG, UNSUP, WS = 0, 1, 2, 3
F32, BF16, F16DOWN = 0, 1, 2
P = ctypes.c_void_p(0x10000)     # never dereferenced: validation fails first
MIS = ctypes.c_void_p(0x10008)


@pytest.fixture(scope="module")
def L():
    return pcm.lib()


def forward(dt=BF16, out=BF16, x=P, w=P, off=P, tok=P, T=8, R=16, K=64, N=32, n=4, y=P):
    return (dt, out, x, w, off, tok, T, R, K, N, n, y, None)


def grad_x(dt=BF16, out=BF16, dy=P, w=P, off=P, of=P, T=8, k=2, R=16, K=64, N=32, n=4, dx=P, ws=P, wsb=1 << 20):
    return (dt, out, dy, w, off, of, T, k, R, K, N, n, dx, ws, wsb, None)


def grad_w(dt=BF16, out=BF16, x=P, dy=P, off=P, tok=P, T=8, R=16, K=64, N=32, n=4, dw=P, acc=0, ws=None, wsb=0):
    return (dt, out, x, dy, off, tok, T, R, K, N, n, dw, acc, ws, wsb, None)


def eight_bit(out=BF16, x=P, xs=P, w=P, ws=P, off=P, tok=P, T=8, R=16, K=64, N=32, n=4, y=P):
    return (out, x, xs, w, ws, off, tok, T, R, K, N, n, y, None)


CALLS = {"pcm_grouped_gemm": forward, "pcm_grouped_gemm_dx": grad_x, "pcm_grouped_gemm_dw": grad_w,
         "pcm_grouped_gemm_fp8": eight_bit}


@pytest.mark.parametrize("name", CALLS)
def test_sizes(L, name):
    call, args = getattr(L, name), CALLS[name]
    for bad, want in ((dict(K=0), ARG), (dict(N=0), ARG), (dict(n=0), ARG), (dict(T=-1), ARG), (dict(R=-1), ARG),
                      (dict(K=72), UNSUP), (dict(N=40), UNSUP), (dict(n=257), UNSUP), (dict(R=1 << 30), UNSUP),
                      (dict(T=1 << 30), UNSUP)):
        assert call(*args(**bad)) == want, (name, bad)


@pytest.mark.parametrize("name", CALLS)
def test_widths_near_32_bits(L, name):
    """K and N whose number of blocks of 128 would pass 32 bits on the way are refused, the last one below is not."""
    call, args = getattr(L, name), CALLS[name]
    for width in ((1 << 31) - 112, (1 << 31) - 16):
        assert call(*args(K=width)) == UNSUP, width
        assert call(*args(N=width)) == UNSUP, width
    assert call(*args(K=(1 << 31) - 128, N=(1 << 31) - 128, out=-1)) == ARG


def test_quantiser_widths_near_32_bits(L):
    for width in ((1 << 31) - 112, (1 << 31) - 16):
        assert L.pcm_quant_fp8_rows(BF16, P, None, 1, width, P, P, None) == UNSUP
        assert L.pcm_swiglu_quant_fp8(BF16, P, None, 1, width, P, P, None) == UNSUP
        assert L.pcm_quant_fp8_weights(BF16, P, 1, width, 16, P, P, None, None, None) == UNSUP
        assert L.pcm_quant_fp8_weights(BF16, P, 1, 16, width, P, P, None, None, None) == UNSUP


@pytest.mark.parametrize("name", CALLS)
def test_types(L, name):
    call, args = getattr(L, name), CALLS[name]
    assert call(*args(out=F16DOWN)) == ARG
    assert call(*args(out=-1)) == ARG
    if name != "pcm_grouped_gemm_fp8":
        assert call(*args(dt=F16DOWN)) == ARG
        assert call(*args(dt=F32, out=BF16)) == ARG


@pytest.mark.parametrize("name,pointers", [("pcm_grouped_gemm", "x w y"), ("pcm_grouped_gemm_dx", "dy w dx"),
                                           ("pcm_grouped_gemm_dw", "x dy dw"), ("pcm_grouped_gemm_fp8", "x xs w ws y")])
def test_pointers(L, name, pointers):
    call, args = getattr(L, name), CALLS[name]
    for p in pointers.split():
        assert call(*args(**{p: None})) == ARG, p
        assert call(*args(**{p: MIS})) == ARG, p
    assert call(*args(off=MIS)) == ARG


@pytest.mark.parametrize("name", ["pcm_grouped_gemm", "pcm_grouped_gemm_dw", "pcm_grouped_gemm_fp8"])
def test_rows(L, name):
    call, args = getattr(L, name), CALLS[name]
    assert call(*args(tok=MIS)) == ARG
    assert call(*args(off=None)) == ARG                  # several groups without offsets
    assert call(*args(off=None, n=1)) == ARG             # gathered rows without offsets
    assert call(*args(tok=None)) == ARG                  # T != R without a gather
    assert call(*args(T=0)) == ARG                       # rows gathered from nothing


def test_input_gradient(L):
    assert L.pcm_grouped_gemm_dx(*grad_x(k=0)) == ARG
    assert L.pcm_grouped_gemm_dx(*grad_x(k=9)) == UNSUP
    assert L.pcm_grouped_gemm_dx(*grad_x(R=17)) == ARG               # more rows than slots
    assert L.pcm_grouped_gemm_dx(*grad_x(of=None)) == ARG            # T != R
    assert L.pcm_grouped_gemm_dx(*grad_x(of=None, T=16)) == ARG      # k != 1
    assert L.pcm_grouped_gemm_dx(*grad_x(of=MIS)) == ARG
    assert L.pcm_grouped_gemm_dx(*grad_x(off=None)) == ARG
    need = L.pcm_workspace_bytes(binding.OP_GROUPED_DX, 8, 64, 0, 4, 2, BF16)
    assert need == 8 * 2 * 64 * 4
    assert L.pcm_grouped_gemm_dx(*grad_x(wsb=need - 1)) == WS
    assert L.pcm_grouped_gemm_dx(*grad_x(ws=None)) == WS
    assert L.pcm_grouped_gemm_dx(*grad_x(ws=MIS)) == ARG


def test_weight_gradient_workspace(L):
    """Many rows and a small result: parts of the rows, each with sums of its own."""
    assert L.pcm_workspace_bytes(binding.OP_GROUPED_DW, 16, 64, 32, 4, 1, BF16) == 0
    need = L.pcm_workspace_bytes(binding.OP_GROUPED_DW, 8192, 2048, 64, 1, 1, BF16)
    assert need == 16 * 64 * 2048 * 4                      # 32 tiles: 512 / 32 parts
    args = dict(off=None, tok=None, n=1, T=8192, R=8192, K=2048, N=64)
    assert L.pcm_grouped_gemm_dw(*grad_w(**args, ws=P, wsb=need - 1)) == WS
    assert L.pcm_grouped_gemm_dw(*grad_w(**args, ws=None, wsb=need)) == WS
    assert L.pcm_grouped_gemm_dw(*grad_w(**args, ws=MIS, wsb=need)) == ARG


def test_accumulate_is_float32(L):
    assert L.pcm_grouped_gemm_dw(*grad_w(acc=1)) == ARG


def test_nothing_to_do(L):
    assert L.pcm_grouped_gemm(*forward(R=0, x=None, w=None, y=None)) == OK
    assert L.pcm_grouped_gemm_fp8(*eight_bit(R=0, x=None, y=None)) == OK
    assert L.pcm_grouped_gemm_dx(*grad_x(T=0, R=0, dy=None, dx=None)) == OK
    assert L.pcm_grouped_gemm_dw(*grad_w(R=0, out=F32, acc=1)) == OK
    assert L.pcm_quant_fp8_rows(BF16, None, None, 0, 64, None, None, None) == OK
    assert L.pcm_swiglu_quant_fp8(F32, None, None, 0, 64, None, None, None) == OK


def test_quantisers(L):
    for name in ("pcm_quant_fp8_rows", "pcm_swiglu_quant_fp8"):
        call = getattr(L, name)
        assert call(F16DOWN, P, None, 4, 64, P, P, None) == ARG
        assert call(BF16, P, None, -1, 64, P, P, None) == ARG
        assert call(BF16, P, None, 4, 0, P, P, None) == ARG
        assert call(BF16, P, None, 4, 72, P, P, None) == UNSUP
        assert call(BF16, P, None, 1 << 30, 64, P, P, None) == UNSUP
        for i, bad in ((1, None), (1, MIS), (5, None), (5, MIS), (6, None), (6, MIS), (2, ctypes.c_void_p(0x10002))):
            args = [BF16, P, None, 4, 64, P, P, None]
            args[i] = bad
            assert call(*args) == ARG, (name, i, bad)
    good = [BF16, P, 4, 64, 32, P, P, P, P, None]
    for i, bad, want in ((0, 2, ARG), (2, 0, ARG), (2, 257, UNSUP), (3, 0, ARG), (3, 40, UNSUP), (4, 72, UNSUP),
                         (1, None, ARG), (1, MIS, ARG), (5, None, ARG), (6, MIS, ARG), (7, None, ARG), (8, None, ARG),
                         (7, MIS, ARG), (8, MIS, ARG)):
        args = list(good)
        args[i] = bad
        assert L.pcm_quant_fp8_weights(*args) == want, (i, bad)


def test_python_refuses_host_tensors():
    x, w = torch.zeros(4, 64), torch.zeros(1, 32, 64)
    off = torch.tensor([0, 4], dtype=torch.int32)
    q, qs = x.to(torch.float8_e4m3fn), torch.ones(4, 1)
    wq, ws = w.to(torch.float8_e4m3fn), torch.ones(1, 1, 1)
    for call in (lambda: pcm.pcm_grouped_gemm(x, w, off), lambda: pcm.pcm_grouped_gemm_dx(torch.zeros(4, 32), w, off),
                 lambda: pcm.pcm_grouped_gemm_dw(x, torch.zeros(4, 32), off), lambda: pcm.pcm_quant_fp8_rows(x),
                 lambda: pcm.pcm_swiglu_quant_fp8(x), lambda: pcm.pcm_quant_fp8_weights(w),
                 lambda: pcm.pcm_grouped_gemm_fp8(q, qs, wq, ws, off)):
        with pytest.raises(ValueError):
            call()


def test_python_refuses_sizes_past_32_bits():
    """Sizes that the C entry points take in 32 bits are refused above them, not cut to what is left of them."""
    wide, on = (1 << 32) + 64, dict(device="meta")
    x, w = torch.empty((1, wide), **on), torch.empty((1, 64, wide), **on)
    q, wq = torch.empty((1, wide), dtype=torch.float8_e4m3fn, **on), torch.empty((64, wide), dtype=torch.float8_e4m3fn, **on)
    scale = torch.empty((1, wide // 128 + 1), **on)
    for call in (lambda: pcm.pcm_grouped_gemm(x, w), lambda: pcm.pcm_grouped_gemm_dx(x, w.mT),
                 lambda: pcm.pcm_grouped_gemm_dx(torch.empty((1, 64), **on), w),
                 lambda: pcm.pcm_grouped_gemm_dx(torch.empty((1, 64), **on), w[:, :, :64], row_of=x.int()),
                 lambda: pcm.pcm_grouped_gemm_dw(x, torch.empty((1, 64), **on)),
                 lambda: pcm.pcm_grouped_gemm_dw(torch.empty((1, 64), **on), x),
                 lambda: pcm.pcm_quant_fp8_rows(x), lambda: pcm.pcm_swiglu_quant_fp8(torch.empty((1, 2 * wide), **on)),
                 lambda: pcm.pcm_quant_fp8_weights(w), lambda: pcm.pcm_quant_fp8_weights(w.mT),
                 lambda: pcm.pcm_grouped_gemm_fp8(q, scale, wq, scale)):
        with pytest.raises(ValueError, match="32 bits"):
            call()


def test_python_refuses_shapes():
    x = torch.zeros(4, 64)
    with pytest.raises(ValueError):
        pcm.pcm_grouped_gemm(x[0], torch.zeros(1, 32, 64))
    with pytest.raises(ValueError):
        pcm.pcm_grouped_gemm(x, torch.zeros(32))
    with pytest.raises(ValueError):
        pcm.pcm_swiglu_quant_fp8(torch.zeros(4, 63))
    with pytest.raises(ValueError):
        pcm.pcm_quant_fp8_weights(torch.zeros(64))
