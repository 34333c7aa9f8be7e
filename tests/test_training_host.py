"""Refusals of the training step's operators, on the host (no GPU needed): the C entry points reject bad sizes, types,
pointers and overlapping tensors before touching a device, the Python ones tensors that the kernels must not address."""
import ctypes
import struct

import pytest
import torch

import paper_2609_01024_amd as pcm
from paper_2609_01024_amd import binding

OK, ARG, UNSUP, WS = 0, 1, 2, 3
F32, BF16, F16DOWN = 0, 1, 2
P = ctypes.c_void_p(0x10000)     # never dereferenced: validation fails first
MIS = ctypes.c_void_p(0x10008)
ODD = ctypes.c_void_p(0x10002)


@pytest.fixture(scope="module")
def L():
    return pcm.lib()


def dispatch(dt=BF16, out=BF16, x=P, of=P, w=P, off=P, T=8, k=2, R=16, H=64, n=4, y=P):
    return (dt, out, x, of, w, off, T, k, R, H, n, y, None)


def dispatch_grad(dt=BF16, other=F32, out=BF16, dy=P, x=P, of=P, w=P, off=P, T=8, k=2, R=16, H=64, n=4, dx=P, dw=P):
    return (dt, other, out, dy, x, of, w, off, T, k, R, H, n, dx, dw, None)


def combine(dt=BF16, out=BF16, o=P, of=P, w=P, off=P, T=8, k=2, R=16, H=64, n=4, y=P, acc=0):
    return (dt, out, o, of, w, off, T, k, R, H, n, y, acc, None)


def combine_grad(dt=BF16, other=F32, out=BF16, dy=P, o=P, of=P, w=P, off=P, T=8, k=2, R=16, H=64, n=4, do=P, dw=P):
    return (dt, other, out, dy, o, of, w, off, T, k, R, H, n, do, dw, None)


def mix(dt=BF16, out=BF16, u=P, bits=P, beta=P, src=P, tgt=P, T=8, k=2, R=16, R_tgt=16, H=64, z=P):
    return (dt, out, u, bits, beta, src, tgt, T, k, R, R_tgt, H, z, None)


def mix_grad(dt=BF16, out=BF16, dz=P, u=P, bits=P, beta=P, src=P, tgt=P, T=8, k=2, R=16, R_tgt=16, H=64, du=P, dbeta=P):
    return (dt, out, dz, u, bits, beta, src, tgt, T, k, R, R_tgt, H, du, dbeta, None)


def swiglu(dt=BF16, out=BF16, gate_up=P, count=None, R=16, H=64, u=P):
    return (dt, out, gate_up, count, R, H, u, None)


def swiglu_grad(dt=BF16, out=BF16, gate_up=P, du=P, count=None, R=16, H=64, d=P):
    return (dt, out, gate_up, du, count, R, H, d, None)


CALLS = {"pcm_dispatch_rows": dispatch, "pcm_dispatch_rows_grad": dispatch_grad, "pcm_combine_rows": combine,
         "pcm_combine_rows_grad": combine_grad, "pcm_mix_rows": mix, "pcm_mix_rows_grad": mix_grad, "pcm_swiglu": swiglu,
         "pcm_swiglu_grad": swiglu_grad}
ON_TOKENS = [name for name in CALLS if "swiglu" not in name]
ON_GROUPS = [name for name in ON_TOKENS if "mix" not in name]


@pytest.mark.parametrize("name", CALLS)
def test_sizes_and_types(L, name):
    call, args = getattr(L, name), CALLS[name]
    for bad, want in ((dict(H=0), ARG), (dict(R=-1), ARG), (dict(H=72), UNSUP), (dict(R=1 << 30), UNSUP),
                      (dict(H=(1 << 31) - 112), UNSUP), (dict(H=(1 << 28) + 16), UNSUP), (dict(H=1 << 28, out=-1), ARG), (dict(dt=F16DOWN), ARG), (dict(dt=-1), ARG), (dict(out=F16DOWN), ARG),
                      (dict(out=7), ARG)):
        assert call(*args(**bad)) == want, (name, bad)
    if name in ON_TOKENS:
        for bad, want in ((dict(T=-1), ARG), (dict(k=0), ARG), (dict(k=9), UNSUP), (dict(T=1 << 30), UNSUP)):
            assert call(*args(**bad)) == want, (name, bad)
    if name in ("pcm_dispatch_rows_grad", "pcm_combine_rows_grad"):
        assert call(*args(other=F16DOWN)) == ARG and call(*args(other=-1)) == ARG
    if name in ON_GROUPS:
        for bad, want in ((dict(n=0), ARG), (dict(n=257), UNSUP), (dict(off=None), ARG)):
            assert call(*args(**bad)) == want, (name, bad)
    if "mix" in name:
        for bad, want in ((dict(R_tgt=-1), ARG), (dict(R_tgt=1 << 30), UNSUP)):
            assert call(*args(**bad)) == want, (name, bad)


@pytest.mark.parametrize("name,needed,optional", [
    ("pcm_dispatch_rows", "x of y", "w"), ("pcm_dispatch_rows_grad", "dy x of", "w dx dw"), ("pcm_combine_rows", "o of y", "w"),
    ("pcm_combine_rows_grad", "dy o of", "w do dw"), ("pcm_mix_rows", "u bits beta src tgt z", ""),
    ("pcm_mix_rows_grad", "dz u bits beta src tgt", "du dbeta"), ("pcm_swiglu", "gate_up u", ""),
    ("pcm_swiglu_grad", "gate_up du d", "")])
def test_pointers(L, name, needed, optional):
    call, args = getattr(L, name), CALLS[name]
    for p in needed.split():
        assert call(*args(**{p: None})) == ARG, p
    for p in (needed + " " + optional).split():
        assert call(*args(**{p: MIS})) == ARG, p
    if name in ON_GROUPS:
        assert call(*args(off=ODD)) == ARG
    if "swiglu" in name:
        assert call(*args(count=ODD)) == ARG


def test_something_is_wanted(L):
    assert L.pcm_dispatch_rows_grad(*dispatch_grad(dx=None, dw=None)) == ARG
    assert L.pcm_combine_rows_grad(*combine_grad(do=None, dw=None)) == ARG
    assert L.pcm_mix_rows_grad(*mix_grad(du=None, dbeta=None)) == ARG


def test_accumulate_is_float32(L):
    assert L.pcm_combine_rows(*combine(acc=1)) == ARG


def test_nothing_to_do(L):
    assert L.pcm_dispatch_rows(*dispatch(T=0, x=None, of=None, y=None)) == OK
    assert L.pcm_dispatch_rows(*dispatch(R=0, y=None)) == OK
    assert L.pcm_dispatch_rows_grad(*dispatch_grad(T=0, dy=None, x=None, of=None, dx=None, dw=None)) == OK
    assert L.pcm_combine_rows(*combine(T=0, o=None, of=None, y=None)) == OK
    assert L.pcm_combine_rows_grad(*combine_grad(T=0, dy=None, o=None, of=None, do=None, dw=None)) == OK
    assert L.pcm_mix_rows(*mix(T=0, u=None, bits=None, beta=None, src=None, tgt=None, z=None)) == OK
    assert L.pcm_mix_rows(*mix(R_tgt=0, z=None)) == OK
    assert L.pcm_mix_rows_grad(*mix_grad(R=0, u=None, du=None, dbeta=None)) == OK
    assert L.pcm_mix_rows_grad(*mix_grad(T=0, dz=None, u=None, du=None, dbeta=None)) == OK
    assert L.pcm_swiglu(*swiglu(R=0, gate_up=None, u=None)) == OK
    assert L.pcm_swiglu_grad(*swiglu_grad(R=0, gate_up=None, du=None, d=None)) == OK


def test_route_grad(L):
    def args(out=F32, ids=P, w=P, bits=P, dbeta=P, mode=0, dw=P, T=8, n=16, k=2, d=P):
        return (out, ids, w, bits, dbeta, mode, dw, T, n, k, d, None)
    call = L.pcm_route_grad
    for bad, want in ((dict(T=-1), ARG), (dict(n=0), ARG), (dict(k=0), ARG), (dict(n=4, k=5), ARG), (dict(n=257), UNSUP),
                      (dict(k=9), UNSUP), (dict(T=1 << 30, k=1), UNSUP), (dict(out=F16DOWN), ARG), (dict(mode=3), ARG),
                      (dict(mode=-1), ARG), (dict(bits=None), ARG), (dict(dbeta=None), ARG),
                      (dict(bits=None, dbeta=None, dw=None), ARG), (dict(ids=None), ARG), (dict(w=None), ARG), (dict(d=None), ARG)):
        assert call(*args(**bad)) == want, bad
    for p in ("ids", "w", "bits", "dbeta", "dw", "d"):
        assert call(*args(**{p: MIS})) == ARG, p
    assert call(*args(T=0, ids=None, w=None, d=None)) == OK


# ------------------------------------------------------------------------ all gradients
def tensors(*items):
    """A pcm_tensor array of (address, count, type)."""
    return ctypes.create_string_buffer(b"".join(struct.pack("<QqQ", *i) for i in items)) if items else None


def clip(L, grads, out=None, m=None, max_norm=1.0, norm=P, ws=P, wsb=1 << 20):
    m = len(grads) if m is None else m
    to = None if out is None else tensors(*out)
    return {L.pcm_clip_grads(tensors(*grads), to, m, norm, max_norm, None),
            L.pcm_clip_grad_norm(tensors(*grads), to, m, max_norm, norm, ws, wsb, None)}


A, B = (0x10000, 64, F32), (0x20000, 64, BF16)


def test_clip_refuses_tensors(L):
    for bad, want in (((0x10000, 64, F16DOWN), ARG), ((0x10000, 64, 9), ARG), ((0x10000, -1, F32), ARG), ((0, 64, F32), ARG),
                      ((0x10002, 64, F32), ARG), ((0x10001, 64, BF16), ARG), ((0x10000, (1 << 36) + 1, BF16), UNSUP)):
        assert clip(L, [B, bad]) == {want}, bad
        assert clip(L, [bad]) == {want}, bad
        assert clip(L, [(0x900000, bad[1], F32)], out=[bad]) == {want}, bad
        assert L.pcm_grad_norm(tensors(B, bad), 2, P, P, 1 << 20, None) == want, bad
    assert clip(L, [A, B], out=[(0x30000, 64, F32), (0x40000, 63, F32)]) == {ARG}      # another count


def test_clip_refuses_overlaps(L):
    assert clip(L, [A, A]) == {ARG}                                                     # the same one twice
    assert clip(L, [A, B, (0x10000 + 252, 4, F32)]) == {ARG}                            # its last element
    assert clip(L, [A, (0x10000 - 4, 3, BF16)]) == {ARG}                                # its first bytes
    assert clip(L, [A, B], out=[A, A]) == {ARG}                                         # an output on another gradient
    assert clip(L, [A, B], out=[B, A]) == {ARG}
    assert clip(L, [A, B], out=[(0x10000, 64, BF16), B]) == {ARG}                       # itself, in another type
    assert clip(L, [A, B], out=[(0x10004, 64, F32), B]) == {ARG}
    assert clip(L, [A, B], out=[(0x30000, 64, F32), (0x30000 + 128, 64, BF16)]) == {ARG}
    many = [(0x100000 + 4096 * i, 1024, F32) for i in range(4096)]
    assert clip(L, many[:2000] + [(many[2000][0] - 4, 1, F32)] + many[2001:]) == {ARG}


def test_clip_refuses_the_rest(L):
    for max_norm in (-1.0, float("nan"), -float("inf")):
        assert clip(L, [A], max_norm=max_norm) == {ARG}
    assert clip(L, [A], norm=None) == {ARG}
    assert clip(L, [A], norm=ODD) == {ARG}
    assert clip(L, [A], m=-1) == {ARG}
    assert clip(L, [A], m=4097) == {UNSUP}
    assert L.pcm_grad_norm(tensors(A), 4097, P, P, 1 << 20, None) == UNSUP
    assert L.pcm_grad_norm(tensors(A), -1, P, P, 1 << 20, None) == ARG
    assert L.pcm_grad_norm(None, 1, P, P, 1 << 20, None) == ARG
    assert L.pcm_clip_grads(None, None, 1, P, 1.0, None) == ARG
    assert L.pcm_clip_grads(None, None, 0, P, 1.0, None) == OK
    need = binding.workspace_bytes(binding.OP_GRAD_NORM, 1, 0, 0, 1, 1, 0)
    assert need > 0
    for call in (lambda ws, b: L.pcm_grad_norm(tensors(A), 1, P, ws, b, None),
                 lambda ws, b: L.pcm_clip_grad_norm(tensors(A), None, 1, 1.0, P, ws, b, None)):
        assert call(P, need - 1) == WS
        assert call(None, need) == WS
        assert call(MIS, need) == ARG


# ------------------------------------------------------------------------ Python
def test_python_refuses_host_tensors():
    x, of = torch.zeros(4, 64), torch.zeros(4, 2, dtype=torch.int32)
    o, bits, beta = torch.zeros(8, 64), torch.zeros(4, dtype=torch.int64), torch.zeros(4, 2, 2)
    for call in (lambda: pcm.pcm_dispatch_rows(x, of), lambda: pcm.pcm_dispatch_rows_grad(o, of),
                 lambda: pcm.pcm_combine_rows(o, of), lambda: pcm.pcm_combine_rows_grad(x, of), lambda: pcm.pcm_swiglu(x),
                 lambda: pcm.pcm_swiglu_grad(x, x[:, :32]), lambda: pcm.pcm_mix_rows(o, bits, beta, of),
                 lambda: pcm.pcm_mix_rows_grad(o, o, bits, beta, of), lambda: pcm.pcm_route_grad(of, x[:, :2], 8, dw=x[:, :2]),
                 lambda: pcm.pcm_grad_norm([x]), lambda: pcm.pcm_clip_grads([x], x[0, :1], 1.0),
                 lambda: pcm.pcm_clip_grad_norm([x], 1.0)):
        with pytest.raises(ValueError):
            call()


def test_python_refuses_shapes():
    x, of = torch.zeros(4, 64), torch.zeros(4, 2, dtype=torch.int32)
    for call in (lambda: pcm.pcm_dispatch_rows(x[0], of), lambda: pcm.pcm_combine_rows(x[0], of),
                 lambda: pcm.pcm_swiglu(torch.zeros(4, 63)), lambda: pcm.pcm_swiglu(torch.zeros(64)),
                 lambda: pcm.pcm_mix_rows(x[0], of, of, of), lambda: pcm.pcm_route_grad(of[0], x, 8)):
        with pytest.raises(ValueError):
            call()


def test_python_refuses_sizes_past_32_bits():
    wide, on = (1 << 32) + 64, dict(device="meta")
    x, of = torch.empty((1, wide), **on), torch.empty((1, 2), dtype=torch.int32, **on)
    for call in (lambda: pcm.pcm_dispatch_rows(x, of), lambda: pcm.pcm_dispatch_rows_grad(x, of),
                 lambda: pcm.pcm_combine_rows(x, of), lambda: pcm.pcm_combine_rows_grad(x, of),
                 lambda: pcm.pcm_swiglu(torch.empty((1, 2 * wide), **on)), lambda: pcm.pcm_mix_rows(x, of, of, of),
                 lambda: pcm.pcm_mix_rows_grad(x, x, of, of, of), lambda: pcm.pcm_route_grad(x.int(), x, 8)):
        with pytest.raises(ValueError, match="32 bits"):
            call()


def test_python_clips_by_a_norm_that_is_given():
    """The norm is an input: it cannot be left out."""
    with pytest.raises(ValueError, match="norm"):
        pcm.pcm_clip_grads([torch.zeros(4)], None, 1.0)


SMALL_STACK = """
import ctypes, struct, sys, threading
L = ctypes.CDLL(sys.argv[1])
t = ctypes.create_string_buffer(b"".join(struct.pack("<QqQ", 0x100000 + 4096 * (i % 4095), 1024, 0) for i in range(4096)))
to = ctypes.create_string_buffer(b"".join(struct.pack("<QqQ", 0x8000000 + 4096 * i, 1024, 0) for i in range(4096)))
P, F = ctypes.c_void_p, ctypes.c_float
L.pcm_clip_grads.argtypes = [P, P, ctypes.c_int, P, F, P]
got = []
threading.stack_size(96 << 10)
run = threading.Thread(target=lambda: got.append(L.pcm_clip_grads(t, to, 4096, 0x10000, 1.0, None)))
run.start()
run.join()
print("status", got)
"""


def test_clip_checks_on_a_small_stack():
    """4096 tensors with as many results, the last gradient on the first's memory, from a thread with 96 KB of stack."""
    import subprocess
    import sys
    from paper_2609_01024_amd import build
    r = subprocess.run([sys.executable, "-c", SMALL_STACK, build.LIB], capture_output=True, text=True, timeout=60)
    assert r.returncode == 0 and r.stdout.strip() == f"status [{ARG}]", (r.returncode, r.stdout, r.stderr[-500:])


def test_norm_and_workspace_apart_from_the_tensors(L):
    """The norm and the sums behind it on a gradient or a result: read by some workgroups after others wrote there."""
    need = binding.workspace_bytes(binding.OP_GRAD_NORM, 2, 0, 0, 1, 1, 0)
    far, more = ctypes.c_void_p(0x900000), [(0x30000, 64, BF16), (0x40000, 64, F32)]
    on = [0x10000, 0x10000 + 252, 0x20000, 0x20000 + 124]      # first and last elements of A and B
    for p in on:
        norm = ctypes.c_void_p(p)
        assert L.pcm_grad_norm(tensors(A, B), 2, norm, far, need, None) == ARG, hex(p)
        assert clip(L, [A, B], norm=norm, ws=far) == {ARG}, hex(p)
        assert L.pcm_clip_grad_norm(tensors(A, B), tensors(*more), 2, 1.0, norm, far, need, None) == ARG, hex(p)
        assert clip(L, more, out=[B, A], norm=norm, ws=far) == {ARG}, hex(p)
    for p in (0x10000, 0x10000 - need + 16, 0x20000 + 112):
        ws, norm = ctypes.c_void_p(p), ctypes.c_void_p(0x990000)
        assert L.pcm_grad_norm(tensors(A, B), 2, norm, ws, need, None) == ARG, hex(p)
        assert L.pcm_clip_grad_norm(tensors(A, B), None, 2, 1.0, norm, ws, need, None) == ARG, hex(p)
        assert L.pcm_clip_grad_norm(tensors(*more), tensors(B, A), 2, 1.0, norm, ws, need, None) == ARG, hex(p)
    for p in (0x900000, 0x900000 + need - 4):                  # the norm in the workspace
        norm = ctypes.c_void_p(p)
        assert L.pcm_grad_norm(tensors(A, B), 2, norm, far, need, None) == ARG
        assert L.pcm_clip_grad_norm(tensors(A, B), None, 2, 1.0, norm, far, need, None) == ARG
