"""The training step's operators around the experts' products against the same formulas in 64 bits (needs an MI355X).

Bounds, u = 2^-24 (half a step of float32): a sum of m fused products in any order is off by at most m u S (1 + m u), S
the sum of the magnitudes, for which (m + 1) u S stands here; a bf16 result adds half its step, 2^-8 of the value. A copy
is exact, a product by a float32 weight rounds once more. Below the normal range, 2^-126, values lie 2^-149 apart in
float32 and 2^-133 in bf16 (2^-126 times its 2^-7), half a step of which is 2^-134 whatever the value."""
import math
import sys

import pytest
import torch

import paper_2609_01024_amd as pcm
from paper_2609_01024_amd import binding

pytestmark = pytest.mark.gpu
DEV = "cuda"
U = 2.0 ** -24
BF, F32 = torch.bfloat16, torch.float32
TYPES = {"bf16-bf16": (BF, BF), "bf16-f32": (BF, F32), "f32-f32": (F32, F32), "f32-bf16": (F32, BF)}


@pytest.fixture(autouse=True)
def _named(request):
    print(request.node.name, flush=True)
    sys.stdout.flush()
    yield


def gpu(t):
    return None if t is None else t.to(DEV)


def close(got, want, room, what=""):
    """got within `room` of want (both 64 bits), and half a step of bf16 where it is bf16."""
    half, least = (2.0 ** -8, 2.0 ** -134) if got.dtype == BF else (0.0, 0.0)
    got = got.detach().cpu().double()
    assert got.shape == want.shape, (what, got.shape, want.shape)
    bound = room + torch.clamp(half * (want.abs() + room), min=least) + 1e-44
    d = (got - want).abs()
    bad = ~(d <= bound)
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.numel()} outside, worst {float((d / bound).nan_to_num(1e9).max()):.3g} of the bound"


def same_bits(a, b):
    assert a.dtype == b.dtype and a.shape == b.shape
    assert torch.equal(a.cpu().contiguous().view(torch.uint8), b.cpu().contiguous().view(torch.uint8))


# ------------------------------------------------------------------------ tokens to rows and back
# T, k, n, width: one of everything, widths of part of a wave, of several workgroups and odd ones
SHAPES = [(1, 1, 1, 16), (1, 8, 256, 48), (5, 3, 7, 80), (33, 2, 4, 2064), (70, 4, 9, 528), (200, 8, 64, 208), (3, 7, 8, 4112),
          (16, 5, 6, 7168), (129, 6, 40, 1024)]


def routed(T, k, n, seed=0):
    """Rows of T tokens: offsets, row_token, row_slot, row_of, and the ids and weights behind them."""
    g = torch.Generator().manual_seed(seed)
    top, ids = torch.randn((T, n), generator=g).topk(k, 1)
    order = ids.reshape(-1).sort(stable=True).indices
    of = torch.empty_like(order)
    of[order] = torch.arange(T * k)
    counts = torch.bincount(ids.reshape(-1), minlength=n)
    off = torch.cat([torch.zeros(1, dtype=torch.int64), counts.cumsum(0)])
    return dict(off=off.int(), tok=order // k, slot=order % k, of=of.reshape(T, k).int(), ids=ids.int(), p=top.softmax(1))


def tokens_and_rows(shape, dtype, held, seed=0):
    T, k, n, H = shape
    r = routed(T, k, n, seed)
    g = torch.Generator().manual_seed(seed + 1)
    r["x"], r["o"] = torch.randn((T, H), generator=g).to(dtype), torch.randn((T * k, H), generator=g).to(dtype)
    r["w"] = torch.rand((T, k), generator=g)
    if held == "all":
        r["off"] = None
        r["on"] = torch.ones((T, k), dtype=torch.bool)
    else:      # the middle half of the experts
        r["off"] = r["off"][n // 4:max(n // 4 + 2, 3 * n // 4 + 1)] if n > 1 else r["off"]
        r["on"] = (r["of"] >= r["off"][0]) & (r["of"] < r["off"][-1])
    return r


@pytest.mark.parametrize("held", ["all", "some"])
@pytest.mark.parametrize("types", TYPES)
@pytest.mark.parametrize("shape", SHAPES)
def test_dispatch(shape, types, held):
    dt, out = TYPES[types]
    c = tokens_and_rows(shape, dt, held)
    T, k, n, H = shape
    at, slot = c["tok"], c["slot"]
    on = c["on"][at, slot]
    y = pcm.pcm_dispatch_rows(gpu(c["x"]), gpu(c["of"]), gpu(c["w"]), gpu(c["off"]),
                              y=torch.full((T * k, H), 7.0, dtype=out, device=DEV))
    want = c["x"].double()[at] * c["w"].double()[at, slot][:, None]
    close(y[gpu(on)], want[on], U * want[on].abs(), "y")
    assert bool((y[gpu(~on)] == 7.0).all())          # rows of no pair, left as they were
    plain = pcm.pcm_dispatch_rows(gpu(c["x"]), gpu(c["of"]), None, gpu(c["off"]), out_dtype=out)
    same_bits(plain[gpu(on)], c["x"][at].to(out)[on])


@pytest.mark.parametrize("held", ["all", "some"])
@pytest.mark.parametrize("types", TYPES)
@pytest.mark.parametrize("shape", SHAPES)
def test_combine_and_dispatch_gradient(shape, types, held):
    """Both are the weighted sum of a token's rows; the gradient also gives the weights'."""
    dt, out = TYPES[types]
    c = tokens_and_rows(shape, dt, held)
    T, k, n, H = shape
    o = c["o"].clone()
    o[c["of"][~c["on"]].long()] = float("nan")        # never read into a result
    args = gpu(c["of"]), gpu(c["w"]), gpu(c["off"])
    rows = torch.where(c["on"][:, :, None], c["o"].double()[c["of"].long()], 0.0)
    terms = rows * c["w"].double()[:, :, None]
    want, room = terms.sum(1), (k + 1) * U * terms.abs().sum(1)
    close(pcm.pcm_combine_rows(gpu(o), *args, out_dtype=out), want, room, "y")
    dx, dw = pcm.pcm_dispatch_rows_grad(gpu(o), args[0], gpu(c["x"]), args[1], args[2], out_dtype=out)
    close(dx, want, room, "dx")
    prods = rows * c["x"].double()[:, None, :]
    close(dw, prods.sum(2), (H + 1) * U * prods.abs().sum(2), "dweights")
    assert bool((dw[gpu(~c["on"])] == 0).all())
    none, nothing = pcm.pcm_dispatch_rows_grad(gpu(o), args[0], None, None, args[2], out_dtype=out)
    assert nothing is None
    close(none, rows.sum(1), (k + 1) * U * rows.abs().sum(1), "dx without weights")
    if out == F32:
        before = torch.randn((T, H), generator=torch.Generator().manual_seed(3))
        y = pcm.pcm_combine_rows(gpu(o), *args, y=gpu(before), accumulate=True)
        close(y, before.double() + want, room + 2 * U * (before.double().abs() + terms.abs().sum(1)), "accumulated")


@pytest.mark.parametrize("held", ["all", "some"])
@pytest.mark.parametrize("types", TYPES)
@pytest.mark.parametrize("shape", SHAPES)
def test_combine_gradient(shape, types, held):
    dt, out = TYPES[types]
    c = tokens_and_rows(shape, dt, held)
    T, k, n, H = shape
    at, slot = c["tok"], c["slot"]
    on = c["on"][at, slot]
    o = c["o"].clone()
    o[c["of"][~c["on"]].long()] = float("nan")
    do, dw = pcm.pcm_combine_rows_grad(gpu(c["x"]), gpu(c["of"]), gpu(o), gpu(c["w"]), gpu(c["off"]),
                                       do=torch.full((T * k, H), 7.0, dtype=out, device=DEV))
    want = c["x"].double()[at] * c["w"].double()[at, slot][:, None]
    close(do[gpu(on)], want[on], U * want[on].abs(), "do")
    assert bool((do[gpu(~on)] == 7.0).all())
    prods = torch.where(c["on"][:, :, None], c["o"].double()[c["of"].long()], 0.0) * c["x"].double()[:, None, :]
    close(dw, prods.sum(2), (H + 1) * U * prods.abs().sum(2), "dweights")
    assert bool((dw[gpu(~c["on"])] == 0).all())
    alone, nothing = pcm.pcm_combine_rows_grad(gpu(c["x"]), gpu(c["of"]), None, gpu(c["w"]), gpu(c["off"]), rows=T * k, out_dtype=out)
    assert nothing is None
    same_bits(alone[gpu(on)], do[gpu(on)])


@pytest.mark.parametrize("out", ["bf16", "f32"])
@pytest.mark.parametrize("tokens,rows", [(BF, F32), (F32, BF)])
@pytest.mark.parametrize("shape", [(1, 1, 1, 16), (33, 2, 4, 2064), (70, 5, 9, 528), (3, 8, 8, 7168)])
def test_row_gradients_of_two_types(shape, tokens, rows, out):
    """Tokens of one type and rows of the other: a float32 gradient of outputs that were kept in bf16, and the other way."""
    T, k, n, H = shape
    out = {"bf16": BF, "f32": F32}[out]
    c = tokens_and_rows(shape, F32, "all", 9)
    x, o, of = c["x"].to(tokens), c["o"].to(rows), c["of"].long()
    O, X, W = o.double()[of], x.double()[:, None, :], c["w"].double()[:, :, None]
    dots, mag = (O * X).sum(2), (O * X).abs().sum(2)
    do, dw = pcm.pcm_combine_rows_grad(gpu(x), gpu(c["of"]), gpu(o), gpu(c["w"]), out_dtype=out)
    close(do[gpu(of)], X * W, U * (X * W).abs(), "do")
    close(dw, dots, (H + 1) * U * mag, "dweights")
    dx, dw = pcm.pcm_dispatch_rows_grad(gpu(o), gpu(c["of"]), gpu(x), gpu(c["w"]), out_dtype=out)
    close(dx, (O * W).sum(1), (k + 1) * U * (O * W).abs().sum(1), "dx")
    close(dw, dots, (H + 1) * U * mag, "dweights")


def test_widest_rows():
    """2^28 columns of small integers: a lane's sums stay below 2^24 and are exact, about ten additions after them round by
    2^-24 each."""
    H = 1 << 28
    x = torch.ones((1, H), dtype=BF, device=DEV)
    x[0, ::3] = 2.0
    of, w = torch.zeros((1, 1), dtype=torch.int32, device=DEV), torch.full((1, 1), 4.0, device=DEV)
    y = pcm.pcm_dispatch_rows(x, of, w)
    assert torch.equal(y, 4 * x)
    assert torch.equal(pcm.pcm_combine_rows(y, of, w), 16 * x)
    bits = torch.ones(1, dtype=torch.int64, device=DEV)
    assert torch.equal(pcm.pcm_mix_rows(x, bits, w[:, :, None].contiguous(), of), y)
    twos = (H + 2) // 3
    want = float(H - twos + 4 * twos)
    dx, dw = pcm.pcm_dispatch_rows_grad(x, of, x, w)
    assert torch.equal(dx, y) and abs(float(dw) - want) <= want * 2 ** -20
    du, dbeta = pcm.pcm_mix_rows_grad(x, x, bits, w[:, :, None].contiguous(), of)
    assert torch.equal(du, y) and abs(float(dbeta) - want) <= want * 2 ** -20


@pytest.mark.parametrize("types", ["bf16-f32", "f32-f32"])
def test_row_gradients_against_differences(types):
    """<dy, f(v + d) - f(v - d)> = 2 <df, d> in each argument, which the operators are linear in. Small integers and
    weights of quarters keep every sum exact in float32: both sides have to be equal."""
    dt, out = TYPES[types]
    T, k, n, H = 21, 3, 5, 112
    c = tokens_and_rows((T, k, n, H), dt, "all", 4)
    g = torch.Generator().manual_seed(8)
    ints = lambda shape, m: torch.randint(-m, m + 1, shape, generator=g).to(dt)
    x, vx, o, vo, dy, dr = ints((T, H), 3), ints((T, H), 2), ints((T * k, H), 3), ints((T * k, H), 2), ints((T, H), 3), ints((T * k, H), 3)
    w, vw = torch.randint(0, 5, (T, k), generator=g) / 4, torch.randint(-2, 3, (T, k), generator=g) / 4
    of = gpu(c["of"])
    forth = lambda x, w: pcm.pcm_dispatch_rows(gpu(x), of, gpu(w), out_dtype=F32).cpu().double()
    back = lambda o, w: pcm.pcm_combine_rows(gpu(o), of, gpu(w), out_dtype=F32).cpu().double()
    dx, dwx = (t.cpu().double() for t in pcm.pcm_dispatch_rows_grad(gpu(dr), of, gpu(x), gpu(w), out_dtype=F32))
    do, dwo = (t.cpu().double() for t in pcm.pcm_combine_rows_grad(gpu(dy), of, gpu(o), gpu(w), out_dtype=F32))
    dot = lambda a, b: float((a.double() * b.double()).sum())
    assert dot(dr, forth(x + vx, w) - forth(x - vx, w)) == 2 * dot(dx, vx)
    assert dot(dr, forth(x, w + vw) - forth(x, w - vw)) == 2 * dot(dwx, vw)
    assert dot(dy, back(o + vo, w) - back(o - vo, w)) == 2 * dot(do, vo)
    assert dot(dy, back(o, w + vw) - back(o, w - vw)) == 2 * dot(dwo, vw)


@pytest.mark.parametrize("number", [-1, 60, 1 << 30, -(1 << 31), (1 << 31) - 1])
@pytest.mark.parametrize("types", ["bf16-bf16", "f32-f32"])
def test_numbers_that_are_no_row(types, number):
    """Such a pair has no part; a token without rows has a zero sum."""
    dt, _ = TYPES[types]
    T, k, n, H = 20, 3, 6, 272
    c = tokens_and_rows((T, k, n, H), dt, "all", 2)
    of = c["of"].clone()
    of[3], of[7, 1], of[19, 0] = number, number, number
    on = of == c["of"]
    o = c["o"].clone()
    o[c["of"][~on].long()] = float("nan")
    X, O, W, OF = gpu(c["x"]), gpu(o), gpu(c["w"]), gpu(of)
    rows = torch.where(on[:, :, None], c["o"].double()[c["of"].long()], 0.0)
    terms = rows * c["w"].double()[:, :, None]
    y = pcm.pcm_combine_rows(O, OF, W)
    close(y, terms.sum(1), (k + 1) * U * terms.abs().sum(1), "y")
    assert bool((y[3] == 0).all())
    do, dw = pcm.pcm_combine_rows_grad(X, OF, O, W, do=torch.full((T * k, H), 7.0, dtype=dt, device=DEV))
    gone = c["of"][~on].long()
    assert bool((do[gpu(gone)] == 7.0).all()) and int((do == 7.0).all(1).sum()) == len(gone)
    assert bool((dw[gpu(~on)] == 0).all()) and bool(torch.isfinite(dw).all())
    yr = pcm.pcm_dispatch_rows(X, OF, W, y=torch.full((T * k, H), 7.0, dtype=dt, device=DEV))
    same_bits(yr, do)


def test_groups_bounds_are_held_inside():
    """Offsets that lie outside the rows, or descend: no memory outside, no rows where they say none."""
    c = tokens_and_rows((9, 2, 4, 64), F32, "all")
    X, OF, O = gpu(c["x"]), gpu(c["of"]), gpu(c["o"])
    for off, first, end in (([-5, 99], 0, 18), ([7, 3], 0, 0), ([1 << 30, 1 << 30], 0, 0), ([4, 1 << 30], 4, 18), ([-9, -3], 0, 0)):
        OFF = torch.tensor(off, dtype=torch.int32, device=DEV)
        on = ((c["of"] >= first) & (c["of"] < end))
        want = torch.where(on[:, :, None], c["o"].double()[c["of"].long()], 0.0)
        close(pcm.pcm_combine_rows(O, OF, None, OFF), want.sum(1), 3 * U * want.abs().sum(1), str(off))
        y = pcm.pcm_dispatch_rows(X, OF, None, OFF, y=torch.full((18, 64), 7.0, device=DEV))
        assert int((y != 7.0).any(1).sum()) == end - first, off


def test_a_part_of_the_offsets():
    """A rank's part of a table's offsets, as a view that starts at any of them."""
    c = tokens_and_rows((50, 2, 7, 96), BF, "all", 6)
    off = routed(50, 2, 7, 6)["off"].to(DEV)
    for a, b in ((1, 4), (2, 3), (3, 7), (0, 7)):
        on = (c["of"] >= int(off[a])) & (c["of"] < int(off[b]))
        want = torch.where(on[:, :, None], c["o"].double()[c["of"].long()], 0.0)
        y = pcm.pcm_combine_rows(gpu(c["o"]), gpu(c["of"]), None, off[a:b + 1], out_dtype=F32)
        close(y, want.sum(1), 3 * U * want.abs().sum(1), (a, b))


@pytest.mark.parametrize("H", [80, 4112])
@pytest.mark.parametrize("types", ["bf16-f32", "f32-f32"])
def test_products_alone(types, H):
    """The C entry points without the tensor gradient: dweights and dbeta as with it."""
    dt, out = TYPES[types]
    T, k, n = 30, 3, 5
    c = tokens_and_rows((T, k, n, H), dt, "all", 3)
    m = path_case(T, k, n, H, dt, 0.4, 3)
    code = binding.PCM_BF16 if dt == BF else binding.PCM_F32
    x, o, of, w, bits, beta, u, dz = (gpu(v) for v in (c["x"], c["o"], c["of"], c["w"], m["bits"], m["beta"], m["u"], m["dz"]))
    got = torch.full((T, k), 7.0, device=DEV)
    L, P, R = pcm.lib(), torch.Tensor.data_ptr, T * k
    assert L.pcm_dispatch_rows_grad(code, code, 0, P(o), P(x), P(of), P(w), None, T, k, R, H, 1, None, P(got), None) == 0
    torch.cuda.synchronize()
    same_bits(got, pcm.pcm_dispatch_rows_grad(o, of, x, w, out_dtype=F32)[1])
    got.fill_(7.0)
    assert L.pcm_combine_rows_grad(code, code, 0, P(x), P(o), P(of), P(w), None, T, k, R, H, 1, None, P(got), None) == 0
    torch.cuda.synchronize()
    same_bits(got, pcm.pcm_combine_rows_grad(x, of, o, w, out_dtype=F32)[1])
    got = torch.full((T, k, k), 7.0, device=DEV)
    mof = gpu(m["of"])
    assert L.pcm_mix_rows_grad(code, 0, P(dz), P(u), P(bits), P(beta), P(mof), P(mof), T, k, R, R, H, None, P(got), None) == 0
    torch.cuda.synchronize()
    same_bits(got, pcm.pcm_mix_rows_grad(dz, u, bits, beta, mof, out_dtype=F32)[1])


def test_rows_past_32_bits():
    """Rows whose first element lies past 2^31: the last ones of a buffer of 4.6 GB."""
    R, H, k = 1_100_000, 2080, 2
    rows = torch.empty((R, H), dtype=BF, device=DEV)
    g = torch.Generator().manual_seed(1)
    at = torch.tensor([[R - 1, 5], [R - 70_000, R - 2], [0, R - 33]], dtype=torch.int32)
    v, x = torch.randn((6, H), generator=g).to(BF), torch.randn((3, H), generator=g).to(BF)
    rows[gpu(at.reshape(-1).long())] = gpu(v)
    y, of = v.double().reshape(3, 2, H), gpu(at)
    close(pcm.pcm_combine_rows(rows, of), y.sum(1), 3 * U * y.abs().sum(1), "y")
    prods = y * x.double()[:, None, :]
    close(pcm.pcm_dispatch_rows_grad(rows, of, gpu(x))[1], prods.sum(2), (H + 1) * U * prods.abs().sum(2), "dweights")
    pcm.pcm_dispatch_rows(gpu(x), of, y=rows)
    same_bits(rows[gpu(at.reshape(-1).long())], x.repeat_interleave(2, 0))
    bits, beta = torch.tensor([0b1001, 0b1111, 0b0010], device=DEV), torch.rand((3, 2, 2), generator=g)
    allowed = torch.tensor([[[1, 0], [0, 1]], [[1, 1], [1, 1]], [[0, 1], [0, 0]]]).double()
    src = x.double().repeat_interleave(2, 0).reshape(3, 2, H)
    z = torch.empty((R, H), dtype=BF, device=DEV)
    pcm.pcm_mix_rows(rows, bits, gpu(beta), of, z=z)
    w = beta.double() * allowed
    close(z[gpu(at.reshape(-1).long())], torch.matmul(w.mT, src).reshape(6, H), 3 * U * torch.matmul(w.mT, src.abs()).reshape(6, H), "z")
    dz = v.double().reshape(3, 2, H)
    z[gpu(at.reshape(-1).long())] = gpu(v)
    du, dbeta = pcm.pcm_mix_rows_grad(z, rows, bits, gpu(beta), of, du=torch.empty((R, H), dtype=BF, device=DEV))
    close(du[gpu(at.reshape(-1).long())], torch.matmul(w, dz).reshape(6, H), 3 * U * torch.matmul(w, dz.abs()).reshape(6, H), "du")
    close(dbeta, torch.matmul(src, dz.mT) * allowed, (H + 1) * U * torch.matmul(src.abs(), dz.abs().mT), "dbeta")


def test_many_tokens():
    """More tokens than a launch has workgroups (2^21, of four tokens in the mix gradient)."""
    T, H = 8_500_001, 16
    x = torch.randint(-3, 4, (T, H), generator=torch.Generator().manual_seed(1)).to(BF)
    of = torch.randperm(T, generator=torch.Generator().manual_seed(2)).int()[:, None]
    X, OF = gpu(x), gpu(of)
    y = pcm.pcm_dispatch_rows(X, OF)
    assert torch.equal(y[OF[:, 0].long()], X)
    back, dots = pcm.pcm_dispatch_rows_grad(y, OF, X)
    assert torch.equal(back, X)
    assert torch.equal(dots[:, 0], X.float().square().sum(1))        # integers: exact
    bits, beta = torch.ones(T, dtype=torch.int64, device=DEV), torch.full((T, 1, 1), 2.0, device=DEV)
    assert torch.equal(pcm.pcm_mix_rows(y, bits, beta, OF), 2 * y)
    du, dbeta = pcm.pcm_mix_rows_grad(y, y, bits, beta, OF)
    assert torch.equal(du, 2 * y) and torch.equal(dbeta[:, 0, 0], dots[:, 0])
    ids = torch.zeros((T, 1), dtype=torch.int32, device=DEV)
    d = pcm.pcm_route_grad(ids, torch.full((T, 1), 0.5, device=DEV), 3, dw=dots)
    assert torch.equal(d[:, 0], 0.25 * dots[:, 0]) and not bool(d[:, 1:].any())


# From 96 MB read on the kernels load non-temporally: the same at few tokens whose rows lie anywhere in buffers of that size.
LARGE = 96 << 20


def rows_in_a_large_buffer(T, k, H, dtype, seed):
    """(R, of [T, k]) of rows spread over a buffer of at least LARGE bytes, the first and last ones among them."""
    R = LARGE // (H * (2 if dtype == BF else 4)) + 1
    g = torch.Generator().manual_seed(seed)
    at = torch.randperm(R, generator=g)[:T * k]
    if T * k > 1:
        at[at == 0], at[at == R - 1] = at[0].item(), at[-1].item()
        at[0], at[-1] = 0, R - 1
    assert at.unique().numel() == T * k
    return R, at.reshape(T, k).int()


def in_a_large_buffer(R, of, v, fill=float("nan")):
    """[R, H], `fill` but for the rows v [T, k, H] of `of`."""
    o = torch.full((R, v.shape[-1]), fill, dtype=v.dtype, device=DEV)
    o[gpu(of.reshape(-1).long())] = gpu(v.reshape(-1, v.shape[-1]))
    return o


@pytest.mark.parametrize("out", ["bf16", "f32"])
@pytest.mark.parametrize("tokens,rows", [(BF, BF), (F32, F32), (BF, F32), (F32, BF)], ids=str)
@pytest.mark.parametrize("k,H", [(1, 2064), (2, 208), (3, 2064), (4, 528), (5, 208), (8, 2064)])
def test_rows_of_large_buffers(k, H, tokens, rows, out):
    T, out = 37, {"bf16": BF, "f32": F32}[out]
    R, of = rows_in_a_large_buffer(T, k, H, rows, k)
    g = torch.Generator().manual_seed(k + 1)
    x, v, w = torch.randn((T, H), generator=g).to(tokens), torch.randn((T, k, H), generator=g).to(rows), torch.rand((T, k), generator=g)
    o = in_a_large_buffer(R, of, v)
    X, V, W = x.double()[:, None, :], v.double(), w.double()[:, :, None]
    want, room = (V * W).sum(1), (k + 1) * U * (V * W).abs().sum(1)
    dots, dots_room = (V * X).sum(2), (H + 1) * U * (V * X).abs().sum(2)
    if tokens == rows:
        close(pcm.pcm_combine_rows(o, gpu(of), gpu(w), out_dtype=out), want, room, "y")
    dx, dw = pcm.pcm_dispatch_rows_grad(o, gpu(of), gpu(x), gpu(w), out_dtype=out)
    close(dx, want, room, "dx")
    close(dw, dots, dots_room, "dweights")
    do, dw = pcm.pcm_combine_rows_grad(gpu(x), gpu(of), o, gpu(w), do=torch.full((R, H), 7.0, dtype=out, device=DEV))
    close(do[gpu(of.long())], X * W, U * (X * W).abs(), "do")
    close(dw, dots, dots_room, "dweights")
    do[gpu(of.reshape(-1).long())] = 7.0
    assert bool((do == 7.0).all())


def test_training_sized_row_gradients():
    """Every token of a large batch, four rows each; the products of small integers are exact in float32."""
    T, k, H = 16_384, 4, 1040
    g = torch.Generator(device=DEV).manual_seed(3)
    x = torch.randint(-3, 4, (T, H), generator=g, device=DEV).to(BF)
    o = torch.randint(-3, 4, (T * k, H), generator=g, device=DEV).to(BF)
    of = torch.randperm(T * k, generator=g, device=DEV).reshape(T, k).int()
    w = torch.randint(1, 4, (T, k), generator=g, device=DEV).float() / 4
    rows = o[of.long()].float()
    dots = (rows * x.float()[:, None, :]).sum(2)
    do, dw = pcm.pcm_combine_rows_grad(x, of, o, w, out_dtype=F32)
    assert torch.equal(do[of.long()], x.float()[:, None, :] * w[:, :, None]) and torch.equal(dw, dots)
    dx, dw = pcm.pcm_dispatch_rows_grad(o, of, x, w, out_dtype=F32)
    assert torch.equal(dx, (rows * w[:, :, None]).sum(1)) and torch.equal(dw, dots)


def test_no_tokens_and_no_rows():
    e = lambda *s, dt=F32: torch.empty(s, dtype=dt, device=DEV)
    i = lambda *s: torch.empty(s, dtype=torch.int32, device=DEV)
    assert pcm.pcm_dispatch_rows(e(0, 32), i(0, 2)).shape == (0, 32)
    assert pcm.pcm_combine_rows(e(0, 32), i(0, 2)).shape == (0, 32)
    of = torch.full((3, 2), -1, dtype=torch.int32, device=DEV)
    assert not bool(pcm.pcm_combine_rows(e(0, 32), of).any())
    dx, dw = pcm.pcm_dispatch_rows_grad(e(0, 32), of, torch.ones((3, 32), device=DEV))
    assert not bool(dx.any()) and not bool(dw.any())
    do, dw = pcm.pcm_combine_rows_grad(torch.ones((3, 32), device=DEV), of, e(0, 32))
    assert do.shape == (0, 32) and not bool(dw.any())
    assert pcm.pcm_dispatch_rows(torch.ones((3, 32), device=DEV), of, rows=0).shape == (0, 32)
    bits, beta = torch.full((3,), 15, device=DEV), torch.ones((3, 2, 2), device=DEV)
    z = pcm.pcm_mix_rows(e(0, 32), bits, beta, of, gpu(torch.arange(6, dtype=torch.int32).reshape(3, 2)), rows=6)
    assert z.shape == (6, 32) and not bool(z.any())
    du, dbeta = pcm.pcm_mix_rows_grad(e(0, 32), e(0, 32), bits, beta, of)
    assert du.shape == (0, 32) and not bool(dbeta.any())
    assert pcm.pcm_swiglu(e(0, 64)).shape == (0, 32) and pcm.pcm_swiglu_grad(e(0, 64), e(0, 32)).shape == (0, 64)
    assert pcm.pcm_route_grad(i(0, 2), e(0, 2), 4, dw=e(0, 2)).shape == (0, 4)


@pytest.mark.parametrize("value", [float("nan"), float("inf")])
def test_values_that_are_not_finite_stay_in_their_tokens(value):
    c = tokens_and_rows((12, 2, 4, 80), BF, "all", 5)
    x, o = c["x"].clone(), c["o"].clone()
    x[5, 3] = value
    o[c["of"][2, 1].long(), 9] = value
    y = pcm.pcm_combine_rows(gpu(o), gpu(c["of"]), gpu(c["w"])).cpu()
    assert (~torch.isfinite(y)).nonzero().tolist() == [[2, 9]]
    do, dw = (t.cpu() for t in pcm.pcm_combine_rows_grad(gpu(x), gpu(c["of"]), gpu(c["o"]), gpu(c["w"])))
    assert (~torch.isfinite(do)).sum() == 2 and (~torch.isfinite(dw)).any(1).nonzero().tolist() == [[5]]


# ------------------------------------------------------------------------ SwiGLU
def swiglu64(gate, up):
    return gate * torch.sigmoid(gate) * up


def swiglu_room(gate, up, value):
    """float32 inputs: e^-g 2u, the sum and the division u each, the product with up u: 5u and a spare one. bf16 inputs:
    e^-g from 2^i 2^f: log2 e is off by u / 2 relative, so the exponent by |g| log2(e) u / 2 and e^-g by |g| u / 2, f's
    rounding and the exponential 3u, reciprocal 2u, two products 2u: (8 + |g|) u stands for both. Below the normal range:
    the factor SiLU has steps of 2^-149."""
    return (8 + gate.abs()) * U * value.abs() + (1 + gate.abs()) * (1 + up.abs()) * 2.0 ** -148


def swiglu_grads64(gate, up, du):
    s, c = torch.sigmoid(gate), torch.sigmoid(-gate)
    return torch.cat([du * up * s * (1 + gate * c), du * gate * s], 1)


def swiglu_grad_room(gate, up, du):
    """Float32 steps: e^-g 2u, s 4u, 1 - s as e^-g s 7u, so 1 + g (1 - s) is off by 9u (1 + |g| (1 - s)); three products and s
    again: 17u |du up| s (1 + |g| (1 - s)), and 8u of d up. Far gates: two exponentials of g / 2, 2u each, g / 2 exact, three
    more products: less. Plus steps of 2^-149 where a factor is below the normal range."""
    s, c = torch.sigmoid(gate), torch.sigmoid(-gate)
    low = (1 + gate.abs()) * 2.0 ** -147
    return torch.cat([17 * U * (du * up).abs() * s * (1 + gate.abs() * c) + low * (1 + up.abs()),
                      8 * U * (du * gate).abs() * s + low * (1 + du.abs())], 1)


def check_swiglu(gate, up, du, dt, out):
    gu = torch.cat([gate, up], 1).to(dt)
    F = gate.shape[1]
    gate, up, d = gu[:, :F].double(), gu[:, F:].double(), du.to(dt)
    want = swiglu64(gate, up)
    close(pcm.pcm_swiglu(gpu(gu), out_dtype=out), want, swiglu_room(gate, up, want), "u")
    got = pcm.pcm_swiglu_grad(gpu(gu), gpu(d), out_dtype=out)
    close(got, swiglu_grads64(gate, up, d.double()), swiglu_grad_room(gate, up, d.double()), "dgate_up")


@pytest.mark.parametrize("types", TYPES)
@pytest.mark.parametrize("R,F", [(1, 16), (7, 48), (64, 208), (300, 1408), (5, 4112)])
def test_swiglu(R, F, types):
    g = torch.Generator().manual_seed(R)
    check_swiglu(*(torch.randn((R, F), generator=g) * s for s in (3.0, 1.0, 1.0)), *TYPES[types])


@pytest.mark.parametrize("up,du", [(1.0, 1.0), (2.0 ** 60, 1.0), (1.0, 2.0 ** 60), (2.0 ** 60, 2.0 ** 60), (2.0 ** -30, 1.5)])
@pytest.mark.parametrize("types", TYPES)
def test_swiglu_of_every_gate(types, up, du):
    """Every finite bf16 gate up to 2^60 in magnitude."""
    bits = torch.arange(1 << 16, dtype=torch.int32).to(torch.int16)
    gates = bits.view(BF).float()
    gates = gates[torch.isfinite(gates) & (gates.abs() <= 2.0 ** 60)]
    gates = gates[:gates.numel() // 16 * 16].reshape(-1, 16)
    check_swiglu(gates, torch.full_like(gates, up), torch.full_like(gates, du), *TYPES[types])


def test_swiglu_gradient_of_far_gates_in_float32():
    """Around where one form takes over from the other, and where SiLU falls below the normal range: values between bf16's."""
    g = torch.Generator().manual_seed(2)
    gates = torch.cat([-64 + torch.randn(4096, generator=g) * 0.01, -torch.rand(4096, generator=g) * 180,
                       torch.rand(4096, generator=g) * 180, -1.2784645 + torch.randn(4096, generator=g) * 1e-4]).reshape(-1, 16)
    for up in (1.0, 2.0 ** 70):
        check_swiglu(gates, torch.full_like(gates, up), torch.ones_like(gates), F32, F32)


def test_swiglu_gradient_against_differences():
    """Central differences of the forward pass in float32: steps of 2^-8 leave h^2 / 6 of the third derivative (below 1 for
    SiLU) times |up du|, and the two values' roundings, 8u each of at most 3 |up|, over 2h."""
    g = torch.Generator().manual_seed(3)
    gate, up, du = (torch.randn((20, 64), generator=g) for _ in range(3))
    h = 2.0 ** -8
    f = lambda gate, up: pcm.pcm_swiglu(gpu(torch.cat([gate, up], 1))).cpu().double()
    d = pcm.pcm_swiglu_grad(gpu(torch.cat([gate, up], 1)), gpu(du)).cpu().double()
    D = du.double()
    by_gate, by_up = (f(gate + h, up) - f(gate - h, up)) / (2 * h) * D, (f(gate, up + h) - f(gate, up - h)) / (2 * h) * D
    # (gate + h is rounded: another u |gate| over h)
    room = D.abs() * (1 + up.double().abs()) * (h * h / 6 + 2 * (8 * 3 * U + 4 * U) / h)
    assert bool(((d[:, :64] - by_gate).abs() <= room).all()) and bool(((d[:, 64:] - by_up).abs() <= room * 4).all())


@pytest.mark.parametrize("R,count", [(50, 0), (50, 1), (50, 37), (50, 50), (50, 99), (50, -3)])
def test_swiglu_of_counted_rows(R, count):
    g = torch.Generator().manual_seed(4)
    gu, du = torch.randn((R, 160), generator=g).to(BF), torch.randn((R, 80), generator=g).to(BF)
    n, done = torch.tensor([9, count, 9], dtype=torch.int32, device=DEV)[1:2], min(max(count, 0), R)
    u = pcm.pcm_swiglu(gpu(gu), n, u=torch.full((R, 80), 7.0, dtype=BF, device=DEV))
    d = pcm.pcm_swiglu_grad(gpu(gu), gpu(du), n, dgate_up=torch.full((R, 160), 7.0, dtype=BF, device=DEV))
    assert bool((u[done:] == 7.0).all()) and bool((d[done:] == 7.0).all())
    same_bits(u[:done], pcm.pcm_swiglu(gpu(gu))[:done])
    same_bits(d[:done], pcm.pcm_swiglu_grad(gpu(gu), gpu(du))[:done])


def test_swiglu_gives_what_its_quantiser_quantises():
    g = torch.Generator().manual_seed(6)
    for dt in (BF, F32):
        gu = gpu(torch.randn((30, 288), generator=g).to(dt))
        u = pcm.pcm_swiglu(gu, out_dtype=F32)
        a, b = pcm.pcm_quant_fp8_rows(u), pcm.pcm_swiglu_quant_fp8(gu)
        same_bits(a[0], b[0])
        same_bits(a[1], b[1])


def test_swiglu_past_32_bits():
    """More than 2^31 elements; the last rows are looked at."""
    R, F = 540_000, 2064
    gu = torch.zeros((R, 2 * F), dtype=BF, device=DEV)
    last = torch.randn((40, 2 * F), generator=torch.Generator().manual_seed(1)).to(BF)
    gu[-40:] = gpu(last)
    gate, up = last[:, :F].double(), last[:, F:].double()
    u = pcm.pcm_swiglu(gu)
    close(u[-40:], swiglu64(gate, up), swiglu_room(gate, up, swiglu64(gate, up)), "u")
    d = pcm.pcm_swiglu_grad(gu, u)
    du = u[-40:].cpu().double()
    close(d[-40:], swiglu_grads64(gate, up, du), swiglu_grad_room(gate, up, du), "dgate_up")
    assert not bool(u[:-40].any()) and not bool(d[:100].any())


@pytest.mark.parametrize("types", TYPES)
def test_swiglu_of_many_rows(types):
    """From 96 MB read on, every element, in 64 bits on the card."""
    dt, out = TYPES[types]
    F = 1040
    R = LARGE // (2 * F * (2 if dt == BF else 4)) + 3
    g = torch.Generator(device=DEV).manual_seed(2)
    gu, du = (torch.randn((R, n), generator=g, device=DEV, dtype=dt) * 3 for n in (2 * F, F))
    gate, up, d = gu[:, :F].double(), gu[:, F:].double(), du.double()

    def near(got, want, room, what):       # close(), where the tensors are
        half = 2.0 ** -8 if got.dtype == BF else 0.0
        bad = ~((got.double() - want).abs() <= room + half * (want.abs() + room) + 2.0 ** -134)
        assert got.shape == want.shape and not bool(bad.any()), (what, int(bad.sum()))

    want = swiglu64(gate, up)
    near(pcm.pcm_swiglu(gu, out_dtype=out), want, swiglu_room(gate, up, want), "u")
    near(pcm.pcm_swiglu_grad(gu, du, out_dtype=out), swiglu_grads64(gate, up, d), swiglu_grad_room(gate, up, d), "dgate_up")


# ------------------------------------------------------------------------ mix along the paths
def path_case(T, k, n, F, dtype, density, seed=0):
    c = routed(T, k, n, seed)
    g = torch.Generator().manual_seed(seed + 7)
    mask = torch.rand((n, n), generator=g) < density
    if density >= 0:
        mask.fill_diagonal_(True)
    on = mask[c["ids"].long()[:, :, None], c["ids"].long()[:, None, :]]
    c["on"] = on
    c["bits"] = (on.reshape(T, -1).long() << torch.arange(k * k)).sum(1)
    c["beta"] = torch.rand((T, k, k), generator=g)      # read only where there is a path
    c["u"], c["dz"] = torch.randn((T * k, F), generator=g).to(dtype), torch.randn((T * k, F), generator=g).to(dtype)
    c["src"] = c["tgt"] = c["of"]
    return c


def check_mix(c, out, has_src=None, has_tgt=None):
    """has_src, has_tgt [T, k]: which pairs have a row; numbers that are none elsewhere."""
    T, k = c["of"].shape
    F = c["u"].shape[1]
    has_src = torch.ones((T, k), dtype=torch.bool) if has_src is None else has_src
    has_tgt = torch.ones((T, k), dtype=torch.bool) if has_tgt is None else has_tgt
    on = c["on"] & has_src[:, :, None] & has_tgt[:, None, :]
    w = torch.where(on, c["beta"].double(), 0.0)
    src, tgt = c["src"].long(), c["tgt"].long()
    u = torch.where(has_src[:, :, None], c["u"].double()[src.clamp(0, T * k - 1)], 0.0)
    dz = torch.where(has_tgt[:, :, None], c["dz"].double()[tgt.clamp(0, T * k - 1)], 0.0)
    beta = torch.where(on, c["beta"], float("nan"))
    args = gpu(c["bits"]), gpu(beta), gpu(c["src"]), gpu(c["tgt"])
    z = pcm.pcm_mix_rows(gpu(c["u"]), *args, z=torch.full((T * k, F), 7.0, dtype=out, device=DEV))
    close(z[gpu(tgt[has_tgt])], torch.matmul(w.mT, u)[has_tgt], (k + 1) * U * torch.matmul(w.mT, u.abs())[has_tgt], "z")
    assert int((z == 7.0).all(1).sum()) == int((~has_tgt).sum())
    du, dbeta = pcm.pcm_mix_rows_grad(gpu(c["dz"]), gpu(c["u"]), *args, du=torch.full((T * k, F), 7.0, dtype=out, device=DEV))
    close(du[gpu(src[has_src])], torch.matmul(w, dz)[has_src], (k + 1) * U * torch.matmul(w, dz.abs())[has_src], "du")
    assert int((du == 7.0).all(1).sum()) == int((~has_src).sum())
    close(dbeta, torch.where(on, torch.matmul(u, dz.mT), 0.0), (F + 1) * U * torch.matmul(u.abs(), dz.abs().mT), "dbeta")
    assert bool((dbeta[gpu(~on)] == 0).all())
    alone, nothing = pcm.pcm_mix_rows_grad(gpu(c["dz"]), None, *args, rows=T * k, out_dtype=out)
    assert nothing is None
    same_bits(alone[gpu(src[has_src])], du[gpu(src[has_src])])


@pytest.mark.parametrize("types", TYPES)
@pytest.mark.parametrize("density", [0.0, 0.3, 1.0])
@pytest.mark.parametrize("T,k,n,F", [(1, 1, 1, 16), (1, 8, 256, 2048), (9, 2, 3, 4112), (40, 3, 5, 80), (65, 4, 12, 272),
                                     (6, 5, 9, 1040), (30, 6, 7, 144), (17, 7, 20, 528), (130, 8, 16, 1024), (2, 2, 8, 14336)])
def test_mix(T, k, n, F, density, types):
    dt, out = TYPES[types]
    check_mix(path_case(T, k, n, F, dt, density), out)


@pytest.mark.parametrize("types", ["bf16-bf16", "f32-f32"])
@pytest.mark.parametrize("k", [2, 3, 8])
def test_mix_without_some_rows_and_paths(k, types):
    """Targets and sources without any path (zeros), pairs without a row, sources and targets in other orders; what no path
    reads is NaN."""
    dt, out = TYPES[types]
    T, n, F = 24, 10, 336
    c = path_case(T, k, n, F, dt, -1.0 if k == 2 else 0.2, 3)
    if k == 2:
        assert not bool(c["on"].any())
    g = torch.Generator().manual_seed(5)
    c["tgt"] = torch.randperm(T * k, generator=g).reshape(T, k).int()
    has_src, has_tgt = torch.rand((T, k), generator=g) < 0.8, torch.rand((T, k), generator=g) < 0.8
    c["u"][c["src"].long()[~has_src]] = float("nan")
    c["dz"][c["tgt"].long()[~has_tgt]] = float("nan")
    read = (c["on"] & has_src[:, :, None] & has_tgt[:, None, :])
    lone_src, lone_tgt = has_src & ~read.any(2), has_tgt & ~read.any(1)
    assert bool(lone_src.any()) and bool(lone_tgt.any())
    c["src"], c["tgt"] = c["src"].clone(), c["tgt"].clone()
    c["src"][~has_src] = torch.tensor([-1, T * k, -(1 << 31)], dtype=torch.int32).repeat(T * k)[:int((~has_src).sum())]
    c["tgt"][~has_tgt] = torch.tensor([T * k, -1, 1 << 30], dtype=torch.int32).repeat(T * k)[:int((~has_tgt).sum())]
    check_mix(c, out, has_src, has_tgt)
    # a source that no path reads may hold anything
    u = c["u"].clone()
    u[c["src"].long()[lone_src]] = float("nan")
    beta = torch.where(read, c["beta"], float("nan"))
    z = pcm.pcm_mix_rows(gpu(u), gpu(c["bits"]), gpu(beta), gpu(c["src"]), gpu(c["tgt"]))
    assert bool(torch.isfinite(z[gpu(c["tgt"].long()[has_tgt])]).all())
    dz = c["dz"].clone()
    dz[c["tgt"].long()[lone_tgt]] = float("inf")
    du, dbeta = pcm.pcm_mix_rows_grad(gpu(dz), gpu(u), gpu(c["bits"]), gpu(beta), gpu(c["src"]), gpu(c["tgt"]))
    assert bool(torch.isfinite(du[gpu(c["src"].long()[has_src])]).all()) and bool(torch.isfinite(dbeta).all())


@pytest.mark.parametrize("K", [3, 8])
def test_mix_on_scored_tables(K):
    """The scored router's tables: fewer sources than slots, -1 behind them."""
    T, n, F = 50, 12, 208
    g = torch.Generator().manual_seed(9)
    layout = pcm.pcm_path_layout_build(gpu((torch.rand((n, n), generator=g) < 0.5).to(torch.uint8)), gpu(torch.randn((n, n), generator=g)))
    t = pcm.pcm_route_scored(gpu(torch.randn((T, n), generator=g)), gpu(torch.randn((T, n), generator=g)), 0.5, layout, K)
    c = dict(of=t.src_row_of.cpu(), src=t.src_row_of.cpu(), tgt=t.tgt_row_of.cpu(), bits=t.path_bits.cpu(), beta=t.beta.cpu())
    c["on"] = ((c["bits"][:, None] >> torch.arange(K * K)) & 1).bool().reshape(T, K, K)
    c["u"], c["dz"] = torch.randn((T * K, F), generator=g).to(BF), torch.randn((T * K, F), generator=g).to(BF)
    assert bool((c["src"] < 0).any()) and bool((c["tgt"] < 0).any())
    check_mix(c, F32, c["src"] >= 0, c["tgt"] >= 0)


@pytest.mark.parametrize("types", TYPES)
@pytest.mark.parametrize("k,F", [(1, 2064), (2, 208), (3, 528), (4, 2064), (5, 272), (6, 80), (7, 1040), (8, 2064)])
def test_mix_of_large_buffers(k, F, types):
    """From 96 MB read on the mixes load non-temporally; the gradient of more than four slots one of its operands."""
    dt, out = TYPES[types]
    T = 29
    c = path_case(T, k, 11, F, dt, 0.4, seed=k)
    R, src = rows_in_a_large_buffer(T, k, F, dt, k)
    tgt = rows_in_a_large_buffer(T, k, F, dt, k + 50)[1]
    u, dz = c["u"].reshape(T, k, F), c["dz"].reshape(T, k, F)
    beta = torch.where(c["on"], c["beta"], float("nan"))
    B, U64, D64 = torch.where(c["on"], c["beta"].double(), 0.0), u.double(), dz.double()
    args = gpu(c["bits"]), gpu(beta), gpu(src), gpu(tgt)
    ub, db = in_a_large_buffer(R, src, u), in_a_large_buffer(R, tgt, dz)
    z = pcm.pcm_mix_rows(ub, *args, z=torch.full((R, F), 7.0, dtype=out, device=DEV))
    close(z[gpu(tgt.long())], torch.matmul(B.mT, U64), (k + 1) * U * torch.matmul(B.mT, U64.abs()), "z")
    z[gpu(tgt.reshape(-1).long())] = 7.0
    assert bool((z == 7.0).all())
    du, dbeta = pcm.pcm_mix_rows_grad(db, ub, *args, du=torch.full((R, F), 7.0, dtype=out, device=DEV))
    room = (k + 1) * U * torch.matmul(B, D64.abs())
    close(du[gpu(src.long())], torch.matmul(B, D64), room, "du")
    close(dbeta, torch.where(c["on"], torch.matmul(U64, D64.mT), 0.0), (F + 1) * U * torch.matmul(U64.abs(), D64.abs().mT), "dbeta")
    alone, nothing = pcm.pcm_mix_rows_grad(db, None, *args, rows=R, du=torch.full((R, F), 7.0, dtype=out, device=DEV))
    assert nothing is None
    close(alone[gpu(src.long())], torch.matmul(B, D64), room, "du alone")
    for d in (du, alone):
        d[gpu(src.reshape(-1).long())] = 7.0
        assert bool((d == 7.0).all())


@pytest.mark.parametrize("types", ["bf16-f32", "f32-f32"])
def test_mix_gradients_against_differences(types):
    """As for the rows: integers and quarters, exact sums."""
    dt, _ = TYPES[types]
    T, k, n, F = 15, 4, 6, 96
    c = path_case(T, k, n, F, dt, 0.4, 2)
    g = torch.Generator().manual_seed(8)
    ints = lambda m: torch.randint(-m, m + 1, (T * k, F), generator=g).to(dt)
    u, vu, dz = ints(3), ints(2), ints(3)
    beta, vb = (torch.randint(-4, 5, (T, k, k), generator=g) / 4 * c["on"] for _ in range(2))
    f = lambda u, beta: pcm.pcm_mix_rows(gpu(u), gpu(c["bits"]), gpu(beta), gpu(c["of"]), out_dtype=F32).cpu().double()
    du, dbeta = (t.cpu().double() for t in pcm.pcm_mix_rows_grad(gpu(dz), gpu(u), gpu(c["bits"]), gpu(beta), gpu(c["of"]), out_dtype=F32))
    dot = lambda a, b: float((a.double() * b.double()).sum())
    assert dot(dz, f(u + vu, beta) - f(u - vu, beta)) == 2 * dot(du, vu)
    assert dot(dz, f(u, beta + vb) - f(u, beta - vb)) == 2 * dot(dbeta, vb)


# ------------------------------------------------------------------------ the router
def betas64(p, on, mode):
    """beta [T, k, k] of 64-bit weights p, differentiable."""
    pair = torch.where(on, p[:, :, None] * p[:, None, :], 0.0)
    if mode == 0:
        return pair / torch.where(on, p[:, None, :], 0.0).sum(2, keepdim=True)
    return pair if mode == 1 else pair / pair.sum((1, 2), keepdim=True)


def route_grad64(ids, p, n, on, dbeta, dw, mode):
    """By autograd in 64 bits at the weights p (which are rounded: the softmax' derivative p_a (delta_ac - p_c) at them)."""
    q = p.double().requires_grad_()
    loss = torch.zeros((), dtype=torch.float64)
    if dbeta is not None:
        loss = loss + (betas64(q, on, mode) * torch.where(on, dbeta.double(), 0.0)).sum()
    if dw is not None:
        loss = loss + (q * dw.double()).sum()
    dp, = torch.autograd.grad(loss, q)
    q = q.detach()
    dl = q * (dp - (q * dp).sum(1, keepdim=True))
    return torch.zeros((p.shape[0], n), dtype=torch.float64).scatter_(1, ids.long(), dl), dp


@pytest.mark.parametrize("out", ["f32", "bf16"])
@pytest.mark.parametrize("given", ["paths", "weights", "both"])
@pytest.mark.parametrize("mode", [0, 1, 2])
@pytest.mark.parametrize("T,k,n", [(1, 1, 1), (1, 8, 256), (31, 2, 8), (33, 4, 60), (200, 8, 64), (65, 3, 5), (64, 7, 255), (40, 1, 9)])
def test_router_gradient(T, k, n, mode, given, out):
    """64-bit arithmetic on the same float32 inputs (both sides within 2^-40 of the largest term), rounded to float32."""
    c = path_case(T, k, n, 16, F32, 0.4, k)
    g = torch.Generator().manual_seed(T)
    dbeta = torch.where(c["on"], torch.randn((T, k, k), generator=g), float("nan")) if given != "weights" else None
    dw = torch.randn((T, k), generator=g) if given != "paths" else None
    got = pcm.pcm_route_grad(gpu(c["ids"]), gpu(c["p"]), n, gpu(c["bits"]) if dbeta is not None else None, gpu(dbeta), gpu(dw), mode,
                             out_dtype={"f32": F32, "bf16": BF}[out])
    want, dp = route_grad64(c["ids"], c["p"], n, c["on"], dbeta, dw, mode)
    close(got, want, U * want.abs() + 2.0 ** -40 * (1 + dp.abs().amax(1, keepdim=True)), "dlogits")
    chosen = torch.zeros((T, n), dtype=torch.bool).scatter_(1, c["ids"].long(), True)
    assert bool((got.cpu()[~chosen] == 0).all())


@pytest.mark.parametrize("mode", [0, 1, 2])
def test_router_gradient_of_weights_that_vanish(mode):
    """Logits so far apart that the smaller weights are 0 in float32: their gradients are 0, the others' what they are."""
    ids = torch.tensor([[2, 0, 3], [1, 3, 0]], dtype=torch.int32)
    p = torch.tensor([[1.0, 0.0, 0.0], [0.75, 0.25, 0.0]])
    on = torch.eye(3).bool().repeat(2, 1, 1)
    on[:, 0, 2] = True
    on[:, 2, 1] = True
    bits = (on.reshape(2, 9).long() << torch.arange(9)).sum(1)
    dbeta = torch.randn((2, 3, 3), generator=torch.Generator().manual_seed(1))
    got = pcm.pcm_route_grad(gpu(ids), gpu(p), 5, gpu(bits), gpu(dbeta), beta_mode=mode).cpu()
    assert bool(torch.isfinite(got).all()) and bool((got[0] == 0).all()) and got[1, 0] == 0
    tiny = p.clone()
    tiny[tiny == 0] = 2.0 ** -60       # in the limit
    want, _ = route_grad64(ids, tiny, 5, on, dbeta, None, mode)
    assert bool(((got[1].double() - want[1]).abs() <= U * want[1].abs() + 2.0 ** -50).all())


@pytest.mark.parametrize("mode", [0, 1, 2])
def test_router_gradient_against_differences(mode):
    """By differences of the router's own path weights. Steps of 2^-7 in the logits: h^2 / 6 of the third derivative (below 8
    for products of up to three softmax factors) and the weights' roundings, 8u each of at most 1, over 2h, times |dbeta|."""
    T, n, k = 12, 6, 3
    g = torch.Generator().manual_seed(4)
    logits = torch.randn((T, n), generator=g) + torch.arange(n) * 0.5        # no ties nearby: the selection stays
    logits = (logits * 64).round() / 64
    packed = pcm.pcm_mask_pack(gpu((torch.rand((n, n), generator=g) < 0.5).to(torch.uint8)))
    route = lambda l: pcm.pcm_route_paths(gpu(l), packed, k, mode)
    ids, p, t = route(logits)
    dbeta = torch.randn((T, k, k), generator=g).to(DEV)
    got = pcm.pcm_route_grad(ids, p, n, t.path_bits, dbeta, beta_mode=mode).cpu().double()
    h, D = 2.0 ** -7, dbeta.cpu().double()
    checked = 0
    for e in range(n):
        step = torch.zeros((T, n))
        step[:, e] = h
        (i0, _, t0), (i1, _, t1) = route(logits - step), route(logits + step)
        ok = ((i0 == ids) & (i1 == ids)).all(1).cpu()
        diff = ((t1.beta.cpu().double() - t0.beta.cpu().double()) * D).sum((1, 2)) / (2 * h)
        room = D.abs().sum((1, 2)) * (8 * h * h / 6 + 8 * U / h)
        assert bool(((got[:, e] - diff).abs() <= room)[ok].all()), e
        checked += int(ok.sum())
    assert checked > T * n // 2


# ------------------------------------------------------------------------ all gradients
def norm64(grads):
    return math.sqrt(sum(float(g.double().square().sum()) for g in grads))


def check_clip(grads, max_norm, out_types=None, places=None):
    """Norm and clipped values by both ways; the norm in 64 bits is off by N 2^-53 and rounded once."""
    N = sum(g.numel() for g in grads)
    want = norm64(grads)
    here = [gpu(g) for g in grads] if places is None else places
    norm = pcm.pcm_grad_norm(here)
    assert norm.dtype == F32 and norm.shape == (1,)
    over = want >= 2.0 ** 128 * (1 - 2.0 ** -25)      # rounds to infinity, which leaves the values as they are
    assert float(norm) == math.inf if over else \
        abs(float(norm) - want) <= (U + (N + 8) * 2.0 ** -53) * want + 2.0 ** -150, (float(norm), want)
    factor = max_norm / want if want > max_norm and not over else 1.0
    out_types = out_types or [g.dtype for g in grads]
    out = [torch.full(g.shape, 7.0, dtype=t, device=DEV) for g, t in zip(grads, out_types)]
    again = pcm.pcm_clip_grad_norm(here, max_norm, out=out)
    same_bits(again, norm)
    for g, o in zip(grads, out):
        # the norm's rounding, the factor's, the product's
        close(o, g.double() * factor, (4 * U + N * 2.0 ** -53) * g.double().abs() * factor, "out")
    two = [torch.empty_like(o) for o in out]
    pcm.pcm_clip_grads(here, norm, max_norm, out=two)
    for a, b in zip(out, two):
        same_bits(a, b)
    for g, h in zip(grads, here):
        same_bits(h, g)                       # read only, so far
    return here, out, norm


SIZES = [[1], [0], [3, 0, 1], [7, 4096, 4095, 4097], [16, 100_000, 31, 8191, 8192, 8193, 1], [5] * 300, [50_000, 17] * 97]


@pytest.mark.parametrize("types", ["bf16", "f32", "mixed"])
@pytest.mark.parametrize("sizes", SIZES, ids=str)
def test_norm_and_clip(sizes, types):
    g = torch.Generator().manual_seed(len(sizes))
    kinds = {"bf16": [BF], "f32": [F32], "mixed": [F32, BF, BF]}[types]
    grads = [torch.randn(n, generator=g).to(kinds[i % len(kinds)]) for i, n in enumerate(sizes)]
    norm = norm64(grads)
    for max_norm in (norm / 3, norm * 2, 0.0):
        here, out, _ = check_clip(grads, max_norm)
        if max_norm == 0.0:
            assert not any(bool(o.any()) for o in out)
        pcm.pcm_clip_grad_norm(here, max_norm)        # in place: the same
        for h, o in zip(here, out):
            same_bits(h, o)


@pytest.mark.parametrize("shift", [0, 1, 2, 3, 5, 7])
def test_clip_of_views(shift):
    """Views of flat buffers at any element, into others at other offsets and of the other type; what lies around them stays."""
    g = torch.Generator().manual_seed(shift)
    sizes = [1, 40, 9000, 3, 17, 4096, 0, 12_345]
    flat = {t: gpu(torch.randn(30_000, generator=g).to(t)) for t in (BF, F32)}
    kept = {t: f.clone() for t, f in flat.items()}
    to = {t: torch.full((60_000,), 7.0, dtype=t, device=DEV) for t in (BF, F32)}
    grads, outs, at = [], [], shift
    for i, n in enumerate(sizes):
        t = (BF, F32)[i % 2]
        grads.append(flat[t][at:at + n])
        outs.append(to[(F32, BF, BF, F32)[i % 4]][at + 3 * i:at + 3 * i + n])
        at += n
    host = [v.cpu() for v in grads]
    norm = pcm.pcm_clip_grad_norm(grads, 1.0, out=outs)
    want = norm64(host)
    assert abs(float(norm) - want) <= 2 * U * want
    for h, o in zip(host, outs):
        close(o, h.double() / want, 4 * U * h.double().abs() / want, "out")
    for t in flat:
        same_bits(flat[t], kept[t])
        written = sum(o.numel() for o in outs if o.dtype == t)
        assert int((to[t] != 7.0).sum()) <= written and bool((to[t][:shift] == 7.0).all()) and bool((to[t][-20_000:] == 7.0).all())
    pcm.pcm_clip_grad_norm(grads, 1.0)                # in place, in the middle of the buffers
    for t in flat:
        inside = torch.zeros(30_000, dtype=torch.bool)
        for v in grads:
            if v.dtype == t:
                inside[v.storage_offset():v.storage_offset() + v.numel()] = True
        same_bits(flat[t].cpu()[~inside], kept[t].cpu()[~inside])
    for h, v in zip(host, grads):
        close(v, h.double() / want, 4 * U * h.double().abs() / want, "in place")


@pytest.mark.parametrize("scale", [1e-30, 1e-42, 1e25, 1e37])
def test_norm_of_small_and_large_values(scale):
    """Squares that float32 does not hold."""
    g = torch.Generator().manual_seed(1)
    grads = [torch.rand(5000, generator=g) * scale, (torch.rand(300, generator=g) * scale).to(BF)]
    check_clip(grads, float(torch.tensor(norm64(grads) / 2, dtype=F32)))


@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf")])
def test_norm_that_is_not_finite(value):
    """Says so, and the gradients stay as they are."""
    g = torch.Generator().manual_seed(1)
    grads = [torch.randn(5000, generator=g), torch.randn(300, generator=g).to(BF)]
    grads[1][7] = value
    here = [gpu(t) for t in grads]
    norm = pcm.pcm_clip_grad_norm(here, 1.0)
    assert not bool(torch.isfinite(norm).any()) and bool(norm.isnan().any()) == math.isnan(value)
    out = [torch.empty_like(h) for h in here]
    pcm.pcm_clip_grads(here, norm, 1.0, out=out)
    for a, h, o in zip(grads, here, out):
        same_bits(h, a)
        same_bits(o, a)


def test_clip_by_a_norm_of_several_ranks():
    grads = [gpu(torch.randn(1000, generator=torch.Generator().manual_seed(1)))]
    norm = torch.tensor(8.0, device=DEV)
    want = grads[0] * 0.25
    assert pcm.pcm_clip_grads(grads, norm, 2.0) is grads
    assert torch.equal(grads[0], want)
    assert pcm.pcm_clip_grads(grads, norm, float("inf")) is grads and torch.equal(grads[0], want)


def test_clip_of_what_can_be_read_once():
    """Gradients and results from generators come back as lists that hold them; a list comes back itself."""
    norm = torch.tensor(8.0, device=DEV)
    grads = [torch.full((n,), 4.0, device=DEV) for n in (5, 300)]
    outs = [torch.zeros_like(g) for g in grads]
    back = list(pcm.pcm_clip_grads((g for g in grads), norm, 2.0, out=(o for o in outs)))
    assert len(back) == 2 and all(b is o for b, o in zip(back, outs)) and all(bool((o == 1.0).all()) for o in outs)
    back = list(pcm.pcm_clip_grads(iter(grads), norm, 2.0))
    assert len(back) == 2 and all(b is g for b, g in zip(back, grads)) and all(bool((g == 1.0).all()) for g in grads)
    assert pcm.pcm_clip_grads(grads, norm, 100.0, out=outs) is outs


@pytest.mark.parametrize("count", [512, 513, 1024, 1025, 4096])
def test_clip_of_many_tensors(count):
    """Up to the most a call takes, in place and into others, in an order that is not that of their addresses."""
    g = torch.Generator().manual_seed(count)
    flat = torch.randn(count * 5, generator=g)
    order = torch.randperm(count, generator=g).tolist()
    here, there = gpu(flat), torch.full((count * 5,), 7.0, dtype=BF, device=DEV)
    grads, outs = [here[5 * i:5 * i + 1 + i % 5] for i in order], [there[5 * i:5 * i + 1 + i % 5] for i in order]
    host = [v.cpu() for v in grads]
    want = norm64(host)
    norm = pcm.pcm_clip_grad_norm(grads, 1.0, out=outs)
    assert abs(float(norm) - want) <= 2 * U * want
    written = torch.zeros(count * 5, dtype=torch.bool)
    for i in order:
        written[5 * i:5 * i + 1 + i % 5] = True
    value = flat.double() / want
    close(there[gpu(written)], value[written], 4 * U * value[written].abs(), "out")
    assert bool((there[gpu(~written)] == 7.0).all())
    pcm.pcm_clip_grads(grads, norm, 1.0)
    close(here[gpu(written)], value[written], 4 * U * value[written].abs(), "in place")
    same_bits(here[gpu(~written)], flat[~written])


def test_norm_beside_the_gradients():
    """The norm next to a gradient in one buffer; one of the gradients where only results are written; never on a written one."""
    flat = torch.full((100,), 2.0, device=DEV)
    grads, norm = [flat[1:60], flat[61:]], flat[60:61]
    assert pcm.pcm_clip_grad_norm(grads, 1.0, norm=norm) is norm
    want = 2.0 * math.sqrt(98)
    assert abs(float(norm) - want) <= 2 * U * want and float(flat[0]) == 2.0
    close(torch.cat(grads), torch.full((98,), 2.0 / want, dtype=torch.float64), 4 * U * torch.full((98,), 2.0 / want, dtype=torch.float64))
    flat.fill_(2.0)
    out = pcm.pcm_clip_grads([flat[:50]], flat[:1], 1.0, out=[torch.zeros(50, device=DEV)])
    assert bool((out[0] == 1.0).all())
    for call in (lambda: pcm.pcm_clip_grads([flat[:50]], flat[49:50], 1.0), lambda: pcm.pcm_grad_norm([flat[:50]], norm=flat[7:8]),
                 lambda: pcm.pcm_clip_grad_norm([flat[:50]], 1.0, norm=flat[:1])):
        with pytest.raises(RuntimeError):
            call()
    assert bool((flat == 2.0).all())


def test_norm_of_nothing():
    assert float(pcm.pcm_grad_norm([])) == 0.0
    assert float(pcm.pcm_clip_grad_norm([], 1.0)) == 0.0
    assert pcm.pcm_clip_grads([], torch.ones(1, device=DEV), 1.0) == []


def test_norm_past_32_bits():
    """More than 2^32 elements."""
    big = torch.zeros((1 << 32) + 5000, dtype=BF, device=DEV)
    big[-3:] = 2.0
    big[0] = 1.0
    assert float(pcm.pcm_grad_norm([big])) == float(torch.tensor(13.0).sqrt())
    pcm.pcm_clip_grad_norm([big], float(torch.tensor(13.0).sqrt()) / 2)
    assert big[-3:].tolist() == [1.0] * 3 and float(big[0]) == 0.5 and int((big != 0).sum()) == 4


def test_clip_refuses():
    a = torch.zeros(64, device=DEV)
    for call in (lambda: pcm.pcm_clip_grad_norm([a.reshape(8, 8).t()], 1.0), lambda: pcm.pcm_clip_grad_norm([a], 1.0, out=[a[:32]]),
                 lambda: pcm.pcm_clip_grad_norm([a], 1.0, out=[]), lambda: pcm.pcm_clip_grad_norm([a], 1.0, norm=a),
                 lambda: pcm.pcm_grad_norm([a, a.cpu()])):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(TypeError):
        pcm.pcm_grad_norm([a.half()])
    for call in (lambda: pcm.pcm_clip_grad_norm([a, a], 1.0), lambda: pcm.pcm_clip_grad_norm([a[:40], a[39:]], 1.0),
                 lambda: pcm.pcm_clip_grad_norm([a], -1.0), lambda: pcm.pcm_clip_grads([a[:32]], a[:1], 1.0, out=[a[16:48]]),
                 lambda: pcm.pcm_grad_norm([a], ws=torch.zeros(256, dtype=torch.uint8, device=DEV))):
        with pytest.raises(RuntimeError):
            call()


# ------------------------------------------------------------------------ as programs call them
def all_calls(c, stream=None):
    """Every entry point once, on tensors of the case; results by name."""
    r = {}
    r["y"] = pcm.pcm_dispatch_rows(c["x"], c["of"], c["w"], stream=stream)
    r["dx"], r["dwx"] = pcm.pcm_dispatch_rows_grad(c["o"], c["of"], c["x"], c["w"], stream=stream)
    r["back"] = pcm.pcm_combine_rows(c["o"], c["of"], c["w"], stream=stream)
    r["do"], r["dwo"] = pcm.pcm_combine_rows_grad(c["x"], c["of"], c["o"], c["w"], stream=stream)
    r["u"] = pcm.pcm_swiglu(c["o"], stream=stream)
    r["dgu"] = pcm.pcm_swiglu_grad(c["o"], r["u"], stream=stream)
    r["z"] = pcm.pcm_mix_rows(r["u"], c["bits"], c["beta"], c["of"], stream=stream)
    r["du"], r["dbeta"] = pcm.pcm_mix_rows_grad(r["z"], r["u"], c["bits"], c["beta"], c["of"], stream=stream)
    r["dl"] = pcm.pcm_route_grad(c["ids"], c["p"], c["n"], c["bits"], r["dbeta"], r["dwo"], stream=stream)
    grads = [r["du"], r["dl"], r["dx"]]
    r["norm"] = pcm.pcm_grad_norm(grads, stream=stream)
    for i, v in enumerate(grads):
        r[f"out{i}"] = torch.empty_like(v)
    outs = [r[f"out{i}"] for i in range(3)]
    r["again"] = pcm.pcm_clip_grad_norm(grads, 1.0, out=outs, stream=stream)
    pcm.pcm_clip_grads(outs, r["again"], 0.5, stream=stream)
    return r


def calls_case(seed=0):
    T, k, n, H = 150, 4, 16, 544
    c = path_case(T, k, n, H, BF, 0.4, seed)
    d = tokens_and_rows((T, k, n, H), BF, "all", seed)
    return {name: v.to(DEV) if isinstance(v, torch.Tensor) else v for name, v in
            dict(x=d["x"], o=d["o"], w=d["w"], of=c["of"], bits=c["bits"], beta=c["beta"], ids=c["ids"], p=c["p"], n=n).items()}


def same(a, b):
    for name in a:
        same_bits(a[name], b[name])


def test_another_stream():
    c = calls_case()
    want = all_calls(c)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        got = all_calls(c, stream=s)
    s.synchronize()
    same(got, want)


def test_two_streams_at_once():
    """Workspaces of their own: calls that overlap give what each gives alone."""
    cases = [calls_case(1), calls_case(2)]
    want = [all_calls(c) for c in cases]
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in cases], [[] for _ in cases]
    for _ in range(5):
        for i, (c, s) in enumerate(zip(cases, streams)):
            with torch.cuda.stream(s):
                got[i].append(all_calls(c, stream=s))
    torch.cuda.synchronize()
    for w, results in zip(want, got):
        for r in results:
            same(r, w)


def test_deterministic():
    c = calls_case()
    a = all_calls(c)
    for _ in range(3):
        same(all_calls(c), a)


def test_graph_replays():
    """Captured once, replayed on new inputs with other work between the replays."""
    c = calls_case()
    all_calls(c)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        got = all_calls(c)
    for seed in range(1, 5):
        for name, v in calls_case(seed).items():
            if isinstance(v, torch.Tensor):
                c[name].copy_(v)
        want = all_calls(c)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        same(got, want)


def test_refuses_tensors_the_kernels_must_not_address():
    c = calls_case()
    x, of, w, o, bits, beta = (c[v] for v in ("x", "of", "w", "o", "bits", "beta"))
    for call in (lambda: pcm.pcm_dispatch_rows(x.t(), of), lambda: pcm.pcm_dispatch_rows(x, of[:-1]),
                 lambda: pcm.pcm_dispatch_rows(x, of.cpu()), lambda: pcm.pcm_dispatch_rows(x, of, w[:, :2].contiguous()),
                 lambda: pcm.pcm_dispatch_rows(x, of, rows=5, y=o), lambda: pcm.pcm_dispatch_rows(x, of, offsets=of),
                 lambda: pcm.pcm_dispatch_rows_grad(o, of, x[1:]), lambda: pcm.pcm_dispatch_rows_grad(o, of, dweights=w),
                 lambda: pcm.pcm_combine_rows(o, of, y=x[1:]), lambda: pcm.pcm_combine_rows(o, of, accumulate=True),
                 lambda: pcm.pcm_combine_rows_grad(x, of, o, rows=3), lambda: pcm.pcm_combine_rows_grad(x, of, do=o[:, :16]),
                 lambda: pcm.pcm_swiglu(o, u=o), lambda: pcm.pcm_swiglu_grad(o, o),
                 lambda: pcm.pcm_mix_rows(o, bits[1:], beta, of), lambda: pcm.pcm_mix_rows(o, bits, beta[:, 0], of),
                 lambda: pcm.pcm_mix_rows(o, bits, beta, of, of[:-1]), lambda: pcm.pcm_mix_rows_grad(o, o[1:], bits, beta, of, du=o),
                 lambda: pcm.pcm_mix_rows_grad(o, None, bits, beta, of, dbeta=beta),
                 lambda: pcm.pcm_route_grad(c["ids"], w, 16, bits, dw=w), lambda: pcm.pcm_route_grad(c["ids"], w[1:], 16, dw=w)):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: pcm.pcm_dispatch_rows(x, of.long()), lambda: pcm.pcm_dispatch_rows(x, of, w.double()),
                 lambda: pcm.pcm_dispatch_rows(x.half(), of), lambda: pcm.pcm_dispatch_rows_grad(o, of, x.half()),
                 lambda: pcm.pcm_combine_rows(o, of, out_dtype=torch.float16), lambda: pcm.pcm_swiglu_grad(o, o[:, :272].float()),
                 lambda: pcm.pcm_mix_rows(o, bits.int(), beta, of), lambda: pcm.pcm_mix_rows_grad(o, o.float(), bits, beta, of),
                 lambda: pcm.pcm_route_grad(c["ids"], w.bfloat16(), 16, dw=w)):
        with pytest.raises((TypeError, ValueError)):
            call()
    for call in (lambda: pcm.pcm_dispatch_rows(torch.zeros((4, 24), device=DEV), of[:4]),
                 lambda: pcm.pcm_combine_rows(o, of, y=x.clone(), accumulate=True),
                 lambda: pcm.pcm_route_grad(c["ids"], c["p"], 3, dw=w), lambda: pcm.pcm_route_grad(c["ids"], c["p"], 300, dw=w)):
        with pytest.raises(RuntimeError):
            call()


@pytest.mark.parametrize("mode", [0, 1, 2])
def test_training_step_of_a_path_layer(mode):
    """A whole step of a path-compositional layer through the framework's calls: router, expansion products, SwiGLU, mix,
    projection products and combine; every gradient back to the hidden states, the experts' and the router's weights; their
    norm and clipping. Against autograd in 64 bits on the same selection. Each float32 sum is off by its bound; through the
    chain the relative errors add, so that a bound of 64 times the longest sum's relative one on the norms holds with room
    (the products' own test's)."""
    T, H, F, n, k = 45, 160, 96, 16, 3
    g = torch.Generator().manual_seed(6)
    x, dy = torch.randn((T, H), generator=g), torch.randn((T, H), generator=g)
    w1, w2 = torch.randn((n, 2 * F, H), generator=g) * 0.08, torch.randn((n, H, F), generator=g) * 0.08
    wr = torch.randn((n, H), generator=g) * 0.1
    mask = (torch.rand((n, n), generator=g) < 0.4).to(torch.uint8)
    X, D, W1, W2, WR = (gpu(t) for t in (x, dy, w1, w2, wr))
    # forward
    logits = pcm.pcm_grouped_gemm(X, WR)
    ids, p, t = pcm.pcm_route_paths(logits, pcm.pcm_mask_pack(gpu(mask)), k, mode)
    off, tok, of = t.expert_offsets, t.row_token, t.row_of
    gu = pcm.pcm_grouped_gemm(X, W1, off, tok)
    u = pcm.pcm_swiglu(gu)
    z = pcm.pcm_mix_rows(u, t.path_bits, t.beta, of)
    o = pcm.pcm_grouped_gemm(z, W2, off)
    y = pcm.pcm_combine_rows(o, of)
    # backward
    do, _ = pcm.pcm_combine_rows_grad(D, of)
    dz, dW2 = pcm.pcm_grouped_gemm_dx(do, W2, off), pcm.pcm_grouped_gemm_dw(z, do, off)
    du, dbeta = pcm.pcm_mix_rows_grad(dz, u, t.path_bits, t.beta, of)
    dgu = pcm.pcm_swiglu_grad(gu, du)
    dW1 = pcm.pcm_grouped_gemm_dw(X, dgu, off, tok)
    dlogits = pcm.pcm_route_grad(ids, p, n, t.path_bits, dbeta, beta_mode=mode)
    dWR = pcm.pcm_grouped_gemm_dw(X, dlogits)
    dX = pcm.pcm_grouped_gemm_dx(dgu, W1, off, of) + pcm.pcm_grouped_gemm_dx(dlogits, WR)
    grads = [dW1, dW2, dWR]
    before = [v.cpu() for v in grads]
    norm = pcm.pcm_clip_grad_norm(grads, 1.0)
    # 64 bits
    x64, a64, b64, r64 = (v.double().requires_grad_() for v in (x, w1, w2, wr))
    sel = ids.cpu().long()
    l64 = torch.matmul(x64, r64.T)
    p64 = l64.gather(1, sel).softmax(1)
    on = (mask.bool() | torch.eye(n).bool())[sel[:, :, None], sel[:, None, :]]
    beta = betas64(p64, on, mode)
    v = (a64[sel] @ x64[:, None, :, None])[..., 0]
    zz = torch.matmul(beta.mT, torch.nn.functional.silu(v[..., :F]) * v[..., F:])
    y64 = (b64[sel] @ zz[..., None])[..., 0].sum(1)
    y64.backward(dy.double())
    for name, got, want in (("y", y, y64.detach()), ("dX", dX, x64.grad), ("dW1", before[0], a64.grad), ("dW2", before[1], b64.grad),
                            ("dWR", before[2], r64.grad)):
        rel = float((got.cpu().double() - want).norm() / want.norm())
        assert rel <= 64 * (2 * F + 8) * 2 * U, (name, rel)
    total = norm64(before)
    assert abs(float(norm) - total) <= 2 * U * total and total > 1.0
    for got, b in zip(grads, before):
        close(got, b.double() / total, 5 * U * b.double().abs() / total, "clipped")


def test_training_step_with_dispatch_and_weights():
    """The vanilla layer with its rows copied out (as before an exchange) and the weights applied on the way back, bf16 rows:
    the exact gradient of what the calls computed, each against 64 bits on its own inputs."""
    T, H, F, n, k = 60, 96, 64, 8, 2
    g = torch.Generator().manual_seed(7)
    x, dy = (torch.randn((T, H), generator=g).to(BF) for _ in range(2))
    logits = torch.randn((T, n), generator=g)
    ids, p, t = pcm.pcm_route_paths(gpu(logits), pcm.pcm_mask_pack(torch.eye(n, dtype=torch.uint8, device=DEV)), k)
    of, off = t.row_of, t.expert_offsets
    w1, w2 = gpu((torch.randn((n, 2 * F, H), generator=g) * 0.1).to(BF)), gpu((torch.randn((n, H, F), generator=g) * 0.1).to(BF))
    rows = pcm.pcm_dispatch_rows(gpu(x), of)
    same_bits(rows, x[t.row_token.cpu().long()])
    o = pcm.pcm_grouped_gemm(pcm.pcm_swiglu(pcm.pcm_grouped_gemm(rows, w1, off)), w2, off)
    y = pcm.pcm_combine_rows(o, of, p, out_dtype=F32)
    terms = o.cpu().double()[of.cpu().long()] * p.cpu().double()[:, :, None]
    close(y, terms.sum(1), (k + 1) * U * terms.abs().sum(1), "y")
    do, dw = pcm.pcm_combine_rows_grad(gpu(dy), of, o, p)
    dlogits = pcm.pcm_route_grad(ids, p, n, dw=dw)
    want, dp = route_grad64(ids.cpu(), p.cpu(), n, None, None, dw.cpu(), 0)
    close(dlogits, want, U * want.abs() + 2.0 ** -40 * (1 + dp.abs().amax(1, keepdim=True)), "dlogits")
    drows = pcm.pcm_grouped_gemm_dx(do, w2, off)
    assert drows.shape == (T * k, F)
    dx, _ = pcm.pcm_dispatch_rows_grad(rows, of)
    close(dx, k * x.double(), 0 * x.double() + 2 * U * k * x.double().abs(), "dx")


def test_training_step_of_a_vanilla_layer():
    """A whole step of the vanilla layer: router, rows copied to their experts, products, SwiGLU, rows back with the router's
    weights; every gradient back to the hidden states, the experts' and the router's weights. Against autograd in 64 bits on
    the same selection; bounds as for the path layer."""
    T, H, F, n, k = 45, 160, 96, 16, 3
    g = torch.Generator().manual_seed(8)
    x, dy = torch.randn((T, H), generator=g), torch.randn((T, H), generator=g)
    w1, w2 = torch.randn((n, 2 * F, H), generator=g) * 0.08, torch.randn((n, H, F), generator=g) * 0.08
    wr = torch.randn((n, H), generator=g) * 0.1
    X, D, W1, W2, WR = (gpu(t) for t in (x, dy, w1, w2, wr))
    # forward (without paths between experts the path table is the plain dispatch)
    logits = pcm.pcm_grouped_gemm(X, WR)
    ids, p, t = pcm.pcm_route_paths(logits, pcm.pcm_mask_pack(torch.eye(n, dtype=torch.uint8, device=DEV)), k)
    off, of = t.expert_offsets, t.row_of
    rows = pcm.pcm_dispatch_rows(X, of, offsets=off)
    gu = pcm.pcm_grouped_gemm(rows, W1, off)
    u = pcm.pcm_swiglu(gu)
    o = pcm.pcm_grouped_gemm(u, W2, off)
    y = pcm.pcm_combine_rows(o, of, p, off)
    # backward
    do, dp = pcm.pcm_combine_rows_grad(D, of, o, p, off)
    du, dW2 = pcm.pcm_grouped_gemm_dx(do, W2, off), pcm.pcm_grouped_gemm_dw(u, do, off)
    dgu = pcm.pcm_swiglu_grad(gu, du)
    drows, dW1 = pcm.pcm_grouped_gemm_dx(dgu, W1, off), pcm.pcm_grouped_gemm_dw(rows, dgu, off)
    dlogits = pcm.pcm_route_grad(ids, p, n, dw=dp)
    dWR = pcm.pcm_grouped_gemm_dw(X, dlogits)
    dX = pcm.pcm_dispatch_rows_grad(drows, of, offsets=off)[0] + pcm.pcm_grouped_gemm_dx(dlogits, WR)
    # 64 bits
    x64, a64, b64, r64 = (v.double().requires_grad_() for v in (x, w1, w2, wr))
    sel = ids.cpu().long()
    p64 = torch.matmul(x64, r64.T).gather(1, sel).softmax(1)
    v = (a64[sel] @ x64[:, None, :, None])[..., 0]
    h = torch.nn.functional.silu(v[..., :F]) * v[..., F:]
    y64 = ((b64[sel] @ h[..., None])[..., 0] * p64[:, :, None]).sum(1)
    y64.backward(dy.double())
    for name, got, want in (("y", y, y64.detach()), ("dX", dX, x64.grad), ("dW1", dW1, a64.grad), ("dW2", dW2, b64.grad),
                            ("dWR", dWR, r64.grad)):
        rel = float((got.cpu().double() - want).norm() / want.norm())
        assert rel <= 64 * (2 * F + 8) * 2 * U, (name, rel)
