"""The experts' products, their gradients, the 8-bit quantisers and the 8-bit product against the same
sums in 64 bits (needs an MI355X).

A sum of m products in float32, in whatever order and with additions rounded or cut (2^-23 relative each),
is off by at most m 2^-23 S, where S is the sum of the products' magnitudes; eight more steps cover scales
and joins. A bf16 output adds half its step, 2^-8 relative. The quantisers use IEEE operations that torch
repeats on the CPU: their codes and scales are the same bits."""
import sys

import pytest
import torch

import paper_2609_01024_amd as pcm
from paper_2609_01024_amd import binding

pytestmark = pytest.mark.gpu
DEV = "cuda"
STEP = 2.0 ** -23
F8 = torch.float8_e4m3fn
# The 8-bit matrix cores (results in bf16) cut each product at 2^-13 of the largest of its group of at most
# 8 neighbours: 8 x 2^-13 of a group's sum of magnitudes at most. Results in float32 use exact products.
EIGHT = {"bf16": 2.0 ** -10, "f32": 0.0}
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


@pytest.fixture(autouse=True)
def _named(request):
    print(request.node.name, flush=True)
    sys.stdout.flush()
    yield


# ------------------------------------------------------------------------ cases
# (T, k, counts or None, n, K, N): counts of rows per group, or None for random routing of T tokens
SHAPES = {
    "one value": (1, 1, None, 1, 16, 16),
    "one token": (1, 2, None, 4, 64, 48),
    "short contraction": (5, 1, None, 3, 48, 80),
    "slices and a rest": (70, 2, None, 5, 208, 144),
    "one slice": (33, 1, None, 2, 64, 64),
    "tile borders": (128, 2, [64, 0, 1, 63, 65, 63], 6, 128, 272),
    "one group has all": (300, 1, [0, 300, 0, 0], 4, 336, 96),
    "last group empty": (40, 1, [7, 33, 0], 3, 96, 400),
    "many groups": (40, 8, None, 256, 80, 112),
    "long contraction": (24, 1, None, 2, 2064, 32),
    "several row tiles": (700, 2, None, 3, 160, 528),
}


def routing(T, k, counts, n, seed):
    """(offsets, row_token, row_of, counts): rows ordered by (group, token)."""
    g = torch.Generator().manual_seed(seed)
    if counts is None:
        ids = torch.rand((T, n), generator=g).topk(k, 1).indices.reshape(-1)
    else:
        ids = torch.repeat_interleave(torch.arange(n), torch.tensor(counts))[torch.randperm(T * k, generator=g)]
    order = ids.sort(stable=True).indices
    row_of = torch.empty_like(order)
    row_of[order] = torch.arange(T * k)
    counts = torch.bincount(ids, minlength=n)
    offsets = torch.cat([torch.zeros(1, dtype=torch.int64), counts.cumsum(0)])
    return offsets.int(), (order // k).int(), row_of.reshape(T, k).int()


def made(shape, dtype, gather, seed=0):
    T, k, counts, n, K, N = SHAPES[shape] if isinstance(shape, str) else shape
    off, tok, of = routing(T, k, counts, n, seed)
    g = torch.Generator().manual_seed(seed + 1)
    R = T * k
    x = torch.randn((T if gather else R, K), generator=g).to(dtype)
    w = (torch.randn((n, N, K), generator=g) * 0.1).to(dtype)
    dy = torch.randn((R, N), generator=g).to(dtype)
    return dict(T=T, k=k, n=n, K=K, N=N, R=R, off=off, tok=tok if gather else None, of=of if gather else None, x=x, w=w, dy=dy)


def gpu(t):
    return None if t is None else t.to(DEV)


def source(c):
    return c["tok"].long() if c["tok"] is not None else torch.arange(c["R"])


def group_of(c):
    return torch.bucketize(torch.arange(c["R"]), c["off"][1:].long(), right=True)


def forward64(c, x, w):
    y = torch.zeros((c["R"], w.shape[1]), dtype=torch.float64)
    e = group_of(c)
    for i in range(c["n"]):
        y[e == i] = x[source(c)[e == i]] @ w[i].T
    return y


def close(got, want, mag, terms, what="", extra=0.0):
    """got within the bound above of want (64 bits); mag: the same sums of magnitudes."""
    got = got.detach().cpu()
    half = 2.0 ** -8 if got.dtype == torch.bfloat16 else 0.0
    bound = ((terms + 8) * STEP + extra) * mag
    bound = bound + half * (want.abs() + bound) + 1e-37
    d = (got.double() - want).abs()
    bad = ~(d <= bound)
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.numel()} outside, worst {float((d / bound).nan_to_num(1e9).max()):.3g} of the bound"


def check_forward(c, out=None, **kw):
    y = pcm.pcm_grouped_gemm(gpu(c["x"]), gpu(c["w"]), gpu(c["off"]), gpu(c["tok"]), out_dtype=out, **kw)
    x, w = c["x"].double(), c["w"].double()
    close(y, forward64(c, x, w), forward64(c, x.abs(), w.abs()), c["K"], "y")
    return y


def rows_dx64(c, dy, w):
    dx = torch.zeros((c["R"], c["K"]), dtype=torch.float64)
    e = group_of(c)
    for i in range(c["n"]):
        dx[e == i] = dy[e == i] @ w[i]
    return dx


def dx64(c, dy, w):
    rows = rows_dx64(c, dy, w)
    return rows if c["of"] is None else rows[c["of"].long()].sum(1)


def dw64(c, x, dy):
    dw = torch.zeros((c["n"], c["N"], c["K"]), dtype=torch.float64)
    e, s = group_of(c), source(c)
    for i in range(c["n"]):
        dw[i] = dy[e == i].T @ x[s[e == i]]
    return dw


# ------------------------------------------------------------------------ products and gradients
@pytest.mark.parametrize("gather", [True, False])
@pytest.mark.parametrize("types", ["bf16-bf16", "bf16-f32", "f32-f32"])
@pytest.mark.parametrize("shape", SHAPES)
def test_forward(shape, types, gather):
    dt, out = (TYPES[t] for t in types.split("-"))
    c = made(shape, dt, gather)
    assert check_forward(c, out).dtype == out


@pytest.mark.parametrize("gather", [True, False])
@pytest.mark.parametrize("types", ["bf16-bf16", "bf16-f32", "f32-f32"])
@pytest.mark.parametrize("shape", SHAPES)
def test_input_gradient(shape, types, gather):
    dt, out = (TYPES[t] for t in types.split("-"))
    c = made(shape, dt, gather)
    dx = pcm.pcm_grouped_gemm_dx(gpu(c["dy"]), gpu(c["w"]), gpu(c["off"]), gpu(c["of"]), out_dtype=out)
    dy, w = c["dy"].double(), c["w"].double()
    close(dx, dx64(c, dy, w), dx64(c, dy.abs(), w.abs()), c["N"] + c["k"], "dx")


@pytest.mark.parametrize("gather", [True, False])
@pytest.mark.parametrize("types", ["bf16-bf16", "bf16-f32", "f32-f32"])
@pytest.mark.parametrize("shape", SHAPES)
def test_weight_gradient(shape, types, gather):
    dt, out = (TYPES[t] for t in types.split("-"))
    c = made(shape, dt, gather)
    dw = torch.full((c["n"], c["N"], c["K"]), float("nan"), dtype=out, device=DEV)   # every element is written
    pcm.pcm_grouped_gemm_dw(gpu(c["x"]), gpu(c["dy"]), gpu(c["off"]), gpu(c["tok"]), dw=dw)
    x, dy = c["x"].double(), c["dy"].double()
    most = int((c["off"][1:] - c["off"][:-1]).max())
    close(dw, dw64(c, x, dy), dw64(c, x.abs(), dy.abs()), most, "dw")


@pytest.mark.parametrize("types", ["bf16", "f32"])
def test_weight_gradient_accumulates(types):
    c = made("tile borders", TYPES[types], True)
    g = torch.Generator().manual_seed(9)
    before = torch.randn((c["n"], c["N"], c["K"]), generator=g)
    dw = before.to(DEV)
    pcm.pcm_grouped_gemm_dw(gpu(c["x"]), gpu(c["dy"]), gpu(c["off"]), gpu(c["tok"]), dw=dw, accumulate=True)
    x, dy = c["x"].double(), c["dy"].double()
    close(dw, before.double() + dw64(c, x, dy), before.double().abs() + dw64(c, x.abs(), dy.abs()), 70, "dw")
    assert torch.equal(dw[1].cpu(), before[1])      # the empty group


@pytest.mark.parametrize("types", ["bf16", "f32"])
def test_one_group_without_offsets(types):
    dt = TYPES[types]
    g = torch.Generator().manual_seed(3)
    x, w, dy = (torch.randn(s, generator=g).to(dt) for s in ((77, 112), (176, 112), (77, 176)))
    X, W, D = x.double(), w.double(), dy.double()
    close(pcm.pcm_grouped_gemm(gpu(x), gpu(w)), X @ W.T, X.abs() @ W.abs().T, 112, "y")
    close(pcm.pcm_grouped_gemm_dx(gpu(dy), gpu(w)), D @ W, D.abs() @ W.abs(), 176, "dx")
    dw = pcm.pcm_grouped_gemm_dw(gpu(x), gpu(dy))
    assert dw.shape == w.shape
    close(dw, D.T @ X, D.abs().T @ X.abs(), 77, "dw")


@pytest.mark.parametrize("types", ["bf16", "f32"])
def test_gradients_against_differences(types):
    """<dy, f(x + v) - f(x - v)> = 2 <dx, v> and the same for w: the product is linear in each. The operands
    are small integers, so that every sum is exact in float32 and both sides have to be equal."""
    dt = TYPES[types]
    c = made("slices and a rest", dt, True)
    g = torch.Generator().manual_seed(5)
    ints = lambda shape, m: torch.randint(-m, m + 1, shape, generator=g).to(dt)
    x, w, dy = ints(c["x"].shape, 3), ints(c["w"].shape, 3), ints(c["dy"].shape, 3)
    vx, vw = ints(x.shape, 2), ints(w.shape, 2)
    off, tok, of = gpu(c["off"]), gpu(c["tok"]), gpu(c["of"])
    f = lambda x, w: pcm.pcm_grouped_gemm(gpu(x), gpu(w), off, tok, out_dtype=torch.float32).cpu().double()
    dx = pcm.pcm_grouped_gemm_dx(gpu(dy), gpu(w), off, of, out_dtype=torch.float32).cpu().double()
    dw = pcm.pcm_grouped_gemm_dw(gpu(x), gpu(dy), off, tok, out_dtype=torch.float32).cpu().double()
    D = dy.double()
    assert float((D * (f(x + vx, w) - f(x - vx, w))).sum()) == 2 * float((dx * vx.double()).sum())
    assert float((D * (f(x, w + vw) - f(x, w - vw))).sum()) == 2 * float((dw * vw.double()).sum())


# ------------------------------------------------------------------------ every tile
# Sizes at which each kernel is chosen (by the number of its tiles), contractions of one to many slices of
# every kind: whole, cut, and around the eight slices whose 8-bit scales travel together.
LENGTHS = [16, 64, 80, 128, 144, 192, 208, 320, 400, 1040, 1168, 2064]
TILES = {   # counts, columns
    "256 x 256": ([700, 1500, 130, 0, 670, 257], 4112),
    "256 x 256, short groups": ([300, 20, 129, 500, 64, 77, 255, 256], 6160),
    "128 x 128": ([1000], 4112),
    "64 x 128": ([129, 1, 370], 4112),
    "64 x 64": ([90, 33, 40, 200, 61], 1040),
    "32 x 64": ([90, 33, 40], 272),
    "16 rows": ([16, 1, 0, 17, 5, 40, 3, 2], 208),
}
TILES_OF_8_BITS = {"128 x 128": ([1400, 300], 4112), "64 x 128": ([129, 1, 600], 4112), "64 x 64": ([90, 33, 40, 200, 61], 2064),
                   "32 x 64": ([190, 33, 40], 2064)}


def on(c):
    return {k: v.to(DEV) if isinstance(v, torch.Tensor) else v for k, v in c.items()}


def rows64(c, a, b, dx=False):
    """Row-wise products of every group in 64 bits on the GPU, and the sums of magnitudes."""
    bounds = c["off"].tolist()
    cols = b.shape[2] if dx else b.shape[1]
    y = torch.zeros((a.shape[0], cols), dtype=torch.float64, device=DEV)
    m = torch.zeros_like(y)
    for i in range(b.shape[0]):
        r, w = slice(bounds[i], bounds[i + 1]), (b[i] if dx else b[i].T).double().contiguous()
        y[r] = a[r].double() @ w
        m[r] = a[r].double().abs() @ w.abs()
    return y.cpu(), m.cpu()


@pytest.mark.parametrize("types", ["bf16-bf16", "bf16-f32", "f32-f32"])
@pytest.mark.parametrize("length", LENGTHS)
@pytest.mark.parametrize("tile", TILES)
def test_tiles_forward_and_input_gradient(tile, length, types):
    counts, cols = TILES[tile]
    dt, out = (TYPES[t] for t in types.split("-"))
    c = on(made((sum(counts), 1, counts, len(counts), length, cols), dt, True, seed=length))
    y = pcm.pcm_grouped_gemm(c["x"], c["w"], c["off"], c["tok"], out_dtype=out)
    close(y, *rows64(c, c["x"][c["tok"].long()], c["w"]), length, "y")
    c = on(made((sum(counts), 1, counts, len(counts), cols, length), dt, False, seed=length))
    dx = pcm.pcm_grouped_gemm_dx(c["dy"], c["w"], c["off"], out_dtype=out)
    close(dx, *rows64(c, c["dy"], c["w"], dx=True), length, "dx")


@pytest.mark.parametrize("counts,cols", [([39 * 256 + 100], 1280), ([13 * 256 + 1, 12 * 256 + 128, 14 * 256 + 7], 1280),
                                         ([20 * 256 + 5, 19 * 256], 1296), ([9 * 256 + 3] * 5, 1040)])
def test_long_row_tiles_before_short_ones(counts, cols):
    """Every tile is computed, also where neither the long tiles nor the short ones are a multiple of the XCDs."""
    c = on(made((sum(counts), 1, counts, len(counts), 64, cols), torch.bfloat16, False, seed=cols))
    y = torch.full((sum(counts), cols), float("nan"), dtype=torch.float32, device=DEV)
    pcm.pcm_grouped_gemm(c["x"], c["w"], c["off"], y=y)
    close(y, *rows64(c, c["x"], c["w"]), 64, "y")


@pytest.mark.parametrize("gather", [True, False])
@pytest.mark.parametrize("types", ["bf16-bf16", "bf16-f32", "f32-f32"])
@pytest.mark.parametrize("N,K", [(1552, 1296), (848, 528), (80, 144)])
@pytest.mark.parametrize("counts", [[0, 1, 63, 64, 65, 200], [127, 128, 129, 500, 2, 191], [320, 256, 16, 3, 0, 1100],
                                    [0, 4097, 1000], [3000]])
def test_tiles_weight_gradient(counts, N, K, types, gather):
    dt, out = (TYPES[t] for t in types.split("-"))
    c = on(made((sum(counts), 1, counts, len(counts), K, N), dt, gather, seed=N))
    dw = torch.full((c["n"], N, K), float("nan"), dtype=out, device=DEV)
    pcm.pcm_grouped_gemm_dw(c["x"], c["dy"], c["off"], c["tok"], dw=dw)
    x = (c["x"][c["tok"].long()] if gather else c["x"]).double()
    bounds = c["off"].tolist()
    parts = [(x[a:b], c["dy"][a:b].double().T.contiguous()) for a, b in zip(bounds, bounds[1:])]
    want = torch.stack([d @ v for v, d in parts]).cpu()
    mag = torch.stack([d.abs() @ v.abs() for v, d in parts]).cpu()
    close(dw, want, mag, max(counts), "dw")
    if out == torch.float32:
        again = dw.clone()
        pcm.pcm_grouped_gemm_dw(c["x"], c["dy"], c["off"], c["tok"], dw=again, accumulate=True)
        assert torch.equal(again, dw + dw)


@pytest.mark.parametrize("out", ["bf16", "f32"])
@pytest.mark.parametrize("length", LENGTHS)
@pytest.mark.parametrize("tile", ["128 x 128", "64 x 128", "64 x 64", "32 x 64", "16 rows"])
def test_tiles_of_8_bits(tile, length, out):
    counts, cols = TILES_OF_8_BITS.get(tile, TILES[tile])
    c = on(made8((sum(counts), 1, counts, len(counts), length, cols), True, seed=length))
    y = product8(c, out_dtype=TYPES[out])
    x = c["xq"].double() * spread(c["xs"], 0, length)
    w = c["wq"].double() * spread(c["ws"], cols, length, 2)
    close(y, *rows64(c, x[c["tok"].long()], w), length, "y", EIGHT[out])


def test_rows_too_long_for_32_bits():
    """Contractions and columns so long that offsets within a tile pass 32 bits, in every direction."""
    K = (1 << 22) + 48
    g = torch.Generator(device=DEV).manual_seed(1)
    x = torch.randn((3, K), generator=g, device=DEV).bfloat16()
    w = torch.randn((16, K), generator=g, device=DEV).bfloat16()
    X, W = x.double(), w.double()
    close(pcm.pcm_grouped_gemm(x, w, out_dtype=torch.float32), (X @ W.T).cpu(), (X.abs() @ W.abs().T).cpu(), K, "y")
    K = (1 << 24) + 48
    dy = torch.randn((5, 16), generator=g, device=DEV).bfloat16()
    w = torch.randn((16, K), generator=g, device=DEV).bfloat16()
    dx = pcm.pcm_grouped_gemm_dx(dy, w, out_dtype=torch.float32)
    x = torch.randn((5, K), generator=g, device=DEV).bfloat16()
    dw = pcm.pcm_grouped_gemm_dw(x, dy, out_dtype=torch.float32)
    D = dy.double()
    for at in (slice(0, 4096), slice(K // 2, K // 2 + 4096), slice(K - 4096, K)):
        W, X = w[:, at].double(), x[:, at].double()
        close(dx[:, at], (D @ W).cpu(), (D.abs() @ W.abs()).cpu(), 16, "dx")
        close(dw[:, at], (D.T @ X).cpu(), (D.T.abs() @ X.abs()).cpu(), 5, "dw")


def test_rows_gathered_past_32_bits():
    """x of more than 2 GiB, rows from its end."""
    T, K, N = 70000, 16400, 48
    x = torch.empty((T, K), dtype=torch.bfloat16, device=DEV)
    x.view(torch.int16).zero_()
    tok = torch.tensor([T - 1, 0, 65535, 65600, T - 2, 12345] * 9, dtype=torch.int32, device=DEV)
    g = torch.Generator(device=DEV).manual_seed(2)
    for t in set(tok.tolist()):
        x[t] = torch.randn(K, generator=g, device=DEV).bfloat16()
    off = torch.tensor([0, 20, len(tok)], dtype=torch.int32, device=DEV)
    w = torch.randn((2, N, K), generator=g, device=DEV).bfloat16()
    rows = x[tok.long()]
    c = dict(off=off)
    close(pcm.pcm_grouped_gemm(x, w, off, tok, out_dtype=torch.float32), *rows64(c, rows, w), K, "y")
    dy = torch.randn((len(tok), N), generator=g, device=DEV).bfloat16()
    dw = pcm.pcm_grouped_gemm_dw(x, dy, off, tok, out_dtype=torch.float32)
    for i, r in enumerate((slice(0, 20), slice(20, len(tok)))):
        D, X = dy[r].double().T.contiguous(), rows[r].double()
        close(dw[i], (D @ X).cpu(), (D.abs() @ X.abs()).cpu(), 34, "dw")


# ------------------------------------------------------------------------ rows that do not count
@pytest.mark.parametrize("types", ["bf16", "f32"])
def test_rows_behind_the_last_group(types):
    """Rows from offsets[n] on: not read (they hold NaN), not written."""
    dt = TYPES[types]
    c = made((60, 2, None, 3, 80, 96), dt, True)
    pad = 37
    tok = torch.cat([c["tok"], torch.zeros(pad, dtype=torch.int32)])
    y = torch.full((c["R"] + pad, c["N"]), 7.0, dtype=dt, device=DEV)
    pcm.pcm_grouped_gemm(gpu(c["x"]), gpu(c["w"]), gpu(c["off"]), gpu(tok), y=y)
    x, w = c["x"].double(), c["w"].double()
    close(y[:c["R"]], forward64(c, x, w), forward64(c, x.abs(), w.abs()), c["K"], "y")
    assert bool((y[c["R"]:] == 7.0).all())
    dy = torch.cat([c["dy"], torch.full((pad, c["N"]), float("nan"), dtype=dt)])
    dx = torch.full((c["R"] + pad, c["K"]), 7.0, dtype=dt, device=DEV)
    pcm.pcm_grouped_gemm_dx(gpu(dy), gpu(c["w"]), gpu(c["off"]), dx=dx)
    D = c["dy"].double()
    close(dx[:c["R"]], rows_dx64(c, D, w), rows_dx64(c, D.abs(), w.abs()), c["N"], "dx")
    assert bool((dx[c["R"]:] == 7.0).all())
    dw = pcm.pcm_grouped_gemm_dw(gpu(c["x"]), gpu(dy), gpu(c["off"]), gpu(tok))
    close(dw, dw64(c, x, D), dw64(c, x.abs(), D.abs()), c["R"], "dw")


@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("types", ["bf16", "f32"])
def test_values_that_are_not_finite_stay_in_their_rows(types, value):
    """One group's rows of x and dy hold NaN or an infinity: no other group's results change, in any
    direction, though tiles and slices of the neighbours reach over the border."""
    dt = TYPES[types]
    c = made((66, 1, [21, 24, 21], 3, 80, 48), dt, False)
    e = group_of(c)
    x, dy = c["x"].clone(), c["dy"].clone()
    x[e == 1] = value
    dy[e == 1] = value
    ref_x, ref_dy = c["x"].clone(), c["dy"].clone()
    ref_x[e == 1] = 0
    ref_dy[e == 1] = 0
    keep = (e != 1).to(DEV)
    off, w = gpu(c["off"]), gpu(c["w"])
    for call in (lambda x, dy: pcm.pcm_grouped_gemm(gpu(x), w, off)[keep],
                 lambda x, dy: pcm.pcm_grouped_gemm_dx(gpu(dy), w, off)[keep],
                 lambda x, dy: pcm.pcm_grouped_gemm_dw(gpu(x), gpu(dy), off)[[0, 2]]):
        a, b = call(x, dy), call(ref_x, ref_dy)
        assert bool(torch.isfinite(a).all()) and torch.equal(a, b)
    assert not bool(torch.isfinite(pcm.pcm_grouped_gemm_dw(gpu(x), gpu(dy), off)[1]).any())
    assert not bool(torch.isfinite(pcm.pcm_grouped_gemm(gpu(x), w, off)[(e == 1).to(DEV)]).any())


def test_input_gradient_of_tokens_without_rows():
    """Negative row_of entries are skipped; a token with none gets zeros; R = 0 gives zeros everywhere."""
    T, k, n, K, N = 9, 3, 2, 48, 32
    g = torch.Generator().manual_seed(2)
    R = 10
    of = torch.full((T, k), -1, dtype=torch.int32)
    of.view(-1)[torch.randperm(T * k, generator=g)[:R]] = torch.randperm(R, generator=g).int()
    of[4] = -1
    off = torch.tensor([0, 4, R], dtype=torch.int32)
    dy, w = torch.randn((R, N), generator=g), torch.randn((n, N, K), generator=g)
    dx = pcm.pcm_grouped_gemm_dx(gpu(dy), gpu(w), gpu(off), gpu(of)).cpu()
    rows = torch.cat([dy[:4].double() @ w[0].double(), dy[4:].double() @ w[1].double()])
    mags = torch.cat([dy[:4].abs().double() @ w[0].abs().double(), dy[4:].abs().double() @ w[1].abs().double()])
    take = lambda r: torch.where((of >= 0)[:, :, None], r[of.clamp_min(0).long()], 0.0).sum(1)
    close(dx, take(rows), take(mags), N + k, "dx")
    assert bool((dx[4] == 0).all())
    none = pcm.pcm_grouped_gemm_dx(gpu(dy[:0]), gpu(w), gpu(off * 0), gpu(of * 0 - 1))
    assert none.shape == (T, K) and bool((none == 0).all())


@pytest.mark.parametrize("R,pad", [(10, 7), (40, 24)])
@pytest.mark.parametrize("types", ["bf16", "f32"])
def test_input_gradient_skips_rows_of_no_group(types, R, pad):
    """Rows in front of offsets[0] and from offsets[n] on, and numbers that are no row, have no part in a
    token's gradient: their workspace rows (NaN here) are not written."""
    dt, k, n, K, N = TYPES[types], 4, 2, 48, 32
    T = R + pad
    g = torch.Generator().manual_seed(8)
    off = torch.tensor([3, R // 2, R], dtype=torch.int32)          # of R + pad rows
    of = torch.randint(-2, R + pad, (T, k), generator=g).int()
    of[0] = torch.tensor([0, 2, R, R + pad - 1])                   # only rows of no group
    of[1] = torch.tensor([3, R - 1, R + pad, 2 ** 31 - 1])
    dy = torch.randn((R + pad, N), generator=g).to(dt)
    dy[:3] = dy[R:] = float("nan")
    w = torch.randn((n, N, K), generator=g).to(dt)
    ws = torch.full((T * k * K * 4,), 0xFF, dtype=torch.uint8, device=DEV)
    dx = pcm.pcm_grouped_gemm_dx(gpu(dy), gpu(w), gpu(off), gpu(of), out_dtype=torch.float32, ws=ws)
    rows, mags = torch.zeros((R + pad, K), dtype=torch.float64), torch.zeros((R + pad, K), dtype=torch.float64)
    for i, (a, b) in enumerate(((3, R // 2), (R // 2, R))):
        rows[a:b] = dy[a:b].double() @ w[i].double()
        mags[a:b] = dy[a:b].double().abs() @ w[i].double().abs()
    take = lambda r: torch.where(((of >= 3) & (of < R))[:, :, None], r[of.clamp(0, R + pad - 1).long()], 0.0).sum(1)
    close(dx, take(rows), take(mags), N + k, "dx")
    assert bool((dx[0] == 0).all())


def test_input_gradient_of_one_group_skips_numbers_that_are_no_row():
    """The same without offsets: the rows are [0, R)."""
    T, k, R, K, N = 7, 3, 12, 64, 48
    g = torch.Generator().manual_seed(9)
    of = torch.randint(-3, R + 4, (T, k), generator=g).int()
    of[2] = torch.tensor([R, -1, 2 ** 31 - 1])
    dy, w = torch.randn((R, N), generator=g), torch.randn((N, K), generator=g)
    ws = torch.full((T * k * K * 4,), 0xFF, dtype=torch.uint8, device=DEV)
    dx = pcm.pcm_grouped_gemm_dx(gpu(dy), gpu(w), row_of=gpu(of), ws=ws)
    take = lambda r: torch.where(((of >= 0) & (of < R))[:, :, None], r[of.clamp(0, R - 1).long()], 0.0).sum(1)
    close(dx, take(dy.double() @ w.double()), take(dy.double().abs() @ w.double().abs()), N + k, "dx")
    assert bool((dx[2] == 0).all())


def test_no_rows():
    w = torch.randn((3, 32, 48), device=DEV)
    off = torch.zeros(4, dtype=torch.int32, device=DEV)
    x, dy = torch.empty((0, 48), device=DEV), torch.empty((0, 32), device=DEV)
    assert pcm.pcm_grouped_gemm(x, w, off).shape == (0, 32)
    assert pcm.pcm_grouped_gemm_dx(dy, w, off).shape == (0, 48)
    assert bool((pcm.pcm_grouped_gemm_dw(x, dy, off) == 0).all())
    dw = torch.ones((3, 32, 48), device=DEV)
    pcm.pcm_grouped_gemm_dw(x, dy, off, dw=dw, accumulate=True)
    assert bool((dw == 1).all())
    # rows in the buffers, none in a group
    y = torch.full((8, 32), 3.0, device=DEV)
    pcm.pcm_grouped_gemm(torch.randn((8, 48), device=DEV), w, off, y=y)
    assert bool((y == 3.0).all())


def test_indices_are_held_inside():
    """Gathered rows and offsets outside their buffers are clamped."""
    c = made((30, 2, None, 3, 48, 64), torch.float32, True)
    tok = c["tok"].clone()
    tok[::7] = 1000000
    tok[3::7] = -5
    held = dict(c, tok=tok.clamp(0, c["T"] - 1))
    got = check_forward(held)
    y = pcm.pcm_grouped_gemm(gpu(c["x"]), gpu(c["w"]), gpu(c["off"]), gpu(tok))
    assert torch.equal(y, got)
    a = pcm.pcm_grouped_gemm_dw(gpu(c["x"]), gpu(c["dy"]), gpu(c["off"]), gpu(tok))
    assert torch.equal(a, pcm.pcm_grouped_gemm_dw(gpu(c["x"]), gpu(c["dy"]), gpu(c["off"]), gpu(held["tok"])))
    off = c["off"].clone()
    off[-1] = c["R"] + 12345
    assert torch.equal(pcm.pcm_grouped_gemm(gpu(c["x"]), gpu(c["w"]), gpu(off), gpu(c["tok"])),
                       pcm.pcm_grouped_gemm(gpu(c["x"]), gpu(c["w"]), gpu(c["off"]), gpu(c["tok"])))
    assert torch.equal(pcm.pcm_grouped_gemm_dw(gpu(c["x"]), gpu(c["dy"]), gpu(off), gpu(c["tok"])),
                       pcm.pcm_grouped_gemm_dw(gpu(c["x"]), gpu(c["dy"]), gpu(c["off"]), gpu(c["tok"])))


# ------------------------------------------------------------------------ quantisers
def over(m):
    return torch.full_like(m, 448.0) / m   # a division (a number over a tensor is its reciprocal times the number)


def quantised_rows(x):
    """Codes (uint8) and scales of the rows of a float32 CPU tensor, by the definition."""
    R, K = x.shape
    pad = torch.nn.functional.pad(x, (0, -K % 128)).reshape(R, -1, 128)
    m = torch.where(torch.isfinite(pad), pad.abs(), 0.0).amax(2, keepdim=True).clamp_min(2.0 ** -100)
    q = (pad * over(m)).to(F8).reshape(R, -1)[:, :K]
    return q, (m / 448.0)[:, :, 0]


def same_codes(got, want):
    g, w = got.cpu().contiguous().view(torch.uint8), want.contiguous().view(torch.uint8)
    nan = (w & 0x7F) == 0x7F
    assert torch.equal((g & 0x7F) == 0x7F, nan), "NaN codes differ"
    assert torch.equal(g[~nan], w[~nan]), "codes differ"


def hard_rows(R, K, dtype, seed=0):
    """Normal values of very different blocks, ties, zeros and the ends of the type's range."""
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((R, K), generator=g) * torch.exp2(torch.randint(-30, 30, (R, 1), generator=g).float())
    x[0] = 0.0
    if R > 3:
        x[1] = (torch.arange(K) % 15 - 7.0) * 0.5
        x[2, ::3] = torch.finfo(torch.float32).max / 2
        x[3] = torch.exp2(-torch.arange(K).float().clamp_max(140))
    return x.to(dtype)


@pytest.mark.parametrize("types", ["bf16", "f32"])
@pytest.mark.parametrize("R,K", [(1, 16), (4, 128), (5, 144), (33, 1408), (7, 7168), (300, 80), (2000, 272)])
def test_quantise_rows(R, K, types):
    x = hard_rows(R, K, TYPES[types])
    q, scale = pcm.pcm_quant_fp8_rows(gpu(x))
    want, want_scale = quantised_rows(x.float())
    assert torch.equal(scale.cpu(), want_scale)
    same_codes(q, want)


@pytest.mark.parametrize("types", ["bf16", "f32"])
def test_quantise_values_that_are_not_finite(types):
    x = hard_rows(6, 400, TYPES[types])
    x[1, 5], x[1, 200], x[4, 399], x[5] = float("nan"), float("inf"), -float("inf"), float("nan")
    q, scale = pcm.pcm_quant_fp8_rows(gpu(x))
    want, want_scale = quantised_rows(x.float())
    assert torch.equal(scale.cpu(), want_scale)
    same_codes(q, want)
    assert bool(torch.isnan(q[1].float()[[5, 200]]).all()) and int(torch.isnan(q[1].float()).sum()) == 2
    w = torch.cat([x, x, x]).repeat(8, 1)[:144].contiguous()
    same_codes(pcm.pcm_quant_fp8_weights(gpu(w))[0], quantised_weights(w.float()[None])[0][0])


@pytest.mark.parametrize("R,count", [(50, 0), (50, 1), (50, 37), (50, 50), (50, 99), (50, -3)])
def test_quantise_counted_rows(R, count):
    x = hard_rows(R, 160, torch.bfloat16)
    off = torch.tensor([0, 3, count], dtype=torch.int32, device=DEV)
    q = torch.full((R, 160), 3.0, device=DEV).to(F8)
    scale = torch.full((R, 2), 5.0, device=DEV)
    pcm.pcm_quant_fp8_rows(gpu(x), off[-1], q, scale)
    want, want_scale = quantised_rows(x.float())
    m = max(0, min(R, count))
    same_codes(q[:m], want[:m])
    assert torch.equal(scale[:m].cpu(), want_scale[:m])
    assert bool((q[m:].float() == 3.0).all()) and bool((scale[m:] == 5.0).all())


@pytest.mark.parametrize("types", ["bf16", "f32"])
@pytest.mark.parametrize("R,F", [(1, 16), (9, 144), (64, 1408), (500, 96)])
def test_quantise_swiglu_rows(R, F, types):
    """SiLU(g) u in float32: the exponential's argument, rounded, moves it by |g| 2^-23 relative, the
    exponential, the sum, the reciprocal and the products by a few 2^-23 more. A code is within half a
    step, 2^-4 of its value (2^-10 scales below the smallest normal code), of that."""
    g = torch.Generator().manual_seed(1)
    x = (torch.randn((R, 2 * F), generator=g) * 3).to(TYPES[types])
    q, scale = pcm.pcm_swiglu_quant_fp8(gpu(x))
    gate, up = x.double()[:, :F], x.double()[:, F:]
    h = gate * torch.sigmoid(gate) * up
    err = (gate.abs() + 8) * 2.0 ** -22
    pad = torch.nn.functional.pad(h, (0, -F % 128)).reshape(R, -1, 128)
    s = pad.abs().amax(2) / 448
    assert bool(((scale.cpu().double() - s).abs() <= s * err.max()).all())
    wide = s.repeat_interleave(128, 1)[:, :F]
    d = (q.cpu().double() * scale.cpu().double().repeat_interleave(128, 1)[:, :F] - h).abs()
    assert bool((d <= (2.0 ** -4 * h.abs() + 2.0 ** -10 * wide) * (1 + 2 * err) + 2 * err * h.abs()).all())


@pytest.mark.parametrize("types", ["bf16", "f32"])
def test_quantise_swiglu_of_far_gates(types):
    """Gates whose exponentials leave float32's range: SiLU goes to 0 or to the gate; what is not finite is NaN."""
    gates = torch.tensor([-1e38, -1e4, -200.0, -100.0, -89.0, -88.5, -60.0, 60.0, 100.0, 1e4, 0.0, -0.0, float("inf"),
                          -float("inf"), float("nan"), 1.0]).to(TYPES[types])
    x = torch.cat([gates, torch.full((16,), 2.0, dtype=gates.dtype)])[None].contiguous()
    q, scale = pcm.pcm_swiglu_quant_fp8(gpu(x))
    h = gates.double() * torch.sigmoid(gates.double()) * 2
    fine = torch.isfinite(gates)
    s = float(scale[0, 0])
    assert abs(s - 2e4 / 448) <= 2.0 ** -7 * s          # 1e4 rounded to bf16
    got = q[0].cpu().double()
    assert bool(torch.isnan(got[~fine]).all())
    assert bool(((got[fine] * s - h[fine]).abs() <= 2.0 ** -4 * h[fine].abs() * (1 + 2.0 ** -14) + 2.0 ** -10 * s).all())


def swiglu_alone(gates, up, types):
    """(scale * 448, SiLU(gate) up in 64 bits, its bound) of gates that are alone in their blocks with one value of up:
    the scale is the value itself. The bound is test_quantise_swiglu_rows' (from 110 on SiLU is the gate or 0) and the
    gate times 2^-149, the spacing of an exponential below the normal range."""
    x = torch.zeros((len(gates), 32), dtype=TYPES[types])
    x[:, 0], x[:, 16] = gates, up
    q, scale = pcm.pcm_swiglu_quant_fp8(gpu(x))
    g = gates.double()
    h = g * torch.sigmoid(g) * up
    bound = (g.abs().clamp_max(110) + 8) * 2.0 ** -22 * h.abs() + g.abs().clamp_max(110) * 2.0 ** -149 * up
    got = scale[:, 0].cpu().double() * 448
    codes = q[:, 0].cpu().double() / 448
    big = h.abs() >= 2.0 ** -90
    assert torch.equal(codes[big], torch.sign(h[big]))     # the largest of its block
    return got, h, bound


def bf16_gates():
    """Every finite bf16 value but the zeros."""
    g = (torch.arange(65536, dtype=torch.int32) << 16).view(torch.float32)
    return g[torch.isfinite(g) & (g != 0)]


@pytest.mark.parametrize("types", ["bf16", "f32"])
def test_quantise_swiglu_of_every_gate(types):
    """SiLU of a large gate is the gate, however large, and of every other what it is."""
    got, h, bound = swiglu_alone(bf16_gates(), 1.0, types)
    bad = ~((got - h.abs().clamp_min(2.0 ** -100)).abs() <= bound + 2.0 ** -122)
    assert not bad.any(), (int(bad.sum()), bf16_gates()[bad][:8].tolist())


@pytest.mark.parametrize("types", ["bf16", "f32"])
def test_quantise_swiglu_of_far_negative_gates(types):
    """Large up values bring back SiLUs of gates whose exponentials, or their reciprocals, leave float32's range."""
    gates = bf16_gates()
    gates = gates[(gates < -1.0) & (gates > -100.0)]
    got, h, bound = swiglu_alone(gates, 2.0 ** 100, types)
    bad = ~((got - h.abs()).abs() <= bound)
    assert not bad.any(), (int(bad.sum()), gates[bad][:16].tolist())


def quantised_weights(w):
    n, N, K = w.shape
    pad = torch.nn.functional.pad(w, (0, -K % 128, 0, -N % 128))
    b = pad.reshape(n, pad.shape[1] // 128, 128, pad.shape[2] // 128, 128)
    m = torch.where(torch.isfinite(b), b.abs(), 0.0).amax((2, 4), keepdim=True).clamp_min(2.0 ** -100)
    q = (b * over(m)).to(F8).reshape(pad.shape)[:, :N, :K]
    return q, (m / 448.0)[:, :, 0, :, 0]


@pytest.mark.parametrize("types", ["bf16", "f32"])
@pytest.mark.parametrize("n,N,K", [(1, 16, 16), (2, 128, 128), (3, 144, 272), (1, 400, 96), (5, 48, 1040)])
def test_quantise_weights(n, N, K, types):
    w = torch.stack([hard_rows(N, K, TYPES[types], seed=i) for i in range(n)])
    q, scale, q_t, scale_t = pcm.pcm_quant_fp8_weights(gpu(w), transpose=True)
    want, want_scale = quantised_weights(w.float())
    assert torch.equal(scale.cpu(), want_scale) and torch.equal(scale_t.cpu(), want_scale.mT.contiguous())
    same_codes(q, want)
    same_codes(q_t, want.mT)
    q2, s2 = pcm.pcm_quant_fp8_weights(gpu(w))
    assert torch.equal(q2.view(torch.uint8), q.view(torch.uint8)) and torch.equal(s2, scale)
    if n == 1:   # a single matrix
        q3, s3 = pcm.pcm_quant_fp8_weights(gpu(w[0]))
        assert torch.equal(q3.view(torch.uint8), q[0].view(torch.uint8)) and torch.equal(s3, scale[0])


# ------------------------------------------------------------------------ 8-bit products
def made8(shape, gather, seed=0):
    c = made(shape, torch.float32, gather, seed)
    g = torch.Generator().manual_seed(seed + 7)
    rows, n, N, K = c["x"].shape[0], c["n"], c["N"], c["K"]
    codes = lambda s: (torch.randn(s, generator=g) * 100).clamp(-448, 448).to(F8)
    scales = lambda s: torch.rand(s, generator=g) * 0.01 + 1e-3
    kb, nb = -(-K // 128), -(-N // 128)
    c.update(xq=codes((rows, K)), xs=scales((rows, kb)), wq=codes((n, N, K)), ws=scales((n, nb, kb)))
    return c


def spread(scale, rows, cols, along=1):
    s = scale.double().repeat_interleave(128, -1)[..., :cols]
    return s if along == 1 else s.repeat_interleave(128, -2)[..., :rows, :]


def dequantised(c):
    return (c["xq"].double() * spread(c["xs"], 0, c["K"]), c["wq"].double() * spread(c["ws"], c["N"], c["K"], 2))


def product8(c, **kw):
    return pcm.pcm_grouped_gemm_fp8(gpu(c["xq"]), gpu(c["xs"]), gpu(c["wq"]), gpu(c["ws"]), gpu(c["off"]), gpu(c["tok"]), **kw)


@pytest.mark.parametrize("gather", [True, False])
@pytest.mark.parametrize("out", ["bf16", "f32"])
@pytest.mark.parametrize("shape", SHAPES)
def test_product_of_8_bits(shape, out, gather):
    c = made8(shape, gather)
    x, w = dequantised(c)
    close(product8(c, out_dtype=TYPES[out]), forward64(c, x, w), forward64(c, x.abs(), w.abs()), c["K"], "y", EIGHT[out])


# contraction 272: three blocks of codes; row tiles of 16, 32 and 64 or 128 rows (kernels with and without pairs)
SCALE_SHAPES = {"16 rows": ([16, 1, 0, 17, 5], 208), "32 x 64": ([190, 33, 40], 2064), "large": ([1400, 300], 4112)}


@pytest.mark.parametrize("x_exp,w_exp", [(-60, -66), (-109, -17), (0, -126), (60, 45), (118, -14), (-20, 125)])
@pytest.mark.parametrize("out", ["bf16", "f32"])
@pytest.mark.parametrize("shape", SCALE_SHAPES)
def test_product_of_8_bits_at_the_ends_of_the_scales(shape, out, x_exp, w_exp):
    """Products of scales from the smallest normal number to as large as leaves the results finite, and blocks of
    zeros under them, which count as nothing."""
    counts, cols = SCALE_SHAPES[shape]
    c = made8((sum(counts), 1, counts, len(counts), 272, cols), True, seed=3)
    one_up = torch.randint(0, 2, c["xs"].shape, generator=torch.Generator().manual_seed(1))
    c["xs"] = torch.exp2((one_up + x_exp).float())
    c["ws"] = torch.full_like(c["ws"], 2.0 ** w_exp)
    c["xq"].view(torch.uint8)[:, 128:256] = 0
    c["xq"].view(torch.uint8)[::5] = 0
    c = on(c)
    y = product8(c, out_dtype=TYPES[out])
    x = c["xq"].double() * spread(c["xs"], 0, 272)
    want, mag = rows64(c, x[c["tok"].long()], c["wq"].double() * 2.0 ** w_exp)
    assert float(mag.max()) < 2.0 ** 127
    close(y, want, mag, 272, "y", EIGHT[out])
    assert bool((y[(c["tok"] % 5) == 0] == 0).all())


def test_product_of_8_bits_without_offsets():
    c = made8((50, 1, None, 1, 400, 144), False)
    x, w = dequantised(c)
    y = pcm.pcm_grouped_gemm_fp8(gpu(c["xq"]), gpu(c["xs"]), gpu(c["wq"][0]), gpu(c["ws"][0]), out_dtype=torch.float32)
    close(y, x @ w[0].T, x.abs() @ w[0].abs().T, 400, "y")


def test_8_bit_rows_behind_the_last_group_and_nan():
    c = made8((66, 1, [21, 24, 21], 3, 176, 48), False)
    e = group_of(c)
    clean = product8(c, out_dtype=torch.float32)
    c["xq"].view(torch.uint8)[e == 1] = 0x7F
    c["xs"][e == 1] = float("nan")
    got = product8(c, out_dtype=torch.float32)
    keep = (e != 1).to(DEV)
    assert torch.equal(got[keep], clean[keep]) and bool(torch.isnan(got[~keep]).all())
    y = torch.full((66, 48), 7.0, device=DEV)
    pcm.pcm_grouped_gemm_fp8(gpu(c["xq"]), gpu(c["xs"]), gpu(c["wq"]), gpu(c["ws"]),
                             torch.tensor([0, 21, 21, 21], dtype=torch.int32, device=DEV), y=y)
    assert torch.equal(y[:21], clean[:21]) and bool((y[21:] == 7.0).all())


def test_input_gradient_in_8_bits():
    """dy W through the transposed codes: the same call with the contraction over N."""
    c = made((90, 1, None, 3, 272, 208), torch.bfloat16, False)
    _, _, wt, st = pcm.pcm_quant_fp8_weights(gpu(c["w"]), transpose=True)
    dq, ds = pcm.pcm_quant_fp8_rows(gpu(c["dy"]))
    dx = pcm.pcm_grouped_gemm_fp8(dq, ds, wt, st, gpu(c["off"]), out_dtype=torch.float32)
    d = dq.cpu().double() * spread(ds.cpu(), 0, c["N"])
    w = (wt.cpu().double() * spread(st.cpu(), c["K"], c["N"], 2)).mT
    close(dx, rows_dx64(c, d, w), rows_dx64(c, d.abs(), w.abs()), c["N"], "dx")


# ------------------------------------------------------------------------ streams, graphs, other calls
def all_calls(c, stream=None):
    """Every entry point once."""
    x, w, dy, off, tok, of = (c[v] for v in ("x", "w", "dy", "off", "tok", "of"))
    r = {}
    r["y"] = pcm.pcm_grouped_gemm(x, w, off, tok, stream=stream)
    r["dx"] = pcm.pcm_grouped_gemm_dx(dy, w, off, of, stream=stream)
    r["dw"] = pcm.pcm_grouped_gemm_dw(x, dy, off, tok, stream=stream)
    r["q"], r["s"] = pcm.pcm_quant_fp8_rows(x, stream=stream)
    r["hq"], r["hs"] = pcm.pcm_swiglu_quant_fp8(x, stream=stream)
    r["wq"], r["ws"], r["wt"], r["st"] = pcm.pcm_quant_fp8_weights(w, transpose=True, stream=stream)
    r["y8"] = pcm.pcm_grouped_gemm_fp8(r["q"], r["s"], r["wq"], r["ws"], off, tok, stream=stream)
    return r


def on_gpu(c):
    return {k: gpu(v) if isinstance(v, torch.Tensor) else v for k, v in c.items()}


def same(a, b):
    for k in a:
        assert torch.equal(a[k].contiguous().view(torch.uint8), b[k].contiguous().view(torch.uint8)), k


def test_another_stream():
    c = on_gpu(made("several row tiles", torch.bfloat16, True))
    want = all_calls(c)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    got = all_calls(c, stream=s)
    s.synchronize()
    same(got, want)


def test_deterministic():
    c = on_gpu(made("several row tiles", torch.bfloat16, True))
    a = all_calls(c)
    for _ in range(3):
        same(all_calls(c), a)


def test_graph_replays():
    """Captured once, replayed on new inputs with other work between the replays."""
    c = on_gpu(made("several row tiles", torch.bfloat16, True))
    all_calls(c)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        got = all_calls(c)
    for seed in range(1, 5):
        new = made("several row tiles", torch.bfloat16, True, seed)
        for k, v in new.items():
            if isinstance(v, torch.Tensor):
                c[k].copy_(v)
        want = all_calls(c)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        same(got, want)


def test_refuses_tensors_the_kernels_must_not_address():
    c = on_gpu(made("one slice", torch.bfloat16, True))
    x, w, off, tok = c["x"], c["w"], c["off"], c["tok"]
    for call in (lambda: pcm.pcm_grouped_gemm(x.t(), w, off, tok), lambda: pcm.pcm_grouped_gemm(x, w.cpu(), off, tok),
                 lambda: pcm.pcm_grouped_gemm(x, w, off[:-1], tok), lambda: pcm.pcm_grouped_gemm(x, w[:, :, :32].contiguous(), off, tok),
                 lambda: pcm.pcm_grouped_gemm(x, w, None, tok), lambda: pcm.pcm_grouped_gemm(x, w, off, tok, y=x[1:]),
                 lambda: pcm.pcm_grouped_gemm_dw(x, c["dy"][:-1], off, tok),
                 lambda: pcm.pcm_grouped_gemm_dw(x, c["dy"], off, tok, accumulate=True)):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: pcm.pcm_grouped_gemm(x, w.float(), off, tok), lambda: pcm.pcm_grouped_gemm(x, w, off.long(), tok),
                 lambda: pcm.pcm_grouped_gemm(x.half(), w.half(), off, tok), lambda: pcm.pcm_grouped_gemm_fp8(x, x, w, w, off, tok)):
        with pytest.raises(TypeError):
            call()
    with pytest.raises(RuntimeError):   # K not a multiple of 16
        pcm.pcm_grouped_gemm(torch.zeros((4, 24), device=DEV), torch.zeros((16, 24), device=DEV))
    with pytest.raises(RuntimeError):   # bfloat16 results of float32 operands
        pcm.pcm_grouped_gemm(x.float(), w.float(), off, tok, out_dtype=torch.bfloat16)


# ------------------------------------------------------------------------ together, as they are used
def test_expert_layer_in_8_bits():
    """Serving: a SwiGLU expert layer with 8-bit weights on the path tables that the router builds. With only
    the diagonal of the mask each token's result is the sum over its experts of p_a W_down (SiLU(g) u). The
    sum over the slots is off from the layer in 64 bits by the 8-bit roundings: activations, weights and the
    SwiGLU output 2^-4 relative at most each, so that the products' worst is 2 x 2^-4 + 2^-8 of the sums of
    magnitudes, through SiLU' <= 1.1 and both products."""
    T, H, F, n, k = 37, 256, 192, 6, 2
    g = torch.Generator().manual_seed(4)
    x = torch.randn((T, H), generator=g).bfloat16()
    wgu, wd = (torch.randn((n, 2 * F, H), generator=g) * 0.06).bfloat16(), (torch.randn((n, H, F), generator=g) * 0.06).bfloat16()
    logits = torch.randn((T, n), generator=g)
    ids, p, paths = pcm.pcm_route_paths(gpu(logits), pcm.pcm_mask_pack(torch.eye(n, dtype=torch.uint8, device=DEV)), k)
    (q1, s1), (q2, s2) = pcm.pcm_quant_fp8_weights(gpu(wgu)), pcm.pcm_quant_fp8_weights(gpu(wd))
    xq, xs = pcm.pcm_quant_fp8_rows(gpu(x))
    off, tok = paths.expert_offsets, paths.row_token
    gu = pcm.pcm_grouped_gemm_fp8(xq, xs, q1, s1, off, tok, out_dtype=torch.float32)
    hq, hs = pcm.pcm_swiglu_quant_fp8(gu, off[-1:])
    o = pcm.pcm_grouped_gemm_fp8(hq, hs, q2, s2, off, out_dtype=torch.float32)
    y = (o[paths.row_of.long()] * p[:, :, None]).sum(1).cpu().double()
    # each step against the 64-bit value of its own inputs
    c = dict(n=n, R=T * k, K=H, N=2 * F, off=off.cpu(), tok=tok.cpu())
    dq = lambda q, s: q.cpu().double() * spread(s.cpu(), 0, q.shape[-1])
    dw = lambda q, s: q.cpu().double() * spread(s.cpu(), q.shape[-2], q.shape[-1], 2)
    X, W1, W2 = dq(xq, xs), dw(q1, s1), dw(q2, s2)
    close(gu, forward64(c, X, W1), forward64(c, X.abs(), W1.abs()), H, "gate and up")
    c2 = dict(c, tok=None, K=F, N=H)
    Hd = dq(hq, hs)
    close(o, forward64(c2, Hd, W2), forward64(c2, Hd.abs(), W2.abs()), F, "down")
    # and the whole against the layer in 64 bits
    e, s = group_of(c), source(c)
    eps = 2.0 ** -4
    step = lambda q_scale: 2.0 ** -10 * q_scale
    xe = x.double()
    G64 = torch.stack([wgu.double()[e[r]] @ xe[s[r]] for r in range(T * k)])
    Gm = torch.stack([wgu.double().abs()[e[r]] @ xe.abs()[s[r]] for r in range(T * k)])
    low = torch.stack([step(spread(s1.cpu(), 2 * F, H, 2))[e[r]] @ xe.abs()[s[r]] +
                       (wgu.double().abs()[e[r]] @ step(spread(xs.cpu(), 0, H))[s[r]]) for r in range(T * k)])
    dG = (2 * eps + eps * eps + 1e-4) * Gm + 2 * low
    gate, up, dg, du = G64[:, :F], G64[:, F:], dG[:, :F], dG[:, F:]
    sil = gate * torch.sigmoid(gate)
    h = sil * up
    dh = 1.1 * dg * (up.abs() + du) + sil.abs() * du
    dh = dh + eps * (h.abs() + dh) + step(spread(hs.cpu(), 0, F))
    O64 = torch.stack([wd.double()[e[r]] @ h[r] for r in range(T * k)])
    low2 = step(spread(s2.cpu(), H, F, 2))
    dO = torch.stack([wd.double().abs()[e[r]] @ dh[r] + (eps * wd.double().abs()[e[r]] + low2[e[r]]) @ (h[r].abs() + dh[r])
                      for r in range(T * k)])
    of, P = paths.row_of.cpu().long(), p.cpu().double()
    want, room = (O64[of] * P[:, :, None]).sum(1), (dO[of] * P[:, :, None]).sum(1)
    assert bool(((y - want).abs() <= room).all())


def test_expert_layer_gradients():
    """Training: two products around a SwiGLU on the router's path tables, every gradient against 64-bit
    autograd. Each float32 sum is off by its bound; through the chain the relative errors add, so that a
    bound of 64 times the longest sum's relative one on the norms holds with room."""
    T, H, F, n, k = 45, 160, 96, 5, 2
    g = torch.Generator().manual_seed(6)
    x = torch.randn((T, H), generator=g)
    wgu, wd = torch.randn((n, 2 * F, H), generator=g) * 0.08, torch.randn((n, H, F), generator=g) * 0.08
    dy = torch.randn((T, H), generator=g)
    ids, p, paths = pcm.pcm_route_paths(gpu(torch.randn((T, n), generator=g)),
                                        pcm.pcm_mask_pack(torch.eye(n, dtype=torch.uint8, device=DEV)), k)
    off, tok, of = paths.expert_offsets, paths.row_token, paths.row_of
    X, W1, W2, D = gpu(x), gpu(wgu), gpu(wd), gpu(dy)
    gu = pcm.pcm_grouped_gemm(X, W1, off, tok)
    gate, up = gu[:, :F], gu[:, F:]
    sg = torch.sigmoid(gate)
    h = (gate * sg * up).contiguous()
    rows = torch.empty(T * k, dtype=torch.long, device=DEV)
    rows[of.reshape(-1).long()] = torch.arange(T * k, device=DEV)
    pr = p.reshape(-1)[rows]                       # the weight of each row
    do = (D[tok.long()] * pr[:, None]).contiguous()
    dh = pcm.pcm_grouped_gemm_dx(do, W2, off)
    dW2 = pcm.pcm_grouped_gemm_dw(h, do, off)
    dgu = torch.cat([dh * up * (sg + gate * sg * (1 - sg)), dh * gate * sg], 1)
    dX = pcm.pcm_grouped_gemm_dx(dgu, W1, off, of)
    dW1 = pcm.pcm_grouped_gemm_dw(X, dgu, off, tok)
    x64, a64, b64 = (t.double().requires_grad_() for t in (x, wgu, wd))
    y = torch.zeros((T, H), dtype=torch.float64)
    for t in range(T):
        for a in range(k):
            e = int(ids[t, a])
            v = a64[e] @ x64[t]
            y[t] = y[t] + float(p[t, a]) * (b64[e] @ (torch.nn.functional.silu(v[:F]) * v[F:]))
    y.backward(dy.double())
    for got, want in ((dX, x64.grad), (dW1, a64.grad), (dW2, b64.grad)):
        rel = float((got.cpu().double() - want).norm() / want.norm())
        assert rel <= 64 * (2 * F + 8) * STEP, rel
