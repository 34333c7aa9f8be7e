"""The experts' matrix products on their own, with their gradients and in 8 bits, as cases to measure.

Three operators: the product grouped by expert with its two gradients, the quantisers to 8-bit
floating point (e4m3) with a scale for each block of 128, and the product of such operands.
listed() names the cases, draw() gives more of the same ranges, prepare() makes what a program
holds before the call, run() is one call: in plain torch (32 bits, rounded once), or, where `own`
is true, through the framework. exact() is the same result in 64 bits.

Layer shapes are those of workloads/configs.py (Mixtral-, OLMoE-, fine-grained- and decode-shaped,
and the float32 one) with their routing, generic ones beside them. Rows are (token, slot) pairs
ordered by expert, then token, as the framework's path tables order them."""
import math

import torch

own = False

DEV = "cuda"
BLOCK = 128
FLOOR = 2.0 ** -100   # smallest block maximum that a scale is made from
E4M3_MAX = 448.0


def listed():
    return [
        # the up projection of one decode step at the widest layer: a row or two for most experts
        dict(name="grouped, decode 32", op="grouped", T=32, k=8, n=256, K=7168, N=2048, dtype="bf16", out="bf16",
             gather=True, logits="normal"),
        # gate and up projection of a whole prompt, experts of very different popularity
        dict(name="grouped, prefill 8192", op="grouped", T=8192, k=8, n=64, K=2048, N=2048, dtype="bf16", out="bf16",
             gather=True, logits="zipf"),
        # a small model checked in float32: ragged groups, the down projection of a few hundred tokens
        dict(name="grouped, f32 ragged", op="grouped", T=777, k=4, n=16, K=960, N=768, dtype="f32", out="f32",
             gather=False, logits="zipf"),
        # training step, gate and up projection of fine-grained experts: each token's rows share its input
        dict(name="gradients, fine-grained", op="grads", T=8192, k=4, n=60, K=2048, N=1408, dtype="bf16", out="bf16",
             gather=True, logits="normal"),
        # training step, down projection of few large experts, weight gradients in float32
        dict(name="gradients, few experts", op="grads", T=4096, k=2, n=8, K=14336, N=4096, dtype="bf16", out="f32",
             gather=False, logits="normal"),
        # the float32 layer of the tests and the benchmark
        dict(name="gradients, f32 small", op="grads", T=64, k=2, n=8, K=256, N=512, dtype="f32", out="f32",
             gather=True, logits="normal"),
        # the activations between the two products of a prompt's experts: SwiGLU, then 8 bits
        dict(name="quantise, SwiGLU rows", op="swiglu_quant", R=32768, K=1408, dtype="bf16"),
        # the hidden states of one decode step
        dict(name="quantise, decode rows", op="quant", R=32, K=7168, dtype="bf16"),
        # weights after an optimizer step, for the forward pass and for the gradient of the inputs
        dict(name="quantise, weights", op="quant_weights", n=64, N=2048, K=1024, dtype="bf16", transpose=True),
        # one token through a dense projection
        dict(name="8-bit, one token", op="fp8", T=1, k=1, n=1, K=4096, N=14336, out="bf16", gather=False, logits="normal"),
        # gate projection of a prompt, few large experts
        dict(name="8-bit, prefill 4096", op="fp8", T=4096, k=2, n=8, K=4096, N=14336, out="bf16", gather=True,
             logits="normal_bias"),
        # the up projection of one decode step at the widest layer
        dict(name="8-bit, decode 32", op="fp8", T=32, k=8, n=256, K=7168, N=2048, out="f32", gather=True, logits="normal"),
    ]


def _spread(rng, lo, hi):
    """An integer of [lo, hi], uniform over its logarithm."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["grouped", "grouped", "grads", "grads", "fp8", "fp8", "fp8", "quant", "swiglu_quant", "quant_weights"])
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    if op in ("quant", "swiglu_quant"):
        return dict(op=op, R=_spread(rng, 1, 32768), K=16 * _spread(rng, 1, 448), dtype=dtype)
    if op == "quant_weights":
        return dict(op=op, n=_spread(rng, 1, 64), N=16 * _spread(rng, 1, 256), K=16 * _spread(rng, 1, 256), dtype=dtype,
                    transpose=rng.choice([True, False]))
    f32 = op != "fp8" and dtype == "f32"
    n = rng.choice([1, _spread(rng, 2, 256)])
    most = 60 if f32 else 448
    K, N = 16 * _spread(rng, 4, most), 16 * _spread(rng, 4, most)
    K, N = (K, N) if n * K * N < 1 << 30 else (K // 64 * 16, N // 64 * 16)
    T = _spread(rng, 1, 2048 if f32 else 8192)
    k = rng.randint(1, min(n, 8))
    while T * k * K * N > 4.8e11 / (4 if op == "grads" else 1):
        T = (T + 1) // 2
    c = dict(op=op, T=T, k=k, n=n, K=K, N=N, out="f32" if f32 else rng.choice(["bf16", "f32"]), gather=rng.choice([True, False]),
             logits=rng.choice(["normal", "zipf"]))
    return c if op == "fp8" else dict(c, dtype=dtype)


# ------------------------------------------------------------------------ inputs
def _randn(g, shape, std, dtype):
    return torch.randn(shape, generator=g, device=DEV, dtype=dtype).mul_(std)


def _type(name):
    return {"bf16": torch.bfloat16, "f32": torch.float32}[name]


def _routing(case, g):
    """The rows of T tokens with k of n experts each: offsets [n+1], row_token [T*k], row_of [T, k]."""
    T, n, k = case["T"], case["n"], case["k"]
    logits = torch.randn((T, n), generator=g, device=DEV)
    if case["logits"] == "normal_bias":
        logits += 0.5 * torch.randn((n,), generator=g, device=DEV)
    if case["logits"] == "zipf":
        logits -= 1.1 * torch.log((torch.randperm(n, generator=g, device=DEV) + 1).float())
    ids = logits.topk(k, dim=1).indices.reshape(-1)
    order = ids.sort(stable=True).indices
    row_of = torch.empty_like(order)
    row_of[order] = torch.arange(T * k, device=DEV)
    counts = torch.bincount(ids, minlength=n)
    offsets = torch.cat([counts.new_zeros(1), counts.cumsum(0)])
    return dict(offsets=offsets.int(), row_token=(order // k).int(), row_of=row_of.reshape(T, k).int())


def _quantised(g, groups, rows, cols, std, whole):
    """8-bit values [groups, rows, cols] of normal numbers with a scale for each 128 of a row, or, where `whole`,
    for each 128 x 128 block."""
    shape = (groups, -(-rows // BLOCK) if whole else rows, -(-cols // BLOCK))
    scale = torch.rand(shape, generator=g, device=DEV).add_(0.5).mul_(3.5 * std / E4M3_MAX)
    q = torch.empty((groups, rows, cols), dtype=torch.float8_e4m3fn, device=DEV)
    for e in range(groups):
        q[e] = _randn(g, (rows, cols), E4M3_MAX / 5.0, torch.bfloat16).clamp_(-E4M3_MAX, E4M3_MAX).to(torch.float8_e4m3fn)
    return q, scale


def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    op, s = case["op"], {"case": case}
    if op in ("quant", "swiglu_quant"):
        wide = 2 if op == "swiglu_quant" else 1
        s["x"] = _randn(g, (case["R"], wide * case["K"]), 1.0, _type(case["dtype"]))
        return s
    if op == "quant_weights":
        s["w"] = _randn(g, (case["n"], case["N"], case["K"]), 0.02, _type(case["dtype"]))
        return s
    s.update(_routing(case, g))
    s["bounds"] = s["offsets"].tolist()
    K, N, n = case["K"], case["N"], case["n"]
    rows_in = case["T"] if case["gather"] else case["T"] * case["k"]
    if op == "fp8":
        q, scale = _quantised(g, 1, rows_in, K, 1.0, False)
        s["xq"], s["xs"] = q[0], scale[0]
        s["wq"], s["ws"] = _quantised(g, n, N, K, 0.02, True)
        return s
    dt = _type(case["dtype"])
    s["x"] = _randn(g, (rows_in, K), 1.0, dt)
    s["w"] = _randn(g, (n, N, K), 0.02, dt)
    if op == "grads":
        s["dy"] = _randn(g, (case["T"] * case["k"], N), 1.0, dt)
    return s


# ------------------------------------------------------------------------ one call
def run(s):
    return _own(s) if own else _plain(s)


def _own(s):
    import paper_2609_01024_amd as pcm
    c = s["case"]
    op = c["op"]
    if op == "quant":
        return pcm.pcm_quant_fp8_rows(s["x"])
    if op == "swiglu_quant":
        return pcm.pcm_swiglu_quant_fp8(s["x"])
    if op == "quant_weights":
        return pcm.pcm_quant_fp8_weights(s["w"], transpose=c["transpose"])
    rows = s["row_token"] if c["gather"] else None
    out = _type(c["out"])
    if op == "fp8":
        return pcm.pcm_grouped_gemm_fp8(s["xq"], s["xs"], s["wq"], s["ws"], s["offsets"], rows, out_dtype=out)
    if op == "grouped":
        return pcm.pcm_grouped_gemm(s["x"], s["w"], s["offsets"], rows, out_dtype=out)
    dx = pcm.pcm_grouped_gemm_dx(s["dy"], s["w"], s["offsets"], s["row_of"] if c["gather"] else None)
    return dx, pcm.pcm_grouped_gemm_dw(s["x"], s["dy"], s["offsets"], rows, out_dtype=out)


def _plain(s):
    c = s["case"]
    op = c["op"]
    if op == "quant":
        return _quant_rows(s["x"].float())
    if op == "swiglu_quant":
        gate, up = s["x"].float().chunk(2, dim=1)
        return _quant_rows(gate / (1.0 + torch.exp(-gate)) * up)
    if op == "quant_weights":
        return _quant_blocks(s["w"].float(), c["transpose"])
    K, N, bounds = c["K"], c["N"], s["bounds"]
    out = _type(c["out"])
    # the groups' sizes are what a program with a loop of products has on the host; one product for each group that has rows
    groups = [(e, a, b) for e, (a, b) in enumerate(zip(bounds, bounds[1:])) if b > a]
    if op == "fp8":
        x = _dequantised(s["xq"], s["xs"].repeat_interleave(BLOCK, 1))
        x = x[s["row_token"].long()] if c["gather"] else x
        y = x.new_empty((x.shape[0], N), dtype=out)
        for e, a, b in groups:
            w = _dequantised(s["wq"][e], s["ws"][e].repeat_interleave(BLOCK, 0)[:N].repeat_interleave(BLOCK, 1))
            y[a:b] = x[a:b] @ w.T
        return y
    x = s["x"].float()
    x = x[s["row_token"].long()] if c["gather"] else x
    if op == "grouped":
        y = x.new_empty((x.shape[0], N), dtype=out)
        for e, a, b in groups:
            y[a:b] = x[a:b] @ s["w"][e].float().T
        return y
    dy = s["dy"].float()
    dx = x.new_empty((x.shape[0], K))
    dw = x.new_zeros((c["n"], N, K), dtype=out)
    for e, a, b in groups:
        dx[a:b] = dy[a:b] @ s["w"][e].float()
        dw[e] = dy[a:b].T @ x[a:b]
    if c["gather"]:
        dx = dx[s["row_of"].long()].sum(1)
    return dx.to(s["x"].dtype), dw


def _dequantised(q, scale):
    return q.float() * scale[:, :q.shape[1]]


def _to_e4m3(blocks, most):
    """Values of blocks scaled so that `most`, their largest magnitude, becomes 448, and the scales."""
    most = most.clamp_min(FLOOR)
    # (a number over a tensor would be its rounded reciprocal times the number)
    return (blocks * (torch.full_like(most, E4M3_MAX) / most)).to(torch.float8_e4m3fn), most / E4M3_MAX


def _padded(x, rows, cols):
    return torch.nn.functional.pad(x, (0, -x.shape[-1] % cols, 0, -x.shape[-2] % rows))


def _quant_rows(x):
    R, K = x.shape
    b = _padded(x, 1, BLOCK).reshape(R, -1, BLOCK)
    q, scale = _to_e4m3(b, b.abs().amax(2, keepdim=True))
    return q.reshape(R, -1)[:, :K].contiguous(), scale[:, :, 0].contiguous()


def _quant_blocks(w, transpose):
    n, N, K = w.shape
    b = _padded(w, BLOCK, BLOCK)
    b = b.reshape(n, b.shape[1] // BLOCK, BLOCK, b.shape[2] // BLOCK, BLOCK)
    q, scale = _to_e4m3(b, b.abs().amax((2, 4), keepdim=True))
    q = q.reshape(n, b.shape[1] * BLOCK, -1)[:, :N, :K].contiguous()
    scale = scale[:, :, 0, :, 0].contiguous()
    return (q, scale, q.transpose(1, 2).contiguous(), scale.transpose(1, 2).contiguous()) if transpose else (q, scale)


# ------------------------------------------------------------------------ what a pass cannot do without
def work(case):
    op = case["op"]
    if op in ("quant", "swiglu_quant", "quant_weights"):
        size = 2 if case["dtype"] == "bf16" else 4
        if op == "quant_weights":
            count, times = case["n"] * case["N"] * case["K"], 2 if case["transpose"] else 1
            blocks = case["n"] * -(-case["N"] // BLOCK) * -(-case["K"] // BLOCK)
            return {"bytes": count * (size + times) + 4 * blocks * times, "flops": 2 * count}
        count = case["R"] * case["K"]
        wide = 2 if op == "swiglu_quant" else 1
        return {"bytes": count * (size * wide + 1) + 4 * case["R"] * -(-case["K"] // BLOCK), "flops": count * (6 if wide == 2 else 2)}
    T, k, n, K, N = (case[v] for v in ("T", "k", "n", "K", "N"))
    R = T * k
    touched = n * (1.0 - (1.0 - k / n) ** T)   # experts that have a row, as expected of even routing
    size = 1 if op == "fp8" else 2 if case["dtype"] == "bf16" else 4
    out = 2 if case["out"] == "bf16" else 4
    rows_in = T if case["gather"] else R
    if op != "grads":
        scales = 4 * (rows_in * -(-K // BLOCK) + touched * -(-K // BLOCK) * -(-N // BLOCK)) if op == "fp8" else 0
        return {"bytes": int(size * (rows_in * K + touched * N * K) + out * R * N + scales), "flops": 2 * R * K * N}
    return {"bytes": int(size * (2 * rows_in * K + R * N + touched * N * K) + out * n * N * K), "flops": 4 * R * K * N}


# ------------------------------------------------------------------------ 64 bits
def _rounded64(v):
    """v (magnitudes up to 448) to the nearest e4m3 value, ties to even: steps of 2^(e-3), at least 2^-9."""
    e = torch.frexp(v).exponent - 1
    step = torch.exp2(e.clamp_min(-6).double() - 3)
    return torch.round(v / step) * step


def _rows64(x):
    q, scale = torch.empty_like(x), x.new_empty((x.shape[0], -(-x.shape[1] // BLOCK)))
    for j in range(scale.shape[1]):
        part = x[:, j * BLOCK:(j + 1) * BLOCK]
        top = torch.maximum(part.abs().max(1).values, x.new_tensor(FLOOR))
        q[:, j * BLOCK:(j + 1) * BLOCK] = _rounded64(part * (E4M3_MAX / top)[:, None])
        scale[:, j] = top / E4M3_MAX
    return q, scale


def _weights64(w, transpose):
    n, N, K = w.shape
    q, scale = torch.empty_like(w), w.new_empty((n, -(-N // BLOCK), -(-K // BLOCK)))
    for i in range(scale.shape[1]):
        for j in range(scale.shape[2]):
            at = (slice(None), slice(i * BLOCK, (i + 1) * BLOCK), slice(j * BLOCK, (j + 1) * BLOCK))
            top = w[at].abs().amax((1, 2)).clamp_min(FLOOR)
            q[at] = _rounded64(w[at] * (E4M3_MAX / top)[:, None, None])
            scale[:, i, j] = top / E4M3_MAX
    return (q, scale, q.mT, scale.mT) if transpose else (q, scale)


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "quant":
        return _rows64(s["x"].double())
    if op == "swiglu_quant":
        v = s["x"].double()
        gate, up = v[:, :case["K"]], v[:, case["K"]:]
        return _rows64(gate * torch.sigmoid(gate) * up)
    if op == "quant_weights":
        return _weights64(s["w"].double(), case["transpose"])
    T, k, n, K, N = (case[v] for v in ("T", "k", "n", "K", "N"))
    of_group = torch.bucketize(torch.arange(T * k, device=DEV), s["offsets"][1:].long(), right=True)
    source = s["row_token"].long() if case["gather"] else torch.arange(T * k, device=DEV)
    at = torch.arange(max(K, N), device=DEV) // BLOCK   # the block of each column
    if op == "fp8":
        x = s["xq"].double() * s["xs"].double()[:, at[:K]]
    else:
        x = s["x"].double()
    y = x.new_empty((T * k, N)) if op != "grads" else None
    dx = x.new_zeros(x.shape) if op == "grads" else None
    dw = x.new_zeros((n, N, K)) if op == "grads" else None
    for e in range(n):
        rows = (of_group == e).nonzero()[:, 0]
        if not len(rows):
            continue
        if op == "fp8":
            w = s["wq"][e].double() * s["ws"][e].double()[at[:N]][:, at[:K]]
        else:
            w = s["w"][e].double()
        if op != "grads":
            y[rows] = torch.matmul(x[source[rows]], w.mT)
            continue
        dy = s["dy"][rows].double()
        dx.index_add_(0, source[rows], dy.matmul(w))
        torch.matmul(dy.mT, x[source[rows]], out=dw[e])
    return y if op != "grads" else (dx, dw)
