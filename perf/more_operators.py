"""The steps of a layer's training around the experts' products, as cases to measure.

Five operators, each with its gradient where it has one: tokens to their experts' rows and back with
weights applied (dispatch, dispatch_grad, combine, combine_grad), SwiGLU between the products (swiglu,
swiglu_grad), the mix along a token's paths (mix, mix_grad), the router's gradient from those of the
weights (route_grad), and the norm over all gradients with clipping (norm, clip). listed() names the
cases, draw() gives more of the same ranges, prepare() makes what a program holds before the call, run()
is one call: in plain torch (32 bits, rounded once), or, where `own` is true, through the framework.
exact() is the same result in 64 bits.

Layer shapes are those of workloads/configs.py (Mixtral-, OLMoE-, fine-grained- and decode-shaped, and
the float32 one) with their routing, generic ones beside them. Rows are (token, slot) pairs ordered by
expert, then token, as the framework's path tables order them."""
import math
import random

import torch

own = False

DEV = "cuda"


def listed():
    return [
        # a prompt's hidden states copied to the rows of their experts, before an exchange or an 8-bit product
        dict(name="rows, prefill 8192", op="dispatch", T=8192, k=8, n=64, held=64, H=2048, dtype="bf16", out="bf16",
             weights=False, logits="zipf"),
        # the experts' outputs of one decode step back to their tokens, on a rank that holds half of the experts
        dict(name="rows back, decode 32", op="combine", T=32, k=8, n=256, held=128, H=7168, dtype="bf16", out="f32",
             weights=True, logits="normal"),
        # training step: gradients of the experts' outputs and of their weights
        dict(name="rows back gradient, fine-grained", op="combine_grad", T=16384, k=4, n=60, held=60, H=2048, dtype="bf16",
             out="bf16", weights=True, logits="normal"),
        # the float32 layer of the tests and the benchmark
        dict(name="SwiGLU, f32 small", op="swiglu", R=128, F=512, dtype="f32", out="f32"),
        # training step of fine-grained experts
        dict(name="SwiGLU gradient, fine-grained", op="swiglu_grad", R=65536, F=1408, dtype="bf16", out="bf16"),
        # forward step of few large experts, half of the paths allowed
        dict(name="mix, few experts", op="mix", T=4096, k=2, n=8, F=14336, dtype="bf16", out="bf16", density=0.5, beta=0,
             logits="normal_bias"),
        # one token's mix after the expansion, which leaves its rows in float32
        dict(name="mix, one token", op="mix", T=1, k=8, n=256, F=2048, dtype="f32", out="bf16", density=0.2, beta=0,
             logits="normal"),
        # training step of many small experts: gradients of the sources' rows and of the path weights
        dict(name="mix gradient, top-8", op="mix_grad", T=8192, k=8, n=64, F=1024, dtype="bf16", out="bf16", density=0.25,
             beta=0, logits="zipf"),
        # the router of the float32 layer
        dict(name="router gradient, small", op="route_grad", T=64, k=2, n=8, density=0.5, beta=0, paths=True, direct=False,
             out="f32", logits="normal"),
        # the router of a fine-grained layer, path weights and a token's own weights
        dict(name="router gradient, fine-grained", op="route_grad", T=16384, k=4, n=60, density=0.3, beta=0, paths=True,
             direct=True, out="f32", logits="normal"),
        # all gradients of a model with many small tensors, views of one buffer for each type
        dict(name="clip, 300 views", op="clip", count=300, most=1 << 20, spread=11, dtype="mixed", out="same", flat=True,
             max_norm=1.0),
        # the gradients of a layer of few large experts
        dict(name="clip, few experts", op="clip", layers=1, n=8, H=4096, F=14336, dtype="bf16", out="same", flat=False,
             max_norm=1.0),
    ]


def _spread(rng, lo, hi):
    """An integer of [lo, hi], uniform over its logarithm."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["dispatch", "dispatch_grad", "combine", "combine_grad", "swiglu", "swiglu_grad", "mix", "mix_grad",
                     "mix_grad", "route_grad", "norm", "clip", "clip"])
    dtype, out = rng.choice([("bf16", "bf16"), ("bf16", "bf16"), ("bf16", "f32"), ("f32", "f32"), ("f32", "bf16")])
    logits = rng.choice(["normal", "zipf"])
    if op in ("swiglu", "swiglu_grad"):
        F, R = 16 * _spread(rng, 1, 896), _spread(rng, 1, 65536)
        return dict(op=op, R=min(R, 90_000_000 // F), F=F, dtype=dtype, out=out)
    if op in ("norm", "clip"):
        return dict(op=op, count=_spread(rng, 1, 500), most=_spread(rng, 64, 1 << 22), spread=rng.randint(0, 999),
                    dtype=rng.choice(["bf16", "f32", "mixed"]), out=rng.choice(["same", "f32"]), flat=True,
                    max_norm=rng.choice([0.5, 1.0, 1e4]))
    n = _spread(rng, 1, 256)
    k = rng.randint(1, min(n, 8))
    T = _spread(rng, 1, 16384)
    if op == "route_grad":
        paths = rng.choice([True, True, False])
        return dict(op=op, T=T, k=k, n=n, density=rng.choice([0.0, 0.25, 0.5, 1.0]), beta=rng.randint(0, 2), paths=paths,
                    direct=not paths or rng.choice([True, False]), out=rng.choice(["f32", "bf16"]), logits=logits)
    width = 16 * _spread(rng, 4, 448)
    T = max(1, min(T, 100_000_000 // (k * width)))
    if op in ("mix", "mix_grad"):
        return dict(op=op, T=T, k=k, n=n, F=width, dtype=dtype, out=out, density=rng.choice([0.0, 0.25, 0.5, 1.0]),
                    beta=rng.randint(0, 2), logits=logits)
    return dict(op=op, T=T, k=k, n=n, held=rng.choice([n, max(1, n // 2)]), H=width, dtype=dtype, out=out,
                weights=rng.choice([True, True, False]), logits=logits)


# ------------------------------------------------------------------------ inputs
def _randn(g, shape, std, dtype):
    return torch.randn(shape, generator=g, device=DEV, dtype=dtype).mul_(std)


def _type(name):
    return {"bf16": torch.bfloat16, "f32": torch.float32}[name]


def _routing(case, g):
    """T tokens with k of n experts each: their ids and weights [T, k], and the rows' offsets [n+1], row_token [T*k],
    row_slot [T*k] and row_of [T, k]."""
    T, n, k = case["T"], case["n"], case["k"]
    logits = torch.randn((T, n), generator=g, device=DEV)
    if case["logits"] == "normal_bias":
        logits += 0.5 * torch.randn((n,), generator=g, device=DEV)
    if case["logits"] == "zipf":
        logits -= 1.1 * torch.log((torch.randperm(n, generator=g, device=DEV) + 1).float())
    top, ids = logits.topk(k, dim=1)
    order = ids.reshape(-1).sort(stable=True).indices
    row_of = torch.empty_like(order)
    row_of[order] = torch.arange(T * k, device=DEV)
    counts = torch.bincount(ids.reshape(-1), minlength=n)
    offsets = torch.cat([counts.new_zeros(1), counts.cumsum(0)])
    return dict(ids=ids.int(), p=top.softmax(1), offsets=offsets.int(), row_token=(order // k).int(),
                row_slot=(order % k).int(), row_of=row_of.reshape(T, k).int())


def _paths(case, g, ids, p):
    """path_bits [T] and beta [T, k, k] of a mask of the case's density (paths from an expert to itself always)."""
    T, n, k = case["T"], case["n"], case["k"]
    mask = torch.rand((n, n), generator=g, device=DEV) < case["density"]
    mask.fill_diagonal_(True)
    on = mask[ids.long()[:, :, None], ids.long()[:, None, :]]
    bits = (on.reshape(T, -1).long() << torch.arange(k * k, device=DEV)).sum(1)
    beta = p[:, :, None] * p[:, None, :] * on
    if case["beta"] == 0:
        beta = beta / (on * p[:, None, :]).sum(2, keepdim=True)
    if case["beta"] == 2:
        beta = beta / beta.sum((1, 2), keepdim=True)
    return dict(bits=bits, beta=beta.contiguous())


def _tensors(case):
    """(elements, type) of each gradient of a norm or clip case."""
    types = {"mixed": [torch.bfloat16, torch.bfloat16, torch.float32]}.get(case["dtype"]) or [_type(case["dtype"])]
    if "layers" in case:
        n, H, F = case["n"], case["H"], case["F"]
        return [(size, types[0]) for _ in range(case["layers"]) for size in (n * H, n * F * H, n * F * H, n * H * F, H)]
    rng = random.Random(case["spread"])
    return [(_spread(rng, 1, case["most"]), types[rng.randrange(len(types))]) for _ in range(case["count"])]


def _flat(spec, types):
    """One buffer for each type in `types` (those of spec's tensors), and spec's tensors as its consecutive views."""
    size, views = {}, []
    for (count, _), dt in zip(spec, types):
        views.append((dt, size.get(dt, 0), count))
        size[dt] = size.get(dt, 0) + count
    buffers = {dt: torch.zeros(total, dtype=dt, device=DEV) for dt, total in size.items()}
    return buffers, [buffers[dt][at:at + count] for dt, at, count in views]


def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    op, s = case["op"], {"case": case}
    if op in ("norm", "clip"):
        spec = _tensors(case)
        here, there = [t for _, t in spec], [torch.float32 if case["out"] == "f32" else t for _, t in spec]
        if case["flat"]:
            buffers, s["grads"] = _flat(spec, here)
            for b in buffers.values():
                b.copy_(_randn(g, b.shape, 1e-3, b.dtype))
            outs, s["outs"] = _flat(spec, there)
            s["whole"] = list(outs.values())
        else:
            s["grads"] = [_randn(g, (count,), 1e-3, t) for count, t in spec]
            s["outs"] = s["whole"] = [torch.zeros(count, dtype=t, device=DEV) for (count, _), t in zip(spec, there)]
        return s
    if op in ("swiglu", "swiglu_grad"):
        s["gate_up"] = _randn(g, (case["R"], 2 * case["F"]), 1.0, _type(case["dtype"]))
        if op == "swiglu_grad":
            s["du"] = _randn(g, (case["R"], case["F"]), 1.0, _type(case["dtype"]))
        return s
    s.update(_routing(case, g))
    T, k = case["T"], case["k"]
    if op == "route_grad":
        if case["paths"]:
            s.update(_paths(case, g, s["ids"], s["p"]))
            s["dbeta"] = _randn(g, (T, k, k), 1.0, torch.float32)
        if case["direct"]:
            s["dw"] = _randn(g, (T, k), 1.0, torch.float32)
        return s
    dt = _type(case["dtype"])
    if op in ("mix", "mix_grad"):
        s.update(_paths(case, g, s["ids"], s["p"]))
        s["u"] = _randn(g, (T * k, case["F"]), 1.0, dt)
        if op == "mix_grad":
            s["dz"] = _randn(g, (T * k, case["F"]), 1.0, dt)
        return s
    # a rank that holds some of the experts has the offsets of those; the rows of others are not its own
    s["offsets"] = s["offsets"][:case["held"] + 1].contiguous()
    of_tokens, of_rows = (T, case["H"]), (T * k, case["H"])
    s["weights"] = s["p"] if case["weights"] else None
    if op in ("dispatch", "dispatch_grad", "combine_grad"):
        s["tokens"] = _randn(g, of_tokens, 1.0, dt)
    if op != "dispatch":
        s["rows"] = _randn(g, of_rows, 1.0, dt)
    if op in ("dispatch", "combine_grad"):   # rows that are not written keep what the program had in them
        s["to_rows"] = torch.zeros(of_rows, dtype=_type(case["out"]), device=DEV)
    return s


# ------------------------------------------------------------------------ one call
def run(s):
    return _own(s) if own else _plain(s)


def _own(s):
    import paper_2609_01024_amd as pcm
    c = s["case"]
    op = c["op"]
    if op == "norm":
        return pcm.pcm_grad_norm(s["grads"])
    if op == "clip":
        return pcm.pcm_clip_grad_norm(s["grads"], c["max_norm"], out=s["outs"]), s["whole"]
    out = _type(c["out"])
    if op == "swiglu":
        return pcm.pcm_swiglu(s["gate_up"], out_dtype=out)
    if op == "swiglu_grad":
        return pcm.pcm_swiglu_grad(s["gate_up"], s["du"], out_dtype=out)
    if op == "mix":
        return pcm.pcm_mix_rows(s["u"], s["bits"], s["beta"], s["row_of"], out_dtype=out)
    if op == "mix_grad":
        return pcm.pcm_mix_rows_grad(s["dz"], s["u"], s["bits"], s["beta"], s["row_of"], out_dtype=out)
    if op == "route_grad":
        return pcm.pcm_route_grad(s["ids"], s["p"], c["n"], path_bits=s.get("bits"), dbeta=s.get("dbeta"), dw=s.get("dw"),
                                  beta_mode=c["beta"], out_dtype=out)
    if op == "dispatch":
        return pcm.pcm_dispatch_rows(s["tokens"], s["row_of"], weights=s["weights"], offsets=s["offsets"], y=s["to_rows"])
    if op == "dispatch_grad":
        return pcm.pcm_dispatch_rows_grad(s["rows"], s["row_of"], x=s["tokens"], weights=s["weights"], offsets=s["offsets"],
                                          out_dtype=out)
    if op == "combine":
        return pcm.pcm_combine_rows(s["rows"], s["row_of"], weights=s["weights"], offsets=s["offsets"], out_dtype=out)
    return pcm.pcm_combine_rows_grad(s["tokens"], s["row_of"], o=s["rows"], weights=s["weights"], offsets=s["offsets"],
                                     do=s["to_rows"])


def _plain(s):
    c = s["case"]
    op = c["op"]
    if op in ("norm", "clip"):
        norm = torch.stack([g.float().square().sum(dtype=torch.float64) for g in s["grads"]]).sum().sqrt().float().reshape(1)
        if op == "norm":
            return norm
        factor = torch.where(norm > c["max_norm"], c["max_norm"] / norm, 1.0)
        for g, o in zip(s["grads"], s["outs"]):
            o.copy_(g.float() * factor)
        return norm, s["whole"]
    out = _type(c["out"])
    if op == "swiglu":
        gate, up = s["gate_up"].float().chunk(2, dim=1)
        return (gate / (1.0 + torch.exp(-gate)) * up).to(out)
    if op == "swiglu_grad":
        gate, up = s["gate_up"].float().chunk(2, dim=1)
        du, sig = s["du"].float(), 1.0 / (1.0 + torch.exp(-gate))
        return torch.cat([du * up * sig * (1.0 + gate * (1.0 - sig)), du * gate * sig], dim=1).to(out)
    if op == "route_grad":
        return _plain_route_grad(s).to(out)
    row_of = s["row_of"].long()
    if op in ("mix", "mix_grad"):
        on = (s["bits"][:, None] >> torch.arange(c["k"] ** 2, device=DEV) & 1).bool().reshape(s["beta"].shape)
        beta = torch.where(on, s["beta"], 0.0)
        u = s["u"].float()[row_of]                                       # [T, k, F]
        if op == "mix":
            z = torch.empty_like(s["u"], dtype=out)
            z[row_of] = (beta.transpose(1, 2).contiguous() @ u).to(out)
            return z
        dz = s["dz"].float()[row_of]
        du = torch.empty_like(s["u"], dtype=out)
        du[row_of] = (beta @ dz).to(out)
        return du, torch.where(on, u @ dz.transpose(1, 2).contiguous(), 0.0)
    here = (row_of >= s["offsets"][0]) & (row_of < s["offsets"][-1])
    w = (here if s["weights"] is None else torch.where(here, s["weights"], 0.0)).float()
    if op == "dispatch":
        at = s["row_token"].long()
        x = s["tokens"].float()[at]
        x = x if s["weights"] is None else x * s["weights"][at, s["row_slot"].long()][:, None]
        return torch.where(_held(s), x.to(out), s["to_rows"])
    if op == "combine":
        return (s["rows"].float()[row_of] * w[:, :, None]).sum(1).to(out)
    rows, tokens = s["rows"].float()[row_of], s["tokens"].float()
    dw = torch.where(here, (rows * tokens[:, None, :]).sum(2), 0.0)
    if op == "dispatch_grad":
        return (rows * w[:, :, None]).sum(1).to(out), dw
    do = tokens[s["row_token"].long()]
    do = do if s["weights"] is None else do * s["weights"][s["row_token"].long(), s["row_slot"].long()][:, None]
    return torch.where(_held(s), do.to(out), s["to_rows"]), dw


def _held(s):
    r = torch.arange(s["row_token"].shape[0], device=DEV)
    return ((r >= s["offsets"][0]) & (r < s["offsets"][-1]))[:, None]


def _plain_route_grad(s):
    c, p = s["case"], s["p"]
    dp = torch.zeros_like(p) if s.get("dw") is None else s["dw"]
    if c["paths"]:
        on = (s["bits"][:, None] >> torch.arange(c["k"] ** 2, device=DEV) & 1).bool().reshape(s["beta"].shape)
        d = torch.where(on, s["dbeta"], 0.0)
        source, target = p[:, :, None], p[:, None, :]
        if c["beta"] == 0:       # beta_ab = p_a p_b / S_a, S_a the sum of p over a's targets
            share = torch.where(on, target, 0.0) / torch.where(on, target, 0.0).sum(2, keepdim=True)
            mean = (d * share).sum(2)
            factor = p / torch.where(on, target, 0.0).sum(2)
            dp = dp + mean + torch.where(on, factor[:, :, None] * (d - mean[:, :, None]), 0.0).sum(1)
        else:
            if c["beta"] == 2:   # over all paths
                pairs = torch.where(on, source * target, 0.0)
                total = pairs.sum((1, 2), keepdim=True)
                d = torch.where(on, d - (d * pairs).sum((1, 2), keepdim=True) / total, 0.0) / total
            dp = dp + (d * target).sum(2) + (d * source).sum(1)
    dl = p * (dp - (p * dp).sum(1, keepdim=True))
    return torch.zeros((c["T"], c["n"]), device=DEV).scatter_(1, s["ids"].long(), dl)


# ------------------------------------------------------------------------ what a pass cannot do without
def work(case):
    op = case["op"]
    size = {"bf16": 2, "f32": 4}
    if op in ("norm", "clip"):
        read = write = total = 0
        for count, t in _tensors(case):
            read += count * (2 if t == torch.bfloat16 else 4)
            write += count * (4 if case["out"] == "f32" or t == torch.float32 else 2)
            total += count
        return {"bytes": read + (write if op == "clip" else 0), "flops": total * (3 if op == "clip" else 2)}
    out = size[case["out"]]
    if op in ("swiglu", "swiglu_grad"):
        count, b = case["R"] * case["F"], size[case["dtype"]]
        return {"bytes": count * (2 * b + out if op == "swiglu" else 3 * b + 2 * out), "flops": count * (5 if op == "swiglu" else 12)}
    T, k, n = case["T"], case["k"], case["n"]
    if op == "route_grad":
        inputs = T * k * 8 + (T * (8 + 4 * k * k) if case["paths"] else 0) + (T * k * 4 if case["direct"] else 0)
        return {"bytes": inputs + T * n * out, "flops": T * (6 * k * k + 5 * k)}
    b = size[case["dtype"]]
    if op in ("mix", "mix_grad"):
        count, tables = T * k * case["F"], T * (8 + 4 * k * k + 4 * k)
        paths = k + case["density"] * k * (k - 1)   # of a token, as expected
        if op == "mix":
            return {"bytes": count * (b + out) + tables, "flops": int(2 * T * paths * case["F"])}
        return {"bytes": count * (2 * b + out) + tables + 4 * T * k * k, "flops": int(4 * T * paths * case["F"])}
    H, R = case["H"], T * k * case["held"] // n    # rows of the held experts, as expected of even routing
    tables = T * k * (8 if case["weights"] else 4)
    if op == "dispatch":
        return {"bytes": T * H * b + R * H * out + tables, "flops": R * H if case["weights"] else 0}
    if op == "combine":
        return {"bytes": R * H * b + T * H * out + tables, "flops": 2 * R * H}
    if op == "dispatch_grad":
        return {"bytes": (R + T) * H * b + T * H * out + tables + 4 * T * k, "flops": 4 * R * H}
    return {"bytes": (R + T) * H * b + R * H * out + tables + 4 * T * k, "flops": 3 * R * H}


# ------------------------------------------------------------------------ 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op in ("norm", "clip"):
        total = torch.zeros(1, dtype=torch.float64, device=DEV)
        for g in s["grads"]:
            total += torch.linalg.vector_norm(g, dtype=torch.float64) ** 2
        norm = total.sqrt()
        if op == "norm":
            return norm
        scale = min(1.0, case["max_norm"] / float(norm))
        if not case["flat"]:
            return norm, [g.double() * scale for g in s["grads"]]
        # the buffers, in the order in which their types come
        whole = [[] for _ in s["whole"]]
        for g, o in zip(s["grads"], s["outs"]):
            whole[[w.dtype for w in s["whole"]].index(o.dtype)].append(g.double() * scale)
        return norm, [torch.cat(parts) for parts in whole]
    if op in ("swiglu", "swiglu_grad"):
        F = case["F"]
        gate, up = s["gate_up"][:, :F].double(), s["gate_up"][:, F:].double()
        silu = torch.nn.functional.silu(gate)
        if op == "swiglu":
            return silu.mul_(up)
        du = s["du"].double()
        sig = torch.sigmoid(gate)
        slope = sig + silu * torch.sigmoid(-gate)
        d = torch.empty(s["gate_up"].shape, dtype=torch.float64, device=DEV)
        d[:, :F] = slope * up * du
        d[:, F:] = silu * du
        return d
    if op == "route_grad":
        return _exact_route_grad(s)
    T, k = case["T"], case["k"]
    if op in ("mix", "mix_grad"):
        rows = [s["row_of"][:, a].long() for a in range(k)]
        back = torch.zeros(s["u"].shape, dtype=torch.float64, device=DEV)
        dbeta = torch.zeros((T, k, k), dtype=torch.float64, device=DEV)
        for a in range(k):
            u = s["u"][rows[a]].double()
            for b in range(k):
                t = ((s["bits"] >> (a * k + b)) & 1).nonzero()[:, 0]   # the tokens that have this path
                w = s["beta"][t, a, b].double()[:, None]
                if op == "mix":
                    back[rows[b][t]] += w * u[t]
                else:
                    dz = s["dz"][rows[b][t]].double()
                    back[rows[a][t]] += w * dz
                    dbeta[t, a, b] = (dz * u[t]).sum(1)
        return back if op == "mix" else (back, dbeta)
    first, end = int(s["offsets"][0]), int(s["offsets"][-1])
    at, slot = s["row_token"].long()[first:end], s["row_slot"].long()[first:end]
    w = torch.ones(end - first, 1, dtype=torch.float64, device=DEV) if s["weights"] is None else s["weights"].double()[at, slot][:, None]
    if op == "dispatch" or op == "combine_grad":
        y = torch.zeros(s["to_rows"].shape, dtype=torch.float64, device=DEV)
        y[first:end] = s["tokens"].double()[at] * w
        if op == "dispatch":
            return y
    if op != "combine_grad":
        back = torch.zeros((T, case["H"]), dtype=torch.float64, device=DEV)
        back.index_add_(0, at, s["rows"][first:end].double() * w)
        if op == "combine":
            return back
        y = back
    dw = torch.zeros((T, k), dtype=torch.float64, device=DEV)
    dw[at, slot] = (s["rows"][first:end].double() * s["tokens"].double()[at]).sum(1)
    return y, dw


def _exact_route_grad(s):
    """By a token's logits of its k experts: the weights as functions of them, differentiated by torch in 64 bits. The
    weights that the calls were given are rounded to 32, so the derivative is taken at those: dl = J(p) dp."""
    c = s["case"]
    T, k = c["T"], c["k"]
    p = s["p"].double().requires_grad_()
    loss = torch.zeros((), dtype=torch.float64, device=DEV)
    if c["direct"]:
        loss = loss + (p * s["dw"]).sum()
    if c["paths"]:
        terms = {}
        for a in range(k):
            for b in range(k):
                terms[a, b] = ((s["bits"] >> (a * k + b)) & 1).double()
        total = sum(on * p[:, a] * p[:, b] for (a, b), on in terms.items())
        for a in range(k):
            reach = sum(terms[a, b] * p[:, b] for b in range(k))
            for b in range(k):
                beta = terms[a, b] * p[:, a] * p[:, b] / {0: reach, 1: 1.0, 2: total}[c["beta"]]
                loss = loss + (beta * s["dbeta"][:, a, b]).sum()
    dp, = torch.autograd.grad(loss, p)
    p = p.detach()
    dlogits = torch.zeros((T, c["n"]), dtype=torch.float64, device=DEV)
    rows = torch.arange(T, device=DEV)
    for a in range(k):
        own_part = p[:, a] * dp[:, a]
        for b in range(k):
            own_part = own_part - p[:, a] * p[:, b] * dp[:, b]
        dlogits[rows, s["ids"][:, a].long()] = own_part
    return dlogits
