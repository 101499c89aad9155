"""Products of a processed layer, as calls of the HARP library's public entry points.

A processed weight W~ = Q_out^T W Q_in is kept in 8 bits with one scale per output channel, and the
rows that a processor hands to it are quantised token by token.  Three operators make up that path,
and the training counterpart of the last one:

* rows to 8 bits with one scale per row (`harp.quantize_rows`): activations between a processor and
  the product, and the rows of a weight ahead of deployment;
* the 8-bit product with scales per token and channel (`harp.linear_i8`);
* products grouped by expert with ragged numbers of rows, in 8 bits (`harp.grouped_linear_i8`) and
  in bf16 (`harp.grouped_linear`), with the gradients of the bf16 form
  (`harp.grouped_grad_rows`, `harp.grouped_grad_weights`).

Widths are those of the benchmark configurations and of the greedy schedules.  Where `own` is false
the operators run in their plain form: elementary torch operations in 32 bits (the quotient that is
rounded to 8 bits in 64, since values next to half a step would fall to the other side).
"""
import math
import random

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
WIDTHS = (2048, 4096, 5120, 8192, 11008, 14336, 28672)
MAX_PRODUCT = 16384 * 4096 * 14336      # multiplications of the largest product
MAX_ELEMENTS = 64 * 4096 * 2048         # entries of the largest weight
MAX_QUANTISED = 16384 * 4096            # entries of the largest quantised batch


def quantise_case(rows, d, dtype, name=None):
    case = {"op": "quantise", "rows": rows, "d": d, "dtype": dtype}
    return {"name": name, **case} if name else case


def product_case(rows, d_in, d_out, out, name=None):
    case = {"op": "product", "rows": rows, "d_in": d_in, "d_out": d_out, "out": out}
    return {"name": name, **case} if name else case


def grouped_case(op, rows, groups, d_in, d_out, out, split, skew, name=None):
    """`split` and `skew` fix how the rows fall on the groups: see group_sizes."""
    case = {"op": op, "rows": rows, "groups": groups, "d_in": d_in, "d_out": d_out, "out": out, "split": split, "skew": skew}
    return {"name": name, **case} if name else case


def listed():
    return [
        # one token in front of a wide layer: latency
        quantise_case(1, 14336, "bf16", "quantise 1 row d14336"),
        # a prefill batch behind its processor
        quantise_case(16384, 4096, "bf16", "quantise prefill d4096"),
        # a weight kept in fp32, channel by channel, an odd number of them
        quantise_case(4099, 11008, "f32", "quantise fp32 d11008"),
        # one token of a decode step
        product_case(1, 4096, 14336, "bf16", "i8 1 row 4096-14336"),
        # a decode batch of sixteen sequences, into fp32 for the processor behind it
        product_case(16, 14336, 4096, "f32", "i8 16 rows 14336-4096"),
        # an ordinary batch of a ragged number of tokens
        product_case(2051, 11008, 4096, "bf16", "i8 ragged 11008-4096"),
        # a long prefill
        product_case(16384, 4096, 14336, "bf16", "i8 prefill 4096-14336"),
        # a decode batch of sixteen tokens, two experts each
        grouped_case("grouped", 32, 8, 4096, 14336, "bf16", 1, 0.5, "grouped decode 8 experts"),
        # a ragged training or prefill batch over a few wide experts, one of them without a token
        grouped_case("grouped", 8195, 8, 4096, 14336, "bf16", 2, 1.0, "grouped ragged 8 experts"),
        # many experts with few rows each, in 8 bits
        grouped_case("grouped_i8", 4100, 64, 4096, 2048, "bf16", 3, 1.0, "grouped i8 64 experts"),
        # the backward pass of the few wide experts
        grouped_case("grouped_grads", 8195, 8, 4096, 14336, "f32", 2, 1.0, "grouped gradients 8 experts"),
        # the backward pass of many narrow experts, about thirty rows each, weights' gradients in bf16
        grouped_case("grouped_grads", 1001, 32, 2048, 4096, "bf16", 4, 1.0, "grouped gradients 32 experts"),
    ]


def log_uniform(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))))))


def width(rng):
    """A configuration's width mostly; now and then any other one, odd ones among them."""
    return rng.choice(WIDTHS) if rng.random() < 0.75 else log_uniform(rng, 256, 14336)


def draw(rng):
    kind = rng.random()
    if kind < 0.25:
        d = width(rng)
        return quantise_case(log_uniform(rng, 1, MAX_QUANTISED // d), d, rng.choice(("bf16", "bf16", "f32")))
    if kind < 0.6:
        d_in, d_out = width(rng), width(rng)
        return product_case(log_uniform(rng, 1, min(16384, MAX_PRODUCT // (d_in * d_out))), d_in, d_out, rng.choice(("bf16", "bf16", "f32")))
    op = rng.choice(("grouped", "grouped_i8", "grouped_grads"))
    d_in, d_out = width(rng), width(rng)
    groups = log_uniform(rng, 1, max(1, min(64, MAX_ELEMENTS // (d_in * d_out))))
    most = min(16384, MAX_PRODUCT // (d_in * d_out * (2 if op == "grouped_grads" else 1)))
    return grouped_case(op, log_uniform(rng, 1, most), groups, d_in, d_out, rng.choice(("bf16", "bf16", "f32")),
                        rng.randrange(1 << 30), rng.choice((0.0, 0.5, 1.0)))


def group_sizes(case):
    """Rows of each group: every row takes a group with weights exp(skew * normal); with a skew of 1 the
    second group has none.  Groups are met in order, as after a sort of the tokens by expert."""
    r = random.Random(case["split"])
    weights = [math.exp(case["skew"] * r.gauss(0, 1)) for _ in range(case["groups"])]
    if case["skew"] == 1.0 and case["groups"] > 1:
        weights[1] = 0.0
    sizes = [0] * case["groups"]
    for e in r.choices(range(case["groups"]), weights, k=case["rows"]):
        sizes[e] += 1
    return sizes


def activations(gen, rows, d, dtype):
    """Normal rows with a fixed set of outlier channels (0.5 %, x50)."""
    gain = torch.ones(d, device="cuda")
    gain[torch.randperm(d, generator=gen, device="cuda")[: max(1, d // 200)]] = 50.0
    return (torch.randn((rows, d), generator=gen, device="cuda") * gain).to(dtype)


def weights(gen, groups, d_out, d_in):
    w = torch.empty((groups, d_out, d_in), dtype=torch.bfloat16, device="cuda")
    for e in range(groups):
        w[e] = torch.randn((d_out, d_in), generator=gen, device="cuda") * 0.02
    return w


def to_8_bits(x):
    """Rows in 8 bits and their scales, for inputs that a program holds in that form already."""
    most = x.abs().amax(-1, keepdim=True).float().clamp_min(1e-30)
    return (x.float() * (127.0 / most)).round_().to(torch.int8), (most / 127.0).squeeze(-1)


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    s = {"op": case["op"]}
    if case["op"] == "quantise":
        s["x"] = activations(gen, case["rows"], case["d"], DTYPES[case["dtype"]])
        s["q"] = torch.empty(s["x"].shape, dtype=torch.int8, device="cuda")
        s["scale"] = torch.empty(case["rows"], device="cuda")
        return s
    rows, d_in, d_out, out = case["rows"], case["d_in"], case["d_out"], DTYPES[case["out"]]
    x = activations(gen, rows, d_in, torch.bfloat16)
    w = weights(gen, case.get("groups", 1), d_out, d_in)
    s["y"] = torch.empty((rows, d_out), dtype=torch.bfloat16 if case["op"] == "grouped_grads" else out, device="cuda")
    if case["op"] in ("product", "grouped_i8"):
        s["x"], s["sx"] = to_8_bits(x)
        s["w"], s["sw"] = torch.empty(w.shape, dtype=torch.int8, device="cuda"), torch.empty(w.shape[:2], device="cuda")
        for e in range(w.shape[0]):
            s["w"][e], s["sw"][e] = to_8_bits(w[e])
        if case["op"] == "product":
            s["w"], s["sw"] = s["w"][0], s["sw"][0]
            return s
    else:
        s["x"], s["w"] = x, w
    s["sizes"] = group_sizes(case)
    s["offsets"] = torch.tensor([sum(s["sizes"][:e]) for e in range(len(s["sizes"]) + 1)], dtype=torch.int32, device="cuda")
    if case["op"] == "grouped_grads":
        s["gy"] = (torch.randn((rows, d_out), generator=gen, device="cuda") * 1e-2).to(torch.bfloat16)
        s["gx"] = torch.empty_like(x)
        s["gw"] = torch.empty(w.shape, dtype=out, device="cuda")
        del s["y"]
    return s


def run(s):
    return run_own(s) if own else run_plain(s)


def run_own(s):
    import paper_2605_29843_b200 as harp
    op = s["op"]
    if op == "quantise":
        q, scale = harp.quantize_rows(s["x"], out=s["q"], scale=s["scale"])
        return {"q": q, "scale": scale}
    if op == "product":
        return harp.linear_i8(s["x"], s["sx"], s["w"], s["sw"], out=s["y"])
    if op == "grouped_i8":
        return harp.grouped_linear_i8(s["x"], s["sx"], s["w"], s["sw"], s["offsets"], out=s["y"])
    if op == "grouped":
        return harp.grouped_linear(s["x"], s["w"], s["offsets"], out=s["y"])
    return {"gx": harp.grouped_grad_rows(s["gy"], s["w"], s["offsets"], out=s["gx"]),
            "gw": harp.grouped_grad_weights(s["gy"], s["x"], s["offsets"], out=s["gw"])}


def run_plain(s):
    op = s["op"]
    if op == "quantise":
        most = s["x"].abs().amax(1).float()
        q = torch.where(most[:, None] > 0, s["x"].double() * 127.0 / most.double()[:, None], 0.0).round()
        return {"q": q.to(torch.int8), "scale": most / 127.0}
    if op == "product":
        return ((s["x"].float() @ s["w"].float().T) * s["sw"] * s["sx"][:, None]).to(s["y"].dtype)
    # One product an expert, as the definition says: padding every group to the longest one would
    # multiply the work wherever the groups are uneven.
    xs = s["x"].split(s["sizes"])
    if op == "grouped_i8":
        y = [(x.float() @ w.float().T) * sw * sx[:, None] for x, sx, w, sw in zip(xs, s["sx"].split(s["sizes"]), s["w"], s["sw"])]
        return torch.cat(y).to(s["y"].dtype)
    if op == "grouped":
        return torch.cat([(x.float() @ w.float().T).to(s["y"].dtype) for x, w in zip(xs, s["w"])])
    gys = s["gy"].split(s["sizes"])
    return {"gx": torch.cat([(g.float() @ w.float()).to(s["gx"].dtype) for g, w in zip(gys, s["w"])]),
            "gw": torch.stack([(g.float().T @ x.float()).to(s["gw"].dtype) for g, x in zip(gys, xs)])}


def work(case):
    """Each input read once and each output written once; weights only of the experts that have rows,
    their gradients of all experts."""
    if case["op"] == "quantise":
        n = case["rows"] * case["d"]
        return {"bytes": n * (DTYPES[case["dtype"]].itemsize + 1) + 4 * case["rows"], "flops": 3 * n}
    rows, d_in, d_out = case["rows"], case["d_in"], case["d_out"]
    out = DTYPES[case["out"]].itemsize
    flops = 2 * rows * d_in * d_out
    if case["op"] == "product":
        return {"bytes": rows * d_in + d_in * d_out + rows * d_out * out + 4 * (rows + d_out), "flops": flops}
    met = sum(n > 0 for n in group_sizes(case))
    if case["op"] == "grouped_i8":
        return {"bytes": rows * d_in + met * (d_in + 4) * d_out + rows * d_out * out + 4 * rows, "flops": flops}
    if case["op"] == "grouped":
        return {"bytes": 2 * rows * d_in + 2 * met * d_in * d_out + rows * d_out * out, "flops": flops}
    return {"bytes": 2 * rows * (2 * d_in + d_out) + 2 * met * d_in * d_out + case["groups"] * d_in * d_out * out, "flops": 2 * flops}


def exact(case, seed):
    """From the definitions in 64 bits, a slice of the rows or an expert at a time."""
    s = prepare(case, seed)
    if case["op"] == "quantise":
        q, scale = torch.empty(s["x"].shape, dtype=torch.int8, device="cuda"), torch.empty(case["rows"], dtype=torch.float64, device="cuda")
        for r in range(0, case["rows"], 1024):
            x = s["x"][r:r + 1024].to(torch.float64)
            step = torch.linalg.vector_norm(x, math.inf, dim=1)
            scale[r:r + 1024] = step / 127
            q[r:r + 1024] = torch.round(127 * x / torch.where(step == 0, 1.0, step).unsqueeze(1)).to(torch.int8)
        return {"q": q, "scale": scale}

    def product(a, b):  # a b^T
        y = torch.empty((a.shape[0], b.shape[0]), dtype=torch.float64, device="cuda")
        b = b.to(torch.float64)
        for r in range(0, a.shape[0], 4096):
            y[r:r + 4096] = torch.einsum("rk,nk->rn", a[r:r + 4096].to(torch.float64), b)
        return y

    if case["op"] == "product":
        return product(s["x"], s["w"]).mul_(s["sx"].to(torch.float64).unsqueeze(1)).mul_(s["sw"].to(torch.float64))
    rows, at = [], 0
    for n in s["sizes"]:
        rows.append(slice(at, at + n))
        at += n
    if case["op"] == "grouped_grads":
        gx = torch.empty(s["x"].shape, dtype=torch.float64, device="cuda")
        gw = torch.empty(s["w"].shape, dtype=torch.float64, device="cuda")
        for e, r in enumerate(rows):
            gx[r] = product(s["gy"][r], s["w"][e].T)
            gw[e] = product(s["gy"][r].T, s["x"][r].T)
        return {"gx": gx, "gw": gw}
    y = torch.empty((case["rows"], case["d_out"]), dtype=torch.float64, device="cuda")
    for e, r in enumerate(rows):
        y[r] = product(s["x"][r], s["w"][e])
        if case["op"] == "grouped_i8":
            y[r] *= s["sx"][r].to(torch.float64).unsqueeze(1) * s["sw"][e].to(torch.float64)
    return y
