"""The gradients of many tensors, as cases that can be timed: their global norm, clipping by it, and the way from a
model's list of gradient tensors to the flat fp32 vector that an encoder takes (gather) and from the decoded mean back
(scatter), clipped on the way.

The sizes are those of the repository's own workloads and of the networks whose gradients the paper counts (65,536 to
124,439,808 elements).  Gradients are normal with one standard deviation per tensor, in fp32, bf16 or fp16; they lie in
allocations of their own, side by side in one bucket (where odd sizes leave most of them at odd addresses), or are column
blocks of a fused layer's gradient.  Everything is drawn on the GPU from the seed.
"""
import math
import random

import numpy as np
import torch

own = False      # False: the operators in plain torch operations; True: this library's kernels

DTYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
# The networks of the paper whose layers are known: weight and bias of every layer.
NETWORKS = {
    "fc300": [784 * 300, 300, 300 * 100, 100, 100 * 10, 10],
    "lenet": [5 * 5 * 32, 32, 5 * 5 * 32 * 64, 64, 3136 * 512, 512, 512 * 10, 10],
}


def listed():
    return [
        # The norm of a small network's gradient, logged every step: launches and host work decide.
        dict(name="norm_fc300", op="norm", n=266610, sizes="fc300", dtype="fp32", store="own", kind="l2", each=False),
        # Adapters and normalisation weights: two thousand tensors of 1 to 4096 elements side by side in one bucket, and
        # the norm of each beside the global one.
        dict(name="norm_adapters", op="norm", n=980001, sizes="small", count=2000, dtype="bf16", store="bucket",
             kind="l2", each=True),
        # An ordinary norm: ResNet-50-sized, fp32, with the norm of each tensor.
        dict(name="norm_resnet50", op="norm", n=25557032, sizes="layered", count=161, dtype="fp32", store="own", kind="l2",
             each=True),
        # The largest norm: the maximum of a GPT-2-small-sized bf16 gradient, the scale of a one-bucket quantizer.
        dict(name="norm_gpt2_max", op="norm", n=124439808, sizes="layered", count=148, dtype="bf16", store="own",
             kind="max", each=False),
        # The smallest clipping: one layer's weights and biases into the optimizer's own buffers.
        dict(name="clip_tiny", op="clip", n=65536, sizes="layered", count=4, dtype="fp32", out="fp32", store="own",
             kind="l2", ratio=0.3),
        # Gradients that are column blocks of fused layers' gradients (three blocks of 1280 columns, four layers).
        dict(name="clip_blocks", op="clip", n=4 * 3 * 1280 * 1280, sizes="blocks", rows=1280, cols=1280, layers=4,
             dtype="bf16", out="bf16", store="blocks", kind="l2", ratio=0.3),
        # Half-precision gradients of a ResNet-18-sized network, clipped into fp32 for the optimizer.
        dict(name="clip_resnet18", op="clip", n=11689512, sizes="layered", count=62, dtype="fp16", out="fp32", store="own",
             kind="l2", ratio=0.9),
        # A worker's gradient on its way to the encoder: the paper's LeNet-like network, fp32.
        dict(name="gather_lenet", op="gather", n=1663370, sizes="lenet", dtype="fp32", store="own", kind="l2", ratio=0.3),
        # The same, ResNet-50-sized, bf16 in one bucket with odd sizes.
        dict(name="gather_resnet50", op="gather", n=25557032, sizes="layered", count=161, dtype="bf16", store="bucket",
             kind="l2", ratio=0.9),
        # The largest gather: GPT-2-small-sized, matrices in bf16, vectors in fp32, clipped by the largest element.
        dict(name="gather_gpt2", op="gather", n=124439808, sizes="layered", count=148, dtype="mixed", store="own",
             kind="max", ratio=0.3),
        # The decoded mean back into a ResNet-18-sized model's tensors, matrices in bf16, vectors in fp32.
        dict(name="scatter_resnet18", op="scatter", n=11689512, sizes="layered", count=62, dtype="mixed", store="own",
             kind="l2", ratio=0.3),
        # The largest scatter, fp32, of a step whose norm is below the limit: nothing is clipped, all is moved.
        dict(name="scatter_gpt2", op="scatter", n=124439808, sizes="layered", count=148, dtype="fp32", store="own",
             kind="l2", ratio=2.0),
    ]


def draw(rng):
    def log_int(lo, hi):
        return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))

    op = rng.choice(["norm", "clip", "gather", "scatter"])
    case = dict(op=op, dtype=rng.choice(["fp32", "bf16", "fp16", "mixed"]), kind=rng.choice(["l2", "l2", "max"]))
    how = rng.choices(["layered", "small", "blocks"], weights=[6, 2, 2 if op != "scatter" else 0])[0]
    case["sizes"], case["store"] = how, rng.choice(["own", "bucket"])
    if how == "layered":
        case["n"] = log_int(1 << 12, 124000000)
        case["count"] = min(log_int(1, 700), case["n"] // 200)
    elif how == "small":
        case["count"] = log_int(100, 4000)
        case["n"] = case["count"] * rng.randint(50, 800) + rng.randint(0, 99)
    else:
        case.update(store="blocks", rows=log_int(16, 4000), cols=log_int(16, 2500), layers=rng.randint(1, 4))
        case["n"] = case["layers"] * 3 * case["rows"] * case["cols"]
        if case["dtype"] == "mixed":
            case["dtype"] = "bf16"
    if op == "norm":
        case["each"] = rng.random() < 0.5
    else:
        case["ratio"] = rng.choice([0.1, 0.3, 0.9, 2.0])
    if op == "clip":
        case["out"] = rng.choice(["same", "fp32"])
    return case


# ------------------------------------------------------------------------------------------------------ inputs
def _sizes(case):
    """Elements of each tensor; the shapes of a network do not change with the seed of its gradients."""
    how, n = case["sizes"], case["n"]
    if how in NETWORKS:
        return list(NETWORKS[how])
    if how == "blocks":
        return [case["rows"] * case["cols"]] * (3 * case["layers"])
    rng, count = random.Random(n + case["count"]), case["count"]
    lo, hi = (1.0, 4096.0) if how == "small" else (1e2, 3e6)
    raw = [math.exp(rng.uniform(math.log(lo), math.log(hi))) for _ in range(count)]
    total = sum(raw)
    sizes = [max(1, int(r / total * n)) for r in raw]
    sizes[sizes.index(max(sizes))] += n - sum(sizes)
    return sizes


def _dtypes(case, dtype):
    """One type for all tensors, or bf16 for the matrices and fp32 for what is short."""
    sizes = _sizes(case)
    if dtype == "mixed":
        return [torch.bfloat16 if m > 8192 else torch.float32 for m in sizes]
    return [DTYPES[dtype]] * len(sizes)


def _sigmas(case, seed):
    """A standard deviation per tensor; fp16 gradients carry a loss scale."""
    rng, scale = random.Random(seed), 1024.0 if case["dtype"] == "fp16" else 1.0
    return [scale * math.exp(rng.uniform(math.log(1e-4), math.log(1e-1))) for _ in _sizes(case)]


def _max_norm(case, sizes, sigmas):
    """The limit of a training program, as a part of the norm that gradients of these deviations have."""
    if case["kind"] == "l2":
        usual = math.sqrt(sum(m * s * s for m, s in zip(sizes, sigmas)))
    else:
        usual = max(s * math.sqrt(2.0 * math.log(m + 1.0)) for m, s in zip(sizes, sigmas))
    return case["ratio"] * usual


def _placed(sizes, dtypes, store, device="cuda", as_type=None):
    """Contiguous tensors that share one buffer per type: side by side in it ("bucket"), or each at a multiple of 128
    elements, as an allocator places them.  Returns the tensors and the buffers, whose gaps are zero."""
    at, used = [], dict.fromkeys(dtypes, 0)
    for m, t in zip(sizes, dtypes):
        at.append(used[t])
        used[t] += m if store == "bucket" else (m + 127) // 128 * 128
    buffers = {t: torch.zeros(used[t], dtype=as_type or t, device=device) for t in used}
    return [buffers[t][a:a + m] for m, t, a in zip(sizes, dtypes, at)], list(buffers.values())


def _gradients(case, seed, sigmas):
    sizes = _sizes(case)
    gen = torch.Generator(device="cuda").manual_seed(seed)
    values = torch.randn(sum(sizes), device="cuda", generator=gen)
    if case["store"] == "blocks":
        rows, cols = case["rows"], case["cols"]
        fused = values.view(case["layers"], rows, 3 * cols).to(DTYPES[case["dtype"]])
        grads = [fused[t // 3, :, t % 3 * cols:(t % 3 + 1) * cols] for t in range(len(sizes))]
        for g, s in zip(grads, sigmas):
            g.mul_(s)
        return grads
    dtypes = _dtypes(case, case["dtype"])
    if case["store"] == "bucket":
        grads, _ = _placed(sizes, dtypes, "bucket")
    else:
        grads = [torch.empty(m, dtype=t, device="cuda") for m, t in zip(sizes, dtypes)]
    for g, v, s in zip(grads, values.split(sizes), sigmas):
        g.copy_(v.mul_(s))
    return grads


def _out_dtypes(case):
    return _dtypes(case, "fp32" if case.get("out") == "fp32" else case["dtype"])


def prepare(case, seed):
    op, sizes, sigmas = case["op"], _sizes(case), _sigmas(case, seed)
    s = {"case": case, "op": op, "norm": torch.empty(1, device="cuda")}
    if op == "scatter":
        s["flat"] = torch.cat(_gradients(dict(case, dtype="fp32", store="own"), seed, sigmas))
    else:
        s["grads"] = _gradients(case, seed, sigmas)
    if op == "norm":
        s["norms"] = torch.empty(len(sizes), device="cuda") if case["each"] else None
        return s
    s["max_norm"] = _max_norm(case, sizes, sigmas)
    if op == "gather":
        s["flat"] = torch.empty(sum(sizes), device="cuda")
        return s
    s["out"], s["buffers"] = _placed(sizes, _out_dtypes(case), case["store"])
    if op == "clip":
        s["out"] = [o.view(g.shape) for o, g in zip(s["out"], s["grads"])]
    return s


# ------------------------------------------------------------------------------------------------------ one pass
def _plain_norms(tensors, kind):
    """The norm of each tensor and of all, in 64 bits (long sums), rounded once."""
    if kind == "max":
        each = torch.stack([t.abs().max().float() for t in tensors])
        return each, each.max().reshape(1)
    squares = torch.stack([t.double().square().sum() for t in tensors])
    return squares.sqrt().float(), squares.sum().sqrt().float().reshape(1)


def _plain_factor(norm, max_norm):
    limit = torch.full_like(norm, max_norm)
    return torch.where(norm <= limit, torch.ones_like(norm), limit / norm)


def _plain(s):
    case, op = s["case"], s["op"]
    tensors = [s["flat"]] if op == "scatter" else s["grads"]
    each, norm = _plain_norms(tensors, case["kind"])
    if op == "norm":
        return (norm, each) if case["each"] else norm
    c = _plain_factor(norm, s["max_norm"])
    if op == "gather":
        return norm, torch.cat([(g.float() * c).reshape(-1) for g in s["grads"]])
    parts = s["grads"] if op == "clip" else s["flat"].split([o.numel() for o in s["out"]])
    for p, o in zip(parts, s["out"]):
        o.copy_(p.float() * c)
    return norm, s["buffers"]


def run(s):
    if not own:
        return _plain(s)
    import paper_1904_01197_b200 as dq
    op = s["op"]
    kind = dq.DQ_NORM_MAX if s["case"]["kind"] == "max" else dq.DQ_NORM_L2
    if op == "norm":
        norm = dq.grad_norm(s["grads"], kind, out_norm=s["norm"], out_norms=s["norms"])
        return norm if s["norms"] is None else (norm, s["norms"])
    if op == "gather":
        flat = dq.grad_gather(s["grads"], s["flat"], max_norm=s["max_norm"], kind=kind, out_norm=s["norm"])
        return s["norm"], flat
    if op == "clip":
        dq.grad_clip(s["grads"], s["max_norm"], out=s["out"], kind=kind, out_norm=s["norm"])
    else:
        dq.grad_scatter(s["flat"], s["out"], max_norm=s["max_norm"], kind=kind, out_norm=s["norm"])
    return s["norm"], s["buffers"]


# ------------------------------------------------------------------------------------------------------ accounting
def _bytes(case, dtypes):
    return sum(m * t.itemsize for m, t in zip(_sizes(case), dtypes))


def work(case):
    """Bytes: every gradient once, every output once.  Operations: a square and an addition per element of an L2 norm, a
    comparison for the maximum, a product per element of what is clipped."""
    op, n = case["op"], case["n"]
    flops = n * (2 if case["kind"] == "l2" else 1)
    read = _bytes(case, _dtypes(case, "fp32" if op == "scatter" else case["dtype"]))
    if op == "norm":
        return {"bytes": read + 4 + (4 * len(_sizes(case)) if case["each"] else 0), "flops": flops}
    written = 4 * n if op == "gather" else _bytes(case, _out_dtypes(case))
    return {"bytes": read + written + 4, "flops": flops + n}


def exact(case, seed):
    """The definition in 64 bits, on the host: N = sqrt(sum x^2) or max |x|, y = x min(1, limit / N)."""
    s = prepare(case, seed)
    op = s["op"]
    x = [t.cpu().float().numpy().astype(np.float64) for t in ([s["flat"]] if op == "scatter" else s["grads"])]
    if case["kind"] == "max":
        each = [float(np.max(np.abs(v))) for v in x]
        total = max(each)
    else:
        sums = [float(np.sum(v * v)) for v in x]
        each, total = [math.sqrt(q) for q in sums], math.sqrt(math.fsum(sums))
    norm = torch.tensor([total], dtype=torch.float64)
    if op == "norm":
        return (norm, torch.tensor(each, dtype=torch.float64)) if case["each"] else norm
    y = [torch.from_numpy(v * min(1.0, s["max_norm"] / total)).reshape(-1) for v in x]
    if op == "gather":
        return norm, torch.cat(y)
    out, buffers = _placed(_sizes(case), _out_dtypes(case), case["store"], "cpu", torch.float64)
    for o, v in zip(out, y if op == "clip" else y[0].split(_sizes(case))):
        o.copy_(v)
    return norm, buffers
