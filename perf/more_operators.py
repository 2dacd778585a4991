"""Calls of the operators that close a training step of a language model around
the codec: the log probabilities of given tokens with entropy and the most
likely alternatives, their gradient, and the AdamW step of the server over many
tensors, with its states in 32 or in 8 bits.

``own`` False computes them in their plain form with torch operations in 32
bits; ``own`` True makes the calls of ``paper_1802_07389_amd.tlc``.
"""
import math

import numpy as np
import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BYTES = {"f32": 4, "bf16": 2, "f16": 2, "i32": 4, "i64": 8}
IGNORE = -100     # target of a token that is left out
SIGMA = 1e-3      # gradients' standard deviation
WEIGHT = 0.02     # weights' standard deviation
STEPS_DONE = 1000  # optimizer steps before the one that is timed
RATES = dict(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.1)

BLOCK = 256       # values that share a scale of the 8-bit states
DITHER_K, DITHER_T = 0xC13FA9A9, 0x91E10DA5

# Tensors of a residual network with two 3x3 convolutions a block: widths of
# the three stages, blocks a stage (335 tensors from 10 to 36,864 values).
RESNET_WIDTHS, RESNET_BLOCKS = (16, 32, 64), 18


# ---------------------------------------------------------------- cases
def listed():
    return [
        # one generated token and its alternatives: latency
        dict(name="logp_1", op="logprobs", tokens=1, vocab=32768, type="bf16", pitch=0, scale=1.0,
             ignored=0.0, masked=0.0, top=20, ids_type="i64"),
        # one step of generation for 64 sequences, a large vocabulary, temperature
        dict(name="logp_64", op="logprobs", tokens=64, vocab=131072, type="f32", pitch=0,
             scale=1.25, ignored=0.0, masked=0.0, top=20, ids_type="i64"),
        # ragged: an odd vocabulary with masked entries, empty rows and padding
        dict(name="logp_odd", op="logprobs", tokens=1001, vocab=30011, type="f16", pitch=5,
             scale=0.7, ignored=0.3, masked=0.1, top=5, ids_type="i32"),
        # the loss of a training batch: 1 GiB of logits
        dict(name="logp_8k", op="logprobs", tokens=8192, vocab=65536, type="bf16", pitch=0,
             scale=1.0, ignored=0.1, masked=0.0, top=0, ids_type="i64"),
        # a short sequence of a small model: latency
        dict(name="logp_grad_512", op="logprobs_grad", tokens=512, vocab=8192, type="f32", out="f32",
             pitch=0, scale=1.0, ignored=0.0, masked=0.0, entropy=False, ids_type="i64"),
        # ragged, with a bonus for entropy
        dict(name="logp_grad_odd", op="logprobs_grad", tokens=2003, vocab=50021, type="f16",
             out="bf16", pitch=3, scale=0.7, ignored=0.3, masked=0.1, entropy=True,
             ids_type="i32"),
        # a training batch over a large vocabulary: 2 GiB of logits
        dict(name="logp_grad_8k", op="logprobs_grad", tokens=8192, vocab=131072, type="bf16",
             out="bf16", pitch=0, scale=1.0, ignored=0.1, masked=0.0, entropy=False,
             ids_type="i64"),
        # one step of a small network, clipped, its change written for the codec
        dict(name="adamw_resnet110", op="adamw", tensors="resnet110", count=335, n=1_730_714,
             type="f32", grad="f32", bits=32, clip=True, deltas=True),
        # a model's fp32 weights from bf16 gradients
        dict(name="adamw_100m", op="adamw", tensors="log", count=148, n=100_000_000, type="f32",
             grad="bf16", bits=32, clip=True, deltas=False),
        # one tensor of odd length, all in 16 bits but the states
        dict(name="adamw8_1m", op="adamw", tensors="one", count=1, n=1_000_003, type="bf16",
             grad="bf16", bits=8, clip=False, deltas=False),
        # the same step with states in 8 bits
        dict(name="adamw8_100m", op="adamw", tensors="log", count=148, n=100_000_000, type="f32",
             grad="bf16", bits=8, clip=True, deltas=False),
        # the server's step between sum and pull, states in 8 bits
        dict(name="adamw8_resnet110", op="adamw", tensors="resnet110", count=335, n=1_730_714,
             type="f32", grad="f32", bits=8, clip=False, deltas=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more call of any operator over the listed ranges."""
    op = rng.choice(["logprobs", "logprobs_grad", "adamw", "adamw"])
    types = ["f32", "bf16", "f16"]
    if op == "adamw":
        return dict(op=op, tensors="log", count=rng.choice([1, rng.randint(2, 400)]),
                    n=_log_int(rng, 1000, 100_000_000), type=rng.choice(types + ["f32"]),
                    grad=rng.choice(types), bits=rng.choice([32, 8]),
                    clip=rng.random() < 0.5, deltas=rng.random() < 0.5)
    vocab = _log_int(rng, 32, 131072)
    vocab = vocab if rng.random() < 0.5 else max(32, vocab // 64 * 64)
    case = dict(op=op, vocab=vocab, type=rng.choice(types), pitch=rng.choice([0, 0, rng.randint(1, 16)]),
                scale=rng.choice([1.0, 1.0, 0.5, 1.25]), ignored=rng.choice([0.0, 0.1, 0.5]),
                masked=rng.choice([0.0, 0.0, 0.1]), ids_type=rng.choice(["i32", "i64"]))
    if op == "logprobs":
        case["top"] = min(vocab, rng.choice([0, 0, 1, 5, 20, 64]))
        case["tokens"] = min(_log_int(rng, 1, 16384), (1 << 28) // vocab)
    else:
        case["out"] = rng.choice([case["type"], "f32", "bf16"])
        case["entropy"] = rng.random() < 0.3
        case["tokens"] = min(_log_int(rng, 1, 16384), (1 << 29) // vocab)
    return case


# ---------------------------------------------------------------- inputs
def _sizes(case):
    """Value counts of the tensors of one step."""
    if case["tensors"] == "resnet110":
        sizes, cin = [3 * 3 * 3 * 16, 16, 16], 16
        for width in RESNET_WIDTHS:
            for _ in range(RESNET_BLOCKS):
                sizes += [9 * cin * width, width, width, 9 * width * width, width, width]
                sizes += [cin * width, width, width] if cin != width else []
                cin = width
        return sizes + [640, 10]
    if case["count"] == 1:
        return [case["n"]]
    rng = np.random.default_rng([case["count"], case["n"]])
    w = np.exp(rng.uniform(math.log(16), math.log(200_000), case["count"]))
    return [max(1, int(v)) for v in w / w.sum() * case["n"]]


def _blocks(n):
    return -(-n // BLOCK)


def _normal(g, sigma, *shape):
    return torch.empty(*shape, device="cuda").normal_(0.0, sigma, generator=g)


def _adamw_operands(case, seed):
    """Weights, gradients and states, all tensors of a kind after one another."""
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    sizes = _sizes(case)
    n = sum(sizes)
    # tensors learn at their own rates: their gradients' sizes differ
    each = torch.exp(_normal(g, 1.0, len(sizes))).repeat_interleave(
        torch.tensor(sizes, device="cuda"), output_size=n) * SIGMA
    s = dict(params=_normal(g, WEIGHT, n).to(TYPES[case["type"]]),
             grads=_normal(g, 1.0, n).mul_(each).to(TYPES[case["grad"]]))
    m = _normal(g, 0.25, n).mul_(each)
    v = torch.exp(_normal(g, 1.0, n)).mul_(each.square())
    if case["bits"] == 32:
        s.update(exp_avg=m, exp_avg_sq=v)
    else:
        at, blocks, _ = _layout(sizes)
        pad = torch.zeros(2, blocks * BLOCK, device="cuda")
        pad[0, at], pad[1, at] = m, v
        pad = pad.view(2, blocks, BLOCK)
        s["scales"] = torch.stack([pad[0].abs().amax(1) / 448, pad[1].amax(1) / 57344], 1)
        s["exp_avg"], s["exp_avg_sq"] = [
            (pad[i] / s["scales"][:, i:i + 1]).view(-1)[at].to(t)
            for i, t in enumerate([torch.float8_e4m3fn, torch.float8_e5m2])]
    if case["deltas"]:
        s["deltas"] = torch.empty(n, device="cuda")
    # the clock: int64 step, float32 factor of the rate
    s["clock"] = torch.tensor([STEPS_DONE, 0x3f800000], device="cuda")
    # the norm that a call before this one has left
    flat = s["grads"].double()
    s["sumsq"] = torch.dot(flat, flat)
    s["max_norm"] = float(np.float32(0.5 * math.exp(1.0) * SIGMA * math.sqrt(n)))
    return s


def _layout(sizes):
    """Where each value is among whole blocks, how many there are, and each
    place's index in its tensor."""
    n = torch.tensor(sizes, device="cuda")
    blocks = (n + BLOCK - 1) // BLOCK
    first = blocks.cumsum(0) - blocks
    total, count = sum(sizes), sum(_blocks(v) for v in sizes)
    start = (first * BLOCK - (n.cumsum(0) - n)).repeat_interleave(n, output_size=total)
    at = torch.arange(total, device="cuda") + start
    k = torch.arange(count * BLOCK, device="cuda") - (first * BLOCK).repeat_interleave(
        blocks * BLOCK, output_size=count * BLOCK)
    return at, count, k


def _logit_operands(case, seed):
    """Logits and targets: a bulk of values, most targets well above it."""
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    t, v = case["tokens"], case["vocab"]
    x = _normal(g, 2.0, t, v + case["pitch"]).to(TYPES[case["type"]])[:, :v]
    u = torch.rand(3, t, device="cuda", generator=g, dtype=torch.float64)
    open_ = max(1, int(v * (1.0 - case["masked"])))  # entries that are not masked
    targets = (open_ ** u[0]).long().clamp_(0, open_ - 1)
    up = torch.where(u[1] < 0.7, 8.0, 0.0).to(x.dtype)
    row = torch.arange(t, device="cuda")
    x[row, targets] += up
    if case["masked"]:
        x[:, open_:] = -math.inf
        x[96::97] = -math.inf  # nothing left in a row
    targets = torch.where(u[2] < case["ignored"], IGNORE, targets)
    s = dict(logits=x, scale=case["scale"],
             targets=targets.to(torch.int32 if case["ids_type"] == "i32" else torch.int64))
    if case["op"] == "logprobs_grad":
        kept = max(1.0, t * (1.0 - case["ignored"]))
        s["grad_logprob"] = -torch.exp(_normal(g, 0.5, t)) / kept
        s["grad_entropy"] = torch.full((t,), -0.1 / kept, device="cuda") if case["entropy"] else None
    return s


def _operands(case, seed):
    return _adamw_operands(case, seed) if case["op"] == "adamw" else _logit_operands(case, seed)


_kept = {}  # the program's one context


def _context(case):
    from paper_1802_07389_amd import tlc
    tensors = len(_sizes(case)) if case["op"] == "adamw" else 0
    if tensors not in _kept:
        _kept.clear()
        _kept[tensors] = tlc.TrainContext(max_tensors=tensors)
    return _kept[tensors]


def _prepare_adamw(case, s):
    sizes = _sizes(case)
    if not own:
        if case["bits"] == 8:
            s["at"], s["blocks"], s["k"] = _layout(sizes)
        return
    split = lambda name: list(torch.split(s[name], sizes))  # noqa: E731
    states = [split("exp_avg"), split("exp_avg_sq")]
    if case["bits"] == 8:
        states.append(list(torch.split(s["scales"], [_blocks(v) for v in sizes])))
    s["list"] = s["ctx"].adamw_list(
        split("params"), grads=split("grads"), bits=case["bits"], states=states,
        deltas=split("deltas") if case["deltas"] else None, clock=s["clock"])
    s["result"] = s["ctx"].norm_result()
    s["result"].sumsq.copy_(s["sumsq"])


def prepare(case, seed):
    """Inputs, states and output buffers; with the framework's calls also the
    context and the list of tensors, which a program makes once and keeps."""
    s = dict(case=dict(case), **_operands(case, seed))
    if own:
        s["ctx"] = _context(case)
    if case["op"] == "adamw":
        _prepare_adamw(case, s)
    elif case["op"] == "logprobs_grad":
        s["out"] = torch.empty(case["tokens"], case["vocab"], device="cuda",
                               dtype=TYPES[case["out"]])
        # what the forward pass has left: both sides get the same, from 64 bits
        s["results"] = torch.stack(_statistics(s, torch.float64), 1).float().contiguous()
    elif own:
        s["out"] = s["ctx"].token_result(case["tokens"], case["top"])
    return s


# ---------------------------------------------------------------- plain forms
def _statistics(s, dtype):
    """Log probability, entropy, largest logit and log-sum of every row, some
    rows at a time; 0 where the target is left out."""
    parts = []
    for x, target in zip(s["logits"].split(1024), s["targets"].long().split(1024)):
        x = x.to(dtype)
        m = x.amax(1)
        empty = m == -math.inf
        z = (x - torch.where(empty, 0.0, m)[:, None]) * s["scale"]
        e = torch.exp(z)
        total = e.sum(1)
        log_sum = torch.log(total)
        own_z = z.gather(1, target.clamp(min=0)[:, None])[:, 0]
        logp = torch.where(empty, -math.inf, own_z - log_sum)
        entropy = torch.where(empty, 0.0, log_sum - (e * z.clamp(min=-1e30)).sum(1) / total)
        parts.append([torch.where(target == IGNORE, 0.0, c) for c in (logp, entropy, m, log_sum)])
    return [torch.cat(c) for c in zip(*parts)]


def _top(s, k):
    """The k largest logits of every row, the lowest index first among equals:
    their values in 32 bits and their indices."""
    x = s["logits"].float() + 0.0
    bits = x.view(torch.int32).long()
    order = torch.where(bits < 0, -(bits & 0x7fffffff), bits)
    keys = order * (1 << 32) + (0xffffffff - torch.arange(x.shape[1], device="cuda"))
    ids = 0xffffffff - (torch.topk(keys, k, dim=1).values & 0xffffffff)
    return x.gather(1, ids), ids


def _run_logprobs(s):
    logp, entropy, m, log_sum = _statistics(s, torch.float32)
    r = dict(logprob=logp, entropy=entropy, max=m, log_sum=log_sum)
    if s["case"]["top"]:
        x, ids = _top(s, s["case"]["top"])
        skip = (s["targets"] == IGNORE)[:, None]
        z = torch.where(m == -math.inf, -math.inf, (x - m[:, None]).T * s["scale"] - log_sum).T
        r["top_logprobs"] = torch.where(skip, 0.0, z)
        r["top_ids"] = torch.where(skip, -1, ids).int()
    return r


def _run_grad(s):
    _, entropy, m, log_sum = s["results"].unbind(1)
    keep = s["targets"] != IGNORE
    live = keep & (m != -math.inf)
    row = torch.arange(live.numel(), device="cuda")[live]
    target = s["targets"].long()[live]
    z = (s["logits"].float() - torch.where(live, m, 0.0)[:, None]) * s["scale"] - log_sum[:, None]
    p = torch.exp(z)
    a = s["grad_logprob"] * s["scale"]
    d = -a[:, None] * p
    if s["grad_entropy"] is not None:
        b = s["grad_entropy"] * s["scale"]
        d -= b[:, None] * (p * (z.clamp(min=-1e30) + entropy[:, None]))
    d[row, target] += a[live]
    s["out"].copy_(torch.where(live[:, None], d, 0.0))
    return {"out": s["out"]}


def _fp8(x, scale, dither, mantissa, lowest, most):
    """Codes of an 8-bit float with `mantissa` bits, smallest exponent `lowest`
    and largest code `most`: x / scale, dithered to one of its neighbours."""
    y = (x.abs() / scale).nan_to_num(0.0)  # 0 / 0
    cut = 23 - mantissa
    bits = y.view(torch.int32).long()
    fine = ((bits + dither) >> cut) - ((126 + lowest) << mantissa)
    small = ((y * 2.0 ** (mantissa - lowest + cut)).clamp(max=2.0 ** 24).long() + dither) >> cut
    return torch.where(y < 2.0 ** lowest, small, fine).clamp(max=most)


def _states_8(s, m, v, step):
    """Codes and scales of the new states, given in whole blocks."""
    h = (s["k"] * DITHER_K + step * DITHER_T) & 0xffffffff
    h = h.view(-1, BLOCK)
    scales = torch.stack([m.abs().amax(1) / 448, v.amax(1) / 57344], 1)
    scales = torch.where(torch.stack([m.abs().amax(1), v.amax(1)], 1) > 0,
                         scales.clamp(min=2.0 ** -126), 0.0)
    q = _fp8(m, scales[:, :1], h >> 12, 3, -6, 126) | torch.where(m.signbit(), 128, 0)
    r = _fp8(v, scales[:, 1:], (h ^ 0x80000000) >> 11, 2, -14, 123)
    r = torch.where((v > 0) & (r == 0), 1, r)
    return scales, q.to(torch.uint8).view(-1), r.to(torch.uint8).view(-1)


def _run_adamw(s):
    case, r = s["case"], RATES
    s["clock"][0] += 1
    step, factor = s["clock"][0], s["clock"].view(torch.float32)[2]
    lr = r["lr"] * factor.double()
    rate = (lr / -torch.expm1(step * math.log(r["beta1"]))).float()
    root = (1.0 / torch.sqrt(-torch.expm1(step * math.log(r["beta2"])))).float()
    decay = (lr * r["weight_decay"]).float()
    out = {"step": step}
    g = s["grads"].float()
    if case["clip"]:
        norm = torch.sqrt(s["sumsq"])
        out["norm"], out["coef"] = norm.float(), (s["max_norm"] / norm).clamp(max=1.0).float()
        g = g * out["coef"]
    m, v = s["exp_avg"].float(), s["exp_avg_sq"].float()
    if case["bits"] == 8:
        block = s["at"] // BLOCK
        m, v = m * s["scales"][block, 0], v * s["scales"][block, 1]
    m = m + (g - m) * (1.0 - r["beta1"])
    v = v + (g * g - v) * (1.0 - r["beta2"])
    p = s["params"].float()
    p = p - (rate * (m / (torch.sqrt(v) * root + r["eps"])) + decay * p)
    if case["deltas"]:
        torch.sub(p.to(s["params"].dtype).float(), s["params"].float(), out=s["deltas"])
        out["deltas"] = s["deltas"]
    s["params"].copy_(p)
    if case["bits"] == 8:
        pad = torch.zeros(2, s["blocks"] * BLOCK, device="cuda")
        pad[0, s["at"]], pad[1, s["at"]] = m, v
        scales, q, w = _states_8(s, *pad.view(2, -1, BLOCK), step)
        s["scales"].copy_(scales)
        out["scales"] = s["scales"]
        s["exp_avg"].view(torch.uint8).copy_(q[s["at"]])
        s["exp_avg_sq"].view(torch.uint8).copy_(w[s["at"]])
    else:
        s["exp_avg"].copy_(m)
        s["exp_avg_sq"].copy_(v)
    return dict(out, params=s["params"], exp_avg=s["exp_avg"], exp_avg_sq=s["exp_avg_sq"])


# ---------------------------------------------------------------- passes
def _run_own(s):
    case, ctx = s["case"], s["ctx"]
    if case["op"] == "logprobs":
        r = ctx.token_logprobs(s["logits"], s["targets"], scale=s["scale"], ignore_id=IGNORE,
                               top=case["top"], out=s["out"])
        out = dict(logprob=r.logprob, entropy=r.entropy, max=r.max, log_sum=r.log_sum)
        if case["top"]:
            out.update(top_logprobs=r.top_logprobs, top_ids=r.top_ids)
        return out
    if case["op"] == "logprobs_grad":
        ctx.token_logprobs_grad(s["logits"], s["targets"], s["results"], s["grad_logprob"],
                                grad_entropy=s["grad_entropy"], scale=s["scale"],
                                ignore_id=IGNORE, out=s["out"])
        return {"out": s["out"]}
    ctx.adamw(s["list"], max_norm=s["max_norm"] if case["clip"] else None,
              result=s["result"] if case["clip"] else None, **RATES)
    out = dict(step=s["list"].step, params=s["params"], exp_avg=s["exp_avg"],
               exp_avg_sq=s["exp_avg_sq"])
    if case["clip"]:
        out.update(norm=s["result"].norm, coef=s["result"].coef)
    if case["deltas"]:
        out["deltas"] = s["deltas"]
    if case["bits"] == 8:
        out["scales"] = s["scales"]
    return out


def run(s):
    if own:
        return _run_own(s)
    return {"logprobs": _run_logprobs, "logprobs_grad": _run_grad, "adamw": _run_adamw}[
        s["case"]["op"]](s)


# ---------------------------------------------------------------- work, 64 bits
def work(case):
    """Bytes and operations of one pass: every input read once, every output
    written once."""
    if case["op"] == "adamw":
        sizes = _sizes(case)
        n = sum(sizes)
        each = 2 * BYTES[case["type"]] + BYTES[case["grad"]] + 4 * case["deltas"]
        each += 16 if case["bits"] == 32 else 4
        scales = 16 * sum(_blocks(v) for v in sizes) if case["bits"] == 8 else 0
        return {"bytes": n * each + scales, "flops": n * 16}
    t, v = case["tokens"], case["vocab"]
    kept = t * (1.0 - case["ignored"])
    read = kept * v * BYTES[case["type"]] + t * BYTES[case["ids_type"]]
    if case["op"] == "logprobs":
        return {"bytes": read + t * (16 + 8 * case["top"]), "flops": kept * v * 6}
    rows = kept * (20 + 4 * case["entropy"])
    return {"bytes": read + rows + t * v * BYTES[case["out"]], "flops": kept * v * 5}


def _exact_logprobs(case, s):
    x = s["logits"].double()
    skip = s["targets"] == IGNORE
    z = x * s["scale"]
    m = x.max(1).values
    empty = m == -math.inf
    # probabilities from the scaled logits themselves, moved so that none overflows
    p = torch.exp(z - torch.where(empty, 0.0, m * s["scale"])[:, None])
    total = p.sum(1)
    p /= total[:, None]
    lse = torch.log(total) + m * s["scale"]
    log_p = z - lse[:, None]
    entropy = -torch.where(p > 0, p * log_p, 0.0).sum(1)
    logp = torch.where(empty, -math.inf, log_p[torch.arange(len(x)), s["targets"].long().clamp(min=0)])
    r = dict(logprob=logp, entropy=torch.where(empty, 0.0, entropy), max=m, log_sum=torch.log(total))
    r = {k: torch.where(skip, 0.0, c) for k, c in r.items()}
    if case["top"]:
        ids = torch.sort(s["logits"].float(), dim=1, descending=True, stable=True).indices
        ids = ids[:, :case["top"]]
        top = torch.where(empty[:, None], -math.inf, log_p.gather(1, ids))
        r["top_logprobs"] = torch.where(skip[:, None], 0.0, top)
        r["top_ids"] = torch.where(skip[:, None], -1, ids).int()
    return r


def _exact_grad(case, s):
    out = torch.zeros(case["tokens"], case["vocab"], device="cuda", dtype=torch.float64)
    for r in range(0, case["tokens"], 512):
        x = s["logits"][r:r + 512].double() * s["scale"]
        p = torch.softmax(x, 1)
        one = torch.zeros_like(p)
        target = s["targets"][r:r + 512].long()
        one.scatter_(1, target.clamp(min=0)[:, None], 1.0)
        d = s["grad_logprob"][r:r + 512, None].double() * (one - p)
        if s["grad_entropy"] is not None:
            plogp = torch.where(p > 0, p * torch.log(p), 0.0)
            d += s["grad_entropy"][r:r + 512, None].double() * (
                p * plogp.sum(1, keepdim=True) - plogp)
        live = (target != IGNORE) & ~torch.isneginf(x).all(1)
        out[r:r + 512] = torch.where(live[:, None], d * s["scale"], 0.0)
    return {"out": out}


def _exact_fp8(x, scale, dither, mantissa, lowest, most, floor):
    """Values, without their scale, of the codes in 64 bits: the format's codes
    are joined by straight lines, and the dither carries a place on them up."""
    y = (x.abs() / scale).nan_to_num(0.0)
    e = torch.frexp(y).exponent - 1
    e = e.clamp(min=lowest)
    unit = torch.exp2((e - mantissa).double())
    q = torch.floor(y / unit + dither) * unit
    q = torch.where(floor & (q == 0) & (y > 0), 2.0 ** (lowest - mantissa), q)
    return q.clamp(max=most) * torch.sign(x)


def _exact_adamw(case, s):
    r, t = RATES, STEPS_DONE + 1
    g, p = s["grads"].double(), s["params"].double()
    out = {"step": t}
    if case["clip"]:
        norm = math.sqrt(float(s["sumsq"]))
        out["norm"], out["coef"] = norm, min(1.0, s["max_norm"] / norm)
        g = g * out["coef"]
    m, v = s["exp_avg"].double(), s["exp_avg_sq"].double()
    if case["bits"] == 8:
        at, blocks, k = _layout(_sizes(case))
        m *= s["scales"].double()[at // BLOCK, 0]
        v *= s["scales"].double()[at // BLOCK, 1]
    m = r["beta1"] * m + (1.0 - r["beta1"]) * g
    v = r["beta2"] * v + (1.0 - r["beta2"]) * g.square()
    hat = (v / (1.0 - r["beta2"] ** t)).sqrt() + r["eps"]
    change = -r["lr"] * (m / (1.0 - r["beta1"] ** t) / hat + r["weight_decay"] * p)
    out["params"] = p + change
    if case["deltas"]:
        # the change as it is stored: of 16-bit weights it has no value in 64 bits
        out["deltas"] = change if case["type"] == "f32" else None
    if case["bits"] == 32:
        return dict(out, exp_avg=m, exp_avg_sq=v)
    pad = torch.zeros(2, blocks * BLOCK, device="cuda", dtype=torch.float64)
    pad[0, at], pad[1, at] = m, v
    m, v = pad.view(2, blocks, BLOCK)
    h = ((k * DITHER_K + t * DITHER_T) % (1 << 32)).view(blocks, BLOCK)
    scale_m, scale_v = m.abs().amax(1) / 448, v.amax(1) / 57344
    q = _exact_fp8(m, scale_m[:, None], (h // (1 << 12)) / 2.0 ** 20, 3, -6, 448.0,
                   torch.zeros_like(m, dtype=torch.bool))
    h = (h + (1 << 31)) % (1 << 32)
    w = _exact_fp8(v, scale_v[:, None], (h // (1 << 11)) / 2.0 ** 21, 2, -14, 57344.0,
                   torch.ones_like(v, dtype=torch.bool))
    return dict(out, scales=torch.stack([scale_m, scale_v], 1), exp_avg=q.reshape(-1)[at],
                exp_avg_sq=w.reshape(-1)[at])


def exact(case, seed):
    s = _operands(case, seed)
    return {"logprobs": _exact_logprobs, "logprobs_grad": _exact_grad, "adamw": _exact_adamw}[
        case["op"]](case, s)
