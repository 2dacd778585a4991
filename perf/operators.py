"""Calls of the training-step operators that stand before the codec: the
embedding lookup with scaling, its gradient by tokens, the global norm of many
gradients and their clipping into the fp32 tensors that are compressed.

``own`` False computes them in their plain form with torch operations in 32
bits; ``own`` True makes the calls of ``paper_1802_07389_amd.tlc``.
"""
import math

import numpy as np
import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BYTES = {"f32": 4, "bf16": 2, "f16": 2, "i32": 4, "i64": 8}
SIGMA = 1e-3      # gradients' standard deviation
ZIPF_SHIFT = 2.7  # token ranks follow 1 / (rank + ZIPF_SHIFT)

# Tensors of a residual network with two 3x3 convolutions a block: widths of
# the three stages, blocks a stage (335 tensors from 10 to 36,864 values).
RESNET_WIDTHS, RESNET_BLOCKS = (16, 32, 64), 18


# ---------------------------------------------------------------- cases
def listed():
    return [
        # one step of generation for eight sequences: latency
        dict(name="embed_8", op="embedding", tokens=8, rows=32768, dim=1024, type="bf16",
             out="bf16", ids="zipf", ids_type="i64", pitch=0),
        # an ordinary training batch, fp32 master weights read as bf16
        dict(name="embed_16k", op="embedding", tokens=16384, rows=65536, dim=1024, type="f32",
             out="bf16", ids="zipf", ids_type="i64", pitch=0),
        # ragged: odd batch, odd vocabulary, rows of odd length in a wider table
        dict(name="embed_odd", op="embedding", tokens=5001, rows=30011, dim=1001, type="f16",
             out="f16", ids="uniform", ids_type="i32", pitch=6),
        # a long batch over a large table
        dict(name="embed_64k", op="embedding", tokens=65536, rows=131072, dim=2048, type="bf16",
             out="bf16", ids="zipf", ids_type="i64", pitch=0),
        # a short sequence of a small model: latency
        dict(name="grad_512", op="embedding_grad", tokens=512, rows=8192, dim=256, type="f32",
             ids="zipf", ids_type="i64", padding=0.0, add=False, pitch=0),
        # an ordinary training batch with padded tails
        dict(name="grad_16k", op="embedding_grad", tokens=16384, rows=65536, dim=1024,
             type="bf16", ids="zipf", ids_type="i64", padding=0.1, add=False, pitch=0),
        # a table tied to the output projection, whose gradient is there
        # already; ragged sizes, a third of the tokens padding
        dict(name="grad_tied_odd", op="embedding_grad", tokens=10007, rows=50021, dim=515,
             type="f16", ids="zipf", ids_type="i32", padding=0.3, add=True, pitch=3),
        # a long batch over a large table: a gradient of 1 GiB
        dict(name="grad_128k", op="embedding_grad", tokens=131072, rows=131072, dim=2048,
             type="bf16", ids="zipf", ids_type="i64", padding=0.0, add=False, pitch=0),
        # the norm of one step's gradients of a small network: latency
        dict(name="norm_resnet110", op="grad_norm", tensors="resnet110", count=335, n=1_730_714,
             type="f32"),
        # the norm of the benchmark's tensor: 1 GiB
        dict(name="norm_256m", op="grad_norm", tensors="one", count=1, n=1 << 28, type="f32"),
        # one step's gradients of a small network, clipped into a packed bucket
        dict(name="clip_resnet110", op="clip", tensors="resnet110", count=335, n=1_730_714,
             type="f32", limit=0.5, in_place=False),
        # a model's bf16 gradients, clipped into the fp32 tensors to compress
        dict(name="clip_100m", op="clip", tensors="log", count=148, n=100_000_000, type="bf16",
             limit=0.5, in_place=False),
    ]


def _log_int(rng, lo, hi):
    v = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    return v - 1 if v == 3072 else v


def _dim(rng):
    """Row lengths: multiples of 64 and any."""
    v = _log_int(rng, 64, 4096)
    v = v if rng.random() < 0.4 else max(64, v // 64 * 64)
    return v - 64 if v == 3072 else v


def draw(rng):
    """One more call of any operator over the listed ranges."""
    op = rng.choice(["embedding", "embedding_grad", "embedding_grad", "grad_norm", "clip"])
    types = ["f32", "bf16", "f16"]
    if op in ("embedding", "embedding_grad"):
        dim = _dim(rng)
        case = dict(op=op, dim=dim, type=rng.choice(types),
                    tokens=min(_log_int(rng, 1, 131072), 65536 * 2048 // dim),
                    rows=min(_log_int(rng, 1000, 131072), 131072 * 1024 // dim),
                    ids=rng.choice(["zipf", "zipf", "uniform", "few"]),
                    ids_type=rng.choice(["i32", "i64"]),
                    pitch=rng.choice([0, 0, 0, rng.randint(1, 16)]))
        if op == "embedding":
            case["out"] = rng.choice([case["type"], "bf16", "f32"])
        else:
            case["padding"] = rng.choice([0.0, 0.0, 0.1, 0.5])
            case["add"] = rng.choice([False, False, True])
        return case
    case = dict(op=op, tensors="log", count=rng.choice([1, rng.randint(2, 400)]),
                n=_log_int(rng, 1000, 1 << 27), type=rng.choice(types + ["mixed"]))
    if op == "clip":
        case["in_place"] = case["type"] != "mixed" and rng.random() < 0.25
        # in place the norm stays below the limit, as in most steps
        case["limit"] = 2.0 if case["in_place"] else rng.choice([0.1, 0.5, 2.0])
    return case


# ---------------------------------------------------------------- inputs
def _sizes(case):
    """Value counts of the tensors of one call."""
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
    sizes = [max(1, int(v)) for v in w / w.sum() * case["n"]]
    return [v - 1 if v == 3072 else v for v in sizes]


def _kinds(case):
    """Types of the tensors of one call."""
    k = len(_sizes(case))
    return [["bf16", "f32", "f16"][i % 3] for i in range(k)] if case["type"] == "mixed" else (
        [case["type"]] * k)


def _odds(case):
    """Probability of every id of the case's vocabulary."""
    v = case["rows"]
    if case["ids"] == "few":
        v = 3
    r = np.arange(v, dtype=np.float64)
    if case["ids"] != "zipf":
        return np.full(v, 1.0 / v)
    return np.log((r + 1 + ZIPF_SHIFT) / (r + ZIPF_SHIFT)) / math.log((v + ZIPF_SHIFT) / ZIPF_SHIFT)


def _ids(case, g):
    """Token ids: frequent ones first ("zipf"), all alike, or three in all."""
    t, v = case["tokens"], case["rows"]
    u = torch.rand(t, device="cuda", generator=g, dtype=torch.float64)
    if case["ids"] == "zipf":
        ids = ZIPF_SHIFT * ((v + ZIPF_SHIFT) / ZIPF_SHIFT) ** u - ZIPF_SHIFT
    else:
        ids = u * (v if case["ids"] == "uniform" else 3)
    ids = ids.long().clamp_(0, v - 1)
    if case.get("padding"):  # the tails of eight sequences
        at = torch.arange(t, device="cuda") * 8 % max(t, 1)
        ids = torch.where(at >= (1.0 - case["padding"]) * t, v - 1, ids)
    return ids.to(torch.int32 if case["ids_type"] == "i32" else torch.int64)


def _padding_id(case):
    return case["rows"] - 1 if case.get("padding") else -1


def _scale(dim):
    return float(np.float32(math.sqrt(dim)))


def _matrix(rows, dim, pitch, dtype, g, sigma):
    """rows x dim values; pitch > 0: in a matrix of wider rows."""
    m = torch.empty(rows, dim + pitch, device="cuda").normal_(0.0, sigma, generator=g)
    return m.to(TYPES[dtype])[:, :dim]


def _operands(case, seed):
    """The inputs alone."""
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    if case["op"] == "embedding":
        s = dict(ids=_ids(case, g), scale=_scale(case["dim"]),
                 table=_matrix(case["rows"], case["dim"], case["pitch"], case["type"], g, 0.02))
    elif case["op"] == "embedding_grad":
        s = dict(ids=_ids(case, g), scale=_scale(case["dim"]), padding_id=_padding_id(case),
                 grad=_matrix(case["tokens"], case["dim"], case["pitch"], case["type"], g, SIGMA))
        if case["add"]:
            s["table_grad"] = _matrix(case["rows"], case["dim"], 0, "f32", g, SIGMA)
        else:
            s["table_grad"] = torch.empty(case["rows"], case["dim"], device="cuda")
    else:
        sizes = _sizes(case)
        s = dict(tensors=[torch.empty(n, device="cuda").normal_(0.0, SIGMA, generator=g).to(
            TYPES[k]) for n, k in zip(sizes, _kinds(case))])
        if case["op"] == "clip":
            s["max_norm"] = float(np.float32(case["limit"] * SIGMA * math.sqrt(sum(sizes))))
            if case["in_place"]:  # the views of one flat gradient buffer
                s["bucket"] = torch.cat(s["tensors"])
                s["tensors"] = list(torch.split(s["bucket"], sizes))
    return s


_kept = {}  # the program's one context


def _context(case):
    from paper_1802_07389_amd import tlc
    if case["op"] in ("embedding", "embedding_grad"):
        need = dict(max_tokens=case["tokens"], max_rows=case["rows"], max_dim=case["dim"])
    else:
        need = dict(max_tensors=len(_sizes(case)))
    key = tuple(sorted(need.items()))
    if key not in _kept:
        _kept.clear()
        _kept[key] = tlc.TrainContext(**need)
    return _kept[key]


def prepare(case, seed):
    """Inputs and output buffers; with the framework's calls also the context
    and the list of tensors, which a program makes once and keeps."""
    s = dict(case=dict(case), **_operands(case, seed))
    if case["op"] == "embedding":
        s["out"] = torch.empty(case["tokens"], case["dim"], device="cuda",
                               dtype=TYPES[case["out"]])
    if case["op"] == "clip" and not case["in_place"]:  # fp32, packed
        sizes = _sizes(case)
        s["bucket"] = torch.empty(sum(sizes), device="cuda")
        s["outs"] = list(torch.split(s["bucket"], sizes))
    if own:
        s["ctx"] = _context(case)
        if "tensors" in s:
            s["list"] = s["ctx"].tensor_list(s["tensors"], s.get("outs"))
            s["result"] = s["ctx"].norm_result()
    return s


# ---------------------------------------------------------------- passes
def _run_own(s):
    case, ctx = s["case"], s["ctx"]
    if case["op"] == "embedding":
        return {"out": ctx.embedding(s["table"], s["ids"], scale=s["scale"], out=s["out"])}
    if case["op"] == "embedding_grad":
        ctx.embedding_grad(s["grad"], s["ids"], s["table_grad"], scale=s["scale"],
                           padding_id=s["padding_id"], accumulate=case["add"])
        return {"table_grad": s["table_grad"]}
    if case["op"] == "grad_norm":
        return {"norm": ctx.grad_norm(s["list"], result=s["result"]).norm}
    r = ctx.clip_grad_norm(s["list"], s["max_norm"], result=s["result"])
    return {"norm": r.norm, "coef": r.coef, "bucket": s["bucket"]}


def run(s):
    if own:
        return _run_own(s)
    case = s["case"]
    if case["op"] == "embedding":
        s["out"].copy_(s["table"][s["ids"]].float() * s["scale"])
        return {"out": s["out"]}
    if case["op"] == "embedding_grad":
        keep = (s["ids"] != s["padding_id"]).nonzero().squeeze(1) if case["padding"] else None
        grad = s["grad"] if keep is None else s["grad"][keep]
        ids = s["ids"] if keep is None else s["ids"][keep]
        total = torch.zeros_like(s["table_grad"]).index_add_(0, ids, grad.float())
        if case["add"]:
            s["table_grad"].add_(total.mul_(s["scale"]))
        else:
            torch.mul(total, s["scale"], out=s["table_grad"])
        return {"table_grad": s["table_grad"]}
    flat = [t.float() for t in s["tensors"]]
    flat = torch.cat(flat) if len(flat) > 1 else flat[0]
    norm = flat.square().sum().sqrt()
    if case["op"] == "grad_norm":
        return {"norm": norm}
    coef = (s["max_norm"] / norm).clamp(max=1.0)
    s["bucket"].copy_(flat * coef)
    return {"norm": norm, "coef": coef, "bucket": s["bucket"]}


# ---------------------------------------------------------------- work, 64 bits
def work(case):
    """Bytes and operations of one pass: every input read once (of a table the
    rows that are expected to be asked for), every output written once."""
    if case["op"] in ("embedding", "embedding_grad"):
        t, v, d = case["tokens"], case["rows"], case["dim"]
        kept = t * (1.0 - case.get("padding", 0.0))
        distinct = float((-np.expm1(kept * np.log1p(-_odds(case)))).sum())
        ids = t * BYTES[case["ids_type"]]
        if case["op"] == "embedding":
            return {"bytes": ids + distinct * d * BYTES[case["type"]]
                    + t * d * BYTES[case["out"]], "flops": t * d}
        table = 2 * distinct if case["add"] else v
        return {"bytes": ids + kept * d * BYTES[case["type"]] + table * d * 4,
                "flops": kept * d + distinct * d}
    n = sum(_sizes(case))
    read = sum(k * BYTES[b] for k, b in zip(_sizes(case), _kinds(case)))
    if case["op"] == "grad_norm":
        return {"bytes": read + 4, "flops": 2 * n}
    # in place, below the limit, nothing has to be written
    write = 0 if case["in_place"] else 4 * n
    return {"bytes": read + write, "flops": 3 * n}


def exact(case, seed):
    s = _operands(case, seed)
    if case["op"] == "embedding":
        return {"out": torch.index_select(s["table"].double(), 0, s["ids"]) * s["scale"]}
    if case["op"] == "embedding_grad":
        # runs of equal ids in sorted order; a run's sum is the difference of
        # the running sums at its ends, column block by column block
        order = torch.sort(s["ids"].long(), stable=True).indices
        order = order[s["ids"].long()[order] != s["padding_id"]]
        rows, runs = torch.unique_consecutive(s["ids"].long()[order], return_counts=True)
        ends = runs.cumsum(0)
        out = s["table_grad"].double() if case["add"] else torch.zeros(
            case["rows"], case["dim"], device="cuda", dtype=torch.float64)
        for c in range(0, case["dim"] if rows.numel() else 0, 256):
            sums = s["grad"][order, c:c + 256].double().cumsum(0)[ends - 1]
            sums[1:] -= sums[:-1].clone()
            out[rows, c:c + 256] += s["scale"] * sums
        return {"table_grad": out}
    norm = math.sqrt(sum(float(torch.dot(t.double(), t.double())) for t in s["tensors"]))
    if case["op"] == "grad_norm":
        return {"norm": norm}
    coef = min(1.0, s["max_norm"] / norm)
    done = [t.double() * coef for t in s["tensors"]]
    return {"norm": norm, "coef": coef, "bucket": torch.cat(done)}
