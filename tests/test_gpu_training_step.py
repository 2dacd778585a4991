"""The training-step operators one after the other, as a program uses them: a
table of next-token logits is looked up, the loss, its gradient, the table's
gradient and their norm are formed, pushed through the codec, and the server's
AdamW step gives the change that is pulled.
"""
import importlib.util
import math
import os

import numpy as np
import pytest
import torch

import adamw_ref as ref

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
ROWS, TOKENS, WORKERS = 515, 1500, 2
RATES = dict(lr=1e-2, beta1=0.9, beta2=0.99, eps=1e-8, weight_decay=0.1)
U = 2.0 ** -24


def T():
    from paper_1802_07389_amd import tlc
    return tlc


def tokens(seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    ids = torch.randint(0, ROWS, (TOKENS,), device="cuda", generator=g)
    target = (ids * 3 + torch.randint(0, 4, (TOKENS,), device="cuda", generator=g)) % ROWS
    return ids, torch.where(torch.rand(TOKENS, device="cuda", generator=g) < 0.2, -100, target)


def worker_step(ctx, table, ids, target, grad):
    """Loss and the table's gradient of the logits table[ids]."""
    logits = ctx.embedding(table, ids)
    r = ctx.token_logprobs(logits, target)
    each = torch.full((TOKENS,), -1.0 / TOKENS, device="cuda")
    g = ctx.token_logprobs_grad(logits, target, r, each, out=logits)
    ctx.embedding_grad(g, ids, grad)
    return r


def reference(table, ids, target):
    t = table.double().requires_grad_(True)
    lp = torch.log_softmax(t[ids], 1)
    keep = target != -100
    picked = lp[torch.arange(TOKENS, device="cuda"), target.clamp(min=0)]
    loss = -(picked * keep).sum() / TOKENS
    loss.backward()
    return float(loss.detach()), t.grad


@pytest.mark.parametrize("bits", [32, 8])
def test_push_step_and_pull(bits):
    """Bars: a token's gradient is off by 32 U of p or 1 (the logits are within 10
    of the largest, the sum has 515 / 256 + 64 roundings at most: 160 U), the
    table's row, a sum of at most 40 of them in fp32, by 200 U of the sum of their
    magnitudes."""
    tlc = T()
    g = torch.Generator(device="cuda").manual_seed(0)
    model = torch.randn(ROWS, ROWS, device="cuda", generator=g)
    copies = [model.clone() for _ in range(WORKERS)]
    ctx = tlc.TrainContext(max_tokens=TOKENS, max_rows=ROWS, max_dim=ROWS, max_tensors=1)
    n = model.numel()
    codecs = [tlc.Context(max_n=WORKERS * n, max_tensors=WORKERS) for _ in range(WORKERS + 1)]
    residuals = [torch.zeros_like(model) for _ in range(WORKERS + 1)]
    total = torch.empty_like(model)
    weights = ctx.adamw_list([model], [total], bits=bits, deltas=[total])
    grad = torch.empty_like(model)
    for step in range(1, 4):
        pushed = []
        for k in range(WORKERS):
            ids, target = tokens(10 * step + k)
            r = worker_step(ctx, copies[k], ids, target, grad)
            ctx.sync()
            loss, want = reference(copies[k], ids, target)
            got = -float(r.logprob.double().sum()) / TOKENS
            assert abs(got - loss) <= 300 * U * max(1.0, loss)
            bar = 200 * U * (want.abs() + 40.0 / TOKENS)
            assert bool(((grad.double() - want).abs() <= bar).all())
            pushed.append(codecs[k].compress(grad.view(-1), residuals[k].view(-1), 1.0))
            pushed[-1] = (pushed[-1][0].clone(), pushed[-1][1])
        server = codecs[-1]
        server.decompress_sum([c for c, _ in pushed], [m for _, m in pushed], total.view(-1))
        server.sync()
        norm = ctx.grad_norm([total])
        ctx.sync()
        coef = min(1.0, float(np.float32(0.05)) / math.sqrt(float(norm.sumsq)))
        f = ref.factors(step, **RATES)
        p0, g0 = ref.numpy_of(model), ref.numpy_of(total)
        if bits == 32:
            m, v = ref.numpy_of(weights.exp_avgs[0]), ref.numpy_of(weights.exp_avg_sqs[0])
        else:
            s = weights.scales[0].cpu().numpy()
            m = ref.decode(weights.exp_avgs[0].view(torch.uint8).cpu(), torch.float8_e4m3fn, s, 0)
            v = ref.decode(weights.exp_avg_sqs[0].view(torch.uint8).cpu(), torch.float8_e5m2, s, 1)
        new, _, _ = ref.fp32_step(p0, g0, m, v, np.float32(coef), f)
        ctx.adamw(weights, max_norm=0.05, result=norm, **RATES)
        ctx.sync()
        assert np.array_equal(ref.numpy_of(model), new)
        assert np.array_equal(ref.numpy_of(total), new - p0)
        # what is pulled and what stays behind are the change
        before = residuals[-1] + total
        c, scale = server.compress(total.view(-1), residuals[-1].view(-1), 1.0)
        for k in range(WORKERS):
            codecs[k].decompress(c, scale, n, copies[k].view(-1), accumulate=True)
            codecs[k].sync()
        sent = torch.zeros_like(model)
        server.decompress(c, scale, n, sent.view(-1))
        server.sync()
        assert torch.equal(before - sent, residuals[-1])
        assert torch.equal(copies[0], copies[1])
    for c in codecs:
        c.close()
    ctx.close()


@pytest.mark.parametrize("bits", [32, 8])
def test_captured_training_step(bits):
    """A whole step in a graph, replayed beside eager steps of a twin."""
    tlc = T()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        ctx = tlc.TrainContext(max_tokens=TOKENS, max_rows=ROWS, max_dim=ROWS, max_tensors=1)
        g = torch.Generator(device="cuda").manual_seed(1)
        tables = [torch.randn(ROWS, ROWS, device="cuda", generator=g)]
        tables.append(tables[0].clone())
        grads = [torch.empty_like(t) for t in tables]
        lists = [ctx.adamw_list([t], [d], bits=bits) for t, d in zip(tables, grads)]
        norms = [ctx.norm_result() for _ in tables]
        ids, target = tokens(3)
        logits = torch.empty(TOKENS, ROWS, device="cuda")
        result = ctx.token_result(TOKENS, 3)
        each = torch.full((TOKENS,), -1.0 / TOKENS, device="cuda")

        def step(k):
            ctx.embedding(tables[k], ids, out=logits)
            ctx.token_logprobs(logits, target, top=3, out=result)
            ctx.token_logprobs_grad(logits, target, result, each, out=logits)
            ctx.embedding_grad(logits, ids, grads[k])
            ctx.grad_norm([grads[k]], result=norms[k])
            ctx.adamw(lists[k], max_norm=0.01, result=norms[k], **RATES)

        step(0)
        step(1)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        step(0)
    for k in range(4):
        with torch.cuda.stream(s):
            new_ids, new_target = tokens(20 + k)
            ids.copy_(new_ids)
            target.copy_(new_target)
            step(1)
            want = result.buffer.clone(), result.top_ids.clone()
            graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(tables[0], tables[1]), k
        assert torch.equal(lists[0].clock, lists[1].clock) and int(lists[0].step) == 2 + k
        assert torch.equal(result.buffer, want[0]) and torch.equal(result.top_ids, want[1])
        assert float(norms[0].norm) == float(norms[1].norm)
    ctx.sync()
    ctx.close()


def example():
    spec = importlib.util.spec_from_file_location(
        "embedding_training", os.path.join(ROOT, "examples", "embedding_training.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def test_the_example_runs_with_adamw():
    losses, share = example().train(steps=3, report=lambda text: None, adamw=True)
    assert all(math.isfinite(x) for x in losses) and 0 < share < 1.6 / 8


def test_the_examples_gradients():
    """The library's loss and torch's on the same hidden states: logits of both
    are bf16, so a probability may differ by its exponent's step, 2^-8 of |logit|,
    on either side, and the products by bf16's half step a term and once more."""
    ex = example()
    g = torch.Generator(device="cuda").manual_seed(4)
    model = [torch.randn(ex.ROWS, ex.DIM, device="cuda", generator=g) / ex.DIM,
             torch.randn(ex.DIM, ex.ROWS, device="cuda", generator=g) / ex.DIM]
    a, b = ex.Worker(model, 1, own_loss=True), ex.Worker(model, 1)
    h = torch.randn(512, ex.DIM, device="cuda", generator=g).bfloat16()
    w = torch.randn(ex.DIM, ex.ROWS, device="cuda", generator=g).bfloat16() / 8
    target = torch.randint(0, ex.ROWS, (512,), device="cuda", generator=g)
    target[::9] = ex.PADDING
    la, ha, wa = a.loss(h.clone(), w.clone(), target)
    lb, hb, wb = b.loss(h, w, target)
    assert abs(float(la) - float(lb)) <= 1e-4 * float(lb)
    for x, y in ((ha, hb), (wa, wb)):
        assert float((x.double() - y.double()).norm()) <= 2 ** -6 * float(y.double().norm())
