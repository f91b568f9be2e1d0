"""The graph transformer path: lookup, layers, head and all gradients together, against torch's in 64 bits, captured, and by differences."""
import pytest
import torch

from paper_2412_12218_amd.models import GraphTransformerPath

pytestmark = pytest.mark.gpu
VOCAB, D, HEADS, KV, HIDDEN, OUT, LAYERS = 30, 48, 4, 2, 80, 7, 2


def weights(dtype, seed=0):
    gen = torch.Generator().manual_seed(seed)
    new = lambda *s: (torch.randn(s, generator=gen) / s[0] ** 0.5).to(dtype).cuda()
    kd = KV * D // HEADS
    layer = lambda: dict(qkv=new(D, D + 2 * kd), qkv_bias=new(D + 2 * kd), out=new(D, D), out_bias=new(D), up=new(D, HIDDEN), up_bias=new(HIDDEN),
                         down=new(HIDDEN, D), down_bias=new(D))
    return dict(table=new(VOCAB, D), layers=[layer() for _ in range(LAYERS)], head=new(D, OUT), head_bias=new(OUT))


def flat(w):
    return [w["table"], w["head"], w["head_bias"]] + [t for l in w["layers"] for _, t in sorted(l.items())]


def batch(dtype, lens=(5, 0, 40, 1, 64, 90), seed=1):
    gen = torch.Generator().manual_seed(seed)
    n = sum(lens)
    ptr = torch.tensor([0] + list(torch.cumsum(torch.tensor(lens), 0)), dtype=torch.int32).cuda()
    ids = torch.randint(-1, VOCAB, (n,), generator=gen, dtype=torch.int32).cuda()
    mask = (torch.rand(n, generator=gen) > 0.2).to(torch.uint8).cuda()
    return lens, n, ptr, ids, mask, torch.randn((n, OUT), generator=gen).to(dtype).cuda()


def reference(lens, ids, w, mask, d_out):
    """Logits and gradients in 64 bits, on the CPU."""
    wide = lambda t: t.detach().cpu().double().requires_grad_()
    w = dict(table=wide(w["table"]), head=wide(w["head"]), head_bias=wide(w["head_bias"]), layers=[{k: wide(v) for k, v in l.items()} for l in w["layers"]])
    ids, mask, dh = ids.cpu().long(), mask.cpu() != 0, D // HEADS
    h = torch.where((ids >= 0)[:, None], w["table"][ids.clamp(min=0)] * D ** 0.5, 0.0)
    for l in w["layers"]:
        q, k, v = (h @ l["qkv"] + l["qkv_bias"]).split([D, KV * dh, KV * dh], 1)
        out, at = [], 0
        for n in lens:
            if n == 0:
                continue
            s = slice(at, at + n)
            at += n
            heads = lambda t, c: t[s].view(n, c, dh).transpose(0, 1)
            qh, kh, vh = heads(q, HEADS), heads(k, KV).repeat_interleave(HEADS // KV, 0), heads(v, KV).repeat_interleave(HEADS // KV, 0)
            if not bool(mask[s].any()):
                out.append(torch.zeros((n, D), dtype=torch.float64))
                continue
            p = torch.softmax((qh @ kh.transpose(1, 2) / dh ** 0.5).masked_fill(~mask[s], -torch.inf), 2)
            out.append((p @ vh).transpose(0, 1).reshape(n, D))
        h = h + torch.cat(out) @ l["out"] + l["out_bias"]
        h = h + torch.nn.functional.gelu(h @ l["up"] + l["up_bias"]) @ l["down"] + l["down_bias"]
    logits = h @ w["head"] + w["head_bias"]
    return logits.detach(), torch.autograd.grad(logits, flat(w), d_out.detach().cpu().double())


# Of the 2-norm.  A step with sums of up to 154 fp32 terms is off by (154 + 8) 2^-24 of the terms' absolute sum, some sqrt(154) times the
# result: 1.2e-4; a result of 16 bits, and operands rounded to them, by 3 half steps more (fp16 1.5e-3, bf16 1.2e-2).  Some 20 steps one behind
# the other, whose errors are independent (sqrt 20 = 4.5), are amplified by at most 2 on their way (the residual connections carry
# them on with weight one, the blocks add their own slope times them).
TOL = {torch.float32: 9 * 1.2e-4, torch.float16: 9 * 1.5e-3, torch.bfloat16: 9 * 1.2e-2}


@pytest.mark.parametrize("dtype", list(TOL))
def test_forward_and_gradients(dtype):
    lens, n, ptr, ids, mask, d_out = batch(dtype)
    w = weights(dtype)
    path = GraphTransformerPath(ptr, n, VOCAB, D, HEADS, KV, HIDDEN, OUT, LAYERS, act_dtype=dtype)
    want, want_grads = reference(lens, ids, w, mask, d_out)
    logits = path.forward(ids, w, mask=mask)
    grads = flat(path.backward(ids, w, d_out, mask=mask))
    off = lambda a, b: float((a.cpu().double() - b).norm() / b.norm())
    errors = [off(logits, want)] + [off(a, b) for a, b in zip(grads, want_grads)]
    print(dtype, [f"{e:.1e}" for e in errors], flush=True)
    assert all(g.dtype == torch.float32 for g in grads) and max(errors) < TOL[dtype]


def test_captured_training_step():
    """One graph of the whole step: replays follow new ids and weights written in place, with eager work between them."""
    dtype = torch.float16
    lens, n, ptr, ids, mask, d_out = batch(dtype)
    w = weights(dtype)
    path = GraphTransformerPath(ptr, n, VOCAB, D, HEADS, KV, HIDDEN, OUT, LAYERS, act_dtype=dtype)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        path.forward(ids, w, mask=mask)
        grads = flat(path.backward(ids, w, d_out, mask=mask))
    other = GraphTransformerPath(ptr, n, VOCAB, D, HEADS, KV, HIDDEN, OUT, LAYERS, act_dtype=dtype)
    for seed in range(3):
        _, _, _, new_ids, _, new_d = batch(dtype, seed=10 + seed)
        ids.copy_(new_ids)
        d_out.copy_(new_d)
        for a, b in zip(flat(w), flat(weights(dtype, seed=20 + seed))):
            a.copy_(b)
        path.ws.fill_(255)
        for g in grads:
            g.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        logits = other.forward(ids, w, mask=mask)
        eager = flat(other.backward(ids, w, d_out, mask=mask))
        assert torch.equal(path.logits, logits) and all(torch.equal(a, b) for a, b in zip(grads, eager))


def test_two_paths_on_two_streams():
    """Two programs at once, each with its own buffers and workspace."""
    dtype = torch.bfloat16
    lens, n, ptr, ids, mask, d_out = batch(dtype)
    w = weights(dtype)
    paths = [GraphTransformerPath(ptr, n, VOCAB, D, HEADS, KV, HIDDEN, OUT, LAYERS, act_dtype=dtype) for _ in range(3)]
    paths[0].forward(ids, w, mask=mask)
    want = flat(paths[0].backward(ids, w, d_out, mask=mask))
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = []
    for s, p in zip(streams, paths[1:]):
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            p.forward(ids, w, mask=mask)
            got.append(flat(p.backward(ids, w, d_out, mask=mask)))
    torch.cuda.synchronize()
    for p, grads in zip(paths[1:], got):
        assert torch.equal(p.logits, paths[0].logits) and all(torch.equal(a, b) for a, b in zip(grads, want))
