"""The graph transformer path with norms, gates, residual scale and feed-forward weights by node type, and the clipping of its gradients: all of it together against
torch's gradients in 64 bits, and captured."""
import math

import pytest
import torch

from paper_2412_12218_amd import binding as B
from paper_2412_12218_amd.models import GraphTransformerPath

pytestmark = pytest.mark.gpu
VOCAB, D, HEADS, KV, HIDDEN, OUT, LAYERS, TYPES = 30, 48, 4, 2, 80, 7, 2, 5
RMS, LAYER, NONE = B.FTC_NORM_RMS, B.FTC_NORM_LAYER, B.FTC_NORM_NONE
# norm, post_norm, gates, residual_scale, types
FORMS = [(RMS, NONE, False, 1.0, False), (LAYER, RMS, True, 0.75, True), (NONE, LAYER, True, 1.0, False), (NONE, NONE, False, 1.0, True), (RMS, LAYER, False, 0.9, True)]


def weights(dtype, form, seed=0):
    norm, post, gates, _, typed = form
    gen = torch.Generator().manual_seed(seed)
    new = lambda *s: (torch.randn(s, generator=gen) / s[-2 if len(s) > 1 else 0] ** 0.5).to(dtype).cuda()
    near_one = lambda: (1 + 0.2 * torch.randn(D, generator=gen)).to(dtype).cuda()
    kd, t = KV * D // HEADS, (TYPES,) if typed else ()

    def normed(w, name, kind):
        if kind:
            w[name] = near_one()
        if kind == LAYER:
            w[name + "_bias"] = new(D)
    layers = []
    for _ in range(LAYERS):
        w = dict(qkv=new(D, D + 2 * kd), qkv_bias=new(D + 2 * kd), out=new(D, D), out_bias=new(D), up=new(*t, D, HIDDEN), up_bias=new(*t, HIDDEN),
                 down=new(*t, HIDDEN, D), down_bias=new(*t, D))
        for block in ("attention", "feed"):
            normed(w, block + "_norm", norm)
            normed(w, block + "_post", post)
            if gates:
                w[block + "_gate"] = near_one()
        layers.append(w)
    w = dict(table=new(VOCAB, D), layers=layers, head=new(D, OUT), head_bias=new(OUT))
    normed(w, "head_norm", norm)
    return w


def flat(w):
    return [t for k, t in sorted(w.items()) if k != "layers"] + [t for l in w["layers"] for _, t in sorted(l.items())]


def batch(dtype, lens=(5, 0, 40, 1, 64, 90), seed=1):
    gen = torch.Generator().manual_seed(seed)
    n = sum(lens)
    ptr = torch.tensor([0] + list(torch.cumsum(torch.tensor(lens), 0)), dtype=torch.int32).cuda()
    ids = torch.randint(-1, VOCAB, (n,), generator=gen, dtype=torch.int32).cuda()
    mask = (torch.rand(n, generator=gen) > 0.2).to(torch.uint8).cuda()
    types = torch.randint(0, TYPES - 1, (n,), generator=gen, dtype=torch.int32).cuda()   # no node has the last type
    return lens, n, ptr, ids, mask, torch.randn((n, OUT), generator=gen).to(dtype).cuda(), types


def reference(form, lens, ids, w, mask, d_out, types):
    """Logits and gradients in 64 bits, on the CPU."""
    norm, post, gates, scale, typed = form
    wide = lambda t: t.detach().cpu().double().requires_grad_()
    w = {k: wide(v) for k, v in w.items() if k != "layers"} | dict(layers=[{k: wide(v) for k, v in l.items()} for l in w["layers"]])
    ids, mask, types, dh, f = ids.cpu().long(), mask.cpu() != 0, types.cpu().long(), D // HEADS, torch.nn.functional

    def normed(t, owner, name, kind):
        if kind == LAYER:
            return f.layer_norm(t, (D,), owner[name], owner[name + "_bias"], 1e-5)
        return f.rms_norm(t, (D,), owner[name], 1e-5) if kind else t

    def joined(h, given, l, block):
        given = normed(given, l, block + "_post", post)
        return h * scale + (given * l[block + "_gate"] if gates else given)
    h = torch.where((ids >= 0)[:, None], w["table"][ids.clamp(min=0)] * D ** 0.5, 0.0)
    for l in w["layers"]:
        q, k, v = (normed(h, l, "attention_norm", norm) @ l["qkv"] + l["qkv_bias"]).split([D, KV * dh, KV * dh], 1)
        out, at = [], 0
        for n in lens:
            s = slice(at, at + n)
            at += n
            heads = lambda t, c: t[s].view(n, c, dh).transpose(0, 1)
            qh, kh, vh = heads(q, HEADS), heads(k, KV).repeat_interleave(HEADS // KV, 0), heads(v, KV).repeat_interleave(HEADS // KV, 0)
            if not bool(mask[s].any()):
                out.append(torch.zeros((n, D), dtype=torch.float64))
                continue
            p = torch.softmax((qh @ kh.transpose(1, 2) / dh ** 0.5).masked_fill(~mask[s], -torch.inf), 2)
            out.append((p @ vh).transpose(0, 1).reshape(n, D))
        h = joined(h, torch.cat(out) @ l["out"] + l["out_bias"], l, "attention")
        x = normed(h, l, "feed_norm", norm)
        if typed:
            given = torch.stack([f.gelu(x[i] @ l["up"][t] + l["up_bias"][t]) @ l["down"][t] + l["down_bias"][t] for i, t in enumerate(types.tolist())])
        else:
            given = f.gelu(x @ l["up"] + l["up_bias"]) @ l["down"] + l["down_bias"]
        h = joined(h, given, l, "feed")
    logits = normed(h, w, "head_norm", norm) @ w["head"] + w["head_bias"]
    return logits.detach(), torch.autograd.grad(logits, flat(w), d_out.detach().cpu().double())


def path_of(form, n, ptr, types, dtype):
    norm, post, gates, scale, typed = form
    return GraphTransformerPath(ptr, n, VOCAB, D, HEADS, KV, HIDDEN, OUT, LAYERS, act_dtype=dtype, norm=norm, post_norm=post, gates=gates, residual_scale=scale,
                                types=types if typed else None, n_types=TYPES if typed else 0)


# Of the 2-norm.  A step with sums of up to 200 fp32 terms is off by (200 + 8) 2^-24 of the terms' absolute sum, some sqrt(200) times the result: 1.8e-4; a result of 16
# bits, and operands rounded to them, by 3 half steps more (fp16 1.5e-3, bf16 1.2e-2).  Some 40 steps one behind the other, whose errors are independent (sqrt 40 = 6.3), are
# amplified by at most 2 on their way.
TOL = {torch.float32: 13 * 1.8e-4, torch.float16: 13 * 1.5e-3, torch.bfloat16: 13 * 1.2e-2}


@pytest.mark.parametrize("form", FORMS, ids=str)
@pytest.mark.parametrize("dtype", list(TOL))
def test_training_step(dtype, form):
    lens, n, ptr, ids, mask, d_out, types = batch(dtype)
    w = weights(dtype, form)
    path = path_of(form, n, ptr, types, dtype)
    want, want_grads = reference(form, lens, ids, w, mask, d_out, types)
    logits = path.forward(ids, w, mask=mask)
    grads = path.backward(ids, w, d_out, mask=mask)
    assert sorted(grads) == sorted(w) and all(sorted(a) == sorted(b) for a, b in zip(grads["layers"], w["layers"]))
    off = lambda a, b: float((a.cpu().double() - b).norm() / b.norm())
    errors = [off(logits, want)] + [off(a, b) for a, b in zip(flat(grads), want_grads)]
    print(dtype, form, [f"{e:.1e}" for e in errors], flush=True)
    assert all(g.dtype == torch.float32 and g.shape == b.shape for g, b in zip(flat(grads), want_grads)) and max(errors) < TOL[dtype]
    # all of them clipped by their one norm: the product of a gradient and a factor in 64 bits, rounded once
    kept = [g.clone() for g in flat(grads)]
    total = math.sqrt(sum(float((g.double() ** 2).sum()) for g in kept))
    norm = path.clip(grads, 0.25 * total, scale=0.5)
    assert abs(norm.item() - 0.5 * total) <= 0.5 * total * 2.0 ** -23
    for a, b in zip(flat(grads), kept):
        assert bool((a.double() - b.double() * 0.25).abs().le(b.double().abs() * 0.25 * 2.0 ** -22 + 2.0 ** -149).all())


def test_captured_training_step():
    """One graph of a whole step: replays follow new ids and weights written in place, with eager work between them."""
    dtype, form = torch.float16, FORMS[1]
    lens, n, ptr, ids, mask, d_out, types = batch(dtype)
    w = weights(dtype, form)
    path, other = (path_of(form, n, ptr, types, dtype) for _ in range(2))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        path.forward(ids, w, mask=mask)
        grads = path.backward(ids, w, d_out, mask=mask)
        norm = path.clip(grads, 1.0)
    for seed in range(3):
        _, _, _, new_ids, _, new_d, _ = batch(dtype, seed=10 + seed)
        ids.copy_(new_ids)
        d_out.copy_(new_d)
        for a, b in zip(flat(w), flat(weights(dtype, form, seed=20 + seed))):
            a.copy_(b)
        path.ws.fill_(255)
        for g in flat(grads):
            g.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        logits = other.forward(ids, w, mask=mask)
        eager = other.backward(ids, w, d_out, mask=mask)
        eager_norm = other.clip(eager, 1.0)
        assert torch.equal(path.logits, logits) and torch.equal(norm, eager_norm) and all(torch.equal(a, b) for a, b in zip(flat(grads), flat(eager)))


def test_layers_that_share_weights():
    """One dict for all layers: each has gradients of its own, those of layers with equal weights."""
    dtype, form = torch.float16, FORMS[1]
    lens, n, ptr, ids, mask, d_out, types = batch(dtype)
    w = weights(dtype, form)
    one = w | dict(layers=[w["layers"][0]] * LAYERS)
    equal = w | dict(layers=[dict(w["layers"][0]) for _ in range(LAYERS)])
    grads = []
    for v in (one, equal):
        path = path_of(form, n, ptr, types, dtype)
        path.forward(ids, v, mask=mask)
        grads.append(path.backward(ids, v, d_out, mask=mask))
    assert all(sorted(g) == sorted(w["layers"][0]) for g in grads[0]["layers"])
    assert all(torch.equal(a, b) for a, b in zip(flat(grads[0]), flat(grads[1])))


@pytest.mark.parametrize("lens", [(), (0, 0), (1,)])
def test_smallest_batches(lens):
    """No graph, graphs without a node, one node."""
    dtype, form = torch.float16, FORMS[1]
    gen = torch.Generator().manual_seed(2)
    n, w = sum(lens), weights(dtype, form)
    ptr = torch.tensor([0] + list(torch.cumsum(torch.tensor(lens, dtype=torch.int64), 0)), dtype=torch.int32).cuda()
    ids, types = (torch.randint(0, TYPES, (n,), generator=gen, dtype=torch.int32).cuda() for _ in range(2))
    d_out, mask = torch.randn((n, OUT), generator=gen).to(dtype).cuda(), torch.ones(n, dtype=torch.uint8).cuda()
    path = path_of(form, n, ptr, types, dtype)
    logits = path.forward(ids, w)
    grads = path.backward(ids, w, d_out)
    norm = path.clip(grads, 1.0)
    if n:
        want, want_grads = reference(form, lens, ids, w, mask, d_out, types)
        assert float((logits.cpu().double() - want).norm() / want.norm()) < TOL[dtype]
        total = math.sqrt(sum(float((g ** 2).sum()) for g in want_grads))
        assert abs(norm.item() - total) < TOL[dtype] * total
    else:
        assert logits.shape == (0, OUT) and norm.item() == 0 and not any(bool(g.any()) for g in flat(grads))


def test_types_are_checked():
    _, n, ptr, _, _, _, types = batch(torch.float16)
    for bad in (types + 1, types - 1, types[:-1]):
        with pytest.raises(ValueError):
            GraphTransformerPath(ptr, n, VOCAB, D, HEADS, types=bad, n_types=TYPES - 1)
