"""What a layer of a graph transformer has beside its dense products and its attention, as calls whose speed and results are
followed: the norms before and after a block with its gate and residual connection, dense layers with weights of their own for every type
of node (or expert), and the norm over all gradients with their clipping; the first two with their gradients.

A case is a dict of plain values.  listed() names the standing ones, draw() makes more of the same ranges, prepare() makes what
a program has in hand before the call, run() is one pass, work() what a pass cannot do without, exact() the same in 64 bits.
run() computes the plain form in elementary torch operations, or, where `own` is set, calls the framework.

Sizes of a case (rows of its groups, shapes of its gradients) follow from the case alone; the seed decides the values.
"""
import math
import random

import torch

own = False

DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "f16": 2, "bf16": 2}
EPS = 1e-5


def listed():
    return [
        # one node's answer: the residual connection and the next norm, a call that is all latency
        dict(name="norm_one_row", kind="norm", n=1, d=4096, block=1, post="none", pre="rms", bias=0, gate="none", dtype="bf16"),
        # layer norm in front of a block over a batch of molecules, narrow rows in fp32
        dict(name="norm_molecules", kind="norm", n=46_000, d=200, block=0, post="none", pre="layer", bias=1, gate="none", dtype="f32"),
        # between two blocks of a wide layer: norm of the block's output, learned gate, residual connection, norm for the next block
        dict(name="norm_large", kind="norm", n=50_000, d=1024, block=1, post="rms", pre="rms", bias=0, gate="vector", dtype="f16"),
        # the same as a training step, with layer norms
        dict(name="norm_train", kind="norm_train", n=20_000, d=768, block=1, post="layer", pre="layer", bias=1, gate="vector", dtype="bf16"),
        # training step with a gate for every node, narrow rows
        dict(name="norm_train_gates", kind="norm_train", n=200_000, d=128, block=1, post="none", pre="rms", bias=0, gate="rows", dtype="f16"),
        # a few nodes of a few types through small weights: latency
        dict(name="grouped_small", kind="grouped", n=37, groups=5, d_in=64, d_out=64, act="relu", bias=1, residual=0, dtype="f32"),
        # answers for 24 nodes that are spread over 64 sets of weights: what counts is reading the weights
        dict(name="grouped_few_rows", kind="grouped", n=24, groups=64, d_in=1024, d_out=4096, act="gelu", bias=1, residual=0, dtype="bf16"),
        # second product of a feed-forward block with 16 experts over 48 000 nodes
        dict(name="grouped_large", kind="grouped", n=48_000, groups=16, d_in=4096, d_out=1024, act="none", bias=1, residual=1, dtype="f16"),
        # training step of a layer with weights for each of 8 node types
        dict(name="grouped_train", kind="grouped_train", n=20_000, groups=8, d_in=768, d_out=768, act="silu", bias=1, residual=0, dtype="bf16"),
        # training step over a batch of molecules with weights for each of 118 elements, fp32
        dict(name="grouped_train_types", kind="grouped_train", n=46_000, groups=118, d_in=100, d_out=128, act="gelu", bias=1, residual=0,
             dtype="f32"),
        # gradients of a small model's two layers
        dict(name="clip_small", kind="clip", layers=2, d=64, vocab=118, types=1, scale=1.0, clips=1, dtype="f32"),
        # gradients of twelve layers and of a table of 50 000 rows, from a scaled loss
        dict(name="clip_large", kind="clip", layers=12, d=512, vocab=50_000, types=1, scale=2.0 ** -10, clips=1, dtype="f32"),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["norm", "norm_train", "grouped", "grouped_train", "clip", "grad_norm"])
    dtype = rng.choice(["f32", "f16", "bf16"])
    if kind in ("norm", "norm_train"):
        d = _log_uniform(rng, 8, 8192)
        d = d if rng.random() < 0.3 else (d + 7) // 8 * 8
        block = rng.choice([0, 1, 1]) if kind == "norm" else 1
        return dict(kind=kind, n=_log_uniform(rng, 1, min(400_000, 25_000_000 // d)), d=d, block=block,
                    post=rng.choice(["none", "rms", "layer"]) if block else "none", pre=rng.choice(["rms", "layer"]), bias=rng.choice([0, 1]),
                    gate=rng.choice(["none", "vector", "rows"]) if block else "none", dtype=dtype)
    if kind in ("grouped", "grouped_train"):
        most = 30_000_000_000 if dtype == "f32" else 100_000_000_000
        d_in, d_out = _log_uniform(rng, 8, 4096), _log_uniform(rng, 8, 4096)
        d_in, d_out = (x if rng.random() < 0.3 else (x + 7) // 8 * 8 for x in (d_in, d_out))
        return dict(kind=kind, n=_log_uniform(rng, 1, min(100_000, most // (d_in * d_out), 50_000_000 // max(d_in, d_out))),
                    groups=_log_uniform(rng, 1, max(2, min(500, 50_000_000 // (d_in * d_out)))), d_in=d_in, d_out=d_out,
                    act=rng.choice(["none", "relu", "gelu", "silu"]), bias=rng.choice([0, 1, 1]), residual=rng.choice([0, 1]), dtype=dtype)
    d = _log_uniform(rng, 8, 512)
    return dict(kind=kind, layers=_log_uniform(rng, 1, 12), d=d, vocab=_log_uniform(rng, 2, 50_000), types=rng.choice([1, 1, 4]) if d < 256 else 1,
                scale=rng.choice([1.0, 2.0 ** -10]), clips=rng.choice([0, 1, 1]), dtype=dtype)


# ---- inputs -------------------------------------------------------------------------------------------
def _generator(seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed * 1_000_003 + 31)
    return gen


def _randn(gen, dtype, *shape):
    return torch.randn(shape, generator=gen, device="cuda").to(dtype)


def _group_lengths(case):
    """Rows of every group: a few groups with many, many with few, some of many without any."""
    g, n, rng = case["groups"], case["n"], random.Random(case["groups"] * 8191 + case["n"])
    share = [rng.expovariate(1.0) ** 1.5 * (0 if g > 3 and i % 11 == 7 else 1) + (1e-9 if i == 0 else 0) for i in range(g)]
    edge, total, upto = [0], sum(share), 0.0
    for x in share:
        upto += x
        edge.append(round(n * upto / total))
    edge[-1] = n
    return [b - a for a, b in zip(edge, edge[1:])]


def _offsets(lens):
    ptr = [0]
    for x in lens:
        ptr.append(ptr[-1] + x)
    return ptr


def _gradient_shapes(case):
    """A model's weights: the table, and of each layer the products of attention and of a feed-forward block for each type, norms, biases."""
    d, t = case["d"], case["types"]
    shapes = [(case["vocab"], d)]
    for _ in range(case["layers"]):
        shapes += [(d, 3 * d), (3 * d,), (d, d), (d,), (t, d, 4 * d), (t, 4 * d), (t, 4 * d, d), (t, d), (d,), (d,), (d,)]
    return shapes


def _limit(case):
    """The largest norm: about a third of what the gradients have, or three times that."""
    entries = sum(math.prod(x) for x in _gradient_shapes(case))
    return math.sqrt(entries) * case["scale"] * (0.3 if case["clips"] else 3.0)


def _inputs(case, seed):
    gen, kind, dt = _generator(seed), case["kind"], DTYPES[case["dtype"]]
    if kind in ("norm", "norm_train"):
        n, d = case["n"], case["d"]
        weight = lambda: (1 + 0.2 * torch.randn(d, generator=gen, device="cuda")).to(dt)
        bias = lambda: (0.2 * torch.randn(d, generator=gen, device="cuda")).to(dt) if case["bias"] else None
        mean = 0.5 * torch.randn(d, generator=gen, device="cuda")  # features have means of their own
        s = dict(X=(2 * torch.randn(n, d, generator=gen, device="cuda") + mean).to(dt), pre_w=weight(), pre_b=bias(), F=None, gate=None,
                 post_w=None, post_b=None, x_scale=1.0)
        if case["block"]:
            s["F"] = _randn(gen, dt, n, d)
            if case["post"] != "none":
                s["post_w"], s["post_b"] = weight(), bias()
            if case["gate"] == "vector":
                s["gate"] = weight()
            if case["gate"] == "rows":
                s["gate"] = torch.sigmoid(torch.randn(n, d, generator=gen, device="cuda")).to(dt)
            s["x_scale"] = 0.875  # of the residual connection, as deep stacks have it
        if kind == "norm_train":
            s["dH"], s["dU"] = _randn(gen, dt, n, d), _randn(gen, dt, n, d)
        return s
    if kind in ("grouped", "grouped_train"):
        n, g, d_in, d_out = case["n"], case["groups"], case["d_in"], case["d_out"]
        s = dict(X=_randn(gen, dt, n, d_in), W=(torch.randn(g, d_in, d_out, generator=gen, device="cuda") / math.sqrt(d_in)).to(dt),
                 bias=_randn(gen, dt, g, d_out) if case["bias"] else None, residual=_randn(gen, dt, n, d_out) if case["residual"] else None,
                 edge=_offsets(_group_lengths(case)))
        s["group_ptr"] = torch.tensor(s["edge"], dtype=torch.int32, device="cuda")
        if kind == "grouped_train":
            s["d_out"] = _randn(gen, dt, n, d_out)
        return s
    # gradients of one layer are larger than another's
    return dict(grads=[(torch.randn(shape, generator=gen, device="cuda") * (0.5 + 0.5 * (i % 3))).to(dt)
                       for i, shape in enumerate(_gradient_shapes(case))], limit=_limit(case))


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = case
    if own:
        _buffers(s)
    return s


def _buffers(s):
    """Outputs, workspaces and the list of gradients, which a program makes once."""
    from paper_2412_12218_amd import binding as B
    case, L, kind, dt = s["case"], B.lib(), s["case"]["kind"], DTYPES[s["case"]["dtype"]]
    new = lambda *shape, dtype=dt: torch.empty(shape, dtype=dtype, device="cuda")
    like = lambda t: None if t is None else torch.empty_like(t)
    s["B"] = B
    if kind in ("norm", "norm_train"):
        n, d = case["n"], case["d"]
        code = dict(none=B.FTC_NORM_NONE, rms=B.FTC_NORM_RMS, layer=B.FTC_NORM_LAYER)
        s["args"] = dict(F=s["F"], x_scale=s["x_scale"], post=code[case["post"]], post_w=s["post_w"], post_b=s["post_b"], gate=s["gate"],
                         pre=code[case["pre"]], pre_w=s["pre_w"], pre_b=s["pre_b"])
        s["H"], s["U"] = new(n, d) if case["block"] else None, new(n, d)
        if kind == "norm_train":
            s["stats"] = new(n, 4, dtype=torch.float32)
            s["grads"] = dict(dX=new(n, d), dF=new(n, d), dgate=like(s["gate"]), dpost_w=like(s["post_w"]), dpost_b=like(s["post_b"]),
                              dpre_w=like(s["pre_w"]), dpre_b=like(s["pre_b"]))
            s["ws"] = B._workspace(L.ftc_block_norm_backward_workspace_bytes(n, d), "cuda")
    elif kind in ("grouped", "grouped_train"):
        sizes = case["n"], case["groups"], case["d_in"], case["d_out"]
        s["act"] = dict(none=B.FTC_ACT_NONE, relu=B.FTC_ACT_RELU, gelu=B.FTC_ACT_GELU, silu=B.FTC_ACT_SILU)[case["act"]]
        s["out"] = new(case["n"], case["d_out"])
        s["ws"] = B._workspace(max(L.ftc_grouped_linear_workspace_bytes(*sizes), L.ftc_grouped_linear_backward_workspace_bytes(*sizes)), "cuda")
        if kind == "grouped_train":
            s["slope"] = B.slope_like(s["out"]) if case["act"] != "none" else None
            s["dX"], s["dW"], s["db"] = like(s["X"]), like(s["W"]), like(s["bias"])
    else:
        s["out"], views = None, None
        if kind == "clip":  # one buffer for all of them, as ranks exchange it
            s["out"] = new(sum(g.numel() for g in s["grads"]))
            views = [v.view(g.shape) for v, g in zip(torch.split(s["out"], [g.numel() for g in s["grads"]]), s["grads"])]
        s["list"] = B.GradList(s["grads"], out=views)
        s["norm"] = new(1, dtype=torch.float32)
        s["ws"] = B._workspace(s["list"].workspace_bytes(), "cuda")


# ---- one pass -------------------------------------------------------------------------------------------
def run(s):
    if own:
        return _run_own(s)
    kind = s["case"]["kind"]
    if kind in ("norm", "norm_train"):
        return _plain_norm(s)
    return _plain_grouped(s) if kind in ("grouped", "grouped_train") else _plain_clip(s)


def _run_own(s):
    B, case, kind = s["B"], s["case"], s["case"]["kind"]
    if kind in ("norm", "norm_train"):
        H, U = B.ftc_block_norm(s["X"], H=s["H"], U=s["U"], eps=EPS, stats=s.get("stats"), **s["args"])
        out = dict(H=H, U=U) if case["block"] else dict(U=U)
        if kind == "norm_train":
            grads = B.ftc_block_norm_backward(s["X"], s["stats"], dH=s["dH"], dU=s["dU"], ws=s["ws"], **s["grads"], **s["args"])
            out.update((k, g) for k, g in grads._asdict().items() if g is not None)
        return out
    if kind in ("grouped", "grouped_train"):
        out = B.ftc_grouped_linear(s["X"], s["W"], s["group_ptr"], bias=s["bias"], act=s["act"], residual=s["residual"], out=s["out"],
                                   slope=s.get("slope"), ws=s["ws"])
        if kind == "grouped":
            return dict(out=out)
        dX, dW, db = B.ftc_grouped_linear_backward(s["X"], s["W"], s["group_ptr"], s["d_out"], slope=s["slope"], dX=s["dX"], dW=s["dW"],
                                                   db=s["db"], want_db=bool(case["bias"]), ws=s["ws"])
        return dict(out=out, dX=dX, dW=dW, db=db) if case["bias"] else dict(out=out, dX=dX, dW=dW)
    if kind == "grad_norm":
        return dict(norm=B.ftc_grad_norm(s["list"], scale=case["scale"], norm=s["norm"], ws=s["ws"]))
    norm = B.ftc_clip_grad_norm(s["list"], s["limit"], scale=case["scale"], norm=s["norm"], ws=s["ws"])
    return dict(norm=norm, grads=s["out"])


def _plain_statistics(x, kind):
    """What a row is moved by and what it is multiplied by."""
    mean = x.mean(1, keepdim=True) if kind == "layer" else torch.zeros_like(x[:, :1])
    return mean, 1 / torch.sqrt(((x - mean) ** 2).mean(1, keepdim=True) + EPS)


def _plain_norm_gradient(g, w, xh, r, kind):
    """dx, dw and db of xh w + b, xh = (x - mean) r, for the gradient g."""
    gw = g * w
    dx = gw - xh * (gw * xh).mean(1, keepdim=True)
    if kind == "layer":
        dx = dx - gw.mean(1, keepdim=True)
    return r * dx, (g * xh).double().sum(0).float(), g.double().sum(0).float()


def _plain_norm(s):
    case, dt = s["case"], s["X"].dtype
    wide = lambda t: None if t is None else t.float()
    x, f, gate, dH, dU = wide(s["X"]), wide(s["F"]), wide(s["gate"]), wide(s.get("dH")), wide(s.get("dU"))
    post_w, post_b, pre_w, pre_b = (wide(s[k]) for k in ("post_w", "post_b", "pre_w", "pre_b"))
    p = h = x
    if f is not None:
        p = f
        if post_w is not None:
            mf, rf = _plain_statistics(f, case["post"])
            fh = (f - mf) * rf
            p = fh * post_w if post_b is None else fh * post_w + post_b
        h = x * s["x_scale"] + (p if gate is None else p * gate)
    mh, rh = _plain_statistics(h, case["pre"])
    hh = (h - mh) * rh
    u = hh * pre_w if pre_b is None else hh * pre_w + pre_b
    out = dict(H=h, U=u) if f is not None else dict(U=u)
    if case["kind"] == "norm_train":
        dh, dw, db = _plain_norm_gradient(dU, pre_w, hh, rh, case["pre"])
        dh = dh + dH
        out.update(dX=dh * s["x_scale"], dpre_w=dw)
        if pre_b is not None:
            out["dpre_b"] = db
        dp = dh
        if gate is not None:
            dp, dgate = dh * gate, dh * p
            out["dgate"] = dgate if case["gate"] == "rows" else dgate.double().sum(0).float()
        out["dF"] = dp
        if post_w is not None:
            out["dF"], out["dpost_w"], db = _plain_norm_gradient(dp, post_w, fh, rf, case["post"])
            if post_b is not None:
                out["dpost_b"] = db
    return {k: v.to(dt) for k, v in out.items()}


def _activation(p, act):
    """act(p) and act'(p)."""
    if act == "relu":
        return p.clamp(min=0), (p > 0).to(p.dtype)
    if act == "gelu":
        cdf = 0.5 * (1 + torch.erf(p * math.sqrt(0.5)))
        return p * cdf, cdf + p * torch.exp(-0.5 * p * p) / math.sqrt(2 * math.pi)
    if act == "silu":
        g = 1 / (1 + torch.exp(-p))
        return p * g, g * (1 + p * (1 - g))
    return p, torch.ones_like(p)


def _plain_grouped(s):
    case, dt, X, train = s["case"], s["X"].dtype, s["X"].float(), s["case"]["kind"] == "grouped_train"
    z = torch.empty((case["n"], case["d_out"]), dtype=torch.float32, device="cuda")
    if train:
        dO = s["d_out"].float()
        dX, dW = torch.empty_like(X), torch.zeros(s["W"].shape, dtype=torch.float32, device="cuda")
        db = torch.zeros((case["groups"], case["d_out"]), dtype=torch.float32, device="cuda")
    for i, (a, b) in enumerate(zip(s["edge"], s["edge"][1:])):
        if a == b:
            continue
        W = s["W"][i].float()
        p = X[a:b] @ W
        if s["bias"] is not None:
            p = p + s["bias"][i].float()
        z[a:b], slope = _activation(p, case["act"])
        if train:
            dP = dO[a:b] * slope
            dX[a:b], dW[i], db[i] = dP @ W.t(), X[a:b].t() @ dP, dP.sum(0)
    if s["residual"] is not None:
        z = z + s["residual"].float()
    out = dict(out=z.to(dt))
    if train:
        out.update(dX=dX.to(dt), dW=dW.to(dt))
        if case["bias"]:
            out["db"] = db.to(dt)
    return out


def _plain_clip(s):
    case, total = s["case"], torch.zeros((), dtype=torch.float64, device="cuda")
    for g in s["grads"]:
        total = total + (g.double() ** 2).sum()
    norm = torch.sqrt(total) * abs(case["scale"])
    out = dict(norm=norm.float().reshape(1))
    if case["kind"] == "clip":
        factor = torch.where(norm > s["limit"], s["limit"] / norm, torch.ones_like(norm)) * case["scale"]
        out["grads"] = torch.cat([(g.double() * factor).to(g.dtype).flatten() for g in s["grads"]])
    return out


# ---- what a pass cannot do without --------------------------------------------------------------------
def work(case):
    kind, e = case["kind"], SIZE[case["dtype"]]
    if kind in ("norm", "norm_train"):
        n, d, rows = case["n"], case["d"], 2 * (1 + case["block"])
        vectors = (1 + case["bias"]) * (1 + (case["post"] != "none")) + (case["gate"] == "vector")
        rows += case["gate"] == "rows"
        if kind == "norm_train":  # two gradients in, those of the inputs out
            rows += 4 + (case["gate"] == "rows")
            vectors *= 2
        return dict(bytes=(rows * n + vectors) * d * e, flops=(8 if kind == "norm" else 30) * n * d)
    if kind in ("grouped", "grouped_train"):
        n, d_in, d_out, lens = case["n"], case["d_in"], case["d_out"], _group_lengths(case)
        used = sum(x > 0 for x in lens)  # sets of weights that some row needs
        data = n * d_in + used * (d_in + case["bias"]) * d_out + (1 + case["residual"]) * n * d_out
        if kind == "grouped":
            return dict(bytes=data * e, flops=2 * n * d_in * d_out)
        return dict(bytes=(data + n * (d_out + d_in) + case["groups"] * (d_in + case["bias"]) * d_out) * e, flops=6 * n * d_in * d_out)
    entries = sum(math.prod(x) for x in _gradient_shapes(case))
    return dict(bytes=(2 if kind == "clip" else 1) * entries * e + 4, flops=(3 if kind == "clip" else 2) * entries)


# ---- the same in 64 bits --------------------------------------------------------------------------------
def exact(case, seed):
    s, kind = _inputs(case, seed), case["kind"]
    f = torch.nn.functional
    if kind in ("norm", "norm_train"):
        wide = {k: s[k].double().requires_grad_() for k in ("X", "F", "gate", "post_w", "post_b", "pre_w", "pre_b") if s[k] is not None}

        def normed(t, which):
            w, b = wide[which + "_w"], wide.get(which + "_b")
            if case[which] == "layer":
                return f.layer_norm(t, (case["d"],), w, b, EPS)
            return f.rms_norm(t, (case["d"],), w, EPS) + (0 if b is None else b)

        h = wide["X"]
        if case["block"]:
            block = wide["F"] if case["post"] == "none" else normed(wide["F"], "post")
            h = h * s["x_scale"] + (torch.mul(block, wide["gate"]) if "gate" in wide else block)
        u = normed(h, "pre")
        out = dict(H=h.detach(), U=u.detach()) if case["block"] else dict(U=u.detach())
        if kind == "norm_train":
            names = [k for k in wide]
            grads = torch.autograd.grad([h, u], [wide[k] for k in names], [s["dH"].double(), s["dU"].double()])
            out.update(("d" + k, g) for k, g in zip(names, grads))
        return out
    if kind in ("grouped", "grouped_train"):
        X, W = s["X"].double().requires_grad_(), s["W"].double().requires_grad_()
        bias = None if s["bias"] is None else s["bias"].double().requires_grad_()
        turn = dict(none=lambda t: t, relu=f.relu, gelu=f.gelu, silu=f.silu)[case["act"]]
        parts = []
        for i, x in enumerate(torch.split(X, _group_lengths(case))):
            parts.append(turn(x.mm(W[i]) if bias is None else torch.addmm(bias[i], x, W[i])))
        z = torch.cat(parts)
        if s["residual"] is not None:
            z = z + s["residual"].double()
        if kind == "grouped":
            return dict(out=z.detach())
        leaves = [X, W] + ([bias] if case["bias"] else [])
        grads = torch.autograd.grad(z, leaves, s["d_out"].double())
        return dict(out=z.detach(), **{k: g for k, g in zip(("dX", "dW", "db"), grads)})
    norm = torch.linalg.vector_norm(torch.stack([torch.linalg.vector_norm(g.double() * case["scale"]) for g in s["grads"]]))
    out = dict(norm=norm.reshape(1))
    if kind == "clip":
        keep = min(1.0, s["limit"] / float(norm))
        out["grads"] = torch.cat([g.double().flatten() * (case["scale"] * keep) for g in s["grads"]])
    return out
