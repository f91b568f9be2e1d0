"""Operators of a graph transformer, as calls whose speed and results are followed: node embeddings, the dense update with
bias, activation and residual, and attention between all nodes of a graph over a packed batch, each with its gradients.

A case is a dict of plain values.  listed() names the standing ones, draw() makes more of the same ranges, prepare() makes what
a program has in hand before the call, run() is one pass, work() what a pass cannot do without, exact() the same in 64 bits.
run() computes the plain form in elementary torch operations, or, where `own` is set, calls the framework.

Sizes of a case (lengths of its graphs among them) follow from the case alone; the seed decides the values.
"""
import math
import random

import torch

own = False

DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "f16": 2, "bf16": 2}


def listed():
    return [
        # ids of one small graph (37 atoms of 118 elements): a call that is all latency
        dict(name="lookup_small", kind="lookup", n=37, vocab=118, d=64, pad=0, dtype="f32"),
        # learned features of a sampled mini-batch out of 200 000 nodes
        dict(name="lookup_large", kind="lookup", n=300_000, vocab=200_000, d=128, pad=0, dtype="f16"),
        # gradient of 118 node types over a batch of molecules: few rows, long runs, padded ids among them
        dict(name="lookup_grad_types", kind="lookup_grad", n=46_000, vocab=118, d=200, pad=1, dtype="f32"),
        # gradient of a table of 50 000 rows by ids of a power law, as tokens and node popularity have it
        dict(name="lookup_grad_tokens", kind="lookup_grad", n=131_072, vocab=50_000, d=512, pad=0, dtype="bf16"),
        # the answer for one node: a single row through a wide layer
        dict(name="linear_one_row", kind="linear", n=1, d_in=1024, d_out=4096, act="gelu", bias=1, residual=0, dtype="bf16"),
        # first layer over the 1433 bag-of-words features of a citation network: odd rows, fp32
        dict(name="linear_citation", kind="linear", n=2708, d_in=1433, d_out=128, act="relu", bias=1, residual=0, dtype="f32"),
        # inner layer of a feed-forward block over 65 536 nodes
        dict(name="linear_large", kind="linear", n=65_536, d_in=1024, d_out=4096, act="gelu", bias=1, residual=0, dtype="f16"),
        # training step of a layer with a residual connection
        dict(name="linear_train", kind="linear_train", n=20_000, d_in=768, d_out=768, act="silu", bias=1, residual=1,
             dtype="bf16"),
        # readout: one query a graph over up to 20 000 nodes, K/V heads shared by four query heads
        dict(name="attention_readout", kind="attention", graphs=12, length=10_000, queries=1, heads=8, kv_heads=2, d=64, masked=0,
             dtype="f16"),
        # a batch of molecules in fp32, some nodes masked and one graph wholly
        dict(name="attention_molecules", kind="attention", graphs=2000, length=23, queries=0, heads=4, kv_heads=4, d=20, masked=1,
             dtype="f32"),
        # training step on mid-sized graphs of very different sizes
        dict(name="attention_train", kind="attention_train", graphs=48, length=400, queries=0, heads=8, kv_heads=8, d=64, masked=1,
             dtype="bf16"),
        # training step on a few large graphs
        dict(name="attention_train_large", kind="attention_train", graphs=5, length=4000, queries=0, heads=12, kv_heads=4, d=128,
             masked=0, dtype="f16"),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["lookup", "lookup_grad", "linear", "linear_train", "attention", "attention_train"])
    dtype = rng.choice(["f32", "f16", "bf16"])
    if kind in ("lookup", "lookup_grad"):
        d = _log_uniform(rng, 1, 1024)
        return dict(kind=kind, n=_log_uniform(rng, 1, min(400_000, 60_000_000 // d)),
                    vocab=_log_uniform(rng, 2, min(200_000, 60_000_000 // d)), d=d, pad=rng.choice([0, 1]), dtype=dtype)
    if kind in ("linear", "linear_train"):
        most = 30_000_000_000 if dtype == "f32" else 150_000_000_000
        d_in, d_out = _log_uniform(rng, 8, 4096), _log_uniform(rng, 1, 4096)
        d_in, d_out = (x if rng.random() < 0.3 else (x + 7) // 8 * 8 for x in (d_in, d_out))
        return dict(kind=kind, n=_log_uniform(rng, 1, min(100_000, most // (d_in * d_out))), d_in=d_in, d_out=d_out,
                    act=rng.choice(["none", "relu", "gelu", "silu"]), bias=rng.choice([0, 1, 1]), residual=rng.choice([0, 1]),
                    dtype=dtype)
    d = rng.choice([8, 16, 20, 32, 37, 40, 64, 64, 80, 96, 128, 128])
    kv_heads = rng.choice([1, 2, 3, 4, 8])
    heads = kv_heads * rng.choice([1, 1, 2, 3, 4])
    graphs = _log_uniform(rng, 1, 2000)
    queries = rng.choice([0, 0, 1, 3])
    room = (150_000_000 if dtype == "f32" else 500_000_000) // (graphs * heads)  # pairs of a head of a padded graph
    if queries:
        length = _log_uniform(rng, 1, min(30_000, 20_000_000 // (graphs * heads * d)) + 1)
    else:
        length = _log_uniform(rng, 1, max(1, min(4000, int(math.sqrt(room) / 2))))
    return dict(kind=kind, graphs=graphs, length=length, queries=queries, heads=heads, kv_heads=kv_heads, d=d,
                masked=rng.choice([0, 1]), dtype=dtype)


# ---- inputs -------------------------------------------------------------------------------------------
def _generator(seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed * 1_000_003 + 29)
    return gen


def _lengths(case):
    """Nodes of every graph: 1 .. 2 length - 1, evenly spread in a shuffled order; every 13th of many graphs has none."""
    g, rng = case["graphs"], random.Random(case["graphs"] * 8191 + case["length"])
    lens = [1 + round((2 * case["length"] - 2) * (i + 0.5) / g) for i in range(g)]
    rng.shuffle(lens)
    return [0 if i % 13 == 12 else x for i, x in enumerate(lens)]


def _query_lengths(case):
    return [case["queries"]] * case["graphs"] if case["queries"] else _lengths(case)


def _offsets(lens):
    ptr = [0]
    for x in lens:
        ptr.append(ptr[-1] + x)
    return torch.tensor(ptr, dtype=torch.int32, device="cuda")


def _randn(gen, dtype, *shape):
    return torch.randn(shape, generator=gen, device="cuda").to(dtype)


def _ids(case, gen):
    """Ids of a power law over a shuffled numbering; with `pad`, every 16th or so is -1 (a padded place)."""
    n, vocab = case["n"], case["vocab"]
    weight = torch.arange(1, vocab + 1, device="cuda", dtype=torch.float64) ** -0.8
    cdf = torch.cumsum(weight, 0)
    u = torch.rand(n, generator=gen, device="cuda", dtype=torch.float64) * cdf[-1]
    rank = torch.searchsorted(cdf, u).clamp_(max=vocab - 1)
    ids = torch.randperm(vocab, generator=gen, device="cuda")[rank]
    if case["pad"]:
        ids = torch.where(torch.rand(n, generator=gen, device="cuda") < 1 / 16, -torch.ones_like(ids), ids)
    return ids.to(torch.int32)


def _inputs(case, seed):
    gen, kind, dt = _generator(seed), case["kind"], DTYPES[case["dtype"]]
    if kind in ("lookup", "lookup_grad"):
        s = dict(ids=_ids(case, gen), scale=math.sqrt(case["d"]))  # the usual factor of tied embeddings
        if kind == "lookup":
            s["E"] = _randn(gen, dt, case["vocab"], case["d"])
        else:
            s["d_out"] = _randn(gen, dt, case["n"], case["d"])
        return s
    if kind in ("linear", "linear_train"):
        n, d_in, d_out = case["n"], case["d_in"], case["d_out"]
        s = dict(X=_randn(gen, dt, n, d_in), W=(torch.randn(d_in, d_out, generator=gen, device="cuda") / math.sqrt(d_in)).to(dt),
                 bias=_randn(gen, dt, d_out) if case["bias"] else None,
                 residual=_randn(gen, dt, n, d_out) if case["residual"] else None)
        if kind == "linear_train":
            s["d_out"] = _randn(gen, dt, n, d_out)
        return s
    lens, qlens, hd, kd = _lengths(case), _query_lengths(case), case["heads"] * case["d"], case["kv_heads"] * case["d"]
    n_kv, n_q = sum(lens), sum(qlens)
    s = dict(kv_ptr=_offsets(lens), longest=max(lens), scale=1.0 / math.sqrt(case["d"]), mask=None)
    if case["queries"]:  # queries of their own; keys and values out of one product
        s["q_ptr"], s["longest_q"] = _offsets(qlens), max(qlens)
        s["Q"] = _randn(gen, dt, n_q, hd)
        kv = _randn(gen, dt, n_kv, 2 * kd)
        s["K"], s["V"] = kv[:, :kd], kv[:, kd:]
    else:  # queries, keys and values out of one product
        s["q_ptr"], s["longest_q"] = s["kv_ptr"], s["longest"]
        qkv = _randn(gen, dt, n_kv, hd + 2 * kd)
        s["Q"], s["K"], s["V"] = qkv[:, :hd], qkv[:, hd:hd + kd], qkv[:, hd + kd:]
    if case["masked"]:
        mask = torch.rand(n_kv, generator=gen, device="cuda") >= 0.1
        mask[:lens[0]] = len(lens) == 1  # the first of several graphs wholly
        s["mask"] = mask.to(torch.uint8)
    if kind == "attention_train":
        s["d_out"] = _randn(gen, dt, n_q, hd)
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = case
    if own:
        _buffers(s)
    return s


def _buffers(s):
    """Outputs and workspaces, which a program allocates once."""
    from paper_2412_12218_amd import binding as B
    case, L, kind, dt = s["case"], B.lib(), s["case"]["kind"], DTYPES[s["case"]["dtype"]]
    new = lambda *shape, dtype=dt: torch.empty(shape, dtype=dtype, device="cuda")
    s["B"] = B
    if kind == "lookup":
        s["out"] = new(case["n"], case["d"])
    elif kind == "lookup_grad":
        s["dE"] = new(case["vocab"], case["d"])
        s["ws"] = B._workspace(L.ftc_embedding_backward_workspace_bytes(case["n"], case["vocab"], case["d"]), "cuda")
    elif kind in ("linear", "linear_train"):
        n, d_in, d_out = case["n"], case["d_in"], case["d_out"]
        s["act"] = dict(none=B.FTC_ACT_NONE, relu=B.FTC_ACT_RELU, gelu=B.FTC_ACT_GELU, silu=B.FTC_ACT_SILU)[case["act"]]
        s["out"] = new(n, d_out)
        s["ws"] = B._workspace(max(L.ftc_linear_workspace_bytes(n, d_in, d_out), L.ftc_linear_backward_workspace_bytes(n, d_in, d_out)),
                               "cuda")
        if kind == "linear_train":
            s["slope"] = B.slope_like(s["out"]) if case["act"] != "none" else None
            s["dX"], s["dW"] = new(n, d_in), new(d_in, d_out)
            s["db"] = new(d_out) if case["bias"] else None
    else:
        n_q, n_kv, heads, d = s["Q"].shape[0], s["K"].shape[0], case["heads"], case["d"]
        sizes = (n_q, n_kv, case["graphs"], heads, case["kv_heads"], d)
        s["out"] = new(n_q, heads * d)
        s["ws"] = B._workspace(max(L.ftc_graph_attention_workspace_bytes(*sizes), L.ftc_graph_attention_backward_workspace_bytes(*sizes)),
                               "cuda")
        if kind == "attention_train":
            s["lse"] = new(n_q, heads, dtype=torch.float32)
            s["dQ"], s["dK"], s["dV"] = new(n_q, heads * d), new(n_kv, s["K"].shape[1]), new(n_kv, s["K"].shape[1])


# ---- one pass -------------------------------------------------------------------------------------------
def run(s):
    if own:
        return _run_own(s)
    kind = s["case"]["kind"]
    if kind == "lookup":
        return _plain_lookup(s)
    if kind == "lookup_grad":
        return _plain_lookup_grad(s)
    return _plain_linear(s) if kind in ("linear", "linear_train") else _plain_attention(s)


def _run_own(s):
    B, case, kind = s["B"], s["case"], s["case"]["kind"]
    dt = DTYPES[case["dtype"]]
    if kind == "lookup":
        return dict(out=B.ftc_embedding(s["ids"], s["E"], scale=s["scale"], out=s["out"]))
    if kind == "lookup_grad":
        return dict(dE=B.ftc_embedding_backward(s["ids"], s["d_out"], case["vocab"], scale=s["scale"], dE=s["dE"], ws=s["ws"]))
    if kind == "linear":
        return dict(out=B.ftc_linear(s["X"], s["W"], bias=s["bias"], act=s["act"], residual=s["residual"], out=s["out"], ws=s["ws"]))
    if kind == "linear_train":
        out = B.ftc_linear(s["X"], s["W"], bias=s["bias"], act=s["act"], residual=s["residual"], out=s["out"], slope=s["slope"], ws=s["ws"])
        dX, dW, db = B.ftc_linear_backward(s["X"], s["W"], s["d_out"], slope=s["slope"], dX=s["dX"], dW=s["dW"], db=s["db"],
                                           want_db=bool(case["bias"]), ws=s["ws"])
        return dict(out=out, dX=dX, dW=dW, db=db) if case["bias"] else dict(out=out, dX=dX, dW=dW)
    heads = dict(heads=case["heads"], kv_heads=case["kv_heads"], scale=s["scale"], kv_mask=s["mask"], ws=s["ws"])
    if kind == "attention":
        return dict(out=B.ftc_graph_attention(s["Q"], s["K"], s["V"], s["q_ptr"], s["kv_ptr"], out=s["out"], **heads))
    out = B.ftc_graph_attention(s["Q"], s["K"], s["V"], s["q_ptr"], s["kv_ptr"], out=s["out"], lse=s["lse"], **heads)
    dQ, dK, dV = B.ftc_graph_attention_backward(s["Q"], s["K"], s["V"], s["q_ptr"], s["kv_ptr"], out, s["lse"], s["d_out"],
                                                dQ=s["dQ"], dK=s["dK"], dV=s["dV"], **heads)
    return dict(out=out, dQ=dQ, dK=dK, dV=dV)


def _plain_lookup(s):
    ids, E = s["ids"].long(), s["E"]
    rows = E[ids.clamp(min=0)].float() * s["scale"]
    return dict(out=torch.where((ids >= 0)[:, None], rows, torch.zeros_like(rows)).to(E.dtype))


def _plain_lookup_grad(s):
    ids, g, vocab = s["ids"].long(), s["d_out"], s["case"]["vocab"]
    dE = torch.zeros((vocab + 1, g.shape[1]), dtype=torch.float32, device="cuda")  # the last row takes the padded places
    dE.index_add_(0, torch.where(ids >= 0, ids, vocab), g.float())
    return dict(dE=(dE[:vocab] * s["scale"]).to(g.dtype))


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


def _plain_linear(s):
    case, X, W = s["case"], s["X"].float(), s["W"].float()
    dt = s["X"].dtype
    p = X @ W
    if s["bias"] is not None:
        p = p + s["bias"].float()
    a, slope = _activation(p, case["act"])
    out = dict(out=(a if s["residual"] is None else a + s["residual"].float()).to(dt))
    if case["kind"] == "linear_train":
        dP = s["d_out"].float() * slope
        out.update(dX=(dP @ W.t()).to(dt), dW=(X.t() @ dP).to(dt))
        if case["bias"]:
            out["db"] = dP.sum(0).to(dt)
    return out


def _padded(x, ptr, longest, heads):
    """Rows of a packed batch as (graphs, heads, longest, d) in fp32, zeros behind the end of a graph, and which places are rows."""
    at = torch.arange(longest, device="cuda")
    start, length = ptr[:-1].long(), (ptr[1:] - ptr[:-1]).long()
    there = at < length[:, None]
    rows = (start[:, None] + at).clamp(max=x.shape[0] - 1)
    y = x[rows].float() * there[:, :, None]
    return y.unflatten(2, (heads, -1)).transpose(1, 2).contiguous(), there, rows


def _packed(y, ptr, n):
    """The rows of a packed batch out of (graphs, heads, longest, d)."""
    row = torch.arange(n, device="cuda")
    graph = torch.searchsorted(ptr[1:].long(), row, right=True)
    return y[graph, :, row - ptr.long()[graph]].flatten(1)


def _plain_attention(s):
    case, dt = s["case"], s["Q"].dtype
    heads, kv_heads, scale = case["heads"], case["kv_heads"], s["scale"]
    group, n_q, n_kv = heads // kv_heads, s["Q"].shape[0], s["K"].shape[0]
    q, _, _ = _padded(s["Q"], s["q_ptr"], s["longest_q"], heads)
    k, there, rows = _padded(s["K"], s["kv_ptr"], s["longest"], kv_heads)
    v, _, _ = _padded(s["V"], s["kv_ptr"], s["longest"], kv_heads)
    if s["mask"] is not None:
        there = there & (s["mask"][rows] != 0)
    k, v = k.repeat_interleave(group, 1), v.repeat_interleave(group, 1)
    p = (q @ k.transpose(2, 3)) * scale
    p = p.masked_fill(~there[:, None, None], -math.inf)
    p = torch.exp(p - p.amax(3, keepdim=True).clamp(min=-3e38))
    p = p / p.sum(3, keepdim=True).clamp(min=1e-30)  # a row with nothing to look at keeps zeros
    out = dict(out=_packed(p @ v, s["q_ptr"], n_q).to(dt))
    if case["kind"] == "attention_train":
        dO, _, _ = _padded(s["d_out"], s["q_ptr"], s["longest_q"], heads)
        dv = p.transpose(2, 3) @ dO
        ds = dO @ v.transpose(2, 3)
        ds = p * (ds - (p * ds).sum(3, keepdim=True)) * scale
        dk = ds.transpose(2, 3) @ q
        shared = lambda y: y.unflatten(1, (kv_heads, group)).sum(2)
        out.update(dQ=_packed(ds @ k, s["q_ptr"], n_q).to(dt), dK=_packed(shared(dk), s["kv_ptr"], n_kv).to(dt),
                   dV=_packed(shared(dv), s["kv_ptr"], n_kv).to(dt))
    return out


# ---- what a pass cannot do without --------------------------------------------------------------------
def work(case):
    kind, e = case["kind"], SIZE[case["dtype"]]
    if kind == "lookup":  # rows that several ids share are read once: at most as many as there are ids
        return dict(bytes=4 * case["n"] + (case["n"] + min(case["n"], case["vocab"])) * case["d"] * e, flops=case["n"] * case["d"])
    if kind == "lookup_grad":
        return dict(bytes=4 * case["n"] + (case["n"] + case["vocab"]) * case["d"] * e, flops=case["n"] * case["d"])
    if kind in ("linear", "linear_train"):
        n, d_in, d_out = case["n"], case["d_in"], case["d_out"]
        data = n * d_in + d_in * d_out + case["bias"] * d_out + (1 + case["residual"]) * n * d_out
        if kind == "linear":
            return dict(bytes=data * e, flops=2 * n * d_in * d_out)
        return dict(bytes=(data + n * d_out + n * d_in + d_in * d_out + case["bias"] * d_out) * e, flops=6 * n * d_in * d_out)
    lens, qlens = _lengths(case), _query_lengths(case)
    n_q, n_kv, pairs = sum(qlens), sum(lens), sum(a * b for a, b in zip(qlens, lens))
    data = 2 * n_q * case["heads"] + 2 * n_kv * case["kv_heads"]
    if kind == "attention":
        return dict(bytes=data * case["d"] * e, flops=4 * pairs * case["heads"] * case["d"])
    return dict(bytes=2 * data * case["d"] * e, flops=14 * pairs * case["heads"] * case["d"])


# ---- the same in 64 bits --------------------------------------------------------------------------------
def exact(case, seed):
    s, kind = _inputs(case, seed), case["kind"]
    if kind == "lookup":
        table = torch.cat([s["E"].double(), torch.zeros((1, case["d"]), dtype=torch.float64, device="cuda")])
        return dict(out=torch.index_select(table, 0, s["ids"].long() % (case["vocab"] + 1)) * s["scale"])  # -1: the last row
    if kind == "lookup_grad":
        order = torch.argsort(s["ids"].long(), stable=True)
        ids, rows = s["ids"].long()[order], s["d_out"][order].double()
        edge = torch.searchsorted(ids, torch.arange(case["vocab"] + 1, device="cuda"))
        upto = torch.cat([torch.zeros((1, case["d"]), dtype=torch.float64, device="cuda"), torch.cumsum(rows, 0)])
        dE = (upto[edge[1:]] - upto[edge[:-1]]) * s["scale"]
        dE[edge[1:] == edge[:-1]] = 0.0
        return dict(dE=dE)
    wide = lambda t: None if t is None else t.double().requires_grad_()
    if kind in ("linear", "linear_train"):
        X, W, b = wide(s["X"]), wide(s["W"]), wide(s["bias"])
        z = X.mm(W) if b is None else torch.addmm(b, X, W)
        f = torch.nn.functional
        z = dict(none=lambda t: t, relu=f.relu, gelu=f.gelu, silu=f.silu)[case["act"]](z)
        if s["residual"] is not None:
            z = z + s["residual"].double()
        if kind == "linear":
            return dict(out=z.detach())
        names = ["X", "W"] + (["b"] if case["bias"] else [])
        grads = torch.autograd.grad(z, [X, W] + ([b] if case["bias"] else []), s["d_out"].double())
        return dict(out=z.detach(), **{"d" + k: g for k, g in zip(names, grads)})
    heads, kv_heads, d = case["heads"], case["kv_heads"], case["d"]
    Q, K, V = wide(s["Q"]), wide(s["K"]), wide(s["V"])
    qp, kp = s["q_ptr"].tolist(), s["kv_ptr"].tolist()
    out = torch.zeros((Q.shape[0], heads * d), dtype=torch.float64, device="cuda")
    grads = [torch.zeros(t.shape, dtype=torch.float64, device="cuda") for t in (Q, K, V)]
    for g in range(case["graphs"]):
        a, b, c, e = qp[g], qp[g + 1], kp[g], kp[g + 1]
        seen = torch.ones(e - c, dtype=torch.bool, device="cuda") if s["mask"] is None else s["mask"][c:e] != 0
        if a == b or not bool(seen.any()):
            continue
        for h in range(heads):
            share = h // (heads // kv_heads)
            at_q, at_k = slice(h * d, h * d + d), slice(share * d, share * d + d)
            q, k, v = (t.detach().requires_grad_() for t in (Q[a:b, at_q], K[c:e, at_k], V[c:e, at_k]))
            weights = torch.softmax(s["scale"] * q.mm(k[seen].t()), 1)
            o = weights.mm(v[seen])
            out[a:b, at_q] = o.detach()
            if kind == "attention_train":
                dq, dk, dv = torch.autograd.grad(o, [q, k, v], s["d_out"][a:b, at_q].double())
                grads[0][a:b, at_q] = dq
                grads[1][c:e, at_k] += dk
                grads[2][c:e, at_k] += dv
    if kind == "attention":
        return dict(out=out)
    return dict(out=out, dQ=grads[0], dK=grads[1], dV=grads[2])
