"""Layer chaining of the two benchmark models (Section VI: 2-layer GCN with hidden size 16,
4-layer AGNN with hidden size 32): HotPath is the forward pass the benchmark times, TrainPath
the forward + backward pass of the same two models, GraphTransformerPath the forward + backward
pass of a graph transformer on a batch of graphs, PlannedGraph the per-graph adaptation that the
paper's outlook (Section VII) names: statistics of the graph decide how it is prepared.

Every step is a call into libftc through `binding`; this module only owns the device
buffers between the calls (allocated once in __init__, so a forward pass allocates nothing).
"""
import torch

from . import binding as B


class PlannedGraph:
    """Per-graph adaptive preparation (Section VII: fit the use of the hardware to the input graph).

    One pass over the graph's statistics (ftc_degree_stats, the window build's summary) goes to the host,
    ftc_plan_graph turns it into choices, and this class carries them out: relabel the nodes by degree
    class, or try the community ordering (label propagation) and keep it only if the windows then share
    more columns (sum_uniq drops), or leave the graph as it is.  `g` and `win` are the graph and window
    index to run the layers on; features enter with enter(X) and results leave with leave(Y), so the
    caller keeps the original numbering (permutation in, permutation out).  All device work is libftc's;
    the host only compares the few numbers the plan is made of."""

    def __init__(self, g, D, dtype, lp_rounds=10, side=None):
        self.g_given = g
        self.g, self.perm, self.inv, self.applied = g, None, None, "none"
        ws = B._workspace(B.lib().ftc_reorder_workspace_bytes(g.n, g.nnz), g.row_ptr.device)
        self.win = B.ftc_build_windows_concurrent(g, side)
        stats = B.ftc_degree_stats(g)
        self.sum_uniq_given = int(self.win.summary[0].item())          # the one host read the plan needs
        self.plan = B.ftc_plan_graph(g.n, g.nnz, int(stats[0].item()), self.sum_uniq_given, D, dtype)
        self.sum_uniq = self.sum_uniq_given
        order = self.plan["reorder"]
        if order == B.FTC_ORDER_DEGREE_CLASSES:
            perm, inv = B.ftc_degree_order(g, B.FTC_ORDER_DEGREE_CLASSES, ws=ws)
            self._relabel(perm, inv, ws, side, "degree classes", keep_if_fewer_columns=False)
        elif order == B.FTC_ORDER_COMMUNITIES:
            labels = B.ftc_label_propagation(g, lp_rounds, ws=ws)
            perm, inv, _ = B.ftc_order_by_key(labels, ws=ws)
            self._relabel(perm, inv, ws, side, "communities", keep_if_fewer_columns=True)

    def _relabel(self, perm, inv, ws, side, name, keep_if_fewer_columns):
        g2, flag = B.ftc_permute_graph(self.g_given, perm, inv, ws=ws)
        win2 = B.ftc_build_windows_concurrent(g2, side)
        su2 = int(win2.summary[0].item())
        assert int(flag.item()) == 0
        # a trial ordering is kept only if it makes the rows of a window share at least 2 % more columns
        if keep_if_fewer_columns and su2 > 0.98 * self.sum_uniq_given:
            self.trial = {"ordering": name, "sum_uniq": su2, "kept": False}
            return
        self.g, self.win, self.perm, self.inv, self.applied, self.sum_uniq = g2, win2, perm, inv, name, su2

    def enter(self, X, out=None):
        """Rows of X (original numbering) in the numbering of self.g."""
        return X if self.perm is None else B.ftc_permute_rows(X, self.perm, out=out)

    def leave(self, Y, out=None):
        """Rows of Y (numbering of self.g) back in the original numbering."""
        return Y if self.inv is None else B.ftc_permute_rows(Y, self.inv, out=out)


class HotPath:
    """window build + GCN normalisation + 2-layer GCN + 4-layer AGNN on one graph."""

    def __init__(self, g, d_feat=128, gcn_hidden=16, agnn_hidden=32, n_out=8, agnn_layers=4,
                 act_dtype=torch.float16, path=B.FTC_PATH_AUTO, concurrent_build=True):
        dev = g.row_ptr.device
        L = B.lib()
        self.g, self.path, self.agnn_layers = g, path, agnn_layers
        self.win = B.Windows(g)
        # the independent kernels of the window build overlap on three side streams owned here
        self.side = B.SideStreams() if concurrent_build else None
        n, nnz = g.n, g.nnz
        f32 = dict(dtype=torch.float32, device=dev)
        act = dict(dtype=act_dtype, device=dev)
        self.ws_win = B._workspace(L.ftc_build_windows_workspace_bytes(n, nnz, 16, 8), dev)
        self.dinv = torch.empty(n, **f32)    # the GCN layers take the factored normalisation: no per-edge values
        self.gcn_h = torch.empty((n, gcn_hidden), **act)
        self.gcn_out = torch.empty((n, n_out), **f32)
        ws_gcn = max(L.ftc_gcn_layer_workspace_bytes(n, nnz, d_feat, gcn_hidden),
                     L.ftc_gcn_layer_workspace_bytes(n, nnz, gcn_hidden, n_out))
        self.agnn_h = [torch.empty((n, agnn_hidden), **act) for _ in range(2)]
        self.agnn_out = torch.empty((n, n_out), **f32)
        ws_agnn = L.ftc_agnn_layer_workspace_bytes(n, nnz, agnn_hidden)
        self.ws = B._workspace(max(ws_gcn, ws_agnn), dev)

    def build(self):
        g, w = self.g, self.win
        B.ftc_build_windows_concurrent(g, self.side, out=w, ws=self.ws_win)
        B._check(B.lib().ftc_gcn_norm(B.C.byref(g.c), B.C.byref(w.c), None, B._ptr(self.dinv),
                                      B._stream()))

    def gcn(self, X, W1, W2):
        B.ftc_gcn_layer(self.g, self.win, None, X, W1, relu=True, out=self.gcn_h, path=self.path,
                        ws=self.ws, dinv=self.dinv)
        B.ftc_gcn_layer(self.g, self.win, None, self.gcn_h, W2, relu=False, out=self.gcn_out,
                        path=self.path, ws=self.ws, dinv=self.dinv)
        return self.gcn_out

    def agnn(self, X, W_in, W_out, betas):
        a, b = self.agnn_h
        B.ftc_update_gemm(X, W_in, out=a, relu=True)
        for layer in range(self.agnn_layers):
            B.ftc_agnn_layer(self.g, self.win, a, beta=betas[layer], out=b, path=self.path, ws=self.ws)
            a, b = b, a
        B.ftc_update_gemm(a, W_out, out=self.agnn_out)
        return self.agnn_out

    def step(self, X, W1, W2, W_in, W_out, betas):
        self.build()
        self.gcn(X, W1, W2)
        self.agnn(X, W_in, W_out, betas)

    def capture(self, X, W1, W2, W_in, W_out, betas):
        """The step as a HIP graph: every call of the library only enqueues kernels (and the window build's
        fork / join events) on the stream it is given and allocates nothing, so the whole step can be
        captured once and replayed with one launch; the results land in the same buffers as step()'s.
        The library keeps no state, so nothing has to run eagerly first."""
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            self.step(X, W1, W2, W_in, W_out, betas)
        return graph


class TrainPath:
    """Forward + backward of the two models on one graph with a symmetric pattern (the paper
    names training in Sections II and V and gives no formulas: the gradients are the derivatives
    of the forward definitions).  The GCN normalisation is the factored one, whose transposed
    operator is the operator itself; the AGNN backward needs the transposed index, built once here."""

    def __init__(self, g, win, dinv, d_feat=128, gcn_hidden=16, agnn_hidden=32, n_out=8, agnn_layers=4,
                 act_dtype=torch.float16, path=B.FTC_PATH_AUTO, fused=True):
        dev = g.row_ptr.device
        L = B.lib()
        self.g, self.win, self.dinv, self.path, self.agnn_layers = g, win, dinv, path, agnn_layers
        n, nnz = g.n, g.nnz
        self.T, flag = B.ftc_transpose_index(g, win)
        self.pattern_flag = flag           # handed to the single-pass backward, which refuses a non-symmetric pattern
        if int(flag.item()) != 0:
            raise ValueError("TrainPath needs a symmetric sparsity pattern with ascending, duplicate-free rows")
        f32 = dict(dtype=torch.float32, device=dev)
        act = dict(dtype=act_dtype, device=dev)
        self.gcn_h = torch.empty((n, gcn_hidden), **act)
        self.gcn_out = torch.empty((n, n_out), **f32)
        self.agnn_h = [None] + [torch.empty((n, agnn_hidden), **act) for _ in range(agnn_layers)]
        # single-pass forward / backward pair when the shape allows it: per-row softmax denominators are
        # kept instead of the per-entry probabilities, and no transposed index is read
        self.fused = bool(fused and win is not None and L.ftc_agnn_layer_backward_fused_workspace_bytes(n, nnz, agnn_hidden) > 0
                          and (agnn_hidden * self.agnn_h_itemsize(act_dtype)) % 16 == 0)
        self.agnn_z = [torch.empty(n, **f32) for _ in range(agnn_layers)] if self.fused else []
        # 16-bit activations: every layer also keeps its unrounded output for the backward pass
        self.keep_f32 = self.fused and act_dtype != torch.float32
        self.agnn_y32 = [torch.empty((n, (agnn_hidden + 3) // 4 * 4), **f32) for _ in range(agnn_layers)] \
            if self.keep_f32 else []
        self.agnn_p = [torch.empty(nnz, **f32) for _ in range(agnn_layers)] if not self.fused else []
        self.d_agnn_h = [torch.empty((n, agnn_hidden), **act) for _ in range(2)]
        self.agnn_h0 = torch.empty((n, agnn_hidden), **act)     # output of the in-projection
        self.d_agnn_h0 = torch.empty((n, agnn_hidden), **f32)   # gradient entering the in-projection
        self.agnn_out = torch.empty((n, n_out), **f32)
        self.dbeta = torch.empty(agnn_layers, **f32)
        self.ws = B._workspace(max(
            L.ftc_gcn_layer_workspace_bytes(n, nnz, d_feat, gcn_hidden),
            L.ftc_gcn_layer_workspace_bytes(n, nnz, gcn_hidden, n_out),
            L.ftc_gcn_layer_backward_workspace_bytes(n, nnz, d_feat, gcn_hidden),
            L.ftc_gcn_layer_backward_workspace_bytes(n, nnz, gcn_hidden, n_out),
            L.ftc_agnn_layer_workspace_bytes(n, nnz, agnn_hidden),
            L.ftc_agnn_layer_backward_workspace_bytes(n, nnz, agnn_hidden),
            L.ftc_agnn_layer_backward_fused_workspace_bytes(n, nnz, agnn_hidden),
            L.ftc_update_gemm_backward_workspace_bytes(n, d_feat, agnn_hidden),
            L.ftc_update_gemm_backward_workspace_bytes(n, agnn_hidden, n_out)), dev)

    @staticmethod
    def agnn_h_itemsize(dtype):
        return torch.empty(0, dtype=dtype).element_size()

    def gcn_forward(self, X, W1, W2):
        B.ftc_gcn_layer(self.g, self.win, None, X, W1, relu=True, out=self.gcn_h, path=self.path, ws=self.ws,
                        dinv=self.dinv)
        B.ftc_gcn_layer(self.g, self.win, None, self.gcn_h, W2, relu=False, out=self.gcn_out, path=self.path,
                        ws=self.ws, dinv=self.dinv)
        return self.gcn_out

    def gcn_backward(self, X, W1, W2, d_out):
        """d_out = dL/d(gcn_out), fp32.  Returns (dW1, dW2); the input features get no gradient."""
        d_h, dW2 = B.ftc_gcn_layer_backward(self.g, self.win, None, self.gcn_h, W2, d_out, dinv=self.dinv,
                                            path=self.path, ws=self.ws)
        _, dW1 = B.ftc_gcn_layer_backward(self.g, self.win, None, X, W1, d_h, Y=self.gcn_h, dinv=self.dinv,
                                          want_dX=False, path=self.path, ws=self.ws)
        return dW1, dW2

    def agnn_forward(self, H0, betas):
        """Propagation layers only; every layer keeps what its backward pass needs: the softmax
        denominators (and its unrounded output when the activations are 16-bit) on the single-pass route,
        the attention probabilities on the edge-array route."""
        self.agnn_h[0] = H0
        for l in range(self.agnn_layers):
            keep = dict(row_z=self.agnn_z[l]) if self.fused else dict(edge_p=self.agnn_p[l])
            if self.keep_f32:
                keep["out_f32"] = self.agnn_y32[l]
            B.ftc_agnn_layer(self.g, self.win, self.agnn_h[l], beta=betas[l], out=self.agnn_h[l + 1],
                             path=self.path, ws=self.ws, **keep)
        return self.agnn_h[self.agnn_layers]

    def agnn_backward(self, betas, d_out, first_in_f32=False):
        """d_out = dL/d(last layer's output), in the activation type.  Returns (dL/dH0, dbeta[layers]);
        dL/dH0 in fp32 when first_in_f32 (what the backward of the in-projection takes)."""
        d = d_out
        for l in reversed(range(self.agnn_layers)):
            nxt = self.d_agnn_h0 if (l == 0 and first_in_f32) else self.d_agnn_h[l & 1]
            if self.fused:
                y = self.agnn_y32[l][:, :self.agnn_h[l].shape[1]] if self.keep_f32 else self.agnn_h[l + 1]
                B.ftc_agnn_layer_backward_fused(self.g, self.win, self.agnn_h[l], self.agnn_z[l], y, d,
                                                beta=betas[l], dH=nxt, dbeta=self.dbeta[l:l + 1], ws=self.ws,
                                                pattern_flag=self.pattern_flag)
            else:
                B.ftc_agnn_layer_backward(self.g, self.win, self.T, self.agnn_h[l], self.agnn_p[l], d, beta=betas[l],
                                          dH=nxt, dbeta=self.dbeta[l:l + 1], path=self.path, ws=self.ws)
            d = nxt
        return d, self.dbeta

    def agnn_model_forward(self, X, W_in, W_out, betas):
        """The whole AGNN model of the benchmark: ReLU in-projection, propagation layers, out-projection."""
        B.ftc_update_gemm(X, W_in, out=self.agnn_h0, relu=True)
        h = self.agnn_forward(self.agnn_h0, betas)
        B.ftc_update_gemm(h, W_out, out=self.agnn_out)
        return self.agnn_out

    def agnn_model_backward(self, X, W_in, W_out, betas, d_out):
        """d_out = dL/d(agnn_out), fp32.  Returns (dW_in, dW_out, dbeta[layers])."""
        h_last = self.agnn_h[self.agnn_layers]
        d_h, dW_out = B.ftc_update_gemm_backward(h_last, W_out, d_out, dX=self.d_agnn_h[self.agnn_layers & 1], ws=self.ws)
        d_h0, dbeta = self.agnn_backward(betas, d_h, first_in_f32=True)
        _, dW_in = B.ftc_update_gemm_backward(X, W_in, d_h0, Z=self.agnn_h0, want_dX=False, ws=self.ws)
        return dW_in, dW_out, dbeta


class GraphTransformerPath:
    """Forward + backward of a graph transformer on a packed batch of graphs: node features looked up by id, layers of attention
    between all nodes of a graph and of a feed-forward block (GELU), each with a residual connection around it, and a linear
    head on every node.  graph_ptr: device int32, the graphs' first nodes and the end, which is n (nodes that fill a batch up are a graph of their
    own, masked); heads share kv_heads K/V heads.

    Weights are a dict: "table" (vocab x d), "head" and "head_bias", and "layers", a list of dicts "qkv" (d x (heads + 2 kv_heads) d / heads),
    "out" (d x d), "up" (d x hidden), "down" (hidden x d) with a bias each ("qkv_bias", ...).  Gradients come in the same shape, in fp32.
    Buffers are allocated here once; forward() keeps in them what backward() needs.

    What a layer can have besides (each with weights of its own):
      norm       a norm (B.FTC_NORM_RMS, B.FTC_NORM_LAYER) in front of both blocks and of the head: "attention_norm" and "feed_norm" of a layer, "head_norm"
      post_norm  a norm of what a block gives: "attention_post" and "feed_post" of a layer; layer norms have biases ("feed_norm_bias", ...)
      gates      learned factors of what a block adds, d of them: "attention_gate" and "feed_gate" of a layer
      residual_scale  what the residual connections multiply their input by
      types      the type of every node (contiguous int32 on graph_ptr's device, from 0 on below n_types): "up" and "down" are of each type, n_types x d x hidden and
                 n_types x hidden x d, their biases n_types x hidden and n_types x d.  Read when the path is made: nodes of other types are another path
    clip() is the clipping of all gradients by their norm."""

    LINEAR = ("qkv", "out", "up", "down")

    def __init__(self, graph_ptr, n, vocab, d=64, heads=4, kv_heads=None, hidden=None, n_out=8, layers=2, act_dtype=torch.float16,
                 norm=B.FTC_NORM_NONE, post_norm=B.FTC_NORM_NONE, gates=False, residual_scale=1.0, types=None, n_types=0):
        dev, L = graph_ptr.device, B.lib()
        if d % heads:
            raise ValueError("d is a multiple of heads")
        self.graph_ptr, self.n, self.vocab, self.d, self.heads, self.n_out = graph_ptr, n, vocab, d, heads, n_out
        self.kv_heads = heads if kv_heads is None else kv_heads
        self.head_dim, self.hidden, self.layers = d // heads, 4 * d if hidden is None else hidden, layers
        self.scale = float(d) ** 0.5                 # of the looked-up rows, as with tables shared with an output layer
        kd = self.kv_heads * self.head_dim
        self.columns = (slice(0, d), slice(d, d + kd), slice(d + kd, d + 2 * kd))      # of q, k, v
        act = lambda c: torch.empty((n, c), dtype=act_dtype, device=dev)
        self.h = [act(d) for _ in range(layers + 1)]           # input of every layer, and of the head
        self.qkv = [act(d + 2 * kd) for _ in range(layers)]
        self.attended = [act(d) for _ in range(layers)]
        self.lse = [torch.empty((n, heads), dtype=torch.float32, device=dev) for _ in range(layers)]
        self.middle = [act(d) for _ in range(layers)]          # between attention and feed-forward block
        self.up = [act(self.hidden) for _ in range(layers)]
        self.slope = [B.slope_like(t) for t in self.up]
        self.logits = act(n_out)
        self.d_h, self.d_attended, self.d_up, self.d_qkv = act(d), act(d), act(self.hidden), act(d + 2 * kd)
        shapes = [(d, d + 2 * kd), (d, d), (d, self.hidden), (self.hidden, d), (d, n_out)]
        sizes = (n, n, graph_ptr.numel() - 1, heads, self.kv_heads, self.head_dim)
        self.ws = B._workspace(max([L.ftc_graph_attention_workspace_bytes(*sizes), L.ftc_graph_attention_backward_workspace_bytes(*sizes),
                                    L.ftc_embedding_backward_workspace_bytes(n, vocab, d)] +
                                   [f(n, *s) for f in (L.ftc_linear_workspace_bytes, L.ftc_linear_backward_workspace_bytes) for s in shapes]), dev)
        self.norm, self.post_norm, self.gates, self.residual_scale, self.n_types = norm, post_norm, gates, residual_scale, n_types
        self.blocks = bool(norm or post_norm or gates or types is not None or residual_scale != 1.0)
        if not self.blocks:
            return
        self.group_ptr = None
        if types is not None:
            B._vector(types, n, (torch.int32,))     # what orders them reads n whole numbers of 32 bits on the device
            if types.device != dev:
                raise ValueError(f"types are on {types.device}, graph_ptr on {dev}")
            low, high = (int(x.item()) for x in types.aminmax()) if n else (0, -1)
            if low < 0 or high >= n_types:
                raise ValueError(f"types of {n} nodes, from 0 on below n_types")
            self.perm, self.inv, _ = B.ftc_order_by_key(types)
            self.group_ptr = torch.zeros(n_types + 1, dtype=torch.int32, device=dev)
            self.group_ptr[1:] = torch.cumsum(torch.bincount(types, minlength=n_types), 0)
            self.by_type, self.d_by_type = [act(d) for _ in range(layers)], act(d)     # inputs of the feed-forward block in the order of the types
            self.unsorted = act(d)
        # what is normed for a block or the head, what a block gives, the statistics of the norms behind it
        self.normed = [act(d) for _ in range(2 * layers + 1)] if norm else None
        self.given = [act(d) for _ in range(2 * layers)]
        self.stats = [torch.empty((n, 4), dtype=torch.float32, device=dev) for _ in range(2 * layers + 1)]
        self.d_given, self.d_normed = act(d), act(d)
        self.ws = B._workspace(max([self.ws.numel(), L.ftc_block_norm_backward_workspace_bytes(n, d)] +
                                   [f(n, n_types, *s) for f in (L.ftc_grouped_linear_workspace_bytes, L.ftc_grouped_linear_backward_workspace_bytes)
                                    for s in shapes[2:4]]), dev)

    def _join(self, weights, at):
        """The arguments of the norms and the residual connection behind block `at` (0: in front of the first; 2 i + 1, 2 i + 2: behind attention and
        feed-forward block of layer i) and, by the name of its gradient, where each of their weights is: in which layer (-1: the whole's) and its key."""
        args, names = dict(x_scale=self.residual_scale if at else 1.0, post=B.FTC_NORM_NONE, pre=self.norm), {}

        def take(layer, name, arg):
            args[arg], names["d" + arg] = (weights["layers"][layer] if layer >= 0 else weights)[name], (layer, name)

        def take_norm(layer, name, arg, kind):
            take(layer, name, arg + "_w")
            if kind == B.FTC_NORM_LAYER:
                take(layer, name + "_bias", arg + "_b")
        if at:
            layer, block = (at - 1) // 2, ("attention", "feed")[(at - 1) % 2]
            args["F"], args["post"] = self.given[at - 1], self.post_norm
            if self.post_norm:
                take_norm(layer, block + "_post", "post", self.post_norm)
            if self.gates:
                take(layer, block + "_gate", "gate")
        if self.norm:
            take_norm(*((-1, "head_norm") if at == 2 * self.layers else (at // 2, ("attention_norm", "feed_norm")[at % 2])), "pre", self.norm)
        return args, names

    def _streams(self):
        """The residual stream in front of and behind every block."""
        between = [self.h[0]]
        for i in range(self.layers):
            between += [self.middle[i], self.h[i + 1]]
        return between

    def _forward_blocks(self, weights, mask):
        between, ws = self._streams(), self.ws

        def join(at):
            """What the next block (or the head) gets."""
            if at == 0 and not self.norm:
                return between[0]
            args, _ = self._join(weights, at)
            B.ftc_block_norm(between[max(at - 1, 0)], H=between[at] if at else None, U=self.normed[at] if self.norm else None, stats=self.stats[at], **args)
            return self.normed[at] if self.norm else between[at]
        x = join(0)
        for i, w in enumerate(weights["layers"]):
            B.ftc_linear(x, w["qkv"], bias=w["qkv_bias"], out=self.qkv[i], ws=ws)
            args, kw = self._attention_args(i, mask)
            B.ftc_graph_attention(*args, out=self.attended[i], lse=self.lse[i], **kw)
            B.ftc_linear(self.attended[i], w["out"], bias=w["out_bias"], out=self.given[2 * i], ws=ws)
            x = join(2 * i + 1)
            if self.group_ptr is None:
                B.ftc_linear(x, w["up"], bias=w["up_bias"], act=B.FTC_ACT_GELU, out=self.up[i], slope=self.slope[i], ws=ws)
                B.ftc_linear(self.up[i], w["down"], bias=w["down_bias"], out=self.given[2 * i + 1], ws=ws)
            else:
                B.ftc_permute_rows(x, self.perm, out=self.by_type[i])
                B.ftc_grouped_linear(self.by_type[i], w["up"], self.group_ptr, bias=w["up_bias"], act=B.FTC_ACT_GELU, out=self.up[i], slope=self.slope[i], ws=ws)
                B.ftc_grouped_linear(self.up[i], w["down"], self.group_ptr, bias=w["down_bias"], out=self.unsorted, ws=ws)
                B.ftc_permute_rows(self.unsorted, self.inv, out=self.given[2 * i + 1])
            x = join(2 * i + 2)
        return B.ftc_linear(x, weights["head"], bias=weights["head_bias"], out=self.logits, ws=ws)

    def _backward_blocks(self, weights, grads, d_out, mask):
        between, ws, back = self._streams(), self.ws, B.ftc_linear_backward

        def join(at):
            """Through the join: d_h is the gradient of the stream in front of it then, d_given that of the block's result.  What reaches the stream behind it on the
            way of the next block's input is in d_normed, or has been added to d_h where there is no norm."""
            if at == 0 and not self.norm:
                return
            args, names = self._join(weights, at)
            last = at == 2 * self.layers       # nothing goes on behind the head's norm
            got = B.ftc_block_norm_backward(between[max(at - 1, 0)], self.stats[at], dH=None if last and self.norm else self.d_h, dU=self.d_normed if self.norm else None,
                                            dX=self.d_h, dF=self.d_given if at else None, ws=ws, **args)
            for name, (layer, key) in names.items():
                (grads["layers"][layer] if layer >= 0 else grads)[key] = getattr(got, name)

        def block_input(at, **k):
            """Where the gradient of what a block (or the head) got goes."""
            if self.norm:
                return dict(dX=self.d_normed, **k)
            return dict(dX=self.d_h, **k) if at == 2 * self.layers else dict(dX=self.d_h, dX_add=self.d_h, **k)
        put = lambda at: self.normed[at] if self.norm else between[at]
        last = 2 * self.layers
        _, grads["head"], grads["head_bias"] = back(put(last), weights["head"], d_out, ws=ws, **block_input(last))
        for i in reversed(range(self.layers)):
            w, g, at = weights["layers"][i], grads["layers"][i], 2 * i
            join(at + 2)
            if self.group_ptr is None:
                _, g["down"], g["down_bias"] = back(self.up[i], w["down"], self.d_given, dX=self.d_up, ws=ws)
                _, g["up"], g["up_bias"] = back(put(at + 1), w["up"], self.d_up, slope=self.slope[i], ws=ws, **block_input(at + 1))
            else:
                grouped = B.ftc_grouped_linear_backward
                B.ftc_permute_rows(self.d_given, self.perm, out=self.unsorted)
                _, g["down"], g["down_bias"] = grouped(self.up[i], w["down"], self.group_ptr, self.unsorted, dX=self.d_up, ws=ws)
                up = lambda **k: grouped(self.by_type[i], w["up"], self.group_ptr, self.d_up, slope=self.slope[i], dX=self.d_by_type, ws=ws, **k)
                if self.norm:
                    _, g["up"], g["up_bias"] = up()
                    B.ftc_permute_rows(self.d_by_type, self.inv, out=self.d_normed)
                else:       # d_h in the order of the types and back: the product is added to it before their one rounding
                    B.ftc_permute_rows(self.d_h, self.perm, out=self.unsorted)
                    _, g["up"], g["up_bias"] = up(dX_add=self.unsorted)
                    B.ftc_permute_rows(self.d_by_type, self.inv, out=self.d_h)
            join(at + 1)
            _, g["out"], g["out_bias"] = back(self.attended[i], w["out"], self.d_given, dX=self.d_attended, ws=ws)
            args, kw = self._attention_args(i, mask)
            dq, dk, dv = (self.d_qkv[:, c] for c in self.columns)
            B.ftc_graph_attention_backward(*args, self.attended[i], self.lse[i], self.d_attended, dQ=dq, dK=dk, dV=dv, **kw)
            _, g["qkv"], g["qkv_bias"] = back(put(at), w["qkv"], self.d_qkv, ws=ws, **block_input(at))
        join(0)

    def clip(self, grads, max_norm, scale=1.0, norm=None):
        """Clips the gradients of backward(), in place, all by their one norm, which is what comes back (before clipping); scale: what a scaled loss is divided by."""
        flat = [t for k, t in sorted(grads.items()) if k != "layers"] + [t for g in grads["layers"] for _, t in sorted(g.items())]
        return B.ftc_clip_grad_norm(flat, max_norm, scale=scale, norm=norm)

    def _attention_args(self, layer, mask):
        q, k, v = (self.qkv[layer][:, c] for c in self.columns)
        return (q, k, v, self.graph_ptr, self.graph_ptr), dict(heads=self.heads, kv_heads=self.kv_heads, kv_mask=mask, ws=self.ws)

    def _check_layers(self, weights):
        if len(weights["layers"]) != self.layers:
            raise ValueError(f"weights of {len(weights['layers'])} layers for a path of {self.layers} layers")

    def forward(self, ids, weights, mask=None):
        """Logits (n x n_out), in the path's buffer.  mask: nodes with 0 are attended to by no node."""
        self._check_layers(weights)
        B.ftc_embedding(ids, weights["table"], scale=self.scale, out=self.h[0])
        if self.blocks:
            return self._forward_blocks(weights, mask)
        for i, w in enumerate(weights["layers"]):
            B.ftc_linear(self.h[i], w["qkv"], bias=w["qkv_bias"], out=self.qkv[i], ws=self.ws)
            args, kw = self._attention_args(i, mask)
            B.ftc_graph_attention(*args, out=self.attended[i], lse=self.lse[i], **kw)
            B.ftc_linear(self.attended[i], w["out"], bias=w["out_bias"], residual=self.h[i], out=self.middle[i], ws=self.ws)
            B.ftc_linear(self.middle[i], w["up"], bias=w["up_bias"], act=B.FTC_ACT_GELU, out=self.up[i], slope=self.slope[i], ws=self.ws)
            B.ftc_linear(self.up[i], w["down"], bias=w["down_bias"], residual=self.middle[i], out=self.h[i + 1], ws=self.ws)
        return B.ftc_linear(self.h[-1], weights["head"], bias=weights["head_bias"], out=self.logits, ws=self.ws)

    def backward(self, ids, weights, d_out, mask=None):
        """d_out = dL/d(logits), in the activation type; gradients of the weights that forward() was given, with the mask that it was given."""
        self._check_layers(weights)
        grads, back = dict(layers=[{} for _ in weights["layers"]]), B.ftc_linear_backward
        if self.blocks:
            self._backward_blocks(weights, grads, d_out, mask)
            grads["table"] = B.ftc_embedding_backward(ids, self.d_h, self.vocab, scale=self.scale, ws=self.ws)
            return grads
        _, grads["head"], grads["head_bias"] = back(self.h[-1], weights["head"], d_out, dX=self.d_h, ws=self.ws)
        for i in reversed(range(self.layers)):
            w, g = weights["layers"][i], grads["layers"][i]
            # d_h goes through both blocks of the layer: what their residual connections carry is added in place
            _, g["down"], g["down_bias"] = back(self.up[i], w["down"], self.d_h, dX=self.d_up, ws=self.ws)
            _, g["up"], g["up_bias"] = back(self.middle[i], w["up"], self.d_up, slope=self.slope[i], dX=self.d_h, dX_add=self.d_h, ws=self.ws)
            _, g["out"], g["out_bias"] = back(self.attended[i], w["out"], self.d_h, dX=self.d_attended, ws=self.ws)
            args, kw = self._attention_args(i, mask)
            dq, dk, dv = (self.d_qkv[:, c] for c in self.columns)
            B.ftc_graph_attention_backward(*args, self.attended[i], self.lse[i], self.d_attended, dQ=dq, dK=dk, dV=dv, **kw)
            _, g["qkv"], g["qkv_bias"] = back(self.h[i], w["qkv"], self.d_qkv, dX=self.d_h, dX_add=self.d_h, ws=self.ws)
        grads["table"] = B.ftc_embedding_backward(ids, self.d_h, self.vocab, scale=self.scale, ws=self.ws)
        return grads
