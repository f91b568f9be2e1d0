"""What the graph transformer's entry points refuse, on the host, before anything is launched (the pointers are never followed), and
the reference that the GPU tests use, against torch's gradients in 64 bits.  CPU only."""
import ctypes as C

import numpy as np
import pytest
import torch

import transformer_reference as ref
from paper_2412_12218_amd import binding as B

P = lambda i: C.c_void_p(0x10000 * i)
BIG = 1 << 40


def embedding(**k):
    a = dict(n=4, ids=P(1), vocab=5, E=P(2), lde=8, dtype=1, D=8, scale=1.0, out=P(3), ldo=8, odt=1) | k
    return B.lib().ftc_embedding(*a.values(), None)


def embedding_backward(**k):
    a = dict(n=4, ids=P(1), vocab=5, g=P(2), ldg=8, dtype=1, D=8, scale=1.0, dE=P(3), lde=8, dt=0, ws=P(4), bytes=BIG) | k
    return B.lib().ftc_embedding_backward(*a.values(), None)


def linear(**k):
    a = dict(n=4, X=P(1), ldx=8, dtype=1, d_in=8, W=P(2), d_out=16, bias=P(3), act=2, R=P(4), ldr=16, slope=P(5), lds=16, Z=P(6), ldz=16, zdt=1,
             ws=P(7), bytes=BIG) | k
    return B.lib().ftc_linear(*a.values(), None)


def linear_backward(**k):
    a = dict(n=4, X=P(1), ldx=8, dtype=1, d_in=8, W=P(2), d_out=16, slope=P(3), lds=16, dZ=P(4), ldz=16, add=None, lda=0, dX=P(5), lddx=8, dxt=1, dW=P(6), db=P(7), dwt=0,
             ws=P(8), bytes=BIG) | k
    return B.lib().ftc_linear_backward(*a.values(), None)


def attention(**k):
    a = dict(n_q=4, q_ptr=P(1), n_kv=6, kv_ptr=P(2), graphs=2, heads=4, kv_heads=2, D=8, dtype=1, Q=P(3), ldq=32, K=P(4), ldk=16, V=P(5), ldv=16,
             mask=None, scale=1.0, out=P(6), ldo=32, lse=P(7), ws=P(8), bytes=BIG) | k
    return B.lib().ftc_graph_attention(*a.values(), None)


def attention_backward(**k):
    a = dict(n_q=4, q_ptr=P(1), n_kv=6, kv_ptr=P(2), graphs=2, heads=4, kv_heads=2, D=8, dtype=1, Q=P(3), ldq=32, K=P(4), ldk=16, V=P(5), ldv=16,
             mask=None, scale=1.0, out=P(6), ldo=32, lse=P(7), dO=P(8), lddo=32, dQ=P(9), lddq=32, dK=P(10), lddk=16, dV=P(11), lddv=16, ws=P(12),
             bytes=BIG) | k
    return B.lib().ftc_graph_attention_backward(*a.values(), None)


INVALID, UNSUPPORTED, ALIGN, WORKSPACE = B.FTC_EINVAL, B.FTC_EUNSUPPORTED, B.FTC_EALIGN, B.FTC_EWORKSPACE
CASES = [
    (embedding, dict(n=-1), INVALID), (embedding, dict(vocab=-1), INVALID), (embedding, dict(ids=None), INVALID), (embedding, dict(E=None), INVALID),
    (embedding, dict(out=None), INVALID), (embedding, dict(out=P(2)), INVALID), (embedding, dict(lde=7), INVALID), (embedding, dict(D=0), INVALID),
    (embedding, dict(dtype=3), UNSUPPORTED), (embedding, dict(odt=-1), UNSUPPORTED), (embedding, dict(vocab=0, dtype=9), UNSUPPORTED),
    (embedding, dict(out=C.c_void_p(0x30001)), ALIGN),
    (embedding_backward, dict(n=-1), INVALID), (embedding_backward, dict(ids=None), INVALID), (embedding_backward, dict(g=None), INVALID),
    (embedding_backward, dict(dE=P(2)), INVALID), (embedding_backward, dict(lde=3), INVALID), (embedding_backward, dict(dtype=5), UNSUPPORTED),
    (embedding_backward, dict(ws=None), WORKSPACE), (embedding_backward, dict(bytes=64), WORKSPACE), (embedding_backward, dict(ws=C.c_void_p(0x40010)), ALIGN),
    (linear, dict(n=-1), INVALID), (linear, dict(act=4), INVALID), (linear, dict(act=-1), INVALID), (linear, dict(X=None), INVALID),
    (linear, dict(W=None), INVALID), (linear, dict(Z=None), INVALID), (linear, dict(ldx=7), INVALID), (linear, dict(ldr=15), INVALID),
    (linear, dict(lds=15), INVALID), (linear, dict(d_in=0), INVALID), (linear, dict(d_out=0), INVALID), (linear, dict(dtype=3), UNSUPPORTED),
    (linear, dict(zdt=2), UNSUPPORTED), (linear, dict(dtype=0, zdt=1), UNSUPPORTED), (linear, dict(Z=P(1)), INVALID), (linear, dict(Z=P(2)), INVALID),
    (linear, dict(Z=P(5)), INVALID), (linear, dict(slope=P(4)), INVALID), (linear, dict(Z=P(4), ldz=17), INVALID), (linear, dict(Z=P(4), zdt=0), INVALID),
    (linear, dict(slope=C.c_void_p(0x50001)), ALIGN), (linear, dict(d_in=5000, ldx=5000, ws=None), WORKSPACE),
    (linear, dict(d_in=5000, ldx=5000, bytes=100), WORKSPACE), (linear, dict(d_in=5000, ldx=5000, ws=C.c_void_p(0x70020)), ALIGN),
    (linear_backward, dict(n=-1), INVALID), (linear_backward, dict(d_in=0), INVALID), (linear_backward, dict(X=None), INVALID),
    (linear_backward, dict(W=None), INVALID), (linear_backward, dict(dZ=None), INVALID), (linear_backward, dict(lds=3), INVALID),
    (linear_backward, dict(lddx=3), INVALID), (linear_backward, dict(dtype=4), UNSUPPORTED), (linear_backward, dict(dxt=2), UNSUPPORTED),
    (linear_backward, dict(add=P(9), lda=7), INVALID), (linear_backward, dict(add=P(5), lda=9), INVALID), (linear_backward, dict(add=P(6), lda=8), INVALID),
    (linear_backward, dict(add=P(5), lda=8, dxt=0), INVALID), (linear_backward, dict(dwt=2), UNSUPPORTED), (linear_backward, dict(dX=P(4)), INVALID), (linear_backward, dict(dW=P(2)), INVALID),
    (linear_backward, dict(db=P(6)), INVALID), (linear_backward, dict(ws=None), WORKSPACE), (linear_backward, dict(ws=C.c_void_p(0x80008)), ALIGN),
]
for call in (attention, attention_backward):
    CASES += [(call, dict(n_q=-1), INVALID), (call, dict(n_kv=-1), INVALID), (call, dict(graphs=-1), INVALID), (call, dict(q_ptr=None), INVALID),
              (call, dict(kv_ptr=None), INVALID), (call, dict(heads=0), INVALID), (call, dict(kv_heads=0), INVALID), (call, dict(kv_heads=3), INVALID),
              (call, dict(D=0), INVALID), (call, dict(D=129, ldq=2000, ldk=2000, ldv=2000), UNSUPPORTED), (call, dict(dtype=3), UNSUPPORTED),
              (call, dict(n_q=(1 << 28) + 1), UNSUPPORTED), (call, dict(heads=1 << 17, kv_heads=1 << 17, n_q=1, n_kv=1), UNSUPPORTED),
              (call, dict(Q=None), INVALID), (call, dict(K=None), INVALID), (call, dict(V=None), INVALID), (call, dict(ldq=31), INVALID),
              (call, dict(ldk=15), INVALID), (call, dict(ldv=15), INVALID), (call, dict(out=None), INVALID), (call, dict(Q=C.c_void_p(0x30001)), ALIGN)]
CASES += [(attention, dict(out=P(3)), INVALID), (attention, dict(out=P(4)), INVALID), (attention, dict(n_kv=100_000, ws=None), WORKSPACE),
          (attention, dict(n_kv=100_000, bytes=1000), WORKSPACE), (attention, dict(n_kv=100_000, ws=C.c_void_p(0x80010)), ALIGN),
          (attention_backward, dict(dO=None), INVALID), (attention_backward, dict(lse=None), INVALID), (attention_backward, dict(dQ=None), INVALID),
          (attention_backward, dict(dK=None), INVALID), (attention_backward, dict(dV=P(10)), INVALID), (attention_backward, dict(dK=P(4)), INVALID),
          (attention_backward, dict(lddq=31), INVALID), (attention_backward, dict(ws=None), WORKSPACE), (attention_backward, dict(bytes=8), WORKSPACE)]


@pytest.mark.parametrize("call,change,code", CASES, ids=lambda v: getattr(v, "__name__", str(v)))
def test_refused(call, change, code):
    assert call(**change) == code
    assert B.lib().ftc_last_error().startswith(b"ftc_")


M30 = 1 << 30
LARGE = [
    (embedding, dict(n=M30 + 1)), (embedding, dict(vocab=M30 + 1)), (embedding, dict(n=M30, D=4096, lde=4096, ldo=4096)),
    (embedding, dict(D=M30, lde=M30, ldo=M30)), (embedding_backward, dict(n=M30 + 1)), (embedding_backward, dict(vocab=M30 + 7)),
    (linear, dict(n=M30 + 1)), (linear, dict(n=M30, d_out=64, ldr=64, lds=64, ldz=64)), (linear, dict(n=1, d_out=M30, ldr=M30, lds=M30, ldz=M30)),
    (linear_backward, dict(n=M30, d_out=64, lds=64, ldz=64)), (linear_backward, dict(d_out=M30, lds=M30, ldz=M30)),
    (attention, dict(graphs=M30)), (attention, dict(graphs=1 << 26, kv_heads=4, ldk=32, ldv=32)), (attention_backward, dict(graphs=M30)),
]


@pytest.mark.parametrize("call,change", LARGE, ids=lambda v: v.__name__ if callable(v) else "-".join(f"{k}={x}" for k, x in v.items())[:40])
def test_sizes_beyond_a_launch_are_refused(call, change):
    assert call(**change) == UNSUPPORTED
    assert b"2^30" in B.lib().ftc_last_error() or b"launch" in B.lib().ftc_last_error()


def test_calls_without_work():
    """Nothing to compute: no pointer is needed, nothing is launched."""
    assert embedding(n=0, ids=None, E=None, out=None) == B.FTC_OK
    assert embedding_backward(vocab=0, dE=None, ids=None, g=None, ws=None) == B.FTC_OK
    assert linear(n=0, X=None, Z=None) == B.FTC_OK
    assert attention(n_q=0, Q=None, out=None) == B.FTC_OK
    assert attention(graphs=0, q_ptr=None, kv_ptr=None) == B.FTC_OK
    assert attention_backward(n_q=0, n_kv=0) == B.FTC_OK
    assert attention_backward(graphs=0, q_ptr=None, kv_ptr=None) == B.FTC_OK


def test_workspace_queries():
    L = B.lib()
    assert L.ftc_embedding_backward_workspace_bytes(-1, 4, 4) == 0 and L.ftc_embedding_backward_workspace_bytes(1000, 5, 64) >= 1000 * 8
    assert L.ftc_linear_workspace_bytes(4, 0, 4) == 0 and L.ftc_linear_backward_workspace_bytes(100, 10, 10) >= 100 * 10 * 2
    assert L.ftc_graph_attention_workspace_bytes(4, 4, 1, 3, 2, 8) == 0
    assert L.ftc_graph_attention_workspace_bytes(1, 100_000, 1, 8, 2, 64) >= 8 * 64 * 4 * 2
    for n in (0, 1, 5):                # none of anything
        for d in (1, 4000):
            assert L.ftc_linear_workspace_bytes(n, d, 1) >= 0 and L.ftc_linear_backward_workspace_bytes(n, d, 1) >= 0
        for graphs in (0, 1):
            for kv in (0, 3):
                assert L.ftc_graph_attention_workspace_bytes(n, kv, graphs, 2, 1, 8) >= 0
                assert L.ftc_graph_attention_backward_workspace_bytes(n, kv, graphs, 2, 1, 8) >= 0
        assert L.ftc_embedding_backward_workspace_bytes(n, 0, 1) >= 0
    assert L.ftc_graph_attention_backward_workspace_bytes(1000, 1000, 10, 8, 2, 64) >= 1000 * 8 * 4


def test_tensors_are_checked_by_the_binding():
    x = torch.zeros((4, 8))
    with pytest.raises(ValueError):
        B._ld(x.t(), 8, 4)
    with pytest.raises(ValueError):
        B._ld(x, 4, 9)
    with pytest.raises(ValueError):
        B._ld(x, 4, 8, torch.float16)
    with pytest.raises(ValueError):
        B._vector(torch.zeros(4, dtype=torch.int64), 4, (torch.int32,))
    with pytest.raises(ValueError):
        B._vector(torch.zeros(8, dtype=torch.int32)[::2], 4, (torch.int32,))
    assert B._ld(torch.zeros((1, 8)).as_strided((1, 8), (0, 1)), 1, 8) == 8
    assert B._ld(torch.zeros((4, 16))[:, :1], 4, 1) == 16
    assert B.slope_like(x).dtype == torch.float32 and B.slope_like(x.half()).dtype == torch.int16


def test_reference_attention_against_torch():
    gen = torch.Generator().manual_seed(0)
    heads, kv_heads, D = 4, 2, 6
    Q, K, V = (torch.randn((12, h * D), generator=gen, dtype=torch.float64).float() for h in (heads, kv_heads, kv_heads))
    G = torch.randn((12, heads * D), generator=gen)
    ptr = torch.tensor([0, 5, 5, 12], dtype=torch.int32)
    mask = torch.tensor([1, 1, 0, 1, 1, 1, 0, 1, 1, 1, 1, 0], dtype=torch.uint8)
    want = ref.attention(Q, K, V, ptr, ptr, heads, kv_heads, 0.4, mask, G)
    q, k, v = (t.double().requires_grad_() for t in (Q, K, V))
    total = 0
    for a, b in ((0, 5), (5, 12)):
        s = torch.einsum("ihd,jhd->hij", q[a:b].view(-1, heads, D), k[a:b].view(-1, kv_heads, D).repeat_interleave(2, 1)) * 0.4
        p = torch.softmax(s.masked_fill(mask[a:b] == 0, -1e300), 2)
        o = torch.einsum("hij,jhd->ihd", p, v[a:b].view(-1, kv_heads, D).repeat_interleave(2, 1)).reshape(b - a, -1)
        assert np.allclose(o.detach().numpy(), want["out"][0][a:b], atol=1e-12)
        total = total + (o * G[a:b].double()).sum()
    for name, g in zip(("dQ", "dK", "dV"), torch.autograd.grad(total, [q, k, v])):
        assert np.allclose(g.numpy(), want[name][0], atol=1e-12), name


@pytest.mark.parametrize("act", ["none", "relu", "gelu", "silu"])
def test_reference_linear_against_torch(act):
    gen = torch.Generator().manual_seed(1)
    X, W, b, G = (torch.randn(s, generator=gen) for s in ((9, 5), (5, 7), (7,), (9, 7)))
    x, w, c = (t.double().requires_grad_() for t in (X, W, b))
    f = torch.nn.functional
    z = dict(none=lambda t: t, relu=f.relu, gelu=f.gelu, silu=f.silu)[act](x @ w + c)
    got = ref.linear(X, W, b, act, None, torch.float32)
    assert np.allclose(got[0], z.detach().numpy(), atol=1e-12)
    p = (x @ w + c).detach().requires_grad_()
    slope = torch.autograd.grad(dict(none=lambda t: t, relu=f.relu, gelu=f.gelu, silu=f.silu)[act](p).sum(), p)[0]
    assert np.allclose(got[2], slope.numpy(), atol=1e-12)
    back = ref.linear_backward(X, W, G, slope.float(), torch.float32, torch.float32)
    for (val, _), g in zip(back, torch.autograd.grad(z, [x, w, c], G.double())):
        assert np.allclose(val, g.numpy(), atol=1e-6)


def test_reference_embedding():
    ids = torch.tensor([1, -1, 3, 1, 9], dtype=torch.int32)
    E = torch.arange(12.0).view(4, 3)
    out, _ = ref.embedding(ids, E, 2.0, torch.float32)
    assert np.array_equal(out, np.array([[6, 8, 10], [0, 0, 0], [18, 20, 22], [6, 8, 10], [0, 0, 0]], float))
    dE, _ = ref.embedding_backward(ids, torch.ones((5, 3)), 4, 2.0, torch.float32)
    assert np.array_equal(dE, np.array([0, 4, 0, 2], float)[:, None] * np.ones(3))
