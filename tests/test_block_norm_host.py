"""What the calls of the norms around a block refuse, on the host, before anything is launched (the pointers are never followed).  CPU only."""
import ctypes as C

import pytest
import torch

from paper_2412_12218_amd import binding as B

P = lambda i: 0x10000 * i
INVALID, UNSUPPORTED, ALIGN, WORKSPACE = B.FTC_EINVAL, B.FTC_EUNSUPPORTED, B.FTC_EALIGN, B.FTC_EWORKSPACE
BLOCK = dict(n=4, d=8, dtype=1, post=1, pre=2, eps=1e-5, x_scale=1.0, X=P(1), F=P(2), gate=P(3), post_w=P(4), post_b=P(5), pre_w=P(6), pre_b=P(7), ldx=8,
             ldf=8, ldg=0)
GRADS = dict(dX=P(20), dF=P(21), dgate=P(22), dpost_w=P(23), dpost_b=P(24), dpre_w=P(25), dpre_b=P(26), lddx=8, lddf=8, lddg=8, dw_dtype=0)


def split(k, base):
    return B.ftc_block(*(base | {x: v for x, v in k.items() if x in base}).values()), {x: v for x, v in k.items() if x not in base}


def forward(**k):
    b, rest = split(k, BLOCK)
    a = dict(H=P(10), ldh=8, U=P(11), ldu=8, stats=P(12)) | rest
    return B.lib().ftc_block_norm(C.byref(b), *a.values(), None)


def backward(**k):
    b, rest = split(k, BLOCK)
    g = B.ftc_block_grads(*(GRADS | {x: v for x, v in rest.items() if x in GRADS}).values())
    a = dict(stats=P(12), dH=P(13), lddh=8, dU=P(14), lddu=8) | {x: v for x, v in rest.items() if x in ("stats", "dH", "lddh", "dU", "lddu")}
    w = dict(ws=P(30), bytes=1 << 40) | {x: v for x, v in rest.items() if x in ("ws", "bytes")}
    return B.lib().ftc_block_norm_backward(C.byref(b), *a.values(), C.byref(g), *w.values(), None)


BOTH = [(dict(n=-1), INVALID), (dict(d=0), INVALID), (dict(d=16385, ldx=16385, ldf=16385), UNSUPPORTED), (dict(n=(1 << 30) + 1), UNSUPPORTED), (dict(dtype=3), UNSUPPORTED),
        (dict(post=3), INVALID), (dict(pre=-1), INVALID), (dict(eps=0.0), INVALID), (dict(eps=-1.0), INVALID), (dict(eps=float("nan")), INVALID),
        (dict(eps=float("inf")), INVALID), (dict(x_scale=float("nan")), INVALID), (dict(F=None), INVALID), (dict(F=None, post=0, post_w=None, post_b=None), INVALID),
        (dict(post=0), INVALID), (dict(pre=0), INVALID), (dict(X=None), INVALID), (dict(ldx=7), INVALID), (dict(ldf=7), INVALID), (dict(ldg=7), INVALID),
        (dict(X=P(1) + 1), ALIGN), (dict(pre_w=P(6) + 1), ALIGN), (dict(gate=P(3) + 1), ALIGN), (dict(stats=P(12) + 4), ALIGN)]
CASES = [(f, k, code) for f in (forward, backward) for k, code in BOTH] + [
    (forward, dict(H=None, U=None), INVALID), (forward, dict(pre=0, pre_w=None, pre_b=None), INVALID), (forward, dict(ldh=7), INVALID), (forward, dict(ldu=7), INVALID),
    (forward, dict(H=P(2)), INVALID), (forward, dict(U=P(1)), INVALID), (forward, dict(U=P(10)), INVALID), (forward, dict(U=P(6)), INVALID),
    (forward, dict(H=P(1), ldh=9), INVALID), (forward, dict(stats=P(11)), INVALID), (forward, dict(U=P(11) + 1), ALIGN),
    (backward, dict(pre=0, pre_w=None, pre_b=None, dpre_w=None, dpre_b=None), INVALID), (backward, dict(stats=None), INVALID), (backward, dict(lddh=7), INVALID),
    (backward, dict(lddu=7), INVALID), (backward, dict(lddx=7), INVALID), (backward, dict(lddf=7), INVALID), (backward, dict(ldg=8, lddg=7), INVALID),
    (backward, dict(gate=None), INVALID), (backward, dict(post_w=None), INVALID), (backward, dict(pre_w=None), INVALID), (backward, dict(dw_dtype=2), UNSUPPORTED),
    (backward, dict(dw_dtype=5), UNSUPPORTED), (backward, dict(dX=P(1)), INVALID), (backward, dict(dX=P(14)), INVALID), (backward, dict(dF=P(13)), INVALID),
    (backward, dict(dX=P(13), lddh=9), INVALID), (backward, dict(dgate=P(3)), INVALID), (backward, dict(dF=P(20)), INVALID), (backward, dict(dpre_w=P(23)), INVALID),
    (backward, dict(ws=None), WORKSPACE), (backward, dict(bytes=64), WORKSPACE), (backward, dict(ws=P(30) + 16), ALIGN), (backward, dict(dX=P(20) + 1), ALIGN)]


@pytest.mark.parametrize("call,args,code", CASES, ids=lambda x: getattr(x, "__name__", str(x)))
def test_refused(call, args, code):
    assert call(**args) == code, B.lib().ftc_last_error()
    assert call.__name__ in B.lib().ftc_last_error().decode().replace("ftc_block_norm_backward", "backward").replace("ftc_block_norm", "forward")


def test_null_structs():
    assert B.lib().ftc_block_norm(None, P(1), 8, None, 0, None, None) == INVALID
    assert B.lib().ftc_block_norm_backward(None, None, None, 0, None, 0, None, None, 0, None) == INVALID
    b = B.ftc_block(*BLOCK.values())
    assert B.lib().ftc_block_norm_backward(C.byref(b), P(12), None, 0, None, 0, None, P(30), 1 << 40, None) == INVALID


def test_nothing_to_do():
    assert forward(n=0, X=None, F=None, post_b=None, H=None, U=None) == B.FTC_OK
    assert B.lib().ftc_block_norm_backward_workspace_bytes(0, 8) == 0
    assert B.lib().ftc_block_norm_backward_workspace_bytes(-1, 8) == 0 and B.lib().ftc_block_norm_backward_workspace_bytes(4, 16385) == 0
    # what a launch's groups write, at most two of 256 threads a compute unit
    assert 0 < B.lib().ftc_block_norm_backward_workspace_bytes(1 << 30, 16384) <= 5 * 512 * 16384 * 4


def test_binding_refuses(monkeypatch):
    X, w = torch.zeros(4, 8), torch.zeros(8)
    monkeypatch.setattr(B, "_here", lambda *t: 0)
    for k in (dict(pre_w=torch.zeros(7)), dict(pre_w=w.double()), dict(F=torch.zeros(4, 7)), dict(F=torch.zeros(4, 8).half()), dict(gate=torch.zeros(3, 8)), dict(F=X, gate=torch.zeros(8).expand(4, 8)),
              dict(gate=torch.zeros(7)), dict(stats=torch.zeros(4, 3)), dict(stats=torch.zeros(4, 4).double()), dict(H=torch.zeros(4, 9)),
              dict(U=torch.zeros(4, 8).half()), dict(F=torch.zeros(8, 4).t())):
        with pytest.raises(ValueError):
            B.ftc_block_norm(X, **k)
