"""Rows of a table by id, and the table's gradient, against their formulas in 64 bits."""
import numpy as np
import pytest
import torch

from paper_2412_12218_amd import binding as B
from transformer_reference import check, embedding, embedding_backward

pytestmark = pytest.mark.gpu
DTYPES = [torch.float32, torch.float16, torch.bfloat16]


def power_law_ids(n, vocab, seed, pad=True):
    rng = np.random.default_rng(seed)
    w = np.arange(1, vocab + 1) ** -0.9
    ids = rng.permutation(vocab)[np.searchsorted(np.cumsum(w) / w.sum(), rng.random(n)).clip(max=vocab - 1)].astype(np.int32)
    if pad and n > 3:
        ids[rng.random(n) < 0.1] = -1
        ids[n // 2] = vocab          # behind the table
        ids[n // 3] = 2 ** 31 - 1
        ids[0] = -2 ** 31
    return torch.from_numpy(ids).cuda()


def rows(n, D, ld, dtype, seed, shift=0):
    """n x D of a matrix with rows of ld elements, `shift` elements from its start."""
    gen = torch.Generator().manual_seed(seed)
    whole = torch.randn(n * ld + shift, generator=gen).to(dtype).cuda()
    return whole[shift:].view(n, ld)[:, :D] if n else whole.new_empty((0, D))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n,vocab,D,ld,shift", [(1, 1, 1, 1, 0), (37, 118, 64, 64, 0), (1000, 7, 37, 40, 3), (513, 2000, 200, 200, 0),
                                               (70, 50, 1031, 1031, 1), (5, 3, 8, 24, 8), (3001, 900, 5, 5, 0)])
def test_lookup(dtype, n, vocab, D, ld, shift):
    ids, E = power_law_ids(n, vocab, n), rows(vocab, D, ld, dtype, D, shift)
    for out_dtype in {dtype, torch.float32, torch.bfloat16}:
        out = torch.full((n, D + 3), 7.0, dtype=out_dtype, device="cuda")[:, :D]
        B.ftc_embedding(ids, E, scale=2.5, out=out)
        check(f"lookup {dtype} {n} {vocab} {D} -> {out_dtype}", out, *embedding(ids, E, 2.5, out_dtype))
        whole = out.as_strided((n, D + 3), (D + 3, 1))
        assert bool((whole[:, D:] == 7.0).all())


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n,vocab,D,ld", [(1, 1, 1, 1), (1, 50, 64, 64), (37, 118, 64, 64), (1000, 7, 37, 40), (5000, 1, 9, 9), (4097, 2000, 200, 200),
                                         (20_000, 300, 17, 24), (70, 50, 1031, 1031), (40_000, 3, 128, 128), (150_000, 70_000, 4, 4)])
def test_gradient(dtype, n, vocab, D, ld):
    ids, g = power_law_ids(n, vocab, n + 1), rows(n, D, ld, dtype, D)
    for de_dtype in {dtype, torch.float32}:
        dE = torch.full((vocab, D + 5), float("nan"), dtype=de_dtype, device="cuda")[:, :D]
        B.ftc_embedding_backward(ids, g, vocab, scale=1.5, dE=dE)
        check(f"gradient {dtype} {n} {vocab} {D} -> {de_dtype}", dE, *embedding_backward(ids, g, vocab, 1.5, de_dtype))
        again = B.ftc_embedding_backward(ids, g, vocab, scale=1.5, de_dtype=de_dtype)
        assert torch.equal(again, dE)
        whole = dE.as_strided((vocab, D + 5), (D + 5, 1))
        assert bool(whole[:, D:].isnan().all())


@pytest.mark.parametrize("n", [1, 15, 16, 17, 31, 32, 33, 1024, 1025, 40_000])
def test_one_id_everywhere_and_no_id_at_all(n):
    """Runs that end with, inside and behind a chunk; positions that are all padded."""
    g = rows(n, 12, 12, torch.float32, n)
    for value in (0, 2, -1, 3):
        ids = torch.full((n,), value, dtype=torch.int32, device="cuda")
        dE = torch.full((3, 12), float("nan"), device="cuda")
        B.ftc_embedding_backward(ids, g, 3, dE=dE)
        check(f"id {value} {n} times", dE, *embedding_backward(ids, g, 3, 1.0, torch.float32))


def test_gradient_is_the_transposed_lookup():
    """<lookup(E), G> = <E, gradient(G)>, and differences of the scalar in single entries of E."""
    ids, E, G = power_law_ids(300, 40, 5), rows(40, 24, 24, torch.float32, 1), rows(300, 24, 24, torch.float32, 2)
    dE = B.ftc_embedding_backward(ids, G, 40, scale=0.75)
    f = lambda E: float((B.ftc_embedding(ids, E, scale=0.75).double() * G.double()).sum())
    # 7200 products of numbers up to 5, off by 2^-23 of themselves each
    assert abs(f(E) - float((E.double() * dE.double()).sum())) < 7200 * 25 * 2.0 ** -22
    for v, c in ((0, 0), (17, 5), (39, 23)):
        up, down = E.clone(), E.clone()
        up[v, c] += 1.0
        down[v, c] -= 1.0
        assert abs((f(up) - f(down)) / 2 - float(dE[v, c])) < 7200 * 25 * 2.0 ** -22


def test_nothing_to_do():
    E = rows(5, 8, 8, torch.float16, 0)
    none = torch.empty(0, dtype=torch.int32, device="cuda")
    assert B.ftc_embedding(none, E).shape == (0, 8)
    dE = torch.full((5, 8), 3.0, dtype=torch.float16, device="cuda")
    B.ftc_embedding_backward(none, E[:0], 5, dE=dE)
    assert bool((dE == 0).all())
    assert B.ftc_embedding_backward(power_law_ids(5, 5, 0), E, 0).shape == (0, 8)
    assert bool((B.ftc_embedding(power_law_ids(9, 5, 0), E[:0]) == 0).all())      # a table without rows


def test_infinities_stay_in_their_rows():
    g = rows(600, 8, 8, torch.float32, 3)
    ids = power_law_ids(600, 20, 4, pad=False)
    at = [int((ids == v).nonzero()[0]) for v in range(3)]
    g[at[0], 1], g[at[1], 2], g[at[2], 3] = float("inf"), float("-inf"), float("nan")
    E = B.ftc_embedding_backward(ids, g, 20)
    want, bound = embedding_backward(ids, g, 20, 1.0, torch.float32)
    check("infinities", E, want, bound)


def test_offsets_beyond_32_bits():
    """A table and a gradient whose last row begins behind 2^32 bytes and 2^31 elements."""
    ld = (1 << 30) + 8
    E = torch.empty(2 * ld + 16, dtype=torch.float16, device="cuda").as_strided((3, 16), (ld, 1))
    E.copy_(torch.arange(48, device="cuda").view(3, 16).half())
    ids = torch.tensor([2, 0, 2, 1], dtype=torch.int32, device="cuda")
    assert torch.equal(B.ftc_embedding(ids, E), E[ids.long()])
    g = torch.ones((4, 16), dtype=torch.float16, device="cuda")
    B.ftc_embedding_backward(ids, g, 3, dE=E)
    assert torch.equal(E.cpu(), torch.tensor([1.0, 1.0, 2.0]).half()[:, None].expand(3, 16))


def test_captured_and_on_another_stream():
    ids, E, g = power_law_ids(3000, 400, 9), rows(400, 64, 64, torch.float16, 1), rows(3000, 64, 64, torch.float16, 2)
    ws = B._workspace(B.lib().ftc_embedding_backward_workspace_bytes(3000, 400, 64), "cuda")
    out, dE = torch.empty_like(g), torch.empty_like(E)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        want, want_d = B.ftc_embedding(ids, E), B.ftc_embedding_backward(ids, g, 400, de_dtype=torch.float16)
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.ftc_embedding(ids, E, out=out)
        B.ftc_embedding_backward(ids, g, 400, dE=dE, ws=ws)
    for _ in range(3):
        out.fill_(float("nan"))
        dE.fill_(float("nan"))
        ws.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(dE, want_d)
        (E * 2).sum().item()
    ids.copy_(power_law_ids(3000, 400, 11))
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, B.ftc_embedding(ids, E)) and torch.equal(dE, B.ftc_embedding_backward(ids, g, 400, de_dtype=torch.float16))
