"""The gradient of a table at the numbers of ids where its positions are counted into order or sorted, in one, two and three passes."""
import pytest
import torch

from paper_2412_12218_amd import binding as B
from test_gpu_embedding import power_law_ids, rows
from transformer_reference import check, embedding_backward

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("vocab", [1, 255, 511, 512, 65_535, 262_143, 262_144, 300_000])
@pytest.mark.parametrize("n", [1, 1499, 1500, 1501, 3000, 3001, 4095, 4096, 4097])
def test_gradient_next_to_the_limits(n, vocab):
    """Ids of the table's first and last rows and outside it among them; a workspace of what the query says, with anything in it."""
    ids, g = power_law_ids(n, vocab, n), rows(n, 4, 4, torch.float32, n)
    ids[n // 4], ids[n // 5] = vocab - 1, 0
    ws = B._workspace(B.lib().ftc_embedding_backward_workspace_bytes(n, vocab, 4), "cuda")
    dE = None
    for fill in (255, 0):
        ws.fill_(fill)
        again = B.ftc_embedding_backward(ids, g, vocab, scale=1.5, ws=ws)
        assert dE is None or torch.equal(again, dE)
        dE = again
    check(f"{n} ids of {vocab}", dE, *embedding_backward(ids, g, vocab, 1.5, torch.float32))
