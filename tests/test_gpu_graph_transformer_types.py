"""Feed-forward blocks by node type inside the path: what goes back through them is added to the residual stream's gradient as it is without types, before one rounding."""
import pytest
import torch

from paper_2412_12218_amd import binding as B
from test_gpu_graph_transformer_blocks import FORMS, LAYERS, batch, path_of, weights

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("form", [FORMS[3], (B.FTC_NORM_NONE, B.FTC_NORM_RMS, True, 0.75, True)], ids=str)
@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
def test_gradient_of_the_stream(monkeypatch, dtype, form):
    lens, n, ptr, ids, mask, d_out, types = batch(dtype)
    w, path, norm, grouped, seen = weights(dtype, form), path_of(form, n, ptr, types, dtype), B.ftc_block_norm_backward, B.ftc_grouped_linear_backward, []

    def watched_norm(X, stats, dH=None, **k):
        before = dH.clone()
        got = norm(X, stats, dH=dH, **k)
        seen.append((before, got.dX.clone()))
        return got

    def watched_grouped(X, W, group_ptr, dZ, slope=None, **k):
        if slope is not None:   # the block's first product: its gradient by itself, in fp32
            seen.append(grouped(X, W, group_ptr, dZ, slope=slope, want_dW=False, want_db=False, dx_dtype=torch.float32)[0])
        return grouped(X, W, group_ptr, dZ, slope=slope, **k)
    path.forward(ids, w, mask=mask)
    monkeypatch.setattr(B, "ftc_block_norm_backward", watched_norm)
    monkeypatch.setattr(B, "ftc_grouped_linear_backward", watched_grouped)
    path.backward(ids, w, d_out, mask=mask)
    # of each layer: the join behind its feed-forward block, the block, the join behind its attention
    assert len(seen) == 3 * LAYERS
    for (_, stream), block, (added, _) in zip(seen[::3], seen[1::3], seen[2::3]):
        assert torch.equal(added, (stream.float() + block[path.inv.long()]).to(dtype))
