"""Attention weights of a sequence among others and alone: a batch is cut by its longest context and its most rows, so the last bits
may differ with the others of a call, within the bound that operator_ref derives; the same call gives the same bits."""
import pytest

from test_gpu_attn_weights import call, check, es, setup  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("heads,hd,dtype,n,lens", [
    ((32, 8), 128, "bf16", [6, 6], [3000, 2000]),
    ((32, 8), 128, "bf16", [1, 16], [4100, 70]),          # four waves alone, eight together
    ((28, 4), 128, "bf16", [2, 16, 1], [65, 900, 2300]),
    ((4, 2), 64, "fp32", [1, 9, 16], [128, 700, 17]),     # one launch alone, two together
])
def test_alone_and_together(es, heads, hd, dtype, n, lens):
    import torch
    slots = max(lens) + 1
    q, k, w, layout = setup(es, 81, 2, heads, hd, dtype, n, lens, slots)
    together = call(es, q, k, w, layout, n, lens, heads[0])
    assert torch.equal(together, call(es, q, k, w, layout, n, lens, heads[0]))
    check(q, k, w, n, lens, together)
    for b in range(len(n)):
        only = [x if i == b else 0 for i, x in enumerate(n)]
        rows = q[:, sum(n[:b]): sum(n[: b + 1])].contiguous()
        alone = call(es, rows, k, w, layout, only, lens, heads[0])
        assert torch.equal(alone, call(es, rows, k, w, layout, only, lens, heads[0]))
        check(rows, k, w, only, lens, alone)
