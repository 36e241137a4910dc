"""paged_attention of single tokens: softmax weights keep more than the activations' bits for the product
with V (bf16: two parts), so that what is left is the output's own rounding."""
import pytest
import torch

import serving_helpers as S
from test_prompt_gpu import Case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind,H,G,D", [
    ("bf16", 2, 4, 32), ("bf16", 2, 4, 64), ("bf16", 1, 8, 128), ("bf16", 2, 3, 256),
    ("fp8", 1, 5, 32), ("fp8", 2, 4, 64), ("fp8", 2, 2, 128), ("fp8", 1, 4, 256),
    ("mxfp4", 4, 4, 32), ("mxfp4", 1, 7, 64), ("mxfp4", 2, 8, 128), ("mxfp4", 1, 2, 256)])
def test_bf16(kind, H, G, D):
    """Tolerance: the output's rounding, half a step; the upper part of a weight is cut off at 2^-7 of
    it, the lower rounded at 2^-8 of that: 2^-15 A for the weights, with A the attention of |V|; scores
    and exponentials as in test_prompt_gpu; 4-bit scores off by E = 2^-17 max |q| sum |k| |scale|, 2 E A
    (test_attention_edges_gpu)."""
    print(f"[gpu] {kind} H={H} G={G} D={D}", flush=True)
    counts = [1, 2, 3, 9, 31, 64, 65, 130, 700, 3000]
    c = Case(kind, H, G, D, counts, [1] * len(counts), seed=50)
    for window, sinks in ((0, 0), (100, 4)):
        out = c.run(window, sinks, q_indptr=None, max_queries=1).double().cpu()
        for r, n in enumerate(counts):
            sl = c.slots[c.indptr[r]: c.indptr[r + 1]].long()
            k, v = (S.values(c.rows[i][sl], kind, H, D) for i in (0, 1))
            ref, A = S.attention(c.q[r: r + 1], k, v, window, sinks, D ** -0.5)
            E = 2.0 ** -17 * c.q[r].double().abs().max(-1).values * D ** -0.5 * \
                k.abs().sum(-1).max(0).values.repeat_interleave(G) * (kind == "mxfp4")
            tol = 1.01 * S.HALF_STEP["bf16"] * ref[0].abs() + \
                (2.0 ** -15 + 2.0 ** -17 * D + 2.0 ** -18 + 2 * E[:, None]) * A[0] + 2.0 ** -134
            assert bool(((out[r] - ref[0]).abs() <= tol).all()), (
                r, n, float(((out[r] - ref[0]).abs() / tol).max()))
