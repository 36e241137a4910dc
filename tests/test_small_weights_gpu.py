"""paged_attention over many keys that are each far below the row's largest: their weights are small,
their sum is not."""
import pytest
import torch

from paper_2608_13263_amd import binding as B
import serving_helpers as S

pytestmark = pytest.mark.gpu


def _call(kind, act, H, G, D, n, queries):
    """One key of 2.25, n - 1 of 0, a query of 1: scores of 18 and 0 after a scale of 8 / D, 26 powers
    of two apart. Values 0 and 1: the output is the share of the small weights."""
    x = torch.zeros(2, n, H, D)
    x[0, 0] = 2.25
    x[1, 1:] = 1.0
    size = -(-n // 16) * 16
    planes = torch.stack([S.pack4(p) if kind == "mxfp4" else
                          p.to(S.TYPES[kind]).view(torch.uint8).reshape(n, -1) for p in x])
    planes = torch.nn.functional.pad(planes, (0, 0, 0, size - n))
    cache = S.make_cache(B, planes, kind, H, D, 16)
    dev = lambda v: torch.tensor(v, dtype=torch.int32).cuda()   # noqa: E731
    q = torch.ones(queries, H * G, D, dtype=S.TYPES[act], device="cuda")
    out = B.paged_attention(cache, q, dev([0, n]), torch.arange(n, dtype=torch.int32).cuda(), 0, n,
                            q_indptr=dev([0, queries]), max_queries=queries, scale=8 / D)
    return out.double().cpu()


@pytest.mark.parametrize("kind,act,H,G,D,n,queries", [
    ("fp16", "fp16", 1, 4, 64, 40000, 1), ("fp16", "fp16", 2, 2, 32, 30000, 1),
    ("fp8", "fp16", 1, 1, 128, 40000, 1), ("bf16", "bf16", 1, 4, 128, 40000, 1),
    ("fp16", "fp16", 8, 16, 64, 20000, 520),    # tiles enough for one split
    ("fp16", "fp16", 1, 4, 128, 40000, 9), ("fp8", "fp16", 8, 16, 64, 20000, 520),
    ("bf16", "bf16", 8, 16, 64, 20000, 520)])
def test_many_far_below(kind, act, H, G, D, n, queries):
    """A weight is rounded by at most half a step of its type, relative, and fp16 by 2^-36 of the
    row's largest where its relative steps end (weights are 2^11 and more times what is taken
    relative to the largest, and fp16's last step is 2^-24); the score's and the exponential's
    parts are as in test_prompt_gpu."""
    print(f"[gpu] {kind} {act} H={H} D={D} n={n} queries={queries}", flush=True)
    out = _call(kind, act, H, G, D, n, queries)
    low = (n - queries + torch.arange(queries, dtype=torch.float64)) * torch.exp(
        torch.tensor(-18.0, dtype=torch.float64))
    ref = (low / (1 + low))[:, None, None]
    tol = 2.02 * S.HALF_STEP[act] * ref + (2.0 ** -17 * D + 2.0 ** -18) * ref + S.HALF_TINY[act]
    if act == "fp16":
        tol = tol + n * 2.0 ** -36
    assert bool(((out - ref).abs() <= tol).all()), float(((out - ref).abs() / tol).max())
