"""paged_attention where its variants meet: head counts that share a workgroup's loads, single tokens
through query ranges, requests of more queries than the call allows, used workspaces, queries of far
apart sizes. Tolerances as in test_prompt_gpu (Case.check)."""
import pytest
import torch

from paper_2608_13263_amd import binding as B
import serving_helpers as S
from test_prompt_gpu import Case

pytestmark = pytest.mark.gpu


def dev(x):
    return torch.tensor(x, dtype=torch.int32).cuda()


@pytest.mark.parametrize("H", [2, 4, 6, 8])
@pytest.mark.parametrize("kind,D,act", [("bf16", 32, None), ("fp16", 32, None), ("fp8", 32, "fp16"),
                                        ("fp8", 64, "bf16"), ("mxfp4", 32, None),
                                        ("mxfp4", 64, None), ("mxfp4", 128, None),
                                        ("mxfp4", 256, None)])
def test_heads_loaded_together(kind, D, act, H):
    G = {2: 16, 4: 5, 6: 1, 8: 4}[H]
    c = Case(kind, H, G, D, [1, 63, 64, 130, 0, 1500], [1, 1, 1, 1, 1, 1], act=act, seed=20)
    for window, sinks in ((0, 0), (100, 3)):
        out = c.run(window, sinks, q_indptr=None, max_queries=1)
        c.check(out, window, sinks)
        assert bool((out[6:] == 9).all())


@pytest.mark.parametrize("kind,H,G,D", [("bf16", 2, 4, 128), ("fp8", 4, 2, 64), ("mxfp4", 4, 4, 128),
                                        ("fp16", 1, 3, 256)])
def test_single_tokens_through_ranges(kind, H, G, D):
    """Requests of no or one query, max_queries 1: rows go by q_indptr, not by the request."""
    c = Case(kind, H, G, D, [5, 40, 0, 300, 700, 64], [1, 0, 1, 1, 0, 1], seed=21)
    for window in (0, 50):
        out = c.run(window, 2, max_queries=1)
        c.check(out, window, 2)
        assert bool((out[4:] == 9).all())


def test_more_queries_than_allowed():
    """A request of more queries than max_queries: NaN in all of its rows, the others' as they are."""
    for queries, most in (([300, 2, 1], 2), ([1, 500, 2], 40), ([2, 2, 130], 129)):
        c = Case("bf16", 2, 4, 64, [600, 700, 800], queries, seed=22)
        good = c.run()
        out = c.run(max_queries=most)
        for r, ql in enumerate(queries):
            at = slice(int(c.q_indptr[r]), int(c.q_indptr[r + 1]))
            if ql > most:
                assert bool(torch.isnan(out[at]).all())
            else:   # (the splits differ between the two calls, and with them the sums' order)
                assert float((out[at].double() - good[at].double()).abs().max()) <= \
                    4 * S.HALF_STEP["bf16"] * float(good[at].abs().max())
        assert bool((out[sum(queries):] == 9).all())


@pytest.mark.parametrize("kind", ["bf16", "fp8", "mxfp4"])
@pytest.mark.parametrize("queries", [[1, 1], [9, 40]])
def test_used_workspaces(kind, queries):
    """What a workspace held before, NaN here, has no part in a call; one of the stated size does."""
    c = Case(kind, 2, 4, 128, [3000, 90], queries, seed=23)
    single = queries == [1, 1]
    kw = dict(max_queries=1) if single else {}
    want = c.run(**kw)
    t = B.CAttention(None, None, 0, 0, c.q.data_ptr(), None, None, 0, c.q.shape[0],
                     max(queries), 3000, 8, 2, 128, 1, B.KV_BF16,
                     {"bf16": B.KV_BF16, "fp8": B.KV_FP8_E4M3, "mxfp4": B.KV_MXFP4}[kind], 0, 0, 1.0)
    need = B.attention_workspace_bytes(t, 2)
    assert need > 0
    ws = torch.full((need // 4,), float("nan"), device="cuda")
    for _ in range(2):
        assert torch.equal(c.run(workspace=ws, **kw), want)
    with pytest.raises(B.VTokenError):
        c.run(workspace=ws[:-1], **kw)


@pytest.mark.parametrize("D", [32, 64, 128, 256])
def test_4_bit_scores_of_queries_far_apart(D):
    """A query's values go in as two 8-bit parts: exact down to 2^-9 of the largest, off by at most
    2^-17 of it below. A score is then off by at most E = 2^-17 max |q| sum |k| |scale|, a weight and
    its share of the normaliser by E each: 2 E A."""
    c = Case("mxfp4", 2, 4, D, [200, 700], [1, 1], seed=24)
    g = torch.Generator().manual_seed(25)
    size = 2.0 ** (-14 * torch.rand(c.q.shape, generator=g))
    c.q = (c.q.sign() * size * 4).to(torch.bfloat16)
    c.q[0, 1] = 0
    c.q[1, 2, 5:] = 0
    c.q[1, 3] = float("nan")
    out = c.run(q_indptr=None, max_queries=1).double().cpu()
    scale = D ** -0.5
    for r in range(2):
        sl = c.slots[c.indptr[r]: c.indptr[r + 1]].long()
        k, v = (S.values(c.rows[i][sl], "mxfp4", 2, D) for i in (0, 1))
        ref, A = S.attention(c.q[r: r + 1], k, v, 0, 0, scale)
        E = 2.0 ** -17 * c.q[r].double().abs().max(-1).values * scale * \
            k.abs().sum(-1).max(0).values.repeat_interleave(4)
        h = S.HALF_STEP["bf16"]
        tol = 1.01 * h * (A[0] + ref[0].abs()) + \
            (2.0 ** -17 * D + 2.0 ** -18 + 2 * E[:, None]) * A[0]
        nan = torch.isnan(ref[0])
        assert torch.equal(torch.isnan(out[r]), nan)
        assert bool(((out[r] - ref[0]).abs() <= tol)[~nan].all())


@pytest.mark.parametrize("kind", ["bf16", "fp8", "mxfp4"])
def test_widest_windows(kind):
    """Windows and first tokens up to the type's last value are every token."""
    for queries in ([1], [30], [80]):
        c = Case(kind, 2, 2, 64, [70], queries, seed=26)
        kw = dict(q_indptr=None, max_queries=1) if queries == [1] else {}
        want = c.run(**kw)
        for window, sinks in ((2 ** 31 - 1, 0), (2 ** 30, 2 ** 31 - 1), (1, 2 ** 31 - 1), (70, 0)):
            got = c.run(window, sinks, **kw)
            c.check(got, min(window, 10 ** 6), min(sinks, 10 ** 6))
            assert float((got.double() - want.double()).abs().max()) <= \
                4 * S.HALF_STEP["bf16"] * float(want[:queries[0]].abs().max())


@pytest.mark.parametrize("kind", ["bf16", "fp8", "mxfp4"])
def test_wide_heads_over_splits(kind):
    """256 dims, few queries of many keys: the splits' records and their merge."""
    c = Case(kind, 1, 6, 256, [3000, 500], [7, 25], seed=27)
    for window, sinks in ((0, 0), (900, 4)):
        c.check(c.run(window, sinks), window, sinks, some=6)


def test_a_stream_by_its_handle():
    c = Case("bf16", 2, 4, 128, [3000], [1], seed=28)
    want = c.run(q_indptr=None, max_queries=1)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for stream in (side, side.cuda_stream):
        with torch.cuda.stream(side):
            out = torch.full(c.q.shape, 9.0, dtype=c.q.dtype, device="cuda")
        torch.cuda.synchronize()
        got = c.run(q_indptr=None, max_queries=1, stream=stream, out=out)
        torch.cuda.synchronize()
        assert torch.equal(got, want)
