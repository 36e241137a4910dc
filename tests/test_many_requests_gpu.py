"""paged_attention over batches of more requests than a wave looks at at a time (64), some of them
without queries or slots, in one split and in several. Tolerances as in test_prompt_gpu."""
import numpy as np
import pytest
import torch

from test_prompt_gpu import Case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind,H,G,D,requests", [
    ("bf16", 1, 4, 64, 65), ("fp8", 2, 1, 32, 200), ("mxfp4", 1, 16, 64, 130), ("fp16", 1, 3, 128, 129)])
def test_ragged(kind, H, G, D, requests):
    print(f"[gpu] {kind} H={H} G={G} D={D} requests={requests}", flush=True)
    r = np.random.default_rng(requests)
    counts = r.integers(0, 90, requests)
    queries = np.minimum(r.integers(0, 41, requests), counts)
    queries[r.random(requests) < 0.3] = 0
    counts[requests - 1], queries[requests - 1] = 120, 50   # the last one, past whole rounds of 64
    c = Case(kind, H, G, D, counts.tolist(), queries.tolist(), seed=60)
    for window, sinks in ((0, 0), (20, 3)):
        out = c.check(c.run(window, sinks), window, sinks, some=4)
        assert bool((out[int(queries.sum()):] == 9).all())


@pytest.mark.parametrize("kind", ["bf16", "mxfp4"])
def test_split(kind):
    """Few queries in all, so that the keys are split and merged; the queries are in the last requests
    and in between."""
    counts = [3] * 150
    queries = [0] * 150
    for at, n, ql in ((2, 4000, 3), (63, 2000, 1), (64, 3000, 7), (100, 1100, 2), (149, 5000, 5)):
        counts[at], queries[at] = n, ql
    c = Case(kind, 1, 8, 128, counts, queries, seed=61)
    out = c.check(c.run(), some=3)
    assert bool((out[sum(queries):] == 9).all())


@pytest.mark.parametrize("kind,D", [("bf16", 128), ("fp8", 64), ("mxfp4", 128)])
def test_single_tokens(kind, D):
    r = np.random.default_rng(5)
    counts = r.integers(0, 60, 300)
    counts[299] = 2500
    c = Case(kind, 2, 2, D, counts.tolist(), [1] * 300, seed=62)
    for window in (0, 30):
        c.check(c.run(window, 2, q_indptr=None, max_queries=1), window, 2)
