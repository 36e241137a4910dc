"""paged_attention where a poisoned key (a slot outside the pool, a NaN or an infinity in K or V) lies
far below the row's other scores: its own weight is zero in float32, and it still reaches every query
that sees it, whichever wave or split meets it."""
import pytest
import torch

from paper_2608_13263_amd import binding as B
import serving_helpers as S
from test_prompt_gpu import Case

pytestmark = pytest.mark.gpu

SINGLE = [("bf16", 2, 4, 128), ("fp16", 1, 3, 256), ("fp8", 1, 8, 128),    # a head to a workgroup
          ("bf16", 4, 2, 32), ("fp8", 2, 4, 64), ("fp8", 1, 1, 32),        # heads loaded together
          ("mxfp4", 4, 4, 128), ("mxfp4", 1, 8, 64), ("mxfp4", 3, 1, 256)]
PROMPT = [("bf16", 2, 4, 128), ("fp16", 1, 2, 64), ("bf16", 1, 3, 256), ("fp8", 1, 8, 128),
          ("fp8", 2, 1, 32), ("mxfp4", 1, 4, 128), ("mxfp4", 2, 2, 64)]


def _poisoned(shapes):
    """Every shape with every poison; e4m3 and e2m1 have no infinity."""
    return [(*s, p) for s in shapes for p in ("slot", "k nan", "v nan", "v inf")
            if p != "v inf" or s[0] in ("bf16", "fp16")]


def _far_apart(kind, H, G, D, n, queries, poison, at, high):
    """Keys of -2 but those at `high`, of 2; queries of 8: scores of -16 D^0.5 and 16 D^0.5 after the
    scale, 2 x 16 D^0.5 log2(e) >= 261 powers of two apart (a float32 power ends at 2^-150)."""
    c = Case(kind, H, G, D, [n], [queries], seed=30)
    x = torch.full((2, n, H, D), -2.0)
    x[0, high] = 2.0
    x[1] = 1.0
    packed = [S.pack4(p) if kind == "mxfp4" else p.to(S.TYPES[kind]).view(torch.uint8).reshape(n, -1)
              for p in x]
    rows = S.bytes_of(c.cache).clone()
    for plane, p in enumerate(packed):
        rows[2 + plane][c.slots.long()] = p
    c.q = torch.full_like(c.q, 8.0)
    if poison != "slot":
        row = rows[2 if poison[0] == "k" else 3][int(c.slots[at])]
        if kind == "mxfp4":
            row[H * D // 2: H * D // 2 + H * D // 32] = 255
        elif kind == "fp8":
            row[:] = 127
        else:
            row.view(S.TYPES[kind])[:] = float(poison[2:])
    else:
        c.slots[at] = c.num_slots
    c.cache.kv.view(torch.uint8).reshape(rows.shape).copy_(rows)
    return c


@pytest.mark.parametrize("kind,H,G,D,poison", _poisoned(SINGLE))
def test_single_tokens(kind, H, G, D, poison):
    """Every kernel of single tokens, over one split and over several."""
    for n in (150, 5000):
        for at, high in ((n - 1, [0]), (0, [n - 1]), (n // 2, [1, n - 2])):
            print(f"[gpu] {kind} H={H} D={D} n={n} {poison} at {at}", flush=True)
            c = _far_apart(kind, H, G, D, n, 1, poison, at, high)
            for window, sinks in ((0, 0), (n - 1, 1)):
                out = c.run(window, sinks, q_indptr=None, max_queries=1)[:1]
                if poison == "v inf":
                    assert not bool(torch.isfinite(out).any())
                else:
                    assert bool(torch.isnan(out).all())
            if at < n - 1:   # a window that hides it
                out = c.run(n - 1 - at, 0, q_indptr=None, max_queries=1)[:1]
                assert bool((out == 1).all())


@pytest.mark.parametrize("kind,H,G,D,poison", _poisoned(PROMPT))
def test_prompts(kind, H, G, D, poison):
    queries = 7
    for n in (150, 6000):
        for at, high in ((n - 4, [0]), (2, [n - 7]), (n // 2, [1, n - 7])):
            print(f"[gpu] {kind} H={H} D={D} n={n} {poison} at {at}", flush=True)
            c = _far_apart(kind, H, G, D, n, queries, poison, at, high)
            ranks = torch.arange(n - queries, n)
            for window, sinks in ((0, 0), (n - 5, 1)):
                out = c.run(window, sinks)[:queries].cpu()
                sees = (ranks >= at) & ((at > ranks - window) | (at < sinks) if window else True)
                lost = ~torch.isfinite(out) if poison == "v inf" else torch.isnan(out)
                assert torch.equal(lost.all(-1).all(-1), sees)
                assert torch.equal(lost.any(-1).any(-1), sees)
                assert bool((out[~sees] == 1).all())


@pytest.mark.parametrize("e", [253, 254, 255])
@pytest.mark.parametrize("H,D,queries", [(2, 64, 90), (1, 128, 30), (4, 32, 1)])
def test_largest_exponents_that_are_hidden(e, H, D, queries):
    """4-bit values that bf16 holds as infinities, in V (and K) of a key that some queries do not see."""
    n, at = 200, 195 if queries > 1 else 20
    for window, sinks in ((0, 0), (150, 4)):
        c = Case("mxfp4", H, 4, D, [n], [queries], seed=31)
        kw = dict(q_indptr=None, max_queries=1) if queries == 1 else {}
        clean = c.run(window, sinks, **kw)[:queries].cpu()
        rows = S.bytes_of(c.cache).clone()
        for plane in (2, 3):
            row = rows[plane][int(c.slots[at])]
            row[: H * D // 2] = 0x7F    # 6 and -6
            row[H * D // 2: H * D // 2 + H * D // 32] = e
        c.cache.kv.view(torch.uint8).reshape(rows.shape).copy_(rows)
        out = c.run(window, sinks, **kw)[:queries].cpu()
        p = torch.arange(n - queries, n)
        sees = (p >= at) & (((p - window) < at) | (at < sinks) if window else True)
        if e == 255:   # (6 x 2^126 and more are numbers, which a weight of zero leaves out)
            assert not bool(torch.isfinite(out[sees]).any())
        assert bool(((out[~sees].double() - clean[~sees].double()).abs() <= 4 * S.HALF_STEP["bf16"]
                     * float(clean.abs().max())).all())
