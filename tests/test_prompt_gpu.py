"""paged_attention against its definition in 64 bits.

Tolerance. With A the attention of |V| (what the weights sum to): each weight is rounded once to
16 bits before the product with V, half a step each, so at most HALF_STEP A; the output's rounding
is HALF_STEP of it; a score is a float32 sum of D exact products, off by at most D 2^-24 of the sum
of their magnitudes (here below 64 after the scale: 2^-24 D 64), and the exponential by 2^-20, both
relative to a weight and its share of the normaliser: twice (2^-18 D + 2^-20) A, taken as
(2^-17 D + 2^-18) A for scores that float32 sums in any order."""
import numpy as np
import pytest
import torch

from paper_2608_13263_amd import binding as B
from paper_2608_13263_amd import workloads as W
import serving_helpers as S

pytestmark = pytest.mark.gpu


class Case:
    """A ragged batch over one layer of a two-layer cache, its slots spread over the pool."""

    def __init__(self, kind, H, G, D, counts, queries, act=None, seed=0, extra=3, block=16):
        act = act or ("fp16" if kind == "fp16" else "bf16")
        self.kind, self.H, self.G, self.D, self.act = kind, H, G, D, act
        self.counts, self.queries = list(counts), list(queries)
        g = torch.Generator().manual_seed(seed + D + G)
        total = sum(counts)
        self.num_slots = (total // block + 2) * block
        self.rows = torch.stack([S.make_rows(kind, self.num_slots, H, D, g) for _ in range(2)])
        other = torch.stack([S.make_rows(kind, self.num_slots, H, D, g) for _ in range(2)])
        self.cache = S.make_cache(B, torch.cat([other, self.rows]), kind, H, D, block)
        self.slots = torch.randperm(self.num_slots, generator=g)[:total].to(torch.int32)
        self.indptr = np.concatenate([[0], np.cumsum(counts)])
        self.q_indptr = np.concatenate([[0], np.cumsum(queries)])
        self.q = torch.randn(sum(queries) + extra, H * G, D, generator=g).to(S.TYPES[act])

    def run(self, window=0, sinks=0, **kw):
        dev = lambda x: torch.as_tensor(np.asarray(x), dtype=torch.int32).cuda()   # noqa: E731
        if "q_indptr" not in kw:
            kw["q_indptr"] = dev(self.q_indptr)
        out = torch.full(self.q.shape, 9.0, dtype=self.q.dtype, device="cuda")
        kw.setdefault("out", out)
        kw.setdefault("max_queries", max(self.queries + [1]))
        return B.paged_attention(self.cache, kw.pop("q", self.q.cuda()), dev(self.indptr),
                                 kw.pop("slots", self.slots.cuda()), 1,
                                 kw.pop("max_tokens", max(self.counts)), window=window,
                                 sinks=sinks, **kw)

    def check(self, out, window=0, sinks=0, scale=None, some=None):
        scale = self.D ** -0.5 if scale is None else scale
        out = out.double().cpu()
        for r, (n, ql) in enumerate(zip(self.counts, self.queries)):
            sl = self.slots[self.indptr[r]: self.indptr[r + 1]].long()
            k, v = (S.values(self.rows[i][sl], self.kind, self.H, self.D) for i in (0, 1))
            at = int(self.q_indptr[r])
            pick = range(ql) if some is None or ql <= some else sorted(
                {0, 1, ql - 1, ql - 2, *np.random.default_rng(r).integers(0, ql, some).tolist()})
            for i in pick:
                m = n - ql + i + 1   # the query as the last of the tokens it may see
                ref, size = S.attention(self.q[at + i: at + i + 1], k[: max(m, 0)], v[: max(m, 0)],
                                        window, sinks, scale)
                h = S.HALF_STEP[self.act]
                tol = 1.01 * h * (size + ref.abs()) + (2.0 ** -17 * self.D + 2.0 ** -18) * size \
                    + S.HALF_TINY[self.act]
                err = (out[at + i] - ref[0]).abs()
                assert bool((err <= tol[0]).all()), (r, i, n, ql, float((err - tol[0]).max()))
        return out


ALL = [("fp16", 2, 4, 64, None), ("bf16", 1, 8, 128, None), ("bf16", 3, 1, 32, None),
       ("fp16", 1, 2, 256, None), ("bf16", 2, 3, 256, None), ("fp8", 2, 2, 128, "bf16"),
       ("fp8", 1, 16, 64, "fp16"), ("fp8", 1, 5, 32, "bf16"), ("fp8", 1, 4, 256, "bf16"),
       ("mxfp4", 2, 8, 128, None), ("mxfp4", 1, 7, 64, None), ("mxfp4", 3, 4, 32, None),
       ("mxfp4", 1, 1, 256, None)]
MASKS = [(0, 0), (0, 5), (1, 0), (1, 1), (70, 0), (64, 4), (33, 130)]


@pytest.mark.parametrize("kind,H,G,D,act", ALL)
def test_single_tokens(kind, H, G, D, act):
    """One query per request, without q_indptr: lengths of zero, one, around the tiles of 16 to 64
    and the splits, under every mask."""
    print(f"[gpu] single tokens {kind} H={H} G={G} D={D}", flush=True)
    counts = [0, 1, 15, 16, 17, 63, 64, 65, 129, 300, 701]
    c = Case(kind, H, G, D, counts, [1] * len(counts), act)
    for window, sinks in MASKS:
        out = c.check(c.run(window, sinks, q_indptr=None, max_queries=1), window, sinks)
        assert bool((out[0] == 0).all()) and bool((out[len(counts):] == 9).all())


@pytest.mark.parametrize("kind,H,G,D,act", ALL)
def test_ragged_prompts(kind, H, G, D, act):
    """Whole prompts, chunks at the end of longer contexts, single tokens, more queries than slots
    and empty requests in one batch, under every mask."""
    print(f"[gpu] ragged prompts {kind} H={H} G={G} D={D}", flush=True)
    counts = [70, 0, 200, 1, 33, 129, 5, 260, 90]
    queries = [70, 0, 3, 1, 32, 1, 8, 65, 0]
    c = Case(kind, H, G, D, counts, queries, act, seed=1)
    for window, sinks in MASKS:
        out = c.check(c.run(window, sinks), window, sinks, some=12)
        assert bool((out[sum(queries):] == 9).all())
        assert bool((out[c.q_indptr[6]: c.q_indptr[6] + 3] == 0).all())   # ranks below zero


@pytest.mark.parametrize("kind,H,G,D,counts,queries,window,sinks", [
    ("bf16", 1, 4, 128, [5000, 3], [2, 1], 0, 0),       # split over the slots
    ("mxfp4", 1, 8, 128, [9001], [13], 0, 0),
    ("fp8", 2, 1, 64, [4100, 4099], [1, 130], 3000, 7),
    ("fp16", 1, 1, 256, [2500], [700], 0, 0),
    ("bf16", 2, 2, 64, [1500, 800, 10], [1500, 100, 10], 257, 70),
    ("mxfp4", 1, 3, 64, [1111], [1111], 100, 1),
])
def test_long(kind, H, G, D, counts, queries, window, sinks):
    print(f"[gpu] long {kind} {counts} {queries}", flush=True)
    c = Case(kind, H, G, D, counts, queries, seed=2)
    c.check(c.run(window, sinks), window, sinks, some=10)


@pytest.mark.parametrize("kind,counts", [("bf16", [20000, 9, 0]), ("mxfp4", [33000]),
                                         ("fp8", [12345, 12000]), ("fp16", [8000] * 3)])
def test_long_single_tokens(kind, counts):
    print(f"[gpu] long single tokens {kind} {counts}", flush=True)
    c = Case(kind, 1, 4, 128, counts, [1] * len(counts), seed=3)
    for window, sinks, bound in ((0, 0, max(counts)), (5000, 64, max(counts)),
                                 (0, 0, 4 * max(counts))):
        c.check(c.run(window, sinks, q_indptr=None, max_queries=1, max_tokens=bound), window,
                sinks)


def test_slots_outside_reach_only_who_sees_them():
    """A slot outside the pool: NaN for the queries that see it, none dereferenced."""
    for queries, single in (([40], False), ([1], True)):
        c = Case("bf16", 2, 4, 128, [200], queries, seed=4)
        for bad, window in ((-1, 0), (2 ** 31 - 1, 0), (c.num_slots, 30)):
            slots = c.slots.clone()
            slots[180] = bad
            kw = dict(q_indptr=None, max_queries=1) if single else {}
            out = c.run(window, 0, slots=slots.cuda(), **kw).cpu()
            ranks = torch.arange(200 - queries[0], 200)
            sees = (ranks >= 180) & ((window == 0) | (180 > ranks - (window or 1)))
            got = torch.isnan(out[: queries[0]]).all(-1).all(-1)
            assert torch.equal(got, sees)
            assert torch.equal(torch.isnan(out[: queries[0]]).any(-1).any(-1), sees)


@pytest.mark.parametrize("kind", ["bf16", "fp8", "mxfp4"])
def test_masked_keys_may_hold_anything(kind):
    """NaN and infinities in K and V of tokens that a query does not see leave it alone; those that
    see them have them."""
    for at, n, queries, window, sinks in ((130, 200, 90, 0, 0), (60, 200, 90, 64, 4),
                                          (199, 200, 5, 0, 0), (10, 400, 1, 100, 4)):
        c = Case(kind, 2, 4, 64, [n], [queries], seed=5)
        clean = c.run(window, sinks)
        rows = S.bytes_of(c.cache).clone()
        for plane in (2, 3):
            row = rows[plane][int(c.slots[at])]
            if kind == "mxfp4":
                row[2 * 32:2 * 32 + 4] = 255
            elif kind == "fp8":
                row[:] = 127
            else:
                row.view(torch.bfloat16)[:] = float("inf") if plane == 3 else float("nan")
        c.cache.kv.view(torch.uint8).reshape(rows.shape).copy_(rows)
        for single in ([False, True] if queries == 1 else [False]):
            kw = dict(q_indptr=None, max_queries=1) if single else {}
            got = c.run(window, sinks, **kw)
            p = torch.arange(n - queries, n)
            sees = (p >= at) & (((p - window) < at) | (at < sinks) if window else True)
            some = torch.isfinite(got[:queries]).cpu()
            assert bool(some[~sees].all()) and not bool(some[sees].any())
            for i in (~sees).nonzero()[:, 0].tolist():
                a, b = got[i].double(), clean[i].double()
                assert float((a - b).abs().max()) <= 4 * S.HALF_STEP["bf16"] * float(
                    b.abs().max()) + 1e-3


@pytest.mark.parametrize("kind,D", [("bf16", 32), ("bf16", 128), ("fp16", 32), ("fp16", 64)])
def test_infinities_that_are_seen(kind, D):
    """An infinity of V in a token that a query sees is that output's, of its KV head and value, also
    where the tokens end inside a tile."""
    for n in (1, 5, 77, 130, 2049):
        for queries in ([1], [min(n, 3)]):
            c = Case(kind, 2, 4, D, [n], queries, seed=6)
            rows = S.bytes_of(c.cache).clone()
            last = rows[3][int(c.slots[n - 1])].view(S.TYPES[kind])
            last[3], last[D + D - 1] = float("inf"), float("-inf")
            c.cache.kv.view(torch.uint8).reshape(rows.shape).copy_(rows)
            kw = dict(q_indptr=None, max_queries=1) if queries == [1] else {}
            got = c.run(0, 0, **kw).cpu()
            want = torch.zeros(8, D)
            want[:4, 3], want[4:, D - 1] = float("inf"), float("-inf")
            sees = got[queries[0] - 1]
            assert torch.equal(torch.where(torch.isfinite(sees), 0.0, sees.float()), want)
            assert bool(torch.isfinite(got[: queries[0] - 1]).all())


def test_scores_far_apart():
    """Scores over the whole of float32's exponent: one key far above, keys far below; equal scores
    of a large size; a scale of zero and one below zero."""
    c = Case("bf16", 1, 2, 64, [300], [20], seed=6)
    x = c.rows.view(torch.bfloat16).view(2, -1, 1, 64)
    x[0] *= 100
    c.cache.kv[2] = x[0].view(c.cache.kv[2].shape).cuda()
    q = (c.q.float() * 100).to(torch.bfloat16)
    c.q = q
    out = c.run().double().cpu()
    sl = c.slots.long()
    k, v = (S.values(c.rows[i][sl], "bf16", 1, 64) for i in (0, 1))
    for i in range(20):
        m = 280 + i + 1
        s = torch.einsum("hd,nd->hn", c.q[i].double(), k[:m, 0]) * 64 ** -0.5
        top2 = s.topk(2).values
        for h in range(2):   # differences of many thousands: one weight is 1, the others 0
            if top2[h, 0] - top2[h, 1] > 200:
                assert torch.equal(out[i, h], v[int(s[h].argmax()), 0])
    assert bool(torch.isfinite(out[:20]).all())
    c = Case("bf16", 1, 2, 64, [300], [20], seed=7)
    for scale in (0.0, -0.25):
        c.check(c.run(scale=scale), scale=scale)


def test_malformed_ranges():
    """Negative starts and counts, more slots than max_tokens, more queries than max_queries: NaN
    for the request's queries; a query range outside the tensor: nothing is written."""
    c = Case("bf16", 1, 4, 64, [50, 60, 70], [4, 5, 6], seed=8)
    dev = lambda x: torch.tensor(x, dtype=torch.int32).cuda()   # noqa: E731

    def call(indptr, q_indptr, max_tokens=70, max_queries=6, slot_count=None):
        out = torch.full_like(c.q, 9.0).cuda()
        return B.paged_attention(c.cache, c.q.cuda(), dev(indptr), c.slots.cuda(), 1, max_tokens,
                                 q_indptr=dev(q_indptr), max_queries=max_queries, out=out,
                                 slot_count=slot_count)

    good = call([0, 50, 110, 180], [0, 4, 9, 15])
    nan = lambda x: bool(torch.isnan(x).all())   # noqa: E731
    out = call([0, 50, 110, 180], [0, 4, 9, 15], max_tokens=60)
    assert torch.equal(out[:9], good[:9]) and nan(out[9:15]) and bool((out[15:] == 9).all())
    out = call([0, 50, 110, 180], [0, 4, 9, 15], max_queries=5)
    assert torch.equal(out[:9], good[:9]) and nan(out[9:15]) and bool((out[15:] == 9).all())
    out = call([0, 50, 40, 110], [0, 4, 9, 15])
    assert torch.equal(out[:4], good[:4]) and nan(out[4:9])
    out = call([-3, 50, 110, 180], [0, 4, 9, 15])
    assert nan(out[:4]) and torch.equal(out[4:15], good[4:15])
    out = call([0, 50, 110, 180], [0, 4, 9, 15], slot_count=dev([50, -1, 70]))
    assert torch.equal(out[:4], good[:4]) and nan(out[4:9]) and torch.equal(out[9:15], good[9:15])
    out = call([0, 50, 110, 180], [-2, 4, 9, 40])
    assert bool((out[:4] == 9).all()) and torch.equal(out[4:9], good[4:9])
    assert bool((out[9:] == 9).all())


def test_strided_and_split_tensors():
    """Queries as views of a projection, outputs at a stride of their own; the same through a slot
    table with room, a caller's workspace and another stream."""
    c = Case("fp8", 2, 4, 64, [400, 90, 1], [30, 90, 1], seed=9)
    n = c.q.shape[0]
    wide = torch.zeros(n, 8 * 64 + 72, dtype=torch.bfloat16, device="cuda")
    wide[:, 8: 8 + 512] = c.q.view(n, -1).cuda()
    out = torch.full((n, 8 * 64 + 16), 9.0, dtype=torch.bfloat16, device="cuda")
    want = c.run(100, 2)
    got = c.run(100, 2, q=wide[:, 8: 520].view(n, 8, 64), out=out[:, 8: 520].view(n, 8, 64))
    assert torch.equal(got, want)
    assert bool((out[:, :8] == 9).all()) and bool((out[:, 520:] == 9).all())
    start = np.array([0, 420, 515, 520])
    table = torch.full((520,), -1, dtype=torch.int32)
    for r in range(3):
        table[start[r]: start[r] + c.counts[r]] = c.slots[c.indptr[r]: c.indptr[r + 1]]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    work = torch.empty(64 << 20, dtype=torch.uint8, device="cuda")
    c.indptr = start
    got = c.run(100, 2, slots=table.cuda(), slot_count=torch.tensor(
        c.counts, dtype=torch.int32).cuda(), workspace=work, stream=side)
    side.synchronize()
    assert torch.equal(got, want)


@pytest.mark.parametrize("queries", [[1, 1, 1], [3, 40, 7]])
def test_captured_and_repeated(queries):
    """A captured call replayed over changed inputs gives what the eager call gives, every time."""
    c = Case("mxfp4", 2, 8, 128, [3000, 700, 64], queries, seed=10)
    q = c.q.cuda()
    slots = c.slots.cuda()
    out = torch.zeros_like(q)
    kw = dict(q=q, slots=slots, out=out, q_indptr=None if max(queries) == 1 else torch.tensor(
        c.q_indptr, dtype=torch.int32).cuda())
    indptr = torch.tensor(c.indptr, dtype=torch.int32).cuda()

    def call():
        return B.paged_attention(c.cache, q, indptr, slots, 1, 3000, q_indptr=kw["q_indptr"],
                                 max_queries=max(queries), window=900, sinks=4, out=out)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        call()
    for i in range(4):
        q.copy_(torch.randn(q.shape, generator=torch.Generator().manual_seed(i)))
        want = call().clone()
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)


def test_two_calls_at_once():
    """Calls on two streams, each with its own outputs and workspace."""
    a = Case("bf16", 8, 4, 128, [4000, 90], [5, 90], seed=11)
    b = Case("mxfp4", 4, 8, 128, [6000], [1], seed=12)
    want = a.run(), b.run(q_indptr=None, max_queries=1)
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    got = []
    for _ in range(4):
        with torch.cuda.stream(streams[0]):
            x = a.run()
        with torch.cuda.stream(streams[1]):
            y = b.run(q_indptr=None, max_queries=1)
        got.append((x, y))
    torch.cuda.synchronize()
    for x, y in got:
        assert torch.equal(x, want[0]) and torch.equal(y, want[1])


def test_far_slots():
    """K and V whose offsets pass 32 bits."""
    H, D, blocks = 8, 256, 70000
    if torch.cuda.mem_get_info()[0] < 24 << 30:
        pytest.skip("needs 10 GB of device memory")
    kv = torch.zeros(2, blocks, 16, H, D, dtype=torch.bfloat16, device="cuda")
    cache = B.KVCache(kv, 1, H, D, 16)
    g = torch.Generator().manual_seed(3)
    n = 40
    slots = (blocks * 16 - 1 - 7 * torch.arange(n)).to(torch.int32)
    k, v = (torch.randn(n, H, D, generator=g).to(torch.bfloat16) for _ in range(2))
    B.write_kv(cache, k.cuda(), v.cuda(), slots.cuda(), 0)
    for ql in (1, 9):
        q = torch.randn(ql, H, D, generator=g).to(torch.bfloat16)
        out = B.paged_attention(
            cache, q.cuda(), torch.tensor([0, n], dtype=torch.int32).cuda(), slots.cuda(), 0, n,
            q_indptr=torch.tensor([0, ql], dtype=torch.int32).cuda(), max_queries=ql)
        ref, size = S.attention(q, k.double(), v.double(), 0, 0, D ** -0.5)
        tol = 1.01 * 2.0 ** -8 * (size + ref.abs()) + (2.0 ** -17 * D + 2.0 ** -18) * size
        assert bool(((out.double().cpu() - ref).abs() <= tol).all())


@pytest.mark.parametrize("kind", ["bf16", "fp8", "mxfp4"])
def test_serving_loop(kind):
    """A prompt in two chunks, then evictions, a repack, the slot table, and new tokens one at a
    time with a window: every step against the definition over the rows that are live."""
    H, G, D, bs, base = 2, 4, 64, 16, 10000.0
    g = torch.Generator().manual_seed(13)
    planes = torch.zeros(2, 40 * bs, S.row_bytes(H, D) if kind == "mxfp4" else
                         H * D * (1 if kind == "fp8" else 2), dtype=torch.uint8)
    cache = S.make_cache(B, planes, kind, H, D, bs)
    table = B.rotary_table(400, D, base)
    w = (1 + 0.1 * torch.randn(D, generator=g)).cuda()
    dev = lambda x: torch.as_tensor(x, dtype=torch.int32).cuda()   # noqa: E731
    blocks = np.random.default_rng(0).permutation(40)
    held, free = blocks[:12], blocks[12:]
    live = []

    def step(slots, first, sees, window=0, sinks=0, slot_count=None, spread=None):
        """Writes len(slots) tokens from position `first`, then attends over the slots `sees`."""
        x = torch.randn(len(slots), (G + 2) * H * D, generator=g).to(torch.bfloat16).cuda()
        q, k, v = (t.view(len(slots), -1, D) for t in x.split([G * H * D, H * D, H * D], 1))
        qo = B.write_kv(cache, k, v, dev(slots), 0, q=q, positions=dev(
            np.arange(first, first + len(slots))), cos_sin=table, q_weight=w, k_weight=w)
        n = len(sees)
        indptr, sl = (dev([0, n]), dev(sees)) if spread is None else spread
        got = B.paged_attention(cache, qo, indptr, sl, 0, n, q_indptr=dev([0, len(slots)]),
                                max_queries=len(slots), window=window, sinks=sinks,
                                slot_count=slot_count)
        rows = S.bytes_of(cache)
        kr, vr = (S.values(rows[i][np.asarray(sees)], kind, H, D) for i in (0, 1))
        ref, size = S.attention(qo.cpu(), kr, vr, window, sinks, D ** -0.5)
        tol = 1.01 * 2.0 ** -8 * (size + ref.abs()) + (2.0 ** -17 * D + 2.0 ** -18) * size
        assert bool(((got.double().cpu() - ref).abs() <= tol).all())

    slot = lambda p: int(held[p // bs]) * bs + p % bs   # noqa: E731
    live = [slot(p) for p in range(180)]
    step(live[:100], 0, live[:100])
    step(live[100:], 100, live, window=64, sinks=4)
    mask = (np.random.default_rng(1).random(180) < 0.3).astype(np.uint8)
    mask[:4] = 1
    batch = B.Batch.from_host([180], [0, 180], [0, 12], held, mask, free)
    plan = B.run_pass(cache, batch)
    start, count, slots = B.build_slot_table(batch, plan, 8)
    n = int(count[0])
    assert int(plan.counters[1]) == 1 and n == int(mask.sum())
    last = int(plan.new_block_ids[int(plan.new_bt_indptr[1]) - 1])
    taken = set(plan.new_block_ids[: int(plan.new_bt_indptr[1])].tolist())
    spare = [int(b) for b in free if int(b) not in taken][0]
    for i in range(5):
        at = n + i
        new = last * bs + at % bs if at % bs and at < -(-n // bs) * bs else spare * bs + at % bs
        B.append_slots(start, count, slots, dev([0, 1]), dev([new]))
        sees = slots[: at + 1].cpu().numpy().tolist()
        step([new], 180 + i, sees, window=20, sinks=4, slot_count=count, spread=(start, slots))
