"""Calls on a stream that is not the current one, with memory that the binding allocates: work that
other streams still have to do on blocks they gave back has no part in the results."""
import pytest
import torch

from paper_2608_13263_amd import binding as B
from paper_2608_13263_amd import workloads as W
import serving_helpers as S
from test_prompt_gpu import Case

pytestmark = pytest.mark.gpu

SPIN = 20_000_000   # cycles that a stream is held up for: some milliseconds


def _late_writes(sizes):
    """Blocks of these many bytes go back to the current stream's memory with a write to come."""
    blocks = [torch.empty(n, dtype=torch.uint8, device="cuda") for n in sizes for _ in range(3)]
    torch.cuda._sleep(SPIN)
    for b in blocks:
        b.fill_(255)   # NaN of every type here


def _held_up(stream):
    with torch.cuda.stream(stream):
        torch.cuda._sleep(SPIN)


def _streams():
    """A stream, and one by its handle."""
    keep = torch.cuda.Stream(), torch.cuda.Stream()
    return [(keep[0], keep[0]), (keep[1], keep[1].cuda_stream)]


@pytest.mark.parametrize("queries", [[1], [9]])
def test_attention(queries):
    c = Case("bf16", 2, 4, 128, [6000], queries, seed=40, extra=0)
    q, slots = c.q.cuda(), c.slots.cuda()
    indptr = torch.tensor(c.indptr, dtype=torch.int32).cuda()
    q_indptr = torch.tensor(c.q_indptr, dtype=torch.int32).cuda()

    def call(stream=None):
        return B.paged_attention(c.cache, q, indptr, slots, 1, 6000, q_indptr=q_indptr,
                                 max_queries=queries[0], stream=stream)

    want = call()
    t = B.CAttention(None, None, 0, 0, q.data_ptr(), None, None, 0, q.shape[0], queries[0], 6000,
                     8, 2, 128, 1, B.KV_BF16, B.KV_BF16, 0, 0, 1.0)
    need = B.attention_workspace_bytes(t, 1)
    assert need > 0
    torch.cuda.synchronize()
    for side, given in _streams():
        for _ in range(2):
            _late_writes([need, want.numel() * 2])
            got = call(given)
            side.synchronize()
            late = got.clone()
            torch.cuda.synchronize()
            assert torch.equal(late, want) and torch.equal(got, want)
            # blocks asked for right after the call are not its workspace
            _held_up(side)
            got = call(given)
            for n in (need, need, got.numel() * 2):
                torch.empty(n, dtype=torch.uint8, device="cuda").fill_(255)
            torch.cuda.synchronize()
            assert torch.equal(got, want)


def test_outputs_that_the_current_stream_still_reads():
    """An output given back while the current stream has still to read it is not the next call's."""
    n = 300
    g = torch.Generator().manual_seed(41)
    planes = torch.stack([S.make_rows("bf16", 512, 2, 64, g) for _ in range(2)])
    cache = S.make_cache(B, planes, "bf16", 2, 64, 16)
    a, b = (torch.randperm(512, generator=g)[:n].to(torch.int32).cuda() for _ in range(2))
    want = [x.clone() for x in B.read_kv(cache, a, 0)]
    torch.cuda.synchronize()
    for side, given in _streams():
        for _ in range(2):
            _late_writes([n * 256])
            k, v = B.read_kv(cache, a, 0, stream=given)
            torch.cuda.current_stream().wait_stream(side)
            torch.cuda._sleep(SPIN)
            got = k.clone(), v.clone()
            del k, v
            B.read_kv(cache, b, 0, stream=given)
            torch.cuda.synchronize()
            assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_written_queries():
    n = 200
    g = torch.Generator().manual_seed(42)
    planes = torch.stack([S.make_rows("bf16", 512, 2, 64, g) for _ in range(2)])
    cache = S.make_cache(B, planes, "bf16", 2, 64, 16)
    x = torch.randn(3, n, 2, 64, generator=g).to(torch.bfloat16).cuda()
    slots = torch.arange(n, dtype=torch.int32).cuda()
    kw = dict(q=x[0], positions=slots, cos_sin=B.rotary_table(n, 64))
    want = B.write_kv(cache, x[1], x[2], slots, 0, **kw)
    torch.cuda.synchronize()
    for side, given in _streams():
        _late_writes([n * 256])
        got = B.write_kv(cache, x[1], x[2], slots, 0, stream=given, **kw)
        torch.cuda.synchronize()
        assert torch.equal(got, want)


def test_a_pass_and_what_reads_it():
    """The plan, the layout check, the slot mapping and table, an append's status and the decode."""
    inp = W.tiny_cache(101)
    sh = inp.shape
    batch = B.Batch.from_inputs(inp)
    kv = W.kv_device(sh, inp.num_blocks, 1)
    q = torch.randn(inp.num_reqs, 4 * sh.num_kv_heads, sh.head_dim, device="cuda")
    none = torch.zeros(inp.num_reqs + 1, dtype=torch.int32, device="cuda")

    def run(stream=None):
        cache = B.KVCache(kv.clone(), sh.num_layers, sh.num_kv_heads, sh.head_dim, sh.block_size)
        torch.cuda.synchronize()
        if stream is not None:
            _late_writes([4, 64, 512, 4096, 1 << 15, 1 << 16, 1 << 20])
        status = B.check_layout(cache, batch, stream=stream)
        plan = B.run_pass(cache, batch, stream=stream)
        indptr, slots = B.build_slot_mapping(batch, plan, stream=stream)
        table = B.build_slot_table(batch, plan, 4, stream=stream)
        full = B.append_slots(*table, none, none, stream=stream)
        out = B.paged_decode(cache, q, indptr, slots, 0, 4096, stream=stream)
        torch.cuda.synchronize()
        n, held = int(indptr[-1]), int(plan.new_bt_indptr[-1])
        assert int(status) == 0 and int(full) == 0 and int(plan.counters[3]) == 0 and n > 0
        rows = [t for r in range(inp.num_reqs) for t in
                table[2][int(table[0][r]): int(table[0][r]) + int(table[1][r])].tolist()]
        return (indptr, slots[:n], table[0], table[1], torch.tensor(rows), out,
                plan.new_block_ids[:held], plan.freed[: int(plan.counters[2])],
                plan.token_slot[: inp.num_tokens], cache.kv.view(torch.uint8))

    want = run()
    for side, given in _streams():
        for a, b in zip(run(given), want):
            assert torch.equal(a, b)


def test_captured_on_another_stream():
    """Calls on a side stream that a capture forks to, their outputs and workspaces made there: every
    replay is the eager result, with eager calls between them."""
    c = Case("bf16", 2, 4, 128, [6000], [1], seed=43, extra=0)
    q, slots = c.q.cuda(), c.slots.cuda()
    indptr = torch.tensor(c.indptr, dtype=torch.int32).cuda()
    side = torch.cuda.Stream()

    def call(stream=None):
        out = B.paged_attention(c.cache, q, indptr, slots, 1, 6000, stream=stream)
        return B.paged_attention(c.cache, out, indptr, slots, 1, 6000, stream=stream), out

    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        side.wait_stream(torch.cuda.current_stream())
        got = call(side)
        torch.cuda.current_stream().wait_stream(side)
    for i in range(4):
        q.copy_(torch.randn(q.shape, generator=torch.Generator().manual_seed(i)))
        want = call()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
        call(side)
        torch.cuda.synchronize()
