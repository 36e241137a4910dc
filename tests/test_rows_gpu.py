"""write_kv and read_kv against their definitions.

Tolerances. A 16-bit or 8-bit result is off by the rounding to its type, half a step of the result
(relative HALF_STEP, or half of the smallest step), and by the float32 steps before it: five
roundings of 2^-24 each on products that are at most |a| + |b| of the turned pair, taken as 2^-21 of
the largest value of the head row. 4-bit rows and copies are compared bit for bit: the operator's
roundings are part of its definition."""
import numpy as np
import pytest
import torch

from paper_2608_13263_amd import binding as B
from paper_2608_13263_amd import workloads as W
import serving_helpers as S

pytestmark = pytest.mark.gpu


def _near(got, ref, kind, size):
    tol = S.HALF_STEP[kind] * ref.abs() * (1 + 2.0 ** -12) + S.HALF_TINY[kind] + 2.0 ** -21 * size
    assert bool(((got.double().cpu() - ref).abs() <= tol).all()), float(
        ((got.double().cpu() - ref).abs() - tol).max())


def _inputs(kind, act, n, Hq, H, D, g, pad=8):
    """Views of a wider projection: the tokens' stride is more than their heads."""
    x = torch.randn(n, (Hq + 2 * H) * D + pad, generator=g).to(S.TYPES[act]).cuda()
    q = x[:, : Hq * D].view(n, Hq, D) if n else x[:, : Hq * D].reshape(0, Hq, D)
    k = x[:, Hq * D: (Hq + H) * D].view(n, H, D)
    v = x[:, (Hq + H) * D: (Hq + 2 * H) * D].view(n, H, D)
    return q, k, v


@pytest.mark.parametrize("kind,act,Hq,H,D,n,rot,interleaved,norm", [
    ("bf16", "bf16", 32, 8, 128, 37, 128, False, True),
    ("bf16", "bf16", 5, 1, 256, 3, 128, True, True),
    ("bf16", "bf16", 4, 4, 32, 65, 32, False, False),
    ("fp16", "fp16", 8, 2, 64, 129, 16, False, True),
    ("fp16", "fp16", 3, 3, 96, 17, 96, True, False),
    ("fp16", "fp16", 2, 1, 8, 5, 8, True, True),
    ("fp16", "fp16", 2, 2, 40, 9, 32, False, True),
    ("fp8", "bf16", 8, 4, 128, 33, 64, False, True),
    ("fp8", "fp16", 8, 2, 64, 1, 32, True, False),
    ("mxfp4", "bf16", 8, 1, 128, 50, 128, False, True),
    ("mxfp4", "bf16", 6, 3, 32, 21, 16, False, True),
    ("mxfp4", "bf16", 5, 5, 96, 11, 48, False, True),
    ("mxfp4", "bf16", 0, 2, 256, 7, 256, True, True),
    ("mxfp4", "bf16", 64, 8, 64, 300, 64, False, False),
])
def test_write(kind, act, Hq, H, D, n, rot, interleaved, norm):
    """Both rotations, odd heads, the second of two layers, padding in the middle, positions far
    out; every byte outside the written rows stays."""
    print(f"[gpu] write {kind} {act} Hq={Hq} H={H} D={D} n={n}", flush=True)
    g = torch.Generator().manual_seed(D + n)
    before = torch.stack([S.make_rows(kind, 384, H, D, g) for _ in range(4)])
    cache = S.make_cache(B, before, kind, H, D, 16)
    q, k, v = _inputs(kind, act, n, Hq, H, D, g)
    if not norm:
        v[0, 0, :2] = torch.tensor([500.0, -1e4])   # past fp8's largest value
    slots = torch.randperm(384, generator=g)[:n].to(torch.int32)
    if n > 2:
        slots[n // 2] = -1
    pos = torch.randint(0, 1500, (n,), generator=g, dtype=torch.int32)
    table = B.rotary_table(1500, rot, 500000.0)
    qw, kw = ((1 + 0.3 * torch.randn(2, D, generator=g)) if norm else (None, None))
    dev = lambda x: None if x is None else x.cuda()   # noqa: E731
    out = torch.full((n, Hq, D), 7.0, dtype=S.TYPES[act], device="cuda") if Hq else None
    B.write_kv(cache, k, v, slots.cuda(), 1, q=q if Hq else None, positions=pos.cuda(),
               cos_sin=table, q_weight=dev(qw), k_weight=dev(kw), eps=1e-5,
               interleaved=interleaved, q_out=out)
    torch.cuda.synchronize()
    after = S.bytes_of(cache)
    keep = slots >= 0
    at = slots[keep].long()
    expected = before.clone()
    cs = table.cpu()

    def chain(x, w, t):
        return S.turned(S.normed(x.cpu().float(), w, 1e-5).to(t), cs, pos, interleaved)

    for plane, x in ((2, chain(k, kw, torch.float32)), (3, v.cpu().float())):
        if kind == "mxfp4":
            expected[plane][at, : after.shape[2]] = torch.where(
                torch.arange(after.shape[2]) < H * D // 2 + H * D // 32, S.pack4(x)[keep],
                before[plane][at])
        else:
            wide = chain(k, kw, torch.float64) if plane == 2 else x.double()
            if kind == "fp8":
                wide = wide.clamp(-448, 448)
            size = wide.abs().amax(-1, keepdim=True)
            _near(S.values(after[plane][at], kind, H, D), wide[keep], kind, size[keep])
            expected[plane][at] = after[plane][at]
    assert torch.equal(after, expected)
    if Hq:
        wide = chain(q, qw, torch.float64)
        _near(out[keep.cuda()], wide[keep], act, wide.abs().amax(-1, keepdim=True)[keep])
        assert bool((out[~keep.cuda()] == 7).all())


def test_write_16_bit_values_are_copied():
    """v goes into a 16-bit cache as it is: infinities, NaN payload bits, the smallest values."""
    x = torch.arange(0, 65536, dtype=torch.int32).to(torch.int16).view(torch.bfloat16)
    v = x.view(512, 1, 128).cuda()
    cache = S.make_cache(B, torch.zeros(2, 512, 256, dtype=torch.uint8), "bf16", 1, 128, 16)
    B.write_kv(cache, v, v, torch.arange(512, dtype=torch.int32).cuda(), 0)
    got = cache.kv[1].reshape(512, 1, 128).cpu()
    nan = torch.isnan(v.cpu())
    assert torch.equal(torch.isnan(got), nan)
    assert torch.equal(got.view(torch.int16)[~nan], v.cpu().view(torch.int16)[~nan])


@pytest.mark.parametrize("kind", ["fp8", "mxfp4"])
def test_write_every_rounding(kind):
    """All bf16 values, 32 neighbours to an exponent: ties, saturation, zeros of both signs, the
    smallest exponents, infinities and NaN."""
    x = torch.arange(0, 65536, dtype=torch.int32).to(torch.int16).view(torch.bfloat16)
    v = x.view(512, 1, 128)
    row = 128 if kind == "fp8" else S.row_bytes(1, 128)
    cache = S.make_cache(B, torch.zeros(2, 512, row, dtype=torch.uint8), kind, 1, 128, 16)
    B.write_kv(cache, v.cuda(), v.cuda(), torch.arange(512, dtype=torch.int32).cuda(), 0)
    got = S.bytes_of(cache)
    if kind == "fp8":
        f = v.float()
        # torch's cast of what is clamped; NaN stays
        ref = torch.where(f.isnan(), f, f.clamp(-448, 448)).to(torch.float8_e4m3fn)
        a, b = got[1].reshape(512, 128), ref.view(torch.uint8).reshape(512, 128)
        nan = f.isnan().reshape(512, 128)
        assert torch.equal(a[~nan], b[~nan]) and bool((a[nan] & 127 == 127).all())
    else:
        assert torch.equal(got[1], S.pack4(v.float()))
    assert torch.equal(got[0], got[1])
    # ties of the 4-bit grid in a group of their own, with either neighbour
    if kind == "mxfp4":
        t = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0, 7.5, 4.0, 0.2490234375])
        u = torch.zeros(1, 1, 128)
        u[0, 0, :11], u[0, 0, 32:43], u[0, 0, 64] = t, -t * 2.0 ** -20, 2.0 ** -130
        u = u.to(torch.bfloat16)
        B.write_kv(cache, u.cuda(), u.cuda(), torch.zeros(1, dtype=torch.int32).cuda(), 0)
        assert torch.equal(S.bytes_of(cache)[0][:1], S.pack4(u.float()))


def test_write_bad_tokens():
    """A slot past the pool or a position without angles: NaN queries, nothing in the cache."""
    g = torch.Generator().manual_seed(0)
    before = torch.stack([S.make_rows("bf16", 32, 2, 64, g) for _ in range(2)])
    cache = S.make_cache(B, before, "bf16", 2, 64, 16)
    q, k, v = _inputs("bf16", "bf16", 6, 4, 2, 64, g)
    slots = torch.tensor([3, 32, 5, 2 ** 31 - 1, 7, -9], dtype=torch.int32).cuda()
    pos = torch.tensor([0, 1, 10, 2, -1, 3], dtype=torch.int32).cuda()
    out = torch.full_like(q.contiguous(), 7.0)
    B.write_kv(cache, k, v, slots, 0, q=q, positions=pos, cos_sin=B.rotary_table(10, 64), q_out=out)
    after = S.bytes_of(cache)
    assert not torch.equal(after[:, 3], before[:, 3])
    after[:, 3] = before[:, 3]
    assert torch.equal(after, before)
    nan = torch.isnan(out).all(-1).all(-1).cpu()
    assert nan.tolist() == [False, True, True, True, True, False]
    assert bool((out[5] == 7).all()) and not bool(torch.isnan(out[0]).any())


def test_write_in_place_and_captured():
    """q_out = q; the call in a graph, replayed with new inputs, on a stream of its own."""
    g = torch.Generator().manual_seed(5)
    before = torch.stack([S.make_rows("mxfp4", 64, 8, 128, g) for _ in range(2)])
    cache, eager = (S.make_cache(B, before, "mxfp4", 8, 128, 16) for _ in range(2))
    x = torch.randn(20, 48 * 128, generator=g).to(torch.bfloat16).cuda()
    q, k, v = (t.view(20, -1, 128) for t in x.split([32 * 128, 8 * 128, 8 * 128], 1))
    slots = torch.arange(20, dtype=torch.int32).cuda()
    pos = torch.arange(20, dtype=torch.int32).cuda()
    table, w = B.rotary_table(64, 128), torch.rand(128, generator=g).cuda()
    kw = dict(positions=pos, cos_sin=table, q_weight=w, k_weight=w)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        B.write_kv(cache, k, v, slots, 0, q=q, q_out=q, **kw)
    for i in range(3):
        x.copy_(torch.randn(20, 48 * 128, generator=g).to(torch.bfloat16))
        slots += 3 * i
        want = B.write_kv(eager, k, v, slots, 0, q=q, **kw)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(want, q) and torch.equal(S.bytes_of(cache), S.bytes_of(eager))


@pytest.mark.parametrize("kind,H,D", [("bf16", 8, 128), ("fp16", 1, 8), ("fp16", 3, 96),
                                      ("fp8", 2, 256), ("fp8", 8, 64), ("mxfp4", 1, 32),
                                      ("mxfp4", 8, 128), ("mxfp4", 5, 96), ("mxfp4", 3, 256)])
def test_read(kind, H, D):
    """Exact values, bit for bit, of every code of the type; slots that repeat and that are outside;
    strided outputs."""
    g = torch.Generator().manual_seed(D)
    row = S.row_bytes(H, D) if kind == "mxfp4" else H * D * (1 if kind == "fp8" else 2)
    planes = torch.randint(0, 256, (4, 96, row), generator=g, dtype=torch.uint8)
    if kind == "mxfp4":   # exponents that bf16 holds
        a = H * D // 2
        planes[..., a:] = torch.randint(60, 200, planes[..., a:].shape, generator=g,
                                        dtype=torch.uint8)
        planes[0, 3, a] = 255
    cache = S.make_cache(B, planes, kind, H, D, 16)
    slots = torch.tensor([0, 95, 3, 3, -1, 96, 41], dtype=torch.int32)
    dtype = torch.float16 if kind == "fp16" else torch.bfloat16
    wide = torch.zeros(7, H * D + 8, dtype=dtype, device="cuda")
    for layer in (0, 1):
        k, v = B.read_kv(cache, slots.cuda(), layer, v_out=wide[:, : H * D].view(7, H, D))
        for got, plane in ((k, planes[2 * layer]), (v, planes[2 * layer + 1])):
            ref = S.values(plane[slots.clamp(0, 95).long()], kind, H, D)
            ref[4], ref[5] = np.nan, np.nan
            assert torch.allclose(got.double().cpu(), ref, rtol=0, atol=0, equal_nan=True)
    assert bool((wide[:, H * D:] == 0).all())
    if kind == "fp8":
        k16, _ = B.read_kv(cache, slots.cuda(), 0, dtype=torch.float16)
        k, _ = B.read_kv(cache, slots.cuda(), 0)
        assert torch.allclose(k16.double(), k.double(), rtol=0, atol=0, equal_nan=True)


def test_rows_of_nothing():
    cache = S.make_cache(B, torch.zeros(2, 16, 256, dtype=torch.uint8), "bf16", 1, 128, 16)
    none = torch.empty(0, dtype=torch.int32, device="cuda")
    x = torch.empty(0, 1, 128, dtype=torch.bfloat16, device="cuda")
    assert B.write_kv(cache, x, x, none, 0, q=x).shape == (0, 1, 128)
    assert B.read_kv(cache, none, 0)[0].shape == (0, 1, 128)


def test_far_slots():
    """Rows whose offset passes 32 bits: the last slots of a plane of more than 2^32 bytes."""
    H, D, blocks = 8, 256, 70000
    if torch.cuda.mem_get_info()[0] < 24 << 30:
        pytest.skip("needs 10 GB of device memory")
    kv = torch.zeros(2, blocks, 16, H, D, dtype=torch.bfloat16, device="cuda")
    cache = B.KVCache(kv, 1, H, D, 16)
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn(3, H, D, device="cuda", generator=g).to(torch.bfloat16)
    slots = torch.tensor([blocks * 16 - 1, blocks * 16 - 40, 2], dtype=torch.int32, device="cuda")
    B.write_kv(cache, x, -x, slots, 0)
    k, v = B.read_kv(cache, slots, 0)
    assert torch.equal(k, x) and torch.equal(v, -x)
    assert torch.equal(kv[0, -1, -1], x[0]) and int((kv != 0).any(-1).any(-1).sum()) == 6


def test_packed_cache_through_a_pass():
    """A 4-bit cache through the repack: the live rows move whole, attention's slots find them."""
    inp = W.from_masks([[1, 0, 0, 1] * 20, [0] * 30 + [1] * 5, [1] * 33],
                       W.KVShape(1, 2, 64, 16, "fp16"), free_blocks=12, seed=3, name="packed")
    H, D = 8, 128
    g = torch.Generator().manual_seed(2)
    planes = torch.stack([S.make_rows("mxfp4", inp.num_blocks * 16, H, D, g) for _ in range(4)])
    cache = S.make_cache(B, planes, "mxfp4", H, D, 16)
    batch = B.Batch.from_inputs(inp)
    before = []
    for r in range(inp.num_reqs):
        a = int(inp.tok_indptr[r])
        table = inp.block_ids[inp.bt_indptr[r]: inp.bt_indptr[r + 1]]
        before += [int(table[p // 16]) * 16 + p % 16 for p in range(int(inp.seq_lens[r]))
                   if inp.live[a + p]]
    old = [B.read_kv(cache, torch.tensor(before, dtype=torch.int32).cuda(), x) for x in (0, 1)]
    plan = B.run_pass(cache, batch)
    indptr, slots = B.build_slot_mapping(batch, plan)
    n = int(indptr[-1])
    assert int(plan.counters[3]) == 0 and n == len(before) and int(plan.counters[1]) > 0
    for layer in (0, 1):
        new = B.read_kv(cache, slots[:n].contiguous(), layer)
        assert torch.equal(new[0], old[layer][0]) and torch.equal(new[1], old[layer][1])
