"""The serving operators around the paged cache, as calls that are timed and compared with their
plain forms.

Three kinds of call, all through paper_2608_13263_amd.binding:

  write   write_kv: per-head RMS norm of queries and keys, rotary positions, the rows stored at
          their slots of the cache (4-bit caches: the rows are read back with read_kv, since their
          outputs are the values they stand for)
  read    read_kv: the rows of listed slots as dense 16-bit tensors
  attend  paged_attention: a ragged batch of queries over the cache, causal, with a sliding window
          and first tokens that stay visible; one query per request where `queries` is 0

Geometries are those of workloads.py and bench.py (tiny cache, Llama-3-8B, Llama-3-70B and one
GPU's share of it under 8-way tensor parallelism). Everything is made from the seed on the device.

The plain forms compute in 32 bits (the norm's mean and root in 64, since its result decides
roundings to 8 and 4 bits) and round once at the end.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

_DTYPE = {"fp16": torch.float16, "bf16": torch.bfloat16, "fp8": torch.float8_e4m3fn}
_E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _case(name, kind, kv, act, heads, group, dim, block, **kw):
    """A case: cache type, activation type, KV heads, query heads per KV head, head_dim, block."""
    c = {"kind": kind, "kv": kv, "act": act, "heads": heads, "group": group, "dim": dim,
         "block": block}
    if name is not None:
        c["name"] = name
    c.update(kw)
    return c


def _write(name, kv, act, heads, group, dim, block, tokens, rotary, norm, interleaved, first, pad):
    """`tokens` tokens from position `first` on; the last `pad` of them are padding (slot -1)."""
    return _case(name, "write", kv, act, heads, group, dim, block, tokens=tokens, rotary=rotary,
                 norm=norm, interleaved=interleaved, first=first, pad=pad)


def _read(name, kv, act, heads, dim, block, tokens):
    return _case(name, "read", kv, act, heads, 1, dim, block, tokens=tokens)


def _attend(name, kv, act, heads, group, dim, block, reqs, lo, hi, queries, window, sinks):
    """`reqs` requests of U[lo, hi] live tokens, of which the last U[1, queries] are queries
    (exactly `queries` in a batch of one; 0: one query per request, the decode step's call)."""
    return _case(name, "attend", kv, act, heads, group, dim, block, reqs=reqs, lo=lo, hi=hi,
                 queries=queries, window=window, sinks=sinks)


def listed():
    return [
        # One new token of one request: launch and latency.
        _write("write_one", "bf16", "bf16", 8, 4, 128, 16, 1, 128, True, False, 4096, 0),
        # A prompt of Llama-3-8B's geometry goes into the cache.
        _write("write_8b", "bf16", "bf16", 8, 4, 128, 16, 8192, 128, True, False, 0, 0),
        # Partial, interleaved rotation without norms into an fp8 cache; a padded batch.
        _write("write_fp8", "fp8", "fp16", 2, 4, 64, 16, 3001, 32, False, True, 100000, 17),
        # A prompt of Llama-3-70B's geometry into a 4-bit cache, and its values back.
        _write("write_4bit", "mxfp4", "bf16", 8, 8, 128, 32, 4097, 128, True, False, 20000, 0),
        # A few hundred tokens of an fp8 cache looked at.
        _read("read_fp8", "fp8", "bf16", 8, 128, 32, 500),
        # A long request's 4-bit rows exported.
        _read("read_4bit", "mxfp4", "bf16", 8, 128, 32, 65536),
        # The smallest decode step: a tiny cache, a short window.
        _attend("decode_tiny", "fp16", "fp16", 2, 4, 64, 16, 8, 50, 250, 0, 64, 4),
        # A decode step of Llama-3-8B over long requests, a window of 2,048 and four sinks.
        _attend("decode_window", "bf16", "bf16", 8, 4, 128, 16, 64, 4096, 8192, 0, 2048, 4),
        # A decode step of Llama-3-70B over long requests, every token visible, 4 bits.
        _attend("decode_4bit", "mxfp4", "bf16", 8, 8, 128, 32, 29, 5043, 19788, 0, 0, 0),
        # A whole prompt with a window of 4,096 and four sinks.
        _attend("prompt_8b", "bf16", "bf16", 8, 4, 128, 16, 1, 8192, 8192, 8192, 4096, 4),
        # Prompts, chunks and single tokens in one batch over an fp8 cache.
        _attend("prompt_ragged", "fp8", "bf16", 8, 8, 128, 32, 12, 600, 3000, 600, 0, 0),
        # A short chunk at the end of two long requests, one GPU's share at TP = 8, 4 bits.
        _attend("chunk_4bit", "mxfp4", "bf16", 1, 8, 128, 32, 2, 30000, 60000, 61, 0, 0),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the same ranges, at most as costly as the largest listed one."""
    kind = rng.choice(["write", "write", "read", "decode", "decode", "prompt", "prompt"])
    kv = rng.choice(["bf16", "fp16", "fp8", "mxfp4", "mxfp4"])
    act = {"bf16": "bf16", "fp16": "fp16", "fp8": rng.choice(["bf16", "fp16"]), "mxfp4": "bf16"}[kv]
    block = rng.choice([8, 16, 16, 24, 32, 48])
    heads = rng.choice([1, 2, 3, 4, 5, 8, 8])
    if kind in ("write", "read"):
        dim = rng.choice([32, 64, 96, 128, 128, 256])
        group = rng.choice([1, 2, 4, 5, 7, 8])
        most = (8192 * 48 * 128) // (heads * (group + 2) * dim)
        tokens = min(_log_int(rng, 1, 20000), most)
        if kind == "read":
            return _read(None, kv, act, heads, dim, block, min(3 * tokens, 60000))
        rotary = rng.choice([dim, dim, dim // 2])
        return _write(None, kv, act, heads, group, dim, block, tokens, rotary, rng.random() < 0.7,
                      rng.random() < 0.3, _log_int(rng, 1, 120000), rng.choice([0, tokens // 9]))
    dim = rng.choice([32, 64, 128, 128, 256])
    group = rng.choice([1, 2, 4, 5, 7, 8, 16])
    window = rng.choice([0, 0, _log_int(rng, 1, 5000)])
    sinks = rng.choice([0, 1, 4, 16, 100])
    reqs = _log_int(rng, 1, 64)
    if kind == "decode":
        most = (256 << 20) // (heads * dim * reqs)
        hi = max(1, min(_log_int(rng, 1, 40000), most))
        return _attend(None, kv, act, heads, group, dim, block, reqs, max(1, hi // 3), hi, 0,
                       window, sinks)
    # the padded scores of the plain form stay within those of the listed prompts
    queries = _log_int(rng, 1, 6000)
    most = 1800000000 // (heads * group * max(dim, 128) // 128)
    queries = max(1, min(queries, int(math.sqrt(most / reqs))))
    hi = max(queries, min(_log_int(rng, 1, 40000), most // (reqs * queries),
                          (128 << 20) // (heads * dim * reqs)))
    return _attend(None, kv, act, heads, group, dim, block, reqs, max(1, hi // 4), hi, queries,
                   window, sinks)


# ------------------------------------------------------------------------------------------
# 4-bit rows: [heads][dim/2] codes (even value in the low half of its byte), then one e8m0
# exponent per 32 values, padded to 16 bytes.
# ------------------------------------------------------------------------------------------
def _row_bytes(heads, dim):
    return -(-heads * (dim // 2 + dim // 32) // 16) * 16


def _pack(x):
    """float32 [..., heads, dim] -> uint8 [..., row bytes]."""
    heads, dim = x.shape[-2:]
    g = x.reshape(*x.shape[:-1], dim // 32, 32)
    field = g.abs().amax(-1, keepdim=True).view(torch.int32) >> 23
    e = torch.where(field == 255, 255, (field - 2).clamp_min(1))
    inverse = torch.where(e == 255, 0, (254 - e) << 23).to(torch.int32).view(torch.float32)
    t = torch.where(e == 255, 0.0, g.abs() * inverse)
    code = ((t > 0.25).to(torch.uint8) + (t >= 0.75) + (t > 1.25) + (t >= 1.75) + (t > 2.5)
            + (t >= 3.5) + (t > 5.0))
    code = torch.where((e != 255) & torch.signbit(g), code + 8, code).to(torch.uint8)
    code = code.reshape(*x.shape[:-2], heads * dim // 2, 2)
    row = torch.cat([code[..., 0] | (code[..., 1] << 4),
                     e.to(torch.uint8).reshape(*x.shape[:-2], heads * dim // 32)], -1)
    return torch.nn.functional.pad(row, (0, _row_bytes(heads, dim) - row.shape[-1]))


def _unpack(rows, heads, dim):
    """uint8 [..., row bytes] -> float32 [..., heads, dim]."""
    nib = rows[..., : heads * dim // 2]
    code = torch.stack([nib & 15, nib >> 4], -1).reshape(*rows.shape[:-1], heads, dim // 32, 32)
    e = rows[..., heads * dim // 2: heads * dim // 2 + heads * dim // 32].to(torch.int32)
    scale = torch.where(e == 255, math.nan, (e << 23).view(torch.float32))
    table = torch.tensor(_E2M1 + tuple(-v for v in _E2M1), device=rows.device)
    x = table[code.to(torch.int32)] * scale.reshape(*rows.shape[:-1], heads, dim // 32, 1)
    return x.reshape(*rows.shape[:-1], heads, dim)


# ------------------------------------------------------------------------------------------
# inputs
# ------------------------------------------------------------------------------------------
def _tokens(c):
    """Live tokens and queries of every request of an attend case (the case's own, so that the
    shapes of its outputs are)."""
    r = np.random.default_rng([c["reqs"], c["lo"], c["hi"], c["queries"]])
    n = r.integers(c["lo"], c["hi"] + 1, size=c["reqs"])
    if c["queries"] == 0:
        return n, np.ones_like(n)
    if c["reqs"] == 1:
        return n, np.minimum(c["queries"], n)
    return n, np.minimum(r.integers(1, c["queries"] + 1, size=c["reqs"]), n)


def _pool(c, tokens, g):
    """A pool of one layer with room for `tokens` tokens (and some blocks more), filled with
    normal values: [2][blocks][block][heads][dim], 4-bit caches [2][blocks][block][row bytes]."""
    blocks = -(-tokens // c["block"]) * 9 // 8 + 1
    shape = (blocks, c["block"], c["heads"], c["dim"])
    planes = [torch.randn(shape, device="cuda", generator=g) for _ in range(2)]
    if c["kv"] == "mxfp4":
        return torch.stack([_pack(p) for p in planes])
    return torch.stack([p.to(_DTYPE[c["kv"]]).view(torch.uint8) for p in planes]).view(
        _DTYPE[c["kv"]])


def _slots(c, pool, sizes, g):
    """Slots of the requests' tokens, one after the other: blocks in random order, each request's
    tokens filling its own blocks from the front."""
    S = c["block"]
    perm = torch.randperm(pool.shape[1], device="cuda", generator=g)
    sizes = torch.as_tensor(np.asarray(sizes), device="cuda")
    need = (sizes + S - 1) // S
    start = torch.repeat_interleave(torch.cumsum(sizes, 0) - sizes, sizes)
    first = torch.repeat_interleave(torch.cumsum(need, 0) - need, sizes)
    i = torch.arange(int(sizes.sum()), device="cuda") - start
    return (perm[first + i // S] * S + i % S).to(torch.int32)


def prepare(case, seed):
    c = dict(case)
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    act = _DTYPE[c["act"]]
    H, G, D = c["heads"], c["group"], c["dim"]
    s = {"case": c}
    if c["kind"] == "write":
        n = c["tokens"]
        s["pool"] = _pool(c, n, g)
        s["slots"] = _slots(c, s["pool"], [n], g)
        if c["pad"]:
            s["slots"][n - c["pad"]:] = -1
        # the rows of a fused projection: queries, keys and values of a token side by side
        x = torch.randn(n, (G + 2) * H * D, device="cuda", generator=g).to(act)
        s["q"] = x[:, : G * H * D].view(n, G * H, D)
        s["k"] = x[:, G * H * D: (G + 1) * H * D].view(n, H, D)
        s["v"] = x[:, (G + 1) * H * D:].view(n, H, D)
        s["q_out"] = torch.zeros(n, G * H, D, device="cuda", dtype=act)
        s["positions"] = torch.arange(c["first"], c["first"] + n, device="cuda", dtype=torch.int32)
        half = c["rotary"] // 2
        angle = (torch.arange(c["first"] + n, device="cuda", dtype=torch.float64)[:, None]
                 * 500000.0 ** (-torch.arange(half, device="cuda", dtype=torch.float64) / half))
        s["cos_sin"] = torch.cat([angle.cos(), angle.sin()], 1).float()
        for w in ("q_weight", "k_weight"):
            s[w] = (1 + 0.2 * torch.randn(D, device="cuda", generator=g)) if c["norm"] else None
        return s
    if c["kind"] == "read":
        s["pool"] = _pool(c, c["tokens"], g)
        s["slots"] = _slots(c, s["pool"], [c["tokens"]], g)
        return s
    n, ql = _tokens(c)
    s["pool"] = _pool(c, int((-(-n // c["block"]) * c["block"]).sum()), g)
    s["slots"] = _slots(c, s["pool"], n, g)
    s["slot_indptr"] = torch.tensor(np.concatenate([[0], np.cumsum(n)]), dtype=torch.int32).cuda()
    s["q_indptr"] = torch.tensor(np.concatenate([[0], np.cumsum(ql)]), dtype=torch.int32).cuda()
    s["max_tokens"], s["max_queries"] = int(n.max()), int(ql.max())
    s["q"] = (1.5 * torch.randn(int(ql.sum()), H * G, D, device="cuda", generator=g)).to(act)
    return s


# ------------------------------------------------------------------------------------------
# one pass
# ------------------------------------------------------------------------------------------
def _rotate(y, cs, interleaved):
    """Rotary positions over the first `rotary` values of each head; cs [n, rotary]."""
    rot = cs.shape[-1]
    c, s = cs[:, None, : rot // 2], cs[:, None, rot // 2:]
    if interleaved:
        a, b = y[..., 0:rot:2], y[..., 1:rot:2]
        r = torch.stack([a * c - b * s, b * c + a * s], -1).flatten(-2)
    else:
        a, b = y[..., : rot // 2], y[..., rot // 2: rot]
        r = torch.cat([a * c - b * s, b * c + a * s], -1)
    return torch.cat([r, y[..., rot:]], -1)


def _norm(x, weight, eps):
    if weight is None:
        return x
    mean = x.double().square().mean(-1, keepdim=True)
    return x * (1.0 / (mean + eps).sqrt()).float() * weight


def _store(plane, slots, x, kv):
    """Rows of x into a plane at slots (all of them valid)."""
    flat = plane.view(-1, *plane.shape[2:])
    if kv == "mxfp4":
        flat[slots] = _pack(x)
    elif kv == "fp8":
        x = x.clamp(-448.0, 448.0).to(plane.dtype)
        flat.view(torch.uint8)[slots] = x.view(torch.uint8)
    else:
        flat[slots] = x.to(plane.dtype)


def _load(plane, slots, c):
    """float32 rows of a plane at slots."""
    flat = plane.view(-1, *plane.shape[2:])
    if c["kv"] == "mxfp4":
        return _unpack(flat[slots], c["heads"], c["dim"])
    if c["kv"] == "fp8":
        return flat.view(torch.uint8)[slots].view(plane.dtype).float()
    return flat[slots].float()


def _plain_write(s):
    c = s["case"]
    cs = s["cos_sin"][s["positions"]]
    q = _rotate(_norm(s["q"].float(), s["q_weight"], 1e-6), cs, c["interleaved"])
    k = _rotate(_norm(s["k"].float(), s["k_weight"], 1e-6), cs, c["interleaved"])
    real = c["tokens"] - c["pad"]   # rows past them are left as they were
    s["q_out"][:real] = q[:real].to(s["q_out"].dtype)
    slots = s["slots"][:real].long()
    _store(s["pool"][0], slots, k[:real], c["kv"])
    _store(s["pool"][1], slots, s["v"][:real].float(), c["kv"])
    if c["kv"] != "mxfp4":
        return {"q": s["q_out"], "pool": s["pool"]}
    return {"q": s["q_out"], **_plain_read(s)}


def _plain_read(s):
    c = s["case"]
    slots = s["slots"].long()
    bad = (slots < 0)[:, None, None]
    k, v = (torch.where(bad, math.nan, _load(s["pool"][i], slots.clamp_min(0), c)).to(
        _DTYPE[c["act"]]) for i in (0, 1))
    return {"k": k, "v": v}


def _plain_attend(s):
    c = s["case"]
    H, G, D = c["heads"], c["group"], c["dim"]
    start, qstart = s["slot_indptr"].long(), s["q_indptr"].long()
    n, ql = start.diff()[:, None], qstart.diff()[:, None]
    R, nm, qm = c["reqs"], s["max_tokens"], s["max_queries"]
    t = torch.arange(nm, device="cuda")[None]
    i = torch.arange(qm, device="cuda")[None]
    slots = s["slots"][(start[:-1, None] + t).clamp_max(s["slots"].numel() - 1)].long()
    k = _load(s["pool"][0], slots, c).permute(0, 2, 3, 1).contiguous()   # [R, H, D, nm]
    v = _load(s["pool"][1], slots, c).permute(0, 2, 1, 3).contiguous()   # [R, H, nm, D]
    row = (qstart[:-1, None] + i).clamp_max(s["q"].shape[0] - 1)
    q = s["q"][row].float().view(R, qm, H, G, D).permute(0, 2, 3, 1, 4).reshape(R, H, G * qm, D)
    x = (q @ k).mul_(D ** -0.5).view(R, H, G, qm, nm)
    p = (n - ql + i)[:, :, None]                                          # ranks [R, qm, 1]
    key = t[:, None, :]
    seen = (key <= p) & (key < n[:, :, None])
    if c["window"]:
        seen &= (key < c["sinks"]) | (key > p - c["window"])
    x.masked_fill_(~seen[:, None, None], -math.inf)
    m = x.amax(-1, keepdim=True).clamp_min(-3e38)
    x.sub_(m).exp_()
    total = x.sum(-1, keepdim=True)
    o = (x.view(R, H, G * qm, nm) @ v).view(R, H, G, qm, D)
    o = torch.where(total > 0, o / total, 0.0).permute(0, 3, 1, 2, 4).reshape(R, qm, H * G, D)
    return o[i.expand(R, qm) < ql].to(s["q"].dtype)


def _own(s):
    from paper_2608_13263_amd import binding as B
    c = s["case"]
    if "cache" not in s:   # what a program keeps for as long as its pool
        make = B.PackedKVCache if c["kv"] == "mxfp4" else B.KVCache
        s["cache"] = make(s["pool"], 1, c["heads"], c["dim"], c["block"])
    cache, act = s["cache"], _DTYPE[c["act"]]
    if c["kind"] == "attend":
        return B.paged_attention(
            cache, s["q"], s["slot_indptr"], s["slots"], 0, s["max_tokens"],
            q_indptr=s["q_indptr"] if c["queries"] else None, max_queries=s["max_queries"],
            window=c["window"], sinks=c["sinks"])
    if c["kind"] == "write":
        B.write_kv(cache, s["k"], s["v"], s["slots"], 0, q=s["q"], q_out=s["q_out"],
                   positions=s["positions"], cos_sin=s["cos_sin"], q_weight=s["q_weight"],
                   k_weight=s["k_weight"], eps=1e-6, interleaved=c["interleaved"])
        if c["kv"] != "mxfp4":
            return {"q": s["q_out"], "pool": s["pool"]}
    k, v = B.read_kv(cache, s["slots"], 0, dtype=act)
    return {"k": k, "v": v} if c["kind"] == "read" else {"q": s["q_out"], "k": k, "v": v}


def run(state):
    if own:
        return _own(state)
    return {"write": _plain_write, "read": _plain_read, "attend": _plain_attend}[
        state["case"]["kind"]](state)


# ------------------------------------------------------------------------------------------
# work and the definition in 64 bits
# ------------------------------------------------------------------------------------------
def _row(c):
    if c["kv"] == "mxfp4":
        return c["heads"] * (c["dim"] // 2 + c["dim"] // 32)
    return c["heads"] * c["dim"] * (1 if c["kv"] == "fp8" else 2)


def work(case):
    c = case
    H, G, D = c["heads"], c["group"], c["dim"]
    if c["kind"] == "write":
        n = c["tokens"] - c["pad"]
        b = n * ((G + 2) * H * D * 2 + 4 * c["rotary"] + 8 + G * H * D * 2 + 2 * _row(c))
        if c["kv"] == "mxfp4":
            b += c["tokens"] * 2 * (_row(c) + H * D * 2)
        return {"bytes": b, "flops": 6 * n * (G + 1) * H * D}
    if c["kind"] == "read":
        return {"bytes": c["tokens"] * 2 * (_row(c) + 2 * H * D), "flops": 0}
    n, ql = (x.astype(np.float64) for x in _tokens(c))
    w = np.full_like(n, c["window"]) if c["window"] else n
    k = np.minimum(c["sinks"], n) if c["window"] else 0 * n
    read = np.minimum(n, k + w + ql - 1)
    # query of rank p sees min(p + 1, k + w) keys: the ranks below `full` see fewer
    full = np.minimum(n, k + w)
    few = np.clip(full - (n - ql), 0, ql)
    pairs = ql * full - few * (few - 1) / 2
    return {"bytes": float((read * 2 * _row(c) + ql * 2 * G * H * D * 2).sum()),
            "flops": float(4 * D * H * G * pairs.sum())}


def _exact_e2m1(x):
    """Nearest value that 4 bits and a shared exponent per 32 hold, in 64 bits."""
    g = x.reshape(*x.shape[:-1], -1, 32)
    top = g.abs().amax(-1, keepdim=True)
    e = torch.floor(torch.log2(top.clamp_min(2.0 ** -100))) - 2
    t = g / torch.exp2(e)
    step = torch.exp2(torch.floor(torch.log2(t.abs().clamp_min(1.0))) - 1)
    return (torch.round(t / step) * step).clamp(-6, 6).mul(torch.exp2(e)).reshape(x.shape)


def _exact_values(plane, c):
    """float64 values of a plane's rows [slots, heads, dim], from the formats' definitions."""
    H, D = c["heads"], c["dim"]
    if c["kv"] != "mxfp4":
        return plane.reshape(-1, H, D).double()
    rows = plane.reshape(-1, plane.shape[-1])
    b = rows[:, : H * D // 2]
    code = torch.empty(rows.shape[0], H * D, dtype=torch.int64, device=rows.device)
    code[:, 0::2], code[:, 1::2] = b % 16, b // 16
    size = torch.tensor(_E2M1, dtype=torch.float64, device=rows.device)[code % 8]
    e = rows[:, H * D // 2: H * D // 2 + H * D // 32].double() - 127
    x = torch.where(code >= 8, -size, size).view(-1, H, D // 32, 32)
    return (x * torch.exp2(e).view(-1, H, D // 32, 1)).view(-1, H, D)


def exact(case, seed):
    s = prepare(case, seed)
    c = s["case"]
    H, G, D = c["heads"], c["group"], c["dim"]
    if c["kind"] == "read":
        rows = s["slots"].long()
        return {n: _exact_values(s["pool"][i], c)[rows] for i, n in enumerate("kv")}
    if c["kind"] == "write":
        pos, keep = s["positions"].long(), s["slots"] >= 0
        rot = c["rotary"]
        cos, sin = s["cos_sin"][pos].double()[:, None].chunk(2, -1)

        def turned(x, w):
            x = x.double()
            if w is not None:
                x = x / torch.sqrt((x * x).sum(-1, keepdim=True) / D + 1e-6) * w.double()
            i = torch.arange(rot // 2, device="cuda")
            a, b = (2 * i, 2 * i + 1) if c["interleaved"] else (i, i + rot // 2)
            y = x.clone()
            y[..., a] = x[..., a] * cos - x[..., b] * sin
            y[..., b] = x[..., a] * sin + x[..., b] * cos
            return y

        q = torch.where(keep[:, None, None], turned(s["q"], s["q_weight"]), s["q_out"].double())
        k, v = turned(s["k"], s["k_weight"]), s["v"].double()
        if c["kv"] == "mxfp4":
            lost = torch.where(keep, 0.0, math.nan)[:, None, None]
            return {"q": q, "k": _exact_e2m1(k) + lost, "v": _exact_e2m1(v) + lost}
        pool = torch.stack([_exact_values(p, c) for p in s["pool"]])
        for plane, x in zip(pool, (k, v)):
            plane[s["slots"][keep].long()] = x[keep]
        return {"q": q, "pool": pool.view(s["pool"].shape)}
    n, ql = _tokens(c)
    if 4 * D * H * G * float((n * ql).sum()) > 6e12:
        return None
    k, v = (_exact_values(p, c) for p in s["pool"])
    out, at, row = [], 0, 0
    for nr, qr in zip(n.tolist(), ql.tolist()):
        slots = s["slots"][at: at + nr].long()
        kr, vr = k[slots].transpose(0, 1), v[slots].transpose(0, 1)
        q = s["q"][row: row + qr].double()
        at, row = at + nr, row + qr
        got = []
        for j in range(0, qr, 1024):
            qj = q[j: j + 1024]
            rank = torch.arange(nr - qr + j, nr - qr + j + qj.shape[0], device="cuda")[:, None]
            key = torch.arange(nr, device="cuda")[None]
            hidden = key > rank
            if c["window"] > 0:
                hidden |= (key >= c["sinks"]) & (key <= rank - c["window"])
            x = torch.matmul(qj.view(-1, H, G, D).permute(1, 2, 0, 3).reshape(H, -1, D),
                             kr.transpose(1, 2).contiguous()) / math.sqrt(D)
            x = x.view(H, G, -1, nr).masked_fill(hidden, -math.inf)
            p = torch.softmax(x, -1).nan_to_num(0.0)
            y = torch.matmul(p.view(H, -1, nr), vr.contiguous()).view(H, G, -1, D)
            got.append(y.permute(2, 0, 1, 3).reshape(-1, H * G, D))
        out.append(torch.cat(got))
    return torch.cat(out)
