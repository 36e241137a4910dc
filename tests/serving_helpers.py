"""Plain definitions of the row and attention calls, in 64 bits on the host (and, for the 4-bit
format, in the formula's own 32-bit steps), and inputs for their tests."""
import numpy as np
import torch

E2M1 = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]
TYPES = {"fp16": torch.float16, "bf16": torch.bfloat16, "fp8": torch.float8_e4m3fn}
HALF_STEP = {"fp16": 2.0 ** -11, "bf16": 2.0 ** -8, "fp8": 2.0 ** -4}   # relative
# half of the step between the smallest values, where the relative step ends
HALF_TINY = {"fp16": 2.0 ** -25, "bf16": 2.0 ** -134, "fp8": 2.0 ** -10}


def row_bytes(H, D):
    return -(-H * (D // 2 + D // 32) // 16) * 16


def pack4(x):
    """float32 [n][H][D] -> uint8 [n][row bytes], one value at a time from the format's words."""
    x = np.asarray(x, np.float32)
    n, H, D = x.shape
    out = np.zeros((n, row_bytes(H, D)), np.uint8)
    g = x.reshape(n, H * D // 32, 32)
    top = np.abs(g).max(-1)
    finite = np.isfinite(g).all(-1)
    _, ex = np.frexp(np.where(finite, top, 1.0))
    e = np.clip(ex - 1 - 2 + 127, 1, 254)
    e = np.where(top == 0, 1, e)
    t = np.where(finite[..., None], np.abs(g), 0).astype(np.float64) / 2.0 ** (e - 127.0)[..., None]
    grid = np.array(E2M1)
    lo = np.clip(np.searchsorted(grid, t, side="right") - 1, 0, 7)
    hi = np.minimum(lo + 1, 7)
    mid = (grid[lo] + grid[hi]) / 2
    code = np.where(t > mid, hi, np.where(t < mid, lo, np.where(lo % 2 == 0, lo, hi)))
    code = np.where(np.signbit(g) & finite[..., None], code + 8, code).reshape(n, H * D // 2, 2)
    out[:, : H * D // 2] = code[..., 0] + 16 * code[..., 1]
    out[:, H * D // 2: H * D // 2 + H * D // 32] = np.where(finite, e, 255)
    return torch.from_numpy(out)


def values(rows, kind, H, D):
    """Rows of a plane (bytes [n][row bytes]) -> float64 [n][H][D]."""
    rows = rows.cpu()
    if kind != "mxfp4":
        return rows.contiguous().view(TYPES[kind]).double().reshape(-1, H, D)
    b = rows.numpy()
    c = b[:, : H * D // 2].astype(np.int64)
    code = np.stack([c & 15, c >> 4], -1).reshape(-1, H * D // 32, 32)
    v = np.where(code >= 8, -1.0, 1.0) * np.array(E2M1)[code & 7]
    e = b[:, H * D // 2: H * D // 2 + H * D // 32].astype(np.float64)
    scale = np.where(e == 255, np.nan, 2.0 ** (e - 127))
    return torch.from_numpy((v * scale[..., None]).reshape(-1, H, D))


def normed(x, w, eps):
    """float32 [n][heads][D] in the formula's steps: mean and root in 64 bits, the rest in 32."""
    if w is None:
        return x
    r = (1.0 / torch.sqrt(x.double().square().sum(-1, keepdim=True) / x.shape[-1] + eps)).float()
    return (x * r) * w


def turned(x, cos_sin, pos, interleaved):
    """The rotation in the dtype of x."""
    rot = cos_sin.shape[1]
    i = torch.arange(rot // 2)
    a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + rot // 2)
    cs = cos_sin.to(x.dtype)[pos.long()][:, None]
    c, s = cs[..., : rot // 2], cs[..., rot // 2:]
    y = x.clone()
    y[..., a] = x[..., a] * c - x[..., b] * s
    y[..., b] = x[..., b] * c + x[..., a] * s
    return y


def attention(q, k, v, window, sinks, scale):
    """float64 [ql][Hq][D] over k, v [n][H][D] (values), and the same with |v|: what the roundings
    of the weights are relative to. Masked keys have no part, whatever they hold."""
    ql, Hq, D = q.shape
    n, H = k.shape[:2]
    out, size = torch.zeros(2, ql, Hq, D, dtype=torch.float64)
    for i in range(ql):
        p = n - ql + i
        seen = [j for j in range(n)
                if j <= p and (window == 0 or j > p - window or j < sinks)]
        if not seen:
            continue
        ks = k[seen].repeat_interleave(Hq // H, 1)
        vs = v[seen].repeat_interleave(Hq // H, 1)
        w = torch.softmax((q[i][None].double() * ks).sum(-1) * scale, 0)
        out[i] = (w[..., None] * vs).sum(0)
        size[i] = (w[..., None] * vs.abs()).sum(0)
    return out, size


def make_rows(kind, n, H, D, g):
    """Random rows (bytes [n][row bytes])."""
    x = torch.randn(n, H, D, generator=g)
    if kind == "mxfp4":
        return pack4(x)
    return x.to(TYPES[kind]).view(torch.uint8).reshape(n, -1)


def make_cache(B, planes, kind, H, D, S):
    """A cache over planes [2L][slots][row bytes] (host bytes), slots a multiple of S."""
    P, slots, row = planes.shape
    dev = planes.cuda()
    if kind == "mxfp4":
        return B.PackedKVCache(dev.view(P, slots // S, S, row), P // 2, H, D, S)
    kv = dev.view(TYPES[kind]).view(P, slots // S, S, H, D)
    return B.KVCache(kv, P // 2, H, D, S)


def bytes_of(cache):
    """The cache's bytes on the host, [2L][slots][row bytes]."""
    P = 2 * cache.num_layers
    return cache.kv.view(torch.uint8).reshape(P, cache.num_blocks * cache.block_size, -1).cpu()
