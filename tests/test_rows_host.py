"""Refusals of the row and attention calls, on the host: documented statuses before any device
work, and the binding's own checks."""
import ctypes
import os
from types import SimpleNamespace

import pytest
import torch

from paper_2608_13263_amd import binding as B

pytestmark = pytest.mark.skipif(not os.path.exists(B.LIB_PATH),
                                reason="libvtoken.so not built (run __graft_entry__.build())")
CODE = B.STATUS_CODE
P = (ctypes.addressof(ctypes.create_string_buffer(4096)) + 15) // 16 * 16   # only compared


def _cache(**kw):
    c = dict(kv=P, num_layers=2, num_kv_heads=8, head_dim=128, block_size=16, num_blocks=100,
             elem_bytes=2)
    c.update(kw)
    return B.CCache(**c)


def _write(**kw):
    w = dict(q=P, k=P, v=P, q_out=P, q_stride=4096, k_stride=1024, v_stride=1024,
             q_out_stride=4096, q_weight=P, k_weight=P, cos_sin=P, positions=P, slots=P,
             num_tokens=0, num_q_heads=32, num_kv_heads=8, head_dim=128, rotary_dim=128,
             num_positions=10, interleaved=0, layer=1, dtype=B.KV_BF16, kv_dtype=B.KV_BF16,
             eps=1e-6)
    w.update(kw)
    return B.CKVWrite(**w)


def _read(**kw):
    r = dict(slots=P, k_out=P, v_out=P, k_stride=1024, v_stride=1024, num_tokens=0,
             num_kv_heads=8, head_dim=128, layer=1, dtype=B.KV_BF16, kv_dtype=B.KV_BF16)
    r.update(kw)
    return B.CKVRead(**r)


def _attention(**kw):
    a = dict(q=P, out=P, q_stride=4096, out_stride=4096, q_indptr=P, slot_count=None,
             workspace=None, workspace_bytes=0, num_queries=0, max_queries=4, max_tokens=100,
             num_q_heads=32, num_kv_heads=8, head_dim=128, layer=1, dtype=B.KV_BF16,
             kv_dtype=B.KV_BF16, window=0, sinks=0, scale=1.0)
    a.update(kw)
    return B.CAttention(**a)


def _status(call, struct, cache=None, *more):
    c = _cache() if cache is None else cache
    return getattr(B.load_library(), call)(ctypes.byref(c), ctypes.byref(struct), *more)


SHARED = [
    (dict(layer=2), "SHAPE"), (dict(layer=-1), "SHAPE"), (dict(num_kv_heads=4), "SHAPE"),
    (dict(head_dim=64), "SHAPE"), (dict(dtype=B.KV_FP16), "SHAPE"), (dict(dtype=2), "SHAPE"),
    (dict(kv_dtype=B.KV_FP16), "SHAPE"), (dict(kv_dtype=B.KV_FP8_E4M3), "SHAPE"),
    (dict(kv_dtype=B.KV_MXFP4), "SHAPE"), (dict(kv_dtype=4), "SHAPE"),
]


@pytest.mark.parametrize("change,code", SHARED + [
    (dict(num_tokens=-1), "SHAPE"), (dict(num_q_heads=-1), "SHAPE"),
    (dict(rotary_dim=136), "SHAPE"), (dict(rotary_dim=8), "SHAPE"), (dict(rotary_dim=0), "SHAPE"),
    (dict(rotary_dim=12, interleaved=1), "SHAPE"), (dict(interleaved=2), "ARGUMENT"),
    (dict(num_tokens=2 ** 31 - 1), "SHAPE"), (dict(num_positions=-1), "SHAPE"),
    (dict(num_tokens=2, slots=None), "NULL"), (dict(num_tokens=2, positions=None), "NULL"),
    (dict(num_tokens=2, k=None), "NULL"), (dict(num_tokens=2, v=None), "NULL"),
    (dict(num_tokens=2, q=None), "NULL"), (dict(num_tokens=2, q_out=None), "NULL"),
    (dict(num_tokens=2, k=P + 8), "ARGUMENT"), (dict(num_tokens=2, v_stride=1020), "ARGUMENT"),
    (dict(num_tokens=2, q_stride=4088), "ARGUMENT"), (dict(num_tokens=2, k_stride=-1024), "ARGUMENT"),
    (dict(num_tokens=2, q_out_stride=0), "ARGUMENT"),
])
def test_write_refuses(change, code):
    assert _status("vtoken_write_kv", _write(**change), None, None) == CODE["VTOKEN_ERR_" + code]


@pytest.mark.parametrize("change,code", SHARED + [
    (dict(num_tokens=-1), "SHAPE"), (dict(num_tokens=2, slots=None), "NULL"),
    (dict(num_tokens=2, k_out=None), "NULL"), (dict(num_tokens=2, v_out=P + 2), "ARGUMENT"),
    (dict(num_tokens=2, k_stride=1016), "ARGUMENT"), (dict(num_tokens=2 ** 31 - 1), "SHAPE"),
])
def test_read_refuses(change, code):
    assert _status("vtoken_read_kv", _read(**change), None, None) == CODE["VTOKEN_ERR_" + code]


@pytest.mark.parametrize("change,code", SHARED + [
    (dict(num_queries=-1), "SHAPE"), (dict(max_tokens=-1), "SHAPE"), (dict(max_queries=-1), "SHAPE"),
    (dict(num_queries=5, max_queries=0), "SHAPE"), (dict(window=-1), "ARGUMENT"),
    (dict(sinks=-1), "ARGUMENT"), (dict(num_q_heads=36), "SHAPE"), (dict(num_q_heads=0), "SHAPE"),
    (dict(num_q_heads=136), "SHAPE"), (dict(head_dim=96), "SHAPE"),
    (dict(q_indptr=None), "SHAPE"), (dict(q_indptr=None, max_queries=1, num_queries=1), "SHAPE"),
    (dict(num_queries=5, q=None), "NULL"), (dict(num_queries=5, out=None), "NULL"),
    (dict(num_queries=5, q=P + 4), "ARGUMENT"), (dict(num_queries=5, out_stride=4000), "ARGUMENT"),
])
def test_attention_refuses(change, code):
    st = _status("vtoken_paged_attention", _attention(**change), None, 2, P, P, None)
    assert st == CODE["VTOKEN_ERR_" + code]


def test_null_structs_and_indptr():
    lib = B.load_library()
    c = _cache()
    for call in (lib.vtoken_write_kv, lib.vtoken_read_kv):
        assert call(ctypes.byref(c), None, None) == CODE["VTOKEN_ERR_NULL"]
        assert call(None, None, None) == CODE["VTOKEN_ERR_NULL"]
    assert lib.vtoken_paged_attention(ctypes.byref(c), None, 1, P, P, None) == CODE["VTOKEN_ERR_NULL"]
    assert _status("vtoken_paged_attention", _attention(num_queries=5), None, 2, None, P,
                   None) == CODE["VTOKEN_ERR_NULL"]
    assert _status("vtoken_paged_attention", _attention(num_queries=5), None, -1, P, P,
                   None) == CODE["VTOKEN_ERR_SHAPE"]
    assert lib.vtoken_attention_workspace_bytes(None, 1) == -1
    assert lib.vtoken_attention_workspace_bytes(ctypes.byref(_attention(window=-1)), 1) == -1


def test_calls_of_nothing_return_ok():
    """No tokens, queries or requests: nothing is enqueued (there is no device here)."""
    assert _status("vtoken_write_kv", _write(), None, None) == 0
    assert _status("vtoken_read_kv", _read(), None, None) == 0
    assert _status("vtoken_paged_attention", _attention(), None, 2, P, P, None) == 0
    assert _status("vtoken_paged_attention", _attention(num_queries=3), None, 0, P, P, None) == 0


def test_workspace_too_small_is_refused():
    a = _attention(num_queries=2, q_indptr=None, max_queries=1, max_tokens=100000)
    need = B.attention_workspace_bytes(a, 2)
    if need == 0:
        pytest.skip("this size takes no workspace")
    assert _status("vtoken_paged_attention", a, None, 2, P, P, None) == CODE["VTOKEN_ERR_NULL"]
    a.workspace, a.workspace_bytes = P, need - 1
    assert _status("vtoken_paged_attention", a, None, 2, P, P, None) == CODE["VTOKEN_ERR_CAPACITY"]


def test_row_bytes():
    assert B.kv_row_bytes(8, 128, B.KV_BF16) == 2048
    assert B.kv_row_bytes(8, 128, B.KV_FP8_E4M3) == 1024
    assert B.kv_row_bytes(8, 128, B.KV_MXFP4) == 8 * 68
    assert B.kv_row_bytes(1, 128, B.KV_MXFP4) == 80       # 68, padded
    assert B.kv_row_bytes(3, 32, B.KV_MXFP4) == 64        # 51, padded
    for args in ((8, 48, B.KV_MXFP4), (8, 264, B.KV_BF16), (0, 128, B.KV_BF16), (8, 4, B.KV_FP16),
                 (8, 128, 4)):
        with pytest.raises(B.VTokenError, match="SHAPE"):
            B.kv_row_bytes(*args)


def test_a_packed_cache_needs_its_geometry():
    c = _cache(num_kv_heads=1, head_dim=544, elem_bytes=1)
    assert _status("vtoken_read_kv", _read(kv_dtype=B.KV_MXFP4), c, None) == 0
    assert _status("vtoken_read_kv", _read(kv_dtype=B.KV_MXFP4, num_kv_heads=4), c,
                   None) == CODE["VTOKEN_ERR_SHAPE"]
    assert _status("vtoken_read_kv", _read(kv_dtype=B.KV_MXFP4, dtype=B.KV_FP16), c,
                   None) == CODE["VTOKEN_ERR_SHAPE"]


def test_struct_layouts_match_header(tmp_path):
    import shutil
    import subprocess
    if shutil.which("gcc") is None:
        pytest.skip("gcc not available")
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    structs = {"vtoken_kv_write": B.CKVWrite, "vtoken_kv_read": B.CKVRead,
               "vtoken_attention": B.CAttention}
    lines = ['#include <stdio.h>', '#include <stddef.h>', '#include "vtoken.h"', "int main(void){"]
    for name, cls in structs.items():
        lines.append(f'printf("%zu\\n", sizeof({name}));')
        lines += [f'printf("%zu\\n", offsetof({name}, {f}));' for f, _ in cls._fields_]
    lines.append('printf("%d\\n", VTOKEN_KV_MXFP4); return 0;}')
    (tmp_path / "x.c").write_text("\n".join(lines))
    subprocess.run(["gcc", "-D__HIP_PLATFORM_AMD__", "-I", os.path.join(root, "include"), "-I",
                    "/opt/rocm/include", str(tmp_path / "x.c"), "-o", str(tmp_path / "x")],
                   check=True)
    got = [int(x) for x in subprocess.run([str(tmp_path / "x")], check=True, capture_output=True,
                                          text=True).stdout.split()]
    want = []
    for cls in structs.values():
        want += [ctypes.sizeof(cls)] + [getattr(cls, f).offset for f, _ in cls._fields_]
    assert got == want + [B.KV_MXFP4]


def test_binding_checks_tensors():
    """Shapes, types and strides that the C calls cannot see (host tensors: refused before any)."""
    cpu = torch.device("cpu")
    x = torch.zeros(4, 8, 128, dtype=torch.bfloat16)
    assert B._activation(x, "x", cpu, torch.bfloat16, 8, 128) == 1024
    assert B._activation(x[::2], "x", cpu, torch.bfloat16, 8, 128) == 2048
    assert B._activation(x[:1], "x", cpu, torch.bfloat16, 8, 128) == 1024
    for bad in (x[0], x[:, :4], x.float(), x.transpose(1, 2), x[..., ::2],
                x.transpose(0, 1).contiguous().transpose(0, 1)):
        with pytest.raises(ValueError):
            B._activation(bad, "x", cpu, torch.bfloat16, 8, 128)
    with pytest.raises(ValueError):
        B._ints(torch.zeros(3, dtype=torch.int64), "slots", cpu)
    with pytest.raises(ValueError):
        B._ints(torch.zeros(6, dtype=torch.int32)[::2], "slots", cpu)
    with pytest.raises(ValueError):
        B._ints(torch.zeros(3, dtype=torch.int32), "slots", cpu, 4)
    with pytest.raises(ValueError):
        B._act_code(torch.float32)


def test_rotary_table():
    t = B.rotary_table(200001, 64, 500000.0, device="cpu")
    assert t.shape == (200001, 64) and t.dtype == torch.float32
    import math
    for p, i in ((0, 0), (200000, 0), (123457, 5), (199999, 31)):
        a = p * 500000.0 ** (-2 * i / 64)
        # angles in float64 are off by 2^-52 of 200,000: the cosines by less than a float's step
        assert abs(float(t[p, i]) - math.cos(a)) < 2.0 ** -23
        assert abs(float(t[p, 32 + i]) - math.sin(a)) < 2.0 ** -23


@pytest.mark.parametrize("name", ["max_tokens", "max_queries", "num_queries"])
def test_ranks_past_32_bits_are_refused(name):
    """Slots of a request and queries up to 2^30: the sum of a rank and a window fits an int32."""
    lib = B.load_library()
    for value, ok in ((2 ** 30, True), (2 ** 30 + 1, False), (2 ** 31 - 1, False)):
        a = _attention(**{name: value})
        assert (lib.vtoken_attention_workspace_bytes(ctypes.byref(a), 1) >= 0) is ok


def test_a_table_without_positions_is_refused():
    """Every position is outside of it, and there is no row to read in a bad one's place."""
    for tokens in (0, 2):
        st = _status("vtoken_write_kv", _write(num_positions=0, num_tokens=tokens), None, None)
        assert st == CODE["VTOKEN_ERR_SHAPE"]
    cache = SimpleNamespace(kv=torch.zeros(2, 1, 16, 2, 64, dtype=torch.bfloat16), num_kv_heads=2,
                            head_dim=64)
    x, i = torch.zeros(3, 2, 64, dtype=torch.bfloat16), torch.zeros(3, dtype=torch.int32)
    for shape in ((0, 64), (10, 0)):
        with pytest.raises(ValueError, match="no angles"):
            B.write_kv(cache, x, x, i, 0, positions=i, cos_sin=torch.zeros(shape))


def test_most_head_rows():
    """2^27 - 8 head rows, 32 lanes each at 256 dims, are a grid of less than 2^32 threads; a call of
    one more row is refused before the launch (slots of NULL are looked at later)."""
    c = _cache(num_kv_heads=1, head_dim=256)
    w = dict(num_q_heads=0, num_kv_heads=1, head_dim=256, rotary_dim=256, slots=None)
    r = dict(num_kv_heads=1, head_dim=256, slots=None)
    for tokens, code in ((2 ** 26 - 4, "NULL"), (2 ** 26 - 3, "SHAPE"), (2 ** 26, "SHAPE")):
        assert _status("vtoken_write_kv", _write(num_tokens=tokens, **w), c,
                       None) == CODE["VTOKEN_ERR_" + code]
        assert _status("vtoken_read_kv", _read(num_tokens=tokens, **r), c,
                       None) == CODE["VTOKEN_ERR_" + code]


def test_sizes_past_32_bits_are_refused():
    """The structs would keep the lower 32 bits: another layer, a window of 5, one of everything."""
    cache = SimpleNamespace(kv=torch.zeros(2, 1, 16, 2, 64, dtype=torch.bfloat16), num_kv_heads=2,
                            head_dim=64)
    x, i = torch.zeros(3, 2, 64, dtype=torch.bfloat16), torch.zeros(3, dtype=torch.int32)
    for far in (2 ** 31, 2 ** 32, 2 ** 32 + 5, -2 ** 32):
        with pytest.raises(ValueError, match="32 bits"):
            B.write_kv(cache, x, x, i, far)
        with pytest.raises(ValueError, match="32 bits"):
            B.read_kv(cache, i, far)
        for kw in (dict(layer=far), dict(max_tokens=far), dict(window=far), dict(sinks=far),
                   dict(max_queries=far, q_indptr=i)):
            with pytest.raises(ValueError, match="32 bits"):
                B.paged_attention(cache, x, i, i, **{"layer": 0, "max_tokens": 5, **kw})


def test_a_cache_off_16_bytes_is_refused():
    """A view that starts inside a row's 16 bytes: the kernels read and write 16 at a time."""
    for off in (2, 8, 15):
        c = _cache(kv=P + off)
        for st in (_status("vtoken_write_kv", _write(num_tokens=2), c, None),
                   _status("vtoken_read_kv", _read(num_tokens=2), c, None),
                   _status("vtoken_paged_attention", _attention(num_queries=5), c, 2, P, P, None)):
            assert st == CODE["VTOKEN_ERR_ARGUMENT"]
