"""Argument errors of the paged cache's entry points, all found before a device is touched, and the oracle's own pins."""
import ctypes
import math

import pytest
import torch

import paper_2603_24517_b200 as lib
from oracle import cache_oracle as orc
from paper_2603_24517_b200 import binding
from paper_2603_24517_b200 import build as lib_build


@pytest.fixture(scope="module")
def cdll():
    lib_build.build()
    return lib.load_library()


def _cache(**other):
    at = dict(k=0x1000, v=0x2000, k_scale=0x3000, v_scale=0x4000, block_table=0x5000, seq_lens=0x6000, starts=None,
              k_strides=(64 * 2 * 128, 128, 64 * 128), v_strides=(64 * 2 * 128, 128, 64 * 128), table_stride=4, type=0,
              n_pages=8, page_size=64, Hkv=2, D=128, B=2, max_blocks=4)
    at.update(other)
    c = binding._KvCacheStruct()
    for name, x in at.items():
        setattr(c, name, (ctypes.c_longlong * 3)(*x) if name.endswith("strides") else x)
    return c


def _strides(s):
    return None if s is None else (ctypes.c_longlong * 3)(*s)


def _append(c, k=0x7000, v=0x8000, S=5, ks=None, vs=None, fn="attn_kv_append", **other):
    return getattr(c, fn)(ctypes.byref(_cache(**other)), k, v, S, _strides(ks), _strides(vs), None)


def _attend(c, q=0x7000, o=0x8000, lse=0x9000, Hq=4, S=5, max_new=5, causal=1, scale=0.1, qs=None, os=None, ws=0xa000,
            ws_bytes=1 << 30, **other):
    return c.attn_fwd_cached(ctypes.byref(_cache(**other)), q, o, lse, Hq, S, max_new, causal, scale, _strides(qs), _strides(os), ws,
                             ws_bytes, None)


@pytest.mark.parametrize("call", [_append, lambda c, **o: _append(c, fn="attn_kv_read", **o), _attend])
def test_cache_argument_errors(cdll, call):
    for name in ("k", "v") if call is _attend else ():
        assert call(cdll, **{name: None}) == 1, name
    for name in ("k_scale", "v_scale", "block_table", "seq_lens"):
        assert call(cdll, **{name: None}) == 1, name
        assert call(cdll, **{name: 0x3002}) == 4, name
    assert call(cdll, starts=0x3001) == 4
    for name in ("n_pages", "page_size", "Hkv", "D", "B", "max_blocks", "S"):
        assert call(cdll, **{name: 0}) == 2, name
    assert call(cdll, D=64) == 3
    for page in (8, 48, 256, 17):
        assert call(cdll, page_size=page) == 3, page
    assert call(cdll, type=2) == 3 and call(cdll, type=-1) == 3
    assert call(cdll, max_blocks=1 << 25) == 3
    assert call(cdll, S=(1 << 30) // 2 + 1) == 3
    for name in ("k_strides", "v_strides"):
        assert call(cdll, **{name: (0, 128, 8192)}) == 2
        assert call(cdll, **{name: (16384, 64, 8192)}) == 2
        assert call(cdll, **{name: (16384, 136, 8192)}) == 4
        assert call(cdll, **{name: (1 << 39, 128, 8192)}) == 3
    assert call(cdll, table_stride=-1) == 2


def test_row_tensor_errors(cdll):
    for fn in ("attn_kv_append", "attn_kv_read"):
        assert _append(cdll, k=None, fn=fn) == 1 and cdll.attn_kv_append(None, 0x7000, 0x8000, 5, None, None, None) == 1
        assert getattr(cdll, fn)(ctypes.byref(_cache()), 0x7000, None, 5, None, None, None) == 1
    p = ctypes.byref(_cache())
    for fn in (cdll.attn_kv_append, cdll.attn_kv_read):
        assert fn(p, 0x7008, 0x8000, 5, None, None, None) == 4
        assert fn(p, 0x7000, 0x8000, 5, _strides((1280, 260, 128)), None, None) == 4
        assert fn(p, 0x7000, 0x8000, 5, None, _strides((1280, 0, 128)), None) == 2
        assert fn(p, 0x1000, 0x8000, 5, None, None, None) == 3   # the cache itself
    assert cdll.attn_kv_read(p, 0x7000, 0x7000, 5, None, None, None) == 3
    assert cdll.attn_kv_append(ctypes.byref(_cache(v=0x1000)), 0x7000, 0x8000, 5, None, None, None) == 3


def test_attention_argument_errors(cdll):
    for name in ("q", "o", "ws"):
        assert _attend(cdll, **{name: None}) == 1, name
        assert _attend(cdll, **{name: 0xb008}) == 4, name
    assert _attend(cdll, lse=0x9002) == 4
    assert _attend(cdll, Hq=0) == 2 and _attend(cdll, Hq=3) == 2 and _attend(cdll, max_new=0) == 2
    for scale in (0.0, -1.0, math.inf, math.nan):
        assert _attend(cdll, scale=scale) == 3
    assert _attend(cdll, qs=(0, 512, 128)) == 2 and _attend(cdll, os=(2560, 512, 130)) == 4
    assert _attend(cdll, o=0x7000) == 3 and _attend(cdll, ws=0x7000) == 3 and _attend(cdll, o=0x2000) == 3
    assert _attend(cdll, ws_bytes=cdll.attn_fwd_cached_workspace_bytes(4, 2, 5) - 1) == 8


def test_binding_refusals():
    cache = lib.KVCache(*(torch.zeros(4, 16, 2, 128, dtype=torch.int8) for _ in "kv"), *(torch.zeros(4, 2) for _ in "kv"))
    table, lens = torch.zeros(1, 4, dtype=torch.int32), torch.ones(1, dtype=torch.int32)
    rows = torch.zeros(1, 1, 2, 128, dtype=torch.bfloat16)
    with pytest.raises(ValueError):  # not on a GPU
        lib.kv_cache_append(cache, rows, rows, table, lens)
    with pytest.raises(ValueError):
        lib.new_kv_cache(4, 16, 2, torch.float16, device="cpu")
    with pytest.raises(ValueError):
        lib.kv_cache_read(cache, table, lens)


def test_struct_matches_the_header():
    # four pointers, three pointers, 2 x 3 strides, one stride, seven ints
    assert ctypes.sizeof(binding._KvCacheStruct) == 7 * 8 + 6 * 8 + 8 + 7 * 4 + 4
    # the packed form is the same bytes
    values = list(range(1, 22))
    c = binding._KvCacheStruct(*values[:7], (ctypes.c_longlong * 3)(*values[7:10]), (ctypes.c_longlong * 3)(*values[10:13]), *values[13:])
    assert bytes(c)[:140] == binding._pack_cache(*values)[:140] and len(binding._pack_cache(*values)) == ctypes.sizeof(c)


def test_oracle_codes_are_the_types_own():
    g = torch.Generator().manual_seed(0)
    x = torch.cat((torch.randn(4096, generator=g) * 100, torch.randn(4096, generator=g) * 0.01, torch.arange(-448, 449) / 1.0,
                   torch.tensor([0.0, 2.0 ** -10, 3 * 2.0 ** -10, 464.0, 1e9]))).clamp(-448, 448)
    assert torch.equal(orc.e4m3_round(x.double()), x.to(torch.float8_e4m3fn).double())
    assert orc.scale_for(448.0, False) == 1.0 and orc.scale_for(448.5, False) == 2.0 and orc.scale_for(224.0, False) == 0.5
    assert orc.scale_for(127.0, True) == 1.0 and orc.scale_for(0.0, True) == 0.0


def test_oracle_attention_is_a_weighted_mean():
    k = torch.zeros(5, 1, 128, dtype=torch.float64)
    v = torch.arange(5.0, dtype=torch.float64)[:, None, None].expand(5, 1, 128)
    o, lse, _, _ = orc.attend(torch.ones(3, 2, 128), k, v, 1, True, 0.1)  # positions 1, 2, 3 of equal scores
    assert torch.allclose(o[:, 0, 0], torch.tensor([0.5, 1.0, 1.5], dtype=torch.float64))
    assert torch.allclose(lse[1], torch.tensor([2.0, 3.0, 4.0], dtype=torch.float64).log())
    o, lse, _, _ = orc.attend(torch.ones(3, 2, 128), k, v, -2, True, 0.1)  # positions -2, -1, 0
    assert not bool(o.any()) and lse[0].tolist() == [-math.inf, -math.inf, 0.0]
