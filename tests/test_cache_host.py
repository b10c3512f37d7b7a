"""Serving entry points, what needs no GPU: descriptor layout and refusals (reported before any CUDA call)."""
import ctypes as C

import numpy as np
import pytest
import torch


@pytest.fixture(scope="module")
def B():
    from paper_2402_05628_b200.build import build_library
    build_library()
    from paper_2402_05628_b200 import binding
    return binding


def flat(s):
    out = []
    for name, t in s._fields_:
        v = getattr(s, name)
        out += flat(v) if isinstance(v, C.Structure) else [v]
    return out


@pytest.mark.parametrize("pack,desc", [("_pack_plan", "CachePlanDesc"), ("_pack_write", "CacheWriteDesc"),
                                       ("_pack_attention", "CacheAttentionDesc"), ("_pack_logprobs", "TokenLogprobsDesc")])
def test_packed_descriptors_have_the_c_layout(B, pack, desc):
    cls = getattr(B, desc)
    n = len(flat(cls()))
    values = list(range(1, n + 1))
    assert flat(cls.from_buffer_copy(getattr(B, pack)(*values))) == values


def status(B, d, fn):
    return getattr(B.lib(), fn)(C.addressof(d), *((None, 0, None) if fn == "repq_cache_attention" else (None,)))


def cache(B, **kw):
    c = B.CacheDesc(16, 16, 16, 16, 4, 2, 16, 64)
    for k, v in kw.items():
        setattr(c, k, v)
    return c


@pytest.mark.parametrize("change,code", [
    (dict(block_size=24), 2), (dict(d_h=72), 2), (dict(d_h=144), 2), (dict(k_codes=None), 1), (dict(num_blocks=0), 1),
    (dict(v_codes=24), 3), (dict(num_blocks=1 << 30), 2)])
def test_cache_refusals(B, change, code):
    c = cache(B, **change)
    assert status(B, B.CacheWriteDesc(c, 1, 1, 16, 64, 64, 16, 64, 64, 16), "repq_cache_write") == code
    assert "repq_cache_write" in B.repq_last_error()
    d = B.CacheAttentionDesc(c, 1, 1, 4, 1, 1, 1)
    assert status(B, d, "repq_cache_attention") == code


@pytest.mark.parametrize("field,value,code", [("tokens", -1, 1), ("dtype", 2, 1), ("k", None, 1), ("slot_map", None, 1), ("v", 24, 3),
                                              ("k_stride_token", 60, 3), ("v_stride_head", 4, 3)])
def test_write_refusals(B, field, value, code):
    d = B.CacheWriteDesc(cache(B), 1, 1, 16, 64, 64, 16, 64, 64, 16)
    setattr(d, field, value)
    assert status(B, d, "repq_cache_write") == code


def test_write_of_nothing(B):
    assert status(B, B.CacheWriteDesc(cache(B), 0, 1, None, 0, 0, None, 0, 0, None), "repq_cache_write") == B.REPQ_OK


def attention(B, **kw):
    d = B.CacheAttentionDesc(cache(B))
    base = dict(requests=1, tokens=1, heads=4, max_q_len=1, max_kv_len=10, q_dtype=1, q=16, q_stride_token=256, q_stride_head=64,
                block_table=16, ld_table=4, table_width=4, kv_lens=16, cu_q=16, alpha=1.0, out_kind=1, out_bits=8, out_scale=1.0, out=16,
                ldo=256, o_stride_head=64)
    for k, v in dict(base, **kw).items():
        setattr(d, k, v)
    return d


@pytest.mark.parametrize("change,code", [
    (dict(heads=3), 1), (dict(heads=0), 1), (dict(requests=-1), 1), (dict(max_kv_len=-1), 1), (dict(q_dtype=5), 1), (dict(out_kind=7), 1),
    (dict(out_kind=2, out_bits=5), 1), (dict(out_kind=2, out_scale=0.0), 1), (dict(ld_table=3, requests=2), 1), (dict(q=None), 1), (dict(out=None), 1),
    (dict(kv_lens=None), 1), (dict(cu_q=None), 1), (dict(block_table=None), 1), (dict(q=24), 3), (dict(q_stride_head=4), 3), (dict(out=20), 3),
    (dict(ldo=260), 3), (dict(out_kind=2, out=18), 3)])
def test_attention_refusals(B, change, code):
    assert status(B, attention(B, **change), "repq_cache_attention") == code


@pytest.mark.parametrize("change", [dict(requests=0), dict(tokens=0), dict(max_q_len=0)])
def test_attention_of_nothing(B, change):
    assert status(B, attention(B, **change), "repq_cache_attention") == B.REPQ_OK


@pytest.mark.parametrize("field,value,code", [
    ("requests", -1, 1), ("block_size", 48, 2), ("cu_q", None, 1), ("kv_lens", None, 1), ("free_list", None, 1), ("slot_map", None, 1),
    ("ld_table", 3, 1), ("kv_lens_out", 32, 1), ("free_head_out", 80, 1), ("block_table", None, 1)])
def test_plan_refusals(B, field, value, code):
    d = B.CachePlanDesc(2, 16, 4, 8, 32, 32, 48, 64, 4, 16, 80, 96, 112, 128, 144, 160, 176)
    setattr(d, field, value)
    assert status(B, d, "repq_cache_plan") == code


@pytest.mark.parametrize("field,value,code", [
    ("rows", -1, 1), ("vocab", 0, 1), ("dtype", 3, 1), ("top", 33, 2), ("top", -1, 2), ("logits", None, 1), ("ld", 99, 1), ("tokens", None, 1),
    ("top_ids", None, 1), ("logits", 18, 3)])
def test_logprobs_refusals(B, field, value, code):
    d = B.TokenLogprobsDesc(2, 100, 2, 0, 16, 100, 16, 16, 16, 16, 16, 16)
    setattr(d, field, value)
    assert status(B, d, "repq_token_logprobs") == code
    d.rows = 0
    assert field in ("rows", "vocab", "dtype", "top") or status(B, d, "repq_token_logprobs") == B.REPQ_OK


def test_binding_refuses_other_types_and_shapes(B):
    i = torch.zeros(2, dtype=torch.int32)
    c = B.CacheTensors(torch.zeros(2, 1, 16, 32, dtype=torch.uint8), torch.zeros(2, 1, 16, 32, dtype=torch.uint8), torch.zeros(2, 1), torch.zeros(2, 1))
    k = torch.zeros(2, 1, 32)
    with pytest.raises(TypeError):
        B.repq_cache_write(c, k, k, i.long())
    with pytest.raises(ValueError):
        B.repq_cache_write(c, k, k[:, :, :16], i)
    with pytest.raises(TypeError):
        B.repq_cache_write(c, k.half(), k.half(), i)
    with pytest.raises(TypeError):
        B.repq_cache_write(c._replace(k_scale=torch.zeros(2, 2)), k, k, i)
    q, t = torch.zeros(2, 1, 32), torch.zeros(1, 4, dtype=torch.int32)
    kw = dict(max_q_len=2, max_kv_len=4, alpha=1.0)
    ws = torch.zeros(16, dtype=torch.uint8)
    with pytest.raises(ValueError):
        B.repq_cache_attention(c, q, t, i, i, torch.zeros(2, 1, 32), ws, **kw)
    with pytest.raises(TypeError):
        B.repq_cache_attention(c, q, t, i[:1], i, torch.zeros(2, 1, 32).double(), ws, **kw)
    with pytest.raises(ValueError):
        B.repq_token_logprobs(torch.zeros(3, 5), i, torch.zeros(3))
    with pytest.raises(TypeError):
        B.repq_token_logprobs(torch.zeros(2, 5), i, torch.zeros(2, dtype=torch.float64))
    with pytest.raises(ValueError):
        B.repq_cache_plan(i, i, t, i, i[:1], 16, kv_lens_out=i, cu_q=i, slot_map=i, positions=None, free_head_out=i[:1])
