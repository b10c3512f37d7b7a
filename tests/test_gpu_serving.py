"""A decoder served out of the paged 8-bit cache: one block against float64 attention over what its cache holds, and the same answer
whichever way a text reaches it (whole, in chunks, token by token, beside other requests)."""
import os
import sys

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def model():
    from paper_2402_05628_b200.build import build_library
    build_library()
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    import serve_decoder
    return serve_decoder, serve_decoder.build(dim=128, heads=2, positions=160, vocab=500)


def test_block_attends_to_what_its_cache_holds(model):
    """The attention codes inside a block (repeated here through the stages) against float64 attention over the cache's own values."""
    import torch
    from paper_2402_05628_b200 import binding as B
    from paper_2402_05628_b200.serving import PagedCache
    block = model[1].blocks[0]
    c = block.cfg
    D, H = c["D"], c["H"]
    dh = D // H
    cache = PagedCache(1, 40, H, 16, dh, 3, 160)
    g = torch.Generator(device="cuda:0").manual_seed(2)
    first, second = [50, 0, 16], [3, 70, 1]
    for q in (first, second):
        step = cache.plan(q)
        x = torch.randn(sum(q), D, device="cuda:0", generator=g).to(block.act_dtype)
        y = block.forward_cached(x, step, cache, 0)
    assert torch.isfinite(y.float()).all() and cache.free_blocks == 40 - 4 - 5 - 2
    kv = [53, 70, 17]
    assert step.kv_lens.tolist() == kv and step.positions.tolist() == list(range(50, 53)) + list(range(70)) + [16]
    ks, vs = ((t[0].double() - 128.0) * t[1].double()[:, :, None, None] for t in ((cache.layers[0].k_codes, cache.layers[0].k_scale),
                                                                                  (cache.layers[0].v_codes, cache.layers[0].v_scale)))
    q = torch.randn(sum(second), H, dh, device="cuda:0", generator=g).to(torch.bfloat16)
    out = torch.empty(sum(second), H, dh, dtype=torch.bfloat16, device="cuda:0")
    ws = cache.workspace(B.repq_cache_attention_workspace_bytes(cache.layers[0], q, cache.table, 70, 70))
    B.repq_cache_attention(cache.layers[0], q, cache.table, step.kv_lens, step.cu_q, out, ws, max_q_len=70, max_kv_len=70, alpha=dh ** -0.5)
    at = 0
    for b, n in enumerate(second):
        pages = cache.table[b, :-(-kv[b] // 16)].long()
        k, v = (t[pages].transpose(0, 1).reshape(H, -1, dh)[:, :kv[b]] for t in (ks, vs))
        s = torch.einsum("ihd,hjd->hij", q[at:at + n].double(), k) * dh ** -0.5
        s = s.masked_fill(torch.ones(n, kv[b], dtype=torch.bool, device="cuda:0").triu(kv[b] - n + 1), float("-inf"))
        ref = torch.einsum("hij,hjd->ihd", torch.softmax(s, -1), v)
        # bf16 outputs, weights of 11 bits
        assert ((out[at:at + n].double() - ref).abs() <= 2.0 ** -8 * ref.abs() + 2.0 ** -10 * v.abs().max()).all()
        at += n


def test_cached_keys_are_the_projection_within_half_a_step(model):
    """K of the prompt as the library's own projection gives it (rotated by position) lies within half a step of what the cache holds."""
    import torch
    from paper_2402_05628_b200 import binding as B
    from paper_2402_05628_b200.serving import PagedCache
    block = model[1].blocks[0]
    c = block.cfg
    D, H, T = c["D"], c["H"], 45
    cache = PagedCache(1, 4, H, 16, D // H, 1, 64)
    x = torch.randn(T, D, device="cuda:0").to(block.act_dtype)
    block.forward_cached(x, cache.plan([T]), cache, 0)
    ab = c["bits_a"] | B.REPQ_BYTE_CODES
    codes, sums = torch.empty(T, D, dtype=torch.uint8, device="cuda:0"), torch.empty(T, dtype=torch.int32, device="cuda:0")
    B.repq_ln_quant(x, block.ln1_g, block.ln1_b, c["eps"], block.ln1_s, block.ln1_z, ab, codes, sums, B.REPQ_NORM_RMS)
    qkv = torch.empty(T, 3 * D, dtype=block.act_dtype, device="cuda:0")
    block._gemm(T, codes, block.ln1_s, block.ln1_z, sums, block.qkv, 3 * D, D, qkv, out_scale=[1.0] * 3, out_zero=[0] * 3, out_kind=B.REPQ_OUT_BF16,
                rope=block.rope[:T].contiguous(), rope_period=T, rope_dim=D // H, rope_groups=2)
    for i, (cc, ss) in enumerate(((cache.layers[0].k_codes, cache.layers[0].k_scale), (cache.layers[0].v_codes, cache.layers[0].v_scale))):
        want = qkv[:, (1 + i) * D:(2 + i) * D].double().view(T, H, -1)
        pages = cache.table[0, :3].long()
        step = ss[pages].double().repeat_interleave(16, 0)[:T]
        got = ((cc[pages].double() - 128.0) * ss[pages].double()[:, :, None, None]).transpose(1, 2).reshape(48, H, -1)[:T]
        assert ((got - want).abs() <= 0.5001 * step[:, :, None]).all() and want.abs().max() > 0


def test_the_same_text_whole_in_chunks_and_token_by_token(model):
    """Quantized keys and values of a block of tokens depend on when its scale was found, so the three differ by rounding: a step of the
    cache is below 1 % of a channel's spread, and a log probability moves by a few of these."""
    ex, m = model
    text = np.random.default_rng(5).integers(0, m.vocab, 100).tolist()
    whole = ex.text_logprobs(m, text)
    spread = float(whole.std())
    assert spread > 0.5
    for chunk in (33, 7, 1):
        other = ex.text_logprobs(m, text, chunk)
        assert float((other - whole).abs().mean()) < 0.1 * spread


def test_the_first_layer_holds_the_same_whichever_way_a_text_came(model):
    """Keys and values of the first layer depend on a token and its position alone.  A block's final scale is that of its largest element, so
    it is the same every way; each of at most 16 growths re-rounds a code by half a (final) step at most, and most blocks grow a
    few times.  A wrong slot or position moves a value by some 30 steps."""
    import torch
    from paper_2402_05628_b200.serving import PagedCache
    ex, m = model
    block = m.blocks[0]
    D, H, T = block.cfg["D"], block.cfg["H"], 100
    x = torch.randn(T, D, device="cuda:0").to(block.act_dtype)

    def held(chunk):
        cache = PagedCache(1, 20, H, 16, D // H, 3, 112)
        for at in range(0, T, chunk):
            n = min(chunk, T - at)
            step = cache.plan([1, n, 0] if at % 2 else [0, n, 0])              # (another request's tokens come between)
            rows = torch.cat([x[:step.tokens - n], x[at:at + n]])
            block.forward_cached(rows, step, cache, 0)
        pages, t = cache.table[1, :7].long(), cache.layers[0]
        return [(c[pages].double().sub(128.0) * s[pages].double()[:, :, None, None], s[pages].double()[:, :, None, None])
                for c, s in ((t.k_codes, t.k_scale), (t.v_codes, t.v_scale))]
    whole = held(T)
    for chunk in (33, 7, 1):
        for (want, s), (got, s2) in zip(whole, held(chunk)):
            assert torch.equal(s, s2)
            steps = ((got - want).abs() / s).transpose(1, 2).reshape(112, -1)[:T]
            assert float(steps.max()) <= 9.0 and float(steps.mean()) <= 1.0


def test_requests_beside_each_other_and_one_after_the_other(model):
    ex, m = model
    rng = np.random.default_rng(6)
    prompts = [rng.integers(0, m.vocab, n).tolist() for n in (20, 1, 63)]
    together = ex.serve(m, prompts, 8, say=lambda s: None)
    for p, (tokens, logprobs) in zip(prompts, together):
        (alone, lp), = ex.serve(m, [p], 8, say=lambda s: None)
        # greedy choices may part where two tokens are as good; up to there both say the same
        same = 0
        while same < 8 and alone[same] == tokens[same]:
            same += 1
        assert same >= 1 and np.abs(np.array(lp[:same]) - np.array(logprobs[:same])).max() < 0.5


def test_blocks_go_back_and_the_pool_refuses(model):
    import torch
    from paper_2402_05628_b200.serving import PagedCache
    cache = PagedCache(1, 6, 1, 16, 16, 2, 80)
    a = cache.plan([40, 17])
    assert cache.free_blocks == 1
    with pytest.raises(MemoryError):
        cache.plan([9, 16])
    with pytest.raises(ValueError):
        cache.plan([50, 0])
    with pytest.raises(ValueError):
        cache.plan([1])
    cache.release(0)
    b = cache.plan([5, 48])
    assert b.slot_map.min() >= 0 and b.kv_lens.tolist() == [5, 65] and a.kv_lens.tolist() == [40, 17]
    held = cache.table[0, :1].tolist() + cache.table[1, :5].tolist()
    assert sorted(held) == list(range(6)) and cache.free_blocks == 0


def test_example_runs():
    import subprocess
    r = subprocess.run([sys.executable, os.path.join(ROOT, "examples", "serve_decoder.py"), "--steps", "4"], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "perplexity" in r.stdout, r.stdout + r.stderr
