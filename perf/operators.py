"""What serving and scoring with a quantized decoder is made of, operator by operator: the plan of a step (block tables, slot
maps), keys and values written into an 8-bit paged cache, attention over that cache, and log probabilities of tokens.

A case is a dict of plain values.  `prepare` makes the inputs from the seed, `run` is one pass: with `own` through the framework's
entry points, otherwise in elementary torch operations in float32.  Head layouts are those of this repository's LLaMA-7B-shaped and
DeiT-B-shaped blocks (32 heads of 128 channels, 12 of 64), the first also with 8 key / value heads; lengths, batches and the
vocabulary of 32000 are generic."""
import math

import torch

own = False

DEV = "cuda:0"
STEP = 1.0 / 127.0           # of a block's largest magnitude; float32 wherever it is used
LEAST_SCALE = 2.0 ** -60     # scale of a block of zeros


# ------------------------------------------------------------------------------------------------ the cases

def attention(name, requests, q_max, kv_max, heads, kv_heads, d_h, block, act="bf16", ragged=True):
    """q_max new tokens per request at most, kv_max tokens of a request in all; ragged: both spread over requests."""
    return dict(name=name, kind="attention", requests=requests, q_max=q_max, kv_max=kv_max, heads=heads, kv_heads=kv_heads,
                d_h=d_h, block=block, act=act, ragged=ragged)


def listed():
    return [
        # the plan of a decode step: 64 requests, a token each
        dict(name="plan_decode_64", kind="plan", requests=64, q_max=1, kv_max=4096, block=32),
        # the plan of a mixed step of a busy server: 300 requests, chunks among single tokens
        dict(name="plan_mixed_300", kind="plan", requests=300, q_max=129, kv_max=8192, block=16),
        # the cache write of a decode step, 32 heads of 128 channels
        dict(name="write_decode_64", kind="write", requests=64, q_max=1, kv_max=1024, kv_heads=32, d_h=128, block=16, act="bf16"),
        # the cache write of prompts
        dict(name="write_prompt_4x2048", kind="write", requests=4, q_max=2048, kv_max=2048, kv_heads=32, d_h=128, block=64, act="bf16"),
        # one user's next token over an ordinary prompt of an odd length: the smallest attention, where latency counts
        attention("attend_1x777", 1, 1, 777, 32, 32, 128, 16, ragged=False),
        # a decode batch, lengths of 1 to 4096, grouped heads
        attention("attend_64x4096_grouped", 64, 1, 4096, 32, 8, 128, 32),
        # two very long contexts: few rows, a long axis
        attention("attend_2x131072", 2, 1, 131072, 32, 8, 128, 64, ragged=False),
        # prompts of the LLaMA-7B-shaped layer: compute, the largest
        attention("attend_prompt_4x2048", 4, 2048, 2048, 32, 32, 128, 64, ragged=False),
        # chunks of prompts over what the cache already holds, with decode steps of other requests among them
        attention("attend_chunks_16x512", 16, 512, 4096, 32, 8, 128, 32),
        # float32 activations, 12 heads of 64 channels, a few tokens per request to verify
        attention("attend_f32_24x5", 24, 5, 2000, 12, 12, 64, 16, act="f32"),
        # scoring the tokens of a decode step: few rows
        dict(name="score_16x32000", kind="score", rows=16, vocab=32000, top=5, act="f32"),
        # scoring a text, as for perplexity: many rows
        dict(name="score_4096x32000", kind="score", rows=4096, vocab=32000, top=1, act="bf16"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["plan", "write", "write", "attention", "attention", "attention", "attention", "score", "score"])
    block = rng.choice([16, 16, 32, 64, 128])
    if kind == "plan":
        requests = _log(rng, 1, 512)
        return dict(kind="plan", requests=requests, q_max=rng.choice([1, _log(rng, 2, min(2048, 32768 // requests + 2))]),
                    kv_max=_log(rng, 2100, 16384), block=block)
    if kind == "score":
        vocab = rng.choice([32000, 32000, _log(rng, 1000, 131072)])
        return dict(kind="score", rows=_log(rng, 1, 4096 * 32000 // max(vocab, 32000)), vocab=vocab, top=rng.choice([0, 1, 5, 20]),
                    act=rng.choice(["f32", "bf16"]))
    heads, d_h = rng.choice([(32, 128), (32, 128), (12, 64), (16, 64)])
    kv_heads = rng.choice([h for h in (heads, heads, heads // 4, heads // 2, 4) if heads % h == 0])
    act = "f32" if rng.random() < 0.2 else "bf16"
    if kind == "write":
        requests = _log(rng, 1, 256)
        q_max = rng.choice([1, _log(rng, 2, max(2, min(2048, 8192 // requests)))])
        kv_max = max(q_max, _log(rng, 64, max(64, min(4096, 65536 // requests))))
        return dict(kind="write", requests=requests, q_max=q_max, kv_max=kv_max, kv_heads=kv_heads, d_h=d_h, block=block, act=act)
    if rng.random() < 0.6:                       # decode, a few tokens a request
        requests = _log(rng, 1, 128)
        q_max = rng.choice([1, 1, 1, rng.randint(2, 8)])
        kv_max = _log(rng, 16, 131072 * 2 // requests if act == "bf16" else 8192 * 8 // requests + 64)
        kv_max = min(kv_max, 131072 * 2 * 8 // (requests * kv_heads))
    else:                                        # chunks of prompts
        requests = _log(rng, 1, 16)
        q_max = _log(rng, 16, 2048 if act == "bf16" else 512)
        kv_max = max(q_max, _log(rng, 64, 4096))
        while requests > 1 and requests * q_max * kv_max > 4 * 2048 * 2048:
            requests -= 1
    case = attention("", requests, q_max, max(kv_max, q_max), heads, kv_heads, d_h, block, act, rng.random() < 0.7)
    del case["name"]
    return case


# ------------------------------------------------------------------------------------------------ inputs

def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(int(seed))


def _randn(g, *shape):
    return torch.randn(*shape, device=DEV, generator=g)


def _lengths(case):
    """(new tokens, tokens in all) per request, from the case alone: a program's sizes do not change with its data."""
    n, q_max, kv_max = case["requests"], case["q_max"], case["kv_max"]
    if not case.get("ragged", True):
        return [q_max] * n, [kv_max] * n
    h = torch.Generator().manual_seed(17 + n + 31 * q_max + 101 * kv_max)
    u, v = torch.rand(n, generator=h).tolist(), torch.rand(n, generator=h).tolist()
    if case["kind"] == "plan" and q_max > 1:      # most requests bring one token, some a chunk, some nothing
        q = [1 if a < 0.7 else 0 if a > 0.97 else 1 + int(b * (q_max - 1)) for a, b in zip(u, v)]
    elif q_max > 8 and n > 2:                     # half of them chunks, the others single tokens
        q = [1 if a < 0.5 else 1 + int(b * (q_max - 1)) for a, b in zip(u, v)]
        q[0] = q_max
    else:
        q = [q_max] * n
    kv = [a + int(b * (kv_max - a)) for a, b in zip(q, torch.rand(n, generator=h).tolist())]
    kv[-1] = max(kv_max, q[-1])
    return q, kv


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device=DEV)


def _tables(g, kv, block, spare):
    """Block tables of requests that hold kv tokens, blocks dealt out of a shuffled pool; the pool's other blocks are the free list."""
    need = [(n + block - 1) // block for n in kv]
    pool = torch.randperm(sum(need) + spare, device=DEV, generator=g).to(torch.int32)
    width = max(need) + 1
    n = torch.tensor(need, device=DEV)
    at = torch.cumsum(n, 0) - n
    col = torch.arange(width, device=DEV)
    table = torch.where(col < n[:, None], pool[(at[:, None] + col).clamp(max=pool.numel() - 1)], -1)
    return table.contiguous(), pool[sum(need):].contiguous(), pool.numel()


def prepare(case, seed):
    g = _gen(seed)
    kind = case["kind"]
    act = torch.float32 if case.get("act") == "f32" else torch.bfloat16
    if kind == "score":
        # logits of a language model: a few plausible tokens far above a bell-shaped rest; the given token is often one of them
        rows, vocab = case["rows"], case["vocab"]
        logits = torch.empty(rows, vocab, dtype=act, device=DEV)
        for r in range(0, rows, 1024):
            t = 2.0 * _randn(g, min(1024, rows - r), vocab)
            t.scatter_add_(1, torch.randint(0, vocab, (t.shape[0], 8), device=DEV, generator=g), 4.0 + 3.0 * _randn(g, t.shape[0], 8))
            logits[r:r + 1024] = t
        tokens = torch.where(torch.rand(rows, device=DEV, generator=g) < 0.7, logits.argmax(1),
                             torch.randint(0, vocab, (rows,), device=DEV, generator=g)).to(torch.int32)
        k = case["top"]
        out = [torch.empty(rows, device=DEV), torch.empty(rows, device=DEV), torch.empty(rows, dtype=torch.int32, device=DEV),
               torch.empty(rows, k, dtype=torch.int32, device=DEV), torch.empty(rows, k, device=DEV)]
        return dict(kind=kind, logits=logits, tokens=tokens, out=out, top=k)
    q, kv = _lengths(case)
    total, block = sum(q), case["block"]
    cu = _ints([0] + torch.tensor(q).cumsum(0).tolist())
    if kind == "plan":
        before = [a - b for a, b in zip(kv, q)]
        most = sum(-(-a // block) - -(-b // block) for a, b in zip(kv, before))
        table, free, _ = _tables(g, before, block, most + 64)
        table = torch.nn.functional.pad(table, (0, -(-case["kv_max"] // block) + 1 - table.shape[1] + 8), value=-1).contiguous()
        slots = (total + 63) // 64 * 64                  # the step's token budget
        n = case["requests"]
        new = lambda m: torch.zeros(m, dtype=torch.int32, device=DEV)      # noqa: E731
        return dict(kind=kind, before=_ints(before), q=_ints(q), table=table, free=free, head=_ints([3]), block=block,
                    out=[new(n), new(n + 1), new(slots), new(slots), new(1), new(4)])
    heads, kv_heads, d_h = case.get("heads", 0), case["kv_heads"], case["d_h"]
    table, _, blocks = _tables(g, kv, block, 4)
    # a fused projection's output: its query, key and value columns are strided views
    qkv = torch.empty(total, (heads + 2 * kv_heads) * d_h, dtype=act, device=DEV)
    for r in range(0, total, 4096):
        qkv[r:r + 4096] = _randn(g, min(4096, total - r), qkv.shape[1])
    codes, scales = [], []
    for _ in range(2):                                   # K, V: bell-shaped codes around 128, scales of real spread
        c = torch.empty(blocks, kv_heads, block, d_h, dtype=torch.uint8, device=DEV)
        for b in range(0, blocks, 512):
            c[b:b + 512] = (_randn(g, *c[b:b + 512].shape) * 36.0 + 128.0).round_().clamp_(1, 255)
        codes.append(c)
        scales.append(0.028 * torch.exp(0.25 * _randn(g, blocks, kv_heads)))
    if kind == "write":
        new = qkv.view(total, 2 * kv_heads, d_h)
        new *= torch.exp(0.5 * _randn(g, 2 * kv_heads, 1)).to(act)          # heads of different spread
        pos = torch.cat([torch.arange(b - a, b, device=DEV) for a, b in zip(q, kv)])
        req = torch.repeat_interleave(torch.arange(len(q), device=DEV), torch.tensor(q, device=DEV))
        slot = (table[req, pos // block].long() * block + pos % block).to(torch.int32)
        return dict(kind=kind, k=new[:, :kv_heads], v=new[:, kv_heads:], slot=slot, codes=codes, scales=scales, block=block)
    # queries whose rows look at few keys closely and at many a little
    x = qkv.view(total, heads + 2 * kv_heads, d_h)[:, :heads]
    x *= (0.5 + 1.5 * torch.rand(heads, 1, device=DEV, generator=g)).to(act)
    return dict(kind=kind, q=x, table=table, kv=_ints(kv), cu=cu, codes=codes, scales=scales, block=block, q_max=max(q), kv_max=max(kv),
                out=torch.empty(total, heads, d_h, dtype=act, device=DEV), alpha=1.0 / math.sqrt(d_h), keep=qkv, workspace=None)


# ------------------------------------------------------------------------------------------------ one pass

def run(state):
    if own:
        return _run_own(state)
    return {"plan": _plan, "write": _write, "attention": _attend, "score": _score}[state["kind"]](state)


def _run_own(s):
    from paper_2402_05628_b200 import binding as B
    kind = s["kind"]
    if kind == "plan":
        kv, cu, slot, pos, head, totals = s["out"]
        B.repq_cache_plan(s["before"], s["q"], s["table"], s["free"], s["head"], s["block"], kv_lens_out=kv, cu_q=cu, slot_map=slot,
                          positions=pos, free_head_out=head, totals=totals)
        return dict(table=s["table"], kv=kv, cu=cu, slot=slot, pos=pos, head=head, totals=totals)
    if kind == "score":
        logprob, entropy, rank, ids, tops = s["out"]
        B.repq_token_logprobs(s["logits"], s["tokens"], logprob, entropy=entropy, rank=rank, top_ids=ids, top_logprobs=tops)
        return dict(logprob=logprob, entropy=entropy, rank=rank, ids=ids, tops=tops)
    cache = B.CacheTensors(*s["codes"], *s["scales"])
    if kind == "write":
        B.repq_cache_write(cache, s["k"], s["v"], s["slot"])
        return dict(k=cache.k_codes, v=cache.v_codes, k_scale=cache.k_scale, v_scale=cache.v_scale)
    if s["workspace"] is None:                       # a program keeps its workspace from pass to pass
        n = B.repq_cache_attention_workspace_bytes(cache, s["q"], s["table"], s["q_max"], s["kv_max"])
        s["workspace"] = torch.zeros(max(n, 16), dtype=torch.uint8, device=DEV)
    B.repq_cache_attention(cache, s["q"], s["table"], s["kv"], s["cu"], s["out"], s["workspace"], max_q_len=s["q_max"],
                           max_kv_len=s["kv_max"], alpha=s["alpha"])
    return s["out"]


def _plan(s):
    before, q, table, free, head, bs = s["before"].long(), s["q"].long(), s["table"], s["free"], s["head"].long(), s["block"]
    kv = before + q
    old, new = (before + bs - 1) // bs, (kv + bs - 1) // bs
    first = torch.cumsum(new - old, 0) - (new - old)                        # of the free list, beyond its head
    col = torch.arange(table.shape[1], device=DEV)
    fresh = (col >= old[:, None]) & (col < new[:, None])
    table = torch.where(fresh, free[(head + first[:, None] + col - old[:, None]).clamp(0, free.numel() - 1)], table)
    cu = torch.cat([torch.zeros(1, dtype=torch.long, device=DEV), torch.cumsum(q, 0)])
    i = torch.arange(s["out"][2].numel(), device=DEV)
    req = (torch.searchsorted(cu, i, right=True) - 1).clamp(max=q.numel() - 1)
    there = i < cu[-1]
    pos = torch.where(there, before[req] + i - cu[req], -1)
    at = pos.clamp(min=0)
    slot = torch.where(there, table[req, (at // bs).clamp(max=table.shape[1] - 1)].long() * bs + at % bs, -1)
    taken = (new - old).sum()
    totals = torch.stack([cu[-1], taken, torch.zeros_like(taken), kv.max()])
    as_int = lambda t: t.to(torch.int32)      # noqa: E731
    return dict(table=table, kv=as_int(kv), cu=as_int(cu), slot=as_int(slot), pos=as_int(pos), head=as_int(head + taken), totals=as_int(totals))


def _write(s):
    bs = s["block"]
    slot = s["slot"].long()
    run_of, at = torch.unique_consecutive(slot // bs, return_inverse=True)   # the blocks that get rows, and each row's
    earlier = torch.full_like(run_of, bs).scatter_reduce_(0, at, slot % bs, "amin")
    had = (earlier > 0)[:, None]
    for x, codes, scales in ((s["k"], s["codes"][0], s["scales"][0]), (s["v"], s["codes"][1], s["scales"][1])):
        x = x.float()
        top = torch.zeros(run_of.numel(), x.shape[1], device=DEV).index_reduce_(0, at, x.abs().amax(-1), "amax")
        before = scales[run_of]
        step = torch.tensor(STEP, device=DEV)
        after = torch.maximum(torch.where(had, before, 0.0), (top * step).clamp(min=LEAST_SCALE))
        c = codes[run_of]
        kept = ((c.float() - 128.0) * (before / after)[:, :, None, None]).round().clamp(-127, 127) + 128.0
        old = (torch.arange(bs, device=DEV) < earlier[:, None])[:, None, :, None]
        codes[run_of] = torch.where(old & had[:, :, None, None], kept.to(torch.uint8), c)
        scales[run_of] = after
        codes[slot // bs, :, slot % bs] = ((x / after[at][:, :, None]).round().clamp(-127, 127) + 128.0).to(torch.uint8)
    return dict(k=s["codes"][0], v=s["codes"][1], k_scale=s["scales"][0], v_scale=s["scales"][1])


def _values(codes, scales, pages):
    """[requests, kv_heads, tokens, d_h] float32 of the pages of a table."""
    x = (codes[pages].float() - 128.0) * scales[pages][..., None, None]
    return x.transpose(1, 2).flatten(2, 3)


def _attend(s):
    q, cu, kv, bs = s["q"].float(), s["cu"].long(), s["kv"].long(), s["block"]
    n, (_, heads, d_h) = kv.numel(), q.shape
    q_len = cu[1:] - cu[:-1]
    pages = s["table"][:, :(s["kv_max"] + bs - 1) // bs].long().clamp(min=0)
    k, v = _values(s["codes"][0], s["scales"][0], pages), _values(s["codes"][1], s["scales"][1], pages)
    kv_heads = k.shape[1]
    i, j = torch.arange(s["q_max"], device=DEV), torch.arange(k.shape[2], device=DEV)
    at = (cu[:-1, None] + i).clamp(max=q.shape[0] - 1)
    x = q[at].view(n, s["q_max"], kv_heads, heads // kv_heads, d_h).permute(0, 2, 3, 1, 4).flatten(2, 3)
    scores = torch.matmul(x, k.transpose(2, 3)).view(n, kv_heads, -1, s["q_max"], j.numel())
    seen = j <= (kv - q_len)[:, None, None] + i[:, None]
    scores = scores.mul_(s["alpha"]).masked_fill_(~seen[:, None, None], float("-inf"))
    top = scores.amax(-1, keepdim=True)
    p = scores.sub_(torch.where(torch.isinf(top), 0.0, top)).exp_()
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p.flatten(2, 3), v).view(n, kv_heads, -1, s["q_max"], d_h) / torch.where(total > 0, total, 1.0)
    o = o.permute(0, 3, 1, 2, 4).reshape(n, s["q_max"], heads, d_h)
    t = torch.arange(q.shape[0], device=DEV)
    req = torch.searchsorted(cu, t, right=True) - 1
    return o[req, t - cu[req]].to(s["q"].dtype)


def _score(s):
    x, t = s["logits"].float(), s["tokens"].long()[:, None]
    top = x.amax(1, keepdim=True)
    e = (x - top).exp()
    z = e.sum(1, keepdim=True)
    lse = top + z.log()
    given = x.gather(1, t)
    entropy = z.log() - (e * (x - top)).sum(1, keepdim=True) / z
    at = torch.arange(x.shape[1], device=DEV)
    rank = 1 + ((x > given) | ((x == given) & (at < t))).sum(1)
    ids = torch.sort(x, dim=1, descending=True, stable=True).indices[:, :s["top"]] if s["top"] else t[:, :0]
    return dict(logprob=(given - lse)[:, 0], entropy=entropy[:, 0], rank=rank.to(torch.int32), ids=ids.to(torch.int32), tops=x.gather(1, ids) - lse)


# ------------------------------------------------------------------------------------------------ the same in 64 bits

def exact(case, seed):
    s = prepare(case, seed)
    kind = s["kind"]
    if kind == "plan":
        return None                                   # whole numbers
    if kind == "score":
        # row by row in groups, by the library's 64-bit log softmax
        lp, ent, tops = [], [], []
        for r in range(0, s["logits"].shape[0], 256):
            y = torch.log_softmax(s["logits"][r:r + 256].double(), 1)
            lp.append(y.gather(1, s["tokens"][r:r + 256].long()[:, None])[:, 0])
            ent.append(-(y.exp() * y).sum(1))
            tops.append(torch.topk(y, s["top"], dim=1).values)
        return dict(logprob=torch.cat(lp), entropy=torch.cat(ent), rank=None, ids=None, tops=torch.cat(tops))
    if kind == "write":
        # block by block over what the step brings: only the scales are numbers that 64 bits say more about
        out, bs = {}, s["block"]
        slot = s["slot"].tolist()
        starts = [i for i in range(len(slot)) if i == 0 or slot[i] // bs != slot[i - 1] // bs] + [len(slot)]
        for name, x, scales in (("k_scale", s["k"], s["scales"][0]), ("v_scale", s["v"], s["scales"][1])):
            big, now = x.double().abs().amax(-1).cpu(), scales.double().cpu()
            for a, b in zip(starts, starts[1:]):
                page = slot[a] // bs
                need = (big[a:b].amax(0) / 127.0).clamp(min=LEAST_SCALE)
                now[page] = torch.maximum(now[page], need) if slot[a] % bs else need
            out[name] = now
        return dict(k=None, v=None, **out)
    bs, cu, kv = s["block"], s["cu"].tolist(), s["kv"].tolist()
    heads = s["q"].shape[1]
    kv_heads, d_h = s["codes"][0].shape[1], s["codes"][0].shape[3]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEV)
    for b in range(len(kv)):
        lo, hi, L = cu[b], cu[b + 1], kv[b]
        if hi == lo or L == 0:
            continue
        pages = s["table"][b, :(L + bs - 1) // bs].long()
        hidden = torch.ones(hi - lo, L, dtype=torch.bool, device=DEV).triu(L - (hi - lo) + 1)
        for h in range(kv_heads):
            k, v = (((c[pages, h].double() - 128.0) * t[pages, h].double()[:, None, None]).reshape(-1, d_h)[:L] for c, t in zip(s["codes"], s["scales"]))
            for x in range(h * (heads // kv_heads), (h + 1) * (heads // kv_heads)):
                y = (s["q"][lo:hi, x].double() @ k.T * s["alpha"]).masked_fill(hidden, float("-inf"))
                out[lo:hi, x] = torch.softmax(y, -1) @ v
    return out


# ------------------------------------------------------------------------------------------------ what a pass needs

def work(case):
    kind = case["kind"]
    a = 4 if case.get("act") == "f32" else 2
    if kind == "score":
        n = case["rows"] * case["vocab"]
        return {"bytes": n * a + case["rows"] * (16 + 8 * case["top"]), "flops": 6.0 * n}
    q, kv = _lengths(case)
    total, n, bs = sum(q), case["requests"], case["block"]
    if kind == "plan":
        fresh = sum(-(-b // bs) - -(-(b - a_) // bs) for a_, b in zip(q, kv))
        return {"bytes": 16 * n + 8 * fresh + 8 * total, "flops": 4.0 * (n + total)}
    row = case["kv_heads"] * case["d_h"]
    if kind == "write":
        # rows in, codes out, scales of the blocks that get rows
        blocks = sum((b - 1) // bs - (b - a_) // bs + 1 for a_, b in zip(q, kv) if a_)
        return {"bytes": 2 * total * row * (a + 1) + 16 * blocks * case["kv_heads"] + 4 * total, "flops": 6.0 * total * row}
    # the keys that some row sees, once per key / value head; queries in, outputs out
    pairs = sum(a_ * (b - a_) + a_ * (a_ + 1) / 2 for a_, b in zip(q, kv))
    pages = sum(-(-b // bs) for b in kv)
    return {"bytes": 2 * sum(kv) * row + 8 * pages * case["kv_heads"] + 4 * pages + 2 * total * case["heads"] * case["d_h"] * a,
            "flops": 4.0 * case["d_h"] * case["heads"] * pairs}
