"""The paged 8-bit cache on the GPU: the plan of a step, the write, and attention over it, against plain implementations in numpy
(integers exactly, the quantizer in float32 as it is defined, attention in float64)."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

F32 = np.float32


@pytest.fixture(scope="module")
def B():
    from paper_2402_05628_b200.build import build_library
    build_library()
    from paper_2402_05628_b200 import binding
    return binding


def dev(a):
    import torch
    return torch.from_numpy(np.ascontiguousarray(a)).to("cuda:0")


def ints(a):
    return dev(np.asarray(list(a) if isinstance(a, range) else a, dtype=np.int32))


# ------------------------------------------------------------------------------------------------ plan

def plan_ref(kv, q, table, free, head, bs, slots):
    table, out, pos, cu, e, lost = table.copy(), [], [], [0], 0, 0
    width = table.shape[1]
    for b in range(len(kv)):
        old, new = -(-kv[b] // bs), -(-(kv[b] + q[b]) // bs)
        for j in range(old, new):
            if j >= width:
                lost += 1
                continue
            table[b, j] = free[head + e] if head + e < len(free) else -1
            lost += head + e >= len(free)
            e += 1
        for i in range(q[b]):
            p = kv[b] + i
            page = table[b, p // bs] if p // bs < width else -1
            out.append(page * bs + p % bs if page >= 0 else -1)
            pos.append(p)
        cu.append(cu[-1] + q[b])
    pad = lambda a: np.array((a + [-1] * slots)[:slots], dtype=np.int32)     # noqa: E731
    taken = min(e, len(free) - head)
    return dict(table=table, cu=cu, slot=pad(out), pos=pad(pos), kv=np.add(kv, q), head=head + taken,
                totals=[cu[-1], taken, lost, max(np.add(kv, q), default=0)])


def run_plan(B, kv, q, table, free, head, bs, slots, positions=True):
    import torch
    n = len(kv)
    t = ints(table)
    new = lambda m: torch.full((m,), 77, dtype=torch.int32, device="cuda:0")     # noqa: E731
    o = dict(kv=new(n), cu=new(n + 1), slot=new(slots), pos=new(slots), head=new(1), totals=new(4))
    B.repq_cache_plan(ints(kv), ints(q), t, ints(free), ints([head]), bs, kv_lens_out=o["kv"], cu_q=o["cu"], slot_map=o["slot"],
                      positions=o["pos"] if positions else None, free_head_out=o["head"], totals=o["totals"])
    return {k: v.cpu().numpy() for k, v in dict(o, table=t).items()}


@pytest.mark.parametrize("n,q_max,bs,slots", [(1, 1, 16, 1), (3, 40, 16, 200), (64, 1, 32, 64), (300, 129, 16, 9000), (1000, 3, 128, 5000),
                                              (600, 0, 64, 0), (2, 3000, 64, 4096)])
def test_plan(B, n, q_max, bs, slots):
    rng = np.random.default_rng(n + q_max)
    kv = rng.integers(0, 1000, n)
    kv[0] = 0
    kv[-1] = 3 * bs
    q = rng.integers(0, q_max + 1, n)
    width = int((kv + q).max() + bs - 1) // bs + 2
    old, need = -(-kv // bs), -(-(kv + q) // bs)
    pool = rng.permutation(int(need.sum()) + 50).astype(np.int32)
    table = np.full((n, width), -7, dtype=np.int32)
    at = 0
    for b in range(n):
        table[b, :old[b]] = pool[at:at + old[b]]
        at += old[b]
    free = pool[at:]
    got, ref = run_plan(B, kv, q, table, free, 5, bs, slots), plan_ref(kv, q, table, free, 5, bs, slots)
    for k in ref:
        assert np.array_equal(got[k].reshape(-1), np.asarray(ref[k]).reshape(-1)), k


@pytest.mark.parametrize("free,width", [(7, 40), (1, 40), (0, 40), (60, 5), (60, 0)])
def test_plan_out_of_blocks(B, free, width):
    """Blocks that the list or the table's rows do not hold: no entry is read or written past them, their tokens have no slot."""
    rng = np.random.default_rng(3)
    kv, q, bs = np.array([30, 0, 64, 5]), np.array([40, 33, 20, 0]), 16
    table = rng.integers(0, 100, (4, width)).astype(np.int32)
    args = (kv, q, table, np.arange(200, 200 + free, dtype=np.int32), 0, bs, 100)
    got, ref = run_plan(B, *args, positions=False), plan_ref(*args)
    ref["pos"] = np.full(100, 77)
    for k in ref:
        assert np.array_equal(got[k].reshape(-1), np.asarray(ref[k]).reshape(-1)), k


# ------------------------------------------------------------------------------------------------ write

def write_ref(codes, scales, x, slots):
    """The quantizer as it is defined, in float32: codes and scales of one of K, V after the rows x [tokens, heads, d_h]."""
    codes, scales = codes.copy(), scales.copy()
    bs = codes.shape[2]
    i = 0
    while i < len(slots):
        if slots[i] < 0 or slots[i] >= codes.shape[0] * bs:
            i += 1
            continue
        n = 1
        while i + n < len(slots) and slots[i + n] == slots[i] + n and slots[i + n] % bs:
            n += 1
        page, off = divmod(int(slots[i]), bs)
        rows = x[i:i + n].astype(F32)
        rows = np.where(np.isnan(rows), F32(0), rows)
        for h in range(x.shape[1]):
            a = np.minimum(np.abs(rows[:, h]).max(), np.finfo(F32).max)
            s = max(F32(a) * F32(1.0 / 127.0), F32(2.0 ** -60))
            if off:
                old = scales[page, h]
                s = max(s, old)
                c = codes[page, h, :off].astype(F32) - F32(128)
                codes[page, h, :off] = np.clip(np.rint(c * F32(old / s)), -127, 127) + 128
            scales[page, h] = s
            codes[page, h, off:off + n] = np.clip(np.rint(rows[:, h] / s), -127, 127) + 128
        i += n
    return codes, scales


def bf16(x):
    import torch
    return torch.from_numpy(np.asarray(x, dtype=F32)).to(torch.bfloat16)


def case_write(B, kv, q, bs, heads, dh, act, rng, mutate=None):
    import torch
    n, total = len(kv), int(np.sum(q))
    need = -(-(np.add(kv, q)) // bs)
    blocks = int(need.sum()) + 2
    pool = rng.permutation(blocks)
    slots, at = [], 0
    for b in range(n):
        pages = pool[at:at + need[b]]
        at += need[b]
        slots += [int(pages[p // bs]) * bs + p % bs for p in range(kv[b], kv[b] + q[b])]
    slots = np.array(slots, dtype=np.int32)
    if mutate is not None:
        slots = mutate(slots)
    x = (rng.standard_normal((total, 2 * heads + 1, dh)) * np.exp(rng.standard_normal((1, 2 * heads + 1, 1)))).astype(F32)
    x[rng.random(x.shape) < 0.002] = 30.0
    t = torch.from_numpy(x) if act == "f32" else bf16(x)
    g = t.to("cuda:0")
    x = t.float().numpy()
    codes = rng.integers(1, 256, (2, blocks, heads, bs, dh)).astype(np.uint8)
    scales = np.exp(rng.standard_normal((2, blocks, heads)) - 4).astype(F32)
    c = B.CacheTensors(dev(codes[0]), dev(codes[1]), dev(scales[0]), dev(scales[1]))
    B.repq_cache_write(c, g[:, :heads], g[:, heads + 1:], ints(slots))
    for i, (gc, gs) in enumerate(((c.k_codes, c.k_scale), (c.v_codes, c.v_scale))):
        rc, rs = write_ref(codes[i], scales[i], x[:, :heads] if i == 0 else x[:, heads + 1:], slots)
        assert np.array_equal(gs.cpu().numpy(), rs)
        assert np.array_equal(gc.cpu().numpy(), rc)


@pytest.mark.parametrize("act", ["bf16", "f32"])
@pytest.mark.parametrize("kv,q,bs,heads,dh", [
    ([0], [1], 16, 1, 16), ([15, 16, 17, 0], [1, 1, 1, 1], 16, 3, 64), ([5, 100, 0], [40, 0, 33], 16, 2, 128),
    ([3, 61], [300, 130], 64, 4, 128), ([100], [200], 128, 5, 80), ([7, 0], [50, 90], 32, 2, 48)])
def test_write(B, kv, q, bs, heads, dh, act):
    case_write(B, np.array(kv), np.array(q), bs, heads, dh, act, np.random.default_rng(len(kv) + dh))


def test_write_many_tokens(B):
    """Enough tokens that a CTA takes windows of them: runs that begin in one window and end in the next, single tokens among them."""
    rng = np.random.default_rng(8)
    q = np.array([500] + [1] * 200 + [777, 3, 64])
    case_write(B, rng.integers(0, 200, len(q)), q, 64, 8, 64, "bf16", rng)


def test_write_skips_tokens_without_a_slot(B):
    def holes(slots):
        slots = slots.copy()
        slots[16:23] = -1
        slots[23:32] = 1 << 30
        return slots
    case_write(B, np.array([0, 9, 4]), np.array([16, 16, 20]), 16, 2, 32, "f32", np.random.default_rng(2), holes)


def test_write_zeros_infinities_and_nan(B):
    import torch
    x = torch.zeros(2, 2, 16)
    x[0, 0, 3], x[0, 0, 4], x[0, 1, 5] = float("inf"), 1.0, float("nan")
    x[0, 1, 6], x[1, 0, 0] = -2.0, -float("inf")
    x = x.cuda()
    c = B.new_cache(3, 1, 16, 16)
    c.k_codes.fill_(9)
    B.repq_cache_write(c, x[:, :1], x[:, 1:], ints([16, 32]))
    big = np.finfo(F32).max * F32(1 / 127.)
    k, v = c.k_codes.cpu().numpy(), c.v_codes.cpu().numpy()
    assert c.k_scale.cpu().numpy()[:, 0].tolist() == [0, big, big] and c.v_scale.cpu().numpy()[1, 0] == F32(2) * F32(1 / 127.)
    assert k[1, 0, 0].tolist() == [128] * 3 + [255] + [128] * 12 and k[2, 0, 0].tolist() == [1] + [128] * 15
    assert v[1, 0, 0].tolist() == [128] * 6 + [1] + [128] * 9
    assert c.v_scale.cpu().numpy()[2, 0] == F32(2.0 ** -60) and set(v[2, 0, 0]) == {128}
    assert (k[0] == 9).all() and (k[1:, :, 1:] == 9).all()


# ------------------------------------------------------------------------------------------------ attention

class Case:
    """A cache filled with codes, tables, queries; and what attention over it is, in float64."""

    def __init__(self, kv, q, heads, kv_heads, dh, bs, act="bf16", seed=0, spread=0.3, peak=1.0):
        import torch
        rng = np.random.default_rng(seed)
        self.kv, self.q, self.bs, self.dh, self.group = np.array(kv), np.array(q), bs, dh, heads // kv_heads
        need = -(-self.kv // bs)
        self.blocks = int(need.sum()) + 3
        pool = rng.permutation(self.blocks)
        self.table = np.full((len(kv), int(need.max(initial=0)) + 2), -1, dtype=np.int32)
        at = 0
        used = np.zeros(self.blocks, dtype=bool)
        for b in range(len(kv)):
            self.table[b, :need[b]] = pool[at:at + need[b]]
            used[pool[at:at + need[b]]] = True
            at += need[b]
        self.codes = rng.integers(0, 256, (2, self.blocks, kv_heads, bs, dh)).astype(np.uint8)     # (slots that hold nothing: any byte)
        self.scales = (np.exp(spread * rng.standard_normal((2, self.blocks, kv_heads))) / 73.0).astype(F32)
        self.scales[:, ~used] = np.nan
        total = int(self.q.sum())
        x = (peak * rng.standard_normal((total + 1, heads + 3, dh))).astype(F32)
        t = torch.from_numpy(x) if act == "f32" else bf16(x)
        self.x = t.float().numpy()[:total, 1:1 + heads].astype(np.float64)
        self.gx = t.to("cuda:0")[:total, 1:1 + heads]
        self.cu = np.concatenate([[0], np.cumsum(self.q)])
        self.act, self.heads, self.alpha = act, heads, 1.0 / np.sqrt(dh)

    def reference(self, max_kv=None, chunks=False):
        """(out, lse, a bound on each element's error but for the output's rounding): weights of 11 bits and scores of float32, or 22 bits."""
        out, lse, tol, floor = np.zeros(self.x.shape), np.full(self.x.shape[:2], -np.inf), np.zeros(self.x.shape), np.zeros(self.x.shape)
        for b in range(len(self.kv)):
            L = int(self.kv[b]) if max_kv is None else min(int(self.kv[b]), max_kv)
            pages = self.table[b, :-(-L // self.bs)]
            there = np.repeat((pages >= 0) & (pages < self.blocks), self.bs)[:L]
            p = np.where((pages >= 0) & (pages < self.blocks), pages, 0)
            kk, vv = (((c[p].astype(np.float64) - 128) * s[p].astype(np.float64)[:, :, None, None]).transpose(1, 0, 2, 3).reshape(
                c.shape[1], -1, self.dh)[:, :L] for c, s in zip(self.codes, self.scales))
            for i in range(int(self.q[b])):
                r = self.cu[b] + i
                n = max(0, min(int(self.kv[b] - self.q[b]) + i + 1, L))
                on = there[:n]
                if not on.any():
                    continue
                for h in range(self.heads):
                    k, v = kk[h // self.group][:n][on], vv[h // self.group][:n][on]
                    s = self.alpha * k @ self.x[r, h]
                    m = s.max()
                    e = np.exp(s - m)
                    out[r, h] = e @ v / e.sum()
                    lse[r, h] = m + np.log(e.sum())
                    size = np.abs(v).T @ e / e.sum()                           # sum p |v|
                    terms = (self.alpha * np.abs(k) @ np.abs(self.x[r, h])).max()    # what a score is made of
                    wt = 2.0 ** -11 if self.act == "bf16" else 2.0 ** -21
                    tol[r, h] = size * (wt + 2.0 ** -20 * (4 + terms + abs(m)))
                    # chunks: weights under 2^-21 of the largest are multiples of 2^-31 of it at least
                    c = np.maximum(np.abs(v).max(1, initial=0), 1e-300)
                    floor[r, h] = 2.0 ** -32 * len(e) * 128 * (e * c / 64).max() / e.sum()
        return out, lse, tol + floor if chunks else tol

    def run(self, B, out=None, lse=None, max_q=None, max_kv=None, workspace=None, stream=None, **kw):
        import torch
        cache = B.CacheTensors(dev(self.codes[0]), dev(self.codes[1]), dev(self.scales[0]), dev(self.scales[1]))
        mq, mk = max_q if max_q is not None else int(self.q.max()), max_kv if max_kv is not None else int(self.kv.max())
        table = ints(self.table)
        n = B.repq_cache_attention_workspace_bytes(cache, self.gx, table, mq, mk)
        ws = torch.zeros(max(n, 16), dtype=torch.uint8, device="cuda:0") if workspace is None else workspace
        if out is None:
            out = torch.full(self.gx.shape, 7.0, dtype=self.gx.dtype, device="cuda:0")
        kv, cu = ints(self.kv), ints(self.cu)
        torch.cuda.synchronize()                       # (inputs made on the default stream)
        B.repq_cache_attention(cache, self.gx, table, kv, cu, out, ws, max_q_len=mq, max_kv_len=mk, alpha=self.alpha,
                               lse=lse, stream=stream, **kw)
        return out

    def check(self, B, chunks=False, **kw):
        import torch
        lse = torch.full(self.gx.shape[:2], 7.0, device="cuda:0")
        got = self.run(B, lse=lse, **kw).float().cpu().numpy().astype(np.float64)
        ref, ref_lse, tol = self.reference(kw.get("max_kv"), chunks)
        u = 2.0 ** -8 if self.act == "bf16" else 2.0 ** -24
        assert np.isfinite(got).all()
        worst = np.abs(got - ref) - (tol + u * np.abs(ref) + 1e-12)
        assert worst.max(initial=-1) <= 0, "off by %g where %g is allowed" % (np.abs(got - ref).max(), tol.max())
        fin = np.isfinite(ref_lse)
        gl = lse.cpu().numpy()
        assert np.array_equal(fin, np.isfinite(gl)) and (gl[~fin] == -np.inf).all()
        assert np.abs(gl[fin] - ref_lse[fin]).max(initial=0) <= 2.0 ** -18 * (8 + np.abs(ref_lse[fin]).max(initial=0) + (tol / 2 ** -20).max(initial=0))


@pytest.mark.parametrize("act", ["bf16", "f32"])
@pytest.mark.parametrize("dh", [16, 32, 48, 64, 80, 96, 112, 128])
def test_attention_widths(B, dh, act):
    Case([37, 1, 130], [1, 1, 2], 4, 2, dh, 16, act, seed=dh).check(B)


@pytest.mark.parametrize("act", ["bf16", "f32"])
@pytest.mark.parametrize("kv,q,heads,kv_heads,bs", [
    ([1], [1], 1, 1, 16),                                    # one key
    ([0, 5, 0], [1, 1, 0], 2, 1, 16),                        # a request that holds nothing, one that asks nothing
    ([64, 65, 63, 128], [1, 1, 1, 1], 8, 2, 64),             # the edges of a unit
    ([17], [17], 6, 6, 16), ([40], [13], 6, 2, 32),          # a prompt; a chunk with a group of three
    ([3, 50], [9, 4], 2, 2, 16),                             # more queries than tokens: the first rows see nothing
    ([777], [1], 32, 32, 16), ([1500, 2, 300], [1, 3, 2], 8, 8, 128),
    ([700, 90], [7, 5], 16, 2, 32),                          # groups of eight
])
def test_attention_lengths(B, kv, q, heads, kv_heads, bs, act):
    Case(kv, q, heads, kv_heads, 64, bs, act, seed=sum(kv)).check(B)


@pytest.mark.parametrize("act", ["bf16", "f32"])
def test_attention_long_axis_split_over_the_chip(B, act):
    Case([20000], [1], 4, 1, 128, 64, act, seed=5).check(B)


@pytest.mark.parametrize("act", ["bf16", "f32"])
def test_attention_prompts(B, act):
    Case([300, 129, 128, 1], [300, 129, 1, 1], 4, 2, 128, 32, act, seed=6).check(B)
    Case([700, 450], [200, 333], 3, 3, 64, 16, act, seed=7).check(B)


@pytest.mark.parametrize("dh", [16, 32, 48, 64, 80, 96, 112, 128])
def test_attention_chunk_widths(B, dh):
    Case([150, 260], [150, 130], 4, 2, dh, 16, seed=dh).check(B)


@pytest.mark.parametrize("kv,q,heads,kv_heads,dh,bs", [
    ([49], [49], 1, 1, 64, 16),                              # a few rows more than the kernel for few rows takes
    ([3000], [60], 2, 1, 128, 64),                           # one item, cut along the keys over all SMs
    ([700, 0, 1000, 64], [257, 0, 100, 64], 6, 2, 64, 32),   # groups of three: rows of a token in two tiles; requests of nothing
    ([900, 333, 5000, 2, 640], [200, 1, 1, 2, 129], 10, 2, 128, 16),   # chunks and single tokens in one call, groups of five
    ([130, 140], [140, 129], 2, 2, 128, 128),                # more queries than tokens: the first rows see nothing
    ([256] * 90, [64] * 90, 4, 4, 64, 16),                   # more items than SMs
    ([4000, 100], [1000, 100], 4, 1, 80, 64),
])
def test_attention_chunks(B, kv, q, heads, kv_heads, dh, bs):
    Case(kv, q, heads, kv_heads, dh, bs, seed=sum(q)).check(B)


@pytest.mark.parametrize("kv,q,heads,kv_heads,dh,bs", [([9000], [64], 2, 2, 64, 32), ([20000, 300], [50, 44], 2, 1, 128, 64)])
def test_attention_chunks_of_long_items_in_few_parts(B, kv, q, heads, kv_heads, dh, bs):
    Case(kv, q, heads, kv_heads, dh, bs, seed=sum(kv)).check(B)


def test_attention_chunks_rising_maxima(B):
    """Keys that matter more the later they come, by far: the running maximum moves within steps and between them."""
    c = Case([600], [200], 2, 2, 64, 32, seed=21)
    c.scales[0, c.table[0, :19], :] = (np.exp(0.35 * np.arange(19)) / 200.0)[:, None]
    c.check(B, chunks=True)
    d = Case([600], [200], 2, 2, 64, 32, seed=22)
    d.scales[1, d.table[0, :19], :] = (2.0 ** np.arange(-9, 10))[:, None]
    d.check(B, chunks=True)


def test_attention_chunks_repeat_bit_for_bit(B):
    import torch
    c = Case([3000, 50, 800], [300, 50, 1], 2, 1, 128, 64, seed=23)
    ws = torch.zeros(64 << 20, dtype=torch.uint8, device="cuda:0")
    first = c.run(B, workspace=ws)
    for _ in range(5):
        assert torch.equal(c.run(B, workspace=ws), first)
    assert B.repq_device_status() == 0


def test_attention_scales_of_every_size(B):
    """Blocks whose scales differ by many powers of two, and queries that look at few keys."""
    Case([500, 70], [2, 1], 4, 4, 64, 16, "bf16", seed=8, spread=6.0, peak=0.05).check(B)
    Case([500, 70], [2, 1], 4, 4, 64, 16, "f32", seed=9, spread=6.0, peak=0.05).check(B)
    Case([500, 300], [1, 40], 4, 4, 64, 32, "bf16", seed=9, spread=0.1, peak=20.0).check(B)


def test_attention_blocks_of_zeros(B):
    """A block that was written as zeros has the least scale: its keys count in the sum and add nothing."""
    for q in (1, 40):
        c = Case([100], [q], 2, 2, 32, 16, seed=10)
        c.codes[:, c.table[0, 1:4]] = 128
        c.scales[:, c.table[0, 1:4]] = F32(2.0 ** -60)
        c.check(B)


def test_attention_hides_tokens_of_missing_blocks(B):
    for q in (1, 50):
        c = Case([130, 60], [q, 1], 2, 1, 64, 16, seed=11)
        c.table[0, 2], c.table[0, 5], c.table[1, 0] = -1, 1 << 30, c.blocks
        c.check(B)


def test_attention_bound_on_the_keys(B):
    Case([300, 40], [3, 1], 4, 2, 64, 32, seed=12).check(B, max_kv=77)


def test_attention_code_outputs(B):
    import torch
    for bits, q in ((8, 3), (4 | 0x100, 3), (4, 3), (8, 70)):
        c = Case([90, 200], [q, 2], 4, 2, 64, 16, seed=13)
        ref, _, tol = c.reference()
        s, z, top = 0.01 if bits == 8 else 0.2, (128 if bits == 8 else 8), (255 if bits == 8 else 15)
        out = torch.zeros(c.gx.shape[0], 4, 32 if bits == 4 else 64, dtype=torch.uint8, device="cuda:0")
        sums = torch.full((c.gx.shape[0],), 5, dtype=torch.int32, device="cuda:0")
        got = c.run(B, out=out, out_bits=bits, out_scale=s, out_zero=z, out_row_sum=sums).cpu().numpy()
        if bits == 4:
            got = np.stack([got & 15, got >> 4], -1).reshape(got.shape[0], 4, 64)
        lo, hi = (np.clip(np.rint((ref + e * (tol + 1e-6)) / s) + z, 0, top) for e in (-1, 1))
        assert ((got >= lo) & (got <= hi)).all()
        assert np.array_equal(sums.cpu().numpy(), 5 + got.reshape(got.shape[0], -1).sum(1, dtype=np.int64))


def test_attention_strided_output_other_stream_and_one_workspace(B):
    import torch
    c = Case([513, 20, 300], [1, 1, 1], 8, 2, 128, 32, seed=14)
    first = c.run(B)
    st = torch.cuda.Stream()
    buf = torch.zeros(3, 10, 256, dtype=torch.bfloat16, device="cuda:0")
    ws = torch.zeros(64 << 20, dtype=torch.uint8, device="cuda:0")
    torch.cuda.synchronize()
    for _ in range(3):
        out = c.run(B, out=buf[:, 1:9, 128:], workspace=ws, stream=st)
    st.synchronize()
    assert torch.equal(out, first)                       # the same bits from call to call, whoever finishes last
    assert not buf[:, 0].any() and not buf[:, 9].any() and not buf[:, :, :128].any()


def test_cache_beyond_32_bit_offsets(B):
    """Write and attention at the far end of a cache of more than 4 GiB of codes for K and for V."""
    import torch
    blocks, heads, bs, dh = 9000, 32, 128, 128
    c = B.new_cache(blocks, heads, bs, dh)
    assert c.k_codes.numel() > 1 << 32
    g = torch.Generator(device="cuda:0").manual_seed(1)
    k, v, q = (torch.randn(200, heads, dh, device="cuda:0", generator=g).to(torch.bfloat16) for _ in range(3))
    pages = [blocks - 1, blocks - 2]
    slots = torch.tensor([pages[i // bs] * bs + i % bs for i in range(200)], dtype=torch.int32, device="cuda:0")
    B.repq_cache_write(c, k, v, slots)
    table, kv = ints([pages]), ints([200])
    small = B.new_cache(2, heads, bs, dh)
    B.repq_cache_write(small, k, v, ints(range(200)))
    for n in (1, 200):
        outs = []
        for cache, t in ((c, table), (small, ints([[0, 1]]))):
            ws = torch.zeros(B.repq_cache_attention_workspace_bytes(cache, q[:n], t, n, 200), dtype=torch.uint8, device="cuda:0")
            outs.append(torch.empty(n, heads, dh, dtype=torch.bfloat16, device="cuda:0"))
            B.repq_cache_attention(cache, q[200 - n:], t, kv, ints([0, n]), outs[-1], ws, max_q_len=n, max_kv_len=200, alpha=dh ** -0.5)
        assert torch.equal(*outs) and outs[0].float().abs().max() > 0
