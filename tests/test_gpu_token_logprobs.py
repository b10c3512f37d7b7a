"""repq_token_logprobs against a plain float64 implementation: log probabilities, entropy, rank, top alternatives."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_2402_05628_b200.build import build_library
    build_library()
    from paper_2402_05628_b200 import binding
    return binding


def order(x):
    """Indices by (value descending, index ascending), NaN last."""
    key = np.where(np.isnan(x), -np.inf, x)
    return np.lexsort((np.arange(x.size), np.isnan(x), -key))


def reference(x, tokens, top):
    rows = []
    for r in range(x.shape[0]):
        o = order(x[r])
        t = int(tokens[r])
        if np.isnan(x[r]).any() or (x[r] == np.inf).any():
            lp = np.full(x.shape[1], np.nan)
            ent = np.nan
        elif (x[r] == -np.inf).all():
            lp, ent = np.full(x.shape[1], -np.inf), 0.0
        else:
            m = x[r].max()
            lp = x[r] - m - np.log(np.exp(x[r] - m).sum())
            p = np.exp(lp)
            ent = -(p[p > 0] * lp[p > 0]).sum()
        in_ = 0 <= t < x.shape[1]
        rows.append((lp[t] if in_ else 0.0, ent, int(np.where(o == t)[0][0]) + 1 if in_ else 0, o[:top], lp[o[:top]]))
    return [np.array(c) for c in zip(*rows)]


def check(B, x, tokens, top, ld=None, offset=0, stream=None):
    """x: float32 or bf16 CPU tensor [rows, vocab]."""
    import torch
    rows, vocab = x.shape
    buf = torch.full((rows, (ld or vocab) + offset), float("nan"), dtype=x.dtype, device="cuda:0")
    buf[:, offset:offset + vocab] = x.cuda()
    g = buf[:, offset:offset + vocab]
    new = lambda *s, d=torch.float32: torch.full(s, 99, dtype=d, device="cuda:0")     # noqa: E731
    lp, ent, rank, ids, tops = new(rows), new(rows), new(rows, d=torch.int32), new(rows, top, d=torch.int32), new(rows, top)
    B.repq_token_logprobs(g, torch.from_numpy(np.asarray(tokens, dtype=np.int32)).cuda(), lp, entropy=ent, rank=rank,
                          top_ids=ids if top else None, top_logprobs=tops if top else None)
    xd = x.double().numpy()
    r = reference(xd, tokens, top)
    finite = np.where(np.isfinite(xd), np.abs(xd), 0).max(1)
    # exponents are formed in float32 from logits and a maximum of that size, sums of float32 numbers in a few long chains
    tol = 2.0 ** -21 * (4 + finite) + 2.0 ** -20
    for got, ref in ((lp, r[0]), (ent, r[1])):
        got = got.cpu().numpy()
        assert np.array_equal(np.isnan(got), np.isnan(ref)) and np.array_equal(np.isinf(got), np.isinf(ref))
        ok = np.isfinite(ref)
        assert (np.abs(got - ref)[ok] <= (tol + 2.0 ** -22 * np.abs(np.where(ok, ref, 0)))[ok]).all()
    assert np.array_equal(rank.cpu().numpy(), r[2])
    if top:
        assert np.array_equal(ids.cpu().numpy(), r[3])
        got = tops.cpu().numpy()
        assert np.array_equal(np.isnan(got), np.isnan(r[4])) and np.array_equal(np.isinf(got), np.isinf(r[4]))
        ok = np.isfinite(r[4])
        assert (np.abs(got - r[4])[ok] <= (np.broadcast_to(tol[:, None], got.shape) + 2.0 ** -22 * np.abs(np.where(ok, r[4], 0)))[ok]).all()


@pytest.mark.parametrize("act", ["float32", "bfloat16"])
@pytest.mark.parametrize("rows,vocab,top", [(1, 1, 1), (1, 7, 3), (3, 1000, 0), (2, 1021, 32), (5, 32000, 5), (1, 131072, 20), (300, 4097, 2),
                                            (700, 513, 1)])
def test_token_logprobs(B, rows, vocab, top, act):
    import torch
    rng = np.random.default_rng(vocab)
    x = torch.from_numpy((3 * rng.standard_normal((rows, vocab))).astype(np.float32)).to(getattr(torch, act))
    tokens = rng.integers(0, vocab, rows)
    tokens[0] = int(x[0].float().argmax())
    check(B, x, tokens, top)


@pytest.mark.parametrize("act", ["float32", "bfloat16"])
def test_token_logprobs_strides(B, act):
    import torch
    rng = np.random.default_rng(1)
    x = torch.from_numpy(rng.standard_normal((4, 2500)).astype(np.float32)).to(getattr(torch, act))
    check(B, x, rng.integers(0, 2500, 4), 4, ld=2512)
    check(B, x, rng.integers(0, 2500, 4), 4, ld=2503, offset=1)


@pytest.mark.parametrize("rows", [3, 400])
def test_token_logprobs_ties_masks_and_padding(B, rows):
    """Equal logits go by index; masked ones (-inf, the type's lowest) have no probability; tokens outside the vocabulary are padding."""
    import torch
    rng = np.random.default_rng(rows)
    x = rng.integers(-3, 4, (rows, 3000)).astype(np.float32)      # hundreds of equal largest logits
    x[1] = 2.5
    x[2, :] = -np.inf
    x[2, [5, 2900]] = [1.0, 1.0]
    tokens = rng.integers(0, 3000, rows)
    tokens[:3] = [-1, 3000, 2900]
    check(B, torch.from_numpy(x), tokens, 8)
    y = x.copy()
    y[0, 10:] = np.finfo(np.float32).min
    y[1, :] = np.finfo(np.float32).min
    tokens[0] = 11
    check(B, torch.from_numpy(y), tokens, 3)


@pytest.mark.parametrize("act", ["float32", "bfloat16"])
@pytest.mark.parametrize("rows,vocab,top", [(1300, 600, 6), (1250, 1501, 1), (1201, 515, 0), (1300, 2048, 32)])
def test_token_logprobs_many_rows(B, rows, vocab, top, act):
    """Enough rows that each has few warps."""
    import torch
    rng = np.random.default_rng(vocab + top)
    x = (2 * rng.standard_normal((rows, vocab))).astype(np.float32)
    x[::7, rng.integers(0, vocab, vocab // 2)] = -np.inf
    x[3::11] = np.round(x[3::11])                                  # (many equal ones)
    tokens = rng.integers(0, vocab, rows)
    tokens[::5] = -1
    check(B, torch.from_numpy(x).to(getattr(torch, act)), tokens, top)


@pytest.mark.parametrize("act", ["float32", "bfloat16"])
@pytest.mark.parametrize("rows", [1, 320, 1200])
def test_token_logprobs_largest_far_apart(B, rows, act):
    """The largest logits lie at a power of two of elements from each other, so that they fall to few threads, or to one."""
    import torch
    rng = np.random.default_rng(rows)
    x = rng.standard_normal((rows, 8192)).astype(np.float32)
    for r in range(rows):
        step = (512, 1024, 2048)[r % 3]
        x[r, r % 16::step] += 20.0
    check(B, torch.from_numpy(x).to(getattr(torch, act)), rng.integers(0, 8192, rows), 12)


@pytest.mark.parametrize("rows", [5, 500])
def test_token_logprobs_rows_of_nothing_nan_and_infinity(B, rows):
    import torch
    rng = np.random.default_rng(7)
    x = rng.standard_normal((rows, 2048)).astype(np.float32)
    x[0] = -np.inf
    x[1, 7] = np.nan
    x[2, 2000] = np.inf
    x[3] = np.nan
    check(B, torch.from_numpy(x), rng.integers(0, 2048, rows), 6)


def test_token_logprobs_parts_alone(B):
    import torch
    x = torch.randn(4, 500, device="cuda:0")
    ent = torch.empty(4, device="cuda:0")
    B.repq_token_logprobs(x, None, entropy=ent)
    ids, tops = torch.empty(4, 2, dtype=torch.int32, device="cuda:0"), torch.empty(4, 2, device="cuda:0")
    B.repq_token_logprobs(x, None, top_ids=ids, top_logprobs=tops)
    y = torch.log_softmax(x.double(), 1)
    assert (ent - -(y.exp() * y).sum(1)).abs().max() < 1e-5 and torch.equal(ids.long(), y.topk(2).indices)
