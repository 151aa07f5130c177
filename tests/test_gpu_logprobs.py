"""Log probabilities, entropy and top alternatives on the GPU against their plain form in 64 bits (oracle/tree.py).

Tolerances, u = 2^-24.  A weight w = 2^y, y = c (x - b), has a relative error of 3 u |y| ln 2 (difference, product, c) and 2 u (the power);
b is at most 8 below the largest y, so |y| is taken as 8 more than its distance from that.  A lane adds up to 32 weights a chunk, then its
chunks (V / 4096 where a workgroup has the row, fewer otherwise), then 8 joins with a scaling of 2 u each and up to 10 scalings on the way:
N u, N = V / 4096 + 60.  With p the probabilities, A1 = sum p |y| and A2 = sum p y^2:
  log S        (N + 2 + 3 ln 2 A1) u, and 4 u of its size for the logarithm
  U / S        (N + 5) A1 u + 3 ln 2 A2 u + A1 times the error of S
A result adds 2 u of each term that it is made of."""
import numpy as np
import pytest
import torch

from oracle import tree as ref

pytestmark = pytest.mark.gpu
DEV = "cuda"
u = 2.0 ** -24


@pytest.fixture(scope="module")
def osc():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2604_12782_amd as m
    m.lib()
    return m


def i32(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device=DEV)


def check(osc, X, tokens=None, k=0, scale=1.0, **kw):
    scale = float(np.float32(scale))
    lp, ids, top, lse, ent = osc.osc_token_logprobs(X, None if tokens is None else i32(tokens), k, scale, **kw)
    x = X.double().cpu().numpy()
    T, V = x.shape
    tok = np.zeros((T, 0), int) if tokens is None else np.asarray(tokens).reshape(T, -1)
    wlp, wids, wtop, wlse, went = ref.token_logprobs(x, tok, k, scale)
    most = 2.0 ** 128 - 2.0 ** 103  # what is further from 0 is infinity in single precision
    wlp, wtop, wlse = (np.where(w <= -most, -np.inf, w) for w in (wlp, wtop, wlse))
    N = V / 4096 + 60
    fine = ~(np.isnan(x).any(1) | np.isposinf(x).any(1) | np.isneginf(x).all(1))
    z = scale * np.where(fine[:, None], x, 0.0)
    m = z.max(1)
    with np.errstate(invalid="ignore"):
        y = np.where(np.isneginf(z), 0.0, (m[:, None] - z) / np.log(2) + 8)
    p = np.exp(z - m[:, None])
    p /= p.sum(1, keepdims=True)
    A1, A2 = (p * y).sum(1), (p * y * y).sum(1)
    logS = np.log(V) + 6
    eS = (N + 2 + 3 * np.log(2) * A1) * u + 4 * u * logS
    f = lambda t: t.double().cpu().numpy()
    near = lambda g, w, tol: (np.array_equal(np.isnan(g), np.isnan(w)) and np.array_equal(np.isneginf(g), np.isneginf(w))
                              and (np.abs(np.where(np.isfinite(w), g, 0) - np.where(np.isfinite(w), w, 0)) <= tol).all())
    assert near(f(lse), wlse, eS + 2 * u * (np.abs(m) + 6 + logS)), "lse"
    assert near(f(ent), went, eS + (N + 5) * A1 * u + 3 * np.log(2) * A2 * u + A1 * eS + 4 * u * (logS + A1)), "entropy"
    per_row = (eS + 2 * u * logS)[:, None]
    if tokens is not None:
        assert tuple(lp.shape) == np.asarray(tokens).shape
        assert near(f(lp).reshape(T, -1), wlp, per_row + 4 * u * (np.abs(np.where(np.isfinite(wlp), wlp, 0)) + logS)), "given"
    else:
        assert lp is None
    if k:
        assert np.array_equal(ids.cpu().numpy(), wids), "ids"
        assert near(f(top), wtop, per_row + 4 * u * (np.abs(np.where(np.isfinite(wtop), wtop, 0)) + logS)), "top"
    else:
        assert ids is None and top is None
    return lp, ids, top, lse, ent


def logits(seed, T, V, dtype, std=3.0, pad=0, shift=0):
    g = torch.Generator().manual_seed(seed)
    x = (torch.randn(T, V + pad, generator=g) * std).to(dtype)
    flat = torch.zeros(T * (V + pad) + shift, dtype=dtype, device=DEV)  # rows from any element on
    flat[shift:] = x.view(-1).to(DEV)
    return flat[shift:].view(T, V + pad)[:, :V]


DTYPES = [torch.float32, torch.bfloat16]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("V", [1, 2, 3, 7, 8, 9, 15, 63, 64, 65, 511, 1023, 1024, 1025, 4096, 4111, 10007, 50257])
def test_sizes(osc, V, dtype):
    gen = np.random.default_rng(V)
    for T in (1, 3, 19):
        for k in (0, 1, 5, 64):
            check(osc, logits(V + T, T, V, dtype), gen.integers(-1, V + 1, (T, 1 + k % 4)), min(k, V), scale=(1.0, 0.7, 2.5)[T % 3])


@pytest.mark.parametrize("dtype", DTYPES)
def test_alignment_and_strides(osc, dtype):
    for shift in range(9):
        for pad in (0, 1, 5, 8):
            check(osc, logits(shift, 5, 2001 + pad, dtype, pad=pad, shift=shift), [2000, 0, 1, 7, 1999], 9)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("T", [1, 2, 7, 100, 1100])
def test_parts_of_rows(osc, T, dtype):
    """rows in up to 64 parts, and in one"""
    V = 131075 if T < 100 else 9001
    x = logits(T, T, V, dtype)
    got = check(osc, x, np.arange(T) * 17 % V, 20)
    again = osc.osc_token_logprobs(x, i32(np.arange(T) * 17 % V), 20)
    assert all(torch.equal(a, b) for a, b in zip(got, again))


@pytest.mark.parametrize("dtype", DTYPES)
def test_ties(osc, dtype):
    """equal logits: the lowest tokens, wherever lanes, wavefronts and parts of the row meet"""
    for V in (5000, 70001):
        x = torch.zeros(5, V, dtype=dtype, device=DEV)
        x[1] = -2.5
        x[2, ::3] = 1.0
        x[3, V // 2:] = 4.0
        x[4, :] = 0.0
        x[4, ::2] = -0.0  # zeros are equal
        for k in (1, 33, 64):
            check(osc, x, [0, 1, 2, 3, V - 1], k)
    few = torch.randint(0, 3, (6, 40000), device=DEV, generator=torch.Generator(DEV).manual_seed(1)).to(dtype)
    check(osc, few, None, 50)


@pytest.mark.parametrize("dtype", DTYPES)
def test_order_of_the_values(osc, dtype):
    """rising and falling rows, where every chunk, or only the first, has the best; large and tiny distances"""
    V = 30000
    ramp = torch.linspace(-40, 40, V)
    x = torch.stack([ramp, ramp.flip(0), ramp.abs(), -ramp.abs(), ramp * 1e-6, ramp * 20, ramp * 0 + 1000]).to(dtype).to(DEV)
    for k in (1, 20, 64):
        check(osc, x, np.arange(7), k)
    check(osc, x, np.arange(7), 3, scale=1e-4)
    check(osc, x, np.arange(7), 3, scale=30.0)


@pytest.mark.parametrize("dtype", DTYPES)
def test_masked_logits(osc, dtype):
    """-infinity and the type's lowest value where no token may come; rows with one token, with none"""
    V = 20011
    low = torch.finfo(dtype).min
    for mask in (-float("inf"), low):
        x = logits(3, 9, V, dtype).clone()
        x[0, 5:] = mask
        x[1, :-1] = mask
        x[2] = mask
        x[3, 100:19000] = mask
        x[4, ::2] = mask
        x[5, :19999] = mask
        x[6, 7] = mask
        x[7] = mask
        x[7, 11], x[7, 12000] = 3.0, 3.0
        for k in (0, 3, 64):
            check(osc, x, [[0, 6, V - 1]] * 9, k)
        check(osc, x, [[0, 6, V - 1]] * 9, 3, scale=3.0)


@pytest.mark.parametrize("dtype", DTYPES)
def test_rows_that_are_not_finite(osc, dtype):
    """NaN or infinity anywhere makes its own row NaN and no other"""
    nan, inf = float("nan"), float("inf")
    for T, V in ((12, 6007), (1030, 300)):
        x = logits(5, T, V, dtype).clone()
        for row, (at, v) in enumerate(((0, nan), (V - 1, nan), (V // 2, -nan), (3, inf), (V - 2, inf), (100, nan))):
            x[row, at] = v
        x[6] = nan
        x[7, 5], x[7, 6] = inf, -inf
        x[8, :] = -inf
        x[8, 200] = nan
        lp, ids, top, lse, ent = check(osc, x, np.arange(T) % V, 7)
        assert torch.isnan(lse[:9]).all() and (ids[:9] == -1).all() and torch.isnan(top[:9]).all() and torch.isfinite(lse[9:]).all()


@pytest.mark.parametrize("dtype", DTYPES)
def test_sure_and_even_rows(osc, dtype):
    x = torch.zeros(4, 33000, dtype=dtype, device=DEV)
    x[0, 32999] = 60.0   # entropy 0
    x[2, 7] = 12.0
    x[3] = 3.0e4         # far from 0
    x[3, 100] = 3.1e4
    check(osc, x, [32999, 5, 7, 100], 2)


def test_out_tensors_and_workspace(osc):
    x = logits(1, 6, 40000, torch.bfloat16)
    tok = np.arange(12).reshape(6, 2)
    n = osc.osc_token_logprobs_workspace_bytes(6, 40000, 4)
    assert n > 0
    want = osc.osc_token_logprobs(x, i32(tok), 4)
    for fill in (0, 255, 127):
        out = [torch.full(t.shape, 7, dtype=t.dtype, device=DEV) for t in want]
        got = osc.osc_token_logprobs(x, i32(tok), 4, workspace=torch.full((n,), fill, dtype=torch.uint8, device=DEV), out=tuple(out))
        assert all(a is b for a, b in zip(got, out)) and all(torch.equal(a, b) for a, b in zip(got, want))
    lp, ids, top, lse, ent = osc.osc_token_logprobs(x, None, 0, out=(None, None, None, None, torch.empty(6, device=DEV)))
    assert lse is None and torch.equal(ent, want[4])
    assert osc.osc_token_logprobs(x[:0], i32(np.zeros((0, 3))), 4)[0].shape == (0, 3)


def test_many_given_tokens(osc):
    x = logits(2, 3, 5000, torch.float32)
    check(osc, x, np.arange(3 * 300).reshape(3, 300) * 5 - 9, 2)


def test_logits_past_32_bits(osc):
    """rows whose first element lies past 2^32 bytes"""
    x = torch.zeros(20, 128 * 2 ** 20 + 1, dtype=torch.bfloat16, device=DEV)
    x[19, 100 * 2 ** 20] = 20.0
    x[18, -1] = 20.0
    lp, ids, top, lse, ent = osc.osc_token_logprobs(x, i32([0] * 20), 2)
    assert ids[19].tolist() == [100 * 2 ** 20, 0] and ids[18].tolist() == [128 * 2 ** 20, 0] and ids[0].tolist() == [0, 1]
    V = x.shape[1]
    want = np.log(V - 1 + np.exp(20.0))
    # sums of 2^20 terms a lane at most, in single precision
    assert abs(lse[19].item() - want) < 1e-3 and abs(lse[0].item() - np.log(V)) < V / 4096 * u + 1e-5


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("T", [300, 700, 1100])
def test_many_long_rows(osc, T, dtype):
    """a workgroup a row, more chunks than a lane has marks: the same as of a few rows, which are checked above"""
    V = 280001 if T == 1100 else 66000
    x = logits(T, 8, V, dtype).repeat(-(-T // 8), 1)[:T]
    tok = i32(np.arange(T) % 8 * 1000)
    few, got = osc.osc_token_logprobs(x[:8].contiguous(), tok[:8], 20), osc.osc_token_logprobs(x, tok, 20)
    assert torch.equal(got[1], few[1].repeat(-(-T // 8), 1)[:T])
    for a, b in zip(got, few):
        if a.dtype == torch.float32:
            b = b.repeat(-(-T // 8), *[1] * (b.dim() - 1))[:T].double()
            assert ((a.double() - b).abs() <= 2 * (V / 4096 + 250) * u + 16 * u * b.abs()).all()
    check(osc, x[3:5], tok[3:5].cpu().numpy(), 20)


def test_more_rows_than_a_launch_has(osc):
    T, V = 2 ** 23 + 300, 4
    g = torch.Generator(device=DEV)
    g.manual_seed(5)
    X = torch.randint(-8, 9, (T, V), generator=g, device=DEV).bfloat16()
    tokens = torch.randint(0, V, (T,), generator=g, device=DEV).int()
    lp, ids, top, lse, entropy = osc.osc_token_logprobs(X, tokens, 2)
    rows = torch.cat([torch.arange(0, 200), torch.arange(2 ** 23 - 200, T)]).to(DEV)
    out = [torch.empty_like(v[rows]) for v in (lp, ids, top, lse, entropy)]
    osc.osc_token_logprobs(X[rows], tokens[rows], 2, out=out)
    for a, b in zip((lp, ids, top, lse, entropy), out):
        assert torch.equal(a[rows], b)
    check(osc, X[rows], tokens[rows].cpu().numpy(), 2)
    want = torch.log_softmax(X.double(), 1).gather(1, tokens.long()[:, None])[:, 0]
    # check()'s bound for V = 4 and logits 16 apart at most: A1 <= 32, 173 u a row and 99 u for the size of the result
    assert (lp - want).abs().max() <= 300 * u


def far_rows(V, dtype, scale):
    """rows of ordinary logits with fills at any distance, rows of large logits alone, rows on both sides of where c x is 2^20"""
    inf, low = float("inf"), torch.finfo(dtype).min
    rows, x = [], logits(8, 1, V, dtype)[0].clone()
    for fill in (-1e4, -1e9, -1e10, -1e12, -1e15, -1e20, -1e30, low, -inf):
        for i, part in enumerate((slice(5, None), slice(None, V - 1), slice(None), slice(100, V - 100), slice(None, None, 2), slice(None, V // 2), slice(V // 2, None), slice(7, 8))):
            r = x.roll(i)
            r[part] = fill
            rows.append(r)
        r = torch.full_like(x, fill)  # two tokens that can come
        r[[3, V // 2]] = 3.0
        rows.append(r)
    for v in (1e6, 1e9, 1e10, 1e15, 1e20, 1e30, 1e37):
        rows += [torch.full_like(x, v), torch.full_like(x, -v)]
        for a in (v, -v, 1.5 * v):
            r = x.clone()
            r[V // 3] = a
            rows.append(r)
        r = torch.full_like(x, -v)
        r[::3], r[1::5] = v, 0.0
        rows.append(r)
    line = 2.0 ** 20 * np.log(2) / scale
    for at in (line, -line):
        g = torch.Generator().manual_seed(int(scale * 10))
        near = (at + torch.randn(V, generator=g) * 2 / scale).to(dtype).to(DEV)
        rows += [near, torch.cat([near[:V // 2] * 1.25, near[V // 2:]]), torch.cat([near[:V // 2] * 0.75, near[V // 2:]]), torch.where(torch.arange(V, device=DEV) % 64 < 32, near, near * 0.999)]
    return torch.stack(rows)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("scale", [0.7, 1.0, 1.6, 3.0])
def test_far_logits(osc, dtype, scale):
    """logits are as good as their distance from the row's largest one, however far all of them are from 0: rows in parts, and of every number of wavefronts"""
    V = 33003
    x = far_rows(V, dtype, scale)
    tok = lambda n: [[0, 3, V // 2, V - 1]] * n
    check(osc, x, tok(len(x)), 5, scale=scale)
    for r in range(0, len(x), 12):
        check(osc, x[r:r + 12], tok(len(x[r:r + 12])), 5, scale=scale)
    x = far_rows(5001, dtype, scale)
    tok = [[0, 3, 2500, 5000]]
    for T in (300, 700, 1100):
        many = torch.cat([x, logits(T, T - len(x), 5001, dtype)])
        check(osc, many, tok * T, 64 if T == 700 else 0, scale=scale)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("scale", [1e-38, 0.01, 0.3, 0.5, 1.0, 2.0])
def test_distances_past_the_types_range(osc, dtype, scale):
    """logits further apart than the type's largest number: their log probabilities are numbers where scale makes them so"""
    x = logits(4, 6, 3001, dtype).clone()
    top = torch.finfo(dtype).max
    x[0, 5], x[0, 6] = 3e38, -3e38
    x[1, 5], x[1, 6] = top, -top
    x[2] = -top
    x[2, 9], x[2, 6] = 2e38, -1e38
    x[3, 5], x[3, 6] = 3e38, -float("inf")
    x[4, 6] = -top
    tok = i32([[0, 5, 6, 9]] * 6)
    past = scale * x.double().max(1).values >= 2.0 ** 128  # their lse is infinity in single precision: 2 * 2e38 and more
    assert past.any() == (scale == 2.0)
    for k in (0, 64):
        check(osc, x[~past], tok[~past].cpu().numpy(), k, scale=scale)
        lp, ids, top, lse, ent = osc.osc_token_logprobs(x, tok, k, scale)
        want = scale * (x.double() - x.double().max(1, keepdim=True).values)  # a single token: 0, and no other above -2^128
        assert torch.isposinf(lse[past]).all() and (ent[past] == 0).all()
        for got, at in ((lp, tok), (top, ids)) if k else ((lp, tok),):
            w = want.gather(1, at.long())[past]
            assert ((w == 0) | (w < -2.0 ** 128)).all() and torch.equal(got[past], torch.where(w == 0, 0.0, -float("inf")).float())
    if not past.any():
        check(osc, x[:2, 4:7], [[0, 1, 2]] * 2, 3, scale=scale)
