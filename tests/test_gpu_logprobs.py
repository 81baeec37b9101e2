"""GPU: token log probabilities, entropy, top alternatives and the gradient of the logits, through the C ABI,
against the fp64 definition.

Tolerances.  U = 2^-24 is the rounding of fp32.  With t = scale (x - m), the difference and its product are
rounded, the constant log2 e is, and the exponential has two units in the last place: a relative error of (4 |t| +
8) U per term of S.  Weighted by the probabilities |t| averages to at most log V, and the sum is a chain of at
most V / 256 + 64 additions, so log S is off by at most U A with A = 4 log V + 72 + V / 256.  Then
    lse = scale m + log S:          U (A + 4 |scale m| + 2 |lse|)
    logprob, top = t - log S:       U (A + 4 |t| + 2 |value|)
    entropy = log S - E / S:        E has the same relative errors on terms that sum to at most (1 + log V) S:
                                    U 4 A (1 + log V)
    dlogits: t = scale x - lse is rounded at the size of its terms, which p takes as a relative error; with Q = 16 +
             4 (|scale x| + |lse| + |t|): U scale Q (p (|g| + |h| (1 + |t| + H)) + [token] |g|), then the rounding to
             the type, half a step: bf16 2^-8, fp32 2^-24 of the value.  Below 2^-126 p and the result are flushed to zero:
             2^-126 (1 + scale (|g| + |h| (1 + |t| + H)))."""
import math

import numpy as np
import pytest
import torch

from oracle import ops_oracle as oo
from paper_2602_01469_b200 import binding

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
U = 2.0 ** -24
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}
BF16, F32 = torch.bfloat16, torch.float32
INF = float("inf")


@pytest.fixture(scope="module")
def ctx():
    c = binding.Context(0)
    yield c
    c.close()


def put(x, pad=0, offset=0):
    """The rows of a host tensor in a longer device buffer: ``pad`` elements apart, ``offset`` in."""
    rows, cols = x.shape
    buf = torch.full((rows * (cols + pad) + offset,), 3.0, dtype=x.dtype, device=DEV)
    v = buf[offset:].view(rows, cols + pad)[:, :cols]
    v.copy_(x)
    return v


def forward(ctx, x, tokens, scale=1.0, k=0):
    rows = x.shape[0]
    nan = float("nan")
    out = [torch.full((rows,), nan, device=DEV) for _ in range(3)]
    top = torch.full((rows, k), nan, device=DEV) if k else None
    ids = torch.full((rows, k), -7, dtype=torch.int32, device=DEV) if k else None
    binding.peagle_token_logprobs_fwd(ctx, x, tokens, scale, out[0], out[1], out[2], top, ids)
    torch.cuda.synchronize()
    return out[0], out[1], out[2], top, ids


def near(got, want, bound):
    got = got.double().cpu().numpy()
    want = np.where(np.abs(want) > 3.4028235677973366e38, np.copysign(np.inf, want), want)   # past fp32's (and bf16's) range
    same = (np.isnan(got) & np.isnan(want)) | (np.isinf(want) & (got == want))
    with np.errstate(invalid="ignore"):
        bad = ~(same | (np.abs(got - want) <= bound))
    assert not bad.any(), (int(bad.sum()), np.argwhere(bad)[:4].tolist(), got[bad][:4], want[bad][:4])


def check_forward(x, tokens, scale, k, got):
    x64, tok = x.double().cpu().numpy(), tokens.cpu().numpy()
    lp, lse, H, top, ids = oo.token_logprobs(x64, tok, float(np.float32(scale)), k)
    V = x.shape[1]
    A = 4 * math.log(V) + 72 + V / 256
    with np.errstate(invalid="ignore", over="ignore"):
        m = np.nan_to_num(np.abs(x64.max(1) * scale), posinf=0.0)
        big = np.nan_to_num(np.abs(lse), posinf=0.0)
        near(got[1], lse, U * (A + 4 * m + 2 * big))
        away = lambda v: np.nan_to_num(np.abs(v), posinf=0.0)
        near(got[0], lp, U * (A + 4 * (away(lp) + math.log(V)) + 2 * away(lp)))
        near(got[2], H, np.full(len(tok), U * 4 * A * (1 + math.log(V))))
        if k:
            near(got[3], top, U * (A + 4 * (away(top) + math.log(V)) + 2 * away(top)))
            assert np.array_equal(got[4].cpu().numpy(), ids)


def check_backward(ctx, x, tokens, scale, lse, H, g, h, in_place=False):
    d = x.clone(memory_format=torch.preserve_format) if in_place else torch.full_like(x, float("nan"))
    want = oo.token_logprobs_bwd(x.double().cpu().numpy(), tokens.cpu().numpy(), float(np.float32(scale)), lse.double().cpu().numpy(),
                                 None if H is None else H.double().cpu().numpy(), None if g is None else g.cpu().numpy(),
                                 None if h is None else h.cpu().numpy())
    binding.peagle_token_logprobs_bwd(ctx, d if in_place else x, tokens, scale, lse, H, g, h, d)
    torch.cuda.synchronize()
    with np.errstate(invalid="ignore", over="ignore"):
        s = x.double().cpu().numpy() * scale
        L = lse.double().cpu().numpy()[:, None].copy()
        big = np.abs(L[:, 0]) >= 8192          # rows that are normalised again: differences to their maximum
        s[big] -= s[big].max(1, keepdims=True)
        L[big, 0] = np.log(np.exp(s[big]).sum(1))
        t = s - L
        p = np.exp(np.minimum(np.nan_to_num(t, nan=0.0), 1.0))
        fin = lambda v: np.nan_to_num(np.abs(v), posinf=0.0)
        Q = 16 + 4 * (fin(s) + fin(L) + fin(t))
        ga = np.zeros(x.shape[0]) if g is None else np.abs(g.double().cpu().numpy())
        ha = np.zeros(x.shape[0]) if h is None else np.abs(h.double().cpu().numpy())
        Ha = np.zeros(x.shape[0]) if H is None else fin(H.double().cpu().numpy())
        one = np.zeros_like(s)
        tok = tokens.cpu().numpy()
        rows = np.nonzero((tok >= 0) & (tok < x.shape[1]))[0]
        one[rows, tok[rows]] = 1.0
        factor = ga[:, None] + ha[:, None] * (1 + np.minimum(fin(t), 300.0) + Ha[:, None])
        bound = U * scale * Q * (p * factor + one * ga[:, None])
    near(d, want, HALF[x.dtype] * fin(want) + bound + 2.0 ** -126 * (1 + scale * factor))
    return d


CASES = [  # rows, vocab, type, k, scale, pad, offset
    (1, 1, BF16, 1, 1.0, 0, 0),
    (2, 5, F32, 5, 1.3, 0, 0),
    (3, 64, BF16, 64, 1.0, 0, 0),
    (40, 257, BF16, 7, 1.0, 3, 1),
    (700, 1000, BF16, 20, 0.7, 0, 0),
    (1, 128000, BF16, 20, 1.0, 0, 0),
    (2, 128000, F32, 64, 1.0, 0, 0),
    (9, 50001, BF16, 5, 0.7, 0, 5),
    (5, 50001, F32, 8, 1.0, 2, 1),
    (150, 32000, BF16, 3, 1.0, 8, 0),
    (400, 20000, BF16, 1, 1.0, 0, 0),
    (31, 8191, F32, 20, 2.0, 0, 3),
    (3, 262147, BF16, 20, 1.0, 0, 0),
]


@pytest.mark.parametrize("rows,vocab,dtype,k,scale,pad,offset", CASES)
def test_forward_and_backward_match_the_definition(ctx, rows, vocab, dtype, k, scale, pad, offset):
    gen = torch.Generator().manual_seed(rows * 7 + vocab)
    x = 2.5 * torch.randn(rows, vocab, generator=gen)
    peak = torch.randint(vocab, (rows,), generator=gen)
    x[torch.arange(rows), peak] += 9.0
    x = put(x.to(dtype), pad, offset)
    tokens = torch.where(torch.rand(rows, generator=gen) < 0.6, peak, torch.randint(vocab, (rows,), generator=gen))
    tokens[torch.rand(rows, generator=gen) < 0.2] = -1
    tokens = tokens.to(torch.int32).to(DEV)
    got = forward(ctx, x, tokens, scale, k)
    check_forward(x, tokens, scale, k, got)
    without = forward(ctx, x, tokens, scale, 0)
    for a, b in zip(got[:3], without[:3]):
        assert torch.allclose(a, b, rtol=1e-5, atol=1e-5)
    g, h = torch.randn(rows, generator=gen).to(DEV), torch.randn(rows, generator=gen).to(DEV)
    check_backward(ctx, x, tokens, scale, got[1], got[2], g, h)
    check_backward(ctx, x, tokens, scale, got[1], None, g, None)
    check_backward(ctx, x, tokens, scale, got[1], got[2], None, h)
    a = check_backward(ctx, x, tokens, scale, got[1], got[2], g, h, in_place=True)
    b = check_backward(ctx, x, tokens, scale, got[1], got[2], g, h)
    assert torch.equal(a, b)
    assert binding.peagle_poll_status(ctx) == 0


def special_rows(vocab, dtype):
    """Rows with masks, ties, orders and numbers where a maximum, a sum or a list of the best can go wrong."""
    gen = torch.Generator().manual_seed(vocab)
    low = torch.finfo(dtype).min
    rows = [torch.full((vocab,), v) for v in (-INF, low, 0.0, -7.5)]
    up = torch.linspace(-20, 20, vocab)
    rows += [up, up.flip(0)]                                       # every entry a new best, and the best first
    few = torch.randint(0, 3, (vocab,), generator=gen).float()     # three values only
    rows += [few, -few, torch.where(few > 0, 0.0, -0.0)]           # signs of zero
    for value in (-INF, low, -1e30, -1e9, -1e4):                   # masks that leave one, three, or half
        for left in (1, 3, vocab // 2):
            r = torch.full((vocab,), value)
            r[torch.randperm(vocab, generator=gen)[:left]] = torch.randn(left, generator=gen)
            rows.append(r)
    r = torch.full((vocab,), low)
    r[vocab // 3] = -INF
    rows.append(r)                                                 # the lowest number is not -inf
    r = torch.full((vocab,), -INF)
    r[vocab - 1] = low
    rows.append(r)
    r = torch.randn(vocab, generator=gen)
    r[vocab // 2] = 3e38
    rows.append(r)
    rows += [torch.full((vocab,), -1e30), torch.full((vocab,), -1e9), 1e6 + 64 * torch.randn(vocab, generator=gen)]
    for bad in (float("nan"), INF):
        for at in (0, vocab // 2, vocab - 1):
            r = torch.randn(vocab, generator=gen)
            r[at] = bad
            rows.append(r)
    r = torch.full((vocab,), -INF)
    r[1] = float("nan")
    rows.append(r)
    x = torch.stack(rows)
    x[4:6] = x[4:6] * 0.5
    return x.to(dtype)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("vocab,k,repeat", [(12, 12, 1), (1003, 20, 1), (20011, 64, 1), (70001, 20, 1), (5000, 20, 14)])
def test_rows_where_it_can_go_wrong(ctx, dtype, vocab, k, repeat):
    x = special_rows(vocab, dtype).repeat(repeat, 1)
    rows = x.shape[0]
    gen = torch.Generator().manual_seed(k)
    tokens = torch.randint(-1, vocab, (rows,), generator=gen).to(torch.int32).to(DEV)
    x = put(x, 0, 0)
    got = forward(ctx, x, tokens, 1.0, k)
    check_forward(x, tokens, 1.0, k, got)
    g, h = torch.randn(rows, generator=gen).to(DEV), torch.randn(rows, generator=gen).to(DEV)
    check_backward(ctx, x, tokens, 1.0, got[1], got[2], g, h)
    check_backward(ctx, x, tokens, 1.0, got[1], None, g, None)


def forward_without_entropy(ctx, x, tokens, scale, k):
    rows = x.shape[0]
    lp, lse = torch.full((rows,), float("nan"), device=DEV), torch.full((rows,), float("nan"), device=DEV)
    top = torch.full((rows, k), float("nan"), device=DEV) if k else None
    ids = torch.full((rows, k), -7, dtype=torch.int32, device=DEV) if k else None
    binding.peagle_token_logprobs_fwd(ctx, x, tokens, scale, lp, lse, None, top, ids)
    torch.cuda.synchronize()
    return lp, lse, top, ids


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("k", [0, 20])
@pytest.mark.parametrize("vocab,repeat", [(1003, 1), (20011, 1), (5000, 14)])
def test_rows_where_it_can_go_wrong_without_entropy(ctx, dtype, k, vocab, repeat):
    x = special_rows(vocab, dtype).repeat(repeat, 1)
    gen = torch.Generator().manual_seed(k + 1)
    tokens = torch.randint(-1, vocab, (x.shape[0],), generator=gen).to(torch.int32).to(DEV)
    x = put(x, 0, 0)
    lp, lse, top, ids = forward_without_entropy(ctx, x, tokens, 1.0, k)
    # the entropy's place is filled with the definition's: it is not asked for
    H = oo.token_logprobs(x.double().cpu().numpy(), tokens.cpu().numpy(), 1.0, k)[2]
    check_forward(x, tokens, 1.0, k, (lp, lse, torch.tensor(H, device=DEV), top, ids))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("k", [0, 20, 64])
@pytest.mark.parametrize("rows", [1, 4, 5])
def test_few_long_rows_in_every_form(ctx, dtype, k, rows):
    """Clusters of 16 blocks, or of 8: with entropy and without, with alternatives and without."""
    vocab = 70001
    gen = torch.Generator().manual_seed(rows)
    x = put((3 * torch.randn(rows, vocab, generator=gen)).to(dtype))
    tokens = torch.randint(-1, vocab, (rows,), generator=gen).to(torch.int32).to(DEV)
    got = forward(ctx, x, tokens, 1.0, k)
    check_forward(x, tokens, 1.0, k, got)
    lp, lse, top, ids = forward_without_entropy(ctx, x, tokens, 1.0, k)
    check_forward(x, tokens, 1.0, k, (lp, lse, got[2], top, ids))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("repeat", [1, 130]) # rows cut into parts, and whole ones
def test_rows_that_overflow_the_list_late(ctx, dtype, repeat):
    vocab, k = 20011, 20
    gen = torch.Generator().manual_seed(5)
    rows = []
    for at in (2048, 9000, 15000, 17500, vocab - 1100):
        for tail in (torch.linspace(10, 30, vocab - at), torch.full((vocab - at,), 12.0)):
            r = torch.randn(vocab, generator=gen)
            r[at:] = tail
            rows.append(r)
    x = torch.stack(rows).repeat(repeat, 1).to(dtype)
    tokens = torch.randint(-1, vocab, (x.shape[0],), generator=gen).to(torch.int32).to(DEV)
    x = put(x, 0, 0)
    check_forward(x, tokens, 0.9, k, forward(ctx, x, tokens, 0.9, k))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("k", [20, 64])
@pytest.mark.parametrize("repeat", [1, 50]) # rows cut into parts, and whole ones
def test_early_best_entries_survive_a_late_overflow(ctx, dtype, k, repeat):
    """Some of the k best come first and an ascending tail follows, which fills the list several times over within a
    chunk: the early ones are put back into the list while the chunk is gone through again."""
    vocab = 20011
    gen = torch.Generator().manual_seed(15)
    rows = []
    for early in (1, k // 2, k - 1, k):
        for at in (4096, 9000, 16500):
            r = torch.randn(vocab, generator=gen)
            r[at:] = torch.linspace(8, 40, vocab - at)
            where = torch.randperm(min(at, 4096), generator=gen)[:early]
            r[where] = 64.0 + 2.0 * torch.arange(early)
            rows.append(r)
    x = torch.stack(rows).repeat(repeat, 1).to(dtype)
    tokens = torch.randint(-1, vocab, (x.shape[0],), generator=gen).to(torch.int32).to(DEV)
    x = put(x, 0, 0)
    check_forward(x, tokens, 1.0, k, forward(ctx, x, tokens, 1.0, k))


def test_a_peaked_row_keeps_its_digits(ctx):
    """Large logits and a probability near one: neither logprob nor 1 - p is a difference of rounded numbers."""
    x = torch.full((2, 5000), 20.0)
    x[:, 77] = 40.0
    x = put(x)
    tokens = torch.tensor([77, 78], dtype=torch.int32, device=DEV)
    got = forward(ctx, x, tokens)
    want = -math.log1p(4999 * math.exp(-20.0))
    # S = 1 + 1.03e-5.  Once the largest term, 1, is in, every further addition rounds by up to U: at most 20 of
    # the thread's own (5,000 / 256) and 13 joins.  (A difference of numbers near 40 would be off by 64 U.)
    assert float(got[0][0]) == pytest.approx(want, rel=0, abs=33 * U)
    d = torch.empty_like(x)
    binding.peagle_token_logprobs_bwd(ctx, x, tokens, 1.0, got[1], None, torch.ones(2, device=DEV), None, d)
    # lse is the nearest fp32 number, 2^-19 of spacing at 40
    assert float(d[0, 77]) == pytest.approx(-math.expm1(40.0 - float(got[1][0])), rel=1e-5, abs=1e-12)


@pytest.mark.parametrize("step", [1.203125, 0.703125, 3.109375])
def test_long_rows_far_from_zero_keep_their_sums(ctx, step):
    """Rows of 2^21 entries around 100,000, which are summed again one by one: the sum of as many like terms stays as good
    as its terms.  A term is off by U (4 |t| + 8), |t| = step at most; logS, about 14, and what is formed with it are
    rounded: 64 U of logprob, and of a gradient, in which t = scale x - logS becomes relative, 128 U.  The entropy has
    log S and E / S, each to 64 U."""
    vocab = 1 << 21
    row = torch.full((vocab,), 100000.0)
    row[1::2] -= step
    row[3::8] -= step
    x = torch.stack((row, row.flip(0), row)).to(DEV)
    x[2] *= -1
    tokens = torch.tensor([0, 1, 3], dtype=torch.int32, device=DEV)
    lp, lse, H, top, ids = forward(ctx, x, tokens, 1.0, 2)
    want, _, wH, wtop, wids = oo.token_logprobs(x.double().cpu().numpy(), tokens.cpu().numpy(), 1.0, 2)
    assert np.array_equal(ids.cpu().numpy(), wids)
    near(lp, want, 64 * U * np.ones(3))
    near(top, wtop, 64 * U * np.ones((3, 2)))
    near(H, wH, 2 * 64 * U * np.ones(3))
    g = torch.tensor([1.0, -2.0, 0.5], device=DEV)
    d = torch.empty_like(x)
    binding.peagle_token_logprobs_bwd(ctx, x, tokens, 1.0, lse, None, g, None, d)
    w = oo.token_logprobs_bwd(x.double().cpu().numpy(), tokens.cpu().numpy(), 1.0, lse.double().cpu().numpy(), None, g.cpu().numpy(), None)
    near(d, w, 128 * U * np.abs(w))


def test_zero_gradients_skip_the_row(ctx):
    x = torch.full((3, 3001), float("nan"), dtype=BF16, device=DEV)
    x[1] = 1.0
    tokens = torch.tensor([5, 6, -1], dtype=torch.int32, device=DEV)
    lse = torch.tensor([1.0, math.log(3001.0) + 1.0, 1.0], device=DEV)
    g = torch.tensor([0.0, 2.0, 3.0], device=DEV)                  # no gradient; a gradient; no token
    d = torch.full_like(x, 9.0)
    binding.peagle_token_logprobs_bwd(ctx, x, tokens, 1.0, lse, None, g, None, d)
    assert float(d[0].float().abs().max()) == 0.0 and float(d[2].float().abs().max()) == 0.0
    assert float(d[1, 6]) == pytest.approx(2.0 * (1 - 1 / 3001), rel=2.0 ** -8)


def test_tokens_outside_the_vocabulary_are_reported(ctx):
    x = torch.randn(4, 100, device=DEV)
    tokens = torch.tensor([1, 100, -2, 5], dtype=torch.int32, device=DEV)
    got = forward(ctx, x, tokens, 1.0, 2)
    assert binding.peagle_poll_status(ctx) == binding.STATUS["BAD_META"]
    assert binding.peagle_poll_status(ctx) == 0
    check_forward(x, tokens, 1.0, 2, got)
    check_backward(ctx, x, tokens, 1.0, got[1], None, torch.ones(4, device=DEV), None)
    forward(ctx, x, torch.full((4,), 2 ** 31 - 1, dtype=torch.int32, device=DEV))
    assert binding.peagle_poll_status(ctx) == binding.STATUS["BAD_META"]


def test_tokens_outside_are_reported_whatever_is_asked_for(ctx):
    x = torch.randn(4, 100, device=DEV)
    lse, top, ids = torch.empty(4, device=DEV), torch.empty(4, 3, device=DEV), torch.empty(4, 3, dtype=torch.int32, device=DEV)
    good = torch.tensor([1, 99, -1, 5], dtype=torch.int32, device=DEV)
    for bad in (100, -2, -2 ** 31):
        tokens = torch.tensor([1, bad, -1, 5], dtype=torch.int32, device=DEV)
        for outputs in ((None, lse), (None, None, lse), (None, None, None, top, ids)):
            binding.peagle_token_logprobs_fwd(ctx, x, tokens, 1.0, *outputs)
            assert binding.peagle_poll_status(ctx) == binding.STATUS["BAD_META"]
            binding.peagle_token_logprobs_fwd(ctx, x, good, 1.0, *outputs)
            binding.peagle_token_logprobs_fwd(ctx, x, None, 1.0, *outputs)
            assert binding.peagle_poll_status(ctx) == 0


@pytest.mark.parametrize("scale", [1e-20, 1e-3, 50.0, 1e20])
def test_scales_far_from_one(ctx, scale):
    """Nearly uniform rows, rows with one token left, and logits that the scale takes past fp32's range."""
    x = special_rows(3001, BF16)
    tokens = torch.arange(x.shape[0], dtype=torch.int32) * 17 % 3001
    x, tokens = put(x), tokens.to(DEV)
    got = forward(ctx, x, tokens, scale, 6)
    s = x.float() * scale                                   # in fp32, as the definition has it
    none = torch.isnan(s).any(1) | (s == INF).any(1)
    empty = (s == -INF).all(1) & ~none
    assert torch.isnan(got[1][none]).all() and (got[4][none] == -1).all()
    assert (got[1][empty] == -INF).all() and (got[2][empty] == 0).all()
    rest = ~(none | empty)
    assert bool(rest.any())
    keep = rest.nonzero()[:, 0]
    check_forward(x[keep].clone(), tokens[keep], scale, 6, [None if t is None else t[keep] for t in got])


def test_no_rows(ctx):
    e, i = torch.empty(0, device=DEV), torch.empty(0, dtype=torch.int32, device=DEV)
    x = torch.empty(0, 70, dtype=BF16, device=DEV)
    binding.peagle_token_logprobs_fwd(ctx, x, i, 1.0, e, e, e, torch.empty(0, 3, device=DEV), i.view(0, 1).expand(0, 3).contiguous())
    binding.peagle_token_logprobs_bwd(ctx, x, i, 1.0, e, e, e, e, x.clone())
    torch.cuda.synchronize()


def test_outputs_are_optional_and_repeat(ctx):
    gen = torch.Generator().manual_seed(1)
    x = put(torch.randn(17, 9000, generator=gen).to(BF16))
    tokens = torch.randint(9000, (17,), generator=gen).to(torch.int32).to(DEV)
    one = forward(ctx, x, tokens, 1.0, 9)
    two = forward(ctx, x, tokens, 1.0, 9)
    for a, b in zip(one, two):
        assert torch.equal(a, b)
    ids, top = torch.empty(17, 9, dtype=torch.int32, device=DEV), torch.empty(17, 9, device=DEV)
    binding.peagle_token_logprobs_fwd(ctx, x, None, 1.0, None, None, None, top, ids)
    assert torch.equal(ids, one[4]) and torch.equal(top, one[3])
    lse = torch.empty(17, device=DEV)
    binding.peagle_token_logprobs_fwd(ctx, x, None, 1.0, None, lse)
    assert torch.allclose(lse, one[1], rtol=1e-6, atol=0)


def test_rows_past_two_to_the_31_elements(ctx):
    rows, ld = 2200, 1000003
    buf = torch.zeros(rows * ld, dtype=BF16, device=DEV)
    x = buf.view(rows, ld)[:, :300]
    x.copy_(torch.randn(rows, 300, device=DEV))
    tokens = torch.randint(300, (rows,), device=DEV).to(torch.int32)
    lp, lse = torch.empty(rows, device=DEV), torch.empty(rows, device=DEV)
    ids, top = torch.empty(rows, 4, dtype=torch.int32, device=DEV), torch.empty(rows, 4, device=DEV)
    binding.peagle_token_logprobs_fwd(ctx, x, tokens, 1.0, lp, lse, torch.empty_like(lp), top, ids)
    at = [0, 1, 2147, 2148, 2199]
    ent = torch.zeros(5, device=DEV)
    binding.peagle_token_logprobs_fwd(ctx, x[2195:], tokens[2195:], 1.0, None, None, ent)
    H = torch.distributions.Categorical(logits=x[at].double()).entropy().float()
    check_forward(x[at].clone(), tokens[at], 1.0, 4, (lp[at], lse[at], H, top[at], ids[at]))
    g, first = torch.ones(rows, device=DEV), x[at].clone()
    binding.peagle_token_logprobs_bwd(ctx, x, tokens, 1.0, lse, None, g, None, x)     # in place
    want = oo.token_logprobs_bwd(first.double().cpu().numpy(), tokens[at].cpu().numpy(), 1.0, lse[at].cpu().numpy(), None,
                                 np.ones(5), None)
    assert np.allclose(x[at].double().cpu().numpy(), want, rtol=2.0 ** -7, atol=1e-6)
    del buf, x


def test_entropies_past_two_to_the_31_elements(ctx):
    rows, ld = 2200, 1000003
    buf = torch.zeros(rows * ld, dtype=BF16, device=DEV)
    x = buf.view(rows, ld)[:, :300]
    x.copy_(torch.randn(rows, 300, device=DEV))
    tokens = torch.randint(300, (rows,), device=DEV).to(torch.int32)
    lp, lse, H, h = (torch.empty(rows, device=DEV) for _ in range(4))
    binding.peagle_token_logprobs_fwd(ctx, x, tokens, 1.0, lp, lse, H)
    binding.peagle_token_logprobs_fwd(ctx, x, tokens, 1.0, None, None, h)
    assert torch.equal(H, h)
    at = [0, 1, 2147, 2148, 2199]
    check_forward(x[at].clone(), tokens[at], 1.0, 0, (lp[at], lse[at], H[at], None, None))
    g, first = torch.randn(rows, device=DEV), x[at].clone()
    binding.peagle_token_logprobs_bwd(ctx, x, tokens, 1.0, lse, H, g, lp, x)     # in place
    torch.cuda.synchronize()
    want = torch.empty_like(first)
    binding.peagle_token_logprobs_bwd(ctx, first, tokens[at], 1.0, lse[at], H[at], g[at], lp[at], want)
    assert torch.equal(x[at], want)
    check_backward(ctx, first, tokens[at], 1.0, lse[at], H[at], g[at], lp[at])
    del buf, x


def test_in_a_captured_graph(ctx):
    gen = torch.Generator().manual_seed(3)
    x = put(torch.randn(6, 30000, generator=gen).to(BF16))
    tokens = torch.randint(30000, (6,), generator=gen).to(torch.int32).to(DEV)
    lp, lse, H = (torch.zeros(6, device=DEV) for _ in range(3))
    ids, top = torch.zeros(6, 5, dtype=torch.int32, device=DEV), torch.zeros(6, 5, device=DEV)
    d = torch.zeros_like(x)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        binding.peagle_token_logprobs_fwd(ctx, x, tokens, 1.0, lp, lse, H, top, ids)
        binding.peagle_token_logprobs_bwd(ctx, x, tokens, 1.0, lse, H, lp, H, d)
    for _ in range(2):
        x.copy_(torch.randn(6, 30000, generator=gen).to(BF16))
        tokens.copy_(torch.randint(30000, (6,), generator=gen).to(torch.int32))
        g.replay()
        torch.cuda.synchronize()
        check_forward(x, tokens, 1.0, 5, (lp, lse, H, top, ids))
        e = torch.empty_like(d)
        binding.peagle_token_logprobs_bwd(ctx, x, tokens, 1.0, lse, H, lp, H, e)
        assert torch.equal(d, e)


def test_binding_refuses(ctx):
    x = torch.zeros(3, 50, dtype=BF16, device=DEV)
    tok = torch.zeros(3, dtype=torch.int32, device=DEV)
    f = torch.zeros(3, device=DEV)

    def refused(status, call, *args):
        with pytest.raises(binding.PeagleError) as e:
            call(ctx, *args)
        assert e.value.status == binding.STATUS[status]

    fwd, bwd = binding.peagle_token_logprobs_fwd, binding.peagle_token_logprobs_bwd
    ids = torch.zeros(3, 4, dtype=torch.int32, device=DEV)
    refused("BAD_SHAPE", fwd, x, tok.long(), 1.0, f)
    refused("BAD_SHAPE", fwd, x, tok[:2], 1.0, f)
    refused("BAD_SHAPE", fwd, x.half(), tok, 1.0, f)
    refused("BAD_SHAPE", fwd, x, tok, 0.0, f)
    refused("BAD_SHAPE", fwd, x, tok, 1.0, f.double())
    refused("BAD_SHAPE", fwd, x.t(), tok, 1.0, f)
    refused("BAD_SHAPE", fwd, x.cpu(), tok, 1.0, f)
    refused("BAD_SHAPE", fwd, x, tok, 1.0, f, None, None, None, ids)
    refused("BAD_SHAPE", fwd, x, tok, 1.0, f, None, None, torch.zeros(3, 5, device=DEV), ids)
    refused("BAD_SHAPE", fwd, x, tok, 1.0, f, None, None, torch.zeros(3, 8, device=DEV)[:, ::2], ids)
    refused("NULL", fwd, x, None, 1.0, f)
    refused("NULL", bwd, x, tok, 1.0, None, None, f, None, x.clone())
    refused("NULL", bwd, x, tok, 1.0, f, None, None, f, x.clone())
    refused("BAD_SHAPE", bwd, x, tok, 1.0, f, None, f, None, x.float())
