"""Scores of given tokens on the GPU against the fp64 oracle."""
import numpy as np
import pytest
import torch

from oracle.score import score_tokens
from paper_2605_23163_b200 import fdd

pytestmark = pytest.mark.gpu

# fp32 arithmetic on one row: t = (l - m) log2 e is rounded twice, 2^-23 |t|, which moves 2^t by 2^-23 |t| ln 2 of itself; under the
# distribution |t| is at most log2 V = 17.3 on the average, so the sum is off by 1.4e-6; the exponential (2 ulp) and the sums of eight add
# 2^-22 + 3 * 2^-24 = 4.2e-7.  The log-probability is off by that, and by roundings of itself; the entropy by |t| as much.
LOGPROB_ABS, ENTROPY_ABS, REL = 2e-6, 3.5e-5, 2.0 ** -22


@pytest.fixture(autouse=True)
def _need_cuda():
    assert torch.cuda.is_available()


def _score(logits, tokens, state=None, n_top=0, dtype="f32", entropy=True, offset=0):
    """logits: fp64 values that are numbers of the type."""
    rows, vocab = logits.shape
    ctx = fdd.fdd_create(4, 1, 64, vocab, 1, 0, 16, 1, fdd.FDD_LOGITS_F32 if dtype == "f32" else fdd.FDD_LOGITS_BF16)
    try:
        lg = torch.from_numpy(logits).to(torch.float32 if dtype == "f32" else torch.bfloat16).cuda()
        assert np.array_equal(lg.double().cpu().numpy(), logits, equal_nan=True)
        outs = [torch.full((rows,), 5.0, device="cuda"), torch.full((rows,), 5.0, device="cuda") if entropy else None,
                torch.full((rows, n_top), -9, dtype=torch.int32, device="cuda"), torch.full((rows, n_top), 5.0, device="cuda")]
        fdd.fdd_score_tokens(ctx, lg, torch.tensor(np.asarray(tokens), dtype=torch.int32, device="cuda"),
                             None if state is None else torch.tensor(np.asarray(state), dtype=torch.uint8, device="cuda"), n_top,
                             outs[0], outs[1], outs[2] if n_top else None, outs[3] if n_top else None)
        fdd.fdd_poll_status(ctx)
        return [None if t is None else t.cpu().numpy() for t in outs]
    finally:
        fdd.fdd_destroy(ctx)


def _check(logits, tokens, state=None, n_top=0, dtype="f32"):
    got = _score(logits, tokens, state, n_top, dtype)
    ref = score_tokens(logits, tokens, n_top, None if state is None else np.asarray(state) == fdd.FDD_COMMITTED)
    assert np.array_equal(got[2], ref["top_ids"])
    for mine, name, tol in ((got[0], "logprob", LOGPROB_ABS), (got[1], "entropy", ENTROPY_ABS), (got[3], "top_logprobs", LOGPROB_ABS)):
        r = ref[name]
        assert np.array_equal(np.isnan(mine), np.isnan(r)), name
        inf = np.isinf(r)
        assert np.array_equal(mine[inf], r[inf]), name
        at = np.isfinite(r)
        assert np.all(np.abs(mine[at] - r[at]) <= tol + REL * np.abs(r[at])), (name, np.max(np.abs(mine[at] - r[at])))
    return got


def _round(x, dtype):
    return torch.from_numpy(np.asarray(x)).to(torch.float32 if dtype == "f32" else torch.bfloat16).double().numpy()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,vocab,n_top", [
    (1, 1, 1), (3, 2, 2), (5, 7, 5), (2, 33, 32), (4, 97, 20), (3, 2047, 0), (9, 4096, 8), (1, 151936, 5), (22, 151936, 20),
    (37, 50257, 32), (200, 4099, 3), (700, 1001, 12),
])
def test_scores_of_given_tokens(rows, vocab, n_top, dtype):
    rng = np.random.default_rng(rows * 7 + vocab)
    x = rng.normal(size=(rows, vocab)) * rng.choice([0.5, 1.0, 3.0], size=(rows, 1))
    peak = rng.integers(0, vocab, size=rows)
    x[np.arange(rows), peak] += rng.choice([0.0, 5.0, 14.0], size=rows)
    tokens = np.where(rng.random(rows) < 0.5, peak, rng.integers(0, vocab, size=rows))
    _check(_round(x, dtype), tokens, None, n_top, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_without_a_committed_token_take_no_part(dtype):
    rng = np.random.default_rng(1)
    x = _round(rng.normal(size=(8, 1000)), dtype)
    x[2] = np.nan                                      # scaffold rows hold anything
    tokens = [0, -1, 5, 1000, 999, 7, 8, 2 ** 31 - 1]
    state = [1, 1, 2, 1, 1, 0, 3, 1]
    got = _check(x, tokens, state, 4, dtype)
    assert np.isfinite(got[0][[0, 4]]).all() and np.isnan(got[0][[1, 2, 3, 5, 6, 7]]).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("vocab", [1000, 20011])
def test_masked_ids_ties_and_values_that_are_not_finite(dtype, vocab):
    rng = np.random.default_rng(2)
    low = float(torch.finfo(torch.float32 if dtype == "f32" else torch.bfloat16).min)
    x = _round(rng.normal(size=(14, vocab)), dtype)
    x[0, 10:] = -np.inf                                # most ids masked
    x[1, 10:] = low
    x[2] = -np.inf                                     # nothing left
    x[3] = low                                         # nothing left, by the lowest value: uniform
    x[4, 77] = np.inf
    x[5, 78] = np.nan
    x[6] = np.nan
    x[7] = 1.5                                         # all equal
    x[8] = 0.0
    x[8, ::2] = -0.0                                   # equal too
    x[9, :-1] = -np.inf                                # one id left
    x[10, 500:] = x[10, 499]                           # a large tie
    x[11] = -low                                       # the largest value everywhere
    x[12, 1:] = -np.inf
    x[12, 0] = low
    x[13, :500] = -np.inf
    x[13, -1] = -low
    tokens = [3, 3, 3, 3, 3, 3, 3, 3, 3, vocab - 1, 3, 3, 0, vocab - 1]
    _check(x, tokens, None, 20, dtype)
    _check(x, [vocab - 1] * 14, None, 32, dtype)


@pytest.mark.parametrize("order", ["up", "down", "zigzag", "one thread", "steps"])
def test_the_likeliest_ids_in_rows_in_any_order(order):
    vocab = 30000
    v = np.arange(vocab, dtype=np.float64)
    if order == "up":
        x = v / 1000
    elif order == "down":
        x = -v / 1000
    elif order == "zigzag":
        x = np.where(v % 2 == 0, v, -v) / 1000
    elif order == "one thread":
        x = np.where((v.astype(int) // 4) % 256 == 17, 5 + v / 1e4, v / 1e5)
    else:
        x = np.floor(v / 5000)                         # long runs of equal logits, the highest last
    x = _round(np.stack([x] * 300), "f32")             # (enough rows for one CTA each, and once few for a cluster each)
    got = _check(x[:2], [5, 29999], None, 32)
    many = _score(x, [5] * 300, None, 32)
    assert np.array_equal(many[2], np.stack([got[2][0]] * 300))


def test_rows_far_into_a_large_array():
    # 3.0e9 logits: offsets of the last rows pass 32 bits, in elements as in bytes.  Few rows take part.
    vocab, rows = 151936, 20000
    rng = np.random.default_rng(7)
    ctx = fdd.fdd_create(4, 1, 64, vocab, 1, 0, 16, 1, fdd.FDD_LOGITS_BF16)
    try:
        lg = torch.zeros((rows, vocab), dtype=torch.bfloat16, device="cuda")
        at = [0, 7067, 14135, 14136, rows - 1]
        x = _round(rng.normal(size=(len(at), vocab)) * 2, "bf16")
        lg[torch.tensor(at, device="cuda")] = torch.from_numpy(x).to(torch.bfloat16).cuda()
        tokens = np.full(rows, -1, dtype=np.int32)
        tokens[at] = rng.integers(0, vocab, size=len(at))
        outs = [torch.zeros(rows, device="cuda") for _ in range(2)] + [torch.zeros((rows, 7), dtype=torch.int32, device="cuda"), torch.zeros((rows, 7), device="cuda")]
        fdd.fdd_score_tokens(ctx, lg, torch.from_numpy(tokens).cuda(), None, 7, *outs)
        fdd.fdd_poll_status(ctx)
        logprob, entropy, ids, likely = (t.cpu().numpy() for t in outs)
        ref = score_tokens(x, tokens[at], 7)
        assert np.array_equal(ids[at], ref["top_ids"])
        assert np.all(np.abs(logprob[at] - ref["logprob"]) <= LOGPROB_ABS + REL * np.abs(ref["logprob"]))
        assert np.all(np.abs(entropy[at] - ref["entropy"]) <= ENTROPY_ABS)
        others = np.ones(rows, dtype=bool)
        others[at] = False
        assert np.all(np.isnan(logprob[others])) and np.all(ids[others] == -1) and np.all(np.isnan(likely[others]))
    finally:
        fdd.fdd_destroy(ctx)


def test_the_same_bits_every_time_and_without_entropy():
    rng = np.random.default_rng(5)
    x = _round(rng.normal(size=(40, 40001)) * 2, "bf16")
    tokens = rng.integers(0, 40001, size=40)
    first = _score(x, tokens, None, 20, "bf16")
    again = _score(x, tokens, None, 20, "bf16", entropy=False)
    none = _score(x, tokens, None, 0, "bf16")
    assert np.array_equal(first[0], again[0]) and np.array_equal(first[2], again[2]) and np.array_equal(first[3], again[3])
    assert np.array_equal(first[0], none[0]) and np.array_equal(first[1], none[1])


def test_refusals():
    ctx = fdd.fdd_create(4, 1, 64, 10, 1, 0, 16, 1, fdd.FDD_LOGITS_F32)
    try:
        x, t = torch.zeros((2, 10), device="cuda"), torch.zeros(2, dtype=torch.int32, device="cuda")
        lp, ids, tl = torch.zeros(2, device="cuda"), torch.zeros((2, 40), dtype=torch.int32, device="cuda"), torch.zeros((2, 40), device="cuda")
        before = fdd.fdd_launch_count(ctx)
        for status, args in ((fdd.FDD_ERR_CAPACITY, (x, t, None, 33, lp, None, ids, tl)), (fdd.FDD_ERR_SHAPE, (x, t, None, 11, lp, None, ids, tl)),
                             (fdd.FDD_ERR_INVALID_ARG, (x, t, None, -1, lp, None, ids, tl)), (fdd.FDD_ERR_INVALID_ARG, (None, t, None, 1, lp, None, ids, tl)),
                             (fdd.FDD_ERR_INVALID_ARG, (x, t, None, 1, None, None, ids, tl)), (fdd.FDD_ERR_INVALID_ARG, (x, t, None, 1, lp, None, None, tl)),
                             (fdd.FDD_ERR_INVALID_ARG, (x, t, None, 1, lp, None, ids, None)), (fdd.FDD_ERR_INVALID_ARG, (x.data_ptr() + 4, t, None, 0, lp))):
            with pytest.raises(fdd.FddError) as e:
                fdd.fdd_score_tokens(ctx, *args)
            assert e.value.status == status, args[3]
        fdd.fdd_score_tokens(ctx, None, t[:0], None, 0, None)          # no rows: nothing to do
        assert fdd.fdd_launch_count(ctx) == before
    finally:
        fdd.fdd_destroy(ctx)


# Nearly certain rows.  With a peak `gap` nats above small logits that add up to S of it, the log-probability is -ln(1 + S) and the entropy
# about S (1 + gap).  The 16 bytes around the peak are masked but for itself (inside them a sum is plain fp32), so every small term counts:
# its t is off by 5 * 2^-24 of |t| <= 44 (difference, factor and constant, once in the pass and once where parts are moved), 9.1e-6 of the
# term; the exponentials add 2^-21 and the sums of small terms, at most 75 + 20 additions, 95 * 2^-24 = 5.7e-6, the product with t and the
# end 2^-21: 1.6e-5 in all.  A sum in one fp32 number would be off by 2^-24 of the peak a step, a tenth of S and more at 25 nats.
CERTAIN_REL = 3e-5


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows", [1, 30, 100])                          # eight, two and one CTA a row at the larger vocabulary
@pytest.mark.parametrize("vocab,gap", [(4096, 18.0), (151936, 18.0), (151936, 25.0), (151937, 29.5)])
def test_rows_that_are_nearly_certain(rows, vocab, gap, dtype):
    rng = np.random.default_rng(int(vocab + gap + rows))
    per_piece = 8 if dtype == "bf16" else 4
    logits = _round(rng.normal(size=(rows, vocab)) * 0.3, dtype)
    peak = rng.integers(0, vocab, size=rows)
    runner = np.empty(rows, dtype=np.int64)
    for r in range(rows):
        # the piece of a row begins at a multiple of 16 bytes of memory, the peak's is masked on both sides whatever that is
        lo, hi = max(0, peak[r] - per_piece + 1), min(vocab, peak[r] + per_piece)
        logits[r, lo:hi] = -np.inf
        logits[r, peak[r]] = gap
        # the likeliest of the rest: another piece of the same thread, a neighbour's, another CTA's
        at = (peak[r] + (256 * per_piece, 2 * per_piece, vocab // 2)[r % 3]) % vocab
        if lo <= at < hi:
            at = (hi + 2 * per_piece) % vocab
        runner[r] = at
        logits[r, at] = _round(np.array(gap - 12.0), dtype)
    tokens = np.where(np.arange(rows) % 4 == 3, runner, peak)
    got = _score(logits, tokens, None, 2, dtype)
    ref = score_tokens(logits, tokens, 2)
    assert np.array_equal(got[2], ref["top_ids"])
    assert np.all(got[0] <= 0.0) and np.all(got[1] >= 0.0) and np.all(got[3] <= 0.0)
    sure = tokens == peak
    assert np.all(np.abs(got[0][sure] - ref["logprob"][sure]) <= CERTAIN_REL * np.abs(ref["logprob"][sure]))
    assert np.all(np.abs(got[3][:, 0] - ref["top_logprobs"][:, 0]) <= CERTAIN_REL * np.abs(ref["top_logprobs"][:, 0]))
    assert np.all(np.abs(got[1] - ref["entropy"]) <= CERTAIN_REL * ref["entropy"])
    assert np.all(np.abs(got[0] - ref["logprob"]) <= LOGPROB_ABS + REL * np.abs(ref["logprob"]))
