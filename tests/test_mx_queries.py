"""Attention over the 4-bit cache where its queries are hard to hold: channels that are many times the others, results compared as ratios.

Tolerance, from the arithmetic, as a ratio of norms against 64 bits: softmax weights and the result are rounded to bf16, 0.0017 each on average, 0.0024 together.  A query
value is off by at most 2^-14 where the largest of its 32 is at least 3.875, 1.6e-5 of that one, and evenly spread; with channels of f times the others, that
one is about 1.3 f, so a score is off by 1.2e-5 f of the keys' size, 0.0012 at f = 100: 0.0027 in all.  The bound is 0.0035.
"""
import numpy as np
import pytest

from paper_2508_15919_amd.synth import bf16_bits_to_f64, f32_to_bf16_bits
from tests.test_mx_cache import Step, attend, dense, hb, place_tables, random_pool  # noqa: F401  (hb is a fixture)

BOUND = 0.0035


def off(got, want):
    return float(np.linalg.norm(got - want) / np.linalg.norm(want))


def steady_keys(step, pool, channels):
    """Every key gets the scale 2^-1 (which those of random_pool mostly have) and the value 1 (code 4 times the scale) in the channels: what queries have there
    moves all scores of a row alike."""
    D = step.d
    kb, ks, _, _, ke, _ = place_tables(D)
    pool[:, :, ke.ravel()] = 126
    for c in channels:
        for slot in range(16):
            at, sh = kb[slot, c], ks[slot, c]
            pool[:, :, at] = (pool[:, :, at] & (0xF0 if sh == 0 else 0x0F)) | (4 << sh)


@pytest.mark.gpu
@pytest.mark.parametrize("steady", [False, True])
@pytest.mark.parametrize("factor", [1, 8, 30, 64, 100])
@pytest.mark.parametrize("hq,hkv,d,q_len,ctx", [
    (8, 2, 128, [1, 40, 1], [2000, 1100, 90]),
    (8, 2, 64, [1, 1, 70], [1500, 333, 700]),
    (4, 1, 128, [150], [900]),                   # prompts alone
])
def test_queries_with_channels_of_many_times_the_others(hb, hq, hkv, d, q_len, ctx, factor, steady):
    step = Step(hb, hq, hkv, d, q_len, ctx, 300 + factor)
    pool = random_pool(step)
    channels = [32 * w + c for w in range(d // 32) for c in (5, 18)]
    if steady:
        steady_keys(step, pool, channels)
    q = step.g.standard_normal((step.tokens, hq, d))
    q[:, :, channels] *= factor
    q = f32_to_bf16_bits(q.astype(np.float32))
    got = bf16_bits_to_f64(attend(step, q, step.torch.from_numpy(pool).cuda()))
    found = off(got, dense(step, bf16_bits_to_f64(q), pool))
    print(f"{found:.5f} off")
    assert found <= BOUND


@pytest.mark.gpu
@pytest.mark.parametrize("hq,hkv,d,q_len,ctx", [
    (8, 2, 128, [1, 33, 1], [5000, 3001, 2999]),
    (4, 4, 64, [1, 1, 65], [4097, 1777, 2500]),
    (8, 1, 128, [1, 1, 1, 1], [6000, 16, 17, 1]),
    (8, 2, 64, [130], [3000]),
])
def test_long_contexts_as_a_ratio(hb, hq, hkv, d, q_len, ctx):
    """Results over thousands of keys are a fiftieth of a value: bounds in units of the values say little there."""
    step = Step(hb, hq, hkv, d, q_len, ctx, 350)
    pool = random_pool(step)
    q = step.bits(step.tokens, hq, d)
    got = bf16_bits_to_f64(attend(step, q, step.torch.from_numpy(pool).cuda()))
    found = off(got, dense(step, bf16_bits_to_f64(q), pool))
    print(f"{found:.5f} off")
    assert found <= BOUND


@pytest.mark.gpu
@pytest.mark.parametrize("hq,hkv,d,q_len,ctx", [
    (8, 2, 128, [1, 40, 1], [333, 1200, 90]),
    (8, 2, 64, [1, 33, 70], [40, 33, 700]),
    (4, 1, 128, [130], [900]),                   # prompts alone, an item's steps in two halves
    (8, 1, 128, [70, 1], [6000, 5000]),          # items split along the keys
    (4, 4, 64, [100], [100]),
])
def test_queries_that_are_not_finite_stay_by_themselves(hb, hq, hkv, d, q_len, ctx):
    """A head of a row with an infinity or a NaN gives NaN there, as over the bf16 pool; every other head and row keeps its bits.  (One whose scores overflow:
    nothing is said of it.)"""
    step = Step(hb, hq, hkv, d, q_len, ctx, 370)
    pool = step.torch.from_numpy(random_pool(step)).cuda()
    q = step.bits(step.tokens, hq, d)
    want = attend(step, q, pool)
    assert np.isfinite(bf16_bits_to_f64(want)).all()
    first = int(np.concatenate(([0], np.cumsum(q_len)))[np.argmax(q_len)])         # of the longest chunk
    bad = {(first, 0): 0x7FC0, (first + 5, 1): 0x7F80, (first + 21, 1): 0xFF80, (first + 20, 2): 0xFFFF, (first + 32, 3): 0x7F80}
    if first > 0:
        bad[0, 1] = 0x7FC0                                                         # a decode
    over = (first + 8, 2)
    for (row, head), bits in bad.items():
        q[row, head, (7 * row + head) % d] = bits
    q[over] = 0x7F7F
    got = attend(step, q, pool)
    others = np.ones((step.tokens, hq), bool)
    others[over] = False
    for at in bad:
        others[at] = False
        assert np.isnan(bf16_bits_to_f64(got[at])).all(), at
    assert np.array_equal(got[others], want[others]), np.argwhere((got != want).any(-1) & others).tolist()
