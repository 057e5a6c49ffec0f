"""The statement of the 8-bit cache against closed forms and hand-made cases (CPU only), and the arithmetic its exactness rests on."""
import numpy as np
import pytest

import paper_2503_06433_amd as ss
import workloads as wl
from oracle import kv8


def test_a_block_of_whole_numbers_is_kept():
    x = np.arange(16 * 8).reshape(16, 8).astype(float) - 64
    x[3, 3] = 127
    q, a = kv8.quantise(x)
    assert a == 127 and np.array_equal(q, x)
    q, a = kv8.quantise(x * 2.0 ** -9)
    assert a == 127 * 2.0 ** -9 and np.array_equal(q, x)


def test_halves_go_to_even_and_zero_and_not_finite_blocks():
    x = np.zeros((16, 4))
    x[0] = [127, 0.5, 1.5, -2.5]
    assert np.array_equal(kv8.quantise(x)[0][0], [127, 0, 2, -2])
    assert kv8.quantise(np.zeros((16, 4)))[1] == 0 and not kv8.held_head(np.zeros((16, 4))).any()
    x[5, 1] = np.inf
    assert np.isnan(kv8.held_head(x)).all()


def test_a_block_is_off_by_half_a_step_at_most_and_again_not_at_all():
    x = np.random.default_rng(1).normal(size=(40, 3, 64))
    h = kv8.held(x)
    assert np.array_equal(h[32:], x[32:])
    for b in (0, 16):
        for g in range(3):
            a = np.abs(x[b:b + 16, g]).max()
            assert np.abs(h[b:b + 16, g] - x[b:b + 16, g]).max() <= a / 254 * (1 + 1e-12)
    np.testing.assert_allclose(kv8.held(h), h, rtol=1e-15)


@pytest.mark.parametrize("dtype", [wl.BF16, wl.F16])
def test_the_quotient_in_32_bits_rounds_as_in_real_arithmetic(dtype):
    """v * 127 / A of two numbers of at most 11 bits: v * 127 is exact in 24 bits, and a quotient that is not on half a step is
    off it by 1 / (2 mA) >= 2^-12 of A's whole mantissa mA < 2^11, against an error of 127 * 2^-24 < 2^-17."""
    rng = np.random.default_rng(2)
    vals = wl.quantize(rng.normal(size=(4000, 16)) * np.exp(rng.normal(size=(4000, 1))), dtype)[0]
    for v in vals:
        a = np.abs(v).max()
        lo = np.rint((v.astype(np.float32) * np.float32(127)) / np.float32(a))
        assert np.array_equal(lo, np.rint(v * 127 / a))


def test_kept_positions():
    w = np.array([3.0, 1.0, 3.0, 0.0, 3.0, 9.0, 0.0])
    assert list(kv8.kept_positions(w, 4, 1)) == [0, 2, 5, 6]            # equal weights: the earlier ones
    assert list(kv8.kept_positions(w, 3, 3)) == [4, 5, 6]
    assert list(kv8.kept_positions(w, 2, 5)) == [5, 6]                  # recent beyond what is kept
    assert list(kv8.kept_positions(w, 7, 0)) == list(range(7))
    w[3] = np.nan
    assert list(kv8.kept_positions(w, 2, 1)) == [3, 6]
    assert list(kv8.kept_positions(np.array([-0.0, 0.0, 0.0]), 1, 0)) == [0]


def test_attention_over_kept_tokens_is_attention_without_the_others():
    rng = np.random.default_rng(3)
    k, v, q = rng.normal(size=(20, 1, 8)), rng.normal(size=(20, 1, 8)), rng.normal(size=(1, 2, 8))
    out, _, w = kv8.attention(q, k, v, 19)
    assert np.allclose(w.sum(-1), 1)
    k2, v2, w2 = kv8.evict(127 * k, 127 * v, w.sum(1)[0][None], 9, 2)
    assert k2.shape == (9, 1, 8) and np.all(np.diff(kv8.kept_positions(w.sum(1)[0], 9, 2)) > 0)
    out2 = kv8.attention(q, k2, v2, 8)[0]
    assert np.abs(out2 - out).max() < np.abs(out).max()


def test_calls_without_a_context_are_refused():
    lib = ss.load_library()
    assert lib.ss_kv8_enable(None, None, None) == ss.SS_EINVAL
    assert lib.ss_kv8_write(None, None, 0, None, None, None) == ss.SS_EINVAL
    assert lib.ss_kv8_attn_prefill(None, None, 0, None, None, None, None) == ss.SS_EINVAL
    assert lib.ss_kv8_attn_decode(None, None, 0, None, None, None, None) == ss.SS_EINVAL
    assert lib.ss_kv8_weights(None, None, 0, None, 0, None, None) == ss.SS_EINVAL
    assert lib.ss_kv8_evict(None, None, None, None, 0, 0, None) == ss.SS_EINVAL
