"""The 4-bit cache format of the oracle against hand-worked values and against a search over all codes (no GPU)."""
import numpy as np
import pytest

from oracle import nova_fourbit as F


def _row(*vals):
    x = np.zeros(64)
    x[:len(vals)] = vals
    return x


def test_levels_ties_and_signs():
    # largest magnitude 6: scale 1; ties go to the level of even rank
    x = _row(6.0, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, -0.3, -5.1, 0.26, 0.0)
    codes, scales = F.quantise(x)
    assert scales[0] == 127
    assert F.values(codes, scales)[:12].tolist() == [6.0, 0.0, 1.0, 1.0, 2.0, 2.0, 4.0, 4.0, -0.5, -6.0, 0.5, 0.0]
    assert codes[0] == 0x07 and codes[1] == 0x22 and codes[4] == 0xf9      # even channel in the low nibble


@pytest.mark.parametrize("a,e", [(6.0, 0), (6.0001, 1), (12.0, 1), (3.0, -1), (3.0001, 0), (1.0, -2), (0.75, -3), (1e-38, -124),
                                 (0.0, -124), (3.0e38, 125)])
def test_scale_is_the_smallest_that_reaches(a, e):
    _, scales = F.quantise(_row(a))
    assert int(scales[0]) - 127 == e


def test_not_finite_groups_read_as_nan_and_leave_their_neighbours():
    for bad in (np.nan, np.inf, -np.inf):
        x = np.ones(64)
        x[3] = bad
        v = F.values(*F.quantise(x))
        assert np.isnan(v[:32]).all() and (v[32:] == 1.0).all()


def test_every_value_is_the_nearest_code():
    rng = np.random.default_rng(3)
    x = (rng.standard_normal((50, 64)) * np.exp(3 * rng.standard_normal((50, 1)))).astype(np.float32).astype(np.float64)
    codes, scales = F.quantise(x)
    v = F.values(codes, scales)
    step = np.repeat(np.exp2(scales.astype(np.float64) - 127), 32, -1)
    grid = np.concatenate([F.LEVELS, -F.LEVELS])
    assert np.array_equal(np.abs(v - x), np.abs(grid * step[..., None] - x[..., None]).min(-1))
    assert (np.abs(x).reshape(50, 2, 32).max(-1) <= 6 * np.exp2(scales.astype(np.float64) - 127)).all()
    assert (np.abs(x).reshape(50, 2, 32).max(-1) > 3 * np.exp2(scales.astype(np.float64) - 127)).all()


def test_values_are_stable():
    rng = np.random.default_rng(4)
    v = F.values(*F.quantise(rng.standard_normal((20, 128))))
    assert np.array_equal(F.values(*F.quantise(v)), v)


def test_attention_mass_is_one_per_query_and_head():
    rng = np.random.default_rng(5)
    K, V = (F.values(*F.quantise(rng.standard_normal((2, 2, 9, 64)))) for _ in range(2))
    q = rng.standard_normal((2, 3, 4, 64))
    out, lse, _, _ = F.attention(q, K, V, 0.125, [9, 0], [3, 3])
    assert (out[1] == 0).all() and np.isneginf(lse[1]).all()
    m, got = F.mass(q, K, 0.125, lse, None, [9, 0], [3, 3])
    assert np.isclose(got[0].sum(), 3 * 4) and (m[1] == -1).all()


def test_sums_that_are_no_numbers_add_nothing():
    rng = np.random.default_rng(6)
    K = F.values(*F.quantise(rng.standard_normal((2, 1, 5, 64))))
    q = rng.standard_normal((2, 3, 2, 64))
    _, lse, _, _ = F.attention(q, K, K, 0.125, [4, 5], [3, 3])
    q[0, 1, 0, 2] = lse[0, 1, 0] = np.nan
    m_in = np.array([[0.5, -1.0, np.inf, np.nan, 3.0], [0.0] * 5])
    m, got = F.mass(q, K, 0.125, lse, m_in, [4, 5], [3, 3])
    assert np.isnan(got[0, :4]).all() and m[0].tolist() == [0.5, 0.0, np.inf, 0.0, -1.0]
    assert np.isclose(m[1].sum(), 3 * 2)


def test_block_is_the_16_bit_block_on_the_same_rows():
    """On cached rows that are the block's own keys and values, not rounded, all variants give nova_oracle.pruned_block's result."""
    from oracle import nova_oracle as O
    rng = np.random.default_rng(7)
    B, N, C, heads, k, P, T = 2, 9, 64, 2, 4, 5, 3
    W = {n: 0.1 * rng.standard_normal(s) for n, s in dict(w_qkv=(3 * C, C), b_qkv=(3 * C,), w_o=(C, C), b_o=(C,), w_fc1=(4 * C, C),
                                                         b_fc1=(4 * C,), w_fc2=(C, 4 * C), b_fc2=(C,)).items()}
    x, kp, vp = (rng.standard_normal((B, m, C)) for m in (N, P, P))
    idx = np.stack([np.sort(rng.permutation(N)[:k]) for _ in range(B)])
    cross = {"w_cq": 0.1 * rng.standard_normal((C, C)), "b_cq": rng.standard_normal(C), "w_co": 0.1 * rng.standard_normal((C, C)),
             "b_co": rng.standard_normal(C), "k_text": rng.standard_normal((B, T, C)), "v_text": rng.standard_normal((B, T, C))}
    for kw in ({}, dict(gelu_form="tanh", ada=rng.standard_normal((B, 6, C))), dict(cross=cross),
               dict(qk_scale=np.array([3.0, 5.0]), gelu_form="tanh", ada=rng.standard_normal((B, 6, C)), cross=cross)):
        unit = (lambda t: O.unit_rows(t.reshape(B, -1, heads, C // heads)).reshape(t.shape)) if "qk_scale" in kw else (lambda t: t)
        prior = unit(kp)
        y, kn, vn = O.pruned_block(x, idx, W, prior, vp, heads, **kw)
        K, V = (np.concatenate(p, 1).reshape(B, P + k, heads, C // heads).transpose(0, 2, 1, 3) for p in ((prior, kn), (vp, vn)))
        y4, k4, v4, got = F.block(x, idx, W, K, V, heads, [P + k] * B, [k] * B, **kw)
        assert np.allclose(y4, y, atol=1e-12) and np.allclose(k4, kn, atol=1e-12) and np.allclose(v4, vn, atol=1e-12)
        assert np.isclose(got.sum(), B * heads * k)
