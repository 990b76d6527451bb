"""Pins of the plain cache model the GPU tests compare with (no GPU)."""
import numpy as np
import pytest

import kv_ref as ref
from paper_2505_13204_b200 import binding


@pytest.mark.parametrize("D", [64, 128, 256])
def test_head_bytes_of_the_library_and_of_the_model_agree(D):
    assert binding.kv_head_bytes(D) == ref.head_bytes(D)


def test_head_dim_the_kernels_do_not_have_is_refused():
    with pytest.raises(binding.AasdError) as e:
        binding.kv_head_bytes(96)
    assert e.value.code == binding.ERR_UNSUPPORTED


def test_plan_by_hand():
    # seq 0 ends, seq 1 crosses a page boundary, seq 2 wants more than is left, seq 3 has room already
    table, held, stack = [[5, 6], [1], [2], [3]], [2, 1, 1, 1], [7]
    got = ref.plan([0, 64, 60, 10], [0, 3, 200, 5], table, held, stack, 4, 0, 208)
    assert table == [[], [1, 6], [2], [3]] and stack == [7, 5] and held == [0, 2, 1, 1]
    assert got["kv_len"].tolist() == [0, 67, 60, 15] and got["full"]
    assert got["tok_offsets"].tolist() == [0, 0, 3, 203, 208]
    assert got["slot_map"][:3].tolist() == [6 * 64, 6 * 64 + 1, 6 * 64 + 2]
    assert (got["slot_map"][3:203] == -1).all() and got["slot_map"][203] == 3 * 64 + 10
    assert got["positions"][203:].tolist() == [10, 11, 12, 13, 14]


def test_quantised_rows_stay_within_half_a_step_and_bad_rows_become_zeros():
    rng = np.random.default_rng(0)
    x = (rng.standard_normal((50, 128)) * 10.0 ** rng.integers(-6, 6, (50, 1))).astype(np.float32)
    x[7] = 3.25
    x[9, 5] = np.nan
    c, s, m, bad = ref.quantise(x)
    v = s[:, None].astype(np.float64) * c + m[:, None]
    # half a step, plus what rounding the minimum (2^-9 of it) and the scale (2^-9 of 15 steps) may cost at the ends
    err = np.abs(v - x)
    lim = 0.5 * s + np.abs(m) * 2.0 ** -8 + 15 * s * 2.0 ** -8
    ok = np.arange(50) != 9
    assert (err[ok] <= lim[ok, None]).all()
    assert bad[9] and (v[9] == 0).all()
    assert (v[7] == 3.25).all()


def test_store_and_load_are_each_others_inverse():
    rng = np.random.default_rng(1)
    pages = rng.integers(0, 256, (3, 2, ref.head_bytes(64))).astype(np.uint8)
    e = ref.Entry(rng.standard_normal((2, 64)), rng.standard_normal((2, 64)))
    before = pages.copy()
    ref.store(pages, 70, e, 64)
    k, v = ref.load(pages, 70, 64)
    assert np.array_equal(k, e.values("k")) and np.array_equal(v, e.values("v"))
    for slot in (69, 71, 6, 134):                     # neighbours keep their bytes
        for a, b in zip(ref.load(pages, slot, 64), ref.load(before, slot, 64)):
            assert np.array_equal(a, b, equal_nan=True)


def test_attention_of_equal_keys_is_the_mean_and_of_nothing_is_zero():
    rng = np.random.default_rng(2)
    v = rng.standard_normal((5, 1, 8))
    out, lse, _ = ref.attend(rng.standard_normal((2, 8)), np.zeros((5, 1, 8)), v, [0, 2, 4], 0.3)
    assert np.allclose(out[1], v[[0, 2, 4], 0].mean(0)) and np.allclose(lse, np.log(3))
    out, lse, _ = ref.attend(rng.standard_normal((2, 8)), np.zeros((5, 1, 8)), v, [], 0.3)
    assert (out == 0).all() and np.isneginf(lse).all()
