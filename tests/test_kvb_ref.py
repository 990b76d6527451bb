"""The plain model of the 8-bit cache against torch's e4m3 type, and its own definitions."""
import numpy as np
import torch

import kvb_ref as ref
from paper_2505_13204_b200 import binding


def test_codes_are_those_of_the_type():
    every = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(every, ref.VALUES, equal_nan=True)
    rng = np.random.default_rng(0)
    mid = (ref._POS[1:] + ref._POS[:-1]) / 2
    x = np.concatenate([ref._POS, mid, -mid, np.nextafter(mid, 0), np.nextafter(mid, 999), rng.standard_normal(5000) * 10.0 ** rng.integers(-4, 3, 5000)])
    x = np.clip(x, -448, 448)
    x32 = x.astype(np.float32)
    want = torch.as_tensor(x32).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    assert np.array_equal(ref.encode(x32.astype(np.float64)), want)


def test_the_scale_is_the_least_one_that_fits():
    for top in (0.0, 1e-30, 2.0 ** -56 * 1.75, 448.0, np.nextafter(448.0, 999), 1.0, 1.75, 1.7500001, 3.4e38):
        e = ref.fit(top)
        assert top <= 448 * 2.0 ** e and (e == ref.LEAST or top > 448 * 2.0 ** (e - 1))


def test_places_are_a_permutation_in_16_byte_chunks():
    for D in (64, 128, 256):
        at = np.stack([ref.places(D, t) for t in range(ref.PAGE)])
        assert sorted(at.ravel()) == list(range(ref.PAGE * D))
        assert (at.reshape(ref.PAGE, D // 16, 16)[..., 0] % 16 == 0).all() and (np.diff(at.reshape(ref.PAGE, D // 16, 16)) == 1).all()


def test_growing_a_scale_changes_no_normal_value():
    rng = np.random.default_rng(1)
    raw = np.zeros(ref.head_bytes(64), np.uint8)
    b = ref.Block(raw, 1, 64)
    b.e = -3
    x = rng.standard_normal((ref.PAGE, 64))
    for t in range(ref.PAGE):
        b.put(t, x[t])
    was = np.stack([b.value(t) for t in range(ref.PAGE)])
    b.grow(1, range(ref.PAGE))
    now = np.stack([b.value(t) for t in range(ref.PAGE)])
    normal = np.abs(was) >= 2.0 ** (1 - 6)
    assert normal.any() and np.array_equal(was[normal], now[normal]) and (np.abs(was - now) <= 2.0 ** (1 - 10)).all()


def test_books_keep_every_page_once():
    b = ref.Books([[0, 1, 2], [], []], [3, 0, 0], [4, 3], [0] * 5, [150, 0, 0], 4)
    out, full, bad = b.fork([0, 0], [1, 2], [150, 128])
    assert out == [(150, 2, 3), (128, -1, -1)] and not full and not bad and b.shares == [2, 2, 0, 0, 0]
    b.free([0, -1, 0])
    assert b.table == [[], [0, 1, 3], []] and b.stack == [4, 2] and b.shares == [0] * 5
    to, moves = b.compact()
    assert moves == [(3, 2)] and to == [0, 1, -1, 2, -1] and b.table[1] == [0, 1, 2] and b.stack == [4, 3]


def test_sizes_and_refusals_without_a_gpu():
    assert [binding.kvb_head_bytes(D) for D in (64, 128, 256)] == [ref.head_bytes(D) for D in (64, 128, 256)]
    lib = binding.load_library()
    import ctypes as C
    n = C.c_size_t()
    assert lib.aasd_kvb_head_bytes(96, C.byref(n)) == binding.ERR_UNSUPPORTED
    none = [None] * 8
    assert lib.aasd_kvb_attend(None, *none[:7], None, None, 0, None) == 1
    assert lib.aasd_kvb_commit(None, *none[:7], None, None) == 1
    assert lib.aasd_kvb_write(None, *([None] * 11), 0, None, None, None, None) == 1
    assert lib.aasd_kv_free(None, None, None, None, None) == 1 and lib.aasd_kv_copy(None, None, 0, None, None, 0) == 1
    assert lib.aasd_kv_fork(None, None, None, None, 0, None, None, None, None, None) == 1
    assert lib.aasd_kv_compact(None, None, None, None, None, None, None) == 1
