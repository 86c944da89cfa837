"""The oracle of the paged 8-bit cache against closed forms and torch's conversion."""

import numpy as np
import pytest
import torch

import oracle as O


def test_values_and_rounding_are_those_of_the_type():
    bits = torch.arange(256, dtype=torch.uint8)
    want = bits.view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(O.e4m3_values(bits.numpy()), want, equal_nan=True)
    ok = ~np.isnan(want)
    assert np.array_equal(O.e4m3_codes(want[ok]), bits.numpy()[ok])
    r = np.random.default_rng(1)
    mid = (O.E4M3[1:] + O.E4M3[:-1]) / 2
    x = np.concatenate([O.E4M3, mid, np.nextafter(mid, 0), np.nextafter(mid, 999), r.standard_normal(5000) * 50])
    x = np.concatenate([x, -x]).astype(np.float32)
    x = x[np.abs(x) <= 448]
    assert np.array_equal(O.e4m3_round(x), torch.from_numpy(x).to(torch.float8_e4m3fn).double().numpy())
    assert np.array_equal(O.e4m3_round([449.0, -1e30, np.inf, np.nan]), [448.0, -448.0, np.nan, np.nan], equal_nan=True)


def test_scale_is_the_smallest_that_holds_the_rows():
    for m, s in ((448.0, 127), (448.1, 128), (224.0, 126), (1.0, 119), (0.0, 27), (2.0 ** -140, 27), (3.3e38, 246)):
        assert O.block_scale(np.array([[m, -m / 2], [np.nan, np.inf]])) == s
    for x in np.exp(np.random.default_rng(2).uniform(-60, 80, 50)):
        s = O.block_scale(np.array([x]))
        assert x <= 448 * 2.0 ** (s - 127) and x > 448 * 2.0 ** (s - 128)


def test_writes_keep_what_was_there():
    """Rows written piece by piece are those written at once, but for what a rise of the scale rounds again."""
    r = np.random.default_rng(3)
    k, v = r.standard_normal((90, 16)), r.standard_normal((90, 16))
    a, b = O.BlockRows(32, 16, 3), O.BlockRows(32, 16, 3)
    a.write(0, k, v)
    at = 0
    for n in (1, 5, 0, 40, 1, 43):
        b.write(at, k[at:at + n], v[at:at + n])
        at += n
    assert np.array_equal(a.s, b.s)
    small = 2.0 ** (a.s - 127.0 - 6)
    for x in (0, 1):
        unit = np.repeat(small[x], 32)[:90, None]
        va, vb = a.values(90)[x], b.values(90)[x]
        assert np.all((va == vb) | ((np.abs(va) <= unit) & (np.abs(va - vb) <= unit / 8)))
    lo, hi = b.bounds()
    kb = b.values(90)[0]
    for i in range(3):
        rows = kb[32 * i:32 * i + 32]
        assert np.array_equal(lo[i], rows.min(0)) and np.array_equal(hi[i], rows.max(0))
    c = O.BlockRows(32, 16, 1)
    c.write(0, np.ones((2, 16)), np.ones((2, 16)))
    c.write(1, np.full((1, 16), 2.0 ** 30), np.zeros((1, 16)))
    assert not c.values(1)[0].any() and c.values(1)[1].all()         # 2^-30 of the scale and less is zero
    assert c.bounds()[0].max() == 0.0


@pytest.mark.parametrize("pairs", [False, True])
def test_rotation_keeps_lengths_and_differences(pairs):
    r = np.random.default_rng(4)
    freq = 100.0 ** (-np.arange(8) / 8)
    angle = np.arange(50)[:, None] * freq
    q, k = r.standard_normal((1, 20)), r.standard_normal((1, 20))

    def at(x, p):
        return O.rotate(x, np.cos(angle), np.sin(angle), np.array([p]), pairs)[0]
    for a, b in ((3, 1), (40, 38), (17, 15)):
        assert np.isclose(at(q, a) @ at(k, b), at(q, 2) @ at(k, 0))
        assert np.isclose(np.linalg.norm(at(q, a)), np.linalg.norm(q)) and np.array_equal(at(q, a)[16:], q[0, 16:])
    assert np.array_equal(at(q, 0), q[0]) and np.isnan(at(q, -1)).all() and np.isnan(at(q, 50)).all()


def test_scores_bound_the_products():
    r = np.random.default_rng(5)
    k = r.standard_normal((4, 32, 8))
    q = r.standard_normal((3, 8))
    s = O.block_scores(q, k.min(1), k.max(1))
    assert np.all(np.einsum("gd,btd->bt", q, k).max(1) <= s + 1e-6)


def test_choice_and_what_is_seen():
    s = np.array([0.0, 5.0, np.nan, 3.0, 5.0, -np.inf, 1.0], dtype=np.float32)
    assert O.top_blocks(s, 4, 1, 1) == [0, 1, 4, 6]
    assert O.top_blocks(s, 2, 0, 0) == [1, 4]
    assert O.top_blocks(s, 1, 0, 0) == [1]
    assert O.top_blocks(s, 9, 2, 3) == [0, 1, 2, 3, 4, 5, 6, -1, -1]
    assert O.top_blocks(s, 6, 0, 0, missing=(1,)) == [0, 1, 3, 4, 5, 6]
    assert [O.rows_seen(10, 3, t, 99) for t in range(3)] == [8, 9, 10]
    assert [O.rows_seen(1, 3, t, 99) for t in range(3)] == [0, 0, 1]
    assert O.rows_seen(10, 3, 1, 99, start=20) == 10 and O.rows_seen(10, 3, 1, 99, start=-1) == 0
    assert O.rows_seen(10, 1, 0, 4) == 4 and O.rows_seen(10, 4, 2, 99, start=5) == 8


def test_attention_of_equal_keys_is_the_mean():
    v = np.random.default_rng(6).standard_normal((7, 4))
    out, mag, top = O.attend(np.ones((2, 4)), np.ones((7, 4)), v, 0.5)
    assert np.allclose(out, v.mean(0)) and np.allclose(mag, np.abs(v).mean(0)) and top == 2.0
    assert not O.attend(np.ones((2, 4)), v[:0], v[:0], 1.0)[0].any()


def test_rounding_to_fewer_bits():
    x = np.random.default_rng(7).standard_normal(2000)
    assert np.array_equal(O.round_to(x, 24), x.astype(np.float32).astype(np.float64))
    y = x.astype(np.float32)
    assert np.array_equal(O.round_to(y, 8), torch.from_numpy(y).bfloat16().double().numpy())
