"""Pins of the paged 4-bit cache's oracle: the row format against an exhaustive
search and hand-worked blocks, the page layout byte by byte, the bookkeeping
against its invariants and hand-worked steps."""

from fractions import Fraction

import numpy as np
import pytest

import oracle as O

MAGNITUDES = [Fraction(0), Fraction(1, 2), Fraction(1), Fraction(3, 2), Fraction(2), Fraction(3), Fraction(4), Fraction(6)]


def _block(x):
    """(scale byte, codes) of 32 finite numbers in exact rational arithmetic."""
    x = [Fraction(float(v)) for v in x]
    top = max(abs(v) for v in x)
    e = -1000
    if top:
        e = 0
        while Fraction(2) ** (e + 1) <= top:
            e += 1
        while Fraction(2) ** e > top:
            e -= 1
        if top >= Fraction(7, 4) * Fraction(2) ** e:
            e += 1
    s = min(max(e + 125, 2), 252)
    unit = Fraction(2) ** (s - 127)
    codes = []
    for v in x:
        y = abs(v) / unit
        d = [abs(y - m) for m in MAGNITUDES]
        near = [c for c in range(8) if d[c] == min(d)]
        c = near[0] if len(near) == 1 or near[0] % 2 == 0 else near[1]
        codes.append(c + (8 if v < 0 else 0))
    return s, codes


@pytest.mark.parametrize("seed", range(4))
def test_quantise_matches_rational_arithmetic(seed):
    r = np.random.default_rng(seed)
    for _ in range(25):
        x = r.standard_normal(32) * 2.0 ** r.integers(-130, 120)
        if r.random() < 0.5:  # ties and borders: multiples of an eighth of the unit
            x = r.integers(-56, 57, 32) / 8.0 * 2.0 ** r.integers(-40, 40)
        x = x.astype(np.float32)
        codes, scales = O.mx4_quantise(x[None])
        s, want = _block(x)
        got = [int(c) if c != 8 else 8 if np.signbit(v) else 0 for c, v in zip(codes[0], x)]
        want = [w + 8 if np.signbit(v) and w < 8 else w for w, v in zip(want, x)]
        assert int(scales[0, 0]) == s and got == want


def test_hand_worked_block():
    """Largest magnitude 6: unit 1, and the ties of that unit go to the even code."""
    x = np.zeros(32)
    x[:12] = [6, -6, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, -0.25, 0.26, -5.01]
    codes, scales = O.mx4_quantise(x[None])
    assert scales[0, 0] == 127
    assert codes[0, :12].tolist() == [7, 15, 0, 2, 2, 4, 4, 6, 6, 8, 1, 15]
    assert O.mx4_values(codes, scales)[0, :12].tolist() == [6, -6, 0, 1, 1, 2, 2, 4, 4, 0, 0.5, -6]
    # 7 is as near to 8 as to 6: the next power of two is taken from there on
    x[0] = np.nextafter(7.0, 0.0)
    assert O.mx4_round(x[None])[0, 0] == 6.0
    x[0] = 7.0
    assert O.mx4_round(x[None])[0, 0] == 8.0


def test_largest_element_is_off_by_at_most_a_fifth_and_by_a_seventh_near_the_next_power():
    """Units of the held values around the largest element: 4, 6 and 8.  Halfway from 4 to 6 it is off by 1 of 5;
    from 6 to 8 (the powers' border at 1.75 is halfway) by at most 1 of 7."""
    m = np.linspace(1.0, 2.0, 4001)[:-1]
    x = np.zeros((len(m), 32))
    x[:, 5] = m
    off = np.abs(O.mx4_round(x)[:, 5] - m) / m
    assert off.max() <= 1.0 / 5.0 + 1e-12
    assert off[m >= 1.5].max() <= 1.0 / 7.0 + 1e-12


def test_values_held_come_back_unchanged_and_blocks_with_nan_or_inf_are_nan():
    r = np.random.default_rng(3)
    x = O.mx4_round(r.standard_normal((5, 128)))
    assert np.array_equal(O.mx4_round(x), x)
    for bad in (np.nan, np.inf, -np.inf):
        y = x.copy()
        y[2, 40] = bad
        z = O.mx4_round(y)
        assert np.isnan(z[2, 32:64]).all() and np.array_equal(np.delete(z, np.s_[32:64], 1), np.delete(x, np.s_[32:64], 1))


def test_smallest_and_largest_units():
    x = np.zeros((2, 32))
    x[0, 0] = 2.0 ** -140
    x[1, :2] = np.float64(np.finfo(np.float32).max), 2.0 ** 127
    codes, scales = O.mx4_quantise(x)
    assert scales[:, 0].tolist() == [2, 252]
    assert codes[0, 0] == 0 and codes[1, :2].tolist() == [7, 6]


@pytest.mark.parametrize("page,d", [(32, 64), (64, 128), (128, 64)])
def test_page_layout(page, d):
    r = np.random.default_rng(page + d)
    k, v = r.standard_normal((2, page, d))
    block = O.page_pack(k, v)
    assert block.shape == (O.page_bytes(page, d),) == (page * d * 17 // 16,)
    kc, ks = O.mx4_quantise(k)
    vc, vs = O.mx4_quantise(v)
    t, c = 13, 37
    for codes, base in ((kc, 0), (vc, page * d // 2)):
        byte = block[base + t * d // 2 + c // 2]
        assert (byte >> 4 if c % 2 else byte & 15) == codes[t, c]
    for scales, base in ((ks, page * d), (vs, page * d + page * d // 32)):
        assert block[base + (c // 32) * page + t] == scales[t, c // 32]
    k2, v2 = O.page_unpack(block, page, d)
    assert np.array_equal(k2, O.mx4_round(k)) and np.array_equal(v2, O.mx4_round(v))


def _book(n_pages=10, S=4, M=4, page=32):
    return O.PageBook(np.zeros(n_pages), -np.ones((S, M)), np.zeros(S), np.zeros(S), page)


def test_hand_worked_bookkeeping():
    b = _book()
    assert b.extend([0, 1], [33, 64]) == ([0, 0], 0)
    assert b.table[0, :2].tolist() == [0, 1] and b.table[1, :2].tolist() == [2, 3]
    assert b.extend([0], [31]) == ([33], 0) and b.held[0] == 2        # room was left
    assert b.extend([0, 1], [1, 0]) == ([64, 64], 0) and b.table[0, 2] == 4
    done, missing, copies = b.fork([0, 0, 1], [2, 3, 2])
    assert (done, missing, copies) == ([1, 1, 0], 0, [(4, 5, 1), (4, 6, 1)])
    assert b.refs.tolist() == [3, 3, 1, 1, 1, 1, 1, 0, 0, 0]
    b.free([0, 0, 7, -1])
    assert b.refs.tolist() == [2, 2, 1, 1, 0, 1, 1, 0, 0, 0] and b.held[0] == b.length[0] == 0
    # refusals: slot twice, negative, too long for the table, outside
    assert b.extend([1, 1, 2, 3, 9], [1, 1, -1, 64, 1]) == ([64, -1, -1, -1, -1], 0)
    assert b.table[1, 2] == 4


def test_pages_run_out_in_order():
    b = _book(n_pages=3)
    assert b.extend([0, 1, 2, 3], [32, 65, 1, 0]) == ([0, -1, -1, 0], 2)
    assert b.refs.tolist() == [1, 0, 0]
    b.extend([1], [33])
    done, missing, _ = b.fork([1, 0], [2, 3])
    assert (done, missing) == ([0, 1], 1)


@pytest.mark.parametrize("seed", range(3))
def test_bookkeeping_invariants(seed):
    r = np.random.default_rng(seed)
    S, M, page, n_pages = 12, 5, 32, 30
    b = _book(n_pages, S, M, page)
    for _ in range(200):
        n = int(r.integers(1, 6))
        seq = r.integers(-1, S + 1, n)
        what = r.integers(0, 3)
        if what == 0:
            b.extend(seq, r.integers(0, 90, n))
        elif what == 1:
            b.fork(seq, r.integers(-1, S + 1, n))
        else:
            b.free(seq)
        refs = np.zeros(n_pages, dtype=np.int64)
        for s in range(S):
            mine = b.table[s, :b.held[s]]
            assert len(set(mine.tolist())) == len(mine)
            np.add.at(refs, mine, 1)
            assert b.length[s] <= b.held[s] * page <= M * page
            # shared pages are full
            for i, p in enumerate(mine):
                assert b.refs[p] == 1 or (i + 1) * page <= b.length[s]
        assert np.array_equal(refs, b.refs)


@pytest.mark.parametrize("bad", [-1, 10, 1 << 30, -(1 << 31)])
def test_fork_passes_a_missing_last_page_on(bad):
    """Rows that the parent does not have are none of the child's either: no fresh page stands for them."""
    b = _book()
    b.extend([0, 1], [75, 40])
    b.table[0, 2] = bad
    refs = b.refs.copy()
    done, missing, copies = b.fork([0, 1], [2, 3])
    assert (done, missing, copies) == ([1, 1], 0, [(4, 5, 8)])
    assert b.table[2, :3].tolist() == [0, 1, bad] and b.held[2] == 3 and b.length[2] == 75
    assert (b.refs - refs).tolist() == [1, 1, 0, 1, 0, 1, 0, 0, 0, 0]
    b.free([0, 1, 2, 3])
    assert b.refs.tolist() == [0, 0, 1, 0, 0, 0, 0, 0, 0, 0]          # the page that nobody names any more


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("G", [1, 2, 3, 4, 5, 8, 9, 16])
def test_low_bits_cases_tell_a_lost_part(G, dtype):
    """The paged decode's cases are held exactly, and losing the last 8 of a weight's or a float32 query's 24 bits
    moves every head by more than twice their bound."""
    from tests import paged_decode_cases as C
    q, k, v, want = C.case(G, 64, dtype, 70, (3, 45))
    assert np.array_equal(O.mx4_round(k), k) and np.array_equal(O.mx4_round(v), v)
    assert np.array_equal(q, q.astype(np.float32)) and (dtype == "f32" or np.array_equal(q, C.trunc(q, 8)))
    x = k @ q.T
    w = np.exp(x - x.max(0))
    assert np.allclose(want, (w / w.sum(0)).T @ v, rtol=0, atol=1e-14)
    differ = v[3] != v[45]
    assert differ.any()
    for a, w in C.planted(q[:, 0], dtype):
        off = np.abs(C.result(a, v[3], v[45], w) - want)
        assert (off[:, differ] > 2 * C.BOUND).all()
