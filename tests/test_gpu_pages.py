"""The paged 4-bit cache on the GPU against its oracle: packed bytes, moved rows
and bookkeeping bit for bit, decode within the dense decode's bound."""

import numpy as np
import pytest

torch = pytest.importorskip("torch")

import oracle as O  # noqa: E402
from tests.parity import check_decode, report  # noqa: E402

pytestmark = pytest.mark.gpu

TORCH = {"bf16": torch.bfloat16, "f32": torch.float32}


@pytest.fixture(scope="module")
def K():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2607_13205_amd.build import ensure_built
    ensure_built()
    import paper_2607_13205_amd as K
    return K


def dev(x, dtype=torch.int32):
    return torch.as_tensor(np.ascontiguousarray(x)).to(dtype).cuda()


def make(K, L, Hkv, d, page, n_pages, S, M, seed=0, garbage=True):
    """An empty cache whose pool and table hold anything (scale bytes 255, NaN, among it)."""
    g = np.random.default_rng(seed)
    pool = g.integers(0, 256, (L, n_pages, Hkv, K.page_bytes(page, d)), dtype=np.uint8)
    if garbage:
        pool[..., page * d:] = g.choice([255, 0, 254, 127], pool[..., page * d:].shape)
    z = lambda n: torch.zeros(n, dtype=torch.int32, device="cuda")  # noqa: E731
    table = dev(g.integers(-(1 << 31), 1 << 31, (S, M)))
    return K.Pages(torch.from_numpy(pool).cuda(), z(n_pages), table, z(S), z(S), page, d)


def book(pages):
    return O.PageBook(*(getattr(pages, n).cpu().numpy() for n in ("refs", "table", "held", "length")), pages.page)


def same_book(pages, b):
    for n in ("refs", "held", "length"):
        assert np.array_equal(getattr(pages, n).cpu().numpy(), getattr(b, n)), n
    t = pages.table.cpu().numpy()
    for s in range(b.S):
        assert np.array_equal(t[s, :b.held[s]], b.table[s, :b.held[s]]), s


def rows_of(pages, slot, upto=None):
    """float64 keys and values [L, Hkv, length, d] of a slot, unpacked by the oracle."""
    n = int(pages.length[slot]) if upto is None else upto
    ids = pages.table[slot, :-(-n // pages.page)].cpu().numpy()
    block = pages.pool.cpu().numpy()[:, ids].transpose(0, 2, 1, 3)
    k, v = O.page_unpack(block, pages.page, pages.d)
    return tuple(x.reshape(x.shape[:2] + (-1, pages.d))[:, :, :n] for x in (k, v))


def normal(shape, dtype, seed, scale=1.0):
    return (scale * torch.randn(shape, generator=torch.Generator().manual_seed(seed))).to(TORCH[dtype])


# ---------------------------------------------------------------------------
# the row format
# ---------------------------------------------------------------------------

def _hard_rows(dtype, d):
    """Rows that meet every border of the format."""
    r = np.random.default_rng(5)
    rows = []
    for _ in range(24):  # multiples of an eighth and a sixteenth of the unit: ties and the values next to them
        rows.append(r.integers(-56, 57, d) / 8.0 * 2.0 ** r.integers(-40, 40))
        rows.append(r.integers(-112, 113, d) / 16.0)
    for _ in range(8):
        rows.append(r.standard_normal(d) * 2.0 ** r.integers(-135, 125))
        rows.append(r.standard_normal(d) * 2.0 ** r.integers(-30, 30, d))
    rows += [np.zeros(d), np.full(d, -0.0), np.full(d, 3.38e38), np.full(d, 1e-44), np.full(d, 2.0 ** -126)]
    for bad in (np.nan, np.inf, -np.inf):
        x = r.standard_normal(d)
        x[7] = bad
        x[40] = -bad
        rows.append(x)
    x = torch.from_numpy(np.stack(rows)).to(TORCH[dtype])
    if dtype == "f32":  # one step of float32 below and above the borders
        t = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0], dtype=torch.float32)
        e = torch.cat([t, torch.nextafter(t, t * 0), torch.nextafter(t, t * 9), torch.tensor([6.0, 7.0, 6.9999995])])
        x = torch.cat([x, torch.cat([e, e.new_full((8,), 6.0)]).repeat(d // 32)[None]])
        x = torch.cat([x, x[-1:] * 2.0 ** 90, x[-1:] * 2.0 ** -120])
    return x


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
def test_packed_bytes(K, dtype, d):
    x = _hard_rows(dtype, d)
    n, page = len(x), 32
    pages = make(K, 1, 1, d, page, 5, 1, 4)
    start, _ = K.pages_extend(pages, dev([n]))
    before = pages.pool.cpu().numpy().copy()
    k, v = x[None, None, None].cuda(), x.flip(0)[None, None, None].cuda()
    K.pages_append(k, v, pages, start)
    x = x.double().numpy()
    M = -(-n // page)
    pad = np.zeros((M * page - n, d))
    want = O.page_pack(np.concatenate([x, pad]).reshape(M, page, d), np.concatenate([x[::-1], pad]).reshape(M, page, d))
    written = torch.zeros_like(pages.pool, dtype=torch.bool)
    for t in range(n):
        _mark(written, pages, 0, 0, 0, t)
    written = written.cpu().numpy()[0, :M, 0]
    got, before = pages.pool.cpu().numpy()[0, :, 0], before[0, :, 0]
    assert np.array_equal(got[:M][written], want[written])
    assert np.array_equal(got[:M][~written], before[:M][~written]) and np.array_equal(got[M:], before[M:])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
def test_read_gives_every_code_and_scale(K, dtype, d):
    """All 256 scale bytes times all sixteen codes, through pages_read."""
    page = 256
    block = np.zeros(K.page_bytes(page, d), dtype=np.uint8)
    codes = (np.arange(d)[None] + np.arange(page)[:, None]) % 16
    packed = (codes[:, 0::2] | codes[:, 1::2] << 4).astype(np.uint8)
    half, ns = page * d // 2, page * d // 32
    block[:half] = packed.reshape(-1)
    block[half:2 * half] = packed[::-1].reshape(-1)
    block[2 * half:2 * half + ns] = np.tile(np.arange(256), d // 32)
    block[2 * half + ns:] = np.tile(np.arange(256)[::-1], d // 32)
    z = dev([0])
    pages = K.Pages(torch.from_numpy(block)[None, None, None].cuda(), z, dev([[0]]), dev([1]), dev([page]), page, d)
    k, v = K.pages_read(pages, page, dtype=TORCH[dtype])
    wk, wv = O.page_unpack(block, page, d)
    big = float(torch.finfo(TORCH[dtype]).max)
    for got, want in ((k, wk), (v, wv)):
        want = np.where(np.abs(want) > big, np.copysign(np.inf, want), want)
        assert np.array_equal(got[0, 0, 0].double().cpu().numpy(), want, equal_nan=True)


# ---------------------------------------------------------------------------
# rows
# ---------------------------------------------------------------------------

def _filled(K, L, Hkv, d, page, lengths, seed=0, spare=3, dtype="bf16", extra_slots=0):
    """A cache with one sequence per length (slots in order), its rows normal numbers."""
    S, n_pages = len(lengths) + extra_slots, sum(-(-n // page) for n in lengths) + spare
    M = max(1, max(-(-n // page) for n in lengths) + 1)
    pages = make(K, L, Hkv, d, page, n_pages, S, M, seed)
    B, T = len(lengths), max(max(lengths), 1)
    start, missing = K.pages_extend(pages, dev(lengths), seq=dev(range(B)))
    assert start.tolist() == [0] * B and missing.item() == 0
    k, v = normal((L, B, Hkv, T, d), dtype, seed + 1).cuda(), normal((L, B, Hkv, T, d), dtype, seed + 2).cuda()
    K.pages_append(k, v, pages, start, n_new=dev(lengths), seq=dev(range(B)))
    return pages, k, v


CASES = [  # L, B, Hkv, N, d, page, cap, dtype
    (1, 1, 1, 1, 64, 32, 1, "bf16"),
    (2, 3, 2, 77, 128, 32, 50, "bf16"),
    (1, 2, 3, 400, 64, 128, 300, "bf16"),
    (1, 2, 2, 150, 128, 64, 149, "f32"),
    (2, 1, 1, 333, 64, 1024, 200, "f32"),
]


@pytest.mark.parametrize("L,B,Hkv,N,d,page,cap,dtype", CASES)
@pytest.mark.parametrize("major", ["head", "token"])
def test_compact(K, L, B, Hkv, N, d, page, cap, dtype, major):
    r = np.random.default_rng(N)
    shape = (L, B, Hkv, N, d) if major == "head" else (L, B, N, Hkv, d)
    k, v = normal(shape, dtype, 1).cuda(), normal(shape, dtype, 2).cuda()
    if major == "token":
        k, v = k.permute(0, 1, 3, 2, 4), v.permute(0, 1, 3, 2, 4)
    S, M = B + 2, -(-(cap + 37) // page) + 1
    pages = make(K, L, Hkv, d, page, B * M + 2, S, M, seed=3)
    slots = r.permutation(S)[:B]
    seq = dev(slots)
    K.pages_extend(pages, dev(r.integers(0, 37, B)), seq=seq)       # some rows are there already
    first = pages.length[seq.long()].clone()
    start, _ = K.pages_extend(pages, dev([cap] * B), seq=seq)
    assert torch.equal(start, first)
    idx = np.stack([np.sort(r.permutation(N)[:cap]) for _ in range(L * B * Hkv)]).reshape(L, B, Hkv, cap)
    count = np.full((L, B, Hkv), cap)
    count[0, 0, 0] = max(0, cap - 3)
    count[-1, -1, -1] = cap + 9                                      # more than the row holds: cut
    if cap > 8:
        idx[0, -1, 0, 2], idx[0, -1, 0, 5] = -1, N                   # skipped
    before = pages.pool.clone()
    K.pages_compact(k, v, dev(idx), dev(count), pages, start, seq=seq)
    kn, vn = k.double().cpu().numpy(), v.double().cpu().numpy()
    written = torch.zeros_like(before, dtype=torch.bool)
    touched = (before != pages.pool)
    for b in range(B):
        gk, gv = rows_of(pages, int(slots[b]))
        for l in range(L):
            for j in range(Hkv):
                for m in range(min(count[l, b, j], cap)):
                    t = idx[l, b, j, m]
                    if 0 <= t < N:
                        at = int(start[b]) + m
                        assert np.array_equal(gk[l, j, at], O.mx4_round(kn[l, b, j, t][None])[0])
                        assert np.array_equal(gv[l, j, at], O.mx4_round(vn[l, b, j, t][None])[0])
                        _mark(written, pages, int(slots[b]), l, j, at)
    assert not (touched & ~written).any(), "bytes of other rows were written"


def _mark(mask, pages, slot, l, j, at):
    page, d = pages.page, pages.d
    pg, t = int(pages.table[slot, at // page]), at % page
    half, ns = page * d // 2, page * d // 32
    for i in (0, 1):
        mask[l, pg, j, i * half + t * d // 2:i * half + (t + 1) * d // 2] = True
        mask[l, pg, j, 2 * half + i * ns + t:2 * half + (i + 1) * ns:page] = True


def test_append_drops_what_has_no_place(K):
    """Refused starts, positions without a page, page numbers outside the pool, slots outside: nothing is written there."""
    L, Hkv, d, page = 1, 2, 64, 32
    pages, k, v = _filled(K, L, Hkv, d, page, [40, 10, 33, 5], spare=4)
    pages.table[2, 1] = 1 << 30
    pages.table[3, 0] = -5
    pages.held[1] = 1 << 30                                          # more than the table's row: cut to it
    before = pages.pool.clone()
    T = 70
    x = normal((L, 5, Hkv, T, d), "bf16", 9).cuda()
    K.pages_append(x, x, pages, dev([-1, 60, 20, 0, 0]), seq=dev([0, 1, 2, 3, 4]), n_new=dev([70, 2, 30, 30, 9]))
    torch.cuda.synchronize()
    changed = (before != pages.pool).any(-1)[0]                      # [n_pages, Hkv]
    own = {int(pages.table[1, 1]) if 0 <= int(pages.table[1, 1]) < pages.c.n_pages else -1, int(pages.table[2, 0])}
    assert {int(i) for i in changed.any(-1).nonzero().flatten()} <= own
    K.pages_append(x[:, :2], x[:, :2], pages, dev([0, 0]), seq=dev([-3, 99]))
    K.pages_append(x[:, :1], x[:, :1], pages, dev([0]), n_new=dev([-4]), seq=dev([0]))
    K.pages_append(x[:, :1, :, :0], x[:, :1, :, :0], pages, dev([0]), seq=dev([0]))
    assert torch.equal((before != pages.pool).any(-1)[0], changed)


@pytest.mark.parametrize("L,B,Hkv,N,d,page,cap,dtype", CASES)
def test_read_ranges(K, L, B, Hkv, N, d, page, cap, dtype):
    r = np.random.default_rng(cap)
    lengths = [N] + [int(r.integers(0, N + 1)) for _ in range(B)]
    pages, k, v = _filled(K, L, Hkv, d, page, lengths, dtype=dtype)
    want = [O.mx4_round(x.double().cpu().numpy()) for x in (k, v)]
    n = len(lengths)
    start = np.array([0] + [int(r.integers(-1, N + 2)) for _ in range(B)])
    count = np.array([cap] + [int(r.integers(-1, cap + 2)) for _ in range(B)])
    order = r.permutation(n)
    outs = [torch.full((L, n, Hkv, cap, d), 7.0, dtype=TORCH[dtype], device="cuda") for _ in (0, 1)]
    K.pages_read(pages, cap, seq=dev(order), start=dev(start[order]), count=dev(count[order]), k_out=outs[0],
                 v_out=outs[1])
    for got, w in zip(outs, want):
        exp = np.full(got.shape, 7.0)
        for i, s in enumerate(order):
            m = min(int(count[s]), cap, lengths[s] - int(start[s]))
            if start[s] >= 0 and m > 0:
                exp[:, i, :, :m] = w[:, s, :, start[s]:start[s] + m]
        assert np.array_equal(got.double().cpu().numpy(), exp)
    # all slots, whole sequences; slots outside and invalid pages give nothing
    k2, _ = K.pages_read(pages, N, dtype=TORCH[dtype])
    for s in range(n):
        assert np.array_equal(k2[:, s, :, :lengths[s]].double().cpu().numpy(), want[0][:, s, :, :lengths[s]])
        assert not k2[:, s, :, lengths[s]:].any()
    pages.table[0, 0] = pages.c.n_pages
    k3, v3 = K.pages_read(pages, N, seq=dev([-1, n, 0]), dtype=TORCH[dtype])
    assert not k3[:, :2].any() and not v3[:, :2].any() and not k3[:, 2, :, :page].any()
    assert torch.equal(k3[:, 2, :, page:], k2[:, 0, :, page:])


def test_read_of_keys_or_values_alone(K):
    import ctypes
    pages, _, _ = _filled(K, 2, 2, 64, 32, [70, 5])
    k, v = K.pages_read(pages, 70)
    for which, want in ((0, k), (1, v)):
        out = torch.zeros_like(want)
        at = [out.data_ptr() if i == which else None for i in (0, 1)]
        assert K.binding.LIB.kve_pages_read(ctypes.byref(pages.c), 0, 2, 70, None, None, None, *at,
                                            torch.cuda.current_stream().cuda_stream) == 0
        assert torch.equal(out, want)


@pytest.mark.parametrize("L,B,Hkv,N,d,page,cap,dtype", CASES)
def test_select(K, L, B, Hkv, N, d, page, cap, dtype):
    r = np.random.default_rng(7 * N)
    lengths = [N] * B
    pages, k, v = _filled(K, L, Hkv, d, page, lengths, spare=B * (-(-cap // page)) + 1, extra_slots=B)
    dst = dev(range(B, 2 * B))
    start, missing = K.pages_extend(pages, dev([cap] * B), seq=dst)
    assert missing.item() == 0
    idx = np.stack([np.sort(r.permutation(N)[:cap]) for _ in range(L * B * Hkv)]).reshape(L, B, Hkv, cap)
    count = np.full((L, B, Hkv), cap)
    if cap > 8:
        idx[0, 0, 0, 3], idx[0, 0, 0, 4], count[-1, -1, -1] = N, -7, cap - 4
    K.pages_select(pages, dev(range(B)), dev(idx), dev(count), dst, start)
    src = [rows_of(pages, b) for b in range(B)]
    for b in range(B):
        got = rows_of(pages, B + b)
        for g, s in zip(got, src[b]):
            for l in range(L):
                for j in range(Hkv):
                    m = np.arange(min(count[l, b, j], cap))
                    m = m[(idx[l, b, j, m] >= 0) & (idx[l, b, j, m] < N)]
                    assert np.array_equal(g[l, j, m], s[l, j, idx[l, b, j, m]])
    for b in range(B):  # the sources are what they were
        for s, x in zip(rows_of(pages, b), (k, v)):
            assert np.array_equal(s, O.mx4_round(x[:, b].double().cpu().numpy()))


# ---------------------------------------------------------------------------
# bookkeeping
# ---------------------------------------------------------------------------

@pytest.mark.parametrize("seed,S,M,page,n_pages", [(0, 12, 5, 32, 30), (1, 40, 7, 64, 90), (2, 200, 9, 32, 5000)])
def test_bookkeeping_follows_the_oracle(K, seed, S, M, page, n_pages):
    """Random extends, forks and frees with refusals of every kind, and the rows of forked tails."""
    r = np.random.default_rng(seed)
    pages = make(K, 2, 2, 64, page, n_pages, S, M, seed)
    b = book(pages)
    for step in range(60):
        n = int(r.integers(1, S // 2))
        seq = r.integers(-1, S + 1, n)
        what = r.integers(0, 5)
        if what < 3:
            add = r.integers(-1, int(0.6 * M * page), n)
            start, missing = K.pages_extend(pages, dev(add), seq=dev(seq))
            want, lack = b.extend(seq, add)
            assert start.tolist() == want and missing.item() == lack
        elif what == 3:
            dst = r.integers(-1, S + 1, n)
            before = pages.pool.clone()
            done, missing = K.pages_fork(pages, dev(seq), dev(dst))
            want, lack, copies = b.fork(seq, dst)
            assert done.tolist() == want and missing.item() == lack
            keep = torch.ones(n_pages, dtype=torch.bool, device="cuda")
            for a, o, rows in copies:
                keep[o] = False
                ka, va = O.page_unpack(before[:, a].cpu().numpy(), page, 64)
                ko, vo = O.page_unpack(pages.pool[:, o].cpu().numpy(), page, 64)
                assert np.array_equal(ka[:, :, :rows], ko[:, :, :rows], equal_nan=True)
                assert np.array_equal(va[:, :, :rows], vo[:, :, :rows], equal_nan=True)
            assert torch.equal(before[:, keep], pages.pool[:, keep])
        else:
            K.pages_free(pages, dev(seq[:max(1, n // 3)]))
            b.free(seq[:max(1, n // 3)])
        same_book(pages, b)
    K.pages_free(pages)
    assert not pages.refs.any() and not pages.held.any() and not pages.length.any()


def test_outputs_may_take_the_place_of_inputs(K):
    """done in the array of sources, start in that of the counts: read before they are written."""
    pages, k, _ = _filled(K, 1, 1, 64, 32, [75, 40], extra_slots=4, spare=8)
    src, dst = dev([1, 0, 0]), dev([5, 3, 4])
    done, _ = K.pages_fork(pages, src, dst, done=src)
    assert done.tolist() == [1, 1, 1] and pages.length.tolist() == [75, 40, 0, 75, 75, 40]
    for slot, of in ((3, 0), (4, 0), (5, 1)):
        n = int(pages.length[slot])
        assert np.array_equal(rows_of(pages, slot)[0], O.mx4_round(k[:, of, :, :n].double().cpu().numpy()))
    add = dev([7, 0, 9])
    start, _ = K.pages_extend(pages, add, seq=dev([3, 4, 5]), start=add)
    assert start.tolist() == [75, 75, 40] and pages.length.tolist() == [75, 40, 0, 82, 75, 49]


def test_many_entries_and_a_large_pool(K):
    """1024 entries; free pages scattered over 300000, found in ascending order over many rounds."""
    r = np.random.default_rng(11)
    n_pages, S = 300_000, 1024
    pages = make(K, 1, 1, 64, 32, n_pages, S, 4, garbage=False)
    refs = (r.random(n_pages) < 0.99).astype(np.int32)
    pages.refs.copy_(dev(refs))
    b = book(pages)
    add = r.integers(0, 100, S)
    order = r.permutation(S)
    start, missing = K.pages_extend(pages, dev(add), seq=dev(order))
    want, lack = b.extend(order, add)
    assert start.tolist() == want and missing.item() == lack
    same_book(pages, b)


def test_corrupt_bookkeeping_stays_in_bounds(K):
    """Lengths, counts and page numbers that no call made: what the header promises, nothing else touched."""
    pages, _, _ = _filled(K, 1, 1, 64, 32, [50, 50, 50], extra_slots=3)
    pages.length.copy_(dev([1 << 30, -7, 50, 0, 0, 0]))
    pages.held.copy_(dev([1 << 30, 2, -3, 0, 0, 0]))
    pages.table[0].fill_(-(1 << 31))
    refs = pages.refs.clone()
    done, _ = K.pages_fork(pages, dev([0, 1, 2]), dev([3, 4, 5]))
    assert done.tolist() == [1, 1, 1] and pages.length[3:].tolist() == [pages.c.M * 32, 0, 0]
    assert torch.equal(pages.refs, refs)
    q = normal((1, 6, 2, 64), "bf16", 1).cuda()
    assert not K.decode_pages(q, pages).any()
    K.pages_free(pages, dev([0, 2, 3]))
    assert torch.equal(pages.refs, refs)
    start, _ = K.pages_extend(pages, dev([1]), seq=dev([1]))
    assert start.tolist() == [0]


# ---------------------------------------------------------------------------
# decode
# ---------------------------------------------------------------------------

def _decode_ref(q, k, v, G):
    """float64 decode of one (layer, sample): q [Hq, d], k, v [Hkv, n, d]; (out, weighted magnitudes, largest logit)."""
    out, mag, top = [], [], 0.0
    for h in range(q.shape[0]):
        kk, vv = k[h // G], v[h // G]
        if kk.shape[0] == 0:
            out.append(np.zeros(q.shape[1]))
            mag.append(np.zeros(q.shape[1]))
            continue
        x = kk @ q[h] / np.sqrt(q.shape[1])
        top = max(top, float(np.abs(x).max()))
        w = np.exp(x - x.max())
        w /= w.sum()
        out.append(w @ vv)
        mag.append(w @ np.abs(vv))
    return np.stack(out), np.stack(mag), top


DECODES = [  # Hkv, G, d, page, lengths, max_tokens, dtype, scale of the queries
    (1, 1, 64, 32, [0, 1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65], None, "bf16", 1.0),
    (2, 4, 128, 32, [0, 1, 31, 32, 33, 127, 128, 129, 300], None, "bf16", 1.0),
    (2, 3, 128, 64, [5, 700, 1639], 1639, "bf16", 1.0),
    (1, 8, 128, 1024, [4000, 1, 2047], None, "bf16", 1.0),
    (1, 16, 128, 64, [333, 20], None, "bf16", 1.0),
    (3, 5, 64, 128, [1000, 64, 0], None, "bf16", 1.0),
    (1, 16, 64, 64, [190], None, "f32", 1.0),
    (2, 4, 128, 64, [600, 31], None, "f32", 1.0),
    (2, 4, 64, 32, [5003, 1200], None, "f32", 1.0),
    (2, 4, 128, 64, [600, 90], None, "bf16", 40.0),     # logits of hundreds: the reference is raised again and again
    (1, 7, 128, 64, [900, 90], None, "f32", 40.0),
    (1, 2, 128, 64, [600], 350, "bf16", 1.0),           # fewer tokens than the sequence has
    (1, 4, 128, 32, [70000, 3], None, "bf16", 1.0),     # many splits
    # a compute unit to a sequence: 16 or 12 waves, some without a step
    (1, 4, 128, 32, [500, 31, 480, 0, 513 - 1], 512, "bf16", 1.0),
    (1, 8, 64, 64, [511, 64, 65], 512, "bf16", 20.0),
    (2, 3, 128, 64, [512, 100, 384, 385], 512, "f32", 1.0),
    (1, 13, 128, 32, [512, 1, 200], 512, "bf16", 1.0),
    (64, 2, 64, 128, [2000, 70, 0], 2048, "bf16", 1.0),
]


@pytest.mark.parametrize("Hkv,G,d,page,lengths,most,dtype,qs", DECODES)
def test_decode(K, Hkv, G, d, page, lengths, most, dtype, qs):
    L, B, Hq = (2 if max(lengths) < 5000 else 1), len(lengths), Hkv * G
    pages, _, _ = _filled(K, L, Hkv, d, page, lengths, seed=G, extra_slots=1)
    r = np.random.default_rng(G)
    order = r.permutation(B)
    q = normal((L, B, Hq, d), dtype, 77, qs).cuda()
    out = torch.full((L, B, Hq, d), float("nan"), device="cuda")
    K.decode_pages(q, pages, max_tokens=most, seq=dev(order), out=out)
    worst = 0.0
    qn, on = q.double().cpu().numpy(), out.double().cpu().numpy()
    for i, s in enumerate(order):
        n = lengths[s] if most is None else min(lengths[s], most)
        k, v = rows_of(pages, int(s), n)
        for l in range(L):
            want, mag, top = _decode_ref(qn[l, i], k[l], v[l], G)
            worst = max(worst, check_decode(on[l, i], want, mag, top, f"length {n} layer {l}"))
    report(f"paged decode worst err/bound g{G} d{d} {dtype} x{qs:g}", round(worst, 4))


@pytest.mark.parametrize("G,d", [(1, 64), (4, 128), (8, 64), (16, 128)])
def test_decode_of_large_values_under_rising_logits(K, G, d):
    """Each token's logit is above the one before, by 90 in all, over values around 2^100: the unnormalised sums of a
    reference that is never raised would leave float32."""
    n = 500
    pages, _, _ = _filled(K, 1, 1, d, 32, [n], seed=G)
    k = torch.zeros((1, 1, 1, n, d))
    k[..., 0] = torch.linspace(0.5, 6.0, n)
    v = normal((1, 1, 1, n, d), "f32", 5, 2.0 ** 100)
    K.pages_append(k.cuda(), v.cuda(), pages, dev([0]))
    q = torch.zeros((1, 1, G, d))
    q[..., 0] = 15.0 * np.sqrt(d)
    q[..., 1:] = normal((1, 1, G, d - 1), "f32", 6)
    out = K.decode_pages(q.bfloat16().cuda(), pages).double().cpu().numpy()
    kk, vv = rows_of(pages, 0)
    want, mag, top = _decode_ref(q.bfloat16().double().numpy()[0, 0], kk[0], vv[0], G)
    check_decode(out[0, 0], want, mag, top)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("G,d,n,drowned,most", [(1, 64, 150, 70, None), (4, 128, 150, 70, 150), (8, 64, 600, 520, None),
                                                (16, 128, 3000, 2500, None), (3, 128, 40, 39, 40)])
def test_decode_of_logits_below_float32(K, G, d, n, drowned, most, dtype):
    """The first `drowned` logits are products that leave float32 downwards, all those of some waves and splits: they
    have no weight, and the others, which are zero, share it."""
    pages, _, _ = _filled(K, 1, 1, d, 32, [n], seed=G)
    k = torch.zeros((1, 1, 1, n, d))
    k[..., :drowned, 0] = -6.0
    v = normal((1, 1, 1, n, d), "f32", 5)
    K.pages_append(k.cuda(), v.cuda(), pages, dev([0]))
    q = torch.zeros((1, 1, G, d))
    q[..., 0] = 2.0 ** 127
    out = K.decode_pages(q.to(TORCH[dtype]).cuda(), pages, max_tokens=most).double().cpu().numpy()
    _, vv = rows_of(pages, 0)
    rest = vv[0, 0, drowned:]
    check_decode(out[0, 0], np.tile(rest.mean(0), (G, 1)), np.tile(np.abs(rest).mean(0), (G, 1)), 0.0)


@pytest.mark.parametrize("L,B,Hkv,G,page,longest,most", [
    (1, 150, 1, 2, 32, 700, None),     # more sequences than a wave has lanes, several splits each
    (1, 64, 2, 4, 64, 200, 200),
    (1, 65, 1, 1, 32, 1500, None),
    (130, 2, 8, 1, 64, 2300, None),    # more (layer, KV head) pairs than resident workgroups: one split per sequence
    (40, 30, 1, 4, 128, 1100, 1100),   # a workgroup per sequence, of four waves
    (3, 50, 2, 4, 32, 500, 500),       # of eight
    (2, 100, 1, 11, 64, 300, 320),     # of sixteen, G = 11
    (5, 75, 1, 8, 32, 2000, 2048),
])
def test_decode_of_many_sequences_and_pairs(K, L, B, Hkv, G, page, longest, most):
    """Ragged lengths with empty sequences among them, slots named twice and in any order."""
    r = np.random.default_rng(B)
    d, Hq = 64, Hkv * G
    lengths = [longest] + [int(r.integers(0, longest + 1)) if r.random() < 0.8 else 0 for _ in range(B - 1)]
    pages, _, _ = _filled(K, L, Hkv, d, page, lengths, seed=B)
    order = np.concatenate([r.permutation(B)[:B - 1], [0]])
    q = normal((L, B, Hq, d), "bf16", 78).cuda()
    out = torch.full((L, B, Hq, d), float("nan"), device="cuda")
    K.decode_pages(q, pages, max_tokens=most, seq=dev(order), out=out)
    k, v = (x.float().cpu().numpy().astype(np.float64) for x in K.pages_read(pages, longest, seq=dev(order)))
    qn, on = q.double().cpu().numpy(), out.double().cpu().numpy()
    for l in sorted({0, L // 2, L - 1}):
        for i, s in enumerate(order):
            n = lengths[s]
            want, mag, top = _decode_ref(qn[l, i], k[l, i, :, :n], v[l, i, :, :n], G)
            check_decode(on[l, i], want, mag, top, f"sample {i} of {n} layer {l}")
    assert torch.isfinite(out).all()


def test_decode_of_thousands_of_samples(K):
    """More samples than lengths are kept in LDS for, on few slots, some of them outside the cache, beside long ones."""
    B, G, d = 4500, 2, 64
    lengths = [2600, 1, 0, 33, 300, 64, 900]
    pages, _, _ = _filled(K, 1, 1, d, 32, lengths)
    r = np.random.default_rng(8)
    order = r.integers(-1, len(lengths) + 1, B)
    order[[0, 63, 64, B - 1]] = 0
    q = normal((1, B, G, d), "bf16", 79).cuda()
    out = torch.full((1, B, G, d), float("nan"), device="cuda")
    K.decode_pages(q, pages, seq=dev(order), out=out)
    rows = [rows_of(pages, s) for s in range(len(lengths))]
    qn, on = q.double().cpu().numpy(), out.double().cpu().numpy()
    assert np.isfinite(on).all()
    for i in [0, 1, 62, 63, 64, 65, B - 2, B - 1, *r.integers(0, B, 150)]:
        s = order[i]
        if 0 <= s < len(lengths):
            want, mag, top = _decode_ref(qn[0, i], rows[s][0][0], rows[s][1][0], G)
            check_decode(on[0, i], want, mag, top, f"sample {i} slot {s}")
        else:
            assert not on[0, i].any()


@pytest.mark.parametrize("dtype,B,slots", [("bf16", 8194, True), ("f32", 9000, True), ("bf16", 5001, False)])
def test_decode_of_more_samples_than_a_launch_cuts(K, dtype, B, slots):
    """Slices of samples one after the other over the same workspace, two layers, rows of several splits in each,
    captured too."""
    L, Hkv, G, d, page = 2, 2, 2, 64, 32
    lengths = [1, 2600, 0, 33, 300]
    if slots:
        pages, _, _ = _filled(K, L, Hkv, d, page, lengths)
    else:                                                       # sample b in slot b: the slots share their pages
        few, _, _ = _filled(K, L, Hkv, d, page, lengths)
        which = np.random.default_rng(2).choice([0, 2, 3, 4], B)
        which[[0, B // 2, B // 2 + 1, B - 1]] = 1
        at = dev(which).long()
        pages = K.Pages(few.pool, few.refs, few.table[at].contiguous(), few.held[at].contiguous(),
                        few.length[at].contiguous(), page, d)
        rows_in = few
    r = np.random.default_rng(9)
    order = r.choice([-1, 0, 2, 3, 4, len(lengths)], B) if slots else which
    if slots:
        order[[0, B // 3, B // 3 + 1, 2 * B // 3, 2 * B // 3 + 1, B - 1]] = 1
        rows_in = pages
    q = normal((L, B, Hkv * G, d), dtype, 79).cuda()
    out = torch.full(q.shape, float("nan"), device="cuda")
    ws = torch.empty(K.decode_pages_workspace_size(L, B, Hkv * G, Hkv, pages.c.M * page, d), dtype=torch.uint8,
                     device="cuda")
    ws.fill_(255)
    seq = dev(order) if slots else None
    K.decode_pages(q, pages, seq=seq, out=out, workspace=ws)
    rows = [rows_of(rows_in, s) for s in range(len(lengths))]
    qn, on = q.double().cpu().numpy(), out.double().cpu().numpy()
    assert np.isfinite(on).all()
    ends = [x + e for x in (0, B // 3, B // 2, 2 * B // 3, B - 2) for e in (0, 1)]
    for i in [*ends, *r.integers(0, B, 100)]:
        s = order[i]
        for l in range(L):
            if 0 <= s < len(lengths):
                want, mag, top = _decode_ref(qn[l, i], rows[s][0][l], rows[s][1][l], G)
                check_decode(on[l, i], want, mag, top, f"sample {i} slot {s} layer {l}")
            else:
                assert not on[l, i].any()
    want = out.clone()
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=side):
        K.decode_pages(q, pages, seq=seq, out=out, workspace=ws)
    for i in range(3):
        out.fill_(float("nan"))
        ws.fill_(i)
        graph.replay()
        assert torch.equal(out, want)


def test_decode_equals_decode_over_the_rows_read_back(K):
    """The same rows dense in bf16: decode_attention gives the same to float32 rounding."""
    lengths = [700, 64, 0, 333]
    pages, _, _ = _filled(K, 1, 4, 128, 64, lengths)
    k, v = K.pages_read(pages, 700)
    q = normal((1, 4, 16, 128), "bf16", 3).cuda()
    a = K.decode_pages(q, pages, max_tokens=700)
    count = dev(lengths)[None, :, None].expand(1, 4, 4).contiguous()
    b = K.decode_attention(q, k, v, count)
    k64, v64 = k.double().cpu().numpy(), v.double().cpu().numpy()
    for s, n in enumerate(lengths):
        want, mag, top = _decode_ref(q[0, s].double().cpu().numpy(), k64[0, s, :, :n], v64[0, s, :, :n], 4)
        check_decode(a[0, s].cpu().numpy(), want, mag, top)
        check_decode(b[0, s].cpu().numpy(), want, mag, top)


def test_decode_leaves_out_missing_pages_and_passes_nan_on(K):
    L, Hkv, G, d, page = 1, 2, 4, 128, 32
    lengths = [100, 100, 100, 100, 20]
    pages, _, _ = _filled(K, L, Hkv, d, page, lengths)
    q = normal((L, 5, Hkv * G, d), "bf16", 4).cuda()
    pages.table[0, 1] = -1
    pages.table[1, 0], pages.table[1, 3] = pages.c.n_pages, 1 << 30
    pages.table[2, :4] = -1
    k, v = rows_of(pages, 3)
    half = page * d // 2
    pages.pool[0, int(pages.table[3, 2]), 0, 2 * half + 5] = 255     # a key block of KV head 0
    pages.pool[0, int(pages.table[4, 0]), 1, 2 * half + page * d // 32 + 3 * page + 7] = 255  # a value block of head 1
    out = K.decode_pages(q, pages).double().cpu().numpy()[0]
    qn = q.double().cpu().numpy()[0]
    for s, keep in ((0, [0, 2, 3]), (1, [1, 2])):
        ids = [int(pages.table[s, i]) for i in keep]
        kk, vv = O.page_unpack(pages.pool.cpu().numpy()[0][ids].transpose(1, 0, 2), page, d)
        n = sum(min(32, 100 - 32 * i) for i in keep)
        kk, vv = kk.reshape(Hkv, -1, d)[:, :n], vv.reshape(Hkv, -1, d)[:, :n]
        want, mag, top = _decode_ref(qn[s], kk, vv, G)
        check_decode(out[s], want, mag, top)
    assert not out[2].any()
    assert np.isnan(out[3, :G]).all()
    want, mag, top = _decode_ref(qn[3], k[0], v[0], G)
    check_decode(out[3, G:], want[G:], mag[G:], top)
    assert np.isfinite(out[4, :G]).all()
    assert np.isnan(out[4, G:, 96:]).all() and np.isfinite(out[4, G:, :96]).all()
    # slots outside read as empty
    assert not K.decode_pages(q[:, :2], pages, seq=dev([-1, 5])).any()


# ---------------------------------------------------------------------------
# offsets beyond 32 bits
# ---------------------------------------------------------------------------

def test_pages_beyond_four_gigabytes(K):
    """The last pages of a pool of 4.9 GB: rows written, forked, moved, read and attended to where they belong."""
    Hkv, d, page, n_pages = 8, 128, 64, 70_000
    pool = torch.zeros((1, n_pages, Hkv, K.page_bytes(page, d)), dtype=torch.uint8, device="cuda")
    assert pool.numel() > 1 << 32
    refs = torch.ones(n_pages, dtype=torch.int32, device="cuda")
    refs[-8:] = 0                                                    # only the last pages are free
    z = lambda *s: torch.zeros(s, dtype=torch.int32, device="cuda")  # noqa: E731
    pages = K.Pages(pool, refs, z(3, 4), z(3), z(3), page, d)
    n = 100
    start, _ = K.pages_extend(pages, dev([n]), seq=dev([0]))
    x = normal((2, 1, 1, Hkv, n, d), "bf16", 1).cuda()
    K.pages_append(x[0], x[1], pages, start, seq=dev([0]))
    assert pages.table[0, :2].tolist() == [n_pages - 8, n_pages - 7]
    K.pages_fork(pages, dev([0]), dev([1]))
    start, missing = K.pages_extend(pages, dev([n]), seq=dev([2]))
    idx = torch.arange(n - 1, -1, -1, dtype=torch.int32, device="cuda").expand(1, 1, Hkv, n).contiguous()
    K.pages_select(pages, dev([0]), idx, torch.full((1, 1, Hkv), n, dtype=torch.int32, device="cuda"), dev([2]), start)
    assert missing.item() == 0
    k, v = K.pages_read(pages, n, dtype=torch.float32)
    want = [O.mx4_round(t[0, 0].double().cpu().numpy()) for t in x]
    for got, w in ((k, want[0]), (v, want[1])):
        got = got[0].double().cpu().numpy()
        assert np.array_equal(got[0], w) and np.array_equal(got[1], w) and np.array_equal(got[2], w[:, ::-1])
    assert not pool[:, :n_pages - 8].any()                           # nothing landed 4 GB lower
    q = normal((1, 3, Hkv, d), "bf16", 2).cuda()
    out = K.decode_pages(q, pages)
    for s in range(3):
        ref, mag, top = _decode_ref(q[0, s].double().cpu().numpy(), want[0], want[1], 1)
        check_decode(out[0, s].cpu().numpy(), ref, mag, top)


def test_millions_of_tokens(K):
    """A table that names one page over and over: 8.4 million tokens to read (4.3 GB of float32 rows) and to attend
    to.  The softmax over copies of a page is that over the page."""
    Hkv, d, page = 1, 128, 32
    M = (1 << 18) + 4
    z = lambda *s: torch.zeros(s, dtype=torch.int32, device="cuda")  # noqa: E731
    one = K.Pages(torch.zeros((1, 1, Hkv, K.page_bytes(page, d)), dtype=torch.uint8, device="cuda"), z(1), z(1, M), z(1),
                  z(1), page, d)
    start, _ = K.pages_extend(one, dev([page]))
    x = normal((2, 1, 1, Hkv, page, d), "bf16", 3).cuda()
    K.pages_append(x[0], x[1], one, start)
    one.held.fill_(M)
    one.length.fill_(M * page)
    T = M * page
    k_out = torch.empty((1, 1, Hkv, T, d), dtype=torch.float32, device="cuda")
    v_out = torch.empty((1, 1, Hkv, T, d), dtype=torch.float32, device="cuda")
    assert k_out.numel() * 4 > 1 << 32
    K.pages_read(one, T, k_out=k_out, v_out=v_out)
    for got, t in ((k_out, x[0]), (v_out, x[1])):
        want = torch.from_numpy(O.mx4_round(t[0, 0, 0].double().cpu().numpy())).float().cuda()
        assert bool((got.view(M, page, d) == want).all())
    del k_out, v_out
    q = normal((1, 1, 4, d), "bf16", 4).cuda()
    out = K.decode_pages(q, one)
    k, v = (O.mx4_round(t[0, 0].double().cpu().numpy()) for t in x)
    ref, mag, top = _decode_ref(q[0, 0].double().cpu().numpy(), k, v, 4)
    # 2^18 steps of 32 tokens over 4096 waves are 64 additions each, 32 within a product and at most 1024 splits
    # merged: 1120 roundings of 2^-24 are 6.7e-5, inside the bound's 1e-4
    check_decode(out[0, 0].cpu().numpy(), ref, mag, top)


def test_source_rows_far_apart(K):
    """A strided view whose rows lie 32 MiB apart, the last one beyond 4 GiB."""
    d, N, far = 64, 140, 1 << 25
    buf = torch.zeros((N * far + 256) // 2, dtype=torch.bfloat16, device="cuda")
    view = torch.as_strided(buf, (1, 1, 1, N, d), (0, 0, 0, far // 2, 1))
    x = normal((1, 1, 1, N, d), "bf16", 5).cuda()
    view.copy_(x)
    pages = make(K, 1, 1, d, 32, 6, 1, 6)
    start, _ = K.pages_extend(pages, dev([N]))
    K.pages_append(view, view, pages, start)
    assert np.array_equal(rows_of(pages, 0)[1], O.mx4_round(x[0].double().cpu().numpy()))
    idx = torch.tensor([[[[N - 1, 3]]]], dtype=torch.int32, device="cuda")
    K.pages_compact(view, view, idx, torch.full((1, 1, 1), 2, dtype=torch.int32, device="cuda"), pages, start)
    got = rows_of(pages, 0)[0][0, 0, :2]
    assert np.array_equal(got, O.mx4_round(x[0, 0, 0, [N - 1, 3]].double().cpu().numpy()))


# ---------------------------------------------------------------------------
# together
# ---------------------------------------------------------------------------

def _step(K, pages, k, v, q, seq, one, out, start, missing, ws_book, ws, most):
    """One decode step: room for the new token, its rows, attention over all of them."""
    K.pages_extend(pages, one, seq=seq, start=start, missing=missing, workspace=ws_book)
    K.pages_append(k, v, pages, start, seq=seq)
    K.decode_pages(q, pages, max_tokens=most, seq=seq, out=out, workspace=ws)


def test_captured_decode_loop(K):
    """A captured step replayed over 70 tokens (pages are taken on the way) equals the eager loop, and an eager step
    on a second cache between the replays changes neither."""
    L, B, Hkv, G, d, page, n0, steps = 2, 3, 2, 4, 128, 32, 50, 70
    lengths = [n0, 1, 33]
    qs = normal((steps, L, B, Hkv * G, d), "bf16", 1).cuda()
    ks, vs = normal((steps, L, B, Hkv, 1, d), "bf16", 2).cuda(), normal((steps, L, B, Hkv, 1, d), "bf16", 3).cuda()

    def fresh():
        pages, _, _ = _filled(K, L, Hkv, d, page, lengths, spare=20)
        table = torch.full((B, 6), -1, dtype=torch.int32, device="cuda")
        table[:, :pages.c.M] = pages.table
        pages = K.Pages(pages.pool, pages.refs, table, pages.held, pages.length, page, d)
        most = 6 * page
        bufs = dict(out=torch.zeros((L, B, Hkv * G, d), device="cuda"), start=dev([0] * B), missing=dev([0]),
                    ws_book=torch.empty(K.pages_workspace_size(pages.c.n_pages, B, B), dtype=torch.uint8, device="cuda"),
                    ws=torch.empty(K.decode_pages_workspace_size(L, B, Hkv * G, Hkv, most, d), dtype=torch.uint8,
                                   device="cuda"), seq=dev([2, 0, 1]), one=dev([1] * B), most=most)
        return pages, bufs

    pages, bufs = fresh()
    want = []
    for i in range(steps):
        _step(K, pages, ks[i], vs[i], qs[i], **bufs)
        want.append(bufs["out"].clone())
    end = [x.clone() for x in (pages.refs, pages.held, pages.length)]

    pages, bufs = fresh()
    other, obufs = fresh()
    q, k, v = qs[0].clone(), ks[0].clone(), vs[0].clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        _step(K, pages, k, v, q, **bufs)
    for i in range(steps):
        q.copy_(qs[i]); k.copy_(ks[i]); v.copy_(vs[i])
        graph.replay()
        if i % 9 == 0:
            _step(K, other, ks[i], vs[i], qs[i], **obufs)
            torch.cuda.synchronize()
        assert torch.equal(bufs["out"], want[i]), i
        assert bufs["missing"].item() == 0
    for a, b in zip(end, (pages.refs, pages.held, pages.length)):
        assert torch.equal(a, b)


def test_calls_on_another_stream(K):
    lengths = [700, 64]
    pages, _, _ = _filled(K, 1, 2, 128, 64, lengths, extra_slots=2, spare=30)
    q = normal((1, 2, 8, 128), "bf16", 3).cuda()
    want = K.decode_pages(q, pages, seq=dev([0, 1]))
    src, dst, one = dev([0, 1]), dev([2, 3]), dev([2])
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())      # all inputs are made before this
    done, _ = K.pages_fork(pages, src, dst, stream=s)
    got = K.decode_pages(q, pages, seq=dst, stream=s)
    k, _ = K.pages_read(pages, 700, seq=one, stream=s)
    s.synchronize()
    assert done.tolist() == [1, 1] and torch.equal(got, want)
    assert np.array_equal(k[0, 0].double().cpu().numpy(), rows_of(pages, 0)[0][0])


def test_forked_sequences_go_their_own_ways(K):
    """Children share the parent's full pages, write behind them, and outlive it; freed pages are used again."""
    L, Hkv, d, page = 2, 2, 64, 32
    pages, k0, v0 = _filled(K, L, Hkv, d, page, [75], extra_slots=3, spare=6)
    done, _ = K.pages_fork(pages, dev([0, 0]), dev([1, 2]))
    assert done.tolist() == [1, 1]
    x = normal((L, 3, Hkv, 40, d), "bf16", 8).cuda()
    new = dev([1, 40, 23])
    start, missing = K.pages_extend(pages, new, seq=dev([0, 1, 2]))
    K.pages_append(x, x, pages, start, n_new=new, seq=dev([0, 1, 2]))
    K.pages_free(pages, dev([0]))
    y = normal((L, 1, Hkv, 64, d), "bf16", 9).cuda()
    start, missing = K.pages_extend(pages, dev([64]), seq=dev([3]))   # takes what the parent left
    assert missing.item() == 0
    K.pages_append(y, y, pages, start, seq=dev([3]))
    base = O.mx4_round(k0[:, 0].double().cpu().numpy())
    more = O.mx4_round(x.double().cpu().numpy())
    for slot, n in ((1, 40), (2, 23)):
        k, _ = rows_of(pages, slot)
        assert np.array_equal(k[:, :, :75], base) and np.array_equal(k[:, :, 75:], more[:, slot, :, :n])
    assert np.array_equal(rows_of(pages, 3)[1], O.mx4_round(y[:, 0].double().cpu().numpy()))
    K.pages_free(pages)
    assert not pages.refs.any()


# ---------------------------------------------------------------------------
# the eviction step into pages
# ---------------------------------------------------------------------------

def _workload(name, **kw):
    import workload as WL
    base = WL.get_workload("layer8k")
    f = dict(L=3, B=2, Hq=8, Hkv=2, N=700, W=16, d=64, pool_k=5, dtype="bf16", mix=base.mix, budgets=(0.2,))
    f.update(kw)
    wl = WL.Workload(name, **f)
    return WL, wl, WL.make_inputs(wl, device="cuda:0")


@pytest.mark.parametrize("chunks", [1, 2])
@pytest.mark.parametrize("dtype,d", [("bf16", 64), ("bf16", 128), ("f32", 128)])
def test_evict_into_pages_keeps_the_rows_of_the_dense_step(K, chunks, dtype, d):
    from paper_2607_13205_amd import pipeline
    WL, wl, inp = _workload("paged", dtype=dtype, d=d)
    alpha = WL.default_alpha(0.0)
    k_cap = K.role_allocate(inp["roles"], 4, alpha, 0.2, wl.W)[2]
    args = (inp["q"], inp["k"], inp["v"], inp["roles"], inp["roles_t"], alpha, 0.2, wl.W, wl.pool_k)
    dense = pipeline.alloc_buffers(inp["k"], wl.Hq, wl.W, 4, k_cap)
    _, kept = pipeline.evict(*args, dense)
    cache = pipeline.alloc_pages(wl.L, wl.Hkv, d, 40, 5, 2 * k_cap, page=32)
    bufs = pipeline.alloc_buffers(inp["k"], wl.Hq, wl.W, 4, k_cap, pages=cache)
    assert bufs.k_out is None and bufs.v_out is None
    slots = dev([3, 1])
    side = torch.cuda.Stream() if chunks > 1 else None
    for times in (1, 2):  # a second step packs behind the first
        _, kept2 = pipeline.evict(*args, bufs, chunks=chunks, side_stream=side, slots=slots)
        assert np.array_equal(kept, kept2) and bufs.missing.item() == 0
        assert bufs.start.tolist() == [(times - 1) * int(n) for n in kept]
        assert cache.length[slots.long()].tolist() == [times * int(n) for n in kept]
    for b, slot in enumerate((3, 1)):
        n = int(kept[b])
        for got, x in zip(rows_of(cache, slot), (dense.k_out, dense.v_out)):
            want = O.mx4_round(x[:, b, :, :n].double().cpu().numpy())
            assert np.array_equal(got[:, :, :n], want) and np.array_equal(got[:, :, n:], want)
    # no room: the first sample's pages are there, the second's are not
    small = pipeline.alloc_pages(wl.L, wl.Hkv, d, -(-int(kept[0]) // 32), 2, k_cap, page=32)
    bufs = pipeline.alloc_buffers(inp["k"], wl.Hq, wl.W, 4, k_cap, pages=small)
    pipeline.evict(*args, bufs)
    assert bufs.start.tolist() == [0, -1] and bufs.missing.item() == -(-int(kept[1]) // 32)
    assert small.length.tolist() == [int(kept[0]), 0]


def test_evict_into_pages_refusals(K):
    from paper_2607_13205_amd import pipeline
    WL, wl, inp = _workload("paged_no")
    cache = pipeline.alloc_pages(wl.L, wl.Hkv, wl.d, 4, 2, 64)
    with pytest.raises(ValueError):
        pipeline.alloc_buffers(inp["k"], wl.Hq, wl.W, 4, 60, with_v=False, pages=cache)
    with pytest.raises(ValueError):
        pipeline.alloc_buffers(inp["k"][:2], wl.Hq, wl.W, 4, 60, pages=cache)
    bufs = pipeline.alloc_buffers(inp["k"], wl.Hq, wl.W, 4, 60, pages=cache)
    with pytest.raises(ValueError):
        pipeline.StepGraph(inp["q"], inp["k"], inp["v"], inp["roles_t"], WL.default_alpha(0.0), wl.W, wl.pool_k, bufs)
    for kw in (dict(page=48), dict(d=96)):
        with pytest.raises(ValueError):
            pipeline.alloc_pages(**dict(dict(L=1, Hkv=1, d=64, n_pages=4, slots=1, max_tokens=10), **kw))


def test_a_sequence_from_prompt_to_end(K):
    """Eviction into pages, decode steps, two continuations, a second eviction of what has grown, and the end."""
    from paper_2607_13205_amd import pipeline
    WL, wl, inp = _workload("paged_life", B=1, N=900)
    L, Hkv, G, d, page = wl.L, wl.Hkv, wl.Hq // wl.Hkv, wl.d, 32
    alpha = WL.default_alpha(0.0)
    k_cap = K.role_allocate(inp["roles"], 4, alpha, 0.2, wl.W)[2]
    cache = pipeline.alloc_pages(L, Hkv, d, 60, 4, 400, page=page)
    bufs = pipeline.alloc_buffers(inp["k"], wl.Hq, wl.W, 4, k_cap, pages=cache)
    slot0 = dev([2])
    _, kept = pipeline.evict(inp["q"], inp["k"], inp["v"], inp["roles"], inp["roles_t"], alpha, 0.2, wl.W, wl.pool_k,
                             bufs, slots=slot0)
    n = int(kept[0])
    rows = [x[:, :, :] for x in rows_of(cache, 2)]                   # [L, Hkv, n, d], as held

    def step(slots, seed, rows):
        B = len(slots)
        seq = dev(slots)
        k, v = normal((L, B, Hkv, 1, d), "bf16", seed).cuda(), normal((L, B, Hkv, 1, d), "bf16", seed + 1).cuda()
        q = normal((L, B, wl.Hq, d), "bf16", seed + 2).cuda()
        start, missing = K.pages_extend(cache, dev([1] * B), seq=seq)
        K.pages_append(k, v, cache, start, seq=seq)
        out = K.decode_pages(q, cache, seq=seq)
        assert missing.item() == 0
        for b in range(B):
            for i, x in enumerate((k, v)):
                rows[b][i] = np.concatenate([rows[b][i], O.mx4_round(x[:, b].double().cpu().numpy())], axis=2)
            for l in range(L):
                want, mag, top = _decode_ref(q[l, b].double().cpu().numpy(), rows[b][0][l], rows[b][1][l], G)
                check_decode(out[l, b].cpu().numpy(), want, mag, top)

    first = [list(rows)]
    for t in range(5):
        step([2], 10 * t, first)
    done, _ = K.pages_fork(cache, dev([2, 2]), dev([0, 3]))
    assert done.tolist() == [1, 1]
    K.pages_free(cache, slot0)
    two = [list(first[0]), list(first[0])]
    for t in range(40):
        step([0, 3], 1000 + 10 * t, two)
    # a second eviction of slot 0: scored on its keys as read back, one bucket, window kept
    N2 = n + 45
    k2, _ = K.pages_read(cache, N2, seq=dev([0]))
    q2 = normal((L, 1, wl.Hq, wl.W, d), "bf16", 5).cuda()
    score = K.snapkv_score(q2, k2, wl.pool_k)
    zero = torch.zeros((1, N2), dtype=torch.int8, device="cuda")
    keep = 70
    idx, count = K.topk_select(score, zero, dev([[keep - wl.W]]), wl.W, 1, keep)
    start, missing = K.pages_extend(cache, dev([keep]), seq=slot0)
    K.pages_select(cache, dev([0]), idx, count, slot0, start)
    K.pages_free(cache, dev([0]))
    assert missing.item() == 0 and (count == keep).all()
    at = idx[:, 0].cpu().numpy()
    third = [[np.take_along_axis(x, at[..., None].astype(np.int64), axis=2) for x in two[0]]]
    for got, want in zip(rows_of(cache, 2), third[0]):
        assert np.array_equal(got, want)
    step([2], 7, third)
    step([3], 8, [two[1]])
    K.pages_free(cache)
    assert not cache.refs.any() and not cache.length.any()


def _bad_values(v):
    """Tensors of v's shape and type that cannot be packed: name -> tensor."""
    off = torch.empty(v.numel() + 8, dtype=v.dtype, device="cuda")[1:v.numel() + 1].view(v.shape)
    odd = torch.empty(v.shape[:-1] + (v.shape[-1] + 1,), dtype=v.dtype, device="cuda")[..., :-1]
    apart = torch.empty(v.shape[:-1] + (2 * v.shape[-1],), dtype=v.dtype, device="cuda")[..., ::2]
    far = torch.empty(v.shape, dtype=v.dtype, device="cuda").permute(4, 0, 1, 2, 3).contiguous().permute(1, 2, 3, 4, 0)
    return dict(unaligned=off, odd_rows=odd, channels_apart=apart, channels_outermost=far, on_the_host=v.cpu())


@pytest.mark.parametrize("chunks", [1, 2])
def test_a_refused_evict_leaves_the_sequences_alone(K, chunks):
    """Whatever is wrong with the values, the slots or the layers: nothing is queued, and no sequence is longer."""
    from paper_2607_13205_amd import pipeline
    WL, wl, inp = _workload("paged_refused")
    alpha = WL.default_alpha(0.0)
    k_cap = K.role_allocate(inp["roles"], 4, alpha, 0.2, wl.W)[2]
    cache = pipeline.alloc_pages(wl.L, wl.Hkv, wl.d, 40, 5, 2 * k_cap, page=32)
    bufs = pipeline.alloc_buffers(inp["k"], wl.Hq, wl.W, 4, k_cap, pages=cache)
    side = torch.cuda.Stream() if chunks > 1 else None
    bufs.score.fill_(7.0)
    slots = dev([3, 1])

    def refused(q=inp["q"], v=inp["v"], slots=slots, bufs=bufs, **kw):
        with pytest.raises((ValueError, K.KveError)):
            pipeline.evict(q, inp["k"], v, inp["roles"], inp["roles_t"], alpha, 0.2, wl.W, wl.pool_k, bufs,
                           chunks=chunks, side_stream=side, slots=slots, **kw)
        torch.cuda.synchronize()
        assert not cache.length.any() and not cache.held.any() and not cache.refs.any(), "the sequences were extended"
        assert (bufs.score == 7.0).all(), "the score was queued"

    for bad in _bad_values(inp["v"]).values():
        refused(v=bad)
    for bad in (slots.long(), dev([3]), slots.cpu(), dev([3, 9, 1, 9])[::2]):
        refused(slots=bad)
    refused(q=inp["q"][:2].contiguous())                             # the layers of a first chunk, and no more
    refused(lse_win=torch.zeros((2, wl.B, wl.Hq, wl.W), device="cuda"))
    one = pipeline.alloc_pages(wl.L, wl.Hkv, wl.d, 40, 1, 2 * k_cap, page=32)
    few = pipeline.alloc_buffers(inp["k"], wl.Hq, wl.W, 4, k_cap, pages=one)
    few.score.fill_(7.0)
    refused(slots=None, bufs=few)                                    # two samples, one slot
    assert not one.length.any()
    pipeline.evict(inp["q"], inp["k"], inp["v"], inp["roles"], inp["roles_t"], alpha, 0.2, wl.W, wl.pool_k, bufs,
                   chunks=chunks, side_stream=side, slots=slots)     # and the step itself still runs
    assert (cache.length[slots.long()] > 0).all()


def test_more_samples_than_a_bookkeeping_call_takes(K):
    from paper_2607_13205_amd import pipeline
    cache = pipeline.alloc_pages(1, 1, 64, 8, 1100, 64)
    with pytest.raises(ValueError, match="1025"):
        pipeline.alloc_buffers(torch.zeros((1, 1025, 1, 16, 64), dtype=torch.bfloat16, device="cuda"), 1, 4, 1, 8,
                               pages=cache)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("bad", [-1, "n_pages", 1 << 30, -(1 << 31)])
def test_fork_of_a_sequence_whose_last_page_is_missing(K, d, bad):
    """The child has the rows that the parent has, and not what a recycled page held: read, attended to, extended and
    freed like the parent."""
    page = 32
    pages, k, v = _filled(K, 2, 2, d, page, [75, 40], extra_slots=2, spare=4)
    bad = pages.c.n_pages if bad == "n_pages" else bad
    pages.table[0, 2] = bad
    b = book(pages)
    done, missing = K.pages_fork(pages, dev([0, 1]), dev([2, 3]))
    want, lack, _ = b.fork([0, 1], [2, 3])
    assert done.tolist() == want == [1, 1] and missing.item() == lack == 0
    same_book(pages, b)
    outs = [torch.full((2, 4, 2, 75, d), 7.0, dtype=torch.bfloat16, device="cuda") for _ in (0, 1)]
    K.pages_read(pages, 75, k_out=outs[0], v_out=outs[1])
    for got in outs:
        assert torch.equal(got[:, :2], got[:, 2:]) and (got[:, 2, :, 64:] == 7.0).all()
        assert not (got[:, 3, :, :40] == 7.0).all(-1).any()
    q = normal((2, 1, 4, d), "bf16", 3).expand(2, 4, 4, d).contiguous().cuda()
    out = K.decode_pages(q, pages)
    assert torch.equal(out[:, 2], out[:, 0]) and torch.equal(out[:, 3], out[:, 1])
    before = pages.pool.clone()
    start, missing = K.pages_extend(pages, dev([3]), seq=dev([2]))
    K.pages_append(k[:, :1, :, :3], v[:, :1, :, :3], pages, start, seq=dev([2]))
    assert start.tolist() == [75] and missing.item() == 0 and torch.equal(before, pages.pool)
    K.pages_free(pages)
    b.extend([2], [3])
    b.free(range(4))
    same_book(pages, b)


def test_fork_takes_all_layers(K):
    """The bookkeeping is every layer's: a fork of some of them would leave the others without the copied rows."""
    pages, _, _ = _filled(K, 3, 1, 64, 32, [40], extra_slots=1)
    before = [getattr(pages, n).clone() for n in ("refs", "held", "length")]
    for part in (pages.layers(0, 2), pages.layers(1, 3), pages.layers(0, 2).layers(0, 2), pages.layers(2, 3)):
        with pytest.raises(ValueError, match="all layers"):
            K.pages_fork(part, dev([0]), dev([1]))
    for x, n in zip(before, ("refs", "held", "length")):
        assert torch.equal(x, getattr(pages, n))
    done, _ = K.pages_fork(pages.layers(0, 3), dev([0]), dev([1]))
    assert done.tolist() == [1]
    for a, b in zip(rows_of(pages, 0), rows_of(pages, 1)):
        assert np.array_equal(a, b)


# ---------------------------------------------------------------------------
# more forms of the calls
# ---------------------------------------------------------------------------

@pytest.mark.parametrize("d", [64, 128])
def test_select_within_one_sequence(K, d):
    """Source and destination are one slot: the rows kept are moved behind the others."""
    n, cap = 90, 37
    pages, k, v = _filled(K, 2, 2, d, 32, [n, n], spare=8)
    pages2 = K.Pages(pages.pool, pages.refs, torch.cat([pages.table, torch.full_like(pages.table, -1)], 1).contiguous(),
                     pages.held, pages.length, 32, d)
    r = np.random.default_rng(d)
    both = dev([0, 1])
    start, missing = K.pages_extend(pages2, dev([cap, cap]), seq=both)
    assert start.tolist() == [n, n] and missing.item() == 0
    idx = np.stack([np.sort(r.permutation(n)[:cap]) for _ in range(8)]).reshape(2, 2, 2, cap)
    K.pages_select(pages2, both, dev(idx), dev(np.full((2, 2, 2), cap)), both, start)
    for s in (0, 1):
        for got, x in zip(rows_of(pages2, s), (k, v)):
            base = O.mx4_round(x[:, s].double().cpu().numpy())
            assert np.array_equal(got[:, :, :n], base)
            assert np.array_equal(got[:, :, n:], np.take_along_axis(base, idx[:, s, ..., None], axis=2))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("which", ["k", "v"])
def test_keys_and_values_of_different_layouts(K, dtype, which):
    """One dense, the other token-major with room between its rows."""
    L, B, Hkv, N, d = 2, 2, 3, 70, 64
    x = {n: normal((L, B, Hkv, N, d), dtype, i) for i, n in enumerate("kv")}
    at = {n: t.cuda() for n, t in x.items()}
    wide = torch.zeros((L, B, N, Hkv, d + 8), dtype=TORCH[dtype], device="cuda")
    at[which] = wide.permute(0, 1, 3, 2, 4)[..., :d]
    at[which].copy_(x[which])
    pages = make(K, L, Hkv, d, 32, 16, B, 5)
    start, _ = K.pages_extend(pages, dev([N, N]))
    K.pages_append(at["k"], at["v"], pages, start)
    want = {n: O.mx4_round(t.double().numpy()) for n, t in x.items()}
    for s in range(B):
        for got, n in zip(rows_of(pages, s), "kv"):
            assert np.array_equal(got, want[n][:, s])
    start, _ = K.pages_extend(pages, dev([4, 4]))
    idx = dev(np.broadcast_to([69, 0, 33, 5], (L, B, Hkv, 4)))
    K.pages_compact(at["k"], at["v"], idx, dev(np.full((L, B, Hkv), 4)), pages, start)
    for s in range(B):
        for got, n in zip(rows_of(pages, s), "kv"):
            assert np.array_equal(got[:, :, N:], want[n][:, s][:, :, [69, 0, 33, 5]])


@pytest.mark.parametrize("chunks", [1, 2])
def test_evict_of_strided_values_into_pages(K, chunks):
    """Token-major values beside dense keys: the rows of the dense step."""
    from paper_2607_13205_amd import pipeline
    WL, wl, inp = _workload("paged_views")
    alpha = WL.default_alpha(0.0)
    k_cap = K.role_allocate(inp["roles"], 4, alpha, 0.2, wl.W)[2]
    v = inp["v"].permute(0, 1, 3, 2, 4).contiguous().permute(0, 1, 3, 2, 4)
    assert not v.is_contiguous()
    side = torch.cuda.Stream() if chunks > 1 else None
    caches = []
    for values in (inp["v"], v):
        cache = pipeline.alloc_pages(wl.L, wl.Hkv, wl.d, 40, wl.B, k_cap, page=32)
        bufs = pipeline.alloc_buffers(inp["k"], wl.Hq, wl.W, 4, k_cap, pages=cache)
        pipeline.evict(inp["q"], inp["k"], values, inp["roles"], inp["roles_t"], alpha, 0.2, wl.W, wl.pool_k, bufs,
                       chunks=chunks, side_stream=side)
        caches.append(cache)
    assert caches[0].length.tolist() == caches[1].length.tolist() and caches[0].length.min() > 0
    for s in range(wl.B):
        for a, b in zip(rows_of(caches[0], s), rows_of(caches[1], s)):
            assert np.array_equal(a, b)


# ---------------------------------------------------------------------------
# more forms of the decode
# ---------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("G", [1, 2, 3, 4, 5, 8, 9, 16])
def test_decode_keeps_all_bits_of_the_weights(K, G, d, dtype):
    """Results that hang on the last 8 of the 24 bits of a weight, and of a float32 query: two tokens in one wave's step,
    in the steps of two waves, within a split and in different ones."""
    from tests import paged_decode_cases as C
    worst = 0.0
    for n, at, most in ((2, (0, 1), 2), (2, (1, 0), 512), (64, (3, 45), 64), (200, (67, 94), 200),
                        (2300, (130, 147), 2304), (2300, (5, 2200), 2304), (2300, (2299, 0), None)):
        q, k, v, want = C.case(G, d, dtype, n, at)
        pages = make(K, 1, 1, d, 32, 80, 1, 80)
        start, _ = K.pages_extend(pages, dev([n]))
        k, v = (torch.from_numpy(x).float()[None, None, None].cuda() for x in (k, v))
        K.pages_append(k, v, pages, start)
        out = K.decode_pages(torch.from_numpy(q).to(TORCH[dtype])[None, None].cuda(), pages, max_tokens=most, scale=1.0)
        worst = max(worst, float(np.abs(out[0, 0].double().cpu().numpy() - want).max()))
        assert worst <= C.BOUND, (n, at, worst / C.U)
    report(f"paged decode, low bits of the weights, units of 2^-24: g{G} d{d} {dtype}", round(worst / C.U, 2))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("G,d,n,most", [(4, 128, 64, 64), (4, 64, 600, 600), (8, 128, 600, 600), (16, 128, 64, 64),
                                        (3, 128, 2500, 2500)])
def test_decode_of_exact_logits_is_float32(K, G, d, n, most, dtype):
    """Small whole numbers as queries and four-bit values with unit scales: the products are exact, what is left is the
    softmax and the sums in float32.  With logits of at most X (in powers of two), of a weight: log2(e) rounded X / 2,
    reference, product and difference X + X + 2 X, times ln 2, exp2 2, a factor and its product in either merge 3 each:
    3.2 X + 8 units of 2^-24.  Of a sum: 32 tokens and three parts per step of a wave, the waves of a split and the
    splits added: 96 steps + 16 + 32.  Both twice, for numerator and denominator, and the division 5."""
    r = np.random.default_rng(n + G)
    q = r.integers(-3, 4, (2, G, d)).astype(np.float64)
    k, v = (r.choice([-1.0, 1.0], (2, n, d)) * O.E2M1[r.integers(0, 8, (2, n, d))] for _ in "kv")
    k[..., ::32], v[..., ::32] = 4.0, -6.0                           # every block's unit is one
    assert np.array_equal(O.mx4_round(k), k) and np.array_equal(O.mx4_round(v), v)
    pages = make(K, 1, 2, d, 64, -(-n // 64), 1, -(-n // 64))
    start, _ = K.pages_extend(pages, dev([n]))
    K.pages_append(*(torch.from_numpy(x).float()[None, None].cuda() for x in (k, v)), pages, start)
    out = K.decode_pages(torch.from_numpy(q.reshape(1, 1, 2 * G, d)).to(TORCH[dtype]).cuda(), pages, max_tokens=most,
                         scale=2.0 ** -6)
    out = out[0, 0].double().cpu().numpy().reshape(2, G, d)
    x = q @ k.transpose(0, 2, 1) / 64.0
    w = np.exp(x - x.max(-1, keepdims=True))
    w /= w.sum(-1, keepdims=True)
    steps = -(-min(n, 128) // 128) if most > 2048 else -(-n // (32 * 12))    # a split, or all waves of a unit
    units = 2 * (3.2 * np.abs(x).max() * 1.4427 + 8 + 96 * steps + 48) + 5
    err = np.abs(out - w @ v) / (w @ np.abs(v))
    assert err.max() <= units * 2.0 ** -24, (err.max() * 2.0 ** 24, units)
    report(f"paged decode, exact logits, err/bound: g{G} d{d} n{n} {dtype}", round(float(err.max() * 2.0 ** 24 / units), 4))


@pytest.mark.parametrize("L,B,Hkv,G,d,dtype,longest,most", [
    (1, 3, 64, 4, 128, "bf16", 2300, 2304),   # 16 splits a pair: one wave per row merges them
    (5, 2, 16, 2, 128, "bf16", 2200, None),   # 12
    (1, 2, 64, 9, 128, "bf16", 2200, None),   # the same for sixteen heads
    (1, 2, 64, 1, 128, "f32", 2300, 2300),
    (1, 2, 64, 3, 64, "f32", 2300, 2300),
    (2, 20, 8, 4, 128, "f32", 300, 512),      # two sequences to a compute unit, of six waves
    (2, 20, 8, 11, 128, "bf16", 300, 512),
    (2, 20, 8, 4, 128, "bf16", 300, 512),     # of eight
    (2, 20, 8, 2, 64, "f32", 300, 512),
    (3, 40, 8, 2, 128, "f32", 200, 200),      # four
    (3, 40, 8, 12, 128, "f32", 200, 200),
    (1, 70, 1, 16, 128, "f32", 1500, None),   # splits of more sequences than a wave has lanes
])
def test_decode_of_every_workgroup_form(K, L, B, Hkv, G, d, dtype, longest, most):
    """Ragged lengths, empty sequences and slots in any order, for both row sizes and query types."""
    r = np.random.default_rng(L * B + d)
    lengths = [longest, 0] + [int(r.integers(0, longest + 1)) for _ in range(B - 2)]
    page = 64
    pages = make(K, L, Hkv, d, page, sum(-(-n // page) for n in lengths) + 1, B, 40)
    start, missing = K.pages_extend(pages, dev(lengths))
    assert missing.item() == 0
    g = torch.Generator(device="cuda").manual_seed(B)
    k, v = (torch.randn((L, B, Hkv, longest, d), generator=g, device="cuda", dtype=torch.float32).bfloat16()
            for _ in "kv")
    K.pages_append(k, v, pages, start, n_new=dev(lengths))
    order = r.permutation(B)
    q = normal((L, B, Hkv * G, d), dtype, 78).cuda()
    out = torch.full((L, B, Hkv * G, d), float("nan"), device="cuda")
    K.decode_pages(q, pages, max_tokens=most, seq=dev(order), out=out)
    assert torch.isfinite(out).all()
    k, v = K.pages_read(pages, longest, seq=dev(order))
    for l in sorted({0, L - 1}):
        qn, on = q[l].double().cpu().numpy(), out[l].double().cpu().numpy()
        kl, vl = k[l].double().cpu().numpy(), v[l].double().cpu().numpy()
        for i, s in enumerate(order):
            n = lengths[s]
            want, mag, top = _decode_ref(qn[i], kl[i, :, :n], vl[i, :, :n], G)
            check_decode(on[i], want, mag, top, f"sample {i} of {n} layer {l}")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_captured_decode_of_several_splits(K, dtype):
    """A captured step whose bound makes splits, replayed while lengths cross a split's and a page's border: the search,
    the ranges left for the merge and the merge itself, against the eager loop."""
    B, Hkv, G, d, page, M, steps = 3, 2, 4, 128, 512, 6, 14
    lengths = [2040, 120, 1]
    qs = normal((steps, 1, B, Hkv * G, d), dtype, 1).cuda()
    ks, vs = (normal((steps, 1, B, Hkv, 1, d), "bf16", s).cuda() for s in (2, 3))

    def fresh():
        pages = make(K, 1, Hkv, d, page, 16, B, M, seed=2)
        start, _ = K.pages_extend(pages, dev(lengths))
        x = normal((2, 1, B, Hkv, max(lengths), d), "bf16", 4).cuda()
        K.pages_append(x[0], x[1], pages, start, n_new=dev(lengths))
        most = M * page
        size = K.decode_pages_workspace_size(1, B, Hkv * G, Hkv, most, d)
        return pages, dict(out=torch.zeros((1, B, Hkv * G, d), device="cuda"), start=dev([0] * B), missing=dev([0]),
                           ws_book=torch.empty(K.pages_workspace_size(16, B, B), dtype=torch.uint8, device="cuda"),
                           ws=torch.full((size,), 255, dtype=torch.uint8, device="cuda"), seq=dev([2, 0, 1]),
                           one=dev([1] * B), most=most)

    pages, bufs = fresh()
    want = []
    for i in range(steps):
        _step(K, pages, ks[i], vs[i], qs[i], **bufs)
        want.append(bufs["out"].clone())
    assert pages.length.tolist() == [n + steps for n in lengths]
    for s, i in ((0, 1), (1, 2), (2, 0)):
        k, v = rows_of(pages, s)
        ref, mag, top = _decode_ref(qs[-1][0, i].double().cpu().numpy(), k[0], v[0], G)
        check_decode(want[-1][0, i].cpu().numpy(), ref, mag, top)

    pages, bufs = fresh()
    other, obufs = fresh()
    q, k, v = qs[0].clone(), ks[0].clone(), vs[0].clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        _step(K, pages, k, v, q, **bufs)
    for i in range(steps):
        q.copy_(qs[i]); k.copy_(ks[i]); v.copy_(vs[i])
        graph.replay()
        if i % 4 == 0:
            _step(K, other, ks[i], vs[i], qs[i], **obufs)
            torch.cuda.synchronize()
        assert torch.equal(bufs["out"], want[i]), i
