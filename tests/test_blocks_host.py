"""The C ABI of the paged 8-bit cache on the CPU: exported symbols, sizes, and
every refusal, none of which may touch its buffers (the pointers are made up)."""

import ctypes
import os
import re

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P = 1 << 20  # an aligned address that no refused call may look at
N = None
BIG = 1 << 30


@pytest.fixture(scope="module")
def kve():
    from paper_2607_13205_amd.build import ensure_built
    ensure_built()
    import paper_2607_13205_amd as K
    return K


def _cache(kve, **kw):
    from paper_2607_13205_amd.pages import _CPages
    f = dict(pool=P, refs=P, table=P, held=P, length=P, L=2, n_pages=10, Hkv=2, d=128, page=64, S=4, M=3)
    f.update(kw)
    return _CPages(*(f[n] for n, _ in _CPages._fields_))


def _rotation(**kw):
    from paper_2607_13205_amd.blocks import _CRotation
    f = dict(cos=P, sin=P, position=P, P=100, r=64, pairs=0)
    f.update(kw)
    return _CRotation(*(f[n] for n, _ in _CRotation._fields_))


def test_every_declared_symbol_is_exported(kve):
    text = open(os.path.join(ROOT, "include", "kve_blocks.h")).read()
    names = sorted(set(re.findall(r"^(?:kve_status_t|size_t) (kve_[a-z0-9_]+)\(", text, re.M)))
    assert len(names) == 9 and sorted(kve.binding.EXPORTED_BLOCKS) == names
    lib = ctypes.CDLL(kve.binding._LIB_PATH)
    for n in names:
        assert hasattr(lib, n), n


def test_sizes(kve):
    import oracle as O
    for page in (32, 64, 128):
        for d in (64, 128):
            assert kve.block_bytes(page, d) == O.block_bytes(page, d)
            assert kve.block_bytes(page, d) % 128 == 0
    for page, d in ((0, 128), (16, 128), (48, 128), (256, 128), (-32, 64), (64, 96), (64, 0)):
        assert kve.block_bytes(page, d) == 0
    top, dec = kve.blocks_top_workspace_size, kve.decode_blocks_workspace_size
    assert top(1, 2, 3, 1, 1000, 32) >= 2 * 3 * 32 * 4 and top(1, 2, 3, 1, 1000, 32) % 256 == 0
    for args in ((0, 1, 1, 1, 9, 32), (1, 0, 1, 1, 9, 32), (1, 1, 0, 1, 9, 32), (1, 1, 1, 0, 9, 32),
                 (1, 1, 1, 1, 0, 32), (1, 1, 1, 1, 9, 256), (1, 1, 1, 1, (1 << 30) + 1, 32), (1, 1 << 24, 1, 1, 9, 32)):
        assert top(*args) == 0
    assert dec(1, 4, 32, 8, 1, 128) > 0
    for args in ((0, 4, 32, 8, 1, 128), (1, 0, 32, 8, 1, 128), (1, 4, 30, 8, 1, 128), (1, 4, 32, 8, 0, 128),
                 (1, 4, 32, 8, 1, 96), (1, 1 << 24, 32, 8, 1, 128)):
        assert dec(*args) == 0


def _calls(kve, c):
    lib, r = kve.binding.LIB, ctypes.byref(c) if c is not None else None
    rot0 = ctypes.byref(_rotation())

    def append(k=P, ks=N, v=P, vs=N, dt=0, B=2, T=5, new=P, start=P, seq=P, rot=rot0, q=P, qs=N, Hq=4, out=2 * P):
        return lib.kve_blocks_append(k, ks, v, vs, dt, B, T, new, start, seq, r, rot, q, qs, Hq, out, N)
    return {
        "append": append,
        "compact": lambda k=P, ks=N, v=P, vs=N, dt=0, B=2, n=9, idx=P, count=P, cap=5, start=P, seq=P:
            lib.kve_blocks_compact(k, ks, v, vs, dt, B, n, idx, count, cap, start, seq, r, N),
        "read": lambda dt=0, B=2, T=5, seq=P, start=P, count=P, k=P, v=P:
            lib.kve_blocks_read(r, dt, B, T, seq, start, count, k, v, N),
        "bounds": lambda dt=0, B=2, n=5, seq=P, first=P, lo=P, hi=P:
            lib.kve_blocks_bounds(r, dt, B, n, seq, first, lo, hi, N),
        "top": lambda q=P, dt=0, B=2, Hq=8, T=1, most=9, start=P, seq=P, k=4, first=1, last=1, out=P, ws=P, wsb=BIG:
            lib.kve_blocks_top(q, dt, r, B, Hq, T, most, start, seq, k, first, last, out, ws, wsb, N),
        "decode": lambda q=P, dt=0, B=2, Hq=8, T=1, most=9, start=P, seq=P, top=P, k=4, scale=0.0, out=P, ws=P, wsb=BIG:
            lib.kve_decode_blocks(q, dt, r, B, Hq, T, most, start, seq, top, k, scale, out, ws, wsb, N),
    }


def _refused(kve, status, call, **kw):
    got = call(**kw)
    assert got == status, (kw, got, kve.last_error())
    assert kve.last_error()


BAD_CACHES = [(dict(refs=0), 1), (dict(table=0), 1), (dict(held=0), 1), (dict(length=0), 1), (dict(L=0), 1),
              (dict(n_pages=0), 1), (dict(Hkv=-1), 1), (dict(S=0), 1), (dict(M=0), 1), (dict(page=48), 1),
              (dict(page=16), 1), (dict(page=256), 1), (dict(d=96), 2), (dict(M=1 << 26), 2),
              (dict(n_pages=(1 << 30) + 1), 2), (dict(S=1 << 30, M=3), 2), (dict(pool=0), 1), (dict(pool=P + 8), 1)]


def test_bad_caches_are_refused(kve):
    for call in _calls(kve, None).values():
        _refused(kve, 1, call)
    for kw, status in BAD_CACHES:
        for call in _calls(kve, _cache(kve, **kw)).values():
            _refused(kve, status, call)


REFUSALS = {
    "append": [(dict(k=0), 1), (dict(v=0), 1), (dict(start=0), 1), (dict(B=0), 1), (dict(T=-1), 1),
               (dict(seq=0, B=5), 1), (dict(dt=2), 2), (dict(k=P + 8), 1), (dict(v=P + 8), 1), (dict(B=1 << 24), 2),
               (dict(T=(1 << 30) + 1), 2), (dict(q=0), 1), (dict(out=0), 1), (dict(rot=N), 1), (dict(out=P), 1),
               (dict(Hq=0), 1), (dict(q=P + 8), 1), (dict(out=P + 8), 1), (dict(Hq=1 << 20, T=300), 2),
               (dict(T=1 << 28, B=1, q=0, out=0), 2)],
    "compact": [(dict(k=0), 1), (dict(v=0), 1), (dict(start=0), 1), (dict(idx=0), 1), (dict(count=0), 1),
                (dict(n=0), 1), (dict(n=(1 << 30) + 1), 1), (dict(cap=-1), 1), (dict(seq=0, B=5), 1),
                (dict(dt=-1), 2), (dict(k=P + 8), 1), (dict(B=1 << 24), 2), (dict(cap=1 << 28, B=1), 2)],
    "read": [(dict(k=0, v=0), 1), (dict(k=P + 8), 1), (dict(v=P + 4), 1), (dict(B=0), 1), (dict(T=-1), 1),
             (dict(seq=0, B=5), 1), (dict(dt=7), 2), (dict(B=1 << 24), 2), (dict(T=1 << 27), 2)],
    "bounds": [(dict(lo=0, hi=0), 1), (dict(lo=P + 8), 1), (dict(hi=P + 4), 1), (dict(B=0), 1), (dict(n=-1), 1),
               (dict(seq=0, B=5), 1), (dict(dt=7), 2), (dict(B=1 << 24), 2), (dict(n=1 << 27), 2)],
    "top": [(dict(q=0), 1), (dict(out=0), 1), (dict(q=P + 8), 1), (dict(Hq=0), 1), (dict(Hq=7), 1), (dict(T=0), 1),
            (dict(most=0), 1), (dict(most=193), 1), (dict(B=0), 1), (dict(seq=0, B=5), 1), (dict(dt=3), 2),
            (dict(k=1), 1), (dict(k=0, first=0, last=0), 1), (dict(first=-1), 1), (dict(last=-1), 1),
            (dict(first=3, last=2), 1), (dict(first=(1 << 31) - 1, last=(1 << 31) - 1), 1),
            (dict(k=(1 << 25) + 1), 2), (dict(ws=0), 3), (dict(wsb=15), 3), (dict(ws=P + 16), 1),
            (dict(B=1 << 24), 2), (dict(T=1 << 24), 2)],
    "decode": [(dict(q=0), 1), (dict(out=0), 1), (dict(q=P + 8), 1), (dict(Hq=0), 1), (dict(Hq=7), 1),
               (dict(Hq=34), 2), (dict(T=0), 1), (dict(T=-3), 1), (dict(most=0), 1), (dict(most=193), 1),
               (dict(scale=-1.0), 1), (dict(scale=float("nan")), 1), (dict(scale=float("inf")), 1), (dict(B=0), 1),
               (dict(seq=0, B=5), 1), (dict(dt=3), 2), (dict(top=0), 1), (dict(k=0), 1), (dict(k=-1), 1),
               (dict(k=-1, top=0), 1), (dict(k=(1 << 24) + 1), 2), (dict(ws=0), 3), (dict(wsb=15), 3),
               (dict(ws=P + 16), 1), (dict(B=1 << 24), 2), (dict(T=1 << 23), 2)],
}


@pytest.mark.parametrize("name", sorted(REFUSALS))
def test_bad_arguments_are_refused(kve, name):
    call = _calls(kve, _cache(kve))[name]
    for kw, status in REFUSALS[name]:
        _refused(kve, status, call, **kw)


def test_bad_rotations_are_refused(kve):
    call = _calls(kve, _cache(kve))["append"]
    for kw in (dict(r=0), dict(r=8), dict(r=24), dict(r=144), dict(r=-16), dict(P=0), dict(cos=0), dict(sin=0),
               dict(position=0), dict(cos=P + 8), dict(sin=P + 4)):
        rot = _rotation(**kw)
        _refused(kve, 1, call, rot=ctypes.byref(rot))


def test_bad_strides_are_refused(kve):
    calls = _calls(kve, _cache(kve))
    dense = dict(layer=5 * 128 * 4, batch=5 * 128 * 2, head=5 * 128, token=128)
    for bad in (dict(token=-128), dict(head=4), dict(layer=1 << 41), dict(token=1 << 25)):
        st = kve.Strides(**dict(dense, **bad))
        for name, which in (("append", "ks"), ("append", "vs"), ("append", "qs"), ("compact", "ks"), ("compact", "vs")):
            _refused(kve, 1, calls[name], **{which: ctypes.byref(st)})
        _refused(kve, 1, calls["compact"], cap=0, idx=0, ks=ctypes.byref(st))


def test_empty_calls_launch_nothing(kve):
    calls = _calls(kve, _cache(kve))
    assert calls["append"](T=0, k=0, v=0, q=0, out=0) == 0
    assert calls["append"](T=0, k=0, v=0, q=0, out=0, rot=N) == 0
    assert calls["compact"](cap=0, idx=0) == 0
    assert calls["compact"](cap=0, idx=0, k=0, v=0) == 0
    assert calls["read"](T=0, k=0, v=0) == 0
    assert calls["bounds"](n=0, lo=0, hi=0) == 0


def test_empty_calls_are_checked(kve):
    """A call of no rows is refused for what would refuse it with rows, but for tensors that it does not need."""
    calls = _calls(kve, _cache(kve))
    for name, empty in (("append", dict(T=0)), ("append", dict(T=0, k=0, v=0)), ("compact", dict(cap=0))):
        assert calls[name](**empty) == 0
        for kw, status in REFUSALS[name]:
            if "T" in kw or "cap" in kw or kw in (dict(k=0), dict(v=0), dict(idx=0)):
                continue
            _refused(kve, status, calls[name], **dict(empty, **kw))
    dense = dict(layer=5 * 128 * 4, batch=5 * 128 * 2, head=5 * 128, token=128)
    for bad in (dict(token=-128), dict(head=4), dict(layer=1 << 41), dict(token=1 << 25)):
        st = ctypes.byref(kve.Strides(**dict(dense, **bad)))
        for which in ("ks", "vs", "qs"):
            _refused(kve, 1, calls["append"], T=0, **{which: st})
        _refused(kve, 1, calls["append"], T=0, k=0, v=0, qs=st)
        _refused(kve, 1, calls["compact"], cap=0, k=0, vs=st)
    for kw in (dict(r=0), dict(r=24), dict(r=144), dict(P=0), dict(cos=P + 8), dict(sin=P + 4)):
        rot = _rotation(**kw)
        _refused(kve, 1, calls["append"], T=0, rot=ctypes.byref(rot))
    rot = _rotation(cos=0, sin=0, position=0)
    assert calls["append"](T=0, k=0, v=0, q=0, out=0, rot=ctypes.byref(rot)) == 0


def test_workspaces_serve_smaller_calls(kve):
    """The size never falls with L, B, Hq or T, and the call takes it: the next check is reached."""
    size = kve.decode_blocks_workspace_size
    Ls, Bs, Ts, Gs = (1, 2, 5, 33), (1, 2, 15, 60), (1, 2, 3, 5, 16, 33), (1, 2, 3, 5, 8, 11, 16)
    for Hkv in (1, 8):
        for a, L in enumerate(Ls):
            for b, B in enumerate(Bs):
                for c, T in enumerate(Ts):
                    for g, G in enumerate(Gs):
                        here = size(L, B, G * Hkv, Hkv, T, 64)
                        assert here > 0
                        for less in ((Ls[a - 1], B, G, T), (L, Bs[b - 1], G, T), (L, B, G, Ts[c - 1]),
                                     (L, B, Gs[g - 1], T)):
                            if less[0] <= L and less[1] <= B and less[2] <= G and less[3] <= T:
                                assert size(less[0], less[1], less[2] * Hkv, Hkv, less[3], 64) <= here
    for L, Hkv, G, B, T in ((1, 8, 8, 64, 4), (4, 3, 5, 7, 4), (2, 1, 16, 3, 9), (80, 8, 4, 2, 1), (1, 1, 3, 30, 16)):
        call = _calls(kve, _cache(kve, L=L, Hkv=Hkv, S=1 << 10, M=1 << 14))["decode"]
        have = size(L, B, G * Hkv, Hkv, T, 128)
        for b in range(1, B + 1, 3):
            for g in range(1, G + 1):
                for t in range(1, T + 1):
                    for most, top, k in ((1, 0, 0), (700, 0, 0), (3000, 0, 0), (1 << 20, 0, 0), (9, P, 4), (9, P, 900)):
                        _refused(kve, 1, call, B=b, Hq=g * Hkv, T=t, most=most, top=top, k=k, wsb=have, ws=P + 16)
                        assert "aligned" in kve.last_error()
    top = kve.blocks_top_workspace_size
    assert top(2, 3, 4, 2, 5000, 32) <= min(top(3, 3, 4, 2, 5000, 32), top(2, 4, 4, 2, 5000, 32),
                                            top(2, 3, 4, 3, 5000, 32), top(2, 3, 4, 2, 5100, 32))


PLAN_PROGRAM = """
#include <cstdio>
#include <cstdlib>
#include "kve_blocks_plan.h"
int main(int argc, char** argv) {
    for (int i = 1; i + 7 < argc; i += 8) {
        int a[8];
        for (int j = 0; j < 8; ++j) a[j] = atoi(argv[i + j]);
        const kve::BlocksPlan p = kve::decode_blocks_plan(a[0], a[1], a[2], a[3], a[4], a[5], a[6] != 0, a[7]);
        printf("%d %d %d %d %d %zu %zu\\n", (int)p.whole, p.entries, p.slice, p.share, p.groups, p.total,
               kve::decode_blocks_size(a[0], a[1], a[2], a[3], a[4], a[7]));
    }
}
"""


def test_decode_searches_few_entries_at_a_time(tmp_path):
    """Every workgroup of a launch that is cut into splits searches all of its entries: millions of them in one launch
    would be more work than ends in a day.  Slices hold at most 4096, cover the call, and fit the workspace."""
    from tests.test_abi_host import _run_plan
    cases = [(L, B, G * Hkv, Hkv, T, tokens, sparse, d) for L, Hkv in ((1, 1), (2, 8)) for G in (1, 4, 16)
             for B in (1, 3, 4500) for T in (1, 5, 1003, 16400, 1 << 20) for tokens in (40, 2049, 1 << 20)
             for sparse in (0, 1) for d in (64, 128) if L * B * G * Hkv * T < 1 << 24]
    sliced = 0
    for case, line in zip(cases, _run_plan(tmp_path, PLAN_PROGRAM, cases)):
        L, B, Hq, Hkv, T, tokens, sparse, d = case
        whole, entries, per, share, groups, total, size = (int(x) for x in line.split())
        assert entries == B * -(-T // (1 if sparse else min(T, 16 * Hkv // Hq))), case
        assert per == entries if whole else per <= 4096, case
        slices = -(-entries // per)
        assert slices == 1 or slices == -(-entries // 4096), case      # as few as can be, of one size
        assert per * slices < entries + slices and groups <= (per if whole else share + per), case
        assert total <= size, case
        sliced += slices > 1
    assert sliced > 50


def test_python_checks(kve):
    """The binding's own refusals, on CPU tensors: none reaches the library."""
    import torch
    z = lambda *s: torch.zeros(s, dtype=torch.int32)  # noqa: E731
    pool = torch.zeros((1, 3, 2, kve.block_bytes(64, 128)), dtype=torch.uint8)
    ok = dict(pool=pool, refs=z(3), table=z(2, 2), held=z(2), length=z(2), page=64, d=128)
    for bad in (dict(page=48), dict(page=256), dict(d=64), dict(pool=pool.float()), dict(refs=z(4)), dict(held=z(3)),
                dict(length=z(1)), dict(table=z(4)), dict(refs=z(3).long()), dict(pool=pool[..., :-16])):
        with pytest.raises(ValueError):
            kve.Blocks(**dict(ok, **bad))
    with pytest.raises(ValueError, match="device"):
        kve.Blocks(**ok)
    x = torch.zeros(10, 8)
    for cos, sin in ((x[0], x[0]), (x, x[:9]), (x, x)):
        with pytest.raises(ValueError):
            kve.Rotation(cos, sin)


def test_caches_do_not_mix(kve):
    """Calls on rows of one format refuse a cache of the other."""
    import types

    import torch
    x = torch.zeros(1)
    other = types.SimpleNamespace(part=False)
    for call in (lambda: kve.pages_fork(other, x, x), lambda: kve.pages_append(x, x, other, x),
                 lambda: kve.pages_compact(x, x, x, x, other, x), lambda: kve.pages_select(other, x, x, x, x, x),
                 lambda: kve.pages_read(other, 1), lambda: kve.decode_pages(x, other)):
        with pytest.raises(ValueError, match="must be a Pages"):
            call()
    for call in (lambda: kve.blocks_append(x, x, other, x), lambda: kve.blocks_compact(x, x, x, x, other, x),
                 lambda: kve.blocks_read(other, 1), lambda: kve.blocks_bounds(other, 1),
                 lambda: kve.blocks_top(x, other, 1), lambda: kve.decode_blocks(x, other)):
        with pytest.raises(ValueError, match="must be a Blocks"):
            call()
