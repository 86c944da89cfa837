"""The C ABI of the paged 4-bit cache on the CPU: exported symbols, sizes, and
every refusal, none of which may touch its buffers (the pointers are made up)."""

import ctypes
import os
import re

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P = 1 << 20  # an aligned address that no refused call may look at
N = None


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


def test_every_declared_symbol_is_exported(kve):
    text = open(os.path.join(ROOT, "include", "kve_pages.h")).read()
    names = sorted(set(re.findall(r"^(?:kve_status_t|size_t) (kve_[a-z0-9_]+)\(", text, re.M)))
    assert len(names) == 11 and sorted(kve.binding.EXPORTED_PAGES) == names
    lib = ctypes.CDLL(kve.binding._LIB_PATH)
    for n in names:
        assert hasattr(lib, n), n


def test_sizes(kve):
    import oracle as O
    for page in (32, 64, 128, 256, 512, 1024):
        for d in (64, 128):
            assert kve.page_bytes(page, d) == O.page_bytes(page, d)
            assert kve.page_bytes(page, d) % 16 == 0
    for page, d in ((0, 128), (16, 128), (48, 128), (2048, 128), (-32, 64), (64, 96), (64, 0)):
        assert kve.page_bytes(page, d) == 0
    ws = kve.pages_workspace_size
    assert ws(100, 4, 3) % 256 == 0 and ws(100, 4, 3) >= 400 + 48
    for args in ((0, 4, 3), (-1, 4, 3), (100, 0, 3), (100, 4, 0), (100, 4, 1025), ((1 << 30) + 1, 4, 3)):
        assert ws(*args) == 0
    dw = kve.decode_pages_workspace_size
    assert dw(1, 4, 32, 8, 1639, 128) > 0
    for args in ((0, 4, 32, 8, 10, 128), (1, 0, 32, 8, 10, 128), (1, 4, 30, 8, 10, 128), (1, 4, 32, 8, 0, 128),
                 (1, 4, 32, 8, 10, 96), (1, 1 << 24, 32, 8, 10, 128), (1, 4, 32, 8, (1 << 30) + 1, 128)):
        assert dw(*args) == 0


BAD_CACHES = [(dict(refs=0), 1), (dict(table=0), 1), (dict(held=0), 1), (dict(length=0), 1), (dict(L=0), 1),
              (dict(n_pages=0), 1), (dict(Hkv=-1), 1), (dict(S=0), 1), (dict(M=0), 1), (dict(page=48), 1),
              (dict(page=16), 1), (dict(page=2048), 1), (dict(d=96), 2), (dict(M=1 << 26), 2),
              (dict(n_pages=(1 << 30) + 1), 2), (dict(S=1 << 30, M=3), 2)]
BAD_POOLS = [(dict(pool=0), 1), (dict(pool=P + 8), 1)]
BIG = 1 << 30


def _calls(kve, c):
    """Name -> (function of keyword overrides, fields that may be overridden)."""
    lib, r = kve.binding.LIB, ctypes.byref(c) if c is not None else None
    return {
        "extend": lambda seq=P, add=P, n=2, start=P, missing=P, ws=P, wsb=BIG:
            lib.kve_pages_extend(r, seq, add, n, start, missing, ws, wsb, N),
        "fork": lambda src=P, dst=P, n=2, done=P, missing=P, ws=P, wsb=BIG:
            lib.kve_pages_fork(r, src, dst, n, done, missing, ws, wsb, N),
        "free": lambda seq=P, n=2: lib.kve_pages_free(r, seq, n, N),
        "append": lambda k=P, ks=N, v=P, vs=N, dt=0, B=2, T=5, new=P, start=P, seq=P:
            lib.kve_pages_append(k, ks, v, vs, dt, B, T, new, start, seq, r, N),
        "compact": lambda k=P, ks=N, v=P, vs=N, dt=0, B=2, n=9, idx=P, count=P, cap=5, start=P, seq=P:
            lib.kve_pages_compact(k, ks, v, vs, dt, B, n, idx, count, cap, start, seq, r, N),
        "select": lambda B=2, src=P, idx=P, count=P, cap=5, dst=P, start=P:
            lib.kve_pages_select(r, B, src, idx, count, cap, dst, start, N),
        "read": lambda dt=0, B=2, T=5, seq=P, start=P, count=P, k=P, v=P:
            lib.kve_pages_read(r, dt, B, T, seq, start, count, k, v, N),
        "decode": lambda q=P, dt=0, B=2, Hq=8, most=9, seq=P, scale=0.0, out=P, ws=P, wsb=BIG:
            lib.kve_decode_pages(q, dt, r, B, Hq, most, seq, scale, out, ws, wsb, N),
    }


def _refused(kve, status, call, **kw):
    got = call(**kw)
    assert got == status, (kw, got, kve.last_error())
    assert kve.last_error()


def test_bad_caches_are_refused(kve):
    for name, call in _calls(kve, None).items():
        _refused(kve, 1, call)
    for kw, status in BAD_CACHES:
        for name, call in _calls(kve, _cache(kve, **kw)).items():
            _refused(kve, status, call)
    for kw, status in BAD_POOLS:
        for name, call in _calls(kve, _cache(kve, **kw)).items():
            if name not in ("extend", "free"):
                _refused(kve, status, call)


REFUSALS = {
    "extend": [(dict(add=0), 1), (dict(start=0), 1), (dict(missing=0), 1), (dict(n=0), 1), (dict(n=-1), 1),
               (dict(seq=0, n=5), 1), (dict(n=1025), 2), (dict(ws=0), 3), (dict(wsb=16), 3), (dict(ws=P + 16), 1)],
    "fork": [(dict(src=0), 1), (dict(dst=0), 1), (dict(done=0), 1), (dict(missing=0), 1), (dict(n=0), 1),
             (dict(n=1025), 2), (dict(ws=0), 3), (dict(wsb=16), 3), (dict(ws=P + 16), 1)],
    "free": [(dict(n=0), 1), (dict(seq=0, n=5), 1), (dict(n=1 << 24), 2)],
    "append": [(dict(k=0), 1), (dict(v=0), 1), (dict(start=0), 1), (dict(B=0), 1), (dict(T=-1), 1),
               (dict(seq=0, B=5), 1), (dict(dt=2), 2), (dict(k=P + 8), 1), (dict(v=P + 8), 1), (dict(B=1 << 24), 2),
               (dict(T=(1 << 30) + 1), 2)],
    "compact": [(dict(k=0), 1), (dict(v=0), 1), (dict(start=0), 1), (dict(idx=0), 1), (dict(count=0), 1),
                (dict(n=0), 1), (dict(n=(1 << 30) + 1), 1), (dict(cap=-1), 1), (dict(seq=0, B=5), 1),
                (dict(dt=-1), 2), (dict(k=P + 8), 1), (dict(B=1 << 24), 2)],
    "select": [(dict(src=0), 1), (dict(dst=0), 1), (dict(idx=0), 1), (dict(count=0), 1), (dict(start=0), 1),
               (dict(B=0), 1), (dict(cap=-1), 1), (dict(B=1 << 24), 2)],
    "read": [(dict(k=0, v=0), 1), (dict(k=P + 8), 1), (dict(v=P + 4), 1), (dict(B=0), 1), (dict(T=-1), 1),
             (dict(seq=0, B=5), 1), (dict(dt=7), 2), (dict(B=1 << 24), 2)],
    "decode": [(dict(q=0), 1), (dict(out=0), 1), (dict(q=P + 8), 1), (dict(Hq=0), 1), (dict(Hq=7), 1),
               (dict(Hq=34), 2), (dict(most=0), 1), (dict(most=193), 1), (dict(scale=-1.0), 1),
               (dict(scale=float("nan")), 1), (dict(scale=float("inf")), 1), (dict(B=0), 1), (dict(seq=0, B=5), 1),
               (dict(dt=3), 2), (dict(ws=0), 3), (dict(wsb=16), 3), (dict(ws=P + 16), 1), (dict(B=1 << 24), 2)],
}


@pytest.mark.parametrize("name", sorted(REFUSALS))
def test_bad_arguments_are_refused(kve, name):
    call = _calls(kve, _cache(kve))[name]
    for kw, status in REFUSALS[name]:
        _refused(kve, status, call, **kw)


def test_bad_strides_are_refused(kve):
    calls = _calls(kve, _cache(kve))
    dense = dict(layer=5 * 128 * 4, batch=5 * 128 * 2, head=5 * 128, token=128)
    for bad in (dict(token=-128), dict(head=4), dict(layer=1 << 41), dict(token=1 << 25)):
        st = kve.Strides(**dict(dense, **bad))
        for name in ("append", "compact"):
            for which in ("ks", "vs"):
                _refused(kve, 1, calls[name], **{which: ctypes.byref(st)})


def test_empty_calls_launch_nothing(kve):
    """No rows: success without looking at a buffer (there is no GPU here, or the pointers are made up)."""
    calls = _calls(kve, _cache(kve))
    assert calls["append"](T=0, k=0, v=0) == 0
    assert calls["compact"](cap=0, idx=0) == 0
    assert calls["select"](cap=0, idx=0) == 0
    assert calls["read"](T=0, k=0, v=0) == 0


def test_python_checks(kve):
    """The binding's own refusals, on CPU tensors: none reaches the library."""
    import torch
    z = lambda *s: torch.zeros(s, dtype=torch.int32)  # noqa: E731
    pool = torch.zeros((1, 3, 2, kve.page_bytes(64, 128)), dtype=torch.uint8)
    ok = dict(pool=pool, refs=z(3), table=z(2, 2), held=z(2), length=z(2), page=64, d=128)
    for bad in (dict(page=48), dict(d=64), dict(pool=pool.float()), dict(refs=z(4)), dict(held=z(3)), dict(length=z(1)),
                dict(table=z(4)), dict(refs=z(3).long()), dict(pool=pool[..., :-16])):
        with pytest.raises(ValueError):
            kve.Pages(**dict(ok, **bad))
    with pytest.raises(ValueError, match="device"):
        kve.Pages(**ok)


def test_evict_checks_what_goes_into_pages(kve):
    """Refused before anything is queued: the sequences would be extended otherwise."""
    import types

    import torch
    from paper_2607_13205_amd import pipeline
    k = torch.zeros((1, 1, 1, 8, 64))

    def evict(v, pages, **kw):
        bufs = types.SimpleNamespace(pages=pages, hist=None)
        pipeline.evict(None, k, v, None, None, None, 0.5, 4, 1, bufs, **kw)
    for v in (None, k[:, :, :, :4], k.bfloat16()):
        with pytest.raises(ValueError, match="v must match k"):
            evict(v, object())
    with pytest.raises(ValueError, match="slots"):
        evict(k, None, slots=torch.zeros(1, dtype=torch.int32))


def test_compact_of_no_rows_checks_the_views(kve):
    """k_cap = 0 launches nothing, but what a call with rows would refuse is refused."""
    call = _calls(kve, _cache(kve))["compact"]
    dense = dict(layer=5 * 128 * 4, batch=5 * 128 * 2, head=5 * 128, token=128)
    for bad in (dict(token=132), dict(head=4), dict(layer=1 << 41), dict(token=1 << 25)):
        st = kve.Strides(**dict(dense, **bad))
        for which in ("ks", "vs"):
            _refused(kve, 1, call, cap=0, idx=0, **{which: ctypes.byref(st)})
    _refused(kve, 1, call, cap=0, idx=0, v=P + 2)
    _refused(kve, 1, call, cap=0, idx=0, k=P + 8)
    assert call(cap=0, idx=0, k=0, v=0) == 0


def test_evict_checks_before_it_queues(kve, monkeypatch):
    """Whatever the compaction into pages would refuse is refused before the score is queued."""
    import types

    import torch
    from paper_2607_13205_amd import pipeline
    k = torch.zeros((2, 1, 1, 8, 64))
    z = torch.zeros(1, dtype=torch.int32)
    queued, refused = [], ValueError("slots of the wrong kind")
    monkeypatch.setattr(pipeline, "_score", lambda *a, **kw: queued.append("score"))
    monkeypatch.setattr(pipeline, "_upload_quotas", lambda *a, **kw: queued.append("quotas"))

    def refuse(*a, **kw):
        raise refused
    monkeypatch.setattr(pipeline.kp, "check_compact", refuse)
    bufs = types.SimpleNamespace(pages=types.SimpleNamespace(L=2), hist=None, start=z, k_cap=3,
                                 idx=torch.zeros((2, 1, 1, 3), dtype=torch.int32),
                                 count=torch.zeros((2, 1, 1), dtype=torch.int32))
    monkeypatch.setattr(torch.cuda, "current_stream", lambda *a: None)
    with pytest.raises(ValueError, match="wrong kind"):
        pipeline.evict(k, k, k, None, None, pipeline.Policy.role((1.0,)), 0.5, 4, 1, bufs, slots=z)
    with pytest.raises(ValueError, match="layers"):
        pipeline.evict(k[:1], k, k, None, None, pipeline.Policy.role((1.0,)), 0.5, 4, 1, bufs, slots=z)
    with pytest.raises(ValueError, match="layers"):
        pipeline.evict(k, k, k, None, None, pipeline.Policy.role((1.0,)), 0.5, 4, 1, bufs, slots=z, lse_win=k[:1])
    assert not queued


def test_decode_workspace_serves_smaller_calls(kve):
    """One made for the largest batch, stack and bound serves what is left of them: the size never falls with L, B, Hq
    or max_tokens."""
    size = kve.decode_pages_workspace_size
    assert size(1, 16, 32, 8, 2048, 128) >= size(1, 15, 32, 8, 2048, 128)
    assert size(32, 4, 32, 8, 1639, 128) >= size(1, 4, 32, 8, 1639, 128)
    Ls, Bs = (1, 2, 3, 5, 16, 31, 32, 33, 80, 129), (1, 2, 4, 15, 16, 17, 64, 100, 500)
    tokens = (1, 128, 129, 512, 513, 1000, 1639, 2047, 2048, 2049, 5000, 1 << 17, 1 << 24)
    for Hkv in (1, 3, 8):
        for d in (64, 128):
            for Hq in (Hkv, 4 * Hkv):
                table = [[[size(L, B, Hq, Hkv, n, d) for n in tokens] for B in Bs] for L in Ls]
                for a in range(len(Ls)):
                    for b in range(len(Bs)):
                        for c in range(len(tokens)):
                            here = table[a][b][c]
                            assert here > 0 and here <= size(Ls[a], Bs[b], 2 * Hq, Hkv, tokens[c], d)
                            for at in ((a - 1, b, c), (a, b - 1, c), (a, b, c - 1)):
                                if min(at) >= 0:
                                    assert table[at[0]][at[1]][at[2]] <= here, (Ls[a], Bs[b], Hkv, tokens[c], at)
    # short sequences need next to nothing however many they are, ordinary ones some megabytes
    assert size(32, 1000, 32, 8, 512, 128) <= 1 << 14
    assert size(32, 64, 32, 8, 2048, 128) <= 4 << 20


def test_decode_takes_the_workspace_of_a_larger_call(kve):
    """Refusals come before anything is launched: with the size of a larger call the next check is reached."""
    size = kve.decode_pages_workspace_size
    call = _calls(kve, _cache(kve, L=1, Hkv=8, S=64, M=64))["decode"]
    for B, most, Bs in ((16, 2048, (1, 4, 15, 16)), (64, 1639, (1, 7, 30)), (200, 700, (1, 3, 6))):
        have = size(1, B, 32, 8, most, 128)
        for b in Bs:
            _refused(kve, 1, call, B=b, Hq=32, most=most, wsb=have, ws=P + 16)      # not 3: the size suffices
            assert "aligned" in kve.last_error()
            _refused(kve, 1, call, B=b, Hq=32, most=most // 2, wsb=have, ws=P + 16)
            assert "aligned" in kve.last_error()
