"""Host-only checks of the 8-bit cache and of its pages: sizes, what is refused before a launch, and the references."""
import ctypes as C

import numpy as np
import pytest
import torch

import kv8_plain as P

B = pytest.importorskip("paper_1805_08691_amd.binding")
L = B.lib
OK, EINVAL, EUNSUPPORTED, EALIGN, EWORKSPACE = 0, -1, -2, -3, -5
A = C.c_void_p(0x10000)             # never dereferenced: every call below ends on the host
FAR = C.c_void_p(0x90000000)


def _at(n):
    return C.c_void_p(0x10000 + n)


def test_sizes():
    assert L.q8_kv8_cache_bytes(7, 3, 64, 128) == 7 * 3 * 4 * (32 * 128 + 64)
    assert L.q8_kv8_cache_bytes(1 << 20, 8, 64, 128) == (1 << 20) * 8 * 4 * (32 * 128 + 64)
    for heads, page, D in ((0, 64, 128), (1, 8, 128), (1, 48, 128), (1, 64, 48), (1, 64, 288), (1, 64, 0)):
        assert L.q8_kv8_cache_bytes(1, heads, page, D) == 0
    assert L.q8_kv8_attend_workspace_bytes(1, 1, 8, 4, 128, 131072) > 0
    assert L.q8_kv8_attend_workspace_bytes(1, 1, 8, 4, 128, 64) == 0 == L.q8_kv8_attend_workspace_bytes(1, 0, 8, 4, 128, 64)
    assert L.q8_page_workspace_bytes(-1, 5) == 0 == L.q8_page_workspace_bytes(4, (1 << 24) + 1)
    assert L.q8_page_workspace_bytes(4000, 1 << 20) >= (1 << 17) + 16000
    sizes = [L.q8_page_workspace_bytes(n, p) for n, p in ((0, 0), (0, 33), (5, 33), (300, 33), (300, 40000))]
    assert sizes == sorted(sizes)


def _write(k=A, v=A, kind=0, T=4, H=2, D=64, s=(128, 64, 128, 64), slots=A, cache=A, pages=3, page=16):
    return L.q8_kv8_write(k, v, kind, T, H, D, *s, slots, cache, pages, page, None)


def _read(k=A, v=A, kind=0, T=4, H=2, D=64, s=(128, 64, 128, 64), slots=A, cache=A, pages=3, page=16):
    return L.q8_kv8_read(cache, pages, page, slots, T, H, D, k, v, kind, *s, None)


def test_tokens_refused():
    for f in (_write, _read):
        assert f(T=0) == OK
        for bad in (dict(k=None), dict(v=None), dict(slots=None), dict(cache=None), dict(kind=7), dict(H=0), dict(pages=0),
                    dict(s=(63, 64, 128, 64)), dict(s=(128, 63, 128, 64)), dict(s=(128, 64, 128, 1))):
            assert f(**bad) == EINVAL, bad
        for bad in (dict(D=48), dict(D=0), dict(D=288), dict(page=8), dict(page=48), dict(pages=1 << 31), dict(T=1 << 31)):
            assert f(**bad) == EUNSUPPORTED, bad
        for bad in (dict(k=_at(2)), dict(v=_at(1), kind=2), dict(slots=_at(4)), dict(cache=_at(32))):
            assert f(**bad) == EALIGN, bad
    assert _write(T=1 << 24) == EUNSUPPORTED == _write(H=0x7fffffff)


def _attend(q=A, kind=2, T=2, H=2, ratio=4, D=64, qs=512, qh=64, cache=A, pages=3, page=16, table=A, width=4, stride=4,
            lengths=A, starts=None, n=2, scale=0.1, window=0, causal=1, out=A, os_=512, oh=64, ws=None, nb=0):
    return L.q8_kv8_attend(q, kind, T, H, ratio, D, qs, qh, cache, pages, page, table, width, stride, lengths, starts, n,
                           scale, window, causal, out, os_, oh, ws, nb, None)


def test_attention_refused():
    assert _attend(T=0) == OK == _attend(n=0)
    for bad in (dict(q=None), dict(out=None), dict(cache=None), dict(table=None), dict(lengths=None), dict(kind=9), dict(H=0),
                dict(ratio=0), dict(pages=0), dict(width=-1), dict(stride=3), dict(T=3), dict(window=-1), dict(n=-1),
                dict(scale=float("nan")), dict(scale=float("inf")), dict(qs=63), dict(oh=32), dict(os_=1), dict(qh=0),
                dict(causal=2), dict(causal=-1), dict(causal=0, window=5)):
        assert _attend(**bad) == EINVAL, bad
    for bad in (dict(kind=0), dict(D=48), dict(D=512), dict(page=24), dict(width=1 << 28, stride=1 << 28, page=1024)):
        assert _attend(**bad) == EUNSUPPORTED, bad
    for bad in (dict(q=_at(1)), dict(out=_at(1)), dict(cache=_at(16)), dict(table=_at(2)), dict(lengths=_at(3)),
                dict(starts=_at(2)), dict(ws=_at(8), nb=100)):
        assert _attend(**bad) == EALIGN, bad
    for T, H, ratio in ((1 << 24, 1, 1), (1 << 20, 16, 16), (1 << 21, 4, 17)):
        assert _attend(T=T, n=T, H=H, ratio=ratio, qs=1 << 20, os_=1 << 20) == EUNSUPPORTED


def test_workspace_for_many_tokens_serves_fewer():
    size = L.q8_kv8_attend_workspace_bytes
    tokens = sorted({max(1, (1 << e) + d) for e in range(18) for d in (-1, 0, 1)})
    for n in (1, 3, 64, 200, 255, 256, 257, 1000):
        for H, ratio, D in ((8, 4, 128), (1, 1, 64), (16, 8, 256), (2, 40, 96), (4, 17, 32)):
            for longest in (64, 512, 513, 8192, 131072):
                sizes = [size(T, n, H, ratio, D, longest) for T in tokens]
                assert sizes == sorted(sizes), (n, H, ratio, D, longest)


def _select(parents=A, m=3, lengths=A, table=A, stride=4, n=2, width=4, page=16, pages=40, out=FAR, ostride=4, grown=FAR, free=A,
            copies=A, counts=A, ws=A, nb=1 << 20):
    return L.q8_page_select(parents, m, lengths, table, stride, n, width, page, pages, out, ostride, grown, free, copies,
                            counts, ws, nb, None)


def _compact(lengths=A, table=A, stride=4, n=2, width=4, page=16, pages=40, out=FAR, ostride=4, free=A, copies=A, counts=A, ws=A,
             nb=1 << 20):
    return L.q8_page_compact(lengths, table, stride, n, width, page, pages, out, ostride, free, copies, counts, ws, nb, None)


def test_pages_refused():
    for f in (_select, _compact):
        for bad in (dict(lengths=None), dict(table=None), dict(out=None), dict(free=None), dict(copies=None), dict(counts=None),
                    dict(ws=None), dict(n=-1), dict(width=-1), dict(stride=3), dict(ostride=3)):
            assert f(**bad) == EINVAL, bad
        for bad in (dict(page=8), dict(page=24), dict(page=1 << 21), dict(pages=(1 << 24) + 1),
                    dict(width=1 << 28, stride=1 << 28, ostride=1 << 28)):
            assert f(**bad) == EUNSUPPORTED, bad
        for bad in (dict(lengths=_at(2)), dict(table=_at(1)), dict(free=_at(2)), dict(copies=_at(2)), dict(counts=_at(1)),
                    dict(ws=_at(8))):
            assert f(**bad) == EALIGN, bad
        assert f(nb=100) == EWORKSPACE
    assert _select(m=-1) == EINVAL == _select(parents=None) == _select(grown=None)
    assert _select(parents=_at(2)) == EALIGN
    # what is read and what is written lie apart, or (compact) are the same table
    for out in (A, _at(4), _at(16), _at(4 * 7)):
        assert _select(out=out) == EINVAL, out
    assert _select(grown=A) == EINVAL == _select(grown=_at(4))
    for bad in (dict(out=_at(4)), dict(out=_at(16)), dict(out=A, ostride=5)):
        assert _compact(**bad) == EINVAL, bad
    # a call whose memory is all apart would run: here each of them meets something that is read
    apart = dict(parents=_at(1024), lengths=_at(2048), table=_at(4096), free=_at(8192), copies=_at(16384), counts=_at(32768))
    for name in ("parents", "lengths", "table"):
        at = apart[name]
        for bad in (dict(out=at), dict(grown=at), dict(free=at), dict(copies=at), dict(counts=at)):
            assert _select(**dict(apart, **bad)) == EINVAL, (name, bad)
    del apart["parents"]
    for name in ("lengths", "table"):
        at = apart[name]
        for bad in (dict(free=at), dict(copies=at), dict(counts=at)) + ((dict(out=at),) if name == "lengths" else ()):
            assert _compact(**dict(apart, **bad)) == EINVAL, (name, bad)


def test_most_rows():
    most, width = 1 << 24, 1
    for f in (_select, _compact):
        assert f(n=most + 1, width=width) == EUNSUPPORTED
        assert f(n=most, width=width, nb=100) == EWORKSPACE
    assert _select(m=most + 1, width=width) == EUNSUPPORTED


def test_copies_refused():
    def copy(cache=A, pages=3, size=64, pairs=A, n=2):
        return L.q8_page_copy(cache, pages, size, pairs, n, None)

    assert copy(n=0) == OK == copy(pages=0) == copy(size=0)
    assert copy(n=-1) == EINVAL == copy(cache=None) == copy(pairs=None)
    assert copy(size=40) == EALIGN == copy(cache=_at(8)) == copy(pairs=_at(2))
    assert copy(pages=1 << 31) == EUNSUPPORTED == copy(size=1 << 40)


def test_binding_refuses_what_it_cannot_pass_on():
    x = torch.zeros(4, 32)
    i = torch.zeros(4, dtype=torch.int32)
    for call in (lambda: B.kv8_write(x, x, x, x), lambda: B.kv8_read(x, x), lambda: B.page_copy(x, x),
                 lambda: B.kv8_attend(x[None], x, x, x), lambda: B.page_select(i, i, i[None], 16, 3),
                 lambda: B.page_compact(i, i[None], 16, 3)):
        with pytest.raises((AssertionError, RuntimeError)):
            call()
    with pytest.raises(B.Q8Error):
        B.kv8_cache(3, 1, 24, 64, device="cpu")
    assert B.kv8_cache(3, 2, 32, 96, device="cpu").shape == (3, 2, 2, 32 * 96 + 64)


def test_references():
    """The plain forms themselves, on cases worked by hand."""
    for D in (32, 64, 96, 160):
        assert sorted(P.key_order(D).reshape(-1).tolist()) == list(range(16 * D))
    cache = P.empty(2, 1, 16, 32)
    k = np.zeros((1, 1, 32), np.float32)
    k[0, 0, :3] = [127, -64.5, 2.5]
    P.write(cache, k, -k, [16], 16)
    got = P.read(cache, [16, 17, 0, 32], 16)
    assert got[0, 0, 0, :3].tolist() == [127, -64, 2] and got[1, 0, 0, :3].tolist() == [-127, 64, -2]
    assert not got[:, 1:].any()
    P.write(cache, k * 2, k / 2, [18], 16)                       # keys: 1 -> 2, codes 127, -64, 2 -> 64, -32, 1; values stay
    got = P.read(cache, [16, 17, 18], 16)
    assert got[0, 0, 0, :3].tolist() == [128, -64, 2] and got[0, 2, 0, :3].tolist() == [254, -128, 4]
    assert got[1, 0, 0, :3].tolist() == [-127, 64, -2] and got[1, 2, 0, :3].tolist() == [64, -32, 1]
    P.write(cache, k * np.float32(2.1), k, [17], 16)              # 2 -> 2.5 at least
    assert P.codes_of(cache[1, 0, 0], 32)[2].tolist() == [2.5, 1.0]
    table = np.array([[4, 7, -1], [4, 2, -1]], np.int32)
    out, lens, free, copies, counts = P.select([1, 5, 1, 1], [20, 20], table, 16, 9)
    assert out.tolist() == [[4, 2, -1], [-1, -1, -1], [4, 0, -1], [4, 1, -1]] and lens == [20, 0, 20, 20]
    assert free == [3, 5, 6, 7, 8] + [-1] * 4 and copies == [(2, 0), (2, 1), (-1, -1), (-1, -1)] and counts == [5, 2, 0, 4]
    out, free, moves, counts = P.compact([20, 20], table, 16, 9)
    assert out.tolist() == [[0, 1, -1], [0, 2, -1]] and moves == [(4, 0), (7, 1), (-1, -1), (-1, -1)] and counts == [6, 2, 0, 3]
    one = np.ones((3, 1, 32))
    values = [one * np.arange(3.0)[:, None, None]]
    assert np.allclose(P.attend(np.ones((1, 1, 32)), [one], values, [3], [0, 1], 1.0, 2)[0], 1.5)
    assert np.allclose(P.attend(np.ones((2, 1, 32)), [one], values, [3], [0, 2], 1.0, causal=False)[0], 1.0)
