"""Host-only checks of the operators on rows and on the 4-bit cache: sizes, and what is refused before a launch."""
import ctypes as C

import numpy as np
import pytest
import torch

import decoder_plain as P

B = pytest.importorskip("paper_1805_08691_amd.binding")
L = B.lib
OK, EINVAL, EUNSUPPORTED, EALIGN, EWORKSPACE = 0, -1, -2, -3, -5
A = C.c_void_p(0x10000)             # never dereferenced: every call below ends on the host


def _at(n):
    return C.c_void_p(0x10000 + n)


def test_sizes():
    assert L.q8_linear_packed_bytes(1, 1) == 16 * 64
    assert L.q8_linear_packed_bytes(1000, 2048) == 1008 * 2048
    assert L.q8_linear_packed_bytes(0, 8) == 0 == L.q8_linear_packed_bytes(8, 131072) == L.q8_linear_packed_bytes(-1, 8)
    assert L.q8_linear_workspace_bytes(3, 5, 20) >= 3 * 32 + 12
    assert L.q8_kv4_cache_bytes(7, 3, 64, 128) == 7 * 3 * 4 * 18 * 128
    assert L.q8_kv4_cache_bytes(1 << 20, 8, 64, 128) == (1 << 20) * 8 * 4 * 18 * 128
    for heads, page, D in ((0, 64, 128), (1, 8, 128), (1, 48, 128), (1, 64, 48), (1, 64, 288), (1, 64, 0)):
        assert L.q8_kv4_cache_bytes(1, heads, page, D) == 0
    assert L.q8_kv4_attend_workspace_bytes(1, 1, 8, 4, 128, 131072) > 0
    assert L.q8_kv4_attend_workspace_bytes(1, 1, 8, 4, 128, 64) == 0
    assert L.q8_kv4_attend_workspace_bytes(1, 0, 8, 4, 128, 64) == 0


def _rows(x=A, kind=0, M=4, K=32, xs=32, z=A, zs=32, q=A):
    return L.q8_quantize_rows(x, kind, M, K, xs, z, zs, q, None)


def test_rows_refused():
    assert _rows(M=0) == OK
    for bad in (dict(x=None), dict(z=None), dict(q=None), dict(kind=3), dict(kind=-1), dict(K=0), dict(xs=31), dict(zs=16)):
        assert _rows(**bad) == EINVAL, bad
    for bad in (dict(z=_at(8)), dict(zs=40), dict(x=_at(2)), dict(q=_at(2)), dict(x=_at(1), kind=1)):
        assert _rows(**bad) == EALIGN, bad
    assert _rows(M=1 << 31) == EUNSUPPORTED


def _product(z=A, zs=64, q_x=A, M=4, N=8, K=64, w=A, q_w=A, bias=None, y=A, kind=0, ys=8):
    return L.q8_linear_int8(z, zs, q_x, M, N, K, w, q_w, bias, y, kind, ys, None)


def _linear(x=A, kind=0, xs=64, M=4, N=8, K=64, w=A, q_w=A, bias=None, y=A, yk=0, ys=8, ws=A, n=1 << 20):
    return L.q8_linear(x, kind, xs, M, N, K, w, q_w, bias, y, yk, ys, ws, n, None)


def test_products_refused():
    assert L.q8_linear_int8_variant(A, 64, A, 4, 8, 64, A, A, None, A, 0, 8, L.q8_linear_num_variants(), None) == EINVAL
    assert L.q8_linear_variant_name(-1) == L.q8_linear_variant_name(10 ** 6) == b"unsupported"
    for f in (_product, _linear):
        assert f(M=0) == OK == f(N=0)
        for bad in (dict(w=None), dict(q_w=None), dict(y=None), dict(K=0), dict(N=-1), dict(ys=7), dict(kind=5)):
            assert f(**bad) == EINVAL, bad
        assert f(K=131072) == EUNSUPPORTED == f(M=1 << 31)
        for bad in (dict(w=_at(8)), dict(q_w=_at(2)), dict(bias=_at(1)), dict(y=_at(2))):
            assert f(**bad) == EALIGN, bad
    assert _product(z=None) == EINVAL == _product(zs=48) == _product(q_x=None)
    assert _product(z=_at(4)) == EALIGN == _product(zs=72)
    assert _linear(x=None) == EINVAL == _linear(xs=63) == _linear(ws=None) == _linear(yk=9)
    assert _linear(ws=_at(16)) == EALIGN
    assert _linear(n=100) == EWORKSPACE
    assert L.q8_linear_pack(None, 4, 4, A, None) == EINVAL == L.q8_linear_pack(A, 4, 4, None, None)
    assert L.q8_linear_pack(A, 4, 4, _at(4), None) == EALIGN
    assert L.q8_linear_pack(A, 4, 131072, A, None) == EUNSUPPORTED
    assert L.q8_linear_pack(None, 0, 4, None, None) == OK


def test_products_beyond_a_launch_refused():
    """A launch's threads are counted in 32 bits: no weights of 2^36 bytes, no build for few rows on 2^27 channels."""
    assert L.q8_linear_pack(A, 1 << 22, 16384, A, None) == EUNSUPPORTED
    for v in range(L.q8_linear_num_variants()):
        if L.q8_linear_variant_name(v) == b"rows_16x16":
            assert L.q8_linear_int8_variant(A, 16, A, 1, 1 << 27, 1, A, A, None, A, 0, 1 << 27, v, None) == EUNSUPPORTED
    assert _product(N=0x7fffffff, ys=0x7fffffff, K=1) == EUNSUPPORTED


def _tables(lengths=A, added=A, n=3, page=16, free=A, n_free=5, table=A, width=4, stride=4, slots=A, positions=A,
            n_slots=9, starts=A, grown=A, counts=A):
    return L.q8_page_tables(lengths, added, n, page, free, n_free, table, width, stride, slots, positions, n_slots, starts,
                            grown, counts, None)


def test_tables_refused():
    for bad in (dict(lengths=None), dict(added=None), dict(free=None), dict(table=None), dict(slots=None),
                dict(positions=None), dict(starts=None), dict(grown=None), dict(counts=None), dict(n=-1), dict(n_free=-1),
                dict(width=-1), dict(stride=3), dict(n_slots=-1)):
        assert _tables(**bad) == EINVAL, bad
    for page in (0, 8, 24, -16, 1 << 21):
        assert _tables(page=page) == EUNSUPPORTED
    for bad in (dict(lengths=_at(2)), dict(slots=_at(4)), dict(table=_at(1)), dict(counts=_at(2))):
        assert _tables(**bad) == EALIGN, bad


def _write(k=A, v=A, kind=0, T=4, H=2, D=64, s=(128, 64, 128, 64), slots=A, cache=A, pages=3, page=16):
    return L.q8_kv4_write(k, v, kind, T, H, D, *s, slots, cache, pages, page, None)


def _read(k=A, v=A, kind=0, T=4, H=2, D=64, s=(128, 64, 128, 64), slots=A, cache=A, pages=3, page=16):
    return L.q8_kv4_read(cache, pages, page, slots, T, H, D, k, v, kind, *s, None)


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


def _attend(q=A, kind=2, T=2, H=2, ratio=4, D=64, qs=512, qh=64, cache=A, pages=3, page=16, table=A, width=4, stride=4,
            lengths=A, starts=None, n=2, scale=0.1, window=0, out=A, os_=512, oh=64, ws=None, nb=0):
    return L.q8_kv4_attend(q, kind, T, H, ratio, D, qs, qh, cache, pages, page, table, width, stride, lengths, starts, n,
                           scale, window, out, os_, oh, ws, nb, None)


def test_attention_refused():
    assert _attend(T=0) == OK == _attend(n=0)
    for bad in (dict(q=None), dict(out=None), dict(cache=None), dict(table=None), dict(lengths=None), dict(kind=9), dict(H=0),
                dict(ratio=0), dict(pages=0), dict(width=-1), dict(stride=3), dict(T=3), dict(window=-1), dict(n=-1),
                dict(scale=float("nan")), dict(scale=float("inf")), dict(qs=63), dict(oh=32), dict(os_=1), dict(qh=0)):
        assert _attend(**bad) == EINVAL, bad
    for bad in (dict(kind=0), dict(D=48), dict(D=512), dict(page=24), dict(width=1 << 28, stride=1 << 28, page=1024)):
        assert _attend(**bad) == EUNSUPPORTED, bad
    for bad in (dict(q=_at(1)), dict(out=_at(1)), dict(cache=_at(16)), dict(table=_at(2)), dict(lengths=_at(3)),
                dict(starts=_at(2)), dict(ws=_at(8), nb=100)):
        assert _attend(**bad) == EALIGN, bad


def test_attention_refuses_tables_of_too_many_places():
    """What a tile looks up behind its last key, up to 2048 tokens, has to have numbers below 2^31."""
    for page in (16, 64, 1 << 16):
        wide = 0x7fff0000 // page + 1
        assert _attend(width=wide, stride=wide, page=page) == EUNSUPPORTED


def test_attention_refuses_more_tiles_than_a_launch_takes():
    for T, H, ratio in ((1 << 24, 1, 1), (1 << 20, 16, 16), (1 << 21, 4, 17)):
        assert _attend(T=T, n=T, H=H, ratio=ratio, qs=1 << 20, os_=1 << 20) == EUNSUPPORTED


def test_workspace_for_many_tokens_serves_fewer():
    """A program holds one workspace, made for its largest step: more tokens never ask for less."""
    size = L.q8_kv4_attend_workspace_bytes
    tokens = sorted({max(1, (1 << e) + d) for e in range(18) for d in (-1, 0, 1)})
    for n in (1, 3, 64, 200, 255, 256, 257, 1000):
        for H, ratio, D in ((8, 4, 128), (1, 1, 64), (16, 8, 256), (2, 40, 96), (4, 17, 32)):
            for longest in (64, 512, 513, 8192, 131072):
                sizes = [size(T, n, H, ratio, D, longest) for T in tokens]
                assert sizes == sorted(sizes), (n, H, ratio, D, longest)
    assert size(8192, 1, 8, 4, 128, 32768) == size(512, 1, 8, 4, 128, 32768) > size(1, 1, 8, 4, 128, 32768) > 0
    assert size(8192, 256, 8, 4, 128, 8192) >= size(1, 256, 8, 4, 128, 8192) > 0 == size(8192, 257, 8, 4, 128, 8192)


def test_binding_refuses_what_it_cannot_pass_on():
    x = torch.zeros(4, 32)
    for call in (lambda: B.quantize_rows(x), lambda: B.linear_pack(x), lambda: B.kv4_read(x, x),
                 lambda: B.linear(x, x, x), lambda: B.kv4_write(x, x, x, x)):
        with pytest.raises((AssertionError, RuntimeError)):
            call()
    with pytest.raises(B.Q8Error):
        B.kv4_cache(3, 1, 24, 64, device="cpu")
    with pytest.raises(B.Q8Error):
        B.kv4_cache(3, 1, 16, 40, device="cpu")


def test_references():
    """The plain forms themselves, on cases worked by hand."""
    z, q = P.quantize_rows(torch.tensor([[127.0, -2.5, 3.5, float("nan"), float("-inf")], [0, 0, 0, 0, 0]]))
    assert z.tolist() == [[127, -2, 4, 0, -128], [0, 0, 0, 0, 0]] and q.tolist() == [1.0, 1.0]
    x = np.zeros((1, 32), np.float32)
    x[0, :4] = [7, -3.5, 2.5, -7]
    z, q = P.kv4_codes(x)
    assert z[0, :4].tolist() == [7, -4, 2, -7] and float(q[0, 0]) == 1.0
    table, slots, positions, starts, grown, counts = P.page_tables([15, 3], [2, 1], 16, [8, 9],
                                                                   np.array([[4, -1], [5, -1]], np.int32), 5)
    assert table.tolist() == [[4, 8], [5, -1]] and slots == [79, 128, 83, -1, -1] and positions == [15, 16, 3, -1, -1]
    assert starts == [0, 2, 3] and grown == [17, 4] and counts == [1, 3, 0]
    one = np.ones((3, 1, 32))
    out, _ = P.attend(np.ones((1, 1, 32)), [one], [one * np.arange(3.0)[:, None, None]], [3], [0, 1], 1.0, 2)
    assert np.allclose(out, 1.5)
