"""Attention over the 8-bit cache in tiles of 128 columns, and the bounds of each row by itself: what a row sees of keys and
factors is what its outputs are near to."""
import numpy as np
import pytest
import torch

import kv8_plain as P

pytestmark = pytest.mark.gpu
TYPES = {"f16": torch.float16, "bf16": torch.bfloat16}


@pytest.fixture(scope="module")
def B():
    from paper_1805_08691_amd import binding
    return binding


def _rng(*seed):
    return np.random.Generator(np.random.PCG64(np.random.SeedSequence([1805, 8691, 89, *seed])))


def _cache(rng, pages, H, page, D, spread=0.3):
    """Codes of a normal distribution, with a factor for every sixteen."""
    cache = P.empty(pages, H, page, D)
    shape = (pages, H, page // 16, 16, D)
    k, v = [np.clip(np.rint(rng.standard_normal(shape) * 40), -128, 127).astype(np.int32) for _ in range(2)]
    P.put(cache, D, k, v, np.exp(spread * rng.standard_normal((pages, H, page // 16, 2))) / 40)
    return cache


def _table(rng, lengths, page, width=0):
    held = [-(-n // page) for n in lengths]
    order = rng.permutation(sum(held) + 2).astype(np.int32)
    table, at = np.full((len(lengths), max([width, 1, *held])), -1, np.int32), 0
    for b, n in enumerate(held):
        table[b, :n] = order[at:at + n]
        at += n
    return table, len(order)


def _held(cache, table, lengths, page):
    """Keys and values of each request in 64 bits, and which of them lie on a page that there is."""
    pages, kv, there = len(cache), [], []
    for b, n in enumerate(lengths):
        rows = table[b, np.arange(n) // page] if n else np.zeros(0, np.int32)
        there.append((rows >= 0) & (rows < pages))
        kv.append(P.held(cache, np.where((table >= 0) & (table < pages), table, 0), b, n, page))
    return kv, there


def _seen(n_keys, n, window, causal, there):
    behind = np.arange(n_keys)[None] - (np.arange(n) + n_keys - n)[:, None]
    return ((behind <= 0) & (behind > -window if window else True) if causal else np.ones((n, n_keys), bool)) & there


def _attend(q, kv, there, lengths, starts, scale, window=0, causal=True):
    """In 64 bits.  q [T, heads * ratio, D], kv: per request [2][length, heads, D].  -> outputs; the same sums of magnitudes, with the
    weights as they are; and the largest sum of |q k| scale over the keys that a row sees."""
    out, size, noise = np.zeros(q.shape), np.zeros(q.shape), np.zeros(q.shape[:2])
    for b, n_keys in enumerate(lengths):
        rows, n = slice(starts[b], starts[b + 1]), starts[b + 1] - starts[b]
        seen = _seen(n_keys, n, window, causal, there[b])
        for h in range(q.shape[1] if n and n_keys else 0):
            k, v = [x[:, h * x.shape[1] // q.shape[1]] for x in kv[b]]
            s = np.where(seen, q[rows, h] @ k.T * scale, -np.inf)
            p = np.exp(s - np.where(seen.any(1), s.max(1), 0)[:, None])
            p /= np.maximum(p.sum(1), 1e-300)[:, None]
            out[rows, h], size[rows, h] = p @ v, p @ np.abs(v)
            noise[rows, h] = np.where(seen, np.abs(q[rows, h]) @ np.abs(k).T, 0).max(1) * abs(scale)
    return out, size, noise


def _poison(cache, table, lengths, added, page, window, causal):
    """What no row sees of the pages: sixteens behind the last token, in front of the window, and pages that no request has (their
    factors are no numbers)."""
    cache, per = cache.copy(), page // 16
    for page_number in set(range(len(cache))) - {int(x) for x in table.reshape(-1)}:
        cache[page_number] = 255
    for b, n in enumerate(lengths):
        front = max(0, n - added[b] - window + 1) // 16 if window and causal else 0
        for s in [*range(front), *range(-(-n // 16), -(-n // page) * per)]:
            if 0 <= table[b, s // per] < len(cache):
                cache[table[b, s // per], :, s % per] = 255
    return cache


def _bound(out, size, noise, n, dtype):
    """How far a row may be off, element by element.  Queries of these tests are multiplied exactly, as are codes.  Sums of the matrix
    instruction are of fp32 terms cut at the largest addend, in steps of 32 (2^-20 of the sum of magnitudes): a score is off by d at
    most, which moves weights by a factor of exp(2 d); the same for n products of values, 2^-23 each of the sum of magnitudes.  A
    probability times its sixteen's factor is rounded once (2^-11), or off by 2^-25 of 2^-7 of the row's largest such product where
    it is below binary16's normal numbers: with codes up to 128 and n keys, n 2^-25 of the largest sum of magnitudes of the row.
    Logarithms of factors (below 2^7) are off by 2^-17, four such numbers are added; the exponential is off by 2^-22, the output's own
    rounding by half a step of its type (fp16 below 2^-14: steps of 2^-24; bf16 below 2^-126: of 2^-133)."""
    rel = np.expm1(2 * noise * 2.0 ** -20) + 2.0 ** -11 + n * 2.0 ** -23 + 2.0 ** -15 + 2.0 ** -21
    half = 2.0 ** -8 if dtype is torch.bfloat16 else 2.0 ** -11
    few = n * 2.0 ** -25 * size.max(-1, keepdims=True)
    return size * rel[..., None] + few + np.abs(out) * half + (2.0 ** -25 if dtype is torch.float16 else 2.0 ** -134)


def _check(B, rng, lengths, added, H, ratio, D, page, kind, scale=None, window=0, causal=True, workspace=True, peak=1.0, width=0,
           holes=(), form=(128, False), factors=None):
    """form: what the call has to run as (kv8_attend_form).  holes: (request, place, entry) of the table.  factors: what becomes of the
    cache's, [pages, heads, sixteens, 2]."""
    table, pool = _table(rng, lengths, page, width)
    cache = _cache(rng, pool, H, page, D)
    if factors is not None:
        k, v, f = P.codes_of(cache, D)
        P.put(cache, D, k, v, factors(f).astype(np.float32))
    for b, place, entry in holes:
        table[b, place] = entry if entry >= 0 else -1
    starts = np.concatenate([[0], np.cumsum(added)]).astype(np.int32)
    q = torch.from_numpy(rng.standard_normal((int(starts[-1]), H * ratio, D)).astype(np.float32) * peak).to(TYPES[kind])
    scale = D ** -0.5 if scale is None else scale
    poisoned = _poison(cache, table, lengths, added, page, window, causal)
    dev = [torch.from_numpy(x).cuda() for x in (poisoned, table, np.array(lengths, np.int32), starts)]
    ws = B.kv8_attend_workspace(q, dev[0], len(lengths), table.shape[1] * page) if workspace else None
    assert B.kv8_attend_form(q, dev[0], dev[1], dev[3], ws) == form
    out = B.kv8_attend(q.cuda(), *dev, scale, window, causal, workspace=ws)
    kv, there = _held(cache, table, lengths, page)
    want, size, noise = _attend(q.double().numpy(), kv, there, lengths, starts, float(np.float32(scale)), window, causal)
    off, bound = out.double().cpu().numpy() - want, _bound(want, size, noise, max(lengths), TYPES[kind])
    assert (np.abs(off) <= bound).all(), float((np.abs(off) / np.maximum(bound, 1e-300)).max())
    if ws is not None and ws.numel():
        assert not bool(ws[:2048].any())                         # counters are zero again
    return out


@pytest.mark.parametrize("steps", [64, 65, 74, 89, 104, 209, 225, 240])
def test_a_long_request_among_short_ones_in_tiles_of_many_columns(B, steps):
    """One tile of so many steps of 64 keys, and little else to fill the card: in 16 parts of equal numbers of steps, rounded up, some
    would begin behind the tile's last key.  (Tables as wide as 32768 tokens.)"""
    lengths, added = [64 * steps - 3] + [12] * 31, [12] * 32
    _check(B, _rng(steps), lengths, added, 1, 8, 128, 64, "bf16", width=512, form=(128, True))


# (head size, key heads, query heads for each) that make tiles of 128 columns of _PIECES
_HEADS = [(32, 16, 21), (64, 16, 21), (96, 13, 8), (128, 16, 8), (160, 8, 8), (192, 5, 8), (224, 8, 6), (256, 16, 3)]
_PIECES = ([700, 64, 333], [130, 64, 100])


def test_forms(B):
    """The one that a call runs as, which the tests here ask for."""
    def form(T, n, ratio, D, longest, ws, H=16, ragged=1):
        return B.lib.q8_kv8_attend_call_form(T, n, H, ratio, D, longest, ragged, ws)
    large = B.lib.q8_kv8_attend_workspace_bytes(294, 3, 16, 8, 128, 704)
    assert form(294, 3, 8, 128, 704, large) == 129 and form(294, 3, 8, 128, 704, 0) == 128
    assert form(294, 3, 8, 128, 704, large, ragged=0) in (16, 17) and form(3, 3, 8, 128, 704, 0, ragged=0) == 16
    assert form(3, 3, 8, 128, 8192, large) == 17
    for bad in (dict(T=0), dict(n=0), dict(H=0), dict(ratio=0), dict(D=48), dict(D=288)):
        assert form(**{**dict(T=294, n=3, ratio=8, D=128, longest=704, ws=0), **bad}) == 0


@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("D,H,ratio", _HEADS)
def test_prompts_in_tiles_of_many_columns(B, kind, D, H, ratio):
    for workspace in (False, True):
        _check(B, _rng(D, workspace), *_PIECES, H, ratio, D, 16, kind, workspace=workspace, form=(128, workspace))


@pytest.mark.parametrize("workspace", [False, True])
@pytest.mark.parametrize("window", [1, 2, 15, 16, 17, 63, 64, 65, 130, 600, 1000])
def test_windows_in_tiles_of_many_columns(B, window, workspace):
    _check(B, _rng(window, 3), *_PIECES, 16, 8, 128, 32, "f16", window=window, workspace=workspace, form=(128, workspace))


@pytest.mark.parametrize("workspace", [False, True])
@pytest.mark.parametrize("D,H,ratio", [(32, 16, 21), (64, 16, 21), (128, 16, 8), (256, 16, 3)])
def test_all_keys_in_tiles_of_many_columns(B, D, H, ratio, workspace):
    """More keys than rows and fewer, one and none."""
    _check(B, _rng(D, 5), [700, 64, 17, 0, 1], [130, 64, 100, 9, 20], H, ratio, D, 16, "bf16", causal=False, workspace=workspace,
           form=(128, workspace))


@pytest.mark.parametrize("workspace", [False, True])
def test_more_rows_than_tokens_in_tiles_of_many_columns(B, workspace):
    out = _check(B, _rng(6), [5, 0, 40], [90, 80, 120], 16, 8, 128, 16, "bf16", workspace=workspace, width=40, form=(128, workspace))
    assert not bool(out[:85].any()) and not bool(out[90:170].any()) and bool(out[85:90].any())


@pytest.mark.parametrize("window,causal", [(0, True), (8500, True), (100, True), (0, False)])
@pytest.mark.parametrize("workspace", [False, True])
def test_long_contexts_in_tiles_of_many_columns(B, window, causal, workspace):
    """More steps than the ring of sixteens in LDS holds, twice over."""
    _check(B, _rng(window, 7), [17000, 130], [20, 130], 9, 8, 160, 64, "bf16", window=window, causal=causal, workspace=workspace,
           form=(128, workspace))


@pytest.mark.parametrize("D,H,ratio,window", [(64, 8, 16, 0), (128, 8, 8, 0), (128, 8, 8, 600), (256, 8, 8, 0)])
def test_cut_pieces_in_tiles_of_many_columns(B, D, H, ratio, window):
    _check(B, _rng(D, window, 8), [4200, 1100], [70, 210], H, ratio, D, 64, "bf16", window=window, width=8192 // 64 * (2 if D == 64 else 1),
           form=(128, True))


@pytest.mark.parametrize("peak,scale", [(0.0, None), (1e-6, None), (30.0, None), (1.0, -0.3), (1.0, 0.0), (300.0, 1e-3)])
@pytest.mark.parametrize("workspace", [False, True])
def test_flat_and_peaked_rows_in_tiles_of_many_columns(B, peak, scale, workspace):
    _check(B, _rng(9), *_PIECES, 16, 8, 128, 16, "bf16", peak=peak, scale=scale, workspace=workspace, form=(128, workspace))


@pytest.mark.parametrize("workspace", [False, True])
@pytest.mark.parametrize("window,causal", [(0, True), (40, True), (0, False)])
def test_missing_pages_in_tiles_of_many_columns(B, window, causal, workspace):
    """Places in front, within and at the end of a request whose page is not there: their tokens are not seen."""
    holes = [(0, 0, -1), (0, 4, 10 ** 9), (0, 5, -1), (0, 21, -7), (2, 10, 1 << 30), (1, 0, -1), (1, 1, -1)]
    _check(B, _rng(window, 10), *_PIECES, 16, 8, 128, 32, "bf16", window=window, causal=causal, workspace=workspace, holes=holes,
           form=(128, workspace))
    # and behind the refill of the ring
    if not window:
        _check(B, _rng(11), [9000, 130], [20, 130], 9, 8, 160, 64, "f16", causal=causal, workspace=workspace,
               holes=[(0, 139, -1), (0, 60, -1)], form=(128, workspace))


def _pieces(B, seed, kind, workspace=True, D=128, H=16, ratio=8, page=16, lengths=_PIECES[0], added=_PIECES[1], columns=128):
    """What a call takes, on the device, and its cache and table on the host."""
    rng = _rng(seed)
    table, pool = _table(rng, lengths, page, 2560 // page)
    cache = _cache(rng, pool, H, page, D)
    starts = np.concatenate([[0], np.cumsum(added)]).astype(np.int32)
    q = torch.from_numpy(rng.standard_normal((int(starts[-1]), H * ratio, D)).astype(np.float32)).to(TYPES[kind])
    dev = [torch.from_numpy(x).cuda() for x in (cache, table, np.array(lengths, np.int32), starts)]
    ws = B.kv8_attend_workspace(q, dev[0], len(lengths), table.shape[1] * page) if workspace else None
    assert B.kv8_attend_form(q, dev[0], dev[1], dev[3], ws) == (columns, workspace)
    return q, dev, ws, cache, table, starts


@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("size", [1e2, 1e4, 1e6, 1e9])
@pytest.mark.parametrize("workspace", [False, True])
def test_rows_that_see_one_key_alone_in_tiles_of_many_columns(B, kind, size, workspace):
    """Scores so far apart that all of a row's weight is on one key: its value, whatever the scores' own size."""
    q, dev, ws, cache, table, starts = _pieces(B, 13, kind, workspace)
    out = B.kv8_attend(q.cuda(), *dev, scale=size, workspace=ws).double().cpu().numpy()
    half, checked = (2.0 ** -8 if kind == "bf16" else 2.0 ** -11), 0
    for b, n in enumerate(_PIECES[0]):
        keys, values = P.held(cache, table, b, n, 16)
        for t in range(starts[b], starts[b + 1]):
            last = n - (starts[b + 1] - t) + 1
            for h in range(t % 7, 128, 13):
                x = q[t, h].double().numpy()
                s = keys[:last, h // 8] @ x * size
                # (scores are off by 2^-20 of the sum of their terms' magnitudes at most)
                noise = (np.abs(keys[:last, h // 8]) @ np.abs(x)).max() * size * 2.0 ** -20
                top = np.argmax(s)
                if last > 1 and np.delete(s, top).max() > s[top] - 2 * noise - 40:
                    continue
                v = values[top, h // 8]
                # (the probability 2^-11, its product with the factor 2^-16 in the exponent, fp32 sums, the output's own rounding)
                assert (np.abs(out[t, h] - v) <= np.abs(v) * (2.0 ** -11 + 2.0 ** -14 + half) + 2.0 ** -24).all(), (b, t, h)
                checked += 1
    assert checked > 100


@pytest.mark.parametrize("workspace", [False, True])
def test_tiles_of_many_columns_leave_other_rows_alone(B, workspace):
    q, dev, ws, *_ = _pieces(B, 14, "f16", workspace)
    T = len(q)
    want = B.kv8_attend(q.cuda(), *dev, workspace=ws)
    rows = torch.zeros((T + 20, *q.shape[1:]), dtype=q.dtype, device="cuda")
    rows[7:7 + T] = q.cuda()
    whole = torch.full((T + 20, q.shape[1] + 1, q.shape[2] + 8), 5.0, device="cuda", dtype=q.dtype)
    B.kv8_attend(rows, *dev[:3], dev[3] + 7, out=whole[:, :-1, :-8], workspace=ws)
    half = torch.finfo(q.dtype).eps
    # (their columns may lie in other tiles, whose steps begin elsewhere: near, not the same bits)
    assert torch.allclose(whole[7:7 + T, :-1, :-8].float(), want.float(), rtol=4 * half, atol=4 * half * float(want.abs().max()))
    assert bool((whole[:7] == 5).all()) and bool((whole[7 + T:] == 5).all())
    assert bool((whole[:, -1] == 5).all()) and bool((whole[..., -8:] == 5).all())


@pytest.mark.parametrize("workspace", [False, True])
def test_tiles_of_many_columns_are_the_same_every_time(B, workspace):
    """And in a captured launch, replayed among eager work."""
    q, dev, ws, *_ = _pieces(B, 15, "bf16", workspace, lengths=[4200, 64, 1333], added=[130, 64, 100])
    x, out = q.cuda(), torch.empty_like(q.cuda())
    first = B.kv8_attend(x, *dev, workspace=ws)
    for _ in range(10):
        assert torch.equal(B.kv8_attend(x, *dev, workspace=ws), first)
    stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        B.kv8_attend(x, *dev, out=out, workspace=ws)
        stream.synchronize()
        with torch.cuda.graph(graph, stream=stream):
            B.kv8_attend(x, *dev, out=out, workspace=ws)
    torch.cuda.current_stream().wait_stream(stream)
    for _ in range(5):
        out.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, first)
        assert torch.equal(B.kv8_attend(x, *dev, workspace=ws), first)


@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("workspace", [False, True])
@pytest.mark.parametrize("columns,H", [(16, 2), (128, 16)])
def test_rows_that_are_no_numbers(B, kind, workspace, columns, H):
    """Queries with infinities and NaN, zeros and the type's smallest, beside ordinary ones of the same tile, whose outputs are bit for
    bit the ones without them."""
    q, dev, ws, *_ = _pieces(B, 12, kind, workspace, H=H, columns=columns)
    T = len(q)
    want = B.kv8_attend(q.cuda(), *dev, workspace=ws)
    q[1, 1::8, 3], q[1, 2::8, 5], q[4, ::8, 127] = float("nan"), float("inf"), float("-inf")
    q[T - 2, 3::8] = 0
    q[T - 1, 1::8] = torch.finfo(q.dtype).tiny
    out = B.kv8_attend(q.cuda(), *dev, workspace=ws)
    fine = torch.isfinite(q).all(-1)
    assert bool(torch.isfinite(out.cpu()[fine]).all()) and bool(torch.isnan(out.cpu()[~fine]).all())
    same = fine.clone()
    same[T - 2, 3::8] = same[T - 1, 1::8] = False
    assert torch.equal(out.cpu()[same], want.cpu()[same])


@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("workspace", [False, True])
@pytest.mark.parametrize("columns,H", [(16, 2), (128, 16)])
@pytest.mark.parametrize("window", [0, 40])
def test_hidden_keys_have_no_effect(B, kind, workspace, columns, H, window):
    """Sixteens that a row sees nothing of, though others of its tile do: whatever they hold, and however large their factors, the
    row's outputs are the same bits."""
    q, dev, ws, cache, table, starts = _pieces(B, 20, kind, workspace, H=H, columns=columns)
    lengths, added = _PIECES
    args = [torch.from_numpy(x).cuda() for x in (table, np.array(lengths, np.int32), starts)]
    want = B.kv8_attend(q.cuda(), dev[0], *args, window=window, workspace=ws)
    for size in (2.0 ** -30, 2.0 ** 12, 2.0 ** 24, 2.0 ** 70):
        other = cache.copy()
        changed = []
        for b, n in enumerate(lengths):
            first = n - added[b]
            sixteens = [first // 16 + 2, first // 16 + 3] if n > 200 else [first // 16 + 1]
            for s in sixteens:
                block = other[table[b, s], :, 0]
                k, v, f = P.codes_of(block, 128)
                P.put(block, 128, -k.clip(-127) if size > 1 else k, v[:, ::-1], f * np.array([min(size, 4.0), size], np.float32))
            changed.append((min(sixteens) * 16, max(sixteens) * 16 + 15))
        got = B.kv8_attend(q.cuda(), torch.from_numpy(other).cuda(), *args, window=window, workspace=ws)
        for b, n in enumerate(lengths):
            pos = np.arange(n - added[b], n)
            apart = (pos < changed[b][0]) | ((pos - window + 1 > changed[b][1]) if window else False)
            rows = starts[b] + np.flatnonzero(apart)
            assert len(rows) >= 16 and torch.equal(got[rows], want[rows]), (size, b)
            rows = starts[b] + np.flatnonzero(~apart)
            assert not torch.equal(got[rows], want[rows])


@pytest.mark.parametrize("spread", [3, 20, 60])
@pytest.mark.parametrize("window", [0, 40])
@pytest.mark.parametrize("columns,H,workspace", [(16, 2, False), (16, 2, True), (128, 16, False), (128, 16, True)])
def test_rows_are_as_near_as_their_own_keys_allow(B, spread, window, columns, H, workspace):
    """Values' factors that spread over many powers of two in one context, zeros among them, rising and falling."""
    def factors(f):
        f[..., 1] *= 2.0 ** rng.integers(-spread, spread, f[..., 1].shape)
        f[..., 1][rng.random(f[..., 1].shape) < 0.2] = 0
        f[..., 0][rng.random(f[..., 0].shape) < 0.1] = 0
        return f

    for peak in (1.0, 12.0):
        rng = _rng(21, spread, window)
        _check(B, rng, *_PIECES, H, 8, 128, 16, "bf16", window=window, workspace=workspace, peak=peak, factors=factors, width=160,
               form=(columns, workspace))


@pytest.mark.parametrize("size", [1e-36, 1e-30, 1e-9, 1e-3, 1e4, 1e9, 1e30])
@pytest.mark.parametrize("columns,H", [(16, 2), (128, 16)])
def test_factors_of_any_size(B, size, columns, H):
    for workspace in (False, True):
        _check(B, _rng(22), *_PIECES, H, 8, 128, 16, "bf16", workspace=workspace, factors=lambda f: f * np.array([1, size]), width=160,
               form=(columns, workspace))


@pytest.mark.parametrize("columns,H", [(16, 2), (128, 16)])
def test_a_likely_key_of_small_values_beside_unlikely_ones_of_large(B, columns, H):
    """Probabilities and factors whose products differ the other way round than they do themselves."""
    for workspace in (False, True):
        for exponent in (-40, -12, 12, 40):
            def factors(f):
                f[..., 1] *= np.exp2(np.clip(exponent * (f[..., 0] * 40 - 1), -60, 60))
                f[..., 0] *= 8
                return f
            _check(B, _rng(23, exponent + 50), *_PIECES, H, 8, 128, 16, "bf16", workspace=workspace, factors=factors, width=160,
                   form=(columns, workspace))
