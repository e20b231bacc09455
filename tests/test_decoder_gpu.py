"""The linear layer on rows, the block tables, the 4-bit cache and attention over it, against the plain references of
decoder_plain.py: bit for bit where the result is a fixed sequence of operations, within a derived bound else."""
import numpy as np
import pytest
import torch

import decoder_plain as P

pytestmark = pytest.mark.gpu
TYPES = P.TYPES


@pytest.fixture(scope="module")
def B():
    from paper_1805_08691_amd import binding
    return binding


def _rng(*seed):
    return np.random.Generator(np.random.PCG64(np.random.SeedSequence([1805, 8691, 77, *seed])))


def _real(rng, shape, kind):
    return torch.from_numpy((rng.standard_normal(shape) * np.exp(rng.standard_normal(shape[-1]))).astype(np.float32)).to(
        TYPES[kind])


# ------------------------------------------------------------------------------ rows to codes
@pytest.mark.parametrize("kind", sorted(TYPES))
@pytest.mark.parametrize("M,K", [(1, 1), (3, 7), (2, 8), (5, 16), (1, 64), (4, 1000), (7, 2049), (2, 4096), (3, 16400),
                                 (1, 131071), (300, 40)])
def test_rows_to_codes(B, kind, M, K):
    x = _real(_rng(M, K), (M, K), kind)
    z, q = B.quantize_rows(x.cuda())
    want_z, want_q = P.quantize_rows(x)
    assert np.array_equal(q.cpu().numpy(), want_q)
    assert np.array_equal(z.cpu().numpy(), want_z)


@pytest.mark.parametrize("kind", sorted(TYPES))
@pytest.mark.parametrize("offset,pad", [(0, 8), (1, 0), (0, 3), (3, 5)])
def test_rows_to_codes_of_strided_rows(B, kind, offset, pad):
    M, K = 6, 200
    whole = _real(_rng(offset, pad), (M * (K + pad) + offset,), kind).cuda()
    x = torch.as_strided(whole, (M, K), (K + pad, 1), offset)
    out = torch.full((M, 224), 77, dtype=torch.int8, device="cuda")
    z, q = B.quantize_rows(x, out=out[:, :K])
    want_z, want_q = P.quantize_rows(x.cpu())
    assert np.array_equal(z.cpu().numpy(), want_z) and np.array_equal(q.cpu().numpy(), want_q)
    assert bool((out[:, 208:] == 77).all())


@pytest.mark.parametrize("kind", sorted(TYPES))
@pytest.mark.parametrize("K", [40, 4096, 20000])
def test_rows_to_codes_of_special_values(B, kind, K):
    x = torch.zeros(9, K)
    rows = _real(_rng(1, K), (9, K), "f32")
    x[1] = rows[1] * 1e-30
    x[2] = rows[2] * 1e-41                                   # (denormal: 0 in binary16)
    x[3] = rows[3] * 1e30
    x[4] = rows[4]
    x[4, 3] = float("nan")
    x[5] = rows[5]
    x[5, 1], x[5, 2] = float("inf"), float("-inf")
    x[6] = float("nan")
    x[7, K - 1] = float("inf")
    x[8] = torch.arange(K) % 256 / 2.0                       # ties
    x = x.to(TYPES[kind])
    z, q = B.quantize_rows(x.cuda())
    want_z, want_q = P.quantize_rows(x)
    assert np.array_equal(q.cpu().numpy(), want_q)
    assert np.array_equal(z.cpu().numpy(), want_z)


def test_rows_to_codes_of_very_many_rows(B):
    """More rows than the blocks of one launch take."""
    M, K = (1 << 26) + 333, 3
    x = torch.randn((M, K), device="cuda", dtype=torch.float16)
    q = torch.zeros(M, device="cuda")
    z, _ = B.quantize_rows(x, factors=q)
    assert bool((q > 0).all())
    for a in (0, (1 << 25) - 100, (1 << 26) - 500, M - 700):
        rows = slice(a, a + 700)
        want_z, want_q = P.quantize_rows(x[rows].cpu())
        assert np.array_equal(z[rows].cpu().numpy(), want_z) and np.array_equal(q[rows].cpu().numpy(), want_q)


def test_rows_to_codes_of_very_many_longer_rows(B):
    """The same where a block takes a row."""
    M, K = (1 << 24) + 7, 1025
    x = torch.empty((M, K), device="cuda", dtype=torch.bfloat16).normal_()
    q = torch.zeros(M, device="cuda")
    z, _ = B.quantize_rows(x, factors=q)
    assert bool((q > 0).all())
    for a in (0, (1 << 24) - 60, M - 64):
        rows = slice(a, a + 64)
        want_z, want_q = P.quantize_rows(x[rows].cpu())
        assert np.array_equal(z[rows].cpu().numpy(), want_z) and np.array_equal(q[rows].cpu().numpy(), want_q)


# ------------------------------------------------------------------------------ the product
def _weights(rng, N, K):
    z_w = rng.integers(-128, 128, (N, K), dtype=np.int8)
    return z_w, (rng.random(N) + 0.5).astype(np.float32) / 100, rng.standard_normal(N).astype(np.float32)


SHAPES = [(1, 1, 1), (1, 16, 64), (1, 17, 65), (2, 100, 333), (15, 31, 128), (16, 64, 4096), (17, 1000, 2048), (33, 48, 16),
          (40, 272, 130), (63, 65, 257), (64, 64, 64), (65, 129, 1000), (100, 300, 200), (128, 256, 512), (129, 257, 1024),
          (255, 255, 255), (300, 520, 720), (513, 384, 192), (1, 5000, 80), (1000, 16, 31), (257, 1030, 2050)]


@pytest.mark.parametrize("kind", sorted(TYPES))
@pytest.mark.parametrize("M,N,K", SHAPES)
def test_product(B, kind, M, N, K):
    rng = _rng(M, N, K)
    z_w, q_w, bias = _weights(rng, N, K)
    z = rng.integers(-128, 128, (M, K), dtype=np.int8)
    q_x = (rng.random(M) + 0.1).astype(np.float32)
    packed = B.linear_pack(torch.from_numpy(z_w).cuda())
    codes = torch.full((M, -(-K // 16) * 16), -77, dtype=torch.int8, device="cuda")
    codes[:, :K] = torch.from_numpy(z).cuda()
    for b in (None, bias):
        y = B.linear_int8(codes[:, :K], torch.from_numpy(q_x).cuda(), packed, torch.from_numpy(q_w).cuda(),
                          None if b is None else torch.from_numpy(b).cuda(), dtype=TYPES[kind])
        want = P.linear(z, q_x, z_w, q_w, b, TYPES[kind])
        assert torch.equal(y.cpu(), want)


@pytest.mark.parametrize("M,N,K", [(1, 3, 5), (40, 70, 64), (16, 16, 128), (65, 257, 200), (130, 100, 1100), (300, 520, 720),
                                   (513, 384, 449)])
def test_every_build_of_the_product(B, M, N, K):
    rng = _rng(M, N, K, 3)
    z_w, q_w, bias = _weights(rng, N, K)
    z = rng.integers(-128, 128, (M, K), dtype=np.int8)
    q_x = (rng.random(M) + 0.1).astype(np.float32)
    packed = B.linear_pack(torch.from_numpy(z_w).cuda())
    codes = torch.full((M, -(-K // 16) * 16), -77, dtype=torch.int8, device="cuda")
    codes[:, :K] = torch.from_numpy(z).cuda()
    dev = [torch.from_numpy(v).cuda() for v in (q_x, q_w, bias)]
    names = [B.lib.q8_linear_variant_name(v).decode() for v in range(B.lib.q8_linear_num_variants())]
    assert len(set(names)) == len(names) >= 2
    for kind in sorted(TYPES):
        want = P.linear(z, q_x, z_w, q_w, bias, TYPES[kind])
        for v in range(len(names)):
            out = torch.full((M + 2, N), 3.0, dtype=TYPES[kind], device="cuda")
            B.linear_int8(codes[:, :K], dev[0], packed, dev[1], dev[2], out=out[1:-1], variant=v)
            assert torch.equal(out[1:-1].cpu(), want), names[v]
            assert bool((out[0] == 3).all()) and bool((out[-1] == 3).all()), names[v]


def test_product_of_rows_far_apart(B):
    """Rows more than 4 MiB apart: a tile's offsets would pass 32 bits."""
    M, N, K = 40, 50, 100
    rng = _rng(21)
    z_w, q_w, _ = _weights(rng, N, K)
    z = rng.integers(-128, 128, (M, K), dtype=np.int8)
    stride = (1 << 26) + 16
    whole = torch.empty((M - 1) * stride + 112, dtype=torch.int8, device="cuda")
    codes = torch.as_strided(whole, (M, K), (stride, 1), 0)
    codes.copy_(torch.from_numpy(z))
    y = B.linear_int8(codes, torch.ones(M, device="cuda"), B.linear_pack(torch.from_numpy(z_w).cuda()),
                      torch.from_numpy(q_w).cuda(), dtype=torch.float32)
    assert torch.equal(y.cpu(), P.linear(z, np.ones(M, np.float32), z_w, q_w, None, torch.float32))


def test_product_of_very_many_rows(B):
    """More rows than a launch's second dimension has sixteens."""
    M, N, K = 16 * 65535 + 33, 20, 16
    rng = _rng(6, 6)
    z_w, q_w, bias = _weights(rng, N, K)
    z = torch.from_numpy(rng.integers(-128, 128, (M, K), dtype=np.int8))
    q_x = torch.from_numpy(rng.random(M).astype(np.float32) + 0.5)
    y = B.linear_int8(z.cuda(), q_x.cuda(), B.linear_pack(torch.from_numpy(z_w).cuda()), torch.from_numpy(q_w).cuda(),
                      torch.from_numpy(bias).cuda(), dtype=torch.float16)
    assert torch.equal(y.cpu(), P.linear(z.numpy(), q_x.numpy(), z_w, q_w, bias, torch.float16))


@pytest.mark.parametrize("M,N", [((1 << 30) + 77, 5), (1, (1 << 27) + 5)])
def test_product_of_more_than_a_launch_takes(B, M, N):
    """Rows in several launches; channels that the builds for few rows do not reach."""
    rng = _rng(6, 7, N % 100)
    K = 16 if M > 1 else 1
    z_w = rng.integers(-128, 128, (min(N, 5000), K), dtype=np.int8)
    q_w = (rng.random(min(N, 5000)) + 0.5).astype(np.float32)
    repeat = -(-N // len(q_w))
    weights = B.linear_pack(torch.from_numpy(z_w).cuda().repeat(repeat, 1)[:N])
    factors = torch.from_numpy(q_w).cuda().repeat(repeat)[:N].contiguous()
    x = torch.randint(-128, 128, (1000, 16), device="cuda", dtype=torch.int8)
    codes = x.repeat(-(-M // 1000), 1)[:M]
    y = torch.empty((M, N), device="cuda", dtype=torch.float16)
    B.linear_int8(codes[:, :K], torch.ones(M, device="cuda"), weights, factors, out=y)
    want = P.linear(x[:, :K].cpu().numpy(), np.ones(1000, np.float32), z_w, q_w, None, torch.float16).cuda()
    if M > 1:
        for a in range(0, M, 1 << 22):
            part = y[a:a + (1 << 22)]
            assert torch.equal(part, want[(a + torch.arange(len(part), device="cuda")) % 1000]), a
    else:
        assert torch.equal(y[0], want[0].repeat(repeat)[:N])


def test_product_of_the_largest_sums(B):
    """128 * 128 * 131071 just fits the accumulator, on both sides."""
    K = 131071
    for a, b in ((-128, -128), (-128, 127), (127, 127)):
        z, z_w = np.full((3, K), a, np.int8), np.full((20, K), b, np.int8)
        one = np.ones(20, np.float32)
        padded = torch.full((3, 131072), 100, dtype=torch.int8, device="cuda")
        padded[:, :K] = a
        y = B.linear_int8(padded[:, :K], torch.ones(3, device="cuda"), B.linear_pack(torch.from_numpy(z_w).cuda()),
                          torch.ones(20, device="cuda"), dtype=torch.float32)
        assert torch.equal(y.cpu(), P.linear(z, np.ones(3, np.float32), z_w, one, None, torch.float32))


@pytest.mark.parametrize("kind", sorted(TYPES))
@pytest.mark.parametrize("M", [1, 2, 4, 16, 40, 70, 300])
def test_product_into_strided_rows(B, kind, M):
    """Rows inside a wider tensor, at an odd place: nothing beside them is written."""
    N, K = 83, 96
    rng = _rng(M, 5)
    z_w, q_w, _ = _weights(rng, N, K)
    z = rng.integers(-128, 128, (M, K), dtype=np.int8)
    q_x = (rng.random(M) + 0.1).astype(np.float32)
    wide = torch.full((M, N + 10), 3.0, dtype=TYPES[kind], device="cuda")
    strided = torch.zeros((M, 160), dtype=torch.int8, device="cuda")
    strided[:, 32:32 + K] = torch.from_numpy(z).cuda()
    B.linear_int8(strided[:, 32:32 + K], torch.from_numpy(q_x).cuda(), B.linear_pack(torch.from_numpy(z_w).cuda()),
                  torch.from_numpy(q_w).cuda(), out=wide[:, 5:5 + N])
    want = torch.full((M, N + 10), 3.0, dtype=TYPES[kind])
    want[:, 5:5 + N] = P.linear(z, q_x, z_w, q_w, None, TYPES[kind])
    assert torch.equal(wide.cpu(), want)


@pytest.mark.parametrize("kind", sorted(TYPES))
@pytest.mark.parametrize("M,N,K", [(1, 16, 8), (1, 4096, 4096), (2, 33, 1000), (3, 100, 4096), (4, 64, 16384), (5, 200, 77),
                                   (8, 1000, 2048), (37, 520, 4096), (130, 300, 1000), (600, 700, 800)])
def test_linear_is_its_two_parts(B, kind, M, N, K):
    rng = _rng(M, N, K, 9)
    z_w, q_w, bias = _weights(rng, N, K)
    x = _real(rng, (M, K), kind)
    if M > 2:
        x[1] = 0
        x[2, K // 2] = float("nan")
    packed, qw, b = B.linear_pack(torch.from_numpy(z_w).cuda()), torch.from_numpy(q_w).cuda(), torch.from_numpy(bias).cuda()
    y = B.linear(x.cuda(), packed, qw, b)
    z, q_x = P.quantize_rows(x)
    assert y.dtype is x.dtype
    assert torch.equal(y.cpu(), P.linear(z, q_x, z_w, q_w, bias, TYPES[kind]))
    y32 = B.linear(x.cuda()[:, :], packed, qw, out=torch.empty(M, N, device="cuda"))
    assert torch.equal(y32.cpu(), P.linear(z, q_x, z_w, q_w, None, torch.float32))


@pytest.mark.parametrize("kind", sorted(TYPES))
@pytest.mark.parametrize("M", [2, 3, 8, 9, 15, 16, 17])
def test_linear_of_a_few_short_rows(B, kind, M):
    """Rows that a wavefront takes: odd lengths and distances, rows of zeros, infinities and no numbers."""
    rng = _rng(M, 51)
    for K, N, pad in ((1, 5, 0), (7, 16, 1), (64, 40, 3), (511, 33, 0), (512, 100, 8), (513, 17, 2), (1000, 2439, 0), (1024, 64, 1),
                      (1025, 64, 0), (40, 9000, 0)):
        z_w, q_w, bias = _weights(rng, N, K)
        x = _real(rng, (M, K + pad), kind)
        x[0] = 0.0
        x[1, 0] = float("nan")
        x[M - 1, K - 1] = float("inf")
        qw, b = torch.from_numpy(q_w).cuda(), torch.from_numpy(bias).cuda()
        got = B.linear(x.cuda()[:, :K], B.linear_pack(torch.from_numpy(z_w).cuda()), qw, b)
        z, q_x = P.quantize_rows(x[:, :K])
        assert torch.equal(got.cpu(), P.linear(z, q_x, z_w, q_w, bias, TYPES[kind])), (K, N)


def test_linear_of_strided_rows(B):
    rng = _rng(4, 4)
    z_w, q_w, _ = _weights(rng, 70, 90)
    for M, offset, pad in ((1, 1, 3), (2, 3, 1), (50, 1, 6), (200, 8, 6)):
        whole = _real(rng, (M * (90 + pad) + offset,), "bf16").cuda()
        x = torch.as_strided(whole, (M, 90), (90 + pad, 1), offset)
        y = B.linear(x, B.linear_pack(torch.from_numpy(z_w).cuda()), torch.from_numpy(q_w).cuda())
        z, q_x = P.quantize_rows(x.cpu())
        assert torch.equal(y.cpu(), P.linear(z, q_x, z_w, q_w, None, torch.bfloat16))


def test_linear_of_nothing(B):
    packed, q_w = B.linear_pack(torch.ones(20, 40, dtype=torch.int8, device="cuda")), torch.ones(20, device="cuda")
    assert B.linear(torch.zeros(0, 40, device="cuda"), packed, q_w).shape == (0, 20)
    none = B.linear_pack(torch.ones(0, 40, dtype=torch.int8, device="cuda"))
    assert B.linear(torch.zeros(3, 40, device="cuda"), none, q_w[:0]).shape == (3, 0)


def test_linear_refuses_weights_packed_for_other_sizes(B):
    """Also such as are as many bytes or more: 128 outputs of 64 values are none for 64 of 128."""
    packed = B.linear_pack(torch.ones(128, 64, dtype=torch.int8, device="cuda"))
    assert packed.numel() == B.lib.q8_linear_packed_bytes(128, 64)
    for N, K in ((64, 128), (64, 64), (128, 65), (129, 64), (112, 64), (32, 256)):
        x, q_w = torch.ones(3, K, device="cuda"), torch.ones(N, device="cuda")
        z, q_x = B.quantize_rows(x)
        with pytest.raises(AssertionError):
            B.linear(x, packed, q_w)
        with pytest.raises(AssertionError):
            B.linear_int8(z, q_x, packed, q_w)
    for N, K in ((128, 64), (113, 64), (128, 1)):
        B.linear(torch.ones(3, K, device="cuda"), packed, torch.ones(N, device="cuda"))
    # memory without a shape is taken as what it is said to hold
    assert torch.equal(B.linear(torch.ones(3, 64, device="cuda"), packed.flatten(), torch.ones(128, device="cuda")),
                       B.linear(torch.ones(3, 64, device="cuda"), packed, torch.ones(128, device="cuda")))


def test_rows_of_more_values_than_an_int_counts_are_refused(B):
    """2^32 + 64 values a row are none of 64."""
    x = torch.empty((1, (1 << 32) + 64), dtype=torch.float16, device="cuda")
    packed, q_w = B.linear_pack(torch.ones(16, 64, dtype=torch.int8, device="cuda")), torch.ones(16, device="cuda")
    z, q_x = torch.zeros((1, (1 << 32) + 64), dtype=torch.int8, device="cuda"), torch.ones(1, device="cuda")
    for call in (lambda: B.linear(x, packed.flatten(), q_w, workspace=torch.empty(4096, dtype=torch.uint8, device="cuda")),
                 lambda: B.quantize_rows(x, out=z, factors=q_x), lambda: B.linear_int8(z, q_x, packed.flatten(), q_w)):
        with pytest.raises(AssertionError):
            call()
    with pytest.raises(B.Q8Error):
        B.linear_pack(torch.empty(((1 << 32) + 16, 1), dtype=torch.int8, device="cuda"))


# ------------------------------------------------------------------------------ block tables
def _run_tables(B, lengths, added, page, n_free, width, n_slots, pad=0, seed=0):
    rng = _rng(len(lengths), page, n_free, seed)
    n = len(lengths)
    table = rng.integers(-5, 1000, (n, width + pad)).astype(np.int32)
    free = rng.permutation(max(n_free, 1))[:n_free].astype(np.int32) + 5000
    dev = [torch.tensor(v, dtype=torch.int32, device="cuda") for v in (lengths, added)]
    tab = torch.from_numpy(table).cuda()
    slots = torch.full((n_slots,), 99, dtype=torch.int64, device="cuda")
    positions = torch.full((n_slots,), 99, dtype=torch.int32, device="cuda")
    got = B.page_tables(*dev, page, torch.from_numpy(free).cuda(), tab[:, :width], slots, positions)
    want = P.page_tables(lengths, added, page, free, table[:, :width], n_slots)
    for name, w in zip(("table", "slots", "positions", "starts", "lengths", "counts"), want):
        assert got[name].cpu().tolist() == np.asarray(w).tolist(), name
    if pad:
        assert np.array_equal(tab[:, width:].cpu().numpy(), table[:, width:])
    assert dev[0].tolist() == list(lengths) and dev[1].tolist() == list(added)
    return got


@pytest.mark.parametrize("page", [16, 64, 256])
@pytest.mark.parametrize("n", [1, 2, 63, 64, 65, 255, 1000, 1024, 1025, 3000, 9000])
def test_tables_of_ragged_requests(B, page, n):
    rng = _rng(n, page)
    lengths = rng.integers(0, 2000, n)
    added = np.where(rng.random(n) < 0.3, rng.integers(0, 40 if n > 100 else 900, n), rng.integers(0, 2, n))
    need = int((-(-(lengths + added) // page) + (-lengths // page)).sum())
    width = -(-3000 // page)
    _run_tables(B, lengths.tolist(), added.tolist(), page, need + 3, width, int(added.sum()) + 11, pad=1)
    # too few pages, too narrow a table, too few slots: what does not fit gets nothing
    _run_tables(B, lengths.tolist(), added.tolist(), page, need // 2, width, int(added.sum()) + 11)
    _run_tables(B, lengths.tolist(), added.tolist(), page, need, max(1, width // 3), int(added.sum()) + 11)
    _run_tables(B, lengths.tolist(), added.tolist(), page, need, width, int(added.sum()) * 2 // 3)


@pytest.mark.parametrize("lengths,added,page,n_free,width,n_slots", [
    ([0], [0], 16, 0, 1, 3), ([0], [1], 16, 1, 1, 1), ([15], [1], 16, 0, 1, 1), ([16], [1], 16, 1, 2, 1),
    ([16], [1], 16, 0, 2, 4), ([-3, 5], [4, -2], 16, 2, 3, 9), ([0, 0, 0], [0, 0, 0], 32, 4, 1, 0),
    ([0, 7], [100000, 3], 16, 7000, 7000, 100010), ([5], [2000000], 64, 40000, 40000, 2000001), ([3], [4], 1024, 0, 1, 9),
    ([1], [50], 16, 10, 0, 60)])
def test_tables_at_the_edges(B, lengths, added, page, n_free, width, n_slots):
    _run_tables(B, lengths, added, page, n_free, width, n_slots)


def test_tables_of_no_request(B):
    e = torch.empty(0, dtype=torch.int32, device="cuda")
    slots, positions = torch.ones(5, dtype=torch.int64, device="cuda"), torch.ones(5, dtype=torch.int32, device="cuda")
    got = B.page_tables(e, e, 16, e, e.reshape(0, 4), slots, positions)
    assert got["starts"].tolist() == [0] and got["counts"].tolist() == [0, 0, 0]
    assert got["slots"].tolist() == [-1] * 5 == got["positions"].tolist()


def test_tables_with_almost_2_31_slots(B):
    """The last slots' numbers stand close below what an int holds, for one launch and for two."""
    room = 2 ** 31 - 100
    slots = torch.empty(room, dtype=torch.int64, device="cuda")
    positions = torch.empty(room, dtype=torch.int32, device="cuda")
    for n in (3, 5000):
        slots.fill_(99)
        positions.fill_(99)
        lengths, added = torch.arange(n, dtype=torch.int32), torch.full((n,), 2, dtype=torch.int32)
        free, table = np.arange(n * 2 + 400, dtype=np.int32), np.zeros((n, n // 16 + 2), np.int32)
        want = P.page_tables(lengths.tolist(), added.tolist(), 16, free, table, 2 * n)
        got = B.page_tables(lengths.cuda(), added.cuda(), 16, torch.from_numpy(free).cuda(), torch.from_numpy(table).cuda(), slots,
                            positions)
        assert slots[:2 * n].tolist() == want[1] and positions[:2 * n].tolist() == want[2]
        for a in range(2 * n, room, 1 << 28):
            assert bool((slots[a:a + (1 << 28)] == -1).all()) and bool((positions[a:a + (1 << 28)] == -1).all()), a
        assert got["counts"].tolist() == want[5]


# ------------------------------------------------------------------------------ tokens in and out
def _slots(rng, T, places):
    """Runs of consecutive slots, some alone, some outside the cache."""
    order = []
    while len(order) < T:
        a = int(rng.integers(0, places))
        order += [s for s in range(a, min(places, a + int(rng.integers(1, 40)))) if s not in order]
    order = order[:T]
    for i in range(0, T, 7):
        order[i] = [-1, places, -(1 << 40), 1 << 40][i // 7 % 4] if i % 2 else order[i]
    return np.array(order, np.int64)


@pytest.mark.parametrize("kind", sorted(TYPES))
@pytest.mark.parametrize("T,H,D,page", [(1, 1, 32, 16), (5, 2, 64, 16), (40, 3, 96, 32), (70, 1, 128, 64), (33, 2, 160, 16),
                                        (20, 1, 224, 128), (17, 2, 256, 64), (150, 1, 192, 16)])
def test_tokens_in_and_out(B, kind, T, H, D, page):
    rng = _rng(T, H, D)
    pages = -(-3 * T // page) + 1
    k, v = _real(rng, (T, H, D), kind), _real(rng, (T, H, D), kind)
    k[0, 0, :32] = 0
    v[T // 2, H - 1, 3], k[T // 2, 0, 5], v[T // 2, 0, 6] = float("nan"), float("inf"), float("-inf")
    slots = _slots(rng, T, pages * page)
    before = rng.integers(0, 256, (pages, H, page // 16, 18 * D)).astype(np.uint8)
    cache = torch.from_numpy(before.copy()).cuda()
    # keys and values as slices of a joint projection's rows, at an odd place for fp32 and the 16-bit types alike
    joint = torch.zeros((T, 3, H, D + 8), dtype=TYPES[kind], device="cuda")
    joint[:, 1, :, 8:] = k.cuda()
    joint[:, 2, :, 8:] = v.cuda()
    dev = torch.from_numpy(slots).cuda()
    B.kv4_write(cache, joint[:, 1, :, 8:], joint[:, 2, :, 8:], dev)
    want = before.copy()
    P.kv4_write(want, k.float().numpy(), v.float().numpy(), slots, page)
    assert np.array_equal(cache.cpu().numpy(), want)
    # the same through unaligned rows
    odd = torch.zeros((T, H, D + 1), dtype=TYPES[kind], device="cuda")[:, :, 1:]
    other = torch.from_numpy(before.copy()).cuda()
    B.kv4_write(other, odd.copy_(k), v.cuda(), dev)
    assert torch.equal(other, cache)
    inside = (slots >= 0) & (slots < pages * page)
    for out_kind in sorted(TYPES):
        got = B.kv4_read(cache, dev, dtype=TYPES[out_kind])
        for g, x in zip(got, (k, v)):
            held = torch.from_numpy(P.kv4_values(x.float().numpy()) * inside[:, None, None])
            assert torch.equal(g.cpu(), held.to(torch.float32).to(TYPES[out_kind]))
    out = [torch.full((T, H, D + 3), 5.0, dtype=TYPES[kind], device="cuda") for _ in range(2)]
    B.kv4_read(cache, dev, out[0][:, :, 1:-2], out[1][:, :, 1:-2])
    same = B.kv4_read(cache, dev, dtype=TYPES[kind])
    for o, s in zip(out, same):
        assert torch.equal(o[:, :, 1:-2], s) and bool((o[:, :, :1] == 5).all()) and bool((o[:, :, -2:] == 5).all())


def test_more_tokens_than_a_launch_takes(B):
    """2^28 tokens and some, most of which go nowhere."""
    T, D, n = (1 << 28) + 37, 32, 100
    k = torch.zeros((T, 1, D), dtype=torch.float16, device="cuda")
    slots = torch.full((T,), -1, dtype=torch.int64, device="cuda")
    rng = _rng(18)
    rows = torch.cat([torch.arange(n), (1 << 28) - 66 + torch.arange(n), T - 3 + torch.arange(3)]).cuda()
    some = _real(rng, (2 * n + 3, 1, D), "f16")
    k[rows] = some.cuda()
    at = torch.from_numpy(rng.permutation(2 * n + 3)).cuda()
    slots[rows] = at
    cache = B.kv4_cache(13, 1, 16, D)
    B.kv4_write(cache, k, k, slots)
    want = torch.from_numpy(P.kv4_values(some.float().numpy())).half()
    for x in B.kv4_read(cache, at, dtype=torch.float16):
        assert torch.equal(x.cpu(), want)
    del k
    for x in B.kv4_read(cache, slots, dtype=torch.float16):
        assert torch.equal(x[rows].cpu(), want)
        x[rows] = 0
        assert not bool(x.any())


@pytest.mark.parametrize("size", [0.0, 1e-9, 1e-6, 1e-3, 100.0, 6e4, 1e6])
def test_sizes_that_the_cache_holds(B, size):
    """Factors down to binary16's smallest number and up to the largest that 8 of still fit."""
    k = _real(_rng(3), (16, 1, 64), "f32") * size
    cache = B.kv4_cache(1, 1, 16, 64)
    slots = torch.arange(16, device="cuda")
    B.kv4_write(cache, k.cuda(), -k.cuda(), slots)
    got = B.kv4_read(cache, slots, dtype=torch.float32)
    assert np.array_equal(got[0].cpu().numpy(), P.kv4_values(k.numpy()).astype(np.float32))
    assert np.array_equal(got[1].cpu().numpy(), P.kv4_values(-k.numpy()).astype(np.float32))


# ------------------------------------------------------------------------------ attention
def _filled(B, rng, lengths, H, D, page, spare=2, kv=None):
    """A cache of requests of these lengths on shuffled pages; unwritten places hold bytes that are no numbers."""
    held = [-(-n // page) for n in lengths]
    pool = sum(held) + spare
    width = max(max(held), 1) + 1
    order = rng.permutation(pool)
    table = np.full((len(lengths), width), -1, np.int32)
    at = 0
    for b, n in enumerate(held):
        table[b, :n] = order[at:at + n]
        at += n
    cache = torch.full((pool, H, page // 16, 18 * D), 255, dtype=torch.uint8, device="cuda")   # binary16 NaN factors
    keys, values, ks, vs, slots = [], [], [], [], []
    for b, n in enumerate(lengths):
        k, v = kv(b, n) if kv else (_real(rng, (n, H, D), "f32"), _real(rng, (n, H, D), "f32"))
        ks.append(k)
        vs.append(v)
        slots += [int(table[b, i // page]) * page + i % page for i in range(n)]
        keys.append(P.kv4_values(k.numpy()))
        values.append(P.kv4_values(v.numpy()))
    if slots:
        B.kv4_write(cache, torch.cat(ks).cuda(), torch.cat(vs).cuda(), torch.tensor(slots, device="cuda"))
    return cache, torch.from_numpy(table).cuda(), keys, values


def _check_attend(B, rng, lengths, added, H, ratio, D, page, kind, window=0, scale=None, workspace=True, peak=1.0):
    cache, table, keys, values = _filled(B, rng, lengths, H, D, page)
    T = sum(added)
    q = (_real(rng, (T, H * ratio, D), "f32") * peak).to(TYPES[kind])
    starts = np.concatenate([[0], np.cumsum(added)]).tolist()
    scale = D ** -0.5 if scale is None else scale
    lens = torch.tensor(lengths, dtype=torch.int32, device="cuda")
    first = None if all(a == 1 for a in added) else torch.tensor(starts, dtype=torch.int32, device="cuda")
    ws = B.kv4_attend_workspace(q, cache, len(lengths), max(lengths + [1])) if workspace else None
    out = torch.full((T, H * ratio, D), 9.0, dtype=TYPES[kind], device="cuda")
    got = B.kv4_attend(q.cuda(), cache, table, lens, first, scale, window=window, out=out, workspace=ws)
    want, most = P.attend(q.double().numpy(), keys, values, lengths, starts, scale, window)
    off = np.abs(got.double().cpu().numpy() - want)
    bound = P.attend_tolerance(want, values, most, TYPES[kind])
    assert np.all(off <= bound), (float(np.nanmax(off / bound)), bool(np.isnan(off).any()))
    return q, cache, table, lens, first, got


@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("D", range(32, 257, 32))
def test_attention_of_single_tokens(B, kind, D):
    _check_attend(B, _rng(D), [1, 0, 70, 16, 200, 64, 65], [1] * 7, 2, 3, D, 16, kind)


@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("D", range(32, 257, 32))
def test_attention_of_several_tokens(B, kind, D):
    _check_attend(B, _rng(D, 1), [130, 20, 3, 0, 50], [70, 20, 0, 0, 1], 2, 3, D, 32, kind)


@pytest.mark.parametrize("ratio", [1, 2, 4, 5, 8, 16, 17, 40])
@pytest.mark.parametrize("page", [16, 64, 256])
def test_attention_by_heads_and_pages(B, ratio, page):
    _check_attend(B, _rng(ratio, page), [40, 129, 1, 300], [1] * 4, 2, ratio, 64, page, "bf16")
    _check_attend(B, _rng(ratio, page, 1), [40, 129, 2, 300], [3, 40, 2, 33], 1, ratio, 64, page, "bf16")


@pytest.mark.parametrize("lengths", [[5000], [4097, 1, 900], [513, 512, 511, 0], [20000]])
@pytest.mark.parametrize("workspace", [True, False])
def test_attention_over_long_contexts(B, lengths, workspace):
    _check_attend(B, _rng(*lengths), lengths, [1] * len(lengths), 2, 4, 64, 64, "bf16", workspace=workspace)
    _check_attend(B, _rng(*lengths), lengths, [min(n, 5) for n in lengths], 1, 2, 128, 32, "f16", workspace=workspace)


@pytest.mark.parametrize("window", [1, 2, 15, 16, 63, 64, 65, 100, 5000])
def test_attention_in_a_window(B, window):
    lengths = [300, 64, 1, 700, 0]
    _check_attend(B, _rng(window), lengths, [1] * 5, 2, 2, 64, 16, "bf16", window=window)
    _check_attend(B, _rng(window, 1), lengths, [90, 64, 1, 37, 0], 1, 3, 96, 32, "bf16", window=window)


@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("D,H,ratio", [(32, 16, 8), (64, 16, 7), (96, 16, 4), (128, 16, 8), (160, 16, 8), (192, 16, 5), (224, 16, 8),
                                       (256, 16, 8)])
def test_attention_of_prompts(B, kind, D, H, ratio):
    """Columns enough for the wide tiles: ragged prompts, in part over what the cache holds, some empty."""
    lengths, added = [330, 0, 200, 70, 129], [150, 0, 200, 70, 1]
    _check_attend(B, _rng(D, 3), lengths, added, H, ratio, D, 32, kind)


@pytest.mark.parametrize("window", [1, 17, 64, 130, 1000])
def test_attention_of_prompts_in_a_window(B, window):
    _check_attend(B, _rng(window, 2), [400, 150, 90], [300, 150, 100], 16, 4, 64, 16, "bf16", window=window)
    _check_attend(B, _rng(window, 3), [400, 150, 90], [300, 150, 100], 16, 4, 64, 16, "f16", window=window, scale=-0.2)


@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("D,H,ratio,window", [(32, 4, 8, 0), (64, 4, 7, 0), (128, 4, 8, 0), (128, 5, 6, 600), (192, 4, 8, 0), (256, 4, 8, 0),
                                              (96, 12, 3, 40)])
def test_attention_of_cut_prompts(B, kind, D, H, ratio, window):
    """Few wide tiles over tables that hold long contexts: the keys are cut, and the parts are added in the same order
    every time."""
    rng = _rng(D, H, 5)
    lengths, added, page, longest = [1500, 0, 700, 2300, 40], [60, 0, 130, 64, 40], 32, 140000
    cache, table, keys, values = _filled(B, rng, lengths, H, D, page)
    table = torch.nn.functional.pad(table, (0, longest // page - table.shape[1]), value=-1)
    T, starts = sum(added), [0, 60, 60, 190, 254, 294]
    q = _real(rng, (T, H * ratio, D), "f32").to(TYPES[kind])
    lens, first = [torch.tensor(v, dtype=torch.int32, device="cuda") for v in (lengths, starts)]
    ws = B.kv4_attend_workspace(q, cache, len(lengths), longest)
    assert ws.numel() >= 1024 * 128 * (D + 2) * 4
    got = B.kv4_attend(q.cuda(), cache, table, lens, first, window=window, workspace=ws)
    want, most = P.attend(q.double().numpy(), keys, values, lengths, starts, D ** -0.5, window)
    bound = P.attend_tolerance(want, values, most, TYPES[kind])
    assert np.all(np.abs(got.double().cpu().numpy() - want) <= bound)
    for _ in range(10):
        assert torch.equal(got, B.kv4_attend(q.cuda(), cache, table, lens, first, window=window, workspace=ws))
    # the same workspace for single tokens, whose parts are others, and back
    one = torch.arange(6, dtype=torch.int32, device="cuda")
    few = B.kv4_attend(q[:5].cuda(), cache, table, lens, one, window=window, workspace=ws)
    assert torch.equal(few, B.kv4_attend(q[:5].cuda(), cache, table, lens, one, window=window,
                                         workspace=B.kv4_attend_workspace(q[:5], cache, len(lengths), longest)))
    assert torch.equal(got, B.kv4_attend(q.cuda(), cache, table, lens, first, window=window, workspace=ws))


@pytest.mark.parametrize("peak,scale", [(0.0, None), (1e-6, None), (30.0, None), (1.0, -0.3), (1.0, 0.0), (3000.0, 1e-4), (1e-3, 1e-5)])
def test_attention_of_flat_and_peaked_prompts(B, peak, scale):
    """Scales that fit the queries' binary16 and such that do not."""
    for kind in ("bf16", "f16") if peak < 1000.0 else ("bf16",):         # (the largest are no fp16 numbers)
        _check_attend(B, _rng(9, 9), [300, 90], [130, 90], 16, 8, 64, 16, kind, scale=scale, peak=peak)


def test_attention_of_prompts_reads_no_page_that_a_request_has_not(B):
    rng = _rng(16)
    H, ratio, D, page = 16, 8, 64, 16
    cache, table, keys, values = _filled(B, rng, [200, 130], H, D, page)
    table[0, 2], table[1, 0] = 1 << 30, -7
    q = _real(rng, (330, H * ratio, D), "bf16")
    lens, starts = [torch.tensor(v, dtype=torch.int32, device="cuda") for v in ([200, 130], [0, 200, 330])]
    got = B.kv4_attend(q.cuda(), cache, table, lens, starts).double().cpu().numpy()
    for rows, b, gone in ((range(48, 200, 19), 0, slice(32, 48)), (range(216, 330, 23), 1, slice(0, 16))):
        for t in rows:
            n = t + 1 - starts[b].item()
            k, v = [np.delete(x[b][:n], gone, 0) for x in (keys, values)]
            want, most = P.attend(q[t:t + 1].double().numpy(), [k], [v], [len(k)], [0, 1], D ** -0.5, 0)
            assert np.all(np.abs(got[t:t + 1] - want) <= P.attend_tolerance(want, [v], most, torch.bfloat16)), t


def test_attention_of_more_rows_than_tokens(B):
    """A request with more rows than tokens in the cache: the first rows stand in front of its first key."""
    _check_attend(B, _rng(8), [3, 0, 20], [5, 4, 30], 2, 2, 64, 16, "bf16")


@pytest.mark.parametrize("peak,scale", [(0.0, None), (1e-6, None), (30.0, None), (1.0, -0.3), (1.0, 0.0), (3000.0, 1e-4)])
def test_attention_of_flat_and_peaked_rows(B, peak, scale):
    for kind in ("bf16", "f16"):
        _check_attend(B, _rng(5), [200, 33], [1, 1], 2, 4, 64, 16, kind, peak=peak, scale=scale)


@pytest.mark.parametrize("rows", [1, 8])
def test_attention_averages_a_long_context(B, rows):
    """Equal weights over many keys: what is left of values that cancel is 1 / sqrt(keys) of them, and what a sum loses in one
    direction shows.  The output's rounding and that of each product are 2^-12 of their size at most, on average a half of
    it, with signs that cancel like the values': together they stay below 2^-11 of the output's norm."""
    rng = _rng(rows, 61)
    H, ratio, D, page, n = 2, 16, 64, 64, 30000
    cache, table, keys, values = _filled(B, rng, [n], H, D, page)
    T = 1 if rows == 1 else 256                                          # (256 tokens of 16 heads: wide tiles)
    q = torch.zeros((T, H * ratio, D), dtype=torch.float16)
    lens, first = [torch.tensor(v, dtype=torch.int32, device="cuda") for v in ([n], [0, T])]
    got = B.kv4_attend(q.cuda(), cache, table, lens, first, workspace=B.kv4_attend_workspace(q, cache, 1, n))
    upto = np.cumsum(values[0], 0)[n - T:] / np.arange(n - T + 1, n + 1)[:, None, None]
    want = np.repeat(upto, ratio, 1)
    off = got.double().cpu().numpy() - want
    assert np.linalg.norm(off) <= 2.0 ** -11 * np.linalg.norm(want), np.linalg.norm(off) / np.linalg.norm(want)


def test_attention_reads_no_page_that_a_request_has_not(B):
    """Pages outside the cache inside a request's length: their tokens are not seen, whatever the table says."""
    rng = _rng(12)
    H, D, page = 2, 64, 16
    cache, table, keys, values = _filled(B, rng, [100, 50], H, D, page)
    table[0, 2], table[1, 0] = 1 << 30, -7
    q = _real(rng, (2, 4, D), "bf16")
    got = B.kv4_attend(q.cuda(), cache, table, torch.tensor([100, 50], dtype=torch.int32, device="cuda"))
    for k in (keys, values):
        k[0] = np.delete(k[0], range(32, 48), 0)
        k[1] = k[1][16:]
    want, most = P.attend(q.double().numpy(), keys, values, [84, 34], [0, 1, 2], D ** -0.5, 0)
    bound = P.attend_tolerance(want, values, most, torch.bfloat16)
    assert np.all(np.abs(got.double().cpu().numpy() - want) <= bound)
    # a window whose first pages have been given away
    whole = int(table[0, 1])                                     # (a page that the first request has filled)
    table[:] = -1
    table[0, 3] = whole
    lens = torch.tensor([64, 0], dtype=torch.int32, device="cuda")
    got = B.kv4_attend(q.cuda(), cache, table, lens, window=16)
    assert bool(torch.isfinite(got).all()) and not bool(got[1].any())


def test_attention_leaves_other_rows_alone(B):
    """Strided queries and outputs; rows in front of the first request's and behind the last one's stay as they are."""
    rng = _rng(13)
    H, ratio, D = 2, 2, 64
    lengths, starts = [40, 20], [2, 5, 6]
    cache, table, keys, values = _filled(B, rng, lengths, H, D, 16)
    q = torch.zeros((9, H * ratio + 1, D + 1), dtype=torch.bfloat16, device="cuda")
    out = torch.full((9, H * ratio + 2, D + 3), 7.0, dtype=torch.bfloat16, device="cuda")
    rows = _real(rng, (9, H * ratio, D), "bf16")
    q[:, 1:, 1:] = rows.cuda()
    B.kv4_attend(q[:, 1:, 1:], cache, table, torch.tensor(lengths, dtype=torch.int32, device="cuda"),
                 torch.tensor(starts, dtype=torch.int32, device="cuda"), out=out[:, 1:-1, 1:-2])
    want, most = P.attend(rows[2:6].double().numpy(), keys, values, lengths, [0, 3, 4], D ** -0.5, 0)
    got = out[2:6, 1:-1, 1:-2].double().cpu().numpy()
    assert np.all(np.abs(got - want) <= P.attend_tolerance(want, values, most, torch.bfloat16))
    out[2:6, 1:-1, 1:-2] = 7.0
    assert bool((out == 7).all())


def test_the_last_pages_of_a_large_cache(B):
    """Byte offsets beyond 32 bits."""
    H, D, page = 8, 256, 16
    pages = (9 << 29) // (H * 18 * D) + 1                       # 4.5 GiB
    cache = torch.empty((pages, H, 1, 18 * D), dtype=torch.uint8, device="cuda")
    rng = _rng(14)
    n = 45
    k, v = _real(rng, (n, H, D), "bf16"), _real(rng, (n, H, D), "bf16")
    table = torch.tensor([[pages - 1, pages - 4, pages // 2]], dtype=torch.int32, device="cuda")
    at = torch.arange(n, device="cuda")
    slots = table[0].long()[at // page] * page + at % page
    B.kv4_write(cache, k.cuda(), v.cuda(), slots)
    got = B.kv4_read(cache, slots, dtype=torch.float32)
    keys, values = P.kv4_values(k.float().numpy()), P.kv4_values(v.float().numpy())
    assert np.array_equal(got[0].cpu().numpy(), keys.astype(np.float32))
    assert np.array_equal(got[1].cpu().numpy(), values.astype(np.float32))
    q = _real(rng, (1, 2 * H, D), "bf16")
    out = B.kv4_attend(q.cuda(), cache, table, torch.tensor([n], dtype=torch.int32, device="cuda"))
    want, most = P.attend(q.double().numpy(), [keys], [values], [n], [0, 1], D ** -0.5, 0)
    assert np.all(np.abs(out.double().cpu().numpy() - want) <= P.attend_tolerance(want, [values], most, torch.bfloat16))


def test_attention_is_the_same_every_time(B):
    """Whichever part of a split ends last, and however often the workspace is used."""
    rng = _rng(15)
    q, cache, table, lens, first, got = _check_attend(B, rng, [3000, 2000], [1, 1], 2, 4, 128, 64, "bf16")
    ws = B.kv4_attend_workspace(q, cache, 2, 3000)
    for _ in range(20):
        assert torch.equal(got, B.kv4_attend(q.cuda(), cache, table, lens, first, workspace=ws))
    more = [_check_attend(B, rng, [9000, 30, 700], [1, 2, 0], 1, 3, 64, 32, "f16")]
    for q, cache, table, lens, first, got in more:
        for _ in range(20):
            assert torch.equal(got, B.kv4_attend(q.cuda(), cache, table, lens, first, workspace=ws))


# lengths, added, key heads, query heads to each, page, tokens that the table has places for (0: no workspace): which
# kernel takes them, and whether it cuts the keys
PATHS = {"rows": ([300, 200, 70, 1, 513], [1] * 5, 4, 8, 64, 0), "rows, cut": ([5000, 900], [1, 1], 2, 8, 64, 5000),
         "prompts": ([330, 200, 129], [150, 200, 100], 16, 8, 32, 0), "prompts, cut": ([2300, 700], [64, 130], 4, 8, 32, 140000)}


def _path(B, rng, path, kind, D, spread, value_size=None, key_size=1.0, window=0, sign=1):
    """Attention on that path over scores that spread by `spread`, values of `value_size(request, tokens)` and keys of
    `key_size`; -> (outputs, expected ones, a function that gives the expected ones with other arguments)."""
    lengths, added, H, ratio, page, longest = PATHS[path]

    def kv(b, n):
        size = 1.0 if value_size is None else value_size(b, n)
        k, v = rng.standard_normal((n, H, D)) * key_size, rng.standard_normal((n, H, D)) * size
        return torch.from_numpy(k.astype(np.float32)), torch.from_numpy(v.astype(np.float32))

    cache, table, keys, values = _filled(B, rng, lengths, H, D, page, kv=kv)
    q = torch.from_numpy((rng.standard_normal((sum(added), H * ratio, D)) * spread).astype(np.float32)).to(TYPES[kind])
    starts = np.concatenate([[0], np.cumsum(added)]).tolist()
    lens, first = [torch.tensor(v, dtype=torch.int32, device="cuda") for v in (lengths, starts)]
    ws = None
    if longest:
        table = torch.nn.functional.pad(table, (0, max(0, -(-longest // page) - table.shape[1])), value=-1)
        ws = B.kv4_attend_workspace(q, cache, len(lengths), longest)
        assert ws.numel()
    scale = sign * D ** -0.5 / key_size
    got = B.kv4_attend(q.cuda(), cache, table, lens, first if "prompts" in path else None, scale, window=window, workspace=ws)

    def expected(scale=scale, values=values, window=window):
        return P.attend_rows(q.double().numpy(), keys, values, lengths, starts, scale, window)

    return got.double().cpu().numpy(), expected(), lambda **kw: expected(**{**kw, "scale": scale * kw.get("scale", 1.0)}), values


def _close(got, want, kind, path, spread):
    off, bound = np.linalg.norm(got - want), P.attend_norm(want, TYPES[kind], "prompts" in path, spread)
    assert off <= bound, (off / np.linalg.norm(want), bound / np.linalg.norm(want))


@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("path", sorted(PATHS))
def test_attention_over_values_of_any_size(B, path, kind):
    """From the largest that the cache holds to such as have factors that are subnormal in binary16."""
    for i, size in enumerate((5000.0, 0.05, 1e-2, 1e-4, 1e-6)):
        got, want, *_ = _path(B, _rng(i, 71), path, kind, 64, 2.0, lambda b, n: size)
        _close(got, want, kind, path, 2.0)


@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("path", sorted(PATHS))
def test_attention_over_values_of_different_sizes(B, path, kind):
    """A context whose first tokens have tiny values and whose later ones large ones, and the other way round; and groups of
    channels of different size, each held to its own norm."""
    for first, behind in ((1e-5, 1.0), (300.0, 1e-2)):
        got, want, *_ = _path(B, _rng(72), path, kind, 96, 2.0, lambda b, n: np.where(np.arange(n) < 64, first, behind)[:, None, None])
        _close(got, want, kind, path, 2.0)
    sizes = np.repeat([1.0, 1e-3, 30.0], 32)
    got, want, *_ = _path(B, _rng(73), path, kind, 96, 2.0, lambda b, n: sizes)
    for g in range(3):
        _close(got[..., 32 * g:32 * g + 32], want[..., 32 * g:32 * g + 32], kind, path, 2.0)


def _within(got, want, kind, path, spread, window=0):
    """Whether the outputs, and where scores are not so far apart that a row is one key's value, those of each row and of
    each head, are as near as roundings leave them; of rows that see 16 keys or more."""
    lengths, added = PATHS[path][:2]
    seen = np.concatenate([np.minimum(np.arange(n - a, n) + 1, window or n) for n, a in zip(lengths, added)])
    got, want = got[seen >= 16], want[seen >= 16]
    parts = [(got, want)]
    if spread <= 2.0:
        parts += list(zip(got, want)) + list(zip(got.swapaxes(0, 1), want.swapaxes(0, 1)))
    return all(np.linalg.norm(g - w) <= P.attend_norm(w, TYPES[kind], "prompts" in path, spread) for g, w in parts)


@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("path", sorted(PATHS))
@pytest.mark.parametrize("D", range(32, 257, 32))
def test_attention_is_as_near_as_roundings_leave_it(B, D, path, kind):
    """... and nothing else is: neither zeros, nor a scale that is 2 % off, nor a context whose last value is missing."""
    got, want, other, values = _path(B, _rng(D, 81), path, kind, D, 2.0)
    assert _within(got, want, kind, path, 2.0)
    short = [np.concatenate([v[:-1], 0 * v[-1:]]) for v in values]
    for wrong in (0 * want, other(scale=1.02), other(values=short)):
        assert not _within(wrong, want, kind, path, 2.0)


@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("path", sorted(PATHS))
@pytest.mark.parametrize("spread,window,sign", [(0.0, 0, 1), (1.0, 0, -1), (8.0, 0, 1), (32.0, 0, -1), (2.0, 17, 1), (2.0, 100, -1)])
def test_attention_is_as_near_over_other_scores(B, spread, window, sign, path, kind):
    """Equal weights, scores far apart, windows, negative scales."""
    got, want, other, _ = _path(B, _rng(int(spread), window, 82), path, kind, 64, spread, window=window, sign=sign)
    assert _within(got, want, kind, path, spread, window)
    if window:
        assert not _within(other(window=window + 1), want, kind, path, spread, window)


@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("path", sorted(PATHS))
def test_attention_over_keys_of_any_size(B, path, kind):
    """From the largest to such as have factors that are subnormal in binary16, at scales that make up for them."""
    for i, size in enumerate((5000.0, 1e-2, 1e-4, 1e-6)):
        got, want, other, _ = _path(B, _rng(i, 83), path, kind, 64, 2.0, key_size=size)
        assert _within(got, want, kind, path, 2.0), size
        assert not _within(other(scale=1.02), want, kind, path, 2.0), size


@pytest.mark.parametrize("window", [2 ** 31 - 1, 2 ** 31 - 20, 2 ** 30, 65])
def test_attention_in_windows_of_any_length(B, window):
    """Requests with more rows than tokens: rows stand in front of the first key, by more than an int is short of the
    longest window."""
    for H, ratio, lengths, added in ((2, 2, [20, 70], [60, 71]), (16, 8, [20, 200], [150, 330])):
        for kind in ("bf16", "f16"):
            _check_attend(B, _rng(7, H), lengths, added, H, ratio, 64, 16, kind, window=window)


# ------------------------------------------------------------------------------ together
def _block(rng, requests=4, n_pages=60, most=400, **kw):
    from paper_1805_08691_amd.decoder import AttentionBlock
    E, H, ratio, D = 160, 2, 3, 64
    w_qkv = torch.from_numpy(rng.standard_normal((H * (ratio + 2) * D, E)).astype(np.float32) / E ** 0.5).cuda()
    w_out = torch.from_numpy(rng.standard_normal((E, H * ratio * D)).astype(np.float32) / 20).cuda()
    return E, w_qkv, w_out, AttentionBlock(w_qkv, w_out, H, ratio, D, n_pages, 16, requests, 400, most, **kw)


def test_a_block_serves_requests(B):
    """Prompts in pieces, decoding, a request that ends and another in its place: every output within what 8 and 4 bits
    cost of the block in fp32, and the pages add up."""
    from paper_1805_08691_amd.decoder import _plain
    rng = _rng(30)
    E, w_qkv, w_out, block = _block(rng)
    xs = [torch.from_numpy(rng.standard_normal((n, E)).astype(np.float32)).cuda() for n in (120, 70, 33, 200)]
    want = _plain(w_qkv, w_out, xs, 2, 3, 64)
    at, got = [0] * 4, [[] for _ in range(4)]
    for added in ([50, 0, 33, 90], [1, 70, 0, 60], [60, 0, 0, 1], [1, 0, 0, 1], [8, 0, 0, 48]):
        x = torch.cat([v[a:a + n] for v, a, n in zip(xs, at, added)]).bfloat16()
        y = block.step(x, added).float()
        for b, part in enumerate(y.split(added)):
            got[b].append(part)
        at = [a + n for a, n in zip(at, added)]
        assert block.lengths == at == block._lengths.tolist()
        assert block.taken == sum(-(-n // 16) for n in at)
    assert at == [120, 70, 33, 200]
    for g, w in zip(got, want):
        # 4-bit values: a code is off by a third of its factor in the mean, max / 7 / sqrt(12), against values of max / 2.5
        off = (torch.cat(g) - w).norm() / w.norm()
        assert off < 0.25, off
    block.release(1)
    taken = block.taken
    assert taken == sum(-(-n // 16) for n in (120, 33, 200))
    again = block.step(xs[1].bfloat16(), [0, 70, 0, 0]).float()
    assert block.taken == taken + 5 and torch.equal(again, torch.cat(got[1]))
    block.step(torch.zeros(400, E, dtype=torch.bfloat16, device="cuda"), [200, 0, 200, 0])       # 24 of 31 pages left
    state = block.table.clone(), list(block.lengths), block.taken
    with pytest.raises(MemoryError):                                     # 9 pages of 7 that are left
        block.step(torch.zeros(150, E, dtype=torch.bfloat16, device="cuda"), [0, 0, 150, 0])
    with pytest.raises(MemoryError):                                     # 6 pages, but 401 tokens of 400
        block.step(torch.zeros(81, E, dtype=torch.bfloat16, device="cuda"), [81, 0, 0, 0])
    assert torch.equal(state[0], block.table) and state[1:] == (block.lengths, block.taken)
    rows = [block.table[b, :-(-n // 16)] for b, n in enumerate(block.lengths)]
    used = torch.cat(rows).tolist()
    assert len(set(used)) == len(used) == block.taken


def test_a_step_is_its_calls(B):
    rng = _rng(31)
    E, _, _, block = _block(rng, b_out=torch.from_numpy(rng.standard_normal(160).astype(np.float32)).cuda())
    x = torch.from_numpy(rng.standard_normal((57, E)).astype(np.float32)).cuda().half()
    y = block.step(x, [30, 0, 20, 7])
    joint = block.qkv(x).view(57, -1, 64)
    slots = torch.cat([block.table[b].long()[torch.arange(n, device="cuda") // 16] * 16 + torch.arange(n, device="cuda") % 16
                       for b, n in enumerate(block.lengths)])
    other = torch.zeros_like(block.cache)
    B.kv4_write(other, joint[:, 6:8], joint[:, 8:], slots)
    assert torch.equal(other, block.cache)
    starts = torch.tensor([0, 30, 30, 50, 57], dtype=torch.int32, device="cuda")
    o = B.kv4_attend(joint[:, :6], other, block.table, block._lengths, starts)
    assert torch.equal(y, block.out(o.view(57, -1)))


def test_recorded_steps(B):
    """A decoding step recorded once and replayed with other values, between eager work and synchronizations."""
    rng = _rng(32)
    E, _, _, block = _block(rng, window=50)
    block.step(torch.from_numpy(rng.standard_normal((150, E)).astype(np.float32)).cuda().bfloat16(), [70, 30, 49, 1])
    one, dev = torch.ones(4, dtype=torch.int32, device="cuda"), torch.device("cuda")
    x = torch.zeros(4, E, dtype=torch.bfloat16, device=dev)
    slots, positions = torch.empty(4, dtype=torch.int64, device=dev), torch.empty(4, dtype=torch.int32, device=dev)
    free, out = torch.empty(4, dtype=torch.int32, device=dev), torch.empty_like(x)
    free.copy_(block.free[block.taken:block.taken + 4])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    keep = [t.clone() for t in (block.cache, block.table)]
    with torch.cuda.stream(side):
        block.launch(x, one, free, slots, positions, out=out)            # (a first call outside of the recording)
    torch.cuda.current_stream().wait_stream(side)
    for t, k in zip((block.cache, block.table), keep):
        t.copy_(k)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        block.launch(x, one, free, slots, positions, out=out)
    for i in range(6):
        new = torch.from_numpy(rng.standard_normal((4, E)).astype(np.float32)).cuda().bfloat16()
        x.copy_(new)
        free.copy_(block.free[block.taken:block.taken + 4])
        if i % 2:
            torch.cuda.synchronize()
        graph.replay()
        replayed = out.clone()
        cache = block.cache.clone()
        # the same step by eager launches, on another stream than the default one
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            y = block.launch(x, one, free, slots, positions)
        torch.cuda.current_stream().wait_stream(side)
        assert torch.equal(replayed, y) and torch.equal(cache, block.cache), i
        assert positions.tolist() == block.lengths
        block._lengths.copy_(block._grown)                               # (the recording's buffers stay in place)
        need = block.pages_needed([1] * 4)
        assert block._counts.tolist() == [need, 4, 0]
        block.lengths = [n + 1 for n in block.lengths]
        block.taken += need


def test_steps_on_two_streams(B):
    """Two blocks, each on a stream of its own, with buffers and workspaces of their own."""
    rng = _rng(33)
    blocks = [_block(rng)[3] for _ in range(2)]
    xs = [torch.from_numpy(rng.standard_normal((200, 160)).astype(np.float32)).cuda().bfloat16() for _ in range(2)]
    want = []
    for b, x in zip(blocks, xs):
        want.append([b.step(x, [100, 60, 0, 40]), b.step(x[:4], [1] * 4)])
        for r in range(4):
            b.release(r)
        b.cache.zero_()
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(3):
        got = [[], []]
        for added, n in (([100, 60, 0, 40], 200), ([1] * 4, 4)):
            for g, b, x, s in zip(got, blocks, xs, streams):
                with torch.cuda.stream(s):
                    g.append(b.step(x[:n], added))
        torch.cuda.synchronize()
        for g, w in zip(got, want):
            assert all(torch.equal(p, q) for p, q in zip(g, w))
        for b in blocks:
            for r in range(4):
                b.release(r)
        torch.cuda.synchronize()


def test_a_step_without_tokens(B):
    """None at all, on an empty block and between steps: an empty output, and nothing else."""
    rng = _rng(34)
    E, _, _, block = _block(rng)
    x = torch.from_numpy(rng.standard_normal((40, E)).astype(np.float32)).cuda().bfloat16()
    want = _block(_rng(34))[3].step(x, [30, 0, 10, 0])
    for added in ([0] * 4, [30, 0, 10, 0], [0] * 4):
        before = block.cache.clone(), block.table.clone(), list(block.lengths), block.taken
        y = block.step(x[:sum(added)], added)
        assert y.shape == (sum(added), E)
        if sum(added):
            assert torch.equal(y, want)
        else:
            assert torch.equal(before[0], block.cache) and torch.equal(before[1], block.table)
            assert before[2:] == (block.lengths, block.taken) and block._lengths.tolist() == block.lengths


def test_a_step_takes_no_negative_numbers(B):
    """The tables take them as 0 and the host would not: refused, with nothing done."""
    E, _, _, block = _block(_rng(35))
    x = torch.zeros(40, E, dtype=torch.bfloat16, device="cuda")
    block.step(x, [20, 0, 20, 0])
    before = block.cache.clone(), block.table.clone(), list(block.lengths), block.taken
    for added in ([-2, 12, 0, 0], [5, 6, 0, -1]):
        with pytest.raises(AssertionError):
            block.step(x[:10], added)
        assert torch.equal(before[0], block.cache) and torch.equal(before[1], block.table)
        assert before[2:] == (block.lengths, block.taken) and block._lengths.tolist() == block.lengths


def test_a_step_refuses_rows_before_it_does_anything(B):
    """fp32 rows, which the attention has no form for, and rows of another width, also one whose weights take as many bytes."""
    E, _, _, block = _block(_rng(36))
    block.step(torch.ones(40, E, dtype=torch.bfloat16, device="cuda"), [20, 0, 20, 0])
    before = block.cache.clone(), block.table.clone(), block._grown.clone()
    for x in (torch.zeros(50, E, device="cuda"), torch.zeros(50, E - 16, dtype=torch.bfloat16, device="cuda"),
              torch.zeros(50, 2 * E, dtype=torch.bfloat16, device="cuda"), torch.zeros(50, 1, E, dtype=torch.float16, device="cuda")):
        with pytest.raises(AssertionError):
            block.step(x, [0, 50, 0, 0])
        assert all(torch.equal(a, b) for a, b in zip(before, (block.cache, block.table, block._grown)))
        assert block.lengths == [20, 0, 20, 0]
