"""The pages of a cache for more requests and pages than a launch's few blocks count at once: against the plain references of kv8_plain.py,
number for number."""
import numpy as np
import pytest
import torch

import kv8_plain as P

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_1805_08691_amd import binding
    return binding


def _dev(x):
    return torch.from_numpy(np.ascontiguousarray(np.asarray(x, np.int32))).cuda()


def _pool(rng, n, width, spare):
    """Rows of pages of their own, of up to width * 16 tokens, and a pool of `spare` pages more."""
    lengths = rng.integers(0, width * 16 + 1, n)
    held = -(-lengths // 16)
    order = rng.permutation(int(held.sum()) + spare).astype(np.int32)
    table, at = np.full((n, width), -1, np.int32), 0
    for b, k in enumerate(held):
        table[b, :k] = order[at:at + k]
        at += k
    return lengths.tolist(), table, len(order)


@pytest.mark.parametrize("n,m,width,spare", [(50000, 70000, 7, 60000), (3000, 70000, 5, 20000), (3000, 30000, 40, 700), (9000, 17000, 3, 0),
                                             (20, 66000, 4, 64), (70000, 300, 3, 100000),
                                             # the last sizes that one block takes, and the first that it does not
                                             (512, 1024, 3, 23587), (512, 1024, 3, 23588), (100, 1000, 16, 130000)])
def test_very_many_requests(B, n, m, width, spare):
    """More than 64 rows a thread, pages in hundreds of blocks, and requests of which most find no page for their copy."""
    rng = np.random.Generator(np.random.PCG64([1805, 8691, 90, n, m]))
    lengths, table, pool = _pool(rng, n, width, spare)
    parents = rng.integers(-1, n + 1, m)
    parents[m // 2:m // 2 + min(4000, m // 4)] = n // 3                       # (one of them very often)
    rows = _dev(table)
    got = B.page_select(_dev(parents), _dev(lengths), rows, 16, pool)
    out, lens, free, copies, counts = P.select(parents.tolist(), lengths, table, 16, pool)
    assert got["counts"].tolist() == counts
    assert np.array_equal(got["table"].cpu().numpy(), out) and got["lengths"].tolist() == lens
    assert got["free_pages"].tolist() == free and [tuple(x) for x in got["copies"].tolist()] == copies
    assert np.array_equal(rows.cpu().numpy(), table)
    moved = B.page_compact(got["lengths"], got["table"], 16, pool, table=got["table"])
    out, free, moves, counts = P.compact(lens, out, 16, pool)
    assert moved["counts"].tolist() == counts and np.array_equal(moved["table"].cpu().numpy(), out)
    assert moved["free_pages"].tolist() == free and [tuple(x) for x in moved["copies"].tolist()] == moves
