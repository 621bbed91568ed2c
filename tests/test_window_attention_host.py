"""Workspace of the windowed attention's gradient, on the host."""

import pytest

from paper_2501_17392_b200 import brace as B
from paper_2501_17392_b200 import build as brace_build


@pytest.fixture(scope="module", autouse=True)
def _built():
    brace_build.build()


def test_workspace_of_a_window():
    f, g = B.lib().brace_window_attention_window_workspace_bytes, B.lib().brace_window_attention_workspace_bytes
    for bad in [(-1, 1, 1, 1, 1, 1, 0), (1, 1, 3, 2, 1, 1, 0), (1, 1, 1, 1, 0, 1, 0), (1, 1, 1, 1, 1, 0, 0), (1, 1, 1, 1, 1, 1, -1),
                (1, 1, 1, 1, 257, 1, 0), (70000, 1, 1, 1, 1, 1, 0)]:
        assert f(*bad) == 0, bad
    for b, h, k, d, s in [(1, 32, 32, 128, 0), (2, 64, 1, 64, 4), (3, 8, 2, 40, 200), (1, 6, 3, 50, 1)]:
        lengths = [1, 100, 129, 1000, 10000, 65536, 65600, 140000, 300000]
        for n in lengths:
            sizes = [f(b, n, h, k, d, w, s) for w in (1, 100, 1024, 10000, 65536, 65537, 100000, 2 ** 31 - 1)]
            assert sizes == sorted(sizes) and sizes[-1] == g(b, n, h, k, d, s)     # one for a long window serves shorter ones
        for w in (100, 4096, 100000):
            sizes = [f(b, n, h, k, d, w, s) for n in lengths]
            assert sizes == sorted(sizes)


@pytest.mark.parametrize("n", [65536, 65600, 262144, 1 << 20])
@pytest.mark.parametrize("heads,kv,dim", [(32, 32, 128), (16, 4, 64), (8, 8, 200)])
def test_long_texts_with_short_windows_take_little(n, heads, kv, dim):
    """Two numbers of a query, and a third of a GB at most where no key is read by more than 65,536 queries; else 4 kv / heads
    of the queries' size more, or twice that size (head dimensions that the tensor cores do not take need no such sums)."""
    numbers, most = 8 * n * heads, 4 * 592 * 2 * 128 * max(dim, 128) * 4
    assert B.lib().brace_window_attention_window_workspace_bytes(1, n, heads, kv, dim, 1024, 4) <= numbers + most + 4096
    own = 0 if dim > 128 else (n + 127) * dim * 2 * max(4 * kv, 2 * heads)
    assert B.lib().brace_window_attention_workspace_bytes(1, n, heads, kv, dim, 4) <= numbers + most + own + 4096
