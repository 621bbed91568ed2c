"""Workspace of the windowed attention's gradient, and what it refuses, on the host: nothing is launched."""

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


P = 1 << 20        # an address that is aligned and never read


def arguments(batch=3, tokens=5, heads=4, kv=2, dim=8, **over):
    e = B.WindowAttentionArgs()
    e.batch, e.tokens, e.heads, e.kv_heads, e.dim, e.window, e.type, e.scale = batch, tokens, heads, kv, dim, 5, 0, 0.3
    e.d_lse, e.head_lse, e.stride_lse = P, tokens, tokens * heads
    for name in ("q", "k", "v", "out", "dout", "dq", "dk", "dv"):
        h = getattr(e, name)
        h.d, h.ld, h.head, h.stride = P, dim * heads, dim, dim * heads * tokens
    for name, strides in over.items():
        if name == "lse":
            e.head_lse, e.stride_lse = strides
        else:
            h = getattr(e, name)
            h.ld, h.head, h.stride = strides
    return e


# (tokens, heads, batch): of 5 tokens, 4 heads (2 of keys), 3 sequences, heads of 8; rows that two places share
OVERLAP = [(8, 8, 1000), (32, 8, 159), (1000, 8, 31), (8, 40, 50), (32, 9, 8), (31, 8, 1000), (8, 39, 1000), (100, 8, 100)]
# tokens first, heads first, sequences inside of tokens and of all, padded, the longest that there are
APART = [(32, 8, 160), (8, 40, 160), (96, 8, 32), (24, 120, 8), (1000, 9, 36), (40, 10, 200), (1 << 40, 8, 1 << 50)]


@pytest.mark.parametrize("name", ["dq", "dk", "dv"])
def test_results_whose_rows_overlap_are_refused(name):
    f = B.lib().brace_window_attention_grad
    for strides in OVERLAP:
        if name == "dq" or strides not in ((31, 8, 1000), (32, 8, 159), (1000, 8, 31)):      # two heads of keys take 16
            assert f(arguments(**{name: strides}), P, 0, None) == B.ERR_INVALID_ARG, strides
    for strides in APART:      # the workspace is what these are refused for
        assert f(arguments(**{name: strides}), P, 0, None) == B.ERR_WORKSPACE, strides
    for tokens, heads, batch, strides in [(1, 4, 3, (0, 8, 32)), (5, 2, 1, (16, 8, 0)), (5, 2, 3, (16, 8, 80)), (1, 2, 1, (0, 8, 0))]:
        e = arguments(batch, tokens, heads, heads, **{name: strides})
        assert f(e, P, 0, None) == B.ERR_WORKSPACE, strides


def test_outputs_and_sums_that_overlap_are_refused():
    for strides in OVERLAP:
        assert B.lib().brace_window_attention_forward(arguments(out=strides), None) == B.ERR_INVALID_ARG, strides
        assert B.lib().brace_window_attention_grad(arguments(q=strides, k=strides, v=strides, out=strides, dout=strides), P, 0,
                                                   None) == B.ERR_WORKSPACE      # these are only read
    for strides in [(5, 5), (5, 19), (15, 14), (14, 5), (4, 100), (10, 10)]:
        assert B.lib().brace_window_attention_forward(arguments(lse=strides), None) == B.ERR_INVALID_ARG, strides
        assert B.lib().brace_window_attention_grad(arguments(lse=strides), P, 0, None) == B.ERR_INVALID_ARG, strides
    for strides in [(5, 20), (15, 5), (7, 28), (1 << 40, 1 << 45)]:
        assert B.lib().brace_window_attention_grad(arguments(lse=strides), P, 0, None) == B.ERR_WORKSPACE, strides
