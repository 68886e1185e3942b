"""Sizes that do not fit the 32 bits in which the library takes them are refused, not cut: 2^32 + 8 tokens are not 8."""
import pytest
import torch

from paper_2604_02715_amd import moe_block as M

BIG = (1 << 32) + 8


def big(*shape, dtype=torch.float32):
    return torch.zeros(1, 1, dtype=dtype).expand(*shape)


@pytest.fixture
def on_the_gpu(monkeypatch):
    """the sizes are looked at before anything else but the place"""
    monkeypatch.setattr(M, "_place", lambda t, name: -1)


@pytest.mark.parametrize("T,E,K", [(BIG, 8, 2), (4, BIG, 2), (4, 8, 1 << 32)])
def test_router(on_the_gpu, T, E, K):
    ids, gates, x = big(T, K, dtype=torch.int32), big(T, K), torch.zeros(T, E) if K > E else big(T, E)
    for call in (lambda: M.route(x, ids, gates), lambda: M.route_grad(x, ids, gates, x)):
        with pytest.raises(ValueError, match="2\\^32"):
            call()


@pytest.mark.parametrize("T,K,E,align", [(BIG, 2, 8, 1), (4, BIG, 8, 1), (4, 2, BIG, 1), (4, 2, 8, BIG), (4, 2, 8, -1)])
def test_sort(on_the_gpu, T, K, E, align):
    ids, small = big(T, K, dtype=torch.int32), torch.zeros(8, dtype=torch.int32)
    with pytest.raises(ValueError, match="2\\^32"):
        M.sort_tokens(ids, E, small, small, ids, small, align=align)


@pytest.mark.parametrize("T,K,H", [(BIG, 2, 8), (4, BIG, 8), (4, 2, BIG)])
def test_rows(on_the_gpu, T, K, H):
    pair_row, row_pair, x, rows, gates = big(T, K, dtype=torch.int32), torch.zeros(8, dtype=torch.int32), big(T, H), big(8, H), big(T, K)
    for call in (lambda: M.dispatch(x, pair_row, row_pair, rows), lambda: M.combine(rows, pair_row, gates, x),
                 lambda: M.combine_grad(x, rows, pair_row, row_pair, gates, rows, gates)):
        with pytest.raises(ValueError, match="2\\^32"):
            call()


@pytest.mark.parametrize("T,H", [(BIG, 8), (4, BIG)])
def test_norms(on_the_gpu, T, H):
    x, w = big(T, H), big(1, H)[0]
    for call in (lambda: M.block_norm(x, w, x), lambda: M.block_norm_grad(x, w, x, x, w, w)):
        with pytest.raises(ValueError, match="2\\^32"):
            call()


@pytest.mark.parametrize("call,good", [(M.sorted_rows, (100, 8, 160, 16)), (M.sort_workspace_bytes, (9000, 8, 160)),
                                       (M.block_norm_grad_workspace_bytes, (100, 4096))])
def test_queries(call, good):
    assert call(*good) > 0
    for i in range(len(good)):
        for bad in (good[i] + (1 << 32), -1):
            with pytest.raises(ValueError, match="2\\^32"):
                call(*good[:i], bad, *good[i + 1:])
