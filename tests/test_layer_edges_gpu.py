"""The bf16 layer, its gradients and the update at the edges of what their entry points accept."""

import pytest
import torch

pytestmark = pytest.mark.gpu

import paper_2607_24062_gb300 as acrl  # noqa: E402

DEV = "cuda"
BF, F32 = torch.bfloat16, torch.float32
MOST = 2 ** 31 - 8193    # rows or columns of a call


@pytest.mark.parametrize("M,N", [(1, MOST), (2, MOST - 100000), (3, 131073), (200, 5000)])
def test_column_sums_alone_up_to_the_most_columns(M, N):
    """dbias without a product beside it: whole numbers, whose sums are exact; nothing beyond the columns is written.  (About 50 GB
    for a row of the most columns.)"""
    dy = torch.empty((M, (N + 7) // 8 * 8), dtype=BF, device=DEV)
    at = torch.arange(dy.shape[1], device=DEV, dtype=torch.int32) % 251
    for i in range(M):
        dy[i] = (at + 3 * i).to(torch.uint8).to(BF)    # up to 255: exact in bf16
    del at
    dy = dy[:, :N]
    x, w = torch.empty((M, 0), dtype=BF, device=DEV), torch.empty((N, 0), dtype=BF, device=DEV)
    db = torch.full((N + 32,), -7.0, device=DEV)
    dx, dw, out = acrl.linear_backward(dy, x, w, bias=True, need_dx=False, need_dw=False, dbias=db)
    assert dx is None and dw is None and out.data_ptr() == db.data_ptr()
    step = 1 << 27
    for c in range(0, N, step):
        assert torch.equal(db[c: min(N, c + step)], dy[:, c: c + step].float().sum(0))
    assert bool((db[N:] == -7.0).all())
