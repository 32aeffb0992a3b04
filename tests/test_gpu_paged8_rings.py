"""Attention of chunks over 8-bit pools: many short items in a row, pages without a copy among them, so that warps
which share a ring run ahead of one another.  Tolerances: tests/test_gpu_paged8.py."""
import pytest
import torch

from paged8_util import Batch8
from paged_util import ref_attend
from paper_2605_27255_gb300 import capi, paged
from test_gpu_paged8 import check, values_top

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d_h", [64, 128])
@pytest.mark.parametrize("length,n,window", [(400, 64, 70), (400, 64, 130), (331, 65, 10), (700, 130, 0), (64, 64, 0), (2000, 70, 900)])
def test_many_items_of_few_pages(d_h, length, n, window):
    """400 sequences that read the same blocks: the outputs of each are those of the first."""
    x = Batch8([length], [n], 4, 1, d_h, seed=71)
    ref = ref_attend(x.plain, d_h ** -0.5, window)
    seqs = 400
    c = paged.PagedCache8(x.k8.cuda(), x.v8.cuda(), x.k_scale.cuda(), x.v_scale.cuda(), x.table.repeat(seqs, 1).cuda(), n_q=4)
    qs = torch.arange(seqs + 1, dtype=torch.int32, device="cuda") * n
    kl = torch.full((seqs,), length, dtype=torch.int32, device="cuda")
    q = x.q.cuda().repeat(seqs, 1, 1)
    out = [c.attend(q, qs, kl, window=window) for _ in range(5)]
    capi.pipo_op_paged_check()
    for y in out:
        assert torch.equal(y, out[0])
    got = out[0].reshape(seqs, n, 4, d_h)
    for b in range(0, seqs, 7):
        check(got[b], ref, values_top(x))
    # (parts of shared items are joined: the last bit may differ)
    assert (got.float() - got[:1].float()).abs().max() <= 2.0 ** -7 * got.float().abs().max()
