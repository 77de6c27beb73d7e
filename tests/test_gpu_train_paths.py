"""GPU parity of the training operators on the plans that large calls take: rows that
clusters of every size share, sorts of many tiles, several column slabs, long rows.
References and error bounds are those of test_gpu_train.py."""

import pytest
import torch

from paper_2608_08340_gb300.train import distill_loss

from test_gpu_train import _distill_plain, _rand, _teacher, _within

pytestmark = pytest.mark.gpu


# ------------------------------------------------------------- distillation

@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kb,q", [(100, 700), (300, 400), (700, 200), (1000, 120), (1100, 120)])
def test_distill_of_many_rows_that_clusters_share(dtype, kb, q):
    """Rows of 2, 4, 8, 16 and 16 larger CTAs, more of them than run at a time, so that
    CTAs of a cluster begin at different moments: the same bits every time, and the
    reference's values."""
    n = kb * 1000 // (2 if dtype == "bf16" else 4) + 5
    logits = _rand((q, n), dtype, kb, 0.2)
    ids, scores = _teacher(q, n, 20, kb + 1)
    loss, dz = distill_loss(logits, ids, scores, 0.1)
    for _ in range(8):
        again, dz2 = distill_loss(logits, ids, scores, 0.1)
        assert torch.equal(again, loss) and torch.equal(dz2, dz)
    for i in (0, q // 2, q - 1):
        part = slice(i, i + 1)
        want, grad, loss_bound, grad_bound = _distill_plain(logits[part], ids[part], scores[part],
                                                            0.1, None)
        _within(loss[part].cpu(), want, loss_bound, "f32", f"loss {i}")
        _within(dz[part].cpu(), grad, grad_bound, dtype, f"gradient {i}")
