"""Gradient of the token loss: what lies around its rows is not touched."""
import pytest
import torch

from paper_2402_17227_b200 import binding as vb
from tests.test_gpu_token_loss import BF16, F32, logits_of, tokens_of

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("vocab", [6, 1001, 32001])
@pytest.mark.parametrize("rows", [2, 600])
@pytest.mark.parametrize("off", [0, 1, 5])
def test_nothing_beside_the_rows_is_written(dtype, vocab, rows, off):
    """The elements before the first row, between the rows and behind the last keep their bits, at every alignment, near 0 and far."""
    pad = 7
    x = logits_of(rows, vocab, dtype, 0, 2, seed=1)
    x[1::2] = torch.finfo(dtype).min
    tokens = tokens_of(rows, vocab)
    op = vb.TokenLoss(rows, vocab, dtype)
    r = op.fwd(x, tokens)
    store = torch.full((off + rows * (vocab + pad) + 64,), 7.0, dtype=dtype, device="cuda")
    inside = torch.zeros(store.shape, dtype=torch.bool, device="cuda")
    view = lambda t: t[off:off + rows * (vocab + pad)].view(rows, vocab + pad)[:, :vocab]
    view(inside).fill_(True)
    norms = torch.full((rows + 2,), 7.0, device="cuda")
    d, _ = op.bwd(x, tokens, r.lse, torch.ones(rows, device="cuda"), dlogits=view(store), a_out=norms[1:-1])
    assert (store[~inside] == 7.0).all() and norms[0] == 7.0 and norms[-1] == 7.0
    assert torch.equal(d, op.bwd(x, tokens, r.lse, torch.ones(rows, device="cuda"))[0]) and not (d == 7.0).any()
