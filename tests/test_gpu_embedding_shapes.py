"""Embedding calls of one token without a dimension, of batches and of their flat
rows, also further apart than their columns."""
import pytest
import torch

pytestmark = pytest.mark.gpu

from tests.test_gpu_embedding import Emb  # noqa: E402


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


@pytest.mark.parametrize("ids_shape,rows_shape", [((), (24,)), ((), (1, 24)), ((1,), (1, 24)), ((2, 3), (2, 3, 24)),
                                                  ((2, 3), (6, 24)), ((4, 1, 2), (4, 1, 2, 24))])
@pytest.mark.parametrize("padded", [False, True])
def test_shapes(ids_shape, rows_shape, padded):
    e = Emb(9, 24, grad="f32", tokens=8)
    gen = torch.Generator().manual_seed(3)
    ids = torch.randint(0, 9, ids_shape, generator=gen)
    wide = torch.full((*rows_shape[:-1], 24 + 5 * padded), 7.0, device="cuda")
    out = wide[..., :24]
    e.e.lookup(e.state, ids.cuda(), out)
    torch.cuda.synchronize()
    assert torch.equal(out.cpu().reshape(-1, 24), e.w.float()[ids.reshape(-1)])
    assert bool((wide[..., 24:] == 7.0).all())
    x = torch.randint(-8, 9, rows_shape, generator=gen).float()  # sums are exact in any order
    out.copy_(x)
    e.e.grad(ids.cuda(), out, e.grads)
    torch.cuda.synchronize()
    want = torch.zeros(9, 24).index_add_(0, ids.reshape(-1), x.reshape(-1, 24))
    assert torch.equal(e.grad().cpu(), want) and e.around()
