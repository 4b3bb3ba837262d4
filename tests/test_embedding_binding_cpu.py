"""Which tensors the binding's embedding calls take (CPU: shapes and types are
looked at before the device)."""
import pytest
import torch

from paper_2509_03047_amd import flashrestore as F


class NoGpu:
    """What lookups and gradients ask of an embedding before they reach the library."""
    info = dict(cols=16, rows=20, arena_bytes=640, grad_arena_bytes=640)
    handle = None


def refusal(ids, rows):
    said = set()
    for call in (lambda: F.fr_embed_lookup(NoGpu, torch.zeros(640, dtype=torch.uint8), ids, rows),
                 lambda: F.fr_embed_grad(NoGpu, ids, rows, torch.zeros(640, dtype=torch.uint8))):
        with pytest.raises(ValueError) as e:
            call()
        said.add(str(e.value).split(": ")[1].split(" ")[0])
    assert len(said) == 1
    return said.pop()


@pytest.mark.parametrize("ids,rows", [
    ((6,), (6, 16)), ((2, 3), (2, 3, 16)), ((2, 3), (6, 16)), ((), (16,)), ((), (1, 16)), ((1,), (1, 16)),
    ((0,), (0, 16)), ((0, 3), (0, 3, 16)), ((4, 1, 2), (4, 1, 2, 16)), ((4, 1, 2), (8, 16))])
def test_shapes_that_fit(ids, rows):
    """The ids' shape and the columns, or all rows behind one another: only the device is missing."""
    assert refusal(torch.zeros(ids, dtype=torch.int64), torch.zeros(rows)) == "not"


@pytest.mark.parametrize("ids,rows", [
    ((2, 3), (3, 2, 16)), ((6,), (2, 3, 16)), ((2, 3), (1, 6, 16)), ((2, 3), (2, 3, 1, 16)), ((1,), (16,)), ((), (2, 8)),
    ((), (1, 1, 16)), ((6,), (6, 15)), ((6,), (5, 16)), ((2, 8), (16, 16, 1)), ((16,), (16,)), ((0, 3), (3, 0, 16))])
def test_shapes_that_do_not(ids, rows):
    """The same number of elements in another shape is another call's tensor."""
    assert refusal(torch.zeros(ids, dtype=torch.int64), torch.zeros(rows)) == "shape"


@pytest.mark.parametrize("dtype", [torch.float16, torch.float64, torch.int32])
def test_types(dtype):
    assert refusal(torch.zeros(6, dtype=torch.int64), torch.zeros(6, 16, dtype=dtype)).startswith("torch.")


@pytest.mark.parametrize("field,value", [("entry", 1 << 32), ("entry", -(1 << 31) - 1), ("first", 1 << 63),
                                         ("first", -(1 << 63) - 1), ("rows", 1 << 32), ("max_tokens", -1)])
def test_numbers_that_do_not_fit_their_fields(field, value):
    """They would reach the library as others: entry 2^32 as entry 0."""
    args = dict(entry=0, rows=20, cols=16, max_tokens=0)
    args[field] = value
    with pytest.raises(ValueError, match=field):
        F.fr_embed_query(F.as_table([(0, 0, 320, F.FR_BF16, -1)]), 640, **args)
