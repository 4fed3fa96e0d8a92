"""Layouts that the operators around a decoder of the caller's own cannot use, refused on the host."""
import pytest
import torch

import paper_2407_09722_b200 as M


@pytest.fixture(scope="module", autouse=True)
def lib():
    from paper_2407_09722_b200.build import build
    build()
    return M.load_library()


def _calls(k, table, lens, b):
    """Each operator that takes a table, on tensors that are right but for it."""
    q = torch.zeros(b, 1, 4, 64, dtype=torch.bfloat16)
    kv = torch.zeros(b, 1, 2, 64, dtype=torch.bfloat16)
    return [lambda: M.paged_attention(q, k, k, table, lens), lambda: M.paged_append(q, kv, kv, k, k, table, lens),
            lambda: M.paged_evict(k, k, table, lens, torch.zeros(b, 2, 64), 8)]


@pytest.mark.parametrize("kind", ["expanded", "overlapping"])
def test_table_rows_that_do_not_lie_apart_are_refused(kind):
    """A row of a table begins where its stride says: rows closer together than they are long are not read at made-up places."""
    k = torch.zeros(4, 2, 16, 64, dtype=torch.bfloat16)
    one = torch.zeros(16, dtype=torch.int32)
    table = one[:4][None].expand(3, 4) if kind == "expanded" else one.as_strided((3, 4), (2, 1))
    for call in _calls(k, table, torch.zeros(3, dtype=torch.int32), 3):
        with pytest.raises(ValueError, match="table: rows"):
            call()


@pytest.mark.parametrize("table", [torch.zeros(3, 4, dtype=torch.int32), torch.zeros(3, 9, dtype=torch.int32)[:, 2:6], torch.zeros(4, dtype=torch.int32)[None],
                                   torch.zeros(4, dtype=torch.int32).as_strided((1, 4), (1, 1))])
def test_table_rows_that_lie_apart_are_taken(table):
    """... wide or narrow, and the stride of a single row does not matter (the calls end at the tensors' device, the check behind it)."""
    k, b = torch.zeros(4, 2, 16, 64, dtype=torch.bfloat16), table.shape[0]
    for call in _calls(k, table, torch.zeros(b, dtype=torch.int32), b):
        with pytest.raises(ValueError, match="CUDA tensors only"):
            call()
