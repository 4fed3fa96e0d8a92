"""Layouts that the operators around a decoder of the caller's own cannot use, refused on the host."""
import ctypes as C

import pytest
import torch

import paper_2407_09722_b200 as M
from paper_2407_09722_b200 import binding as Bn


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


# ---- arrays that a call writes: no element twice

def _kv(**kw):
    d = dict(k_pages=1 << 20, v_pages=2 << 20, table=256, page_stride=2 * 8 * 16 * 128, head_stride=16 * 128, slot_stride=128, table_stride=64,
             dtype=0, n_pages=100, page_size=16, n_kv_heads=8, head_dim=128, max_pages=64)
    d.update(kw)
    return Bn.PagedKV(**d)


def _attn(**kw):
    d = dict(lens=256, q=4096, out=8192, q_stride_seq=3 * 8192, q_stride_row=8192, q_stride_head=128, out_stride_seq=3 * 8192, out_stride_row=8192,
             out_stride_head=128, batch=2, rows=3, n_q_heads=64, max_len=1000)
    d.update(kw)
    return Bn.PagedAttn(**d)


def _rows(**kw):
    d = dict(lens=256, q=4096, k=8192, v=16384, q_out=4096, q_stride_seq=3 * 8192, q_stride_row=8192, q_stride_head=128, kv_stride_seq=3 * 1024,
             kv_stride_row=1024, kv_stride_head=128, out_stride_seq=3 * 8192, out_stride_row=8192, out_stride_head=128, batch=2, rows=3, n_q_heads=64)
    d.update(kw)
    return Bn.PagedRows(**d)


def _evict(**kw):
    d = dict(lens=256, scores=4096, kept=8192, new_lens=512, scores_out=16384, scores_stride_seq=8000, scores_stride_head=1000, out_stride_seq=800,
             out_stride_head=100, batch=2, max_len=1000, keep=100)
    d.update(kw)
    return Bn.PagedEviction(**d)


W = dict(weights=1024, weights_stride_seq=8000, weights_stride_head=1000)


@pytest.mark.parametrize("kw,code", [
    (dict(), 0), (W, 0), (dict(out_stride_seq=128, out_stride_head=256, out_stride_row=64 * 256), 0),          # [rows][heads][sequences]
    (dict(rows=1, out_stride_row=0), 0), (dict(batch=1, out_stride_seq=0), 0), ({**W, "batch": 1, "weights_stride_seq": 0}, 0),
    (dict(out_stride_seq=0), Bn.MTAD_E_INVALID), (dict(out_stride_row=0), Bn.MTAD_E_INVALID), (dict(out_stride_head=0), Bn.MTAD_E_INVALID),
    (dict(out_stride_head=120), Bn.MTAD_E_INVALID), (dict(out_stride_seq=2 * 8192), Bn.MTAD_E_INVALID),
    (dict(out_stride_seq=(1 << 62) + 8, out_stride_row=1 << 62, batch=3), Bn.MTAD_E_INVALID),
    ({**W, "weights_stride_seq": 0}, Bn.MTAD_E_INVALID), ({**W, "weights_stride_head": 0}, Bn.MTAD_E_INVALID),
    ({**W, "weights_stride_head": 999}, Bn.MTAD_E_INVALID), ({**W, "weights_stride_seq": 7999}, Bn.MTAD_E_INVALID)])
def test_attention_outputs_that_overlap_themselves(lib, kw, code):
    n = C.c_size_t(0)
    assert lib.mtad_paged_attention_workspace(_kv(), _attn(**kw), C.byref(n)) == code


PAGES = [dict(page_stride=0), dict(head_stride=0), dict(slot_stride=128, head_stride=128), dict(page_stride=16 * 128), dict(v_pages=1 << 20)]


@pytest.mark.parametrize("kw", PAGES)
def test_pages_that_overlap_are_read_but_not_written(lib, kw):
    """Attention may read an expanded view of the pages; rows are not stored into one, nor moved in it."""
    n = C.c_size_t(0)
    assert lib.mtad_paged_attention_workspace(_kv(**kw), _attn(), C.byref(n)) == 0
    assert lib.mtad_paged_append(_kv(**kw), _rows(), None) == Bn.MTAD_E_INVALID
    assert lib.mtad_paged_evict(_kv(**kw), _evict(), None) == Bn.MTAD_E_INVALID


@pytest.mark.parametrize("kw", [dict(out_stride_seq=0), dict(out_stride_row=0), dict(out_stride_head=0), dict(out_stride_row=8184)])
def test_append_queries_that_overlap_themselves(lib, kw):
    assert lib.mtad_paged_append(_kv(), _rows(**kw), None) == Bn.MTAD_E_INVALID


@pytest.mark.parametrize("kw", [dict(out_stride_seq=0), dict(out_stride_head=0), dict(out_stride_head=99), dict(out_stride_seq=799)])
def test_eviction_scores_that_overlap_themselves(lib, kw):
    assert lib.mtad_paged_evict(_kv(), _evict(**kw), None) == Bn.MTAD_E_INVALID


@pytest.mark.parametrize("sinks", [2 ** 31 - 1, 2 ** 31 - 63, 2 ** 31 - 64, 1024])
def test_as_many_sinks_as_there_are_slots_or_more(lib, sinks):
    """A window behind which every slot is a sink: the workspace of the whole cache."""
    n, m = C.c_size_t(0), C.c_size_t(0)
    call = dict(W, rows=40, out_stride_seq=40 * 8192, window=100, max_len=1000)
    assert lib.mtad_paged_attention_workspace(_kv(), _attn(**{**call, "window": 0}), C.byref(n)) == 0
    assert lib.mtad_paged_attention_workspace(_kv(), _attn(sinks=sinks, **call), C.byref(m)) == 0 and m.value == n.value


def test_strides_of_single_dimensions_may_differ_between_keys_and_values():
    """One row of one sequence, one page: whatever stands there as a stride is not stepped along (the calls end at the tensors' device)."""
    k = torch.zeros(1, 1, 2, 64, dtype=torch.bfloat16)
    v = k.as_strided(k.shape, (7, 9, 64, 1))
    kp = torch.zeros(1, 2, 16, 64, dtype=torch.bfloat16)
    vp = kp.as_strided(kp.shape, (11, 1024, 64, 1))
    table, lens = torch.zeros(1, 1, dtype=torch.int32), torch.zeros(1, dtype=torch.int32)
    q = torch.zeros(1, 1, 4, 64, dtype=torch.bfloat16)
    for call in (lambda: M.paged_append(q, k, v, kp, vp, table, lens), lambda: M.paged_attention(q, kp, vp, table, lens)):
        with pytest.raises(ValueError, match="CUDA tensors only"):
            call()
    with pytest.raises(ValueError, match="alike"):
        M.paged_attention(q, kp, kp.transpose(1, 2).contiguous().transpose(1, 2), table, lens)
    with pytest.raises(ValueError, match="like k"):
        M.paged_append(q, k, torch.zeros(1, 1, 2, 72, dtype=torch.bfloat16)[..., :64], kp, kp, table, lens)
