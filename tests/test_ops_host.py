"""The operators around a decoder of the caller's own: argument checks that need no GPU."""
import ctypes as C
import math

import pytest
import torch

import paper_2407_09722_b200 as M
from paper_2407_09722_b200 import binding as Bn


@pytest.fixture(scope="module")
def lib():
    from paper_2407_09722_b200.build import build
    build()
    return M.load_library()


def _kv(**kw):
    d = dict(k_pages=4096, v_pages=8192, table=256, page_stride=2 * 8 * 16 * 128, head_stride=16 * 128, slot_stride=128, table_stride=64,
             dtype=0, n_pages=100, page_size=16, n_kv_heads=8, head_dim=128, max_pages=64)
    d.update(kw)
    return Bn.PagedKV(**d)


BAD_KV = [(dict(k_pages=None), Bn.MTAD_E_INVALID), (dict(v_pages=8194), Bn.MTAD_E_INVALID), (dict(table=None), Bn.MTAD_E_INVALID),
          (dict(dtype=2), Bn.MTAD_E_INVALID), (dict(dtype=-1), Bn.MTAD_E_INVALID), (dict(n_pages=0), Bn.MTAD_E_INVALID),
          (dict(page_size=0), Bn.MTAD_E_INVALID), (dict(head_dim=12), Bn.MTAD_E_INVALID), (dict(head_dim=264), Bn.MTAD_E_INVALID),
          (dict(head_dim=0), Bn.MTAD_E_INVALID), (dict(slot_stride=120), Bn.MTAD_E_INVALID), (dict(slot_stride=132), Bn.MTAD_E_INVALID),
          (dict(page_stride=-8), Bn.MTAD_E_INVALID), (dict(table_stride=63), Bn.MTAD_E_INVALID), (dict(max_pages=0), Bn.MTAD_E_INVALID),
          (dict(n_kv_heads=1025), Bn.MTAD_E_CAPACITY), (dict(page_size=1 << 26), Bn.MTAD_E_CAPACITY)]


def _attn(**kw):
    d = dict(lens=256, q=4096, out=8192, q_stride_seq=64 * 128, q_stride_row=64 * 128, q_stride_head=128, out_stride_seq=64 * 128,
             out_stride_row=64 * 128, out_stride_head=128, batch=2, rows=1, n_q_heads=64, max_len=1000, scale=0.0)
    d.update(kw)
    return Bn.PagedAttn(**d)


def _rows(**kw):
    d = dict(lens=256, q=4096, k=8192, v=8192, q_out=4096, q_stride_seq=8192, q_stride_row=8192, q_stride_head=128, kv_stride_seq=1024,
             kv_stride_row=1024, kv_stride_head=128, out_stride_seq=8192, out_stride_row=8192, out_stride_head=128, dtype=0, batch=2, rows=1,
             n_q_heads=64, rope_base=10000.0)
    d.update(kw)
    return Bn.PagedRows(**d)


def _evict(**kw):
    d = dict(lens=256, scores=4096, kept=8192, new_lens=512, scores_stride_seq=8000, scores_stride_head=1000, batch=2, max_len=1000, keep=100,
             first=4, recent=10)
    d.update(kw)
    return Bn.PagedEviction(**d)


@pytest.mark.parametrize("kw,code", BAD_KV)
def test_bad_pages_are_refused_everywhere(lib, kw, code):
    n = C.c_size_t(0)
    assert lib.mtad_paged_attention_workspace(_kv(**kw), _attn(), C.byref(n)) == code
    assert lib.mtad_paged_attention(_kv(**kw), _attn(), None, 0, None) == code
    assert lib.mtad_paged_append(_kv(**kw), _rows(), None) == code
    assert lib.mtad_paged_evict(_kv(**kw), _evict(), None) == code


@pytest.mark.parametrize("kw,code", [
    (dict(lens=None), Bn.MTAD_E_INVALID), (dict(q=None), Bn.MTAD_E_INVALID), (dict(out=8193), Bn.MTAD_E_INVALID),
    (dict(batch=0), Bn.MTAD_E_INVALID), (dict(batch=4097), Bn.MTAD_E_CAPACITY), (dict(rows=0), Bn.MTAD_E_INVALID),
    (dict(rows=257), Bn.MTAD_E_CAPACITY), (dict(n_q_heads=63), Bn.MTAD_E_INVALID), (dict(n_q_heads=0), Bn.MTAD_E_INVALID),
    (dict(window=-1), Bn.MTAD_E_INVALID), (dict(sinks=-1), Bn.MTAD_E_INVALID), (dict(max_len=0), Bn.MTAD_E_INVALID),
    (dict(scale=math.nan), Bn.MTAD_E_INVALID), (dict(scale=math.inf), Bn.MTAD_E_INVALID),
    (dict(q_stride_head=4), Bn.MTAD_E_INVALID), (dict(out_stride_row=-8), Bn.MTAD_E_INVALID), (dict(weights=256, weights_stride_head=-1), Bn.MTAD_E_INVALID)])
def test_attention_refusals(lib, kw, code):
    n = C.c_size_t(0)
    assert lib.mtad_paged_attention_workspace(_kv(), _attn(**kw), C.byref(n)) == code
    assert lib.mtad_paged_attention(_kv(), _attn(**kw), None, 0, None) == code


def test_attention_workspace(lib):
    n = C.c_size_t(0)
    kv = _kv(max_pages=4096, table_stride=4096)
    assert lib.mtad_paged_attention_workspace(kv, _attn(), None) == Bn.MTAD_E_INVALID
    assert lib.mtad_paged_attention_workspace(kv, None, C.byref(n)) == Bn.MTAD_E_INVALID
    assert lib.mtad_paged_attention_workspace(kv, _attn(max_len=60000), C.byref(n)) == 0
    need = n.value
    assert need > 0 and need % 256 == 0
    for ws, size in ((None, need), (4096, need - 1), (4100, need)):
        assert lib.mtad_paged_attention(kv, _attn(max_len=60000), ws, size, None) == Bn.MTAD_E_WORKSPACE
    more = dict(max_len=60000, weights=256, weights_stride_seq=480000, weights_stride_head=60000)
    assert lib.mtad_paged_attention_workspace(kv, _attn(**more), C.byref(n)) == 0
    assert n.value > need
    assert lib.mtad_paged_attention_workspace(kv, _attn(max_len=200), C.byref(n)) == 0 and n.value == 0         # a cluster has a head
    # an hour of tiles more than a launch can count
    big = _kv(page_size=1 << 20, max_pages=1000, table_stride=1000)
    assert lib.mtad_paged_attention_workspace(big, _attn(max_len=1000 << 20, batch=4096), C.byref(n)) == Bn.MTAD_E_CAPACITY


@pytest.mark.parametrize("kw,code", [
    (dict(lens=None), Bn.MTAD_E_INVALID), (dict(k=None), Bn.MTAD_E_INVALID), (dict(v=8200), Bn.MTAD_E_INVALID), (dict(q=None), Bn.MTAD_E_INVALID),
    (dict(q_out=None), Bn.MTAD_E_INVALID), (dict(dtype=1), Bn.MTAD_E_INVALID), (dict(dtype=7), Bn.MTAD_E_INVALID), (dict(rope_base=0.5), Bn.MTAD_E_INVALID),
    (dict(rope_base=-1.0), Bn.MTAD_E_INVALID), (dict(rope_base=math.nan), Bn.MTAD_E_INVALID), (dict(rows=257), Bn.MTAD_E_CAPACITY),
    (dict(kv_stride_row=4), Bn.MTAD_E_INVALID), (dict(dtype=2, kv_stride_row=2), Bn.MTAD_E_INVALID), (dict(out_stride_head=4), Bn.MTAD_E_INVALID),
    (dict(n_q_heads=-1), Bn.MTAD_E_INVALID), (dict(batch=5000), Bn.MTAD_E_CAPACITY)])
def test_append_refusals(lib, kw, code):
    assert lib.mtad_paged_append(_kv(), _rows(**kw), None) == code


@pytest.mark.parametrize("kw,code", [
    (dict(lens=None), Bn.MTAD_E_INVALID), (dict(scores=None), Bn.MTAD_E_INVALID), (dict(kept=None), Bn.MTAD_E_INVALID), (dict(new_lens=None), Bn.MTAD_E_INVALID),
    (dict(new_lens=256), Bn.MTAD_E_INVALID), (dict(keep=0), Bn.MTAD_E_INVALID), (dict(keep=13), Bn.MTAD_E_INVALID), (dict(first=-1), Bn.MTAD_E_INVALID),
    (dict(recent=-1), Bn.MTAD_E_INVALID), (dict(max_len=0), Bn.MTAD_E_INVALID),
    (dict(keep=2 ** 31 - 1, first=2 ** 31 - 1, recent=2 ** 31 - 1), Bn.MTAD_E_INVALID), (dict(batch=0), Bn.MTAD_E_INVALID)])
def test_evict_refusals(lib, kw, code):
    assert lib.mtad_paged_evict(_kv(), _evict(**kw), None) == code


def test_a_bound_beyond_the_table_is_the_table(lib):
    n, m = C.c_size_t(0), C.c_size_t(0)
    assert lib.mtad_paged_attention_workspace(_kv(), _attn(max_len=1 << 30), C.byref(n)) == 0
    assert lib.mtad_paged_attention_workspace(_kv(), _attn(max_len=1024), C.byref(m)) == 0 and n.value == m.value


def test_evict_scores_in_place_only_where_a_block_holds_them(lib):
    big = _kv(page_size=4096, max_pages=100, table_stride=100)
    assert lib.mtad_paged_evict(big, _evict(max_len=327681, scores_out=4096), None) == Bn.MTAD_E_UNIMPLEMENTED


def _accept(**kw):
    d = dict(logits=4096, logits_stride_seq=5000, logits_stride_row=1000, draft_stride_seq=4000, draft_stride_row=1000, draft_tok=256,
             last_uniform=512, dtype=2, batch=2, gamma=4, vocab=1000, temperature=1.0, draft_temperature=1.0)
    d.update(kw)
    return Bn.AcceptRows(**d)


def _result(**kw):
    d = {n: 256 for n, _ in Bn.Result._fields_}
    d.update(kw)
    return Bn.Result(**d)


@pytest.mark.parametrize("kw,code", [
    (dict(logits=None), Bn.MTAD_E_INVALID), (dict(logits=4098), Bn.MTAD_E_INVALID), (dict(draft_tok=None), Bn.MTAD_E_INVALID), (dict(last_uniform=None), Bn.MTAD_E_INVALID),
    (dict(dtype=3), Bn.MTAD_E_INVALID), (dict(batch=0), Bn.MTAD_E_INVALID), (dict(batch=4097), Bn.MTAD_E_CAPACITY), (dict(gamma=-1), Bn.MTAD_E_INVALID),
    (dict(gamma=33), Bn.MTAD_E_CAPACITY), (dict(vocab=0), Bn.MTAD_E_INVALID), (dict(temperature=0.0), Bn.MTAD_E_INVALID), (dict(temperature=math.nan), Bn.MTAD_E_INVALID),
    (dict(temperature=math.inf), Bn.MTAD_E_INVALID), (dict(logits_stride_row=-1), Bn.MTAD_E_INVALID)])
def test_accept_refusals(lib, kw, code):
    r = _result()
    assert lib.mtad_accept_chain(_accept(**kw), 256, -1.0, C.byref(r), None) == code
    assert lib.mtad_accept_chain_spd(_accept(**kw), 256, 256, C.byref(r), None) == code


def test_accept_refuses_missing_arrays_and_taus(lib):
    r = _result()
    for tau in (0.0, 0.5, math.nan):
        assert lib.mtad_accept_chain(_accept(), 256, tau, C.byref(r), None) == Bn.MTAD_E_INVALID
    assert lib.mtad_accept_chain(_accept(), None, -1.0, C.byref(r), None) == Bn.MTAD_E_INVALID
    assert lib.mtad_accept_chain(None, 256, -1.0, C.byref(r), None) == Bn.MTAD_E_INVALID
    assert lib.mtad_accept_chain(_accept(), 256, -1.0, None, None) == Bn.MTAD_E_INVALID
    assert lib.mtad_accept_chain_spd(_accept(), None, 256, C.byref(r), None) == Bn.MTAD_E_INVALID
    assert lib.mtad_accept_chain_spd(_accept(), 256, None, C.byref(r), None) == Bn.MTAD_E_INVALID
    assert lib.mtad_accept_chain_spd(_accept(gamma=0), 256, 256, C.byref(r), None) == Bn.MTAD_E_INVALID
    assert lib.mtad_accept_chain_spd(_accept(draft_temperature=0.0), 256, 256, C.byref(r), None) == Bn.MTAD_E_INVALID
    for n in ("eta", "winner", "path", "n_out", "out_tok", "out_lp", "status"):
        assert lib.mtad_accept_chain(_accept(), 256, -1.0, C.byref(_result(**{n: None})), None) == Bn.MTAD_E_INVALID
    assert lib.mtad_ops_cuda_error() == 0


def test_the_python_side_refuses_before_it_calls(lib):
    k = torch.zeros(4, 2, 16, 64, dtype=torch.bfloat16)
    table, lens = torch.zeros(1, 4, dtype=torch.int32), torch.zeros(1, dtype=torch.int32)
    q = torch.zeros(1, 1, 4, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        M.paged_attention(q, k, k, table, lens)                           # no CUDA tensors: there is no CPU form
    with pytest.raises(ValueError):
        M.paged_attention(q, k, k.transpose(1, 2), table, lens)
    with pytest.raises(ValueError):
        M.paged_attention(q, k, k, table.long(), lens)
    with pytest.raises(ValueError):
        M.paged_attention(q.float(), k, k, table, lens)
    with pytest.raises(ValueError):
        M.paged_attention(q[..., :32], k, k, table, lens)
    with pytest.raises(ValueError):
        M.paged_append(q, q, q, k, k, table, lens)                        # not the pages' heads
    with pytest.raises(ValueError):
        M.paged_evict(k, k, table, lens, torch.zeros(1, 3, 64), 8)
    with pytest.raises(ValueError):
        M.paged_evict(k, k, table, lens, torch.zeros(1, 2, 32), 8, max_len=64)
    with pytest.raises(ValueError):
        M.accept_chain(torch.zeros(1, 3, 8), None, None, -1.0, torch.zeros(1, 8), M.ResultBuffers(1, 2, 2, device="cpu"))
