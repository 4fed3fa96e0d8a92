"""Arguments of the operators around a decoder of the caller's own that the other tests leave at their defaults, and what a call leaves alone."""
import math

import pytest
import torch

import paper_2407_09722_b200 as M
from tests.test_gpu_ops import Cache, attention_ref, check_attention, half_step, queries, seen_by

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("scale", [0.3, 1e-3, -0.25, -1.0])
@pytest.mark.parametrize("rows,hq,most", [(1, 4, 700), (3, 16, 700), (5, 24, 700), (1, 4, 5000), (5, 24, 5000)])
@pytest.mark.parametrize("window,sinks", [(0, 0), (100, 3)])
def test_attention_scale(scale, rows, hq, most, window, sinks):
    """Any finite scale but 0, which stands for 1 / sqrt(head_dim): the sign is the caller's.  (A negative one is the positive one on
    queries of the other sign, which the reference and its bound are taken from.)"""
    c = Cache(15, [most, 64, 130], 2, 64, 16)
    q = queries(15, 3, rows, hq, 64, torch.bfloat16)
    if scale > 0:
        check_attention(c, q, scale=scale, window=window, sinks=sinks)
        return
    ref, lse_ref, _, tol, tol_s = attention_ref(c, -q, [rows] * 3, window, sinks, -scale)
    out, lse = M.paged_attention(q, *c.args(), c.lens, window=window, sinks=sinks, scale=scale, max_len=most, return_lse=True)
    assert bool(((out.double() - ref).abs() <= half_step(q.dtype) * ref.abs() + tol + torch.finfo(q.dtype).smallest_normal).all())
    assert bool(((lse.double() - lse_ref).abs() <= tol_s + 2.0 ** -21 * lse_ref.abs()).all())


@pytest.mark.parametrize("rows,hq,most", [(4, 2, 300), (4, 8, 300), (4, 20, 300), (4, 2, 5000), (4, 20, 5000), (4, 80, 300)])
@pytest.mark.parametrize("window,sinks", [(0, 0), (50, 2)])
@pytest.mark.parametrize("bad", [0, 3])
def test_attention_weights_of_slots_that_a_row_with_nan_does_not_see(rows, hq, most, window, sinks, bad):
    """A row that sees a NaN spoils the weights of the slots that it sees and of no others: those behind it, or before its window, have what
    the other rows give, or are left alone."""
    n = 200
    c = Cache(16, [n, 130], 2, 64, 16)
    q = queries(16, 2, rows, hq, 64, torch.bfloat16)
    see = torch.stack([seen_by(n, n - rows + r, window, sinks) for r in range(rows)])
    lost, seen = see[bad], see.any(0)
    _, _, ref, _, tol_s = attention_ref(c, q, [rows] * 2, window, sinks, 0.125)
    q[0, bad, :, 3] = float("nan")
    w0 = torch.rand(2, 2, most, device="cuda")
    w = w0.clone()
    _, lse = M.paged_attention(q, *c.args(), c.lens, window=window, sinks=sinks, weights=w, max_len=most, return_lse=True)
    assert torch.equal(torch.isnan(lse[0]).all(-1), torch.arange(rows, device="cuda") == bad)
    assert bool(torch.isnan(w[0, :, :n][:, lost]).all())
    d = (w.double() - w0.double())[..., :n]
    near = (d - ref).abs() <= ref * (2 * float(tol_s.max()) + 2.0 ** -18) + 2.0 ** -23 * (1 + rows * hq)
    assert bool(near[0][:, ~lost].all()) and bool(near[1].all())
    assert torch.equal(w[0, :, :n][:, ~seen], w0[0, :, :n][:, ~seen]) and torch.equal(w[..., n:], w0[..., n:])
