"""How exact the operators around a decoder of the caller's own are, on inputs that leave nothing else to round."""
import math

import pytest
import torch

import paper_2407_09722_b200 as M

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}


def half_step(dt):
    return torch.finfo(dt).eps / 2


def small_cache(k, v, page, width):
    """k, v [sequences, slots, kv heads, head_dim] as pages, one sequence after the other, in a table of `width` pages."""
    B, n, hkv, hd = k.shape
    per = -(-n // page)
    pages = torch.zeros(2, B * per, hkv, page, hd, dtype=k.dtype, device="cuda")
    for i, x in enumerate((k, v)):
        full = torch.zeros(B, per * page, hkv, hd, dtype=k.dtype, device="cuda")
        full[:, :n] = x
        pages[i] = full.view(B * per, page, hkv, hd).transpose(1, 2)
    table = torch.full((B, max(width, per)), -1, dtype=torch.int32, device="cuda")
    table[:, :per] = torch.arange(B * per, dtype=torch.int32, device="cuda").view(B, per)
    return pages[0], pages[1], table


# query heads a KV head, the bound of the lengths: every tile height, heads that a cluster has and heads of a list cut over the GPU
FORMS = [(g, most) for g in (1, 16, 20, 40) for most in (16, 4096)]


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("group,most", FORMS)
def test_attention_probabilities_keep_their_bits(dtype, group, most):
    """Three slots: probability 1, p = e^t, 1, values -h, 1, -l with h + l the first two terms of p in the cache's type, so that what is left
    of p after two terms is the output.  Scores are exact; the exponent t log2(e) is off by two roundings of a value below 1.45 (2^-23 of p
    together), the exponential by 2^-22, the sums of three terms by 2^-23 at most: 2^-21 of p in all, with the third term of bf16 (2^-27) to spare.
    Two terms of bf16 alone leave up to 2^-18."""
    dt = DT[dtype]
    t = -torch.arange(1, 513, device="cuda").double() / 512 if dtype == "bf16" else -torch.arange(1, 1025, device="cuda").double() / 1024
    t = t.to(dt).unique()
    B, hd = len(t), 64
    p = t.double().exp()
    h = p.to(dt)
    l = (p - h.double()).to(dt)
    k, v = torch.zeros(B, 3, 1, hd, dtype=dt, device="cuda"), torch.zeros(B, 3, 1, hd, dtype=dt, device="cuda")
    k[:, 1, 0, 5] = 1
    v[:, 0, 0], v[:, 1, 0], v[:, 2, 0] = -h[:, None], 1, -l[:, None]
    q = torch.zeros(B, 1, group, hd, dtype=dt, device="cuda")
    q[..., 5] = t[:, None, None]
    kp, vp, table = small_cache(k, v, 16, most // 16)
    out = M.paged_attention(q, kp, vp, table, torch.full((B,), 3, dtype=torch.int32, device="cuda"), scale=1.0, max_len=most)
    want = ((p - h.double() - l.double()) / (2 + p))[:, None, None, None]
    assert bool(((out.double() - want).abs() <= half_step(dt) * want.abs() + 2.0 ** -21 * (p / (2 + p))[:, None, None, None] +
                 torch.finfo(dt).smallest_normal * torch.finfo(dt).eps).all())
