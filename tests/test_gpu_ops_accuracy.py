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


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("group", [1, 16, 20, 40])
def test_attention_sums_over_long_shares_are_rounded(dtype, group):
    """Values of 1 for 1024 slots, of -1 for the next 1024 with the same scores, sixteen times over: the output is nothing but errors.  The
    shares of a head go up to P, the sum of 1024 probabilities, and back; rounded to the nearest in tiles of 16 slots that is 128 errors a period, each
    within half a step of at most P 2^-23: a standard deviation of sqrt(16 * 128 / 12) 2^-23 P, of a total of 32 P; six of them are 2^-21.7.  (Pieces
    that end inside a period, and references that rise, add 2^-26.)  Sums that are cut off at every product came to 2^-19.5."""
    dt = DT[dtype]
    B, hkv, n, hd = 64, 4, 32768, 64
    g = torch.Generator(device="cuda").manual_seed(2)
    k, v = (torch.zeros(1, n, hkv, hd, dtype=dt, device="cuda") for _ in range(2))
    half = torch.randn(n // 2048, 1, 1024, hkv, device="cuda", generator=g).to(dt)
    k[0, :, :, 9] = half.expand(-1, 2, -1, -1).reshape(n, hkv)
    v[0] = torch.tensor([1.0, -1.0], device="cuda").to(dt).repeat_interleave(1024).repeat(n // 2048)[:, None, None]
    q = torch.zeros(B, 1, hkv * group, hd, dtype=dt, device="cuda")
    q[..., 9] = 1
    kp, vp, table = small_cache(k, v, 64, 0)
    out = M.paged_attention(q, kp, vp, table.expand(B, -1).contiguous(), torch.full((B,), n, dtype=torch.int32, device="cuda"), scale=1.0)
    assert float(out.double().abs().max()) <= 2.0 ** -21, math.log2(float(out.double().abs().max()))


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("group", [1, 16, 20, 40])
@pytest.mark.parametrize("n,most", [(700, 700), (30000, 30000)])
def test_attention_many_slots_far_below_one(dtype, group, n, most):
    """The first slot has a score 17.5 above all others (what an attention sink looks like) and the value 0; the others' probabilities, 2^-25.2 each,
    make the output.  Their exponent 25.2 is off by two roundings (2^-24 of it each, 2^-18.9 of a probability); exponentials and sums of n
    terms of one size, in chains of at most n / 16 with the lanes' and tiles' in between, by 2^-16 with room; in fp16 a probability is a multiple of
    2^-37 of the largest, off by half of that: 2^-12.8 of 2^-25.2.  The output is then rounded once."""
    dt = DT[dtype]
    hd = 64
    k, v = torch.zeros(1, n, 1, hd, dtype=dt, device="cuda"), torch.ones(1, n, 1, hd, dtype=dt, device="cuda")
    k[:, 0, 0, 3], v[:, 0] = 1, 0
    v[:, :, 0, 1::2] *= -0.5
    q = torch.zeros(1, 1, group, hd, dtype=dt, device="cuda")
    q[..., 3] = 17.5
    kp, vp, table = small_cache(k, v, 16, 0)
    out, lse = M.paged_attention(q, kp, vp, table, torch.full((1,), n, dtype=torch.int32, device="cuda"), scale=1.0, max_len=most, return_lse=True)
    p = math.exp(-17.5)
    want = torch.tensor([1.0, -0.5], dtype=torch.float64, device="cuda").repeat(hd // 2) * ((n - 1) * p / (1 + (n - 1) * p))
    near = 2.0 ** -18.9 + 2.0 ** -16 + (2.0 ** -38 / p if dtype == "fp16" else 0.0)
    assert bool(((out.double() - want).abs() <= (half_step(dt) + near) * want.abs() + torch.finfo(dt).smallest_normal * torch.finfo(dt).eps).all())
    assert bool(((lse.double() - 17.5 - math.log1p((n - 1) * p)).abs() <= 17.5 * 2.0 ** -22 + 2.0 ** -20).all())


@pytest.mark.parametrize("rows,group", [(3, 2), (3, 4), (9, 2), (9, 4)])
@pytest.mark.parametrize("most", [64, 4096])
def test_attention_fp16_values_added_by_hand(rows, group, most):
    """An infinite value that only the last row sees: that value's row is added outside the products.  Every other output is what it
    was, but for the order of fp32 sums (2^-20 of the largest value with room) and a rounding each."""
    g = torch.Generator(device="cuda").manual_seed(3)
    k, v = (torch.empty(2, 50, 2, 64, dtype=torch.float16, device="cuda").normal_(generator=g) for _ in range(2))
    q = torch.empty(2, rows, 2 * group, 64, dtype=torch.float16, device="cuda").normal_(generator=g)
    lens = torch.full((2,), 50, dtype=torch.int32, device="cuda")
    kp, vp, table = small_cache(k, v, 16, most // 16)
    want = M.paged_attention(q, kp, vp, table, lens, max_len=most).double()
    v[1, 49, :, 7] = float("inf")
    kp, vp, table = small_cache(k, v, 16, most // 16)
    got = M.paged_attention(q, kp, vp, table, lens, max_len=most).double()
    assert bool((got[1, rows - 1, :, 7] == float("inf")).all())
    got[1, rows - 1, :, 7] = want[1, rows - 1, :, 7]
    assert bool(((got - want).abs() <= 2 * half_step(torch.float16) * want.abs() + 2.0 ** -20 * float(v[v.isfinite()].abs().max())).all())


# ---------------------------------------------------------------------------------------------------------------
# accept rules.  A log-probability is the difference of a logit and the row's largest (one rounding, 2^-24 of it) less the logarithm of a
# sum: its terms are off by 2^-20.5 (an exponent up to 32 in fp32, the exponential), the sum of at most 2^7 in a chain by 2^-19 at the very
# worst and by 2^-21 as terms round, the logarithm by 2^-22.  2^-19 and 2^-22 of the value hold all of it.

def lp_bound(lp):
    return 2.0 ** -19 + 2.0 ** -22 * lp.abs()


def accept_both(z, dr, tok, u, ua, temperature=1.0):
    B, D = tok.shape
    got = []
    for rule in ("mtad", "spd"):
        res = M.ResultBuffers(B, D, D)
        if rule == "spd":
            M.accept_chain_spd(z, tok, dr, ua, u, res, temperature=temperature, draft_temperature=temperature)
        else:
            logq = torch.log_softmax(dr.double() / temperature, -1).gather(2, tok.long()[..., None])[..., 0].cumsum(-1).float()
            M.accept_chain(z, tok, logq, math.log(0.2), u, res, temperature=temperature)
        assert not res.status.any()
        got.append({n: getattr(res, n).clone() for n in ("eta", "n_out", "out_tok", "out_lp", "node_lp", "row_lse")})
    return got


def check_accept_lp(z, tok, got, temperature=1.0, far=0.0):
    B, D = tok.shape
    lse = torch.logsumexp(z.double() / temperature, -1)
    lp = z.double() / temperature - lse[..., None]
    want = lp[:, :D].gather(2, tok.long()[..., None])[..., 0]
    b = torch.arange(B, device="cuda")
    for r in got:
        assert bool(((r["node_lp"].double() - want).abs() <= lp_bound(want) + far).all()), float((r["node_lp"].double() - want).abs().max())
        assert bool(((r["row_lse"].double() - lse).abs() <= 2.0 ** -24 * lse.abs() + 2.0 ** -19 + far).all()), float((r["row_lse"].double() - lse).abs().max())
        last = lp[b, r["eta"].long(), r["out_tok"][b, r["eta"].long()].long()]
        assert bool(((r["out_lp"][b, r["eta"].long()].double() - last).abs() <= lp_bound(last) + far).all())


def accept_inputs(seed, B, D, V, step, top):
    """Target rows that are multiples of `step` below `top` in magnitude, the auxiliary model's near them."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    z = ((torch.randn(B, D + 1, V, device="cuda", generator=g) * 2).clamp_(-top, top) / step).round() * step
    dr = ((z[:, :D] + torch.randn(B, D, V, device="cuda", generator=g)).clamp_(-top, top) / step).round() * step
    tok = torch.randint(0, V, (B, D), device="cuda", generator=g, dtype=torch.int32)
    tok[:, 0] = z[:, 0].argmax(-1).int()
    u, ua = (torch.rand(*d, device="cuda", generator=g).clamp_(2.0 ** -24, 1 - 2.0 ** -24) for d in ((B, V), (B, D)))
    return z, dr, tok, u, ua


@pytest.mark.parametrize("dtype,step,top,constant", [("fp32", 2.0 ** -10, 8, 8192 - 16), ("fp32", 2.0 ** -10, 8, -8192 + 16), ("bf16", 1.0, 8, 192), ("fp16", 0.5, 8, -960),
                                                     ("fp32", 2.0 ** -2, 8, 3000000.0)])
@pytest.mark.parametrize("temperature", [1.0, 0.6875])
def test_accept_rows_with_a_constant_added(dtype, step, top, constant, temperature):
    """Any constant may have been added to a row (here one that leaves every logit exact): log-probabilities, decisions and draws are
    those of the row without it, to the same bound, and only the log-sum-exp moves."""
    z, dr, tok, u, ua = accept_inputs(3, 6, 4, 1500, step, top)
    z, dr, far = z.to(DT[dtype]), dr.to(DT[dtype]), (z + constant).to(DT[dtype])
    assert torch.equal(far.double() - constant, z.double()) and torch.equal((dr.float() - constant).to(DT[dtype]).double() + constant, dr.double())
    here = accept_both(z, dr, tok, u, ua, temperature)
    there = accept_both(far, (dr.float() - constant).to(DT[dtype]), tok, u, ua, temperature)
    check_accept_lp(z, tok, here, temperature)
    check_accept_lp(far, tok, there, temperature)
    for a, b in zip(here, there):
        for n in ("eta", "n_out", "out_tok"):
            assert torch.equal(a[n], b[n])


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
def test_accept_peaks_far_above_the_first_tokens(dtype):
    """Two tokens hold nearly all of a row, some 60 above the ones that begin it.  Their exponents, 64 to 128 over the first tokens', are multiples of
    2^-17, off by half of that: 2^-18 ln 2 of each term, 2^-17.5 of both."""
    z, dr, tok, u, ua = accept_inputs(4, 40, 3, 5000, 2.0 ** -6, 8)
    g = torch.Generator(device="cuda").manual_seed(5)
    at = torch.randint(2000, 5000, (40, 4, 2), device="cuda", generator=g)
    at[..., 1] = (at[..., 0] + 1 - 2000) % 3000 + 2000
    z.scatter_(2, at, 60 + torch.rand(40, 4, 2, device="cuda", generator=g))
    z = z.to(DT[dtype])
    tok = at[:, :3, 0].int().contiguous()
    check_accept_lp(z, tok, accept_both(z, dr.to(DT[dtype]), tok, u, ua), far=2.0 ** -17.5)
