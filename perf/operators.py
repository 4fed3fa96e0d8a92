"""The operators that a program with a decoder of its own calls around this library, as timed cases: the new rows' keys and
values enter a cache kept in pages (with the rotary embedding), the rows attend to it (all of it, or a sliding window and
the first tokens), drafted tokens are accepted from rows of logits, and a full cache gives up the tokens that drew the
least attention.

Every case runs in two forms: the library's entry points, or plain torch operations in 32 bits on the same inputs.  Shapes
are the workloads' of `mtad_synth`, or generic; all values depend on the seed alone.
"""
from __future__ import annotations

import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
ROPE_BASE = 10000.0


# ---------------------------------------------------------------------------------------------------------------
# cases

def _case(op, name, **more):
    c = {"op": op, **more}
    if name:
        c["name"] = name
    return c


def _attention(name, batch, rows, hq, hkv, hd, lo, hi, page, dtype="bf16", window=0, sinks=0, weights=False):
    return _case("attention", name, batch=batch, rows=rows, hq=hq, hkv=hkv, hd=hd, lo=lo, hi=hi, page=page, dtype=dtype,
                 window=window, sinks=sinks, weights=weights)


def _append(name, batch, rows, hq, hkv, hd, lo, hi, page, dtype="bf16", source="bf16"):
    return _case("append", name, batch=batch, rows=rows, hq=hq, hkv=hkv, hd=hd, lo=lo, hi=hi, page=page, dtype=dtype, source=source)


def _evict(name, batch, hkv, hd, lo, hi, page, keep, first, recent, dtype="bf16"):
    return _case("evict", name, batch=batch, hkv=hkv, hd=hd, lo=lo, hi=hi, page=page, keep=keep, first=first, recent=recent, dtype=dtype)


def _accept(name, rule, batch, gamma, vocab, dtype="bf16"):
    return _case("accept", name, rule=rule, batch=batch, gamma=gamma, vocab=vocab, dtype=dtype)


def listed():
    return [
        # the shortest call: one new token of one sequence that has just begun, nothing but latency
        _attention("attn_first_tokens", 1, 1, 32, 32, 128, 97, 97, 16),
        # the ordinary verification: a chain of four drafted tokens and the root against 2048 committed ones
        _attention("attn_chain_2k", 1, 5, 32, 32, 128, 2053, 2053, 16),
        # batched serving: eight ragged sequences, chains of six
        _attention("attn_batch_ragged", 8, 7, 40, 40, 128, 1031, 2999, 16),
        # long contexts with grouped heads, one new token each, weights kept for a later eviction
        _attention("attn_long_weights", 16, 1, 64, 8, 128, 8000, 32500, 64, weights=True),
        # an auxiliary model's heads in fp16, window of 512 and four sinks
        _attention("attn_window_small", 4, 1, 12, 12, 64, 333, 1999, 16, dtype="fp16", window=512, sinks=4),
        # many long conversations behind a window of 4096
        _attention("attn_window_long", 32, 1, 64, 8, 128, 9000, 65000, 64, window=4096, sinks=4),
        # the rows of one chain on their way into the cache, as they leave an fp32 projection
        _append("append_chain", 1, 5, 32, 32, 128, 2053, 2053, 16, source="fp32"),
        # chunks of sixteen prompts
        _append("append_prompts", 16, 256, 64, 8, 128, 300, 4000, 64),
        # one sequence of the 7B shape whose cache is halved
        _evict("evict_one", 1, 32, 128, 2113, 2113, 16, 1024, 4, 256),
        # long ragged contexts, some shorter than what is kept
        _evict("evict_long", 16, 8, 128, 6000, 32500, 64, 8192, 4, 1024),
        # the joint-likelihood rule on a chain of four, fp32 rows of a 32000-token vocabulary
        _accept("accept_chain", "mtad", 1, 4, 32000, dtype="fp32"),
        # the speculative-decoding rule on a serving batch with a large vocabulary
        _accept("accept_spd_batch", "spd", 64, 6, 128000),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["attention", "attention", "window", "append", "evict", "accept"])
    dtype = rng.choice(["bf16", "bf16", "fp16"])
    if op == "accept":
        vocab, gamma = _log_int(rng, 1000, 150000), rng.randint(1, 8)
        batch = _log_int(rng, 1, max(1, min(64, 64_000_000 // (vocab * (2 * gamma + 1)))))
        return _accept(None, rng.choice(["mtad", "spd"]), batch, gamma, vocab, rng.choice(["bf16", "fp16", "fp32"]))
    hkv = rng.choice([1, 2, 4, 8, 8, 12, 32])
    group = 1 if hkv > 8 else rng.choice([1, 2, 4, 7, 8])
    hd = rng.choice([64, 80, 128, 128, 128, 256])
    page = rng.choice([1, 16, 16, 24, 64, 128])
    batch = _log_int(rng, 1, 32)
    most = int(500_000_000 / (4.0 * hkv * hd * batch))                 # committed tokens of a sequence
    hi = _log_int(rng, 20, max(40, min(60000, most)))
    lo = max(17, int(hi * rng.uniform(0.2, 1.0)))
    if op == "append":
        rows = min(lo, _log_int(rng, 1, 256))
        return _append(None, batch, rows, hkv * group, hkv, hd, lo, hi, page, dtype, rng.choice([dtype, "fp32"]))
    if op == "evict":
        keep = max(12, int(lo * rng.uniform(0.3, 1.2)))
        first = rng.randint(0, 4)
        return _evict(None, batch, hkv, hd, lo, hi, page, keep, first, rng.randint(0, keep - first), dtype)
    window = _log_int(rng, 16, max(17, hi)) if op == "window" else 0
    return _attention(None, batch, min(lo, rng.choice([1, 1, 1, 4, 7, 16])), hkv * group, hkv, hd, lo, hi, page, dtype, window,
                      rng.randint(0, 8) if window else 0, rng.random() < 0.3)


# ---------------------------------------------------------------------------------------------------------------
# what a program has in hand before the call

def _lengths(case):
    lo, hi, b = case["lo"], case["hi"], case["batch"]
    return [lo + (hi - lo) * ((i * 2654435761 + 40503) % (1 << 16)) // (1 << 16) for i in range(b)]


def _normal(gen, dtype, std, *dims):
    return torch.empty(*dims, dtype=dtype, device="cuda").normal_(0.0, std, generator=gen)


def _uniforms(gen, *dims):
    return torch.rand(*dims, device="cuda", generator=gen).clamp_(2.0 ** -24, 1.0 - 2.0 ** -24)


def _pages(case, gen):
    """Pages of one layer [page][K|V][kv head][slot][head_dim], in the order in which a pool hands them out."""
    ps, lens = case["page"], _lengths(case)
    need = [-(-n // ps) for n in lens]
    total = sum(need) + 3
    pool = _normal(gen, DTYPES[case["dtype"]], 1.0, total, 2, case["hkv"], ps, case["hd"])
    order = torch.randperm(total, generator=torch.Generator().manual_seed(int(gen.initial_seed()) + 1)).tolist()
    table, at = torch.full((case["batch"], max(need)), -1, dtype=torch.int32), 0
    for b, n in enumerate(need):
        table[b, :n] = torch.tensor(order[at:at + n], dtype=torch.int32)
        at += n
    return {"k_pages": pool[:, 0], "v_pages": pool[:, 1], "table": table.cuda(),
            "lens": torch.tensor(lens, dtype=torch.int32, device="cuda")}


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    s = {"case": case}
    if case["op"] == "accept":
        B, g, V, dt = case["batch"], case["gamma"], case["vocab"], DTYPES[case["dtype"]]
        z = _normal(gen, torch.float32, 3.0, B, g + 1, V)
        zq = z[:, :g] + _normal(gen, torch.float32, 0.7, B, g, V)         # the auxiliary model: near the target, not the same
        s["logits"], rows = z.to(dt), zq.to(dt)
        # the drafted tokens are draws from the auxiliary model's rows
        tok = (rows.float() - _uniforms(gen, B, g, V).log_().neg_().log_()).argmax(-1)
        s["tok"], s["u_last"] = tok.to(torch.int32), _uniforms(gen, B, V)
        if case["rule"] == "spd":
            s["draft_rows"], s["u_accept"] = rows, _uniforms(gen, B, g)
        else:
            s["draft_logq"] = rows.double().log_softmax(-1).gather(2, tok[..., None])[..., 0].cumsum(-1).float()
        return s
    s.update(_pages(case, gen))
    B, hd = case["batch"], case["hd"]
    if case["op"] == "attention":
        s["q"] = _normal(gen, DTYPES[case["dtype"]], 1.5, B, case["rows"], case["hq"], hd)
        if case["weights"]:
            s["weights"] = torch.rand(B, case["hkv"], case["hi"], device="cuda", generator=gen)
    elif case["op"] == "append":
        dt = DTYPES[case["source"]]
        # one projection's output, as it lies: a row holds the query heads, the key heads, the value heads
        s["qkv"] = _normal(gen, dt, 1.0, B, case["rows"], case["hq"] + 2 * case["hkv"], hd)
    else:
        # accumulated weights: a few tokens drew most of the attention
        s["scores"] = torch.randn(B, case["hkv"], case["hi"], device="cuda", generator=gen).mul_(2.0).exp_()
        s["scores_out"] = torch.zeros(B, case["hkv"], case["keep"], device="cuda")
    return s


# ---------------------------------------------------------------------------------------------------------------
# one pass

def run(s):
    return {"attention": _run_attention, "append": _run_append, "evict": _run_evict, "accept": _run_accept}[s["case"]["op"]](s)


def _run_attention(s):
    c = s["case"]
    if own:
        import paper_2407_09722_b200 as M
        out, lse = M.paged_attention(s["q"], s["k_pages"], s["v_pages"], s["table"], s["lens"], window=c["window"], sinks=c["sinks"],
                                     weights=s.get("weights"), return_lse=True, max_len=c["hi"])
    else:
        out, lse = _plain_attention(s["q"], s["k_pages"], s["v_pages"], s["table"], s["lens"], c["window"], c["sinks"],
                                    s.get("weights"), c["hi"])
    return {"out": out, "lse": lse, "weights": s.get("weights")}


def _run_append(s):
    c = s["case"]
    q, k, v = s["qkv"].split([c["hq"], c["hkv"], c["hkv"]], dim=2)
    if own:
        import paper_2407_09722_b200 as M
        q_out = M.paged_append(q, k, v, s["k_pages"], s["v_pages"], s["table"], s["lens"], rope_base=ROPE_BASE)
    else:
        q_out = _plain_append(q, k, v, s["k_pages"], s["v_pages"], s["table"], s["lens"])
    return {"q": q_out, "k_pages": s["k_pages"], "v_pages": s["v_pages"]}


def _run_evict(s):
    c = s["case"]
    if own:
        import paper_2407_09722_b200 as M
        kept, new_lens = M.paged_evict(s["k_pages"], s["v_pages"], s["table"], s["lens"], s["scores"], c["keep"], first=c["first"],
                                       recent=c["recent"], scores_out=s["scores_out"])
    else:
        kept, new_lens = _plain_evict(s["k_pages"], s["v_pages"], s["table"], s["lens"], s["scores"], c["keep"], c["first"],
                                      c["recent"], s["scores_out"])
    return {"kept": kept, "lens": new_lens, "scores": s["scores_out"], "k_pages": s["k_pages"], "v_pages": s["v_pages"]}


def _run_accept(s):
    c = s["case"]
    if own:
        import paper_2407_09722_b200 as M
        if "result" not in s:                                             # a decode loop keeps its result arrays
            s["result"] = M.ResultBuffers(c["batch"], c["gamma"], c["gamma"])
        r = s["result"]
        if c["rule"] == "spd":
            M.accept_chain_spd(s["logits"], s["tok"], s["draft_rows"], s["u_accept"], s["u_last"], r)
        else:
            M.accept_chain(s["logits"], s["tok"], s["draft_logq"], math.log(0.1), s["u_last"], r)
        return {n: getattr(r, n) for n in ("eta", "n_out", "out_tok", "out_lp", "node_lp", "row_lse")}
    return _plain_accept(s["logits"], s["tok"], s["u_last"], s.get("draft_rows"), s.get("u_accept"), s.get("draft_logq"),
                         math.log(0.1))


# ---------------------------------------------------------------------------------------------------------------
# the plain forms

def _plain_attention(q, k_pages, v_pages, table, lens, window, sinks, weights, max_len):
    B, R, Hq, hd = q.shape
    Hkv, ps = k_pages.shape[1], k_pages.shape[2]
    n = lens.long()[:, None]
    if window and sinks + window + R < max_len:                           # only the slots that some row can see
        late = n - R - window + 1 + torch.arange(window + R - 1, device=q.device)
        late = torch.where(late >= sinks, late, -1)
        slot = torch.cat([torch.arange(sinks, device=q.device).expand(B, sinks), late], 1)
    else:
        slot = torch.arange(max_len, device=q.device).expand(B, max_len)
    pos = n - R + torch.arange(R, device=q.device)                        # [B, R]
    sl, p = slot[:, None, :], pos[:, :, None]
    seen = (sl >= 0) & (sl <= p)
    if window:
        seen = seen & ((sl > p - window) | (sl < sinks))
    at = torch.where((slot >= 0) & (slot < n), slot, 0)
    page, off = table.gather(1, at // ps).long(), at % ps
    k = k_pages[page, :, off].float().transpose(1, 2)                     # [B, Hkv, slots, hd]
    z = torch.matmul(q.float().view(B, R, Hkv, -1, hd).permute(0, 2, 1, 3, 4).reshape(B, Hkv, -1, hd), k.transpose(2, 3))
    z = z.view(B, Hkv, R, Hq // Hkv, -1) * (1.0 / math.sqrt(hd))
    z = torch.where(seen[:, None, :, None, :], z, -math.inf)
    m = z.amax(-1, keepdim=True)
    e = torch.exp(z - torch.where(m > -math.inf, m, 0.0))
    total = e.sum(-1, keepdim=True)
    prob = e / torch.where(total > 0, total, 1.0)
    v = v_pages[page, :, off].float().transpose(1, 2)
    out = torch.matmul(prob.view(B, Hkv, -1, prob.shape[-1]), v).view(B, Hkv, R, -1, hd)
    out = out.permute(0, 2, 1, 3, 4).reshape(B, R, Hq, hd).to(q.dtype)
    lse = (m + torch.log(total)).squeeze(-1).permute(0, 2, 1, 3).reshape(B, R, Hq)
    if weights is not None:
        weights.scatter_add_(2, at[:, None, :].expand(B, Hkv, -1), prob.sum((2, 3)))
    return out, lse


def _plain_append(q, k, v, k_pages, v_pages, table, lens):
    B, R, hd, ps = q.shape[0], q.shape[1], q.shape[3], k_pages.shape[2]
    slot = lens.long()[:, None] - R + torch.arange(R, device=q.device)
    inv = torch.exp2(torch.arange(hd // 2, dtype=torch.float64, device=q.device) * (-2.0 / hd * math.log2(ROPE_BASE)))
    angle = slot.double()[:, :, None, None] * inv
    cos, sin = torch.cos(angle).float(), torch.sin(angle).float()

    def turned(x):
        a, b = x[..., :hd // 2].float(), x[..., hd // 2:].float()
        return torch.cat([a * cos - b * sin, b * cos + a * sin], -1).to(k_pages.dtype)

    page, off = table.gather(1, slot // ps).long(), slot % ps
    k_pages[page, :, off] = turned(k)
    v_pages[page, :, off] = v.to(v_pages.dtype)
    return turned(q)


def _plain_evict(k_pages, v_pages, table, lens, scores, keep, first, recent, scores_out):
    B, Hkv, L = scores.shape
    ps = k_pages.shape[2]
    slot, n = torch.arange(L, device=scores.device), lens.long()[:, None]
    rank = (slot < n).long() + ((slot < n) & ((slot < first) | (slot >= n - recent))).long()      # 0 no token, 2 always kept
    rank = rank[:, None, :].expand(B, Hkv, L)
    by_score = scores.argsort(dim=-1, descending=True, stable=True)
    order = by_score.gather(2, rank.gather(2, by_score).argsort(dim=-1, descending=True, stable=True))
    count = n.clamp(max=keep)                                             # [B, 1]
    wide = max(keep, L)
    chosen = torch.full((B, Hkv, wide), wide, dtype=torch.int64, device=scores.device)
    chosen[..., :L] = torch.where(slot < count[:, None], order, wide)
    kept = chosen.sort(-1).values[..., :keep]
    there = kept < wide
    src = torch.where(there, kept, kept[..., :1].clamp(max=L - 1))
    dst = torch.where(there, torch.arange(keep, device=scores.device), 0)
    head = torch.arange(Hkv, device=scores.device)[None, :, None]
    t = table[:, None, :].expand(B, Hkv, -1)
    sp, so, dp, do = t.gather(2, src // ps).long(), src % ps, t.gather(2, dst // ps).long(), dst % ps
    k_pages[dp, head, do] = k_pages[sp, head, so]
    v_pages[dp, head, do] = v_pages[sp, head, so]
    scores_out.copy_(torch.where(there, scores.gather(2, src), 0.0))
    return torch.where(there, kept, -1).to(torch.int32), count[:, 0].to(torch.int32)


def _plain_accept(logits, tok, u_last, draft_rows, u_accept, draft_logq, log_tau):
    B, g = tok.shape
    z = logits.float()
    m = z.amax(-1, keepdim=True)
    lse = (m + torch.log(torch.exp(z - m).sum(-1, keepdim=True)))[..., 0]
    at = tok.long()[..., None]
    lp = z[:, :g].gather(2, at)[..., 0] - lse[:, :g]
    step = torch.arange(g, device=z.device)
    if draft_rows is None:
        ok = lp.cumsum(-1) - draft_logq > log_tau
        eta = torch.where(ok, step + 1, 0).amax(-1)
    else:
        y = draft_rows.float()
        my = y.amax(-1, keepdim=True)
        lse_q = (my + torch.log(torch.exp(y - my).sum(-1, keepdim=True)))[..., 0]
        ok = torch.log(u_accept) < lp - (y.gather(2, at)[..., 0] - lse_q)
        eta = ok.long().cumprod(-1).sum(-1)
    b = torch.arange(B, device=z.device)
    w = torch.exp(z[b, eta] - lse[b, eta][:, None])
    if draft_rows is not None:
        e = eta.clamp(max=g - 1)
        q = torch.exp(y[b, e] - lse_q[b, e][:, None])
        w = torch.where((eta < g)[:, None], (w - q).clamp(min=0.0), w)
    last = (w / -torch.log(u_last)).argmax(-1)
    slot = torch.arange(g + 1, device=z.device)
    pad = torch.nn.functional.pad
    out_tok = torch.where(slot < eta[:, None], pad(tok.long(), (0, 1)), torch.where(slot == eta[:, None], last[:, None], 0))
    last_lp = z[b, eta, last] - lse[b, eta]
    out_lp = torch.where(slot < eta[:, None], pad(lp, (0, 1)), torch.where(slot == eta[:, None], last_lp[:, None], 0.0))
    return {"eta": eta.to(torch.int32), "n_out": (eta + 1).to(torch.int32), "out_tok": out_tok.to(torch.int32), "out_lp": out_lp,
            "node_lp": lp, "row_lse": lse}


# ---------------------------------------------------------------------------------------------------------------
# the definitions in 64 bits

def exact(case, seed):
    s = prepare(case, seed)
    return {"attention": _exact_attention, "append": _exact_append, "evict": _exact_evict, "accept": _exact_accept}[case["op"]](s, case)


def _slots(pages, table, b, n):
    """Slots [0, n) of sequence b: [kv head, n, head_dim]."""
    ps = pages.shape[2]
    x = pages[table[b, :-(-n // ps)].long()]
    return x.transpose(0, 1).reshape(pages.shape[1], -1, pages.shape[3])[:, :n]


def _exact_attention(s, c):
    B, R, Hq, Hkv = c["batch"], c["rows"], c["hq"], c["hkv"]
    G = Hq // Hkv
    out = torch.zeros(B, R, Hq, c["hd"], dtype=torch.float64, device="cuda")
    lse = torch.zeros(B, R, Hq, dtype=torch.float64, device="cuda")
    weights = s["weights"].double() if c["weights"] else None
    for b, n in enumerate(_lengths(c)):
        k, v = _slots(s["k_pages"], s["table"], b, n).double(), _slots(s["v_pages"], s["table"], b, n).double()
        j = torch.arange(n, device="cuda")
        for r in range(R):
            at = n - R + r
            hidden = j > at
            if c["window"]:
                hidden |= (j <= at - c["window"]) & (j >= c["sinks"])
            z = torch.einsum("hgd,hnd->hgn", s["q"][b, r].double().view(Hkv, G, -1), k) / math.sqrt(c["hd"])
            z[:, :, hidden] = -math.inf
            lse[b, r] = torch.logsumexp(z, -1).view(-1)
            p = torch.exp(z - lse[b, r].view(Hkv, G, 1))
            out[b, r] = torch.einsum("hgn,hnd->hgd", p, v).reshape(Hq, -1)
            if weights is not None:
                weights[b, :, :n] += p.sum(1)
    return {"out": out, "lse": lse, "weights": weights}


def _exact_append(s, c):
    B, R, hd, ps = c["batch"], c["rows"], c["hd"], c["page"]
    x = s["qkv"].double()
    q, k, v = x[:, :, :c["hq"]], x[:, :, c["hq"]:c["hq"] + c["hkv"]], x[:, :, c["hq"] + c["hkv"]:]
    inv = torch.tensor([ROPE_BASE ** (-2.0 * i / hd) for i in range(hd // 2)], dtype=torch.float64, device="cuda")
    kp, vp = s["k_pages"].double(), s["v_pages"].double()
    q_out = torch.zeros_like(q)
    for b, n in enumerate(_lengths(c)):
        j = torch.arange(n - R, n, device="cuda")
        w = torch.polar(torch.ones(R, hd // 2, dtype=torch.float64, device="cuda"), j.double()[:, None] * inv)[:, None]
        for src, put in ((q, True), (k, False)):
            t = torch.complex(src[b, ..., :hd // 2].contiguous(), src[b, ..., hd // 2:].contiguous()) * w
            t = torch.cat([t.real, t.imag], -1)
            if put:
                q_out[b] = t
            else:
                kp[s["table"][b, j // ps].long(), :, j % ps] = t
        vp[s["table"][b, j // ps].long(), :, j % ps] = v[b]
    return {"q": q_out, "k_pages": kp, "v_pages": vp}


def _exact_evict(s, c):
    B, Hkv, keep, ps = c["batch"], c["hkv"], c["keep"], c["page"]
    k0, v0, kp, vp = s["k_pages"].clone(), s["v_pages"].clone(), s["k_pages"], s["v_pages"]
    kept = torch.full((B, Hkv, keep), -1, dtype=torch.int32, device="cuda")
    out = torch.zeros(B, Hkv, keep, dtype=torch.float64, device="cuda")
    lens = _lengths(c)
    for b, n in enumerate(lens):
        lo, hi = min(c["first"], n), max(min(c["first"], n), n - c["recent"])
        m = min(keep, n)
        for h in range(Hkv):
            z = s["scores"][b, h, :n].double()
            if n <= keep:
                idx = torch.arange(n, device="cuda")
            else:
                best = torch.sort(z[lo:hi], descending=True, stable=True).indices[:keep - lo - (n - hi)] + lo
                idx = torch.cat([torch.arange(lo, device="cuda"), best.sort().values, torch.arange(hi, n, device="cuda")])
            kept[b, h, :m] = idx.int()
            out[b, h, :m] = z[idx]
            t, d = s["table"][b].long(), torch.arange(m, device="cuda")
            kp[t[d // ps], h, d % ps] = k0[t[idx // ps], h, idx % ps]
            vp[t[d // ps], h, d % ps] = v0[t[idx // ps], h, idx % ps]
    return {"kept": kept, "lens": torch.tensor([min(n, keep) for n in lens], dtype=torch.int32, device="cuda"), "scores": out,
            "k_pages": kp, "v_pages": vp}


def _exact_accept(s, c):
    B, g = c["batch"], c["gamma"]
    f64 = dict(dtype=torch.float64, device="cuda")
    res = {"eta": torch.zeros(B, dtype=torch.int32, device="cuda"), "n_out": torch.zeros(B, dtype=torch.int32, device="cuda"),
           "out_tok": torch.zeros(B, g + 1, dtype=torch.int32, device="cuda"), "out_lp": torch.zeros(B, g + 1, **f64),
           "node_lp": torch.zeros(B, g, **f64), "row_lse": torch.zeros(B, g + 1, **f64)}
    for b in range(B):
        z = s["logits"][b].double()
        lse = torch.logsumexp(z, -1)
        p = z - lse[:, None]
        x = s["tok"][b].long()
        lp = p[:g].gather(1, x[:, None])[:, 0]
        if c["rule"] == "spd":
            q = torch.log_softmax(s["draft_rows"][b].double(), -1)
            ratio = torch.exp(lp - q.gather(1, x[:, None])[:, 0]).clamp(max=1.0)
            no = (s["u_accept"][b].double() >= ratio).tolist() + [True]
            eta = no.index(True)
        else:
            ok = (lp.cumsum(0) - s["draft_logq"][b].double() > math.log(0.1)).tolist()
            eta = max([i + 1 for i, t in enumerate(ok) if t], default=0)
        w = p[eta].exp()
        if c["rule"] == "spd" and eta < g:
            w = (w - q[eta].exp()).clamp(min=0.0)
        t = int((w.log() - torch.log(-torch.log(s["u_last"][b].double()))).argmax())
        res["eta"][b], res["n_out"][b] = eta, eta + 1
        res["out_tok"][b, :eta], res["out_lp"][b, :eta] = x[:eta].int(), lp[:eta]
        res["out_tok"][b, eta], res["out_lp"][b, eta] = t, p[eta, t]
        res["node_lp"][b], res["row_lse"][b] = lp, lse
    return res


# ---------------------------------------------------------------------------------------------------------------
# what one pass cannot do without

def work(case):
    size = {"bf16": 2.0, "fp16": 2.0, "fp32": 4.0}
    B = float(case["batch"])
    if case["op"] == "accept":
        g, V = case["gamma"], float(case["vocab"])
        rows = g + 1 + (g if case["rule"] == "spd" else 0)
        return {"bytes": B * V * (rows * size[case["dtype"]] + 4.0), "flops": 4.0 * B * V * rows}
    lens, hd, el = _lengths(case), case["hd"], size[case["dtype"]]
    token = 2.0 * case["hkv"] * hd                                        # elements of one token's keys and values
    if case["op"] == "append":
        n, rows = B * case["rows"], case["hq"] * hd
        return {"bytes": n * ((rows + token) * size[case["source"]] + (rows + token) * el), "flops": 3.0 * n * (rows + token / 2)}
    if case["op"] == "evict":
        moved = float(sum(min(n, case["keep"]) for n in lens if n > case["keep"]))
        return {"bytes": 2.0 * moved * token * el + 4.0 * case["hkv"] * sum(lens) + 12.0 * B * case["hkv"] * case["keep"], "flops": 0.0}
    R, W = case["rows"], case["window"]
    read = float(sum(min(n, min(case["sinks"], n) + W + R - 1) if W else n for n in lens))
    nbytes = read * token * el + 2.0 * B * R * case["hq"] * hd * el + (8.0 * case["hkv"] * read if case["weights"] else 0.0)
    return {"bytes": nbytes, "flops": 4.0 * R * case["hq"] * hd * read}
