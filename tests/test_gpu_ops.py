"""Operators around a decoder of the caller's own, against their definitions in 64 bits: the paged append with the rotary
embedding, attention over the pages (window, sinks, weights), eviction, the accept rules on rows of logits, and a run of them together."""
import math

import pytest
import torch

import paper_2407_09722_b200 as M
from paper_2407_09722_b200 import binding as Bn

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}


def half_step(dt):
    """A value rounded to the nearest is off by at most this share of it."""
    return torch.finfo(dt).eps / 2


class Cache:
    """Pages of one layer in a scattered order, with slots that no sequence owns full of NaN."""

    def __init__(self, seed, lens, hkv, hd, page, dtype=torch.bfloat16, spare=3, layout="head", pad=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.lens_list, self.hkv, self.hd, self.page, self.dtype = list(lens), hkv, hd, page, dtype
        need = [max(-(-n // page), 1) for n in lens]
        total = sum(need) + spare
        shape = (total, 2, hkv, page, hd + pad) if layout == "head" else (total, 2, page, hkv, hd + pad)
        pool = torch.empty(shape, dtype=dtype, device="cuda").normal_(generator=g)
        self.pool = pool
        self.k, self.v = pool[:, 0, ..., :hd], pool[:, 1, ..., :hd]
        if layout != "head":
            self.k, self.v = self.k.transpose(1, 2), self.v.transpose(1, 2)
        order = torch.randperm(total, generator=torch.Generator().manual_seed(seed)).tolist()
        self.table = torch.full((len(lens), max(need) + 1), 2 ** 31 - 1, dtype=torch.int32)
        at = 0
        for b, n in enumerate(need):
            self.table[b, :n] = torch.tensor(order[at:at + n], dtype=torch.int32)
            at += n
        self.spare_pages = order[at:]
        for b, n in enumerate(lens):                                     # behind the last slot: what must never be seen
            for j in range(n, need[b] * page):
                p, o = int(self.table[b, j // page]), j % page
                self.k[p, :, o] = float("nan")
                self.v[p, :, o] = float("nan")
        for p in self.spare_pages:
            self.k[p] = float("nan")
            self.v[p] = float("inf")
        self.table = self.table.cuda()
        self.lens = torch.tensor(lens, dtype=torch.int32, device="cuda")

    def rows(self, which, b, n):
        """[kv head, n, head_dim] in 64 bits."""
        j = torch.arange(n, device="cuda")
        x = (self.k if which == "k" else self.v)[self.table[b, j // self.page].long(), :, j % self.page]
        return x.double().transpose(0, 1)

    def args(self):
        return self.k, self.v, self.table


def seen_by(n, at, window, sinks):
    j = torch.arange(n, device="cuda")
    see = j <= at
    if window:
        see &= (j > at - window) | (j < sinks)
    return see


def attention_ref(c, q, nb, window, sinks, scale):
    """Output, lse, weights in 64 bits and the bound of the fp32 computation: products of the scores are exact in fp32, a sum of hd
    of them, rounded (or cut off) at every addition, is off by at most hd * 2^-23 of the sum of their magnitudes; the probability's exponential
    carries that error, its own 2^-22 and the two-term rounding (2^-16 at most) into the output as a share of the largest value seen."""
    B, R, Hq, hd = q.shape
    G = Hq // c.hkv
    out, lse = torch.zeros(B, R, Hq, hd, dtype=torch.float64, device="cuda"), torch.full((B, R, Hq), -math.inf, dtype=torch.float64, device="cuda")
    tol, tol_s = torch.zeros_like(out), torch.zeros_like(lse)
    w = torch.zeros(B, c.hkv, max(c.lens_list + [1]), dtype=torch.float64, device="cuda")
    for b, n in enumerate(c.lens_list):
        if n == 0:
            continue
        k, v = c.rows("k", b, n), c.rows("v", b, n)
        for r in range(nb[b]):
            see = seen_by(n, n - nb[b] + r, window, sinks)
            if not bool(see.any()):
                continue
            kk, vv, qq = k[:, see], v[:, see], q[b, r].double().view(c.hkv, G, hd)
            s = torch.einsum("hgd,hnd->hgn", qq, kk) * scale
            lse[b, r] = torch.logsumexp(s, -1).view(-1)
            p = torch.exp(s - lse[b, r].view(c.hkv, G, 1))
            out[b, r] = torch.einsum("hgn,hnd->hgd", p, vv).reshape(Hq, hd)
            w[b, :, :n][:, see] += p.sum(1)
            ds = (torch.einsum("hgd,hnd->hgn", qq.abs(), kk.abs()) * scale).amax(-1) * (hd + 8) * 2.0 ** -23
            tol_s[b, r] = ds.view(-1) + 2.0 ** -20
            tol[b, r] = ((2 * ds + 2.0 ** -16)[..., None] * vv.abs().amax(1)[:, None, :].amax(-1, keepdim=True)).expand(-1, -1, hd).reshape(Hq, hd)
    return out, lse, w, tol, tol_s


def check_attention(c, q, window=0, sinks=0, n_rows=None, scale=0.0, weights=True, **kw):
    B, R, Hq, hd = q.shape
    nb = [R] * B if n_rows is None else list(n_rows)
    sc = scale or 1 / math.sqrt(hd)
    ref, lse_ref, w_ref, tol, tol_s = attention_ref(c, q, nb, window, sinks, sc)
    w0 = torch.rand(B, c.hkv, max(c.lens_list + [1]) + 5, device="cuda")
    w = w0.clone() if weights else None
    status = torch.zeros(B, dtype=torch.int32, device="cuda")
    out = torch.full((B, R, Hq, hd), 7.0, dtype=q.dtype, device="cuda")
    lse = torch.full((B, R, Hq), 7.0, device="cuda")
    M.paged_attention(q, *c.args(), c.lens, window=window, sinks=sinks, weights=w, out=out, lse=lse, scale=scale, status=status,
                      n_rows=None if n_rows is None else torch.tensor(nb, dtype=torch.int32, device="cuda"),
                      max_len=max(c.lens_list + [1]), **kw)
    torch.cuda.synchronize()
    assert not status.any()
    for b in range(B):
        n = nb[b]
        assert bool((out[b, n:] == 7).all()) and bool((lse[b, n:] == 7).all())          # rows behind the last: left alone
        o, r = out[b, :n].double(), ref[b, :n]
        bad = (o - r).abs() > half_step(q.dtype) * r.abs() + tol[b, :n] + torch.finfo(q.dtype).smallest_normal
        assert not bool(bad.any()) and bool(torch.isfinite(o).all()), (b, float((o - r).abs().max()))
        l, lr = lse[b, :n].double(), lse_ref[b, :n]
        assert torch.equal(torch.isinf(l), torch.isinf(lr))
        fin = torch.isfinite(lr)
        assert bool(((l - lr).abs()[fin] <= (tol_s[b, :n] + 2.0 ** -21 * lr.abs())[fin]).all())
    if weights:
        G = Hq // c.hkv
        d = (w.double() - w0.double())
        n = w_ref.shape[2]
        # a probability is off by its exponent's error (2 tol_s covers score and lse), a sum of fp32 additions by 2^-24 each
        top = float(tol_s.max()) * 2 if tol_s.numel() else 0.0
        assert bool(((d[..., :n] - w_ref).abs() <= w_ref * (top + 2.0 ** -18) + 2.0 ** -23 * (1 + R * G)).all())
        assert torch.equal(w[..., n:], w0[..., n:])
        for b in range(B):
            untouched = w_ref[b] == 0
            assert torch.equal(w[b, :, :n][untouched], w0[b, :, :n][untouched])
    return out, lse


def queries(seed, B, R, Hq, hd, dtype, std=1.5):
    g = torch.Generator(device="cuda").manual_seed(seed + 77)
    return torch.empty(B, R, Hq, hd, dtype=dtype, device="cuda").normal_(0, std, generator=g)


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("hd,hq,hkv,rows", [(64, 12, 12, 1), (128, 8, 8, 5), (128, 64, 8, 1), (128, 16, 2, 3), (128, 16, 1, 4), (80, 7, 1, 2),
                                            (256, 4, 2, 1), (256, 8, 1, 3), (256, 8, 1, 7), (8, 2, 1, 1), (64, 8, 1, 33)])
def test_attention_heads_and_types(dtype, hd, hq, hkv, rows):
    """Query rows a KV head from 1 to 264: every tile height, one and several row blocks, heads that are padded to a tile's width."""
    c = Cache(1, [1, 63, 64, 65, 700], hkv, hd, 16, DT[dtype])
    check_attention(c, queries(1, 5, rows, hq, hd, DT[dtype]))


@pytest.mark.parametrize("page", [1, 5, 16, 64, 100, 4096])
@pytest.mark.parametrize("lens", [[0], [1], [333], [0, 2500, 1, 64, 0], [129] * 9])
def test_attention_lengths_and_pages(page, lens):
    """Empty sequences between others, one slot, pages that end inside a tile or hold all of it, lengths on and off the tiles."""
    c = Cache(2, lens, 2, 128, page)
    check_attention(c, queries(2, len(lens), 1, 8, 128, torch.bfloat16))


@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 4), (64, 0), (100, 4), (63, 64), (65, 130), (700, 3), (5000, 2), (257, 0)])
@pytest.mark.parametrize("rows", [1, 6])
def test_attention_window_and_sinks(window, sinks, rows):
    c = Cache(3, [1, 3, 64, 200, 777, 1500], 2, 64, 16)
    check_attention(c, queries(3, 6, rows, 4, 64, torch.bfloat16), window=window, sinks=sinks)


def test_attention_window_longer_than_a_block_takes_whole():
    c = Cache(4, [9000, 4100, 12345], 2, 128, 64)
    check_attention(c, queries(4, 3, 2, 16, 128, torch.bfloat16), window=3000, sinks=70)


@pytest.mark.parametrize("rows", [1, 9])
def test_attention_one_long_sequence_cut_over_the_gpu(rows):
    c = Cache(5, [40003], 1, 128, 48)
    check_attention(c, queries(5, 1, rows, 4, 128, torch.bfloat16))


def test_attention_ragged_rows_and_rows_before_the_first_slot():
    """n_rows from 0 to the call's; a length shorter than the rows leaves the first rows without a slot."""
    c = Cache(6, [300, 2, 0, 64, 5], 2, 64, 16)
    check_attention(c, queries(6, 5, 4, 4, 64, torch.bfloat16), n_rows=[4, 4, 3, 0, 1])


@pytest.mark.parametrize("rows,hq", [(3, 2), (9, 4), (16, 4)])
@pytest.mark.parametrize("window,sinks", [(0, 0), (50, 4)])
def test_attention_infinities_that_only_later_rows_see(rows, hq, window, sinks):
    """Values of the last row's own slot are infinite, or NaN: earlier rows, and rows whose window has moved past such a slot,
    do not change by a bit; rows that see it carry it."""
    c = Cache(7, [200, 64, 129], 2, 64, 16)
    q = queries(7, 3, rows, hq, 64, torch.bfloat16)
    want, _ = check_attention(c, q, window=window, sinks=sinks, weights=False)
    hit = [(199, float("inf"))] + ([(200 - rows - 50 + 1, float("nan"))] if window else [])
    seen = torch.zeros(rows, dtype=torch.bool)
    for j, x in hit:
        p, o = int(c.table[0, j // 16]), j % 16
        c.v[p, :, o, ::3] = x
        if x != x:
            c.k[p, :, o] = x
        seen |= torch.tensor([bool(seen_by(200, 200 - rows + r, window, sinks)[j]) for r in range(rows)])
    got = M.paged_attention(q, *c.args(), c.lens, window=window, sinks=sinks, max_len=200)
    assert torch.equal(got[1:], want[1:])
    assert not bool(seen.all())
    for r in range(rows):
        if not seen[r]:
            # the sums are formed in another order where such a row is added by hand: the bound of two fp32 sums, then a rounding each
            d = (got[0, r].double() - want[0, r].double()).abs()
            assert bool((d <= 2 * half_step(q.dtype) * want[0, r].double().abs() + 2.0 ** -16 * 6).all())
        else:
            assert not bool(torch.isfinite(got[0, r, :, ::3]).all())


def test_attention_strides_layouts_and_offsets_past_31_bits():
    """Pages as [slot][head], padded rows, queries as a slice of a fused projection; a pool whose last page lies past 2^31 elements."""
    c = Cache(8, [70, 200], 4, 64, 16, layout="slot", pad=8)
    qkv = torch.randn(2, 3, 8 + 8, 64, device="cuda").bfloat16()
    check_attention(c, qkv[:, :, :8])
    hkv, page, hd = 2, 256, 128
    pool = torch.empty(18000, 2, hkv, page, hd, dtype=torch.bfloat16, device="cuda")
    assert pool.numel() > 2 ** 31
    c = Cache(8, [700], hkv, hd, page, spare=0)
    far = torch.tensor([17999, 17990, 17777], dtype=torch.int64)
    pool[far.cuda()] = c.pool[c.table[0, :3].long()]
    c.k, c.v, c.table = pool[:, 0], pool[:, 1], far.int().cuda()[None]
    check_attention(c, queries(8, 1, 1, 8, hd, torch.bfloat16))


def test_attention_over_a_layer_of_the_contiguous_cache():
    """One layer of the cache that the verify calls keep is a paged cache whose pages are the sequences."""
    L, Bn_, hkv, cap, hd = 3, 4, 2, 160, 64
    cache = torch.randn(L, Bn_, 2, hkv, cap, hd, device="cuda").bfloat16()
    lens = [100, 7, 160, 64]
    c = Cache(9, lens, hkv, hd, 160)
    c.k, c.v, c.page = cache[1, :, 0], cache[1, :, 1], cap
    c.table = torch.arange(Bn_, dtype=torch.int32, device="cuda")[:, None]
    check_attention(c, queries(9, 4, 1, 4, hd, torch.bfloat16))


def test_attention_shared_prefix_pages():
    c = Cache(10, [200, 150], 2, 64, 16)
    c.table[1, :9] = c.table[0, :9]
    c.lens_list = [200, 144]
    c.lens = torch.tensor(c.lens_list, dtype=torch.int32, device="cuda")
    check_attention(c, queries(10, 2, 1, 4, 64, torch.bfloat16))


def test_attention_flags_bad_pages_and_lengths():
    c = Cache(11, [100, 100, 100, 50], 1, 64, 16)
    q = queries(11, 4, 1, 2, 64, torch.bfloat16)
    good = M.paged_attention(q, *c.args(), c.lens, max_len=100)
    c.table[0, 2] = -5
    c.table[1, 0] = c.k.shape[0]
    lens = torch.tensor([100, 100, 100000, -3], dtype=torch.int32, device="cuda")
    status = torch.zeros(4, dtype=torch.int32, device="cuda")
    out, lse = M.paged_attention(q, *c.args(), lens, max_len=100, status=status, return_lse=True)
    assert status.tolist() == [Bn.MTAD_ST_RANGE, Bn.MTAD_ST_RANGE, 4, 4]
    assert torch.equal(out[2], good[2])
    assert not bool(out[3].any()) and bool((lse[3] == -math.inf).all())


def test_attention_is_the_same_every_time_and_in_a_graph():
    c = Cache(12, [5000, 321, 2048], 2, 128, 16)
    q = queries(12, 3, 2, 8, 128, torch.bfloat16)
    w = torch.zeros(3, 2, 5000, device="cuda")
    a, al = M.paged_attention(q, *c.args(), c.lens, weights=w, max_len=5000, return_lse=True)
    wa = w.clone()
    for _ in range(3):
        w.zero_()
        b, bl = M.paged_attention(q, *c.args(), c.lens, weights=w, max_len=5000, return_lse=True)
        assert torch.equal(a, b) and torch.equal(al, bl) and torch.equal(w, wa)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graphs = []
    with torch.cuda.stream(side):
        for _ in range(2):                                                # two graphs, each with scratch of its own
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=side):
                y = M.paged_attention(q, *c.args(), c.lens, max_len=5000)
            graphs.append((g, y))
    torch.cuda.synchronize()
    q2 = queries(13, 3, 2, 8, 128, torch.bfloat16)
    q.copy_(q2)
    c.lens.copy_(torch.tensor([77, 300, 1999], dtype=torch.int32))
    for g, _ in graphs:
        g.replay()
    torch.cuda.synchronize()
    want = M.paged_attention(q, *c.args(), c.lens, max_len=5000)
    assert all(torch.equal(y, want) for _, y in graphs)


def test_attention_on_streams_of_its_own_at_once():
    c = Cache(14, [20000, 3000], 2, 128, 16)
    qs = [queries(s, 2, 1, 16, 128, torch.bfloat16) for s in range(4)]
    want = [M.paged_attention(q, *c.args(), c.lens, max_len=20000) for q in qs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in qs]
    got = [M.paged_attention(q, *c.args(), c.lens, max_len=20000, stream=s) for q, s in zip(qs, streams) for _ in range(3)]
    torch.cuda.synchronize()
    assert all(torch.equal(g, want[i // 3]) for i, g in enumerate(got))


# ---------------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("src", ["same", "fp32"])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("hd,hq,hkv,rows,page", [(64, 12, 12, 1, 16), (128, 8, 2, 5, 7), (80, 3, 1, 33, 16), (8, 2, 2, 2, 1), (256, 4, 1, 3, 64), (72, 2, 1, 4, 16)])
def test_append(src, dtype, hd, hq, hkv, rows, page):
    """Slots are written with the turned keys and the values, the rest of the pool keeps its bits; angles at far positions."""
    dt = DT[dtype]
    sdt = dt if src == "same" else torch.float32
    lens = [rows, 100, 1000]
    c = Cache(20, lens, hkv, hd, page, dt)
    before = c.pool.clone()
    x = torch.randn(3, rows, hq + 2 * hkv, hd, device="cuda").to(sdt)
    q, k, v = x.split([hq, hkv, hkv], 2)
    n_rows = [rows, max(rows - 1, 0), rows]
    pos = torch.tensor([0, 131071, 999999], dtype=torch.int32, device="cuda")
    base = 500000.0
    out = torch.full((3, rows, hq, hd), 7.0, dtype=dt, device="cuda")
    status = torch.zeros(3, dtype=torch.int32, device="cuda")
    M.paged_append(q, k, v, *c.args(), c.lens, n_rows=torch.tensor(n_rows, dtype=torch.int32, device="cuda"), pos=pos, rope_base=base,
                   q_out=out, status=status)
    assert not status.any()
    inv = base ** (-2.0 * torch.arange(hd // 2, dtype=torch.float64, device="cuda") / hd)
    bits = before.view(torch.int16).clone()
    view = bits.view(before.shape)

    def turned(t, p):
        a, b = t[..., :hd // 2].double(), t[..., hd // 2:].double()
        cs, sn = torch.cos(p * inv), torch.sin(p * inv)
        # sine and cosine are good to 2^-22, two products and a sum are rounded to 2^-24 each
        return torch.cat([a * cs - b * sn, b * cs + a * sn], -1), 2.0 ** -21 * torch.cat([a.abs() + b.abs()] * 2, -1)

    for b in range(3):
        n = n_rows[b]
        assert bool((out[b, n:] == 7).all())
        for r in range(n):
            p = float(int(pos[b]) + r)
            want, tol = turned(q[b, r], p)
            tol = tol + half_step(dt) * want.abs() * (1 + 2.0 ** -10) + torch.finfo(dt).smallest_normal
            assert bool(((out[b, r].double() - want).abs() <= tol).all())
            slot = lens[b] - n + r
            pg, o = int(c.table[b, slot // page]), slot % page
            want, tol = turned(k[b, r], p)
            tol = tol + half_step(dt) * want.abs() * (1 + 2.0 ** -10) + torch.finfo(dt).smallest_normal
            assert bool(((c.k[pg, :, o].double() - want).abs() <= tol).all())
            assert torch.equal(c.v[pg, :, o], v[b, r].to(dt))
            view[pg, :, :, o] = c.pool.view(torch.int16)[pg, :, :, o]
    assert torch.equal(c.pool.view(torch.int16), view)


def test_append_without_rotation_in_place_and_keys_alone():
    c = Cache(21, [40], 2, 64, 16)
    x = torch.randn(1, 3, 8, 64, device="cuda").bfloat16()
    q, k, v = x.split([4, 2, 2], 2)
    q0 = q.clone()
    assert M.paged_append(q, k, v, *c.args(), c.lens, q_out=q) is q and torch.equal(q, q0)
    j = torch.arange(37, 40, device="cuda")
    assert torch.equal(c.k[c.table[0, j // 16].long(), :, j % 16], k[0])
    assert M.paged_append(None, k, v, *c.args(), c.lens, rope_base=10000.0) is None
    turned = M.paged_append(q, k, v, *c.args(), c.lens, rope_base=10000.0)
    again = M.paged_append(q, k, v, *c.args(), c.lens, rope_base=10000.0, q_out=q)
    assert torch.equal(turned, again) and again is q


def test_append_flags_slots_outside():
    c = Cache(22, [20, 20, 20], 1, 64, 16)
    before = c.pool.clone()
    k = torch.randn(3, 4, 1, 64, device="cuda").bfloat16()
    lens = torch.tensor([2, 16 * c.table.shape[1] + 1, 20], dtype=torch.int32, device="cuda")
    c.table[2, 1] = 12345
    status = torch.zeros(3, dtype=torch.int32, device="cuda")
    M.paged_append(None, k, k, *c.args(), lens, n_rows=torch.tensor([4, 1, 2], dtype=torch.int32, device="cuda"), status=status)
    assert status.tolist() == [4, 4, Bn.MTAD_ST_RANGE]
    p = int(c.table[0, 0])
    assert torch.equal(c.k[p, :, 0], k[0, 2]) and torch.equal(c.k[p, :, 1], k[0, 3])
    c.pool[p, :, :, :2] = before[p, :, :, :2]
    assert torch.equal(c.pool.view(torch.int16), before.view(torch.int16))


# ---------------------------------------------------------------------------------------------------------------

def evict_ref(scores, n, keep, first, recent):
    if n <= keep:
        return list(range(n))
    key = [math.inf if s != s else s for s in scores]
    nan = [s != s for s in scores]
    mid = sorted(range(first, n - recent), key=lambda j: (not nan[j], -key[j], j))[:keep - first - recent]
    return sorted(list(range(first)) + mid + list(range(n - recent, n)))


def check_evict(c, scores, keep, first, recent, in_place=False, **kw):
    B = len(c.lens_list)
    s0, pool0 = scores.clone(), c.pool.clone()
    so = scores if in_place else torch.full((B, c.hkv, keep), 7.0, device="cuda")
    kept, new = M.paged_evict(*c.args(), c.lens, scores, keep, first=first, recent=recent, scores_out=so, **kw)
    assert new.tolist() == [min(n, keep) for n in c.lens_list]
    host, k_host = s0.cpu(), kept.cpu()
    bits, want = pool0.view(torch.int16), pool0.view(torch.int16).clone()
    s_want = s0.clone() if in_place else torch.full((B, c.hkv, keep), 7.0, device="cuda")
    for b, n in enumerate(c.lens_list):
        for h in range(c.hkv):
            idx = evict_ref(host[b, h, :n].tolist(), n, keep, first, recent)
            assert k_host[b, h].tolist() == idx + [-1] * (keep - len(idx)), (b, h)
            j = torch.tensor(idx, dtype=torch.int64, device="cuda")
            d = torch.arange(len(idx), device="cuda")
            t = c.table[b].long()
            want[t[d // c.page], :, h, d % c.page] = bits[t[j // c.page], :, h, j % c.page]
            s_want[b, h, :len(idx)] = s0[b, h, j]
    assert torch.equal(c.pool.view(torch.int16), want)
    assert torch.equal(so.view(torch.int32), s_want.view(torch.int32))
    if not in_place:
        assert torch.equal(scores.view(torch.int32), s0.view(torch.int32))


@pytest.mark.parametrize("lens,keep,first,recent", [([300], 100, 4, 32), ([1000, 64, 0, 65, 66], 65, 1, 30), ([5000, 2], 4999, 4, 100),
                                                    ([777], 20, 10, 10), ([777], 1, 0, 0), ([40, 41], 40, 40, 0), ([3000], 1500, 0, 0),
                                                    ([9, 8, 7], 8, 0, 8)])
@pytest.mark.parametrize("in_place", [False, True])
def test_evict_what_stays_and_where_it_goes(lens, keep, first, recent, in_place):
    """Nothing to evict, one slot, all but one, no room for scores beside what always stays."""
    c = Cache(30, lens, 3, 64, 16)
    g = torch.Generator(device="cuda").manual_seed(1)
    check_evict(c, torch.randn(len(lens), 3, max(max(lens), keep), device="cuda", generator=g).exp(), keep, first, recent, in_place, max_len=max(lens))


@pytest.mark.parametrize("hd,page,dtype", [(8, 1, "bf16"), (24, 5, "fp16"), (80, 16, "bf16"), (128, 100, "bf16"), (256, 16, "fp16")])
def test_evict_rows_and_pages(hd, page, dtype):
    c = Cache(31, [600, 350], 2, hd, page, DT[dtype])
    check_evict(c, torch.rand(2, 2, 600, device="cuda"), 200, 3, 50)


@pytest.mark.parametrize("kind", ["equal", "few", "zeros", "special", "negative"])
def test_evict_ties_and_special_scores(kind):
    """Equal scores go to the lower slot; signed zeros are equal; infinities, NaN and subnormals have their places."""
    n = 2000
    g = torch.Generator().manual_seed(3)
    s = torch.randn(1, 2, n, generator=g)
    if kind == "equal":
        s = torch.ones(1, 2, n)
    elif kind == "few":
        s = (s * 2).round()
    elif kind == "zeros":
        s = torch.where(s > 0, torch.tensor(0.0), torch.tensor(-0.0))
        s[:, :, ::7] = 1e-42
    elif kind == "special":
        s[:, :, ::5], s[:, :, 1::7], s[:, :, 2::11] = float("inf"), float("nan"), -float("inf")
    else:
        s = -s.abs()
    c = Cache(32, [n], 2, 64, 16)
    check_evict(c, s.cuda(), 700, 2, 100)


def test_evict_scores_that_do_not_fit_a_block():
    """Beyond 327680 slots the scores are read again from memory."""
    n = 330000
    c = Cache(33, [n], 1, 8, 512)
    check_evict(c, torch.rand(1, 1, n, device="cuda"), 1000, 4, 64)
    with pytest.raises(M.MtadError):
        s = torch.rand(1, 1, n, device="cuda")
        M.paged_evict(*c.args(), c.lens, s, 1000, scores_out=s)


def test_evict_flags_bad_pages_and_lengths():
    c = Cache(34, [100, 100], 1, 64, 16)
    s = torch.rand(2, 1, 112, device="cuda")
    status = torch.zeros(2, dtype=torch.int32, device="cuda")
    c.table[0, 5] = -1
    lens = torch.tensor([100, 5000], dtype=torch.int32, device="cuda")
    _, new = M.paged_evict(*c.args(), lens, s, 20, recent=18, max_len=100, status=status)
    assert status.tolist() == [Bn.MTAD_ST_RANGE, 4] and new.tolist() == [20, 20]


# ---------------------------------------------------------------------------------------------------------------

def accept_ref(z, tok, u_last, g, temperature=1.0, draft=None, u_acc=None, logq=None, log_tau=None, draft_temperature=1.0):
    p = torch.log_softmax(z.double() / temperature, -1)
    lse = torch.logsumexp(z.double() / temperature, -1)
    x = tok[:g].long()
    lp = p[:g].gather(1, x[:, None])[:, 0]
    if draft is not None:
        q = torch.log_softmax(draft.double() / draft_temperature, -1)
        ratio = (lp - q[:g].gather(1, x[:, None])[:, 0]).clamp(max=0.0)
        d = u_acc[:g].double().log() - ratio
        ok = [(bool(t < 0) and bool(l > -math.inf)) for t, l in zip(d, lp)] + [False]
        eta = ok.index(False)
        margin = d[:eta + 1].abs()
    else:
        d = lp.cumsum(0) - (logq[:g].double() if g else 0.0) - log_tau
        eta = max([i + 1 for i in range(g) if d[i] > 0 or log_tau == -math.inf], default=0)
        margin = d.abs()
    w = p[eta].exp()
    if draft is not None and eta < g:
        w = (w - q[eta].exp()).clamp(min=0.0)
    score = w.log() - torch.log(-torch.log(u_last.double()))
    best = torch.sort(score, descending=True, stable=True)
    gap = float(best.values[0] - best.values[1]) if len(score) > 1 else 1.0
    if draft is not None and eta < g:
        # p - q cancels where the models agree: the winner counts where it leads with its own weight lowered and every other one raised by
        # the errors of p and q, 2^-20 of each (an fp32 exponential of a log-probability that is off by 2^-21)
        e, E = 2.0 ** -20, -torch.log(u_last.double())
        pp, qq, i = p[eta].exp(), q[eta].exp(), best.indices[0]
        high = (pp * (1 + e) - qq * (1 - e)).clamp(min=0.0) / E
        high[i] = -1.0
        if not bool((pp[i] * (1 - e) - qq[i] * (1 + e)) / E[i] > high.max()):
            gap = 0.0
    return eta, int(best.indices[0]), lp, lse, p, float(margin.min()) if len(margin) else 1.0, gap


def check_accept(rule, z, tok, u, draft=None, u_acc=None, logq=None, log_tau=math.log(0.2), n_draft=None, temperature=1.0, draft_temperature=1.0,
                 compare=True):
    B, r, V = z.shape
    D = r - 1
    nd = [D] * B if n_draft is None else n_draft
    res = M.ResultBuffers(B, D, D)
    kw = dict(n_draft=None if n_draft is None else torch.tensor(nd, dtype=torch.int32, device="cuda"), temperature=temperature)
    if rule == "spd":
        M.accept_chain_spd(z, tok, draft, u_acc, u, res, draft_temperature=draft_temperature, **kw)
    else:
        M.accept_chain(z, tok, logq, log_tau, u, res, **kw)
    h = {n: getattr(res, n).cpu() for n in ("eta", "winner", "path", "n_out", "out_tok", "out_lp", "node_lp", "node_LP", "row_lse", "status", "margin")}
    compared = 0
    for b in range(B):
        g = nd[b]
        eta, last, lp, lse, p, margin, gap = accept_ref(z[b, :g + 1], tok[b] if D else torch.zeros(0, device="cuda"), u[b], g, temperature,
                                                        draft[b] if draft is not None else None, u_acc[b] if u_acc is not None else None,
                                                        logq[b] if logq is not None else None, log_tau, draft_temperature)
        assert int(h["status"][b]) == 0
        # z / temperature, its difference from the largest and the logarithm are fp32 (2^-24 of up to ~100 each); sums of exponentials 2^-20
        tol = 2.0 ** -19 + 2.0 ** -22 * float(lse.abs().max() + (z[b].abs()[torch.isfinite(z[b])].max() / temperature).float())
        ok = torch.isfinite(lp).cpu()
        assert bool(((h["node_lp"][b, :g].double() - lp.cpu())[ok].abs() <= tol).all()) and bool((h["node_lp"][b, g:] == 0).all())
        assert bool(((h["row_lse"][b, :g + 1].double() - lse.cpu()).abs() <= tol).all()) and bool((h["row_lse"][b, g + 1:] == 0).all())
        if margin < 64 * tol or gap < 1e-4:
            continue
        compared += 1
        assert int(h["eta"][b]) == eta and int(h["n_out"][b]) == eta + 1 and int(h["winner"][b]) == eta - 1
        assert h["out_tok"][b, :eta].tolist() == (tok[b, :eta].tolist() if D else []) and h["path"][b, :eta].tolist() == list(range(eta))
        assert int(h["out_tok"][b, eta]) == last
        assert abs(float(h["out_lp"][b, eta]) - float(p[eta, last])) <= tol
        if rule != "spd" and g:
            assert bool(((h["node_LP"][b, :g].double() - lp.cumsum(0).cpu()).abs() <= g * tol).all())
        if g:
            assert abs(float(h["margin"][b, 0]) - margin) <= (g + 1) * tol
    assert compared >= B // 2 or not compare
    return h


def rows_of(seed, B, D, V, dtype):
    g = torch.Generator(device="cuda").manual_seed(seed)
    z = torch.randn(B, D + 1, V, device="cuda", generator=g) * 2
    dr = (z[:, :D] + 0.8 * torch.randn(B, D, V, device="cuda", generator=g)).to(dtype)
    u = torch.rand(B, V, device="cuda", generator=g).clamp_(2.0 ** -24, 1 - 2.0 ** -24)
    ua = torch.rand(B, max(D, 1), device="cuda", generator=g).clamp_(2.0 ** -24, 1 - 2.0 ** -24)[:, :D].contiguous()
    tok = (dr.float() - torch.rand(B, D, V, device="cuda", generator=g).clamp_(1e-6, 1 - 1e-6).log().neg().log()).argmax(-1).int()
    logq = dr.double().log_softmax(-1).gather(2, tok.long()[..., None])[..., 0].cumsum(-1).float()
    return z.to(dtype), dr, tok, u, ua, logq


@pytest.mark.parametrize("rule", ["mtad", "spd"])
@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("B,D,V", [(1, 1, 1), (3, 1, 7), (1, 4, 64), (5, 3, 1009), (2, 32, 515), (9, 6, 32000), (30, 2, 777), (100, 1, 300),
                                   (2, 2, 100003)])
def test_accept_rows(rule, dtype, B, D, V):
    """Vocabularies of one token, smaller than a cluster, odd (rows begin off 16 bytes), large; one to 32 drafted tokens."""
    z, dr, tok, u, ua, logq = rows_of(B * V + D, B, D, V, DT[dtype])
    check_accept(rule, z, tok, u, dr if rule == "spd" else None, ua if rule == "spd" else None, logq if rule == "mtad" else None)


@pytest.mark.parametrize("rule", ["mtad", "spd"])
def test_accept_ragged_chains_strides_and_temperatures(rule):
    z, dr, tok, u, ua, logq = rows_of(5, 4, 5, 3001, torch.bfloat16)
    wide = torch.zeros(4, 9, 3011, device="cuda", dtype=torch.bfloat16)
    wide[:, 2:8, 3:3004] = z
    z = wide[:, 2:8, 3:3004]
    z[1, 3:] = float("nan")                                               # rows that do not count
    kw = dict(n_draft=[5, 2, 0, 4], temperature=0.7)
    if rule == "spd":
        check_accept(rule, z, tok, u, dr, ua, draft_temperature=1.3, **kw)
    else:
        check_accept(rule, z, tok, u, logq=logq, **kw)


def test_accept_no_draft_and_tau_zero():
    z, dr, tok, u, ua, logq = rows_of(6, 3, 0, 500, torch.float32)
    check_accept("mtad", z, None, u)
    z, dr, tok, u, ua, logq = rows_of(6, 3, 4, 500, torch.float32)
    z[0, 1, int(tok[0, 1])] = -math.inf
    res = M.ResultBuffers(3, 4, 4)
    M.accept_chain(z, tok, logq, -math.inf, u, res)
    assert res.eta.tolist() == [4, 4, 4] and not res.status.any()


def test_accept_masked_logits():
    """Tokens masked by -inf are never drawn, a drafted one is rejected; one that the draft could not have drawn is accepted where the target can."""
    z, dr, tok, u, ua, logq = rows_of(7, 2, 2, 400, torch.float32)
    z[:, :, 100:] = -math.inf
    tok[:] = torch.tensor([[5, 6], [200, 6]], dtype=torch.int32)
    dr[0, 0, 5] = -math.inf
    res = M.ResultBuffers(2, 2, 2)
    M.accept_chain_spd(z, tok, dr, torch.full_like(ua, 0.999), u, res)
    h = res.host()
    assert not h["status"].any() and int(h["eta"][0]) >= 1 and int(h["eta"][1]) == 0
    assert all(int(h["out_tok"][b, int(h["eta"][b])]) < 100 for b in range(2))


def test_accept_identical_rows_accept_everything():
    z, _, tok, u, ua, _ = rows_of(8, 6, 4, 2000, torch.bfloat16)
    res = M.ResultBuffers(6, 4, 4)
    M.accept_chain_spd(z, tok, z[:, :4].contiguous(), torch.full_like(ua, 1 - 2.0 ** -24), u, res)
    assert res.eta.tolist() == [4] * 6


def test_accept_flags_what_it_cannot_use():
    z, dr, tok, u, ua, logq = rows_of(9, 6, 2, 300, torch.float32)
    z[0, 1, 17] = float("nan")
    z[1, 0, 3] = float("inf")
    z[2, 2] = -math.inf
    tok[3, 0], tok[4, 1] = 300, -1
    res = M.ResultBuffers(6, 2, 2)
    res.buf.fill_(0)
    M.accept_chain_spd(z, tok, dr, ua, u, res, n_draft=torch.tensor([2, 2, 2, 2, 2, 3], dtype=torch.int32, device="cuda"))
    assert res.status.tolist() == [128, 128, 128, Bn.ST_BAD_TOKEN, Bn.ST_BAD_TOKEN, Bn.ST_BAD_COUNT]
    assert res.n_out.tolist() == [0] * 6 and not res.out_tok.any()


def test_accept_frequencies_of_the_first_token():
    """The rule's law: the first token out of it is distributed as the target's row, whatever the draft's."""
    V, n = 8, 40000
    g = torch.Generator(device="cuda").manual_seed(4)
    p = torch.randn(V, device="cuda", generator=g)
    q = torch.randn(V, device="cuda", generator=g)
    counts = torch.zeros(V)
    for s in range(10):
        B = n // 10
        take = lambda *d: torch.rand(*d, device="cuda", generator=g).clamp_(2.0 ** -24, 1 - 2.0 ** -24)  # noqa: E731
        tok = (q - take(B, 1, V).log().neg().log()).argmax(-1).int()
        res = M.ResultBuffers(B, 1, 1)
        M.accept_chain_spd(p.expand(B, 2, V).contiguous(), tok, q.expand(B, 1, V).contiguous(), take(B, 1), take(B, V), res)
        counts += torch.bincount(res.out_tok[:, 0].cpu().long(), minlength=V)
    want = torch.softmax(p, 0).cpu() * n
    chi2 = float(((counts - want) ** 2 / want).sum())
    assert chi2 < 29.9                                                    # 7 degrees of freedom, 1e-4


# ---------------------------------------------------------------------------------------------------------------

def test_a_run_of_them_together():
    """A decoder of the caller's own, one layer: rows enter the cache and attend to it with a plain form beside them, drafts are
    accepted, the lengths roll forward, and at the bound the cache is thinned and goes on with positions that are no longer slots."""
    torch.manual_seed(3)
    B, Hq, Hkv, hd, V, gamma, page, keep = 3, 8, 2, 64, 211, 3, 16, 48
    d = Hq * hd
    cap_pages = 8
    emb, lm = torch.randn(V, d, device="cuda") * 0.5, (torch.randn(V, d, device="cuda") * 0.05)
    wqkv = torch.randn((Hq + 2 * Hkv) * hd, d, device="cuda") * d ** -0.5
    pool = torch.zeros(B * cap_pages, 2, Hkv, page, hd, dtype=torch.bfloat16, device="cuda")
    table = torch.randperm(B * cap_pages, device="cuda").int().view(B, cap_pages)
    kp, vp = pool[:, 0], pool[:, 1]
    lens, pos = torch.zeros(B, dtype=torch.int32, device="cuda"), torch.zeros(B, dtype=torch.int32, device="cuda")
    weights = torch.zeros(B, Hkv, cap_pages * page, device="cuda")
    plain = [{"k": torch.zeros(Hkv, 0, hd, dtype=torch.bfloat16, device="cuda"), "v": torch.zeros(Hkv, 0, hd, dtype=torch.bfloat16, device="cuda"),
              "w": torch.zeros(Hkv, 0, device="cuda")} for _ in range(B)]
    root = torch.tensor([1, 2, 3], dtype=torch.int32, device="cuda")
    res = M.ResultBuffers(B, gamma, gamma)
    evicted = 0
    for step in range(40):
        tok = torch.randint(0, V, (B, gamma), device="cuda", dtype=torch.int32)
        ids = torch.cat([root[:, None], tok], 1).long()
        qkv = (emb[ids] @ wqkv.T).view(B, gamma + 1, Hq + 2 * Hkv, hd)
        q, k, v = qkv.split([Hq, Hkv, Hkv], 2)
        total = lens + gamma + 1
        q2 = M.paged_append(q, k, v, kp, vp, table, total, pos=pos, rope_base=10000.0)
        w_before = weights.clone()
        att = M.paged_attention(q2, kp, vp, table, total, weights=weights, max_len=cap_pages * page)
        for b in range(B):                                                # the plain form keeps its own cache
            at = torch.arange(gamma + 1, device="cuda").double()[:, None, None] + float(pos[b])
            ang = at * 10000.0 ** (-2.0 * torch.arange(hd // 2, dtype=torch.float64, device="cuda") / hd)

            def turned(t):
                x, y = t[..., :hd // 2].double(), t[..., hd // 2:].double()
                return torch.cat([x * ang.cos() - y * ang.sin(), y * ang.cos() + x * ang.sin()], -1)

            P = plain[b]
            P["k_all"] = torch.cat([P["k"], turned(k[b]).bfloat16().transpose(0, 1)], 1)
            P["v_all"] = torch.cat([P["v"], v[b].bfloat16().transpose(0, 1)], 1)
            n = P["k_all"].shape[1]
            assert n == int(total[b])
            s = torch.einsum("rhgd,hnd->hgrn", turned(q[b]).bfloat16().double().view(gamma + 1, Hkv, -1, hd), P["k_all"].double()) / math.sqrt(hd)
            see = torch.arange(n, device="cuda")[None] <= (n - gamma - 1 + torch.arange(gamma + 1, device="cuda"))[:, None]
            prob = torch.softmax(s.masked_fill(~see, -math.inf), -1)
            want = torch.einsum("hgrn,hnd->rhgd", prob, P["v_all"].double()).reshape(gamma + 1, Hq, hd)
            # keys and queries that round the other way (half a step each, of values up to ~6, in 64 products) move a score by up to 2e-2
            assert float((att[b].double() - want).abs().max()) < 0.1
            got_w = weights[b, :, :n].double() - w_before[b, :, :n].double()
            assert float((got_w - prob.sum((1, 2))).abs().max()) < 0.1
        logits = att.float().view(B, gamma + 1, d) @ lm.T
        logq = torch.full((B, gamma), -5.0, device="cuda") * torch.arange(1, gamma + 1, device="cuda")
        M.accept_chain(logits.contiguous(), tok, logq, math.log(0.5), torch.rand(B, V, device="cuda").clamp_(1e-6, 1 - 1e-6), res)
        assert not res.status.any()
        n_out = res.n_out.clone()
        root = res.out_tok.gather(1, res.eta.long()[:, None])[:, 0].contiguous()
        for b in range(B):
            n = int(lens[b] + n_out[b])
            P = plain[b]
            P["k"], P["v"] = P["k_all"][:, :n], P["v_all"][:, :n]
            weights[b, :, n:] = 0                                         # rows that were not accepted leave no weight
        lens, pos = lens + n_out, pos + n_out
        if int(lens.max()) > 60:
            old = lens
            kept, lens = M.paged_evict(kp, vp, table, old, weights, keep, first=2, recent=16, scores_out=weights)
            evicted += 1
            for b in range(B):
                m = int(lens[b])
                idx = kept[b, :, :m].long()
                weights[b, :, m:] = 0
                P = plain[b]
                P["k"] = P["k"].gather(1, idx[..., None].expand(-1, -1, hd))
                P["v"] = P["v"].gather(1, idx[..., None].expand(-1, -1, hd))
    assert evicted >= 2


def test_calls_captured_behind_copies_and_joined_streams():
    """A captured call right behind a copy, a fill and a second stream that joins: the graph's replay gives the eager call's results."""
    c = Cache(40, [500, 90], 2, 64, 16)
    q = queries(40, 2, 1, 4, 64, torch.bfloat16)
    src, other = q.clone(), torch.zeros(1 << 20, device="cuda")
    want = M.paged_attention(q, *c.args(), c.lens, max_len=500)
    z, dr, tok, u, ua, logq = rows_of(41, 2, 3, 700, torch.float32)
    res, eager = M.ResultBuffers(2, 3, 3), M.ResultBuffers(2, 3, 3)
    M.accept_chain_spd(z, tok, dr, ua, u, eager)
    scores = torch.rand(2, 2, 500, device="cuda")
    kept0, new0 = M.paged_evict(*c.args(), c.lens, scores, 100, recent=10)
    c = Cache(40, [500, 90], 2, 64, 16)
    main, side = torch.cuda.Stream(), torch.cuda.Stream()
    main.wait_stream(torch.cuda.current_stream())
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=main):
        q.copy_(src)
        side.wait_stream(main)
        with torch.cuda.stream(side):
            other.add_(1)
        main.wait_stream(side)
        out = M.paged_attention(q, *c.args(), c.lens, max_len=500)
        res.buf.zero_()
        M.accept_chain_spd(z, tok, dr, ua, u, res)
        M.paged_append(None, c.k[c.table[:, :1].long()][:, :, :, 0], c.v[c.table[:, :1].long()][:, :, :, 0], *c.args(), torch.ones_like(c.lens))
        kept, new = M.paged_evict(*c.args(), c.lens, scores, 100, recent=10)
    q.zero_()
    for _ in range(2):
        g.replay()
    torch.cuda.synchronize()
    assert torch.equal(res.buf, eager.buf) and torch.equal(kept, kept0) and torch.equal(new, new0)
    g.replay()
    torch.cuda.synchronize()
    c2 = Cache(40, [500, 90], 2, 64, 16)
    assert torch.equal(M.paged_attention(q, *c2.args(), c2.lens, max_len=500), want) and out.shape == want.shape


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("kind", ["peak", "far", "masked_first", "masked_most", "huge", "tiny"])
def test_accept_rows_of_every_range(dtype, kind):
    """The first tokens of a row say nothing about the rest: one logit far above all, all far above or below the first ones, rows that begin
    with masked tokens or hold little else."""
    B, D, V = 3, 2, 5000
    z, dr, tok, u, ua, logq = rows_of(11, B, D, V, torch.float32)
    top = 3e4 if dtype == "fp16" else 1e6
    for x in (z, dr):
        if kind == "peak":
            x[:, :, 3333] = 200.0
        elif kind == "far":
            x[:, :, 1000:] += 300.0
        elif kind == "masked_first":
            x[:, :, :4096] = -math.inf
        elif kind == "masked_most":
            x[:, :, 40:4990] = -math.inf
        elif kind == "huge":
            x += top
        else:
            x -= top
    z, dr = z.to(DT[dtype]), dr.to(DT[dtype])
    tok[:] = torch.tensor([[4995, 4996], [4997, 4998], [4991, 4999]], dtype=torch.int32)
    logq = dr.double().log_softmax(-1).gather(2, tok.long()[..., None])[..., 0].cumsum(-1).float()
    check = dict(compare=kind not in ("peak", "huge", "tiny"))            # (margins within the error of such logits decide nothing)
    check_accept("spd", z, tok, u, dr, ua, **check)
    check_accept("mtad", z, tok, u, logq=logq, **check)


def test_views_whose_single_dimensions_have_odd_strides():
    c = Cache(42, [70], 2, 64, 16)
    q = queries(42, 1, 1, 4, 64, torch.bfloat16)
    want = M.paged_attention(q, *c.args(), c.lens)
    odd = q.as_strided(q.shape, (3, 5, 64, 1))
    assert torch.equal(M.paged_attention(odd, *c.args(), c.lens), want)


def test_calls_from_two_threads_on_two_streams():
    """Append (with another rotary base in each thread), attention, eviction and acceptance side by side, each as when alone."""
    import threading

    def work(k, stream, out):
        with torch.cuda.stream(stream):
            c = Cache(50 + k, [3000, 700], 2, 64, 16)
            x = torch.randn(2, 4, 8, 64, device="cuda", generator=torch.Generator(device="cuda").manual_seed(k)).bfloat16()
            q, kk, v = x.split([4, 2, 2], 2)
            z, dr, tok, u, ua, _ = rows_of(60 + k, 2, 3, 900, torch.float32)
            s = torch.rand(2, 2, 3000, device="cuda", generator=torch.Generator(device="cuda").manual_seed(k))
            got = []
            for _ in range(20):
                q2 = M.paged_append(q, kk, v, *c.args(), c.lens, rope_base=10000.0 * (k + 1))
                att = M.paged_attention(q2, *c.args(), c.lens, max_len=3000)
                res = M.ResultBuffers(2, 3, 3)
                M.accept_chain_spd(z, tok, dr, ua, u, res)
                got = [q2, att, res.buf]
            kept, _ = M.paged_evict(*c.args(), c.lens, s, 500, recent=50)
            out[k] = [*got, kept, c.pool]
        stream.synchronize()

    alone, both = {}, {}
    for k in range(2):
        work(k, torch.cuda.Stream(), alone)
    threads = [threading.Thread(target=work, args=(k, torch.cuda.Stream(), both)) for k in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    for k in range(2):
        for a, b in zip(alone[k], both[k]):
            assert torch.equal(a.contiguous().view(torch.uint8), b.contiguous().view(torch.uint8))


@pytest.mark.parametrize("batch,hq,hkv,rows,page,window,hd", [(300, 1, 1, 1, 16, 0, 64), (300, 2, 1, 5, 5, 0, 64), (70, 32, 8, 1, 16, 1000, 64),
                                                              (300, 20, 1, 1, 16, 0, 64), (100, 12, 2, 4, 24, 900, 128), (40, 8, 8, 2, 64, 0, 256)])
def test_attention_many_sequences_over_a_cut_list(batch, hq, hkv, rows, page, window, hd):
    """More sequences than a warp has lanes, some empty, some long: the list of tiles is found by more than one sequence a lane, with a window
    too, for few and many query rows a head, on even and uneven pages."""
    g = torch.Generator().manual_seed(batch + hq)
    lens = [int(n) for n in torch.randint(0, 2000, (batch,), generator=g)]
    lens[0], lens[1], lens[-1] = 0, 1999, 0
    lens[5:9] = [0, 1, 16, 17]
    c = Cache(70, lens, hkv, hd, page)
    check_attention(c, queries(70, batch, rows, hq, hd, torch.bfloat16), window=window, sinks=3 if window else 0)


def test_attention_as_many_rows_as_a_call_takes():
    """256 rows of a prompt chunk on grouped heads: 32 blocks of query rows a KV head."""
    c = Cache(71, [300, 256, 100], 1, 64, 16)
    check_attention(c, queries(71, 3, 256, 8, 64, torch.bfloat16), n_rows=[256, 256, 77])


@pytest.mark.parametrize("in_place", [False, True])
def test_evict_by_a_cluster_a_head(in_place):
    c = Cache(72, [40000, 39000], 1, 8, 64)
    s = torch.rand(2, 1, 40000, device="cuda", generator=torch.Generator(device="cuda").manual_seed(2)).mul(50).round()      # many equal scores
    check_evict(c, s, 12345, 5, 1000, in_place)


def test_launches_are_counted():
    c = Cache(73, [20], 1, 64, 16)
    n = M.mtad_kernel_launches()
    M.paged_attention(queries(73, 1, 1, 1, 64, torch.bfloat16), *c.args(), c.lens)
    assert M.mtad_kernel_launches() == n + 1
