// What moves keys and values of a cache kept in pages: rows that enter it (with the rotary embedding), and eviction.
#include <cooperative_groups.h>
#include <math.h>
#include <math_constants.h>

#include <algorithm>
#include <type_traits>

#include "paged.cuh"

namespace cg = cooperative_groups;

namespace mtad {

namespace {

// ---------------------------------------------------------------------------------------------------------------
// Append.  Row r of sequence b goes to slot length - rows + r; its keys and queries are turned by the angle position *
// base^(-2i/hd) in the pairs (i, i + hd/2):  a' = a cos - b sin,  b' = b cos + a sin.
// One pass over the rows, bound by their bytes (and by latency for a few rows).  A block takes a row, or a share of its heads
// where rows are few: the angles' sines and cosines are formed once per block (reduced in 64 bits, see rope_cs) and serve all its heads.

constexpr int AP_THREADS = 256;

struct RopeTable {
    double v[MTAD_PAGED_MAX_HEAD_DIM / 2];
};
struct AppendArgs {
    PagedView kv;
    const int32_t *lens, *n_rows, *pos;
    const void *q, *k, *v;
    uint16_t* q_out;
    long long q_sb, q_sr, q_sh, k_sb, k_sr, k_sh, o_sb, o_sr, o_sh;
    uint32_t* status;
    int R, Hq, shares, rope;
    long long cap;                   // slots of a sequence
    FastDiv nv, nv2;                 // vectors of half a head, of a head
};

// V elements from memory of type Src to fp32
template <typename Src, int V>
__device__ __forceinline__ void load_vec(const Src* p, float (&x)[V]) {
    if constexpr (sizeof(Src) == 4) {
#pragma unroll
        for (int i = 0; i < V; i += 4) {
            const float4 w = *reinterpret_cast<const float4*>(p + i);
            x[i] = w.x; x[i + 1] = w.y; x[i + 2] = w.z; x[i + 3] = w.w;
        }
    } else {
        uint32_t w[V / 2];
        if constexpr (V == 8) {
            const uint4 u = *reinterpret_cast<const uint4*>(p);
            w[0] = u.x; w[1] = u.y; w[2] = u.z; w[3] = u.w;
        } else {
            const uint2 u = *reinterpret_cast<const uint2*>(p);
            w[0] = u.x; w[1] = u.y;
        }
#pragma unroll
        for (int i = 0; i < V / 2; ++i) {
            const float2 f = Num<Src>::unpack(w[i]);
            x[2 * i] = f.x; x[2 * i + 1] = f.y;
        }
    }
}
template <typename T, int V>
__device__ __forceinline__ void store_vec(uint16_t* p, const float (&x)[V]) {
    uint32_t w[V / 2];
#pragma unroll
    for (int i = 0; i < V / 2; ++i) w[i] = Num<T>::pack(x[2 * i], x[2 * i + 1]);
    if constexpr (V == 8) *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
    else *reinterpret_cast<uint2*>(p) = make_uint2(w[0], w[1]);
}

template <typename Src, typename T, int V>
__global__ void __launch_bounds__(AP_THREADS) append_kernel(const AppendArgs a, const __grid_constant__ RopeTable rope) {
    const int row = blockIdx.x, b = row / a.R, r = row - b * a.R, share = blockIdx.y, tid = threadIdx.x;
    const int half = a.kv.hd >> 1;
    __shared__ float s_cos[MTAD_PAGED_MAX_HEAD_DIM / 2], s_sin[MTAD_PAGED_MAX_HEAD_DIM / 2];
    __shared__ long long s_off;
    pdl_wait();
    pdl_trigger();
    const int len = __ldg(a.lens + b), nb = a.n_rows ? min(max(__ldg(a.n_rows + b), 0), a.R) : a.R;
    if (r >= nb) return;
    const long long slot = (long long)len - nb + r;
    if (a.rope) {
        const int pos = a.pos ? __ldg(a.pos + b) + r : (int)slot;
        for (int i = tid; i < half; i += AP_THREADS) rope_cs((double)pos, rope.v[i], s_cos[i], s_sin[i]);
    }
    if (tid == 0) {
        long long off = -1;
        uint32_t bits = 0;
        if (slot < 0 || slot >= a.cap) bits = MTAD_ST_KV_OVERFLOW;
        else if ((off = slot_offset(a.kv, a.kv.table + (long long)b * a.kv.table_stride, (int)slot)) < 0) bits = MTAD_ST_RANGE;
        if (bits && a.status) atomicOr(a.status + b, bits);
        s_off = off;
    }
    __syncthreads();
    const long long off = s_off;
    const Src* q = static_cast<const Src*>(a.q) + (long long)b * a.q_sb + (long long)r * a.q_sr;
    const Src* k = static_cast<const Src*>(a.k) + (long long)b * a.k_sb + (long long)r * a.k_sr;
    const Src* v = static_cast<const Src*>(a.v) + (long long)b * a.k_sb + (long long)r * a.k_sr;
    uint16_t* qo = a.q_out + (long long)b * a.o_sb + (long long)r * a.o_sr;
    const int turn = (a.Hq + a.kv.Hkv) * (int)a.nv.d, all = turn + a.kv.Hkv * (int)a.nv2.d;
#pragma unroll 2
    for (int i = share * AP_THREADS + tid; i < all; i += a.shares * AP_THREADS) {
        if (i < turn) {
            const int h = (int)div_by(i, a.nv), c = (i - h * (int)a.nv.d) * V;
            const bool is_q = h < a.Hq;
            const Src* src = is_q ? q + (long long)h * a.q_sh : k + (long long)(h - a.Hq) * a.k_sh;
            if (!is_q && off < 0) continue;
            uint16_t* dst = is_q ? qo + (long long)h * a.o_sh : a.kv.k + off + (long long)(h - a.Hq) * a.kv.head_stride;
            float x[V], y[V];
            load_vec<Src, V>(src + c, x);
            load_vec<Src, V>(src + half + c, y);
            if (a.rope) {
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    const float cs = s_cos[c + e], sn = s_sin[c + e], u = x[e], w = y[e];
                    x[e] = u * cs - w * sn;
                    y[e] = w * cs + u * sn;
                }
            }
            store_vec<T, V>(dst + c, x);
            store_vec<T, V>(dst + half + c, y);
        } else if (off >= 0) {
            const int j = i - turn, h = (int)div_by(j, a.nv2), c = (j - h * (int)a.nv2.d) * V;
            float x[V];
            load_vec<Src, V>(v + (long long)h * a.k_sh + c, x);
            store_vec<T, V>(a.kv.v + off + (long long)h * a.kv.head_stride + c, x);
        }
    }
}

template <typename Src, typename T>
cudaError_t launch_append(const AppendArgs& a, const RopeTable& rope, int B, cudaStream_t st) {
    const dim3 grid(B * a.R, a.shares);
    mtad_ops_count(1);
    return a.kv.hd % 16 == 0 ? launch_pdl(append_kernel<Src, T, 8>, grid, dim3(AP_THREADS), 0, st, true, a, rope)
                             : launch_pdl(append_kernel<Src, T, 4>, grid, dim3(AP_THREADS), 0, st, true, a, rope);
}

// ---------------------------------------------------------------------------------------------------------------
// Eviction.  Of the `len` slots of a KV head the first `first`, the last `recent` and the largest scores stay, `keep` in all (lowest slot
// first among equals), in the order of their slots; they move together to the front.  Two launches:
//
// Selection, a cluster of one to eight blocks per KV head, as many as leave every SM one: each block holds its part of the scores in shared
// memory; the keep-th largest is found by a radix descent over the ordered bits in which they differ (11 at a time), the histograms of a
// cluster added up through distributed shared memory; one exchange of counts gives every block the place of its first kept slot.
//
// Moving.  The blocks of a head divide keys and values and the columns of a row, not the rows.  So a block walks its columns from the
// front with no one else in its way: destination j lies at or before source kept[j], and what a later round reads lies behind
// everything that earlier rounds wrote; only the reads of one round have to be over before its writes.  Bound by the bytes of what moves,
// and by DRAM being read in pieces: whole rows of 256 bytes move 16 long contexts in 211 us, halves in 220, quarters 252, eighths 350 (and
// clusters whose blocks take turns at the rows of a head, waiting for one another every round, in 236).
// (One launch for both kept the blocks that move waiting in a selection that uses no bandwidth: 418 us for 16 long contexts, 36 for one.)

constexpr int EV_THREADS = 1024, EV_BINS = 2048, EV_MAX_CLUSTER = 8;
constexpr int EV_STAGE = 40 * 1024;  // scores that a block holds; more are read again from memory

struct EvictArgs {
    PagedView kv;
    const int32_t* lens;
    const float* scores;
    long long s_sb, s_sh;
    int32_t* kept;                   // [B][Hkv][keep]
    int32_t* new_lens;               // [B]
    float* scores_out;               // or null
    long long o_sb, o_sh;
    uint32_t* status;
    int keep, first, recent, max_len, staged, cluster;
};

// Order-preserving bits: larger score, larger key; -0 as +0; every NaN above all numbers.
__device__ __forceinline__ uint32_t score_key(float x) {
    if (x != x) return 0xffffffffu;
    const uint32_t u = __float_as_uint(x + 0.f);
    return (u & 0x80000000u) ? ~u : u | 0x80000000u;
}

__device__ __forceinline__ float key_score(uint32_t k) {
    return k == 0xffffffffu ? CUDART_NAN_F : __uint_as_float((k & 0x80000000u) ? k & 0x7fffffffu : ~k);
}

__global__ void __launch_bounds__(EV_THREADS) select_kernel(const EvictArgs a) {
    extern __shared__ __align__(16) uint32_t s_key[];
    __shared__ __align__(16) uint32_t hist[3][EV_BINS];
    __shared__ int s_warp[EV_THREADS / 32], s_weq[EV_THREADS / 32];
    __shared__ int s_above, s_bin;
    __shared__ int s_gt, s_eq;                            // these and the histograms are read by the cluster
    __shared__ uint32_t s_lo, s_hi;
    cg::cluster_group cluster = cg::this_cluster();
    const int CS = a.cluster, rank = CS > 1 ? (int)cluster.block_rank() : 0, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    auto sync = [&]() { if (CS > 1) cluster.sync(); else __syncthreads(); };
    pdl_wait();
    pdl_trigger();
    const int bh = blockIdx.x / CS, b = bh / a.kv.Hkv, h = bh - b * a.kv.Hkv;
    const int raw = __ldg(a.lens + b), n = min(max(raw, 0), a.max_len);
    const float* z = a.scores + (long long)b * a.s_sb + (long long)h * a.s_sh;
    int32_t* kept = a.kept + (long long)bh * a.keep;
    float* zo = a.scores_out ? a.scores_out + (long long)b * a.o_sb + (long long)h * a.o_sh : nullptr;
    if (rank == 0 && h == 0 && tid == 0) {
        if (raw != n && a.status) atomicOr(a.status + b, MTAD_ST_KV_OVERFLOW);
        a.new_lens[b] = min(n, a.keep);
    }
    if (n <= a.keep) {                                    // nothing to evict (the same for the whole cluster)
        for (int j = rank * EV_THREADS + tid; j < a.keep; j += CS * EV_THREADS) {
            kept[j] = j < n ? j : -1;
            if (zo && j < n && zo != z) zo[j] = z[j];
        }
        return;
    }
    const int chunk = ((n + CS - 1) / CS + 3) & ~3, c0 = min(rank * chunk, n), mine = min(chunk, n - c0);
    // of this block's scores, those that may go: slots outside [first, n - recent) stay whatever their score
    const int i_lo = min(max(a.first - c0, 0), mine), i_hi = max(min(n - a.recent - c0, mine), i_lo);
    for (int i = tid; i < 3 * EV_BINS / 4; i += EV_THREADS) reinterpret_cast<uint4*>(&hist[0][0])[i] = make_uint4(0u, 0u, 0u, 0u);
    if (tid == 0) { s_lo = 0xffffffffu; s_hi = 0; }
    __syncthreads();
    // four neighbouring keys (of slots beyond the block's last: anything); keys(i, n): the element i * 4 + e is one that may go
    auto four = [&](int i) -> uint4 {
        if (a.staged) return reinterpret_cast<const uint4*>(s_key)[i];
        uint32_t k[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) k[e] = i * 4 + e < mine ? score_key(__ldg(z + c0 + i * 4 + e)) : 0;
        return make_uint4(k[0], k[1], k[2], k[3]);
    };
    uint32_t k_lo = 0xffffffffu, k_hi = 0;                // smallest and largest key of those that may go
    {
        // eight requests of a thread in flight, of 16 bytes where the row begins on such a boundary
        auto meet = [&](int i, const float4& w) {
            const uint4 k = make_uint4(score_key(w.x), score_key(w.y), score_key(w.z), score_key(w.w));
            if (i * 4 >= i_lo && i * 4 + 4 <= i_hi) {
                k_lo = min(k_lo, min(min(k.x, k.y), min(k.z, k.w)));
                k_hi = max(k_hi, max(max(k.x, k.y), max(k.z, k.w)));
            } else {
                const uint32_t key[4] = {k.x, k.y, k.z, k.w};
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (i * 4 + e >= i_lo && i * 4 + e < i_hi) { k_lo = min(k_lo, key[e]); k_hi = max(k_hi, key[e]); }
            }
            if (a.staged) reinterpret_cast<uint4*>(s_key)[i] = k;
        };
        const float* from = z + c0;
        const int nv = (reinterpret_cast<uintptr_t>(from) & 15) == 0 ? mine / 4 : 0;
        for (int i0 = tid; i0 < nv; i0 += 8 * EV_THREADS) {
            float4 w[8];
#pragma unroll
            for (int u = 0; u < 8; ++u)
                if (i0 + u * EV_THREADS < nv) w[u] = __ldg(reinterpret_cast<const float4*>(from) + i0 + u * EV_THREADS);
#pragma unroll
            for (int u = 0; u < 8; ++u)
                if (i0 + u * EV_THREADS < nv) meet(i0 + u * EV_THREADS, w[u]);
        }
        for (int i0 = nv + tid; i0 * 4 < mine; i0 += 2 * EV_THREADS) {
            float4 w[2];
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const int i = (i0 + u * EV_THREADS) * 4;
                w[u].x = i < mine ? __ldg(from + i) : 0.f;
                w[u].y = i + 1 < mine ? __ldg(from + i + 1) : 0.f;
                w[u].z = i + 2 < mine ? __ldg(from + i + 2) : 0.f;
                w[u].w = i + 3 < mine ? __ldg(from + i + 3) : 0.f;
            }
#pragma unroll
            for (int u = 0; u < 2; ++u)
                if ((i0 + u * EV_THREADS) * 4 < mine) meet(i0 + u * EV_THREADS, w[u]);
        }
    }
    k_lo = __reduce_min_sync(0xffffffffu, k_lo);
    k_hi = __reduce_max_sync(0xffffffffu, k_hi);
    if (lane == 0) { atomicMin(&s_lo, k_lo); atomicMax(&s_hi, k_hi); }
    sync();
    k_lo = s_lo;
    k_hi = s_hi;
    if (CS > 1)
        for (int k = 0; k < CS; ++k) { k_lo = min(k_lo, *cluster.map_shared_rank(&s_lo, k)); k_hi = max(k_hi, *cluster.map_shared_rank(&s_hi, k)); }

    // ---- the key of the last slot that stays: bins over the keys' own range (of scores of a few magnitudes, most bits that they have in
    // common would fall into a few bins of a fixed split, and their counters be fought for)
    int need = a.keep - a.first - a.recent;               // slots still to be found among those with this prefix
    const bool some = need > 0;
    uint32_t border = 0;                                  // key - k_lo of that slot, down to bit `shift`
    int shift = 32 - __clz(k_hi - k_lo);
#pragma unroll 1
    for (int pass = 0; some && shift > 0; ++pass) {
        const int from = shift, bits = min(shift, 11);
        shift -= bits;
        const uint32_t mask = (1u << bits) - 1, least = k_lo + border, width = from == 32 ? 0xffffffffu : (1u << from) - 1;
        auto count = [&](uint32_t key) {                  // (keys with the prefix: least .. least + width)
            const uint32_t d = key - least;
            if (d <= width) atomicAdd(&hist[pass][(d >> shift) & mask], 1u);
        };
#pragma unroll 2
        for (int i = (i_lo >> 2) + tid; i * 4 < i_hi; i += EV_THREADS) {
            const uint4 k = four(i);
            if (i * 4 >= i_lo && i * 4 + 4 <= i_hi) {
                count(k.x); count(k.y); count(k.z); count(k.w);
            } else {
                if (i * 4 >= i_lo && i * 4 < i_hi) count(k.x);
                if (i * 4 + 1 >= i_lo && i * 4 + 1 < i_hi) count(k.y);
                if (i * 4 + 2 >= i_lo && i * 4 + 2 < i_hi) count(k.z);
                if (i * 4 + 3 >= i_lo && i * 4 + 3 < i_hi) count(k.w);
            }
        }
        sync();
        // bins from the top: thread t has the two below 2048 - 2 t
        const int bin0 = EV_BINS - 2 * (tid + 1);
        uint2 sum = *reinterpret_cast<const uint2*>(&hist[pass][bin0]);
        if (CS > 1) {
            sum = make_uint2(0u, 0u);
            for (int k = 0; k < CS; ++k) {
                const uint2 x = *reinterpret_cast<const uint2*>(cluster.map_shared_rank(&hist[pass][bin0], k));
                sum.x += x.x; sum.y += x.y;
            }
        }
        const int total = (int)(sum.x + sum.y);
        int incl = total;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int x = __shfl_up_sync(0xffffffffu, incl, o);
            if (lane >= o) incl += x;
        }
        if (lane == 31) s_warp[warp] = incl;
        __syncthreads();
        const int w = s_warp[lane];                       // (32 warps)
        const int before = incl - total + __reduce_add_sync(0xffffffffu, lane < warp ? w : 0);
        if (before < need && need <= before + total) {
            const bool upper = need <= before + (int)sum.y;
            s_bin = bin0 + (upper ? 1 : 0);
            s_above = before + (upper ? 0 : (int)sum.y);
        }
        __syncthreads();
        border |= (uint32_t)s_bin << shift;
        need -= s_above;
    }
    border += k_lo;
    // ---- places: a warp has a run of neighbouring slots
    const int run = (mine + 128 * (EV_THREADS / 32) - 1) / (128 * (EV_THREADS / 32)) * 128, r0 = min(warp * run, mine), r1 = min(r0 + run, mine);
    const int g0 = max(r0, i_lo), g1 = min(r1, i_hi);     // those of them that may go
    int gt = 0, eq = 0;                                   // that stay for certain, that lie on the border
    if (some) {
#pragma unroll 2
        for (int i = (g0 >> 2) + lane; i * 4 < g1; i += 32) {
            const uint4 k = four(i);
            const uint32_t key[4] = {k.x, k.y, k.z, k.w};
            const bool whole = i * 4 >= g0 && i * 4 + 4 <= g1;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const bool in = whole || (i * 4 + e >= g0 && i * 4 + e < g1);
                gt += in && key[e] > border;
                eq += in && key[e] == border;
            }
        }
        gt = __reduce_add_sync(0xffffffffu, gt);
        eq = __reduce_add_sync(0xffffffffu, eq);
    }
    gt += (r1 - r0) - max(g1 - g0, 0);
    __syncthreads();                                      // (the last pass's counts are no longer read)
    if (lane == 0) { s_warp[warp] = gt; s_weq[warp] = eq; }
    __syncthreads();
    int before_g, before_e;
    {
        const int w = s_warp[lane], e = s_weq[lane];
        before_g = __reduce_add_sync(0xffffffffu, lane < warp ? w : 0);
        before_e = __reduce_add_sync(0xffffffffu, lane < warp ? e : 0);
        if (CS > 1) {
            const int all_g = __reduce_add_sync(0xffffffffu, w), all_e = __reduce_add_sync(0xffffffffu, e);
            if (tid == 0) { s_gt = all_g; s_eq = all_e; }
            cluster.sync();
            for (int k = 0; k < rank; ++k) { before_g += *cluster.map_shared_rank(&s_gt, k); before_e += *cluster.map_shared_rank(&s_eq, k); }
        }
    }
    auto put = [&](uint32_t at, int i, uint32_t key) {
        kept[at] = c0 + i;
        if (zo) {
            float x = key_score(key);
            // (what the key does not hold, a zero's sign and a NaN's bits, is read again; in place it may be overwritten by now)
            if (key - 0x80000000u == 0u || key == 0xffffffffu) x = zo != z ? z[c0 + i] : x;
            zo[at] = x;
        }
    };
    for (int i = r0 + lane * 4; i - lane * 4 < r1; i += 128) {
        const uint4 k = i < r1 ? four(i >> 2) : make_uint4(0u, 0u, 0u, 0u);
        const uint32_t key[4] = {k.x, k.y, k.z, k.w};
        uint32_t sure = 0, edge = 0;                      // of the lane's four, a bit each
        if (i >= g0 && i + 4 <= g1) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                sure |= key[e] > border ? 1u << e : 0u;
                edge |= key[e] == border ? 1u << e : 0u;
            }
            if (!some) sure = edge = 0;
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const bool may = i + e >= i_lo && i + e < i_hi;
                if (i + e < r1 && (!may || (some && key[e] > border))) sure |= 1u << e;
                if (i + e < r1 && may && some && key[e] == border) edge |= 1u << e;
            }
        }
        const int own = __popc(sure) | __popc(edge) << 16;
        int incl = own;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int x = __shfl_up_sync(0xffffffffu, incl, o);
            if (lane >= o) incl += x;
        }
        const int all = __shfl_sync(0xffffffffu, incl, 31);
        int g = before_g + ((incl - own) & 0xffff), eb = before_e + ((incl - own) >> 16);
        if (all >> 16 == 0) {                             // nothing on the border: those that stay follow one another
            uint32_t at = g + min(eb, need);
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (sure >> e & 1) put(at++, i + e, key[e]);
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const bool is_sure = sure >> e & 1, is_edge = edge >> e & 1;
                if (is_sure || (is_edge && eb < need)) put(g + min(eb, need), i + e, key[e]);          // of those on the border the first `need` stay
                g += is_sure;
                eb += is_edge;
            }
        }
        before_g += all & 0xffff;
        before_e += all >> 16;
    }
    if (CS > 1) cluster.sync();                           // (no block leaves while another reads its shared memory)
}

// A thread moves MV_UNROLL pieces of 16 bytes a round; offsets of a round's rows are worked out once per block, while the round before is in flight.
constexpr int MV_THREADS = 512, MV_UNROLL = 8;
constexpr int MV_SMEM = 3 * MV_THREADS * MV_UNROLL * (int)sizeof(longlong2);          // with parts of one piece
__global__ void __launch_bounds__(MV_THREADS, 2) move_kernel(const EvictArgs a, int slices) {
    extern __shared__ longlong2 s_off[];                  // [3][rows of a round] element offsets of source and destination, -1: not moved
    const int part = blockIdx.x % slices, bh = blockIdx.x / slices, b = bh / a.kv.Hkv, h = bh - b * a.kv.Hkv, tid = threadIdx.x;
    pdl_wait();
    const int n = min(max(__ldg(a.lens + b), 0), a.max_len);
    if (n <= a.keep) return;
    const int half = slices >> 1, chunks = a.kv.hd >> 3, q = part % half, col0 = q * chunks / half, cols = (q + 1) * chunks / half - col0;
    if (cols == 0) return;
    const int32_t* kept = a.kept + (long long)bh * a.keep;
    const int32_t* row = a.kv.table + (long long)b * a.kv.table_stride;
    uint16_t* base = (part >= half ? a.kv.v : a.kv.k) + (long long)h * a.kv.head_stride;
    const int rows = MV_THREADS / cols, round = rows * MV_UNROLL, rr = tid / cols, cc = (col0 + tid - rr * cols) * 8;
    const bool on = rr < rows;
    bool bad = false;
    auto work_out = [&](int j0, longlong2* to) {
        for (int i = tid; i < round; i += MV_THREADS) {
            const int j = j0 + i, src = j < a.keep ? __ldg(kept + j) : -1;
            longlong2 x = make_longlong2(-1, -1);
            if (src > j) {                                // (the first ones stay where they are)
                x.x = slot_offset(a.kv, row, src);
                x.y = slot_offset(a.kv, row, j);
                if (x.x < 0 || x.y < 0) { bad = true; x.x = -1; }
            }
            to[i] = x;
        }
    };
    work_out(0, s_off);
    __syncthreads();
    int at = 0;
    for (int j0 = 0; j0 < a.keep; j0 += round) {
        const longlong2* off = s_off + at * round + rr;
        uint4 w[MV_UNROLL];
#pragma unroll
        for (int u = 0; u < MV_UNROLL; ++u) {
            const long long so = on ? off[u * rows].x : -1;
            if (so >= 0) w[u] = *reinterpret_cast<const uint4*>(base + so + cc);
        }
        at = at == 2 ? 0 : at + 1;
        if (j0 + round < a.keep) work_out(j0 + round, s_off + at * round);
        __syncthreads();                                  // the round's reads are over, the next offsets are there
#pragma unroll
        for (int u = 0; u < MV_UNROLL; ++u) {
            const longlong2 x = on ? off[u * rows] : make_longlong2(-1, -1);
            if (x.x >= 0) *reinterpret_cast<uint4*>(base + x.y + cc) = w[u];
        }
    }
    if (bad && a.status) atomicOr(a.status + b, MTAD_ST_RANGE);
}

}  // namespace

}  // namespace mtad

using namespace mtad;

extern "C" {

int mtad_paged_append(const mtad_paged_kv* kv, const mtad_paged_rows* c, void* stream) {
    AppendArgs a{};
    if (!c) return MTAD_E_INVALID;
    const int rc = paged_view(kv, &a.kv);
    if (rc != MTAD_OK) return rc;
    if (!c->lens || !c->k || !c->v || c->batch < 1 || c->rows < 1 || c->n_q_heads < 0) return MTAD_E_INVALID;
    if (c->n_q_heads > 0 && (!c->q || !c->q_out)) return MTAD_E_INVALID;
    if (c->dtype != kv->dtype && c->dtype != MTAD_F32) return MTAD_E_INVALID;
    if (!isfinite(c->rope_base) || (c->rope_base != 0.f && c->rope_base < 1.f)) return MTAD_E_INVALID;
    if (c->batch > MTAD_PAGED_MAX_BATCH || c->rows > MTAD_MAX_NODES + 1 || c->n_q_heads > MTAD_PAGED_MAX_HEADS) return MTAD_E_CAPACITY;
    if ((reinterpret_cast<uintptr_t>(c->q) | reinterpret_cast<uintptr_t>(c->k) | reinterpret_cast<uintptr_t>(c->v) |
         reinterpret_cast<uintptr_t>(c->q_out)) & 15) return MTAD_E_INVALID;
    const int64_t in[6] = {c->q_stride_seq, c->q_stride_row, c->q_stride_head, c->kv_stride_seq, c->kv_stride_row, c->kv_stride_head};
    const int64_t outs[3] = {c->out_stride_seq, c->out_stride_row, c->out_stride_head};
    for (int i = 0; i < 6; ++i)
        if (in[i] < 0 || in[i] % (c->dtype == MTAD_F32 ? 4 : 8)) return MTAD_E_INVALID;
    for (int i = 0; i < 3; ++i)
        if (outs[i] < 0 || outs[i] % 8) return MTAD_E_INVALID;
    if (!pages_lie_apart(kv) || !lie_apart(kv->head_dim, {{c->batch, outs[0]}, {c->rows, outs[1]}, {c->n_q_heads, outs[2]}})) return MTAD_E_INVALID;
    a.lens = c->lens; a.n_rows = c->n_rows; a.pos = c->pos;
    a.q = c->q; a.k = c->k; a.v = c->v; a.q_out = static_cast<uint16_t*>(c->q_out);
    a.q_sb = in[0]; a.q_sr = in[1]; a.q_sh = in[2]; a.k_sb = in[3]; a.k_sr = in[4]; a.k_sh = in[5];
    a.o_sb = outs[0]; a.o_sr = outs[1]; a.o_sh = outs[2];
    a.status = c->status;
    a.R = c->rows; a.Hq = c->n_q_heads; a.rope = c->rope_base > 0.f;
    a.cap = (long long)kv->max_pages * kv->page_size;
    const int V = kv->head_dim % 16 == 0 ? 8 : 4, half = kv->head_dim / 2;
    a.nv = fast_div((uint32_t)(half / V));
    a.nv2 = fast_div((uint32_t)(kv->head_dim / V));
    // (frequencies of this thread's last base and head size: a hundred exponentials would take as long as the launch)
    static thread_local struct { float base; int hd; RopeTable t; } rope{0.f, 0, {}};
    if (a.rope && (rope.base != c->rope_base || rope.hd != kv->head_dim)) {
        for (int i = 0; i < half; ++i) rope.t.v[i] = exp2(-(2.0 * i / kv->head_dim) * log2((double)c->rope_base));
        rope.base = c->rope_base;
        rope.hd = kv->head_dim;
    }
    // few rows: their heads are shared out until every SM has two blocks
    const int all = (a.Hq + a.kv.Hkv) * (half / V) + a.kv.Hkv * (kv->head_dim / V);
    const int most = (all + AP_THREADS - 1) / AP_THREADS, want = (296 + c->batch * c->rows - 1) / (c->batch * c->rows);
    a.shares = want < most ? want : most;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    cudaError_t e;
    if (kv->dtype == MTAD_BF16)
        e = c->dtype == MTAD_F32 ? launch_append<float, __nv_bfloat16>(a, rope.t, c->batch, st)
                                 : launch_append<__nv_bfloat16, __nv_bfloat16>(a, rope.t, c->batch, st);
    else
        e = c->dtype == MTAD_F32 ? launch_append<float, __half>(a, rope.t, c->batch, st)
                                 : launch_append<__half, __half>(a, rope.t, c->batch, st);
    return ops_status(e);
}

int mtad_paged_evict(const mtad_paged_kv* kv, const mtad_paged_eviction* c, void* stream) {
    EvictArgs a{};
    if (!c) return MTAD_E_INVALID;
    const int rc = paged_view(kv, &a.kv);
    if (rc != MTAD_OK) return rc;
    if (!c->lens || !c->scores || !c->kept || !c->new_lens || c->batch < 1 || c->max_len < 1) return MTAD_E_INVALID;
    if (c->new_lens == c->lens) return MTAD_E_INVALID;    // heads that start late would read it
    if (c->keep < 1 || c->first < 0 || c->recent < 0 || (long long)c->first + c->recent > c->keep) return MTAD_E_INVALID;
    if (c->scores_stride_seq < 0 || c->scores_stride_head < 0 || (c->scores_out && (c->out_stride_seq < 0 || c->out_stride_head < 0)))
        return MTAD_E_INVALID;
    if (c->batch > MTAD_PAGED_MAX_BATCH || c->keep > MTAD_PAGED_MAX_LEN) return MTAD_E_CAPACITY;
    a.lens = c->lens; a.scores = c->scores; a.s_sb = c->scores_stride_seq; a.s_sh = c->scores_stride_head;
    a.kept = c->kept; a.new_lens = c->new_lens;
    a.scores_out = c->scores_out; a.o_sb = c->out_stride_seq; a.o_sh = c->out_stride_head;
    a.status = c->status;
    a.keep = c->keep; a.first = c->first; a.recent = c->recent;
    a.max_len = (int)std::min((long long)c->max_len, (long long)kv->max_pages * kv->page_size);
    int sms = 148, dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) sms = 148;
    const int heads = c->batch * a.kv.Hkv;
    // Blocks of a selection: as many as hold the scores, and where SMs idle more from 4096 slots a block on (8 heads, the whole call with one block
    // / with more from 4096 / from 1024 on: 2113 slots 14.1 / 14.1 / 18.6 us, 8192 26.4 / 27.1 / 31.3, 16384 44.9 / 42.7 / 45.2, 32000 90.9 / 84.3 / 84.2)
    a.cluster = 1;
    while (a.cluster < EV_MAX_CLUSTER && (a.max_len > a.cluster * EV_STAGE || (heads * a.cluster * 2 <= sms && a.max_len > a.cluster * 4 * EV_THREADS)))
        a.cluster *= 2;
    const int chunk = ((a.max_len + a.cluster - 1) / a.cluster + 3) & ~3;
    a.staged = chunk <= EV_STAGE;
    if (!a.staged && c->scores_out == c->scores) return MTAD_E_UNIMPLEMENTED;      // read again after places are written
    if (!pages_lie_apart(kv) || (c->scores_out && !lie_apart(std::min(a.keep, a.max_len), {{c->batch, a.o_sb}, {kv->n_kv_heads, a.o_sh}})))
        return MTAD_E_INVALID;
    const int smem = a.staged ? chunk * (int)sizeof(float) : 0;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    cudaError_t e = ops_smem<select_kernel>(EV_STAGE * (int)sizeof(float));
    if (e == cudaSuccess) {
        cudaLaunchConfig_t cfg{};
        cfg.gridDim = dim3(heads * a.cluster);
        cfg.blockDim = dim3(EV_THREADS);
        cfg.dynamicSmemBytes = smem;
        cfg.stream = st;
        cudaLaunchAttribute at[2];
        at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        at[0].val.programmaticStreamSerializationAllowed = 1;
        at[1].id = cudaLaunchAttributeClusterDimension;
        at[1].val.clusterDim.x = a.cluster;
        at[1].val.clusterDim.y = at[1].val.clusterDim.z = 1;
        cfg.attrs = at;
        cfg.numAttrs = 2;
        e = cudaLaunchKernelEx(&cfg, select_kernel, a);
        mtad_ops_count(1);
    }
    if (e == cudaSuccess && a.max_len > a.keep) {
        // two tensors; parts of a row, of 64 bytes at least, only where SMs would go without a block
        int slices = 2;
        while (slices < 16 && heads * slices < sms && kv->head_dim * 2 / slices >= 64) slices *= 2;
        // (a part of a row has at least one piece of 16 bytes where it has any)
        const int least = std::max(kv->head_dim / 8 * 2 / slices, 1);
        e = ops_smem<move_kernel>(MV_SMEM);
        if (e == cudaSuccess) e = launch_pdl(move_kernel, dim3(heads * slices), dim3(MV_THREADS), (size_t)MV_SMEM / least, st, true, a, slices);
        mtad_ops_count(1);
    }
    return ops_status(e);
}

}  // extern "C"
