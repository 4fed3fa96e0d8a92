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
    if (a.kv.hd % 16 == 0) append_kernel<Src, T, 8><<<grid, AP_THREADS, 0, st>>>(a, rope);
    else append_kernel<Src, T, 4><<<grid, AP_THREADS, 0, st>>>(a, rope);
    mtad_ops_count(1);
    return cudaGetLastError();
}

// ---------------------------------------------------------------------------------------------------------------
// Eviction.  Of the `len` slots of a KV head the first `first`, the last `recent` and the largest scores stay, `keep` in all (lowest slot
// first among equals), in the order of their slots; they move together to the front.
//
// A cluster of eight blocks has a KV head.  Selection: each block holds an eighth of the scores in shared memory; the keep-th
// largest is found by a radix descent over their ordered bits (11, 11 and 10 of them), histograms added up through distributed
// shared memory; one more exchange of counts gives every block the place of its first kept slot.  Moving: the blocks
// divide keys and values and the columns of a row, not the rows.  So a block walks its columns from the front with no one else in
// its way: destination j lies at or before source kept[j], and what a later round reads lies behind everything that
// earlier rounds wrote; only the reads of one round have to be over before its writes.  Bound by the bytes of what moves.

constexpr int EV_CLUSTER = 8, EV_THREADS = 512, EV_BINS = 2048, EV_UNROLL = 8;
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
    int keep, first, recent, max_len, staged;
};

// Order-preserving bits: larger score, larger key; -0 as +0; every NaN above all numbers.
__device__ __forceinline__ uint32_t score_key(float x) {
    if (x != x) return 0xffffffffu;
    const uint32_t u = __float_as_uint(x + 0.f);
    return (u & 0x80000000u) ? ~u : u | 0x80000000u;
}

__global__ void __cluster_dims__(EV_CLUSTER, 1, 1) __launch_bounds__(EV_THREADS, 2) evict_kernel(const EvictArgs a) {
    extern __shared__ float s_score[];
    __shared__ __align__(16) uint32_t hist[3][EV_BINS];
    __shared__ int s_warp[EV_THREADS / 32], s_weq[EV_THREADS / 32];
    __shared__ int s_above, s_bin;
    __shared__ int s_gt, s_eq, s_gap;                     // read by the cluster
    cg::cluster_group cluster = cg::this_cluster();
    const int rank = (int)cluster.block_rank(), tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int bh = blockIdx.x / EV_CLUSTER, b = bh / a.kv.Hkv, h = bh - b * a.kv.Hkv;
    const int raw = __ldg(a.lens + b), n = min(max(raw, 0), a.max_len);
    const float* z = a.scores + (long long)b * a.s_sb + (long long)h * a.s_sh;
    int32_t* kept = a.kept + (long long)bh * a.keep;
    float* zo = a.scores_out ? a.scores_out + (long long)b * a.o_sb + (long long)h * a.o_sh : nullptr;
    if (rank == 0 && h == 0 && tid == 0) {
        if (raw != n && a.status) atomicOr(a.status + b, MTAD_ST_KV_OVERFLOW);
    }
    if (n <= a.keep) {                                    // nothing to evict (the same for the whole cluster)
        for (int j = rank * EV_THREADS + tid; j < a.keep; j += EV_CLUSTER * EV_THREADS) {
            kept[j] = j < n ? j : -1;
            if (zo && j < n && zo != z) zo[j] = z[j];
        }
        if (rank == 0 && h == 0 && tid == 0) a.new_lens[b] = n;
        return;
    }
    const int chunk = (n + EV_CLUSTER - 1) / EV_CLUSTER, c0 = min(rank * chunk, n), c1 = min(c0 + chunk, n), mine = c1 - c0;
    const int lo = a.first, hi = n - a.recent;            // slots outside [lo, hi) stay whatever their score
    for (int i = tid; i < 3 * EV_BINS; i += EV_THREADS) (&hist[0][0])[i] = 0;
    if (a.staged)
        for (int i = tid; i < mine; i += EV_THREADS) s_score[i] = z[c0 + i];
    __syncthreads();
    auto score = [&](int i) { return a.staged ? s_score[i] : z[c0 + i]; };

    // ---- the key of the last slot that stays
    uint32_t prefix = 0;
    int need = a.keep - a.first - a.recent;               // slots still to be found among those with this prefix
    const bool some = need > 0;
#pragma unroll
    for (int pass = 0; pass < 3; ++pass) {
        const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0, bits = pass == 2 ? 10 : 11;
        if (some)
            for (int i = tid; i < mine; i += EV_THREADS) {
                const int j = c0 + i;
                if (j < lo || j >= hi) continue;
                const uint32_t key = score_key(score(i));
                if (pass == 0 || (key >> (shift + bits)) == prefix) atomicAdd(&hist[pass][(key >> shift) & ((1u << bits) - 1)], 1u);
            }
        cluster.sync();
        if (some) {
            // bins from the top: thread t has the four below 2048 - 4 t
            const int bin0 = EV_BINS - 4 * (tid + 1);
            uint4 sum = make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
            for (int k = 0; k < EV_CLUSTER; ++k) {
                const uint4 x = *reinterpret_cast<const uint4*>(cluster.map_shared_rank(&hist[pass][bin0], k));
                sum.x += x.x; sum.y += x.y; sum.z += x.z; sum.w += x.w;
            }
            const int total = (int)(sum.x + sum.y + sum.z + sum.w);
            int incl = total;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const int x = __shfl_up_sync(0xffffffffu, incl, o);
                if (lane >= o) incl += x;
            }
            if (lane == 31) s_warp[warp] = incl;
            __syncthreads();
            int before = incl - total;
            for (int w = 0; w < warp; ++w) before += s_warp[w];
            if (before < need && need <= before + total) {
                const uint32_t c[4] = {sum.w, sum.z, sum.y, sum.x};
                int at = before;
                for (int k = 0; k < 4; ++k) {
                    if (need <= at + (int)c[k]) { s_bin = bin0 + 3 - k; s_above = at; break; }
                    at += (int)c[k];
                }
            }
            __syncthreads();
            prefix = (prefix << bits) | (uint32_t)s_bin;
            need -= s_above;
            __syncthreads();
        }
    }
    // ---- places: every thread has a run of neighbouring slots
    const int run = (mine + EV_THREADS - 1) / EV_THREADS, i0 = min(tid * run, mine), i1 = min(i0 + run, mine);
    int gt = 0, eq = 0, gap = 0x7fffffff;                  // that stay for certain, that lie on the border, first one that goes
    for (int i = i0; i < i1; ++i) {
        const int j = c0 + i;
        if (j < lo || j >= hi) { ++gt; continue; }
        if (!some) continue;
        const uint32_t key = score_key(score(i));
        gt += key > prefix;
        eq += key == prefix;
    }
    int incl_g = gt, incl_e = eq;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int x = __shfl_up_sync(0xffffffffu, incl_g, o), y = __shfl_up_sync(0xffffffffu, incl_e, o);
        if (lane >= o) { incl_g += x; incl_e += y; }
    }
    if (lane == 31) { s_warp[warp] = incl_g; s_weq[warp] = incl_e; }
    if (tid == 0) s_gap = 0x7fffffff;
    __syncthreads();
    int before_g = incl_g - gt, before_e = incl_e - eq, all_g = 0, all_e = 0;
#pragma unroll
    for (int w = 0; w < EV_THREADS / 32; ++w) {
        if (w < warp) { before_g += s_warp[w]; before_e += s_weq[w]; }
        all_g += s_warp[w];
        all_e += s_weq[w];
    }
    if (tid == 0) { s_gt = all_g; s_eq = all_e; }
    cluster.sync();
    for (int k = 0; k < rank; ++k) { before_g += *cluster.map_shared_rank(&s_gt, k); before_e += *cluster.map_shared_rank(&s_eq, k); }
    for (int i = i0; i < i1; ++i) {
        const int j = c0 + i;
        const float x = score(i);
        const bool forced = j < lo || j >= hi;
        const uint32_t key = score_key(x);
        int at = -1;                                      // of those on the border the first `need` stay
        if (forced || (some && key > prefix)) at = before_g++ + min(before_e, need);
        else if (some && key == prefix) {
            if (before_e < need) at = before_g + before_e;
            ++before_e;
        }
        if (at >= 0) {
            kept[at] = j;
            if (zo) zo[at] = x;
        } else {
            gap = min(gap, j);
        }
    }
    if (gap != 0x7fffffff) atomicMin(&s_gap, gap);
    if (rank == 0 && h == 0 && tid == 0) a.new_lens[b] = a.keep;
    cluster.sync();                                       // kept[] and the gaps of all blocks are there
    int from = a.keep;
#pragma unroll
    for (int k = 0; k < EV_CLUSTER; ++k) from = min(from, *cluster.map_shared_rank(&s_gap, k));
    cluster.sync();                                       // (no block leaves while another reads its shared memory)

    // ---- moving: this block's tensor and columns
    const int chunks = a.kv.hd >> 3, part = rank & 3, col0 = part * chunks / 4, cols = (part + 1) * chunks / 4 - col0;
    if (cols == 0) return;
    uint16_t* base = ((rank >> 2) ? a.kv.v : a.kv.k) + (long long)h * a.kv.head_stride;
    const int32_t* row = a.kv.table + (long long)b * a.kv.table_stride;
    const int rows = EV_THREADS / cols, rr = tid / cols, cc = (col0 + tid - rr * cols) * 8;
    const bool on = rr < rows;
    bool bad = false;
    for (int j0 = from; j0 < a.keep; j0 += rows * EV_UNROLL) {
        int src[EV_UNROLL];
        long long so[EV_UNROLL], d_o[EV_UNROLL];
        uint4 w[EV_UNROLL];
#pragma unroll
        for (int u = 0; u < EV_UNROLL; ++u) {
            const int j = j0 + u * rows + rr;
            src[u] = on && j < a.keep ? kept[j] : -1;
        }
#pragma unroll
        for (int u = 0; u < EV_UNROLL; ++u) {
            so[u] = d_o[u] = -1;
            if (src[u] >= 0) {
                so[u] = slot_offset(a.kv, row, src[u]);
                d_o[u] = slot_offset(a.kv, row, j0 + u * rows + rr);
                bad = bad || so[u] < 0 || d_o[u] < 0;
            }
        }
#pragma unroll
        for (int u = 0; u < EV_UNROLL; ++u)
            if (so[u] >= 0) w[u] = *reinterpret_cast<const uint4*>(base + so[u] + cc);
        __syncthreads();
#pragma unroll
        for (int u = 0; u < EV_UNROLL; ++u)
            if (so[u] >= 0 && d_o[u] >= 0) *reinterpret_cast<uint4*>(base + d_o[u] + cc) = w[u];
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
    RopeTable rope;
    for (int i = 0; i < half && a.rope; ++i) rope.v[i] = exp2(-(2.0 * i / kv->head_dim) * log2((double)c->rope_base));
    // few rows: their heads are shared out until every SM has two blocks
    const int all = (a.Hq + a.kv.Hkv) * (half / V) + a.kv.Hkv * (kv->head_dim / V);
    const int most = (all + AP_THREADS - 1) / AP_THREADS, want = (296 + c->batch * c->rows - 1) / (c->batch * c->rows);
    a.shares = want < most ? want : most;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    cudaError_t e;
    if (kv->dtype == MTAD_BF16)
        e = c->dtype == MTAD_F32 ? launch_append<float, __nv_bfloat16>(a, rope, c->batch, st)
                                 : launch_append<__nv_bfloat16, __nv_bfloat16>(a, rope, c->batch, st);
    else
        e = c->dtype == MTAD_F32 ? launch_append<float, __half>(a, rope, c->batch, st)
                                 : launch_append<__half, __half>(a, rope, c->batch, st);
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
    const int chunk = (a.max_len + EV_CLUSTER - 1) / EV_CLUSTER;
    a.staged = chunk <= EV_STAGE;
    if (!a.staged && c->scores_out == c->scores) return MTAD_E_UNIMPLEMENTED;      // read again after places are written
    const int smem = a.staged ? chunk * (int)sizeof(float) : 0;
    cudaError_t e = ops_smem<evict_kernel>(EV_STAGE * (int)sizeof(float));
    if (e == cudaSuccess) {
        evict_kernel<<<c->batch * a.kv.Hkv * EV_CLUSTER, EV_THREADS, smem, static_cast<cudaStream_t>(stream)>>>(a);
        mtad_ops_count(1);
        e = cudaGetLastError();
    }
    return ops_status(e);
}

}  // extern "C"
