// The accept rules on rows of logits that the caller's decoder wrote: a draft chain per sequence, the joint-likelihood threshold of
// Algorithm 1 or the rule of vanilla speculative decoding (Sec. 2.2, steps 2-4).
//
// With z the target's rows over a temperature, lp_i = z_i[x_i] - lse(z_i):
//     threshold    prefix j passes iff sum_{i <= j} lp_i - log q(x_{1:j}) > log tau, the longest passing one is accepted;
//     speculative  token i is accepted iff log u_i < lp_i - lq_i, up to the first rejection.
// The last token is a draw from w = p (nothing rejected, or the threshold rule) or w = max(0, p - q) at the rejected position: the
// argmax of w_v / -log u_v, the same as the argmax of log w_v - log(-log u_v) without two logarithms per token.
//
// Every row is read once for its log-sum-exp, one row and the uniforms again for the draw: bound by those bytes together with the
// exponentials (16 a clock and SM: 24 us of 64 sequences x 13 rows x 128000 bf16 logits whose bytes take 33), at small
// batches by latency.  A cluster of four or eight blocks has a sequence, a block its part of the vocabulary; warps take (row, part) tasks, a
// reference and a sum a lane; rows' statistics and the draw's candidates cross the cluster in distributed shared memory, so
// the call is one launch and needs no workspace.  Statistics are fp32, merged in a fixed order.  The batch of 64 takes 61 us (4.0 TB/s;
// 14 of them the draw, whose loads wait for the accepted prefix), one chain of 5 rows of 32000 fp32 logits 11 us.
#include <cooperative_groups.h>
#include <math.h>
#include <math_constants.h>

#include "paged.cuh"

namespace cg = cooperative_groups;

namespace mtad {

namespace {

constexpr int AC_ROWS = 2 * MTAD_MAX_DEPTH + 1, AC_PARTS = 8;
constexpr float LN2 = 0.6931471805599453f;

struct AcceptRowsArgs {
    const void *z, *q;               // target rows [B, gamma + 1, V], auxiliary rows [B, gamma, V] or null (threshold rule)
    long long z_sb, z_sr, q_sb, q_sr;
    const int32_t *tok, *n_draft;
    const float *draft_logq, *u_accept, *u_last;
    float z_mul, q_mul, log_tau;     // log2(e) / temperature
    double z_unit;                   // 1 / temperature over z_mul as it is: from powers of two back to the rows' own logarithms
    int gamma, V;
    mtad_result out;
};

// Statistics of logits over the temperature, in powers of two: x = z * c, c = log2(e) / temperature.  The reference is a whole number, so
// x - ref is one fused multiply-add whose only rounding is the result's: no bias enters a sum of many.  Reference and sum stay apart to the
// end: whatever has been added to a row is in the reference alone, and a log-probability, (x - ref) - log2(sum), does not see it.
struct Stat {
    float m, s;                      // reference, sum of 2^(x - m)
};
__device__ __forceinline__ float ex2a(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// The sum within [1/2, 1): log2(sum) is small beside x - ref
__device__ __forceinline__ Stat settled(Stat a) {
    if (fabsf(a.m) < 0x1p23f) {                           // (references beyond are no longer whole numbers apart)
        int k = 0;
        a.s = frexpf(a.s, &k);
        a.m += (float)k;
    }
    return a;
}
__device__ __forceinline__ Stat merge(const Stat& a, const Stat& b) {
    const float m = fmaxf(a.m, b.m);
    if (m == -CUDART_INF_F) return Stat{m, a.s + b.s};    // (sums of 0, or NaN)
    return Stat{m, a.s * (a.m == m ? 1.f : ex2a(a.m - m)) + b.s * (b.m == m ? 1.f : ex2a(b.m - m))};
}
// N logits, the largest of them (times a positive c) known
template <int N>
__device__ __forceinline__ void take(Stat& st, const float (&z)[N], float top, float c) {
    const float x = top * c;
    if (x > st.m) {
        const float m = ceilf(x);
        st.s *= st.m == -CUDART_INF_F ? 0.f : ex2a(st.m - m);
        st.m = m;
    }
    const float r = st.m == -CUDART_INF_F ? 0.f : st.m;
    float s0 = 0.f, s1 = 0.f;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const float e = ex2a(fmaf(z[i], c, -r));
        if (i & 1) s1 += e; else s0 += e;
    }
    st.s += s0 + s1;
}

template <typename T> struct Row;
template <> struct Row<float> {
    static constexpr int N = 4;
    static __device__ __forceinline__ void vec(const uint4& w, float (&x)[4]) {
        x[0] = __uint_as_float(w.x); x[1] = __uint_as_float(w.y); x[2] = __uint_as_float(w.z); x[3] = __uint_as_float(w.w);
    }
    static __device__ __forceinline__ float one(float x) { return x; }
    static __device__ __forceinline__ uint4 nothing() { return make_uint4(0xff800000u, 0xff800000u, 0xff800000u, 0xff800000u); }
    static __device__ __forceinline__ float top(const uint4& w) {
        return fmaxf(fmaxf(__uint_as_float(w.x), __uint_as_float(w.y)), fmaxf(__uint_as_float(w.z), __uint_as_float(w.w)));
    }
};
template <typename T> struct Pair;
template <> struct Pair<__nv_bfloat16> { using type = __nv_bfloat162; };
template <> struct Pair<__half> { using type = __half2; };
template <typename T> struct Row16 {
    static constexpr int N = 8;
    static __device__ __forceinline__ void vec(const uint4& w, float (&x)[8]) {
        const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float2 f = Num<T>::unpack(u[i]);
            x[2 * i] = f.x; x[2 * i + 1] = f.y;
        }
    }
    static __device__ __forceinline__ float one(T x) { return Num<T>::to(x); }
    static __device__ __forceinline__ uint4 nothing() {                  // -infinity, eight times
        constexpr uint32_t w = (0x8000u | Num<T>::kExp) * 0x10001u;
        return make_uint4(w, w, w, w);
    }
    // the largest of eight, two at a time (NaN is passed over: it shows in the sum)
    static __device__ __forceinline__ float top(const uint4& w) {
        using P = typename Pair<T>::type;
        const P* p = reinterpret_cast<const P*>(&w);
        const P m = __hmax2(__hmax2(p[0], p[1]), __hmax2(p[2], p[3]));
        const float2 f = Num<T>::unpack(*reinterpret_cast<const uint32_t*>(&m));
        return fmaxf(f.x, f.y);
    }
};
template <> struct Row<__nv_bfloat16> : Row16<__nv_bfloat16> {};
template <> struct Row<__half> : Row16<__half> {};

// Two fp32 at a time
__device__ __forceinline__ uint64_t pair(float lo, float hi) {
    uint64_t x;
    asm("mov.b64 %0, {%1, %2};" : "=l"(x) : "f"(lo), "f"(hi));
    return x;
}
__device__ __forceinline__ float2 halves(uint64_t x) {
    float2 f;
    asm("mov.b64 {%0, %1}, %2;" : "=f"(f.x), "=f"(f.y) : "l"(x));
    return f;
}
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
    uint64_t x;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(x) : "l"(a), "l"(b), "l"(c));
    return x;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
    uint64_t x;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(x) : "l"(a), "l"(b));
    return x;
}

// Statistics of elements [v0, v1) of a row, by one warp: 16-byte loads, U in flight a lane; what lies before the
// first 16-byte boundary and behind the last (rows of odd vocabularies begin anywhere) one by one.
// A lane's reference is the largest of its first load, kept to the end: looking for the largest of every load took longer than the
// exponentials.  Terms up to 2^90 stay in range; x - ref is then rounded to 2^-17, so that a term so far above the first ones is good to
// 2^-18 of itself (one within 2^16 of them to 2^-21, as with the largest known).  What would keep such terms as exact costs every row: a sum
// watched for them, and the reference moved, 72 us instead of 61 for 64 x 13 rows of 128000; a second pass from 2^32 on 41 -> 63 us for
// 64 x 7 rows with one token 25 above the rest.  Where the sum leaves the range (an
// element more than 2^90 above the first ones, or all of them far below; a row that begins with masked tokens), the warp goes through
// its elements again with a running maximum.
template <typename T>
__device__ __forceinline__ Stat row_stat(const T* row, int v0, int v1, float c, int lane) {
    constexpr int N = Row<T>::N, U = 2;
    const int skip = (int)((16 - (reinterpret_cast<uintptr_t>(row + v0) & 15)) & 15) / (int)sizeof(T);
    const int a0 = min(v0 + skip, v1), nv = (v1 - a0) / N, tail = a0 + nv * N;
    const uint4* p = reinterpret_cast<const uint4*>(row + a0);
    const uint64_t cc = pair(c, c);
    Stat st{0.f, 0.f};
    uint64_t s0 = 0, s1 = 0, ref = 0;
    bool any = false;
    uint4 w[U], next[U];                                  // (the next loads are on their way while these are added)
    auto load = [&](int i, uint4 (&to)[U]) {
#pragma unroll
        for (int u = 0; u < U; ++u) to[u] = i + u * 32 < nv ? __ldg(p + i + u * 32) : Row<T>::nothing();      // (past the end: no weight)
    };
    load(lane, w);
    if (lane < nv) {
        const float m = ceilf(Row<T>::top(w[0]) * c);
        any = true;
        st.m = isfinite(m) ? m : 0.f;
        ref = pair(-st.m, -st.m);
    }
    for (int i = lane; i - lane < nv; i += 32 * U) {
        load(i + 32 * U, next);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            float z[N];
            Row<T>::vec(w[u], z);
#pragma unroll
            for (int k = 0; k < N; k += 4) {
                const float2 x = halves(fma2(pair(z[k], z[k + 1]), cc, ref)), y = halves(fma2(pair(z[k + 2], z[k + 3]), cc, ref));
                s0 = add2(s0, pair(ex2a(x.x), ex2a(x.y)));
                s1 = add2(s1, pair(ex2a(y.x), ex2a(y.y)));
            }
        }
#pragma unroll
        for (int u = 0; u < U; ++u) w[u] = next[u];
    }
    const float2 t = halves(add2(s0, s1));
    st.s = t.x + t.y;
    if (__any_sync(0xffffffffu, any && !(st.s >= 0x1p-60f && st.s <= 0x1p90f))) {
        st = Stat{-CUDART_INF_F, 0.f};
        for (int i = lane; i < nv; i += 32) {
            const uint4 w = __ldg(p + i);
            float z[N];
            Row<T>::vec(w, z);
            take<N>(st, z, Row<T>::top(w), c);
        }
    } else if (!any) {
        st = Stat{-CUDART_INF_F, 0.f};
    }
    for (int v = v0 + lane; v < a0; v += 32) { const float z[1] = {Row<T>::one(row[v])}; take<1>(st, z, z[0], c); }
    for (int v = tail + lane; v < v1; v += 32) { const float z[1] = {Row<T>::one(row[v])}; take<1>(st, z, z[0], c); }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) st = merge(st, Stat{__shfl_xor_sync(0xffffffffu, st.m, o), __shfl_xor_sync(0xffffffffu, st.s, o)});
    return st;
}

struct Best {
    float y;
    int v;
};
__device__ __forceinline__ void better(Best& a, float y, int v) {
    if (y > a.y || (y == a.y && v < a.v)) { a.y = y; a.v = v; }
}

// CLUSTER blocks of THREADS threads a sequence: eight of 512 where that leaves SMs idle, four of 512 up to two blocks an SM (64 sequences:
// 60.5 us; eight of 256: 64), four of 256 beyond
template <typename T, int CLUSTER, int THREADS>
__global__ void __cluster_dims__(CLUSTER, 1, 1) __launch_bounds__(THREADS, 1024 / THREADS) accept_rows_kernel(const AcceptRowsArgs a) {
    constexpr int WARPS = THREADS / 32;
    constexpr bool few = CLUSTER == 8;
    cg::cluster_group cluster = cg::this_cluster();
    const int rank = (int)cluster.block_rank(), b = blockIdx.x / CLUSTER, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    __shared__ Stat s_part[AC_ROWS * AC_PARTS];
    __shared__ Stat s_row[AC_ROWS];                       // read by the cluster
    __shared__ Best s_best[WARPS], s_block;            // s_block: read by the cluster
    __shared__ float s_ref[AC_ROWS], s_sum[AC_ROWS], s_log[AC_ROWS];      // of a row: the reference, the sum, its logarithm
    __shared__ int s_eta;
    const int D = a.gamma, V = a.V;
    pdl_wait();
    pdl_trigger();
    const int given = a.n_draft ? __ldg(a.n_draft + b) : D, g = min(max(given, 0), D);
    const bool spd = a.q != nullptr;
    const int rows = g + 1 + (spd ? g : 0);
    const T* z = static_cast<const T*>(a.z) + (long long)b * a.z_sb;
    const T* q = spd ? static_cast<const T*>(a.q) + (long long)b * a.q_sb : nullptr;
    const int per = ((V + CLUSTER - 1) / CLUSTER + 7) / 8 * 8, v0 = min(rank * per, V), v1 = min(v0 + per, V);
    // tokens and their logits, early: a lane per drafted token
    uint32_t bits = given == g ? 0u : MTAD_ST_BAD_COUNT;
    int x = 0;
    float zx = 0.f, qx = 0.f;
    if (warp == 0) {
        bool bad = false;
        if (lane < g) {
            x = __ldg(a.tok + (long long)b * D + lane);
            bad = (unsigned)x >= (unsigned)V;
            if (!bad) {
                zx = Row<T>::one(z[(long long)lane * a.z_sr + x]);
                if (spd) qx = Row<T>::one(q[(long long)lane * a.q_sr + x]);
            }
        }
        if (__any_sync(0xffffffffu, bad)) bits |= MTAD_ST_BAD_TOKEN;
    }
    if (few) {                                            // (the draw's uniforms are on their way into the L2 meanwhile)
        const float* u = a.u_last + (long long)b * V;
        for (int v = v0 + tid * 32; v < v1; v += THREADS * 32) asm volatile("prefetch.global.L2 [%0];" ::"l"(u + v));
    }
    // ---- log-sum-exp of every row
    // (as few parts of a row as keep most warps at work in the last round, none of less than two loads a lane)
    int parts = 1;
    {
        float best = 0.f;
        const int most = min(AC_PARTS, max(1, (v1 - v0) / (Row<T>::N * 64)));
        for (int p = 1; p <= most; ++p) {
            const float use = (float)(rows * p) / (float)((rows * p + WARPS - 1) / WARPS * WARPS);
            if (best < 0.9f && use > best + 0.02f) { best = use; parts = p; }
        }
    }
    const int step = ((v1 - v0 + parts - 1) / parts + Row<T>::N - 1) / Row<T>::N * Row<T>::N;
    for (int t = warp; t < rows * parts; t += WARPS) {
        const int r = t / parts, p = t - r * parts, e0 = min(v0 + p * step, v1), e1 = min(e0 + step, v1);
        const Stat st = r <= g ? row_stat<T>(z + (long long)r * a.z_sr, e0, e1, a.z_mul, lane)
                               : row_stat<T>(q + (long long)(r - g - 1) * a.q_sr, e0, e1, a.q_mul, lane);
        if (lane == 0) s_part[t] = st;
    }
    __syncthreads();
    if (tid < rows) {
        Stat st = s_part[tid * parts];
        for (int p = 1; p < parts; ++p) st = merge(st, s_part[tid * parts + p]);
        s_row[tid] = st;
    }
    cluster.sync();
    if (tid < rows) {
        Stat st = *cluster.map_shared_rank(&s_row[tid], 0);
        for (int k = 1; k < CLUSTER; ++k) st = merge(st, *cluster.map_shared_rank(&s_row[tid], k));
        st = settled(st);
        s_ref[tid] = st.m;
        s_sum[tid] = st.s;
        s_log[tid] = log2f(st.s);
    }
    __syncthreads();
    // of a logit of row r (a product by itself: fused into a difference of two, equal ones would no longer cancel)
    auto log_p = [&](float x, float c, int r) { return __fmul_rn(fmaf(x, c, -s_ref[r]) - s_log[r], LN2); };
    // ---- the accepted prefix (warp 0 of every block; the first block writes)
    if (warp == 0) {
        const bool w = rank == 0;
        bool finite = true;
        for (int r = lane; r < rows; r += 32) finite = finite && isfinite(s_ref[r]) && isfinite(s_log[r]);
        if (!__all_sync(0xffffffffu, finite)) bits |= MTAD_ST_NONFINITE;
        const float lp = lane < g ? log_p(zx, a.z_mul, lane) : 0.f;
        int eta = 0;
        float gap = CUDART_INF_F, LP = lp;
        if (spd) {
            const float ratio = lane < g ? fminf(0.f, lp - log_p(qx, a.q_mul, g + 1 + lane)) : 0.f;   // (NaN, 0 over 0: rejected, below)
            const float lu = lane < g ? logf(__ldg(a.u_accept + (long long)b * D + lane)) : 0.f;
            const bool ok = lane < g && lp > -CUDART_INF_F && lu < ratio;
            const uint32_t no = __ballot_sync(0xffffffffu, !ok);
            eta = min(no ? __ffs(no) - 1 : 32, g);
            if (lane <= eta && lane < g) gap = fabsf(lu - ratio);
        } else {
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const float y = __shfl_up_sync(0xffffffffu, LP, o);
                if (lane >= o) LP += y;
            }
            const float over = lane < g ? LP - __ldg(a.draft_logq + (long long)b * D + lane) : 0.f;
            // (log_tau = -inf: every prefix passes)
            const bool ok = lane < g && (a.log_tau == -CUDART_INF_F || over > a.log_tau);
            const uint32_t yes = __ballot_sync(0xffffffffu, ok);
            eta = yes ? 32 - __clz(yes) : 0;
            if (lane < g) gap = fabsf(over - a.log_tau);
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) gap = fminf(gap, __shfl_xor_sync(0xffffffffu, gap, o));
        if (lane == 0) s_eta = bits ? -1 : eta;
        if (w) {
            const mtad_result& o = a.out;
            if (bits) eta = 0;
            if (lane == 0) {
                o.status[b] = bits;
                o.eta[b] = eta;
                o.winner[b] = eta - 1;
                o.n_out[b] = bits ? 0 : eta + 1;
                if (o.margin && !bits) { o.margin[b * 2] = gap; o.margin[b * 2 + 1] = CUDART_INF_F; }
            }
            if (!bits) {
                if (lane < eta) {
                    o.path[(long long)b * D + lane] = lane;
                    o.out_tok[(long long)b * (D + 1) + lane] = x;
                    o.out_lp[(long long)b * (D + 1) + lane] = lp;
                }
                if (lane < g && o.node_lp) o.node_lp[(long long)b * D + lane] = lp;
                if (lane < g && o.node_LP && !spd) o.node_LP[(long long)b * D + lane] = LP;
                if (o.row_lse)
                    for (int r = lane; r <= g; r += 32) o.row_lse[(long long)b * (D + 1) + r] = (float)(((double)s_ref[r] + (double)s_log[r]) * a.z_unit);
            }
        }
    }
    __syncthreads();
    const int eta = s_eta;
    // ---- the last token: this block's share of the vocabulary.  w_v / -log u_v with its logarithm in full precision; -log u is taken only
    // where the weight could still win, that is where w > best * (1 - u) (-log u >= 1 - u).
    Best best{-CUDART_INF_F, 0x7fffffff};
    auto search = [&](bool rest) {
        const T* row = z + (long long)eta * a.z_sr;
        const T* qrow = rest ? q + (long long)eta * a.q_sr : row;
        const float cz = a.z_mul, cq = a.q_mul, rz = s_ref[eta], rq = rest ? s_ref[g + 1 + eta] : 0.f;
        const float k = rest ? s_sum[eta] / s_sum[g + 1 + eta] : 0.f;      // (p - q) * sum of p's row: one factor, 1 where the rows are the same
        const float* u = a.u_last + (long long)b * V;
        float lead = 0.f;                                 // the best that this warp has seen
        auto look = [&](float x, float y, float un, int v) {
            const float w = fmaf(-k, ex2a(fmaf(y, cq, -rq)), ex2a(fmaf(x, cz, -rz)));
            if (w > 0.f && !(w < lead * (1.f - un))) better(best, w / -logf(un), v);
        };
        auto share = [&]() { lead = __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(fmaxf(best.y, 0.f)))); };
        constexpr int N = Row<T>::N;
        const bool even = ((reinterpret_cast<uintptr_t>(row + v0) | reinterpret_cast<uintptr_t>(qrow + v0) | reinterpret_cast<uintptr_t>(u + v0)) & 15) == 0;
        const int nv = even ? (v1 - v0) / N : 0;          // 16-byte loads where all three rows allow them
        for (int i = tid; i - tid < nv; i += 2 * THREADS) {
            uint4 x[2], y[2];
            float4 un[2][N / 4];
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const int at = i + k * THREADS;
                x[k] = at < nv ? __ldg(reinterpret_cast<const uint4*>(row + v0) + at) : Row<T>::nothing();
                y[k] = rest && at < nv ? __ldg(reinterpret_cast<const uint4*>(qrow + v0) + at) : Row<T>::nothing();
#pragma unroll
                for (int h = 0; h < N / 4; ++h)
                    un[k][h] = at < nv ? __ldg(reinterpret_cast<const float4*>(u + v0) + at * (N / 4) + h) : make_float4(0.f, 0.f, 0.f, 0.f);
            }
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                float zx[N], zy[N];
                Row<T>::vec(x[k], zx);
                Row<T>::vec(y[k], zy);
                const int v = v0 + (i + k * THREADS) * N;
#pragma unroll
                for (int h = 0; h < N / 4; ++h) {
                    look(zx[4 * h], zy[4 * h], un[k][h].x, v + 4 * h);
                    look(zx[4 * h + 1], zy[4 * h + 1], un[k][h].y, v + 4 * h + 1);
                    look(zx[4 * h + 2], zy[4 * h + 2], un[k][h].z, v + 4 * h + 2);
                    look(zx[4 * h + 3], zy[4 * h + 3], un[k][h].w, v + 4 * h + 3);
                }
                share();
            }
        }
        constexpr int U = 4;
        for (int v = v0 + nv * N + tid; v - tid < v1; v += U * THREADS) {
            float x[U], y[U], un[U];
#pragma unroll
            for (int k = 0; k < U; ++k) {
                const bool in = v + k * THREADS < v1;
                x[k] = in ? Row<T>::one(row[v + k * THREADS]) : -CUDART_INF_F;
                y[k] = rest && in ? Row<T>::one(qrow[v + k * THREADS]) : -CUDART_INF_F;
                un[k] = in ? __ldg(u + v + k * THREADS) : 0.f;
            }
#pragma unroll
            for (int k = 0; k < U; ++k) look(x[k], y[k], un[k], v + k * THREADS);
            share();
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) better(best, __shfl_xor_sync(0xffffffffu, best.y, o), __shfl_xor_sync(0xffffffffu, best.v, o));
        if (lane == 0) s_best[warp] = best;
        __syncthreads();
        if (warp == 0) {
            best = lane < WARPS ? s_best[lane] : Best{-CUDART_INF_F, 0x7fffffff};
#pragma unroll
            for (int o = 8; o > 0; o >>= 1) better(best, __shfl_xor_sync(0xffffffffu, best.y, o), __shfl_xor_sync(0xffffffffu, best.v, o));
            if (lane == 0) s_block = best;
        }
        cluster.sync();
        best = Best{-CUDART_INF_F, 0x7fffffff};
#pragma unroll
        for (int k = 0; k < CLUSTER; ++k) {
            const Best c = *cluster.map_shared_rank(&s_block, k);
            better(best, c.y, c.v);
        }
    };
    if (eta >= 0) {                                       // (the same in every block of the cluster)
        search(spd && eta < g);
        if (best.v == 0x7fffffff) {                       // no mass left where p and q agree to the last bit: a draw from p
            cluster.sync();
            search(false);
        }
        if (rank == 0 && tid == 0) {
            const int t = best.v != 0x7fffffff ? best.v : 0;
            a.out.out_tok[(long long)b * (D + 1) + eta] = t;
            a.out.out_lp[(long long)b * (D + 1) + eta] = log_p(Row<T>::one(z[(long long)eta * a.z_sr + t]), a.z_mul, eta);
        }
    }
    cluster.sync();                                       // (no block leaves while another reads its shared memory)
}

int accept_rows(const mtad_accept_rows* c, const float* draft_logq, float log_tau, const void* q, const float* u_accept,
                const mtad_result* out, void* stream) {
    if (!c || !out || !c->logits || !c->last_uniform || c->batch < 1 || c->gamma < 0 || c->vocab < 1) return MTAD_E_INVALID;
    if (c->gamma > 0 && (!c->draft_tok || !out->path)) return MTAD_E_INVALID;
    if (!out->eta || !out->winner || !out->n_out || !out->out_tok || !out->out_lp || !out->status) return MTAD_E_INVALID;
    if (c->dtype != MTAD_BF16 && c->dtype != MTAD_F16 && c->dtype != MTAD_F32) return MTAD_E_INVALID;
    if (c->batch > MTAD_PAGED_MAX_BATCH || c->gamma > MTAD_MAX_DEPTH) return MTAD_E_CAPACITY;
    if (!(c->temperature > 0.f) || !isfinite(c->temperature)) return MTAD_E_INVALID;
    if (c->logits_stride_seq < 0 || c->logits_stride_row < 0 || (q && (c->draft_stride_seq < 0 || c->draft_stride_row < 0))) return MTAD_E_INVALID;
    const uintptr_t el = c->dtype == MTAD_F32 ? 4 : 2;
    if ((reinterpret_cast<uintptr_t>(c->logits) | reinterpret_cast<uintptr_t>(q)) & (el - 1)) return MTAD_E_INVALID;
    AcceptRowsArgs a{};
    a.z = c->logits; a.q = q;
    a.z_sb = c->logits_stride_seq; a.z_sr = c->logits_stride_row; a.q_sb = c->draft_stride_seq; a.q_sr = c->draft_stride_row;
    a.tok = c->draft_tok; a.n_draft = c->n_draft;
    a.draft_logq = draft_logq; a.u_accept = u_accept; a.u_last = c->last_uniform;
    a.z_mul = (float)(1.4426950408889634 / c->temperature); a.q_mul = q ? (float)(1.4426950408889634 / c->draft_temperature) : 1.f;
    a.z_unit = 1.0 / c->temperature / a.z_mul;
    a.log_tau = log_tau;
    a.gamma = c->gamma; a.V = c->vocab;
    a.out = *out;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    mtad_ops_count(1);
    int sms = 148, dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) sms = 148;
    auto launch = [&](auto type) {
        using T = decltype(type);
        if (c->batch * 8 <= sms) return launch_pdl(accept_rows_kernel<T, 8, 512>, dim3(c->batch * 8), dim3(512), 0, st, true, a);
        if (c->batch * 4 <= 2 * sms) return launch_pdl(accept_rows_kernel<T, 4, 512>, dim3(c->batch * 4), dim3(512), 0, st, true, a);
        return launch_pdl(accept_rows_kernel<T, 4, 256>, dim3(c->batch * 4), dim3(256), 0, st, true, a);
    };
    return ops_status(c->dtype == MTAD_F32 ? launch(0.f) : c->dtype == MTAD_BF16 ? launch(__nv_bfloat16()) : launch(__half()));
}

}  // namespace

}  // namespace mtad

using namespace mtad;

extern "C" {

int mtad_accept_chain(const mtad_accept_rows* call, const float* draft_logq, float log_tau, const mtad_result* out, void* stream) {
    if (!call || (call->gamma > 0 && !draft_logq) || isnan(log_tau) || !(log_tau < 0.f)) return MTAD_E_INVALID;
    return accept_rows(call, draft_logq, log_tau, nullptr, nullptr, out, stream);
}

int mtad_accept_chain_spd(const mtad_accept_rows* call, const void* draft_rows, const float* accept_uniform, const mtad_result* out,
                          void* stream) {
    if (!call || !draft_rows || !accept_uniform || call->gamma < 1) return MTAD_E_INVALID;
    if (!(call->draft_temperature > 0.f) || !isfinite(call->draft_temperature)) return MTAD_E_INVALID;
    return accept_rows(call, nullptr, 0.f, draft_rows, accept_uniform, out, stream);
}

}  // extern "C"
