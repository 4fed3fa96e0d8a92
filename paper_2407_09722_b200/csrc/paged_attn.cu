// Attention of the new rows of every sequence over a cache kept in pages.
//
//     out[r, h] = sum_j p_j V[j],   p = softmax_j(scale * q[r, h] . K[j]) over the slots j that row r sees:
//     j <= pos_r,  and with a window  j > pos_r - window  or  j < sinks;   pos_r = length - rows + r
//
// What bounds it: a call reads the visible keys and values once (2 * 2 * head_dim bytes per token and KV head) and does 4 *
// head_dim operations per query row with them, a few dozen per byte at most, so HBM bounds it and the tensor cores idle; at
// short lengths launches and latency do.  Hence
//  - the query rows of a KV head (rows x heads of the group) share one pass over its keys: they are the M side of the
//    mma.sync tiles (m16n8k16), 16, 32 or 64 a block; the rest of the 16 costs tensor work that nobody waits for;
//  - the work is a list of 64-key tiles over (sequence, KV head, row block) that is cut evenly over a grid that fills the
//    GPU once, whatever the lengths: the batch may be ragged, a single long sequence may be alone.  A block's share
//    may begin and end inside a head: its pieces (running maximum, sum, unnormalised output, all fp32) are joined by a
//    second kernel that the first one's launch overlaps; heads that one block saw whole are finished there and then;
//  - a warp copies the keys and values that it multiplies itself (16 rows per request of the tile, cp.async, three or more
//    stages) where a block has 16 query rows, so that no barrier stands between a copy and its use;
//  - page ids and offsets are looked up one tile ahead, a lane per key, and handed around by shuffles.
// Rounding: scores, statistics and sums are fp32.  Probabilities enter the second product as two terms of the cache's type
// (p and what its rounding left), so the 2^-9 of a bf16 probability does not reach the output; the output is rounded once.
#include <math_constants.h>

#include <algorithm>
#include <type_traits>

#include "paged.cuh"

namespace mtad {

namespace {

constexpr int TK = 64;               // keys of a tile
constexpr int NT = 128;              // threads of a block
constexpr int MAX_ROWS_BLOCK = 64;   // query rows (rows x heads of the group) of a block
constexpr int WHOLE_TILES = 4;       // up to so many tiles a head, a block takes a head as a whole and nothing is joined

struct AttnArgs {
    PagedView kv;
    const int32_t* lens;
    const int32_t* n_rows;           // or null: R
    const uint16_t* q;
    uint16_t* out;
    float* lse;                      // [B, R, Hq] or null
    long long q_sb, q_sr, q_sh, o_sb, o_sr, o_sh;
    uint32_t* status;
    int B, R, G, RB, rows_block;     // heads of a group, row blocks, query rows of a block (16 * MT)
    int window, sinks, max_len;
    float scale2;                    // scale * log2(e)
    int whole;                       // a block per (sequence, KV head, row block)
    int grid;
    // workspace
    long long* plan;                 // [0] tiles of a block, [1 .. B + 1] first tile of every sequence
    float* part_o;                   // [2 * grid][rows_block][HD]
    float2* part_ml;                 // [2 * grid][rows_block] maximum (log2 domain) and sum
    float* row_lse2;                 // [B][Hkv * RB][rows_block] log2 of the sums of heads that one block saw whole, only with weights
    float* scores;                   // [B][Hkv][RB * rows_block][score_ld] log2-domain scores, only with weights
    long long score_ld;
    float* weights;                  // [B][Hkv][..] accumulated, or null
    long long w_sb, w_sh;
};

// Sequence b as this call sees it: its length, its rows and the tiles that some row sees (those of the sinks, then those
// from the window's first slot on).
struct Seq {
    int len, nb, nt, ns, skip;       // tile t of the list is tile t of the cache for t < ns, t + skip beyond
};
__device__ __forceinline__ Seq seq_of(const AttnArgs& a, int b) {
    Seq s;
    const int len = __ldg(a.lens + b);
    s.len = min(max(len, 0), a.max_len);
    s.nb = a.n_rows ? min(max(__ldg(a.n_rows + b), 0), a.R) : a.R;
    const int total = (s.len + TK - 1) / TK;
    s.ns = total;
    s.skip = 0;
    if (a.window > 0) {
        const int first = max(s.len - s.nb - a.window + 1, 0);          // of the first row
        const int ns = (min(a.sinks, s.len) + TK - 1) / TK;
        const int from = max(first / TK, ns);
        if (from < total) { s.ns = ns; s.skip = from - ns; }
    }
    // (a sequence without a visible slot still has a tile: its rows are written)
    s.nt = s.nb == 0 ? 0 : max(total - s.skip, 1);
    return s;
}

struct Cursor {                      // a tile of the list
    int b, hr, t;                    // sequence, KV head * row blocks + row block, tile
    Seq s;
};
__device__ __forceinline__ void advance(const AttnArgs& a, Cursor& c) {
    if (++c.t < c.s.nt) return;
    c.t = 0;
    if (++c.hr < a.kv.Hkv * a.RB) return;
    c.hr = 0;
    do {
        if (++c.b >= a.B) return;
        c.s = seq_of(a, c.b);
    } while (c.s.nt == 0);
}

__device__ __forceinline__ void cp16(uint32_t dst, const void* src, bool there) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(there ? 16 : 0) : "memory");
}
__device__ __forceinline__ void cp_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void cp_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }
__device__ __forceinline__ void ldsm4(uint32_t (&r)[4], uint32_t at) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(at));
}
__device__ __forceinline__ void ldsm4t(uint32_t (&r)[4], uint32_t at) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(at));
}
template <typename T>
__device__ __forceinline__ void mma(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    if constexpr (std::is_same<T, __half>::value)
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
    else
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ float ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

template <int HD> struct Tile {
    static constexpr int CH = HD / 8;                    // 16-byte pieces of a row
    static constexpr int BYTES = TK * HD * 2;            // keys (or values) of a tile
    static constexpr int STAGES = HD == 64 ? 6 : 3;      // 96 KB (192 of heads of 256) on their way or in use
    static constexpr int BLOCKS = HD == 256 ? 1 : 2;     // blocks of an SM
    // byte offset of piece c of row r: pieces of eight neighbouring rows fall into different banks
    static __device__ __forceinline__ uint32_t at(int r, int c) { return (uint32_t)(r * HD * 2 + ((c ^ (r & 7)) << 4)); }
};
template <int HD, int MT> constexpr int attn_smem() {
    return Tile<HD>::STAGES * 2 * Tile<HD>::BYTES + MT * 16 * HD * 2 + (MT < 4 ? 16 * HD * 4 : 0);
}

// T: the cache's type; HD: head_dim rounded up to 64, 128 or 256; MT: 16-row tiles of query rows (the four warps stand MT
// over the rows by 4 / MT over the keys of a tile)
template <typename T, int HD, int MT>
__global__ void __launch_bounds__(NT, Tile<HD>::BLOCKS) attn_kernel(const AttnArgs a) {
    using L = Tile<HD>;
    constexpr int KW = 4 / MT, WK = TK / KW, S = L::STAGES, CH = L::CH, PASS = 32 / CH > 0 ? 32 / CH : 1, RW = 16;
    extern __shared__ __align__(128) unsigned char smem[];
    __shared__ float s_m[4][16], s_l[4][16];
    __shared__ long long s_scan[4];
    __shared__ long long s_first[3];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, wm = warp % MT, wk = warp / MT;
    const int g = lane >> 2, t2 = (lane & 3) * 2;
    const uint32_t sm = (uint32_t)__cvta_generic_to_shared(smem);
    const uint32_t sm_q = sm + S * 2 * L::BYTES;
    float* const obuf = reinterpret_cast<float*>(smem + S * 2 * L::BYTES + MT * 16 * HD * 2);
    const int HR = a.kv.Hkv * a.RB, chunks = a.kv.hd >> 3;

    pdl_trigger();
    // ---- this block's share of the list
    long long start, end, per = 0;
    Cursor P;
    if (a.whole) {
        P.b = blockIdx.x / HR;
        P.hr = blockIdx.x - P.b * HR;
        P.t = 0;
        P.s = seq_of(a, P.b);
        start = 0;
        end = P.s.nt;
        if (end == 0) return;
    } else {
        const int each = (a.B + NT - 1) / NT, b0 = tid * each, b1 = min(a.B, b0 + each);
        long long mine = 0;
        for (int b = b0; b < b1; ++b) mine += (long long)seq_of(a, b).nt * HR;
        long long incl = mine;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const long long x = __shfl_up_sync(0xffffffffu, incl, o);
            if (lane >= o) incl += x;
        }
        if (lane == 31) s_scan[warp] = incl;
        __syncthreads();
        long long before = 0, total = 0;
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            if (w < warp) before += s_scan[w];
            total += s_scan[w];
        }
        per = (total + a.grid - 1) / a.grid;
        start = per * blockIdx.x;
        end = min(total, start + per);
        long long base = before + incl - mine;
        if (blockIdx.x == 0) {                           // for the second kernel
            if (tid == 0) { a.plan[0] = per; a.plan[a.B + 1] = total; }
            long long x = base;
            for (int b = b0; b < b1; ++b) { a.plan[1 + b] = x; x += (long long)seq_of(a, b).nt * HR; }
        }
        if (start >= end) return;
        if (start >= base && start < base + mine) {
            int b = b0;
            for (;; ++b) {
                const long long n = (long long)seq_of(a, b).nt * HR;
                if (start < base + n) break;
                base += n;
            }
            s_first[0] = b;
            s_first[1] = start - base;
        }
        __syncthreads();
        P.b = (int)s_first[0];
        P.s = seq_of(a, P.b);
        const long long in = s_first[1];
        P.hr = (int)(in / P.s.nt);
        P.t = (int)(in - (long long)P.hr * P.s.nt);
    }
    const int count = (int)(end - start);
    if (tid == 0 && a.status) {
        const int len = __ldg(a.lens + P.b);
        if (len < 0 || len > a.max_len) atomicOr(a.status + P.b, MTAD_ST_KV_OVERFLOW);
    }
    Cursor C = P;

    // ---- copies: a warp brings rows 16 * warp .. + 15 of a tile (with MT = 1 the rows that it multiplies)
    // offset of the row of this lane (lanes 0 .. 15) in the next tile to be copied, -1: nothing there (zeros instead)
    auto look_up = [&](const Cursor& c) -> long long {
        const int slot = (c.t < c.s.ns ? c.t : c.t + c.s.skip) * TK + warp * RW + (lane & 15);
        const int hi = c.s.len - 1, lo = c.s.len - c.s.nb - a.window;     // the slots that some row sees
        if (slot > hi || (a.window > 0 && slot >= a.sinks && slot <= lo)) return -1;
        const long long off = slot_offset(a.kv, a.kv.table + (long long)c.b * a.kv.table_stride, slot);
        if (off < 0 && a.status) atomicOr(a.status + c.b, MTAD_ST_RANGE);
        return off < 0 ? off : off + (long long)(c.hr / a.RB) * a.kv.head_stride;
    };
    auto copy = [&](long long off, int stage) {
        const uint32_t dk = sm + stage * 2 * L::BYTES, dv = dk + L::BYTES;
        if constexpr (CH <= 32) {
#pragma unroll
            for (int p = 0; p < RW / PASS; ++p) {
                const int rr = p * PASS + lane / CH, c = lane % CH, r = warp * RW + rr;
                const long long o = __shfl_sync(0xffffffffu, off, rr);
                const bool there = o >= 0 && c < chunks;
                const long long e = there ? o + c * 8 : 0;
                cp16(dk + L::at(r, c), a.kv.k + e, there);
                cp16(dv + L::at(r, c), a.kv.v + e, there);
            }
        }
    };
    int ahead = 0;                                        // tiles handed to the copies
    long long off = look_up(P);
#pragma unroll
    for (int s = 0; s < S - 1; ++s) {
        if (ahead < count) {
            copy(off, s);
            if (++ahead < count) { advance(a, P); off = look_up(P); }
        }
        cp_commit();
    }

    // ---- the queries of a (sequence, KV head, row block)
    int rows = 0, m0 = 0;                                 // valid query rows of the block, its first row
    int pos_a = 0, pos_b = 0;                             // last visible slot of this thread's two rows, -1: no such row
    auto load_q = [&]() {
        const int h = C.hr / a.RB, rb = C.hr - h * a.RB;
        m0 = rb * a.rows_block;
        rows = min(C.s.nb * a.G - m0, MT * 16);           // (may be < 0: a block of rows that this sequence does not have)
        const uint16_t* q = a.q + (long long)C.b * a.q_sb;
        for (int i = tid; i < MT * 16 * CH; i += NT) {
            const int m = i / CH, c = i - m * CH;
            uint4 w = make_uint4(0u, 0u, 0u, 0u);
            if (m < rows && c < chunks) {
                const int r = (m0 + m) / a.G, hq = h * a.G + (m0 + m) - r * a.G;
                w = __ldg(reinterpret_cast<const uint4*>(q + (long long)r * a.q_sr + (long long)hq * a.q_sh + c * 8));
            }
            asm volatile("st.shared.v4.b32 [%0], {%1,%2,%3,%4};" ::"r"(sm_q + L::at(m, c)), "r"(w.x), "r"(w.y), "r"(w.z), "r"(w.w) : "memory");
        }
        const int ma = wm * 16 + g, mb = ma + 8;
        pos_a = ma < rows ? C.s.len - C.s.nb + (m0 + ma) / a.G : -1;
        pos_b = mb < rows ? C.s.len - C.s.nb + (m0 + mb) / a.G : -1;
        __syncthreads();
    };
    load_q();

    float o[HD / 8][4];
    float m_a = -CUDART_INF_F, m_b = -CUDART_INF_F, l_a = 0.f, l_b = 0.f;
#pragma unroll
    for (int n = 0; n < HD / 8; ++n) o[n][0] = o[n][1] = o[n][2] = o[n][3] = 0.f;

    int stage = 0;
    int first_t = C.t;                                    // tile at which this block entered the head
    for (int i = 0; i < count; ++i) {
        cp_wait<S - 2>();
        if constexpr (MT == 1) __syncwarp(); else __syncthreads();
        {
            int into = stage + S - 1;
            if (into >= S) into -= S;
            if (ahead < count) {
                copy(off, into);
                if (++ahead < count) { advance(a, P); off = look_up(P); }
            }
            cp_commit();
        }
        const uint32_t tk = sm + stage * 2 * L::BYTES, tv = tk + L::BYTES;
        if (++stage == S) stage = 0;
        const int j0 = (C.t < C.s.ns ? C.t : C.t + C.s.skip) * TK;
        const int first_pos = C.s.len - C.s.nb, last_pos = C.s.len - 1;
        // every slot of the tile is visible to every row
        const bool inner = j0 + TK - 1 <= first_pos && (a.window <= 0 || j0 + TK <= a.sinks || j0 > last_pos - a.window);
        auto sees = [&](int j, int pos) { return j <= pos && (a.window <= 0 || j > pos - a.window || j < a.sinks); };

        // ---- scores of 16 rows x WK keys
        float s[WK / 8][4];
#pragma unroll
        for (int n = 0; n < WK / 8; ++n) s[n][0] = s[n][1] = s[n][2] = s[n][3] = 0.f;
#pragma unroll
        for (int ks = 0; ks < HD / 16; ++ks) {
            uint32_t qa[4];
            ldsm4(qa, sm_q + L::at(wm * 16 + (lane & 15), ks * 2 + (lane >> 4)));
#pragma unroll
            for (int n = 0; n < WK / 8; n += 2) {
                uint32_t kb[4];
                ldsm4(kb, tk + L::at(wk * WK + (n + (lane >> 4)) * 8 + (lane & 7), ks * 2 + ((lane >> 3) & 1)));
                mma<T>(s[n], qa, kb[0], kb[1]);
                mma<T>(s[n + 1], qa, kb[2], kb[3]);
            }
        }
        float x_a = -CUDART_INF_F, x_b = -CUDART_INF_F;
#pragma unroll
        for (int n = 0; n < WK / 8; ++n) {
#pragma unroll
            for (int e = 0; e < 4; ++e) s[n][e] *= a.scale2;
            if (!inner) {
                const int j = j0 + wk * WK + n * 8 + t2;
                if (!sees(j, pos_a)) s[n][0] = -CUDART_INF_F;
                if (!sees(j + 1, pos_a)) s[n][1] = -CUDART_INF_F;
                if (!sees(j, pos_b)) s[n][2] = -CUDART_INF_F;
                if (!sees(j + 1, pos_b)) s[n][3] = -CUDART_INF_F;
            }
            x_a = fmaxf(x_a, fmaxf(s[n][0], s[n][1]));
            x_b = fmaxf(x_b, fmaxf(s[n][2], s[n][3]));
        }
        if (a.scores) {
            float* row = a.scores + (((long long)C.b * a.kv.Hkv + C.hr / a.RB) * (a.RB * a.rows_block) + m0 + wm * 16 + g) * a.score_ld +
                         j0 + wk * WK + t2;
#pragma unroll
            for (int n = 0; n < WK / 8; ++n) {
                if (pos_a >= 0) *reinterpret_cast<float2*>(row + n * 8) = make_float2(s[n][0], s[n][1]);
                if (pos_b >= 0) *reinterpret_cast<float2*>(row + 8 * a.score_ld + n * 8) = make_float2(s[n][2], s[n][3]);
            }
        }
#pragma unroll
        for (int d = 1; d < 4; d <<= 1) {
            x_a = fmaxf(x_a, __shfl_xor_sync(0xffffffffu, x_a, d));
            x_b = fmaxf(x_b, __shfl_xor_sync(0xffffffffu, x_b, d));
        }
        if (__any_sync(0xffffffffu, x_a > m_a || x_b > m_b)) {            // (few tiles raise the maximum)
            const float n_a = fmaxf(m_a, x_a), n_b = fmaxf(m_b, x_b);
            const float f_a = m_a == n_a ? 1.f : ex2(m_a - n_a), f_b = m_b == n_b ? 1.f : ex2(m_b - n_b);
            m_a = n_a; m_b = n_b;
            l_a *= f_a; l_b *= f_b;
#pragma unroll
            for (int n = 0; n < HD / 8; ++n) { o[n][0] *= f_a; o[n][1] *= f_a; o[n][2] *= f_b; o[n][3] *= f_b; }
        }
        const float r_a = m_a == -CUDART_INF_F ? 0.f : m_a, r_b = m_b == -CUDART_INF_F ? 0.f : m_b;
#pragma unroll
        for (int n = 0; n < WK / 8; ++n) {
            s[n][0] = ex2(s[n][0] - r_a); s[n][1] = ex2(s[n][1] - r_a);
            s[n][2] = ex2(s[n][2] - r_b); s[n][3] = ex2(s[n][3] - r_b);
            l_a += s[n][0] + s[n][1];
            l_b += s[n][2] + s[n][3];
        }
        // ---- values that only some rows see: an infinity or NaN among them must not reach the others as 0 * inf.  Such a value
        // row is added to the rows that see it by hand and zeroed for the product.
        if (!inner && C.s.nb > 1) {
            bool odd = false;                             // a non-finite value in a row of this warp's share that not all see
            for (int r = lane; r < RW; r += 32) {
                const int j = j0 + warp * RW + r;
                if (j <= last_pos && !(sees(j, first_pos) && sees(j, last_pos)))
                    for (int c = 0; c < chunks; ++c) {
                        uint32_t w[4];
                        asm volatile("ld.shared.v4.b32 {%0,%1,%2,%3}, [%4];" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "r"(tv + L::at(warp * RW + r, c)));
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            odd = odd || (w[e] & Num<T>::kExp) == Num<T>::kExp || ((w[e] >> 16) & Num<T>::kExp) == Num<T>::kExp;
                    }
            }
            const bool any = MT == 1 ? __any_sync(0xffffffffu, odd) : __syncthreads_or(odd);
            if (any) {
#pragma unroll
                for (int k8 = 0; k8 < WK / 8; ++k8)
#pragma unroll 1
                    for (int e = 0; e < 8; ++e) {
                        const int kk = k8 * 8 + e, j = j0 + wk * WK + kk;
                        if (j > last_pos || (sees(j, first_pos) && sees(j, last_pos))) continue;
                        const int from = (lane & ~3) | (e >> 1);
                        const float p_a = __shfl_sync(0xffffffffu, (e & 1) ? s[k8][1] : s[k8][0], from);
                        const float p_b = __shfl_sync(0xffffffffu, (e & 1) ? s[k8][3] : s[k8][2], from);
                        const bool see_a = sees(j, pos_a), see_b = sees(j, pos_b);
#pragma unroll
                        for (int n = 0; n < HD / 8; ++n) {
                            uint32_t w;
                            asm volatile("ld.shared.b32 %0, [%1];" : "=r"(w) : "r"(tv + L::at(wk * WK + kk, n) + t2 * 2));
                            const float2 v = Num<T>::unpack(w);
                            if (see_a) { o[n][0] += p_a * v.x; o[n][1] += p_a * v.y; }
                            if (see_b) { o[n][2] += p_b * v.x; o[n][3] += p_b * v.y; }
                        }
                    }
                if constexpr (MT == 1) __syncwarp(); else __syncthreads();
                for (int r = 0; r < RW; ++r) {
                    const int j = j0 + warp * RW + r;
                    if (j > last_pos || (sees(j, first_pos) && sees(j, last_pos))) continue;
                    for (int c = lane; c < CH; c += 32)
                        asm volatile("st.shared.v4.b32 [%0], {%1,%1,%1,%1};" ::"r"(tv + L::at(warp * RW + r, c)), "r"(0u) : "memory");
                }
                if constexpr (MT == 1) __syncwarp(); else __syncthreads();
            }
        }
        // ---- o += P V, P as two terms
#pragma unroll
        for (int ks = 0; ks < WK / 16; ++ks) {
            uint32_t ph[4], pl[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float u = s[2 * ks + (e >> 1)][(e & 1) * 2], v = s[2 * ks + (e >> 1)][(e & 1) * 2 + 1];
                ph[e] = Num<T>::pack(u, v);
                const float2 h = Num<T>::unpack(ph[e]);
                pl[e] = Num<T>::pack(u - h.x, v - h.y);
            }
#pragma unroll
            for (int n = 0; n < HD / 8; n += 2) {
                uint32_t vb[4];
                ldsm4t(vb, tv + L::at(wk * WK + ks * 16 + (lane & 15), n + (lane >> 4)));
                mma<T>(o[n], ph, vb[0], vb[1]);
                mma<T>(o[n + 1], ph, vb[2], vb[3]);
                mma<T>(o[n], pl, vb[0], vb[1]);
                mma<T>(o[n + 1], pl, vb[2], vb[3]);
            }
        }

        // ---- end of the head, or of this block's share of it
        const bool last = i + 1 == count, head_end = C.t + 1 == C.s.nt;
        if (!last && !head_end) { ++C.t; continue; }
        const bool cut = first_t != 0 || !head_end;
        // (a block's first piece goes to its place 0, one that begins inside its share to place 1)
        const long long place = 2ll * blockIdx.x + (i - (C.t - first_t) > 0 ? 1 : 0);
#pragma unroll
        for (int d = 1; d < 4; d <<= 1) {
            l_a += __shfl_xor_sync(0xffffffffu, l_a, d);
            l_b += __shfl_xor_sync(0xffffffffu, l_b, d);
        }
        if (KW > 1) {
            if ((lane & 3) == 0) {
                s_m[warp][g] = m_a; s_m[warp][g + 8] = m_b;
                s_l[warp][g] = l_a; s_l[warp][g + 8] = l_b;
            }
            __syncthreads();
            float n_a = m_a, n_b = m_b;
#pragma unroll
            for (int w = 0; w < KW; ++w) { n_a = fmaxf(n_a, s_m[w * MT + wm][g]); n_b = fmaxf(n_b, s_m[w * MT + wm][g + 8]); }
            float t_a = 0.f, t_b = 0.f;
#pragma unroll
            for (int w = 0; w < KW; ++w) {
                const float wa = s_m[w * MT + wm][g], wb = s_m[w * MT + wm][g + 8];
                t_a += s_l[w * MT + wm][g] * (wa == n_a ? 1.f : ex2(wa - n_a));
                t_b += s_l[w * MT + wm][g + 8] * (wb == n_b ? 1.f : ex2(wb - n_b));
            }
            const float f_a = m_a == n_a ? 1.f : ex2(m_a - n_a), f_b = m_b == n_b ? 1.f : ex2(m_b - n_b);
#pragma unroll
            for (int n = 0; n < HD / 8; ++n) { o[n][0] *= f_a; o[n][1] *= f_a; o[n][2] *= f_b; o[n][3] *= f_b; }
            m_a = n_a; m_b = n_b; l_a = t_a; l_b = t_b;
            // the warps over the keys add their outputs one after the other (of 32 rows, half the columns at a time)
            constexpr int NB = HD / 8 / MT;
#pragma unroll
            for (int cb = 0; cb < MT; ++cb)
#pragma unroll
                for (int w = 0; w < KW; ++w) {
                    if (wk == w) {
                        float* ra = obuf + (wm * 16 + g) * (NB * 8) + t2;
                        float* rb = ra + 8 * (NB * 8);
#pragma unroll
                        for (int k = 0; k < NB; ++k) {
                            const int n = cb * NB + k;
                            if (w > 0) {
                                const float2 u = *reinterpret_cast<float2*>(ra + k * 8), v = *reinterpret_cast<float2*>(rb + k * 8);
                                o[n][0] += u.x; o[n][1] += u.y; o[n][2] += v.x; o[n][3] += v.y;
                            }
                            if (w + 1 < KW) {
                                *reinterpret_cast<float2*>(ra + k * 8) = make_float2(o[n][0], o[n][1]);
                                *reinterpret_cast<float2*>(rb + k * 8) = make_float2(o[n][2], o[n][3]);
                            }
                        }
                    }
                    __syncthreads();
                }
        }
        if (wk == KW - 1) {
            const int h = C.hr / a.RB;
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                const int m = wm * 16 + g + half * 8;
                const float mm = half ? m_b : m_a, ll = half ? l_b : l_a;
                if (m < rows) {
                    if (cut) {
                        float* dst = a.part_o + (place * a.rows_block + m) * HD + t2;
#pragma unroll
                        for (int n = 0; n < HD / 8; ++n) *reinterpret_cast<float2*>(dst + n * 8) = make_float2(o[n][half * 2], o[n][half * 2 + 1]);
                    } else {
                        const int r = (m0 + m) / a.G, hq = h * a.G + (m0 + m) - r * a.G;
                        uint16_t* dst = a.out + (long long)C.b * a.o_sb + (long long)r * a.o_sr + (long long)hq * a.o_sh + t2;
                        const float inv = ll > 0.f ? 1.f / ll : (ll == 0.f ? 0.f : ll);       // (NaN stays NaN)
#pragma unroll
                        for (int n = 0; n < HD / 8; ++n)
                            if (n < chunks)
                                *reinterpret_cast<uint32_t*>(dst + n * 8) = Num<T>::pack(o[n][half * 2] * inv, o[n][half * 2 + 1] * inv);
                        if (a.lse && (lane & 3) == 0)
                            a.lse[((long long)C.b * a.R + r) * (a.kv.Hkv * a.G) + hq] = (mm + log2f(ll)) * 0.6931471805599453f;
                        if (a.weights && (lane & 3) == 0)
                            a.row_lse2[((long long)C.b * HR + C.hr) * a.rows_block + m] = mm + log2f(ll);
                    }
                    if (cut && (lane & 3) == 0) a.part_ml[place * a.rows_block + m] = make_float2(mm, ll);
                }
            }
        }
        if (last) break;
        advance(a, C);
        first_t = 0;
        m_a = m_b = -CUDART_INF_F;
        l_a = l_b = 0.f;
#pragma unroll
        for (int n = 0; n < HD / 8; ++n) o[n][0] = o[n][1] = o[n][2] = o[n][3] = 0.f;
        if (tid == 0 && a.status) {
            const int len = __ldg(a.lens + C.b);
            if (len < 0 || len > a.max_len) atomicOr(a.status + C.b, MTAD_ST_KV_OVERFLOW);
        }
        __syncthreads();                                  // the old queries are no longer read
        load_q();
    }
}

// ---- what the blocks left of heads that were cut, and the weights

struct Pieces {                      // the shares that hold a head's tiles
    long long per, s, c0;
    int n;
};
__device__ __forceinline__ Pieces pieces_of(const AttnArgs& a, const Seq& q, int b, int hr) {
    Pieces p;
    if (a.whole) return Pieces{1, 0, 0, 1};
    p.per = a.plan[0];
    p.s = a.plan[1 + b] + (long long)hr * q.nt;
    p.c0 = p.s / p.per;
    p.n = (int)((p.s + q.nt - 1) / p.per - p.c0) + 1;
    return p;
}
__device__ __forceinline__ long long place_of(const Pieces& p, int i) {
    return 2 * (p.c0 + i) + (i == 0 && p.s > p.c0 * p.per ? 1 : 0);
}
// largest maximum and the sum relative to it of row m, over the pieces (a warp)
__device__ __forceinline__ float2 joined(const AttnArgs& a, const Pieces& p, int m, int lane) {
    float mx = -CUDART_INF_F, sum = 0.f;
    for (int i = lane; i < p.n; i += 32) mx = fmaxf(mx, a.part_ml[place_of(p, i) * a.rows_block + m].x);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, o));
    for (int i = lane; i < p.n; i += 32) {
        const float2 ml = a.part_ml[place_of(p, i) * a.rows_block + m];
        sum += ml.y * (ml.x == mx ? 1.f : ex2(ml.x - mx));
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    return make_float2(mx, sum);
}

constexpr int W_KEYS = 512;          // slots of a block that adds weights

// Blocks [0, n_join): a warp per query row adds the pieces of its output.  Blocks beyond: the weights of W_KEYS slots of a KV head,
// exp(score - lse) summed over the rows and the heads of the group and added to what is there.
template <typename T, int HD>
__global__ void __launch_bounds__(NT) join_kernel(const AttnArgs a, int n_join, int groups) {
    constexpr int PER = HD / 32;     // columns of a lane
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, HR = a.kv.Hkv * a.RB;
    __shared__ float s_lse[MAX_ROWS_BLOCK];
    pdl_wait();
    if ((int)blockIdx.x < n_join) {
        const int seg = blockIdx.x / groups, m = (blockIdx.x - seg * groups) * 4 + warp, b = seg / HR, hr = seg - b * HR;
        const Seq q = seq_of(a, b);
        const int h = hr / a.RB, row = (hr - h * a.RB) * a.rows_block + m;
        if (q.nt == 0 || m >= a.rows_block || row >= q.nb * a.G) return;
        const Pieces p = pieces_of(a, q, b, hr);
        if (p.n == 1) return;
        const float2 ml = joined(a, p, m, lane);
        float acc[PER];
#pragma unroll
        for (int k = 0; k < PER; ++k) acc[k] = 0.f;
#pragma unroll 4
        for (int i = 0; i < p.n; ++i) {
            const long long at = place_of(p, i) * a.rows_block + m;
            const float mi = a.part_ml[at].x, f = mi == ml.x ? 1.f : ex2(mi - ml.x);
            const float* src = a.part_o + at * HD + lane * PER;
#pragma unroll
            for (int k = 0; k < PER; k += 2) {
                const float2 x = *reinterpret_cast<const float2*>(src + k);
                acc[k] += f * x.x;
                acc[k + 1] += f * x.y;
            }
        }
        const int r = row / a.G, hq = h * a.G + row - r * a.G;
        const float inv = ml.y > 0.f ? 1.f / ml.y : (ml.y == 0.f ? 0.f : ml.y);
        if (lane * PER < a.kv.hd) {
            uint16_t* dst = a.out + (long long)b * a.o_sb + (long long)r * a.o_sr + (long long)hq * a.o_sh + lane * PER;
#pragma unroll
            for (int k = 0; k < PER; k += 2) *reinterpret_cast<uint32_t*>(dst + k) = Num<T>::pack(acc[k] * inv, acc[k + 1] * inv);
        }
        if (a.lse && lane == 0) a.lse[((long long)b * a.R + r) * (a.kv.Hkv * a.G) + hq] = (ml.x + log2f(ml.y)) * 0.6931471805599453f;
        return;
    }
    const int per_head = (a.max_len + W_KEYS - 1) / W_KEYS, w = blockIdx.x - n_join, bh = w / per_head, b = bh / a.kv.Hkv, h = bh - b * a.kv.Hkv;
    const int k0 = (w - bh * per_head) * W_KEYS;
    const Seq q = seq_of(a, b);
    if (q.nt == 0 || k0 >= q.len) return;
    // slots of tiles that no row sees have no scores
    bool there[4];
    float acc[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const int j = k0 + k * NT + tid, t = j / TK;
        there[k] = j < q.len && (t < q.ns || t >= q.ns + q.skip);
        acc[k] = 0.f;
    }
    if (!__syncthreads_or(there[0] || there[1] || there[2] || there[3])) return;
    for (int rb = 0; rb < a.RB; ++rb) {
        const int hr = h * a.RB + rb, rows = min(q.nb * a.G - rb * a.rows_block, a.rows_block);
        if (rows <= 0) break;
        const Pieces p = pieces_of(a, q, b, hr);
        __syncthreads();
        if (p.n == 1) {
            if (tid < rows) s_lse[tid] = a.row_lse2[((long long)b * HR + hr) * a.rows_block + tid];
        } else {
            for (int m = warp; m < rows; m += 4) {
                const float2 ml = joined(a, p, m, lane);
                if (lane == 0) s_lse[m] = ml.x + log2f(ml.y);
            }
        }
        __syncthreads();
        const float* z = a.scores + ((long long)bh * (a.RB * a.rows_block) + rb * a.rows_block) * a.score_ld + k0 + tid;
#pragma unroll 4
        for (int m = 0; m < rows; ++m) {
            const float lse = s_lse[m];
            if (lse == -CUDART_INF_F) continue;           // (a row that sees nothing)
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if (there[k]) acc[k] += ex2(z[(long long)m * a.score_ld + k * NT] - lse);
        }
    }
    float* dst = a.weights + (long long)b * a.w_sb + (long long)h * a.w_sh + k0 + tid;
#pragma unroll
    for (int k = 0; k < 4; ++k)
        if (there[k]) dst[k * NT] += acc[k];
}

// ---- host

struct Carve {
    size_t off = 0;
    size_t take(size_t bytes) {
        const size_t at = off;
        off += (bytes + 255) & ~(size_t)255;
        return at;
    }
};
struct AttnPlan {
    AttnArgs a;
    int HD, MT, grid;
    long long max_tiles;
    size_t plan, part_o, part_ml, row_lse2, scores, bytes;
};

int make_plan(const mtad_paged_kv* kv, const mtad_paged_attn* c, AttnPlan* p) {
    AttnArgs& a = p->a;
    a = AttnArgs{};
    if (!c) return MTAD_E_INVALID;
    const int rc = paged_view(kv, &a.kv);
    if (rc != MTAD_OK) return rc;
    if (!c->q || !c->out || !c->lens || c->batch < 1 || c->rows < 1 || c->n_q_heads < 1) return MTAD_E_INVALID;
    if (c->n_q_heads % kv->n_kv_heads || c->window < 0 || c->sinks < 0 || c->max_len < 1) return MTAD_E_INVALID;
    if (!isfinite(c->scale)) return MTAD_E_INVALID;
    if (c->batch > MTAD_PAGED_MAX_BATCH || c->rows > MTAD_MAX_NODES + 1 || c->n_q_heads > MTAD_PAGED_MAX_HEADS) return MTAD_E_CAPACITY;
    if ((reinterpret_cast<uintptr_t>(c->q) | reinterpret_cast<uintptr_t>(c->out)) & 15) return MTAD_E_INVALID;
    const int64_t st[6] = {c->q_stride_seq, c->q_stride_row, c->q_stride_head, c->out_stride_seq, c->out_stride_row, c->out_stride_head};
    for (int i = 0; i < 6; ++i)
        if (st[i] < 0 || st[i] % 8) return MTAD_E_INVALID;
    if (c->weights && (c->weights_stride_seq < 0 || c->weights_stride_head < 0)) return MTAD_E_INVALID;
    a.lens = c->lens; a.n_rows = c->n_rows;
    a.q = static_cast<const uint16_t*>(c->q); a.out = static_cast<uint16_t*>(c->out); a.lse = c->lse;
    a.q_sb = st[0]; a.q_sr = st[1]; a.q_sh = st[2]; a.o_sb = st[3]; a.o_sr = st[4]; a.o_sh = st[5];
    a.status = c->status;
    a.B = c->batch; a.R = c->rows; a.G = c->n_q_heads / kv->n_kv_heads;
    a.window = c->window; a.sinks = c->window > 0 ? c->sinks : 0;
    a.max_len = (int)std::min((long long)c->max_len, (long long)kv->max_pages * kv->page_size);
    if (a.window >= a.max_len) a.window = a.sinks = 0;    // (every slot is inside it)
    a.scale2 = (float)((c->scale > 0.f ? (double)c->scale : 1.0 / sqrt((double)kv->head_dim)) * 1.4426950408889634);
    a.weights = c->weights; a.w_sb = c->weights_stride_seq; a.w_sh = c->weights_stride_head;
    p->HD = kv->head_dim <= 64 ? 64 : kv->head_dim <= 128 ? 128 : 256;
    const int M = a.R * a.G;
    p->MT = M <= 16 ? 1 : M <= 32 ? 2 : 4;
    a.rows_block = 16 * p->MT;
    a.RB = (M + a.rows_block - 1) / a.rows_block;
    long long tiles = (a.max_len + TK - 1) / TK;
    if (a.window > 0) {
        const long long some = (long long)(a.sinks + TK - 1) / TK + ((long long)a.window + a.R + TK - 2) / TK + 1;
        tiles = some < tiles ? some : tiles;
    }
    p->max_tiles = tiles;
    const long long heads = (long long)a.B * a.kv.Hkv * a.RB;
    if (heads * tiles > 0x7fffffffll || heads * ((a.max_len + W_KEYS - 1) / W_KEYS) + heads * 16 > 0x7fffffffll) return MTAD_E_CAPACITY;
    a.whole = tiles <= WHOLE_TILES;
    // (workspace sizes are asked for without a device: the largest grid that the kernels run with)
    int sms = 148, dev = 0;
    if (cudaGetDevice(&dev) == cudaSuccess) {
        if (cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) sms = 148;
    }
    const long long fill = (long long)sms * (p->HD == 256 ? 1 : 2);
    p->grid = (int)(a.whole ? heads : heads * tiles < fill ? heads * tiles : fill);
    a.grid = p->grid;
    Carve w;
    p->plan = w.take(a.whole ? 0 : sizeof(long long) * (a.B + 2));
    p->part_o = w.take(a.whole ? 0 : sizeof(float) * 2 * (size_t)p->grid * a.rows_block * p->HD);
    p->part_ml = w.take(a.whole ? 0 : sizeof(float2) * 2 * (size_t)p->grid * a.rows_block);
    a.score_ld = a.weights ? (long long)((a.max_len + TK - 1) / TK) * TK : 0;
    p->row_lse2 = w.take(a.weights ? sizeof(float) * heads * a.rows_block : 0);
    p->scores = w.take(a.weights ? sizeof(float) * (size_t)heads * a.rows_block * a.score_ld : 0);
    p->bytes = w.off;
    return MTAD_OK;
}

template <typename T, int HD, int MT>
cudaError_t launch_attn(const AttnPlan& p, cudaStream_t st) {
    constexpr int smem = attn_smem<HD, MT>();
    cudaError_t e = ops_smem<attn_kernel<T, HD, MT>>(smem);
    if (e != cudaSuccess) return e;
    attn_kernel<T, HD, MT><<<p.grid, NT, smem, st>>>(p.a);
    return cudaGetLastError();
}
template <typename T, int HD>
cudaError_t launch_hd(const AttnPlan& p, cudaStream_t st) {
    cudaError_t e = p.MT == 1 ? launch_attn<T, HD, 1>(p, st) : p.MT == 2 ? launch_attn<T, HD, 2>(p, st) : launch_attn<T, HD, 4>(p, st);
    if (e != cudaSuccess) return e;
    mtad_ops_count(1);
    const int groups = (min(p.a.R * p.a.G, p.a.rows_block) + 3) / 4;
    const int join = p.a.whole ? 0 : p.a.B * p.a.kv.Hkv * p.a.RB * groups;
    const int add = p.a.weights ? p.a.B * p.a.kv.Hkv * ((p.a.max_len + W_KEYS - 1) / W_KEYS) : 0;
    if (join + add == 0) return cudaSuccess;
    mtad_ops_count(1);
    return launch_pdl(join_kernel<T, HD>, dim3(join + add), dim3(NT), 0, st, true, p.a, join, groups);
}
template <typename T>
cudaError_t launch_t(const AttnPlan& p, cudaStream_t st) {
    return p.HD == 64 ? launch_hd<T, 64>(p, st) : p.HD == 128 ? launch_hd<T, 128>(p, st) : launch_hd<T, 256>(p, st);
}

}  // namespace

}  // namespace mtad

using namespace mtad;

extern "C" {

int mtad_paged_attention_workspace(const mtad_paged_kv* kv, const mtad_paged_attn* call, size_t* out_bytes) {
    if (!out_bytes) return MTAD_E_INVALID;
    AttnPlan p;
    const int rc = make_plan(kv, call, &p);
    if (rc == MTAD_OK) *out_bytes = p.bytes;
    return rc;
}

int mtad_paged_attention(const mtad_paged_kv* kv, const mtad_paged_attn* call, void* workspace, size_t workspace_bytes, void* stream) {
    AttnPlan p;
    const int rc = make_plan(kv, call, &p);
    if (rc != MTAD_OK) return rc;
    if (p.bytes && (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255) || workspace_bytes < p.bytes)) return MTAD_E_WORKSPACE;
    char* w = static_cast<char*>(workspace);
    p.a.plan = reinterpret_cast<long long*>(w + p.plan);
    p.a.part_o = reinterpret_cast<float*>(w + p.part_o);
    p.a.part_ml = reinterpret_cast<float2*>(w + p.part_ml);
    p.a.row_lse2 = reinterpret_cast<float*>(w + p.row_lse2);
    p.a.scores = p.a.weights ? reinterpret_cast<float*>(w + p.scores) : nullptr;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    return ops_status(kv->dtype == MTAD_BF16 ? launch_t<__nv_bfloat16>(p, st) : launch_t<__half>(p, st));
}

}  // extern "C"
