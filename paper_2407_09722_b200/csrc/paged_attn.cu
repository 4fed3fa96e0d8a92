// Attention of the new rows of every sequence over a cache kept in pages.
//
//     out[r, h] = sum_j p_j V[j],   p = softmax_j(scale * q[r, h] . K[j]) over the slots j that row r sees:
//     j <= pos_r,  and with a window  j > pos_r - window  or  j < sinks;   pos_r = length - rows + r
//
// What bounds it: a call reads the visible keys and values once (2 * 2 * head_dim bytes per token and KV head) and does 4 *
// head_dim operations per query row with them, a few dozen per byte at most, so HBM bounds it and the tensor cores idle; at
// short lengths launches and latency do.  Hence mma.sync tiles (m16n8k16) straight from shared memory to registers, not tcgen05:
// tensor memory would add two trips per tile and nothing waits for the products.
//  - The query rows of a KV head (rows x heads of the group) share one pass over its keys.  Up to 16 of them (Narrow) keys stand on the
//    M side; 17 to 64 (Wide) the queries do; more are cut into blocks of 64 rows, each with a pass of its own.
//  - Long or ragged batches (stream_kernel for up to 16 rows, attn_kernel with LIST beyond): the list of tiles over (sequence, KV head, row
//    block) is cut evenly over a grid that fills the GPU once.  Shares may begin and end inside a head: its pieces (reference, sum,
//    unnormalised output, all fp32) are joined by a second kernel whose launch the first one overlaps.
//  - Short contexts (attn_kernel without LIST): a cluster of up to eight blocks has a head and joins its pieces through distributed shared
//    memory, one launch and no workspace.
//  - Copies are cp.async, page ids looked up a tile ahead.  Up to 16 query rows: three stages (four for heads of 64), a warp multiplies what
//    it has copied itself and no barrier stands in between.  More rows: two stages (four for heads of 64) and a barrier a tile.
// Measured (device time, B200): 32 contexts behind a window of 4096, 64 heads on 8 of 128, 538 MB: 96 us, 5.6 TB/s (a plain read of 8 GB
// runs at 6.2); eight ragged sequences x 7 rows, 40 heads, 341 MB: 61 us, 5.6 TB/s; a chain of 5 rows at 2053 slots, 32 heads: 11 us;
// one row at 97 slots: 5.8 us.  What is left at the long ones: SMs that get a tenth less bandwidth than others for the same share (shares
// taken over from blocks not yet launched evened that out, and cost more than it gave), the second kernel (5 us), the first loads (4 us).
// Rounding: scores, statistics and sums are fp32.  Probabilities enter the second product as terms of the cache's type (p, and what
// its rounding left; see Prob), so that they keep the bits of fp32.  The tensor cores cut sums off where fp32 rounds them, so a tile's
// products have accumulators of their own and are added to the output by fp32 additions: what is cut off, always towards zero, turned six times
// as many roundings of bf16 outputs over long shares as sums that are rounded.  The output is rounded once.
#include <cooperative_groups.h>
#include <limits.h>
#include <math_constants.h>

#include <algorithm>
#include <type_traits>

#include "paged.cuh"

namespace cg = cooperative_groups;

namespace mtad {

namespace {

constexpr int TK = 64;               // keys of a tile
constexpr int NT = 128;              // threads of a block
constexpr int MAX_ROWS_BLOCK = 64;   // query rows (rows x heads of the group) of a block
constexpr int MAX_CLUSTER = 8;
// Tiles of a block up to which a cluster has a head (device time of one sequence, cluster / list, heads of 128).  8 rows a KV head, 6144 slots (12
// tiles in clusters of eight): 1 KV head 15.8 / 18.8 us, 4 16.3 / 19.1, 8 16.4 / 17.0; 8192 slots: 19.5 / 22.8, 19.9 / 22.1, 20.1 / 18.0; 16384
// slots: 34 / 38, 35 / 24, 35 / 27.  40 rows, 32 KV heads: 4096 slots 37.6 / 40.9, 8192 67.2 / 67.7, 16384 123 / 116 (two blocks a head); few heads
// would have the list from 1000 to 2000 slots on (4096 slots, 1 KV head 27.5 / 13.6, 8 27.8 / 20.7), which this rule does not know.
constexpr int CLUSTER_TILES = 12, CLUSTER_TILES_WIDE = 8;

struct AttnArgs {
    PagedView kv;
    const int32_t* lens;
    const int32_t* n_rows;           // or null: R
    const uint16_t* q;
    uint16_t* out;
    float* lse;                      // [B, R, Hq] or null
    long long q_sb, q_sr, q_sh, o_sb, o_sr, o_sh;
    uint32_t* status;
    int B, R, G, RB, rows_block;     // heads of a group, row blocks, query rows of a block
    int window, sinks, max_len;
    float scale2;                    // scale * log2(e)
    int even;                        // 16 neighbouring slots, the first a multiple of 16, lie in one page
    int dense;                       // the slot stride where it is a row's length, else 0
    int cluster;                     // blocks of a head; 0: the list is cut evenly over the grid
    int grid;
    // workspace
    int* plan;                       // [0] tiles of a share, [1 .. B] first tile of every sequence
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
template <int UNIT>
__device__ __forceinline__ Seq seq_of(const AttnArgs& a, int b) {
    Seq s;
    const int len = __ldg(a.lens + b);
    s.len = min(max(len, 0), a.max_len);
    s.nb = a.n_rows ? min(max(__ldg(a.n_rows + b), 0), a.R) : a.R;
    const int total = (s.len + UNIT - 1) / UNIT;
    s.ns = total;
    s.skip = 0;
    if (a.window > 0) {
        const int first = max(s.len - s.nb - a.window + 1, 0);          // of the first row
        const int ns = (min(a.sinks, s.len) + UNIT - 1) / UNIT;
        const int from = max(first / UNIT, ns);
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
template <int UNIT>
__device__ __forceinline__ void advance(const AttnArgs& a, Cursor& c) {
    if (++c.t < c.s.nt) return;
    c.t = 0;
    if (++c.hr < a.kv.Hkv * a.RB) return;
    c.hr = 0;
    do {
        if (++c.b >= a.B) return;
        c.s = seq_of<UNIT>(a, c.b);
    } while (c.s.nt == 0);
}

__device__ __forceinline__ void cp16(uint32_t dst, const void* src, bool there, uint64_t policy) {
    asm volatile("cp.async.cg.shared.global.L2::cache_hint [%0], [%1], 16, %2, %3;" ::"r"(dst), "l"(src), "r"(there ? 16 : 0), "l"(policy) : "memory");
}
// What is read once leaves the L2 first (a long list: 61 us instead of 65 for the ragged batch of eight); what a short call has read may be there
// when the next one asks for it, and rows in several blocks read it again.  (Pages that sequences share are taken as read once too: whether an id
// comes again is not known here.)
__device__ __forceinline__ uint64_t copy_policy(bool once) {
    uint64_t p;
    if (once) asm volatile("createpolicy.fractional.L2::evict_first.b64 %0, 1.0;" : "=l"(p));
    else asm volatile("createpolicy.fractional.L2::evict_normal.b64 %0, 1.0;" : "=l"(p));
    return p;
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
__device__ __forceinline__ uint32_t transposed(uint32_t x) {             // of an 8 x 8 block of 16-bit elements
    uint32_t y;
    asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
    return y;
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
constexpr float LN2 = 0.6931471805599453f;
// of a row's sum (times what the output is scaled by): 0 for a row that sees nothing (its output is zero), NaN stays NaN
__device__ __forceinline__ float inverse(float sum) { return sum > 0.f ? 1.f / sum : (sum == 0.f ? 0.f : sum); }
__device__ __forceinline__ float ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// of a slot for a row, from its score: none where the row does not see the slot (score -inf), also where its sum is NaN
__device__ __forceinline__ float weight(float score, float lse) { return score == -CUDART_INF_F ? 0.f : ex2(score - lse); }

// Byte offset of 16-byte piece c of row r of a tile: the pieces of eight neighbouring rows fall into different banks.  Tiles begin at
// multiples of 512 bytes, so that the pieces 2 k, 2 k + 1 of a row lie at (address of the pieces 0, 1) ^ (k << 5).
template <int HD> __device__ __forceinline__ uint32_t at(int r, int c) { return (uint32_t)(r * HD * 2 + ((c ^ (r & 7)) << 4)); }

template <int HD, int ROWS> struct Tile {
    static constexpr int CH = HD / 8;                    // 16-byte pieces of a row
    static constexpr int BYTES = TK * HD * 2;            // keys (or values) of a tile
    // two blocks on an SM (one with heads of 256): 64 to 96 KB of a block's shared memory (128 to 192) on their way or in use
    static constexpr int STAGES = HD == 64 ? 4 : ROWS <= 16 ? 3 : 2;
    static constexpr int BLOCKS = HD == 256 ? 1 : 2;
    static constexpr int MT = ROWS <= 16 ? 1 : ROWS / 16;                // warps over the rows; 4 / MT over the keys of a tile
    static constexpr int Q = ROWS <= 16 ? 0 : ROWS * HD * 2;
    static constexpr int COLS = MT;                      // parts of the columns in which the warps of a block add their outputs
    static constexpr int LDO = HD + 4, LDC = HD / COLS + 4;
    static constexpr int OBUF = ROWS * LDC * 4;
    static constexpr int SMEM = STAGES * 2 * BYTES + Q;  // and OBUF, for blocks of the list
    static_assert((4 / MT) * ROWS * LDO * 4 <= STAGES * 2 * BYTES, "the outputs of all warps fit the stages");
};

__device__ __forceinline__ bool sees(const AttnArgs& a, int j, int pos) {
    return j <= pos && (a.window <= 0 || j > pos - a.window || j < a.sinks);
}

// A tile as the cores see it
struct TileAt {
    uint32_t k, v;                   // shared memory (Narrow: of the warp's own 16 rows)
    int j0, first_pos, last_pos;     // slot of the first row there; positions of the sequence's first and last row
    bool inner, many;                // every slot is visible to every row; the sequence has several rows
};
// a slot that some rows of the sequence see and others do not
__device__ __forceinline__ bool mixed(const AttnArgs& a, const TileAt& t, int j) {
    return j <= t.last_pos && !(sees(a, j, t.first_pos) && sees(a, j, t.last_pos));
}
// whether one of the 16 value rows at `first` that only some rows see holds an infinity or a NaN (per lane)
template <typename T, int HD>
__device__ __forceinline__ bool odd_value(const AttnArgs& a, const TileAt& t, int first, int chunks, int lane) {
    bool odd = false;                                     // (a lane has every other piece of a row)
    if (mixed(a, t, t.j0 + first + (lane & 15)))
#pragma unroll 4
        for (int c = lane >> 4; c < chunks; c += 2) {
            uint32_t w[4];
            asm volatile("ld.shared.v4.b32 {%0,%1,%2,%3}, [%4];" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3])
                         : "r"(t.v + at<HD>(first + (lane & 15), c)));
#pragma unroll
            for (int e = 0; e < 4; ++e) odd = odd || (w[e] & Num<T>::kExp) == Num<T>::kExp || ((w[e] >> 16) & Num<T>::kExp) == Num<T>::kExp;
        }
    return odd;
}
template <int HD>
__device__ __forceinline__ void zero_mixed(const AttnArgs& a, const TileAt& t, int first, int lane) {
    for (int r = 0; r < 16; ++r)
        if (mixed(a, t, t.j0 + first + r))
            for (int c = lane; c < HD / 8; c += 32)
                asm volatile("st.shared.v4.b32 [%0], {%1,%1,%1,%1};" ::"r"(t.v + at<HD>(first + r, c)), "r"(0u) : "memory");
}

// Terms of the cache's type as which a probability enters the second product: three of bf16 hold the 24 bits of fp32, two of fp16 hold 22.
// (Two of bf16 left 2^-18 of a probability out, which turned the rounding of one output in 2000.  The third takes no time where memory bounds
// the call, up to 16 query rows a KV head; a chain of 5 on groups of 8, eight ragged sequences, takes 43 us instead of 38, four prompt
// chunks of 256 rows at 2000 to 4000 slots 600 instead of 498.)
//
// The reference of a row's exponentials is raised only when a score passes it by 2^RAISE: sums and outputs stay far inside fp32's range,
// and most tiles need neither a maximum over lanes nor a rescaling.
//
// fp16 has no steps below 2^-24: a probability enters (and the output is kept) times SCALE, so that the largest, 2^RAISE * SCALE, is just below
// the type's end and the steps are 2^-37 of the reference.  (As it is, 2^-25 and less vanished from the output, and many slots behind a
// dominant one with them.  A lower RAISE than that of bf16 for two bits more: 60 to 61 us for the ragged batch in fp16 either way.)
template <typename T> struct Prob;
template <> struct Prob<__nv_bfloat16> {
    static constexpr int TERMS = 3;
    static constexpr float RAISE = 6.f, SCALE = 1.f;
};
template <> struct Prob<__half> {
    static constexpr int TERMS = 2;
    static constexpr float RAISE = 2.f, SCALE = 8192.f;
};

// Up to 16 query rows: keys stand on the M side of the products, S^T = K Q^T (16 keys x 8 rows a step) and O^T = V^T P^T (16 columns x 8
// rows), so that eight rows - one token with a group of eight heads, a chain of seven - fill a tile that would be half empty with
// the queries on that side: half the tensor instructions and half the accumulators.  Every warp has 16 keys of a tile to itself.
template <typename T, int HD, int ROWS> struct Narrow {
    using L = Tile<HD, ROWS>;
    static constexpr int N8 = ROWS / 8, KW = 4;
    float o[HD / 16][N8][4];         // (column g | g + 8, row 2t | 2t + 1)
    float m[N8][2], l[N8][2];        // reference (log2 domain) and sum (of this thread's keys) of rows 2t, 2t + 1
    float over[N8][2], ref[N8][2];   // the score above which the reference is raised; the reference, 0 while there is none
    uint32_t q[HD / 16][N8][2];
    int pos[N8][2];                  // last visible slot, -1: no such row
    int g, t2, warp, lane;

    __device__ __forceinline__ void init(int tid) { lane = tid & 31; warp = tid >> 5; g = lane >> 2; t2 = (lane & 3) * 2; }
    __device__ __forceinline__ void reset() {
#pragma unroll
        for (int n = 0; n < N8; ++n) {
            m[n][0] = m[n][1] = over[n][0] = over[n][1] = -CUDART_INF_F;
            l[n][0] = l[n][1] = ref[n][0] = ref[n][1] = 0.f;
#pragma unroll
            for (int d = 0; d < HD / 16; ++d) o[d][n][0] = o[d][n][1] = o[d][n][2] = o[d][n][3] = 0.f;
        }
    }
    __device__ __forceinline__ void read_q(const AttnArgs& a, const uint16_t* base, int h, int m0, int rows) {
#pragma unroll
        for (int n = 0; n < N8; ++n) {
            const int row = n * 8 + g, r = (m0 + row) / a.G, hq = h * a.G + (m0 + row) - r * a.G;
            const uint16_t* src = base + (long long)r * a.q_sr + (long long)hq * a.q_sh + t2;
#pragma unroll
            for (int k = 0; k < HD / 16; ++k)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const int c = k * 16 + e * 8;
                    q[k][n][e] = row < rows && c < a.kv.hd ? __ldg(reinterpret_cast<const uint32_t*>(src + c)) : 0u;
                }
        }
    }
    __device__ __forceinline__ void put_q(const AttnArgs& a, uint32_t, int first_pos, int m0, int rows) {
#pragma unroll
        for (int n = 0; n < N8; ++n)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int row = n * 8 + t2 + e;
                pos[n][e] = row < rows ? first_pos + (m0 + row) / a.G : -1;
            }
    }
    __device__ __forceinline__ void tile(const AttnArgs& a, const TileAt& t, uint32_t, float* scores, int chunks) {
        float s[N8][4], s2[N8][4];   // (key g | g + 8, row 2t | 2t + 1), in two sums whose products do not wait for one another
#pragma unroll
        for (int n = 0; n < N8; ++n) s[n][0] = s[n][1] = s[n][2] = s[n][3] = s2[n][0] = s2[n][1] = s2[n][2] = s2[n][3] = 0.f;
        const uint32_t at_k = t.k + at<HD>(lane & 15, lane >> 4);
        const uint32_t at_v = t.v + at<HD>((lane >> 4) * 8 + (lane & 7), (lane >> 3) & 1);
#pragma unroll
        for (int k = 0; k < HD / 16; ++k) {
            uint32_t ka[4];
            ldsm4(ka, at_k ^ (k << 5));
#pragma unroll
            for (int n = 0; n < N8; ++n) mma<T>((k & 1) ? s2[n] : s[n], ka, q[k][n][0], q[k][n][1]);
        }
#pragma unroll
        for (int n = 0; n < N8; ++n)
#pragma unroll
            for (int e = 0; e < 4; ++e) s[n][e] += s2[n][e];
        bool raise = false;
#pragma unroll
        for (int n = 0; n < N8; ++n) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                s[n][e] *= a.scale2;
                if (!t.inner && !sees(a, t.j0 + g + (e >> 1) * 8, pos[n][e & 1])) s[n][e] = -CUDART_INF_F;
                raise = raise || s[n][e] > over[n][e & 1];
            }
            if (scores) {
                float* z = scores + (n * 8 + t2) * a.score_ld + t.j0 + g;
                if (pos[n][0] >= 0) { z[0] = s[n][0]; z[8] = s[n][2]; }
                if (pos[n][1] >= 0) { z[a.score_ld] = s[n][1]; z[a.score_ld + 8] = s[n][3]; }
            }
        }
        if (__any_sync(0xffffffffu, raise)) {
#pragma unroll
            for (int n = 0; n < N8; ++n)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    float x = fmaxf(s[n][e], s[n][e + 2]);
#pragma unroll
                    for (int d = 4; d < 32; d <<= 1) x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, d));
                    const float to = fmaxf(m[n][e], x), f = m[n][e] == to ? 1.f : ex2(m[n][e] - to);
                    m[n][e] = to;
                    over[n][e] = to + Prob<T>::RAISE;
                    ref[n][e] = to == -CUDART_INF_F ? 0.f : to;
                    l[n][e] *= f;
#pragma unroll
                    for (int d = 0; d < HD / 16; ++d) { o[d][n][e] *= f; o[d][n][e + 2] *= f; }
                }
        }
#pragma unroll
        for (int n = 0; n < N8; ++n)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                s[n][e] = ex2(s[n][e] - ref[n][e & 1]);
                l[n][e & 1] += s[n][e];
            }
        // values that only some rows see: an infinity or NaN among them must not reach the others as 0 * inf.  Such a value row
        // is added to the rows that see it by hand and zeroed for the product.
        if (!t.inner && t.many && __any_sync(0xffffffffu, odd_value<T, HD>(a, t, 0, chunks, lane))) {
#pragma unroll
            for (int half = 0; half < 2; ++half)
#pragma unroll 1
                for (int kk = 0; kk < 8; ++kk) {
                    const int r = half * 8 + kk, j = t.j0 + r;
                    if (!mixed(a, t, j)) continue;
#pragma unroll
                    for (int n = 0; n < N8; ++n)
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            const float pr = __shfl_sync(0xffffffffu, s[n][half * 2 + e], (kk << 2) | (lane & 3)) * Prob<T>::SCALE;
                            if (sees(a, j, pos[n][e]))
#pragma unroll
                                for (int d = 0; d < HD / 16; ++d)
#pragma unroll
                                    for (int up = 0; up < 2; ++up) {
                                        uint16_t w;
                                        asm volatile("ld.shared.u16 %0, [%1];" : "=h"(w) : "r"(t.v + at<HD>(r, d * 2 + up) + g * 2));
                                        o[d][n][e + 2 * up] += pr * Num<T>::unpack(w).x;
                                    }
                        }
                }
            __syncwarp();
            zero_mixed<HD>(a, t, 0, lane);
            __syncwarp();
        }
        // P^T as the products' second operand: two neighbouring rows of a key are packed and the 8 x 8 blocks transposed
        constexpr int TERMS = Prob<T>::TERMS;
        uint32_t p[TERMS][N8][2];
#pragma unroll
        for (int n = 0; n < N8; ++n)
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                float u = s[n][half * 2] * Prob<T>::SCALE, v = s[n][half * 2 + 1] * Prob<T>::SCALE;
#pragma unroll
                for (int k = 0; k < TERMS; ++k) {
                    const uint32_t w = Num<T>::pack(u, v);
                    const float2 x = Num<T>::unpack(w);
                    p[k][n][half] = transposed(w);
                    u -= x.x;
                    v -= x.y;
                }
            }
        constexpr int STEP = HD / 16 < 8 ? HD / 16 : 8;   // columns' products in flight
        constexpr bool FRESH = HD * N8 <= 256;            // (16 rows of 256 columns have no registers for it: 191 us -> 326 of nine rows at 3000 to 9000 slots)
#pragma unroll
        for (int d0 = 0; d0 < HD / 16; d0 += STEP) {
            uint32_t va[STEP][4];
#pragma unroll
            for (int d = 0; d < STEP; ++d) ldsm4t(va[d], at_v ^ ((d0 + d) << 5));
#pragma unroll
            for (int n = 0; n < N8; ++n) {
                float x[STEP][4];
#pragma unroll
                for (int d = 0; d < STEP; ++d)
#pragma unroll
                    for (int e = 0; e < 4; ++e) x[d][e] = FRESH ? 0.f : o[d0 + d][n][e];
#pragma unroll
                for (int k = TERMS - 1; k >= 0; --k)
#pragma unroll
                    for (int d = 0; d < STEP; ++d) mma<T>(x[d], va[d], p[k][n][0], p[k][n][1]);
#pragma unroll
                for (int d = 0; d < STEP; ++d)
#pragma unroll
                    for (int e = 0; e < 4; ++e) o[d0 + d][n][e] = FRESH ? o[d0 + d][n][e] + x[d][e] : x[d][e];
            }
        }
    }
    // The rows' statistics over the block's warps to s_ml; o is brought to the block's reference.
    __device__ __forceinline__ void join_warps(float2* s_part, float2* s_ml) {
#pragma unroll
        for (int n = 0; n < N8; ++n)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
#pragma unroll
                for (int d = 4; d < 32; d <<= 1) l[n][e] += __shfl_xor_sync(0xffffffffu, l[n][e], d);
                if (g == 0) s_part[warp * ROWS + n * 8 + t2 + e] = make_float2(m[n][e], l[n][e]);
            }
        __syncthreads();
#pragma unroll
        for (int n = 0; n < N8; ++n)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int row = n * 8 + t2 + e;
                float2 w[KW];
                float to = -CUDART_INF_F, sum = 0.f;
#pragma unroll
                for (int k = 0; k < KW; ++k) { w[k] = s_part[k * ROWS + row]; to = fmaxf(to, w[k].x); }
#pragma unroll
                for (int k = 0; k < KW; ++k) sum += w[k].y * (w[k].x == to ? 1.f : ex2(w[k].x - to));
                const float f = m[n][e] == to ? 1.f : ex2(m[n][e] - to);
#pragma unroll
                for (int d = 0; d < HD / 16; ++d) { o[d][n][e] *= f; o[d][n][e + 2] *= f; }
                if (warp == 0 && g == 0) s_ml[row] = make_float2(to, sum);
            }
    }
    // Sums over the lanes' keys: every lane then has the rows' sums
    __device__ __forceinline__ void join_lanes() {
#pragma unroll
        for (int n = 0; n < N8; ++n)
#pragma unroll
            for (int e = 0; e < 2; ++e)
#pragma unroll
                for (int d = 4; d < 32; d <<= 1) l[n][e] += __shfl_xor_sync(0xffffffffu, l[n][e], d);
    }
    // Puts this warp's output to buf[row][ld]
    __device__ __forceinline__ void put(float* buf, int ld, int, bool) {
#pragma unroll
        for (int d = 0; d < HD / 16; ++d)
#pragma unroll
            for (int n = 0; n < N8; ++n)
#pragma unroll
                for (int e = 0; e < 4; ++e) buf[(n * 8 + t2 + (e & 1)) * ld + d * 16 + (e >> 1) * 8 + g] = o[d][n][e];
    }
};

// 17 to 64 query rows: queries on the M side, S = Q K^T and O = P V; the warps stand MT over the rows by 4 / MT over the keys.
template <typename T, int HD, int ROWS> struct Wide {
    using L = Tile<HD, ROWS>;
    static constexpr int MT = L::MT, KW = 4 / MT, WK = TK / KW, CH = L::CH, QN = ROWS * CH / NT;
    float o[HD / 8][4];              // (row g | g + 8, columns 2t, 2t + 1)
    float m_a, m_b, l_a, l_b;        // of rows g, g + 8; sums of this thread's keys
    uint4 q[QN];
    int pos_a, pos_b;
    int g, t2, warp, lane, wm, wk, tid_;

    __device__ __forceinline__ void init(int tid) {
        tid_ = tid; lane = tid & 31; warp = tid >> 5; g = lane >> 2; t2 = (lane & 3) * 2; wm = warp % MT; wk = warp / MT;
    }
    __device__ __forceinline__ void reset() {
        m_a = m_b = -CUDART_INF_F;
        l_a = l_b = 0.f;
#pragma unroll
        for (int n = 0; n < HD / 8; ++n) o[n][0] = o[n][1] = o[n][2] = o[n][3] = 0.f;
    }
    __device__ __forceinline__ void read_q(const AttnArgs& a, const uint16_t* base, int h, int m0, int rows) {
#pragma unroll
        for (int k = 0; k < QN; ++k) {
            const int i = tid_ + k * NT, m = i / CH, c = i - m * CH;
            q[k] = make_uint4(0u, 0u, 0u, 0u);
            if (m < rows && c * 8 < a.kv.hd) {
                const int r = (m0 + m) / a.G, hq = h * a.G + (m0 + m) - r * a.G;
                q[k] = __ldg(reinterpret_cast<const uint4*>(base + (long long)r * a.q_sr + (long long)hq * a.q_sh + c * 8));
            }
        }
    }
    __device__ __forceinline__ void put_q(const AttnArgs& a, uint32_t sm_q, int first_pos, int m0, int rows) {
#pragma unroll
        for (int k = 0; k < QN; ++k) {
            const int i = tid_ + k * NT, m = i / CH, c = i - m * CH;
            asm volatile("st.shared.v4.b32 [%0], {%1,%2,%3,%4};" ::"r"(sm_q + at<HD>(m, c)), "r"(q[k].x), "r"(q[k].y), "r"(q[k].z), "r"(q[k].w)
                         : "memory");
        }
        const int ma = wm * 16 + g, mb = ma + 8;
        pos_a = ma < rows ? first_pos + (m0 + ma) / a.G : -1;
        pos_b = mb < rows ? first_pos + (m0 + mb) / a.G : -1;
    }
    __device__ __forceinline__ void tile(const AttnArgs& a, const TileAt& t, uint32_t sm_q, float* scores, int chunks) {
        float s[WK / 8][4];
#pragma unroll
        for (int n = 0; n < WK / 8; ++n) s[n][0] = s[n][1] = s[n][2] = s[n][3] = 0.f;
        const uint32_t at_q = sm_q + at<HD>(wm * 16 + (lane & 15), lane >> 4);
        const uint32_t at_k = t.k + at<HD>(wk * WK + (lane >> 4) * 8 + (lane & 7), (lane >> 3) & 1);
        const uint32_t at_v = t.v + at<HD>(wk * WK + (lane & 15), lane >> 4);
#pragma unroll
        for (int ks = 0; ks < HD / 16; ++ks) {
            uint32_t qa[4];
            ldsm4(qa, at_q ^ (ks << 5));
#pragma unroll
            for (int n = 0; n < WK / 8; n += 2) {
                uint32_t kb[4];
                ldsm4(kb, (at_k ^ (ks << 5)) + n * 8 * HD * 2);
                mma<T>(s[n], qa, kb[0], kb[1]);
                mma<T>(s[n + 1], qa, kb[2], kb[3]);
            }
        }
        float x_a = -CUDART_INF_F, x_b = -CUDART_INF_F;
#pragma unroll
        for (int n = 0; n < WK / 8; ++n) {
#pragma unroll
            for (int e = 0; e < 4; ++e) s[n][e] *= a.scale2;
            if (!t.inner) {
                const int j = t.j0 + wk * WK + n * 8 + t2;
                if (!sees(a, j, pos_a)) s[n][0] = -CUDART_INF_F;
                if (!sees(a, j + 1, pos_a)) s[n][1] = -CUDART_INF_F;
                if (!sees(a, j, pos_b)) s[n][2] = -CUDART_INF_F;
                if (!sees(a, j + 1, pos_b)) s[n][3] = -CUDART_INF_F;
            }
            x_a = fmaxf(x_a, fmaxf(s[n][0], s[n][1]));
            x_b = fmaxf(x_b, fmaxf(s[n][2], s[n][3]));
        }
        if (scores) {
            float* row = scores + (wm * 16 + g) * a.score_ld + t.j0 + wk * WK + t2;
#pragma unroll
            for (int n = 0; n < WK / 8; ++n) {
                if (pos_a >= 0) *reinterpret_cast<float2*>(row + n * 8) = make_float2(s[n][0], s[n][1]);
                if (pos_b >= 0) *reinterpret_cast<float2*>(row + 8 * a.score_ld + n * 8) = make_float2(s[n][2], s[n][3]);
            }
        }
        if (__any_sync(0xffffffffu, x_a > m_a + Prob<T>::RAISE || x_b > m_b + Prob<T>::RAISE)) {
#pragma unroll
            for (int d = 1; d < 4; d <<= 1) {
                x_a = fmaxf(x_a, __shfl_xor_sync(0xffffffffu, x_a, d));
                x_b = fmaxf(x_b, __shfl_xor_sync(0xffffffffu, x_b, d));
            }
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
        if (!t.inner && t.many && __syncthreads_or(odd_value<T, HD>(a, t, warp * 16, chunks, lane))) {     // (as in Narrow)
#pragma unroll
            for (int k8 = 0; k8 < WK / 8; ++k8)
#pragma unroll 1
                for (int e = 0; e < 8; ++e) {
                    const int kk = wk * WK + k8 * 8 + e, j = t.j0 + kk;
                    if (!mixed(a, t, j)) continue;
                    const int from = (lane & ~3) | (e >> 1);
                    const float p_a = __shfl_sync(0xffffffffu, (e & 1) ? s[k8][1] : s[k8][0], from) * Prob<T>::SCALE;
                    const float p_b = __shfl_sync(0xffffffffu, (e & 1) ? s[k8][3] : s[k8][2], from) * Prob<T>::SCALE;
                    const bool see_a = sees(a, j, pos_a), see_b = sees(a, j, pos_b);
#pragma unroll
                    for (int n = 0; n < HD / 8; ++n) {
                        uint32_t w;
                        asm volatile("ld.shared.b32 %0, [%1];" : "=r"(w) : "r"(t.v + at<HD>(kk, n) + t2 * 2));
                        const float2 v = Num<T>::unpack(w);
                        if (see_a) { o[n][0] += p_a * v.x; o[n][1] += p_a * v.y; }
                        if (see_b) { o[n][2] += p_b * v.x; o[n][3] += p_b * v.y; }
                    }
                }
            __syncthreads();
            zero_mixed<HD>(a, t, warp * 16, lane);
            __syncthreads();
        }
        constexpr int TERMS = Prob<T>::TERMS;
        uint32_t p[WK / 16][TERMS][4];
#pragma unroll
        for (int ks = 0; ks < WK / 16; ++ks)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                float u = s[2 * ks + (e >> 1)][(e & 1) * 2] * Prob<T>::SCALE, v = s[2 * ks + (e >> 1)][(e & 1) * 2 + 1] * Prob<T>::SCALE;
#pragma unroll
                for (int k = 0; k < TERMS; ++k) {
                    p[ks][k][e] = Num<T>::pack(u, v);
                    const float2 x = Num<T>::unpack(p[ks][k][e]);
                    u -= x.x;
                    v -= x.y;
                }
            }
        constexpr int STEP = HD == 256 ? 4 : 8;           // columns' products in flight (two: a chunk of 256 rows 13 % slower)
#pragma unroll
        for (int n = 0; n < HD / 8; n += STEP) {
            float x[STEP][4];
#pragma unroll
            for (int d = 0; d < STEP; ++d) x[d][0] = x[d][1] = x[d][2] = x[d][3] = 0.f;
#pragma unroll
            for (int ks = 0; ks < WK / 16; ++ks) {
                uint32_t vb[STEP / 2][4];
#pragma unroll
                for (int d = 0; d < STEP; d += 2) ldsm4t(vb[d / 2], (at_v ^ ((n + d) << 4)) + ks * 16 * HD * 2);
#pragma unroll
                for (int k = TERMS - 1; k >= 0; --k)
#pragma unroll
                    for (int d = 0; d < STEP; ++d) mma<T>(x[d], p[ks][k], vb[d / 2][(d & 1) * 2], vb[d / 2][(d & 1) * 2 + 1]);
            }
#pragma unroll
            for (int d = 0; d < STEP; ++d)
#pragma unroll
                for (int e = 0; e < 4; ++e) o[n + d][e] += x[d][e];
        }
    }
    __device__ __forceinline__ void join_warps(float2* s_part, float2* s_ml) {
#pragma unroll
        for (int d = 1; d < 4; d <<= 1) {
            l_a += __shfl_xor_sync(0xffffffffu, l_a, d);
            l_b += __shfl_xor_sync(0xffffffffu, l_b, d);
        }
        if ((lane & 3) == 0) {
            s_part[wk * ROWS + wm * 16 + g] = make_float2(m_a, l_a);
            s_part[wk * ROWS + wm * 16 + g + 8] = make_float2(m_b, l_b);
        }
        __syncthreads();
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            const int row = wm * 16 + g + half * 8;
            float2 w[KW];
            float to = -CUDART_INF_F, sum = 0.f;
#pragma unroll
            for (int k = 0; k < KW; ++k) { w[k] = s_part[k * ROWS + row]; to = fmaxf(to, w[k].x); }
#pragma unroll
            for (int k = 0; k < KW; ++k) sum += w[k].y * (w[k].x == to ? 1.f : ex2(w[k].x - to));
            const float mine = half ? m_b : m_a, f = mine == to ? 1.f : ex2(mine - to);
#pragma unroll
            for (int n = 0; n < HD / 8; ++n) { o[n][half * 2] *= f; o[n][half * 2 + 1] *= f; }
            if (wk == 0 && (lane & 3) == 0) s_ml[row] = make_float2(to, sum);
        }
    }
    // Puts (or adds) this warp's output to buf[row][ld]: all columns, or the part cb of them
    __device__ __forceinline__ void put(float* buf, int ld, int cb, bool add) {
        constexpr int NB = HD / 8 / L::COLS;
        const bool all = ld == L::LDO;                    // every column
#pragma unroll
        for (int n = 0; n < HD / 8; ++n) {
            if (!all && n / NB != cb) continue;
            float* at = buf + (wm * 16 + g) * ld + (all ? n : n - cb * NB) * 8 + t2;
#pragma unroll
            for (int half = 0; half < 2; ++half, at += 8 * ld) {
                float2 x = make_float2(o[n][half * 2], o[n][half * 2 + 1]);
                if (add) { const float2 y = *reinterpret_cast<float2*>(at); x.x += y.x; x.y += y.y; }
                *reinterpret_cast<float2*>(at) = x;
            }
        }
    }
};

// What a lane knows of its row (lane & 15) of the next 16 to be copied: the page id as it came from the table - used only when the copy is
// made, a tile later, so that nobody waits for the load - and the slot in the page; id -1: no row sees the slot (zeros instead).
struct Spot {
    int id, in;
};
__device__ __forceinline__ Spot look_up(const AttnArgs& a, const Seq& s, int b, int slot) {
    const int hi = s.len - 1, lo = s.len - s.nb - a.window;               // the slots that some row sees
    if (slot > hi || (a.window > 0 && slot >= a.sinks && slot <= lo)) return Spot{-1, 0};
    const uint32_t p = div_by((uint32_t)slot, a.kv.page);
    const int id = __ldg(a.kv.table + (long long)b * a.kv.table_stride + p);
    return Spot{id == -1 ? INT_MIN : id, slot - (int)(p * a.kv.page.d)};
}
// A warp brings 16 rows of keys and values (`apart` bytes further on) of a KV head that begins at `head` of a page.
template <int HD>
__device__ __forceinline__ void copy_rows(const AttnArgs& a, const Spot& at_, int b, long long head, uint32_t tile, int apart, int c_row, int c_col,
                                          int chunks, uint64_t policy) {
    constexpr int CH = HD / 8, PASS = 32 / CH;
    const uint32_t to = tile + c_row * HD * 2, piece = (c_col ^ c_row) << 4;      // (c_row < PASS <= 4: at() of row p * PASS + c_row)
    auto dst = [&](int p) { return to + p * PASS * HD * 2 + (piece ^ (((p * PASS) & 7) << 4)); };
    const bool there = (unsigned)at_.id < (unsigned)a.kv.n_pages;
    if (a.even && __all_sync(0xffffffffu, there)) {       // one run of a page
        const long long e = (long long)__shfl_sync(0xffffffffu, at_.id, 0) * a.kv.page_stride + head +
                            (__shfl_sync(0xffffffffu, at_.in, 0) + c_row) * a.kv.slot_stride + c_col * 8;
        if (a.dense == HD) {                              // rows of just this length side by side: constant offsets
            const uint16_t *k = a.kv.k + e, *v = a.kv.v + e;
#pragma unroll
            for (int p = 0; p < 16 / PASS; ++p) {
                cp16(dst(p), k + p * PASS * HD, true, policy);
                cp16(dst(p) + apart, v + p * PASS * HD, true, policy);
            }
        } else {
            const bool in = c_col < chunks;
            const uint16_t *k = a.kv.k + (in ? e : 0), *v = a.kv.v + (in ? e : 0);
            const long long step = in ? PASS * a.kv.slot_stride : 0;
#pragma unroll
            for (int p = 0; p < 16 / PASS; ++p, k += step, v += step) {
                cp16(dst(p), k, in, policy);
                cp16(dst(p) + apart, v, in, policy);
            }
        }
    } else {
        if (!there && at_.id != -1 && a.status) atomicOr(a.status + b, MTAD_ST_RANGE);
        const long long off = there ? (long long)at_.id * a.kv.page_stride + head + at_.in * a.kv.slot_stride : -1;
#pragma unroll 2
        for (int p = 0; p < 16 / PASS; ++p) {
            const long long o = __shfl_sync(0xffffffffu, off, p * PASS + c_row);
            const bool in = o >= 0 && c_col < chunks;
            cp16(dst(p), a.kv.k + (in ? o + c_col * 8 : 0), in, policy);
            cp16(dst(p) + apart, a.kv.v + (in ? o + c_col * 8 : 0), in, policy);
        }
    }
}

constexpr int RW = 16;               // keys of a warp's tile

// T: the cache's type; HD: head_dim rounded up to 64, 128 or 256; ROWS: query rows of a block.  LIST: the block has an even share of
// the list of tiles; otherwise a cluster has a head, a block of it a share of the head's tiles, and the pieces are joined through
// distributed shared memory.
template <typename T, int HD, int ROWS, bool LIST>
__global__ void __launch_bounds__(NT, Tile<HD, ROWS>::BLOCKS) attn_kernel(const AttnArgs a) {
    using L = Tile<HD, ROWS>;
    using Core = typename std::conditional<(ROWS <= 16), Narrow<T, HD, ROWS>, Wide<T, HD, ROWS>>::type;
    constexpr int KW = Core::KW, S = L::STAGES, CH = L::CH;
    constexpr bool OWN = ROWS <= 16;                      // a warp multiplies the rows that it has copied itself
    extern __shared__ __align__(1024) unsigned char smem[];
    __shared__ float2 s_part[KW * ROWS];
    __shared__ float2 s_ml[ROWS];                         // the block's; read by the cluster
    __shared__ float2 s_all[LIST ? 1 : MAX_CLUSTER][LIST ? 1 : ROWS];
    __shared__ int s_scan[4];
    __shared__ int s_first[2];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const uint32_t sm = (uint32_t)__cvta_generic_to_shared(smem);
    const uint32_t sm_q = sm + S * 2 * L::BYTES;
    float* const obuf = reinterpret_cast<float*>(smem + L::SMEM);
    const int HR = a.kv.Hkv * a.RB, chunks = a.kv.hd >> 3;

    pdl_wait();
    pdl_trigger();
    // ---- this block's share of the list
    int count, rank = 0;
    Cursor P;
    if constexpr (!LIST) {
        const int head = blockIdx.x / a.cluster;
        rank = blockIdx.x - head * a.cluster;
        P.b = head / HR;
        P.hr = head - P.b * HR;
        P.s = seq_of<TK>(a, P.b);
        if (P.s.nt == 0) return;                          // (the whole cluster)
        // (the last block, whose last tile takes the longest, has none of the odd ones)
        P.t = (int)(((long long)P.s.nt * rank + a.cluster - 1) / a.cluster);
        count = (int)(((long long)P.s.nt * (rank + 1) + a.cluster - 1) / a.cluster) - P.t;
    } else {
        // first tiles of the sequences: up to 32 by one warp (every warp for itself), more by the block
        const int lanes = a.B <= 32 ? 32 : NT, me = a.B <= 32 ? lane : tid;
        const int each = (a.B + lanes - 1) / lanes, b0 = min(me * each, a.B), b1 = min(b0 + each, a.B);
        int mine = 0;
        for (int b = b0; b < b1; ++b) mine += seq_of<TK>(a, b).nt * HR;
        int incl = mine;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int x = __shfl_up_sync(0xffffffffu, incl, o);
            if (lane >= o) incl += x;
        }
        int total = __shfl_sync(0xffffffffu, incl, 31), base = incl - mine;
        if (a.B > 32) {
            if (lane == 31) s_scan[warp] = incl;
            __syncthreads();
            total = 0;
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                if (w < warp) base += s_scan[w];
                total += s_scan[w];
            }
        }
        const int per = (int)(((unsigned)total + a.grid - 1) / (unsigned)a.grid);
        const long long first = (long long)per * blockIdx.x;
        if (blockIdx.x != 0 && first >= total) return;
        const int start = (int)first, end = min(total, start + min(per, total - start));
        if (blockIdx.x == 0 && (a.B > 32 || warp == 0)) { // for the second kernel
            if (me == 0) a.plan[0] = per;
            int x = base;
            for (int b = b0; b < b1; ++b) { a.plan[1 + b] = x; x += seq_of<TK>(a, b).nt * HR; }
        }
        if (start >= end) return;
        count = end - start;
        int in = 0;
        const bool here = start >= base && start < base + mine;
        int b = b0;
        if (here)
            for (in = start - base;; ++b) {
                const int n = seq_of<TK>(a, b).nt * HR;
                if (in < n) break;
                in -= n;
            }
        if (a.B <= 32) {
            const int from = __ffs(__ballot_sync(0xffffffffu, here)) - 1;
            b = __shfl_sync(0xffffffffu, b, from);
            in = __shfl_sync(0xffffffffu, in, from);
        } else {
            if (here) { s_first[0] = b; s_first[1] = in; }
            __syncthreads();
            b = s_first[0];
            in = s_first[1];
        }
        P.b = b;
        P.s = seq_of<TK>(a, b);
        P.hr = in / P.s.nt;
        P.t = in - P.hr * P.s.nt;
    }
    Cursor C = P;
    Core core;
    core.init(tid);
    core.reset();
    int rows = 0, m0 = 0;                                 // valid query rows of the block, its first row
    auto read_q = [&]() {
        const int h = C.hr / a.RB;
        m0 = (C.hr - h * a.RB) * ROWS;
        rows = min(C.s.nb * a.G - m0, ROWS);              // (may be < 0: a block of rows that this sequence does not have)
        core.read_q(a, a.q + (long long)C.b * a.q_sb, h, m0, rows);
    };
    auto put_q = [&]() {
        core.put_q(a, sm_q, C.s.len - C.s.nb, m0, rows);
        if (tid == 0 && a.status) {
            const int len = __ldg(a.lens + C.b);
            if (len < 0 || len > a.max_len) atomicOr(a.status + C.b, MTAD_ST_KV_OVERFLOW);
        }
        if constexpr (!OWN) __syncthreads();
    };

    // ---- copies: a warp brings rows 16 * warp .. + 15 of a tile
    const int c_row = lane / CH, c_col = lane % CH;       // this lane's row and piece in a request
    const uint64_t policy = copy_policy(false);
    auto find = [&](const Cursor& c) { return look_up(a, c.s, c.b, (c.t < c.s.ns ? c.t : c.t + c.s.skip) * TK + warp * RW + (lane & 15)); };
    auto copy = [&](const Spot& spot, const Cursor& c, int stage) {
        copy_rows<HD>(a, spot, c.b, (long long)(c.hr / a.RB) * a.kv.head_stride, sm + stage * 2 * L::BYTES + warp * RW * HD * 2, L::BYTES, c_row, c_col, chunks, policy);
    };
    int ahead = 0;                                        // tiles handed to the copies
    Spot spot{-1, 0}, begin[S - 1];
    Cursor from[S - 1];
    read_q();
#pragma unroll
    for (int s = 0; s < S - 1; ++s)                       // (the first tiles' pages are asked for together)
        if (s < count) {
            begin[s] = find(P);
            from[s] = P;
            if (s + 1 < count) advance<TK>(a, P);
        }
    if (S - 1 < count) spot = find(P);
#pragma unroll
    for (int s = 0; s < S - 1; ++s) {
        if (s < count) copy(begin[s], from[s], s);
        cp_commit();
    }
    ahead = min(S - 1, count);
    put_q();

    int stage = 0;
    int first_t = C.t;                                    // tile at which this block entered the head
    for (int i = 0; i < count; ++i) {
        cp_wait<S - 2>();
        if constexpr (OWN) __syncwarp(); else __syncthreads();
        {
            int into = stage + S - 1;
            if (into >= S) into -= S;
            if (ahead < count) {
                copy(spot, P, into);
                if (++ahead < count) { advance<TK>(a, P); spot = find(P); }
            }
            cp_commit();
        }
        TileAt t;
        t.k = sm + stage * 2 * L::BYTES;
        t.v = t.k + L::BYTES;
        if (++stage == S) stage = 0;
        t.j0 = (C.t < C.s.ns ? C.t : C.t + C.s.skip) * TK;
        t.first_pos = C.s.len - C.s.nb;
        t.last_pos = C.s.len - 1;
        t.inner = t.j0 + TK - 1 <= t.first_pos && (a.window <= 0 || t.j0 + TK <= a.sinks || t.j0 > t.last_pos - a.window);
        if constexpr (OWN) {
            t.k += warp * RW * HD * 2;
            t.v += warp * RW * HD * 2;
            t.j0 += warp * RW;
        }
        t.many = C.s.nb > 1;
        float* const scores = a.scores ? a.scores + (((long long)C.b * a.kv.Hkv + C.hr / a.RB) * (a.RB * ROWS) + m0) * a.score_ld : nullptr;
        core.tile(a, t, sm_q, scores, chunks);

        // ---- end of the head, or of this block's share of it
        ++C.t;
        if constexpr (LIST) {
            const bool last = i + 1 == count, head_end = C.t == C.s.nt;
            if (!last && !head_end) continue;
            const bool cut = first_t != 0 || !head_end;
            // (a block's first piece goes to its place 0, one that begins inside its share to place 1)
            const long long place = 2ll * blockIdx.x + (i + 1 > C.t - first_t ? 1 : 0);
            core.join_warps(s_part, s_ml);
            // the warps over the keys add their outputs one after the other, a part of the columns at a time
            constexpr int W = HD / L::COLS;
            const int h = C.hr / a.RB;
#pragma unroll
            for (int cb = 0; cb < L::COLS; ++cb) {
#pragma unroll
                for (int w = 0; w < KW; ++w) {
                    if (warp / L::MT == w) core.put(obuf, L::LDC, cb, w > 0);
                    __syncthreads();
                }
                for (int k = tid; k < max(rows, 0) * (W / 4); k += NT) {
                    const int m = k / (W / 4), c = (k - m * (W / 4)) * 4, d = cb * W + c;
                    const float4 x = *reinterpret_cast<const float4*>(obuf + m * L::LDC + c);
                    const float2 ml = s_ml[m];
                    if (cut) {
                        *reinterpret_cast<float4*>(a.part_o + (place * ROWS + m) * HD + d) = x;
                        if (d == 0) a.part_ml[place * ROWS + m] = ml;
                    } else {
                        const int r = (m0 + m) / a.G, hq = h * a.G + (m0 + m) - r * a.G;
                        const float inv = inverse(ml.y * Prob<T>::SCALE);
                        if (d < a.kv.hd)
                            *reinterpret_cast<uint2*>(a.out + (long long)C.b * a.o_sb + (long long)r * a.o_sr + (long long)hq * a.o_sh + d) =
                                make_uint2(Num<T>::pack(x.x * inv, x.y * inv), Num<T>::pack(x.z * inv, x.w * inv));
                        if (d == 0) {
                            const float lse2 = ml.x + log2f(ml.y);
                            if (a.lse) a.lse[((long long)C.b * a.R + r) * (a.kv.Hkv * a.G) + hq] = lse2 * LN2;
                            if (a.weights) a.row_lse2[((long long)C.b * HR + C.hr) * ROWS + m] = lse2;
                        }
                    }
                }
                if (!(last && cb + 1 == L::COLS)) __syncthreads();
            }
            if (last) return;
            C.t = C.s.nt - 1;
            advance<TK>(a, C);
            first_t = 0;
            core.reset();
            read_q();
            put_q();
        }
    }
    if constexpr (!LIST) {
        // ---- the warps' outputs, brought to the block's reference, side by side where the tiles were
        core.join_warps(s_part, s_ml);
        float* const part = reinterpret_cast<float*>(smem);               // [KW][ROWS][LDO]
        core.put(part + (warp / L::MT) * ROWS * L::LDO, L::LDO, 0, false);
        cg::cluster_group cluster = cg::this_cluster();
        const int CS = a.cluster, per_row = a.kv.hd / 4, valid = max(rows, 0) * per_row, h = C.hr / a.RB;
        __syncthreads();
        if constexpr (KW > 1) {                           // the block's sum, over the first warp's
#pragma unroll 2
            for (int i = tid; i < valid; i += NT) {
                const int m = i / per_row;
                float4* at = reinterpret_cast<float4*>(part + m * L::LDO + (i - m * per_row) * 4);
                float4 x[KW];
#pragma unroll
                for (int w = 0; w < KW; ++w) x[w] = at[w * (ROWS * L::LDO / 4)];
#pragma unroll
                for (int w = 1; w < KW; ++w) { x[0].x += x[w].x; x[0].y += x[w].y; x[0].z += x[w].z; x[0].w += x[w].w; }
                *at = x[0];
            }
        }
        if (CS > 1) cluster.sync(); else __syncthreads();
        for (int i = tid; i < CS * ROWS; i += NT) {
            const int k = i / ROWS, m = i - k * ROWS;
            s_all[k][m] = CS > 1 ? *cluster.map_shared_rank(&s_ml[m], k) : s_ml[m];
        }
        __syncthreads();
        // ---- a block adds the cluster's sums of its share of (row, four columns), neighbouring columns by neighbouring lanes (requests to
        // another block's memory that are not whole lines take ten times as long)
        const int share = ((valid + CS - 1) / CS + 7) & ~7;
        for (int i = rank * share + tid; i < min((rank + 1) * share, valid); i += NT) {
            const int m = i / per_row, d = (i - m * per_row) * 4;
            float4 x[MAX_CLUSTER];
#pragma unroll
            for (int k = 0; k < MAX_CLUSTER; ++k)
                if (k < CS) x[k] = *reinterpret_cast<const float4*>((CS > 1 ? cluster.map_shared_rank(part, k) : part) + m * L::LDO + d);
            float mx = s_all[0][m].x, sum = 0.f;
            for (int k = 1; k < CS; ++k) mx = fmaxf(mx, s_all[k][m].x);
            float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
            for (int k = 0; k < MAX_CLUSTER; ++k)
                if (k < CS) {
                    const float2 ml = s_all[k][m];
                    const float f = ml.x == mx ? 1.f : ex2(ml.x - mx);
                    sum += f * ml.y;
                    acc.x += f * x[k].x; acc.y += f * x[k].y; acc.z += f * x[k].z; acc.w += f * x[k].w;
                }
            const int r = (m0 + m) / a.G, hq = h * a.G + (m0 + m) - r * a.G;
            const float inv = inverse(sum * Prob<T>::SCALE);
            *reinterpret_cast<uint2*>(a.out + (long long)C.b * a.o_sb + (long long)r * a.o_sr + (long long)hq * a.o_sh + d) =
                make_uint2(Num<T>::pack(acc.x * inv, acc.y * inv), Num<T>::pack(acc.z * inv, acc.w * inv));
            if (d == 0 && a.lse) a.lse[((long long)C.b * a.R + r) * (a.kv.Hkv * a.G) + hq] = (mx + log2f(sum)) * LN2;
        }
        // (no block leaves while another reads its shared memory)
        if (CS > 1) asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
        // ---- weights of the slots of this block's tiles, from the scores that it wrote itself (one row block a head: see make_plan)
        if (a.weights) {
            float* const s_lse = reinterpret_cast<float*>(s_part);
            if (tid < max(rows, 0)) {
                float mx = s_all[0][tid].x, sum = 0.f;
                for (int k = 1; k < CS; ++k) mx = fmaxf(mx, s_all[k][tid].x);
                for (int k = 0; k < CS; ++k) sum += s_all[k][tid].y * (s_all[k][tid].x == mx ? 1.f : ex2(s_all[k][tid].x - mx));
                s_lse[tid] = mx + log2f(sum);
            }
            __syncthreads();
            const float* z = a.scores + ((long long)C.b * a.kv.Hkv + h) * ROWS * a.score_ld;
            float* dst = a.weights + (long long)C.b * a.w_sb + (long long)h * a.w_sh;
            for (int i = tid; i < count * TK; i += NT) {
                const int tt = first_t + i / TK, j = (tt < C.s.ns ? tt : tt + C.s.skip) * TK + i % TK;
                if (j >= C.s.len) continue;
                float acc = 0.f;
#pragma unroll 4
                for (int m = 0; m < rows; ++m) {
                    const float lse = s_lse[m];
                    if (lse != -CUDART_INF_F) acc += weight(z[(long long)m * a.score_ld + j], lse);
                }
                dst[j] += acc;
            }
        }
        if (CS > 1) asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
    }
}

// Up to 16 query rows, the list cut over all warps of the GPU: a warp has an even share of the list of 16-key tiles and a ring of its own,
// waits for nobody, and writes its pieces of cut heads from its registers.
template <int HD, int ROWS> struct Ring {
    static constexpr int BYTES = RW * HD * 2, STAGES = Tile<HD, ROWS>::STAGES;
    static constexpr int SMEM = (NT / 32) * STAGES * 2 * BYTES;
};
template <typename T, int HD, int ROWS>
__global__ void __launch_bounds__(NT, Tile<HD, ROWS>::BLOCKS) stream_kernel(const AttnArgs a) {
    using L = Ring<HD, ROWS>;
    using Core = Narrow<T, HD, ROWS>;
    constexpr int S = L::STAGES, CH = HD / 8;
    extern __shared__ __align__(1024) unsigned char smem[];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, worker = blockIdx.x * (NT / 32) + warp;
    const uint32_t ring = (uint32_t)__cvta_generic_to_shared(smem) + warp * S * 2 * L::BYTES;
    const int Hkv = a.kv.Hkv, chunks = a.kv.hd >> 3;
    pdl_wait();
    pdl_trigger();
    // ---- this warp's share of the list
    int count;
    Cursor P;
    {
        const int each = (a.B + 31) / 32, b0 = min(lane * each, a.B), b1 = min(b0 + each, a.B);
        int mine = 0;
        for (int b = b0; b < b1; ++b) mine += seq_of<RW>(a, b).nt * Hkv;
        int incl = mine;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int x = __shfl_up_sync(0xffffffffu, incl, o);
            if (lane >= o) incl += x;
        }
        const int total = __shfl_sync(0xffffffffu, incl, 31), base = incl - mine, per = (int)(((unsigned)total + a.grid - 1) / (unsigned)a.grid);
        if (worker == 0) {                                // for the second kernel
            if (lane == 0) a.plan[0] = per;
            int x = base;
            for (int b = b0; b < b1; ++b) { a.plan[1 + b] = x; x += seq_of<RW>(a, b).nt * Hkv; }
        }
        if ((long long)per * worker >= total) return;
        const int start = per * worker;
        count = min(per, total - start);
        const bool here = start >= base && start < base + mine;
        int b = b0;
        int in = start - base;
        if (here)
            for (;; ++b) {
                const int n = seq_of<RW>(a, b).nt * Hkv;
                if (in < n) break;
                in -= n;
            }
        const int from = __ffs(__ballot_sync(0xffffffffu, here)) - 1;
        P.b = __shfl_sync(0xffffffffu, b, from);
        in = __shfl_sync(0xffffffffu, in, from);
        P.s = seq_of<RW>(a, P.b);
        P.hr = in / P.s.nt;
        P.t = in - P.hr * P.s.nt;
    }
    Cursor C = P;
    Core core;
    core.init(threadIdx.x);
    core.reset();
    int rows = 0;
    auto read_q = [&]() {
        rows = C.s.nb * a.G;
        core.read_q(a, a.q + (long long)C.b * a.q_sb, C.hr, 0, rows);
    };
    auto put_q = [&]() {
        core.put_q(a, 0, C.s.len - C.s.nb, 0, rows);
        if (lane == 0 && a.status) {
            const int len = __ldg(a.lens + C.b);
            if (len < 0 || len > a.max_len) atomicOr(a.status + C.b, MTAD_ST_KV_OVERFLOW);
        }
    };
    const int c_row = lane / CH, c_col = lane % CH;
    const uint64_t policy = copy_policy(true);
    auto find = [&](const Cursor& c) { return look_up(a, c.s, c.b, (c.t < c.s.ns ? c.t : c.t + c.s.skip) * RW + (lane & 15)); };
    auto copy = [&](const Spot& spot, const Cursor& c, int stage) {
        copy_rows<HD>(a, spot, c.b, c.hr * a.kv.head_stride, ring + stage * 2 * L::BYTES, L::BYTES, c_row, c_col, chunks, policy);
    };
    int ahead = 0;
    Spot spot{-1, 0}, begin[S - 1];
    Cursor from[S - 1];
    read_q();
#pragma unroll
    for (int s = 0; s < S - 1; ++s)                       // (the first tiles' pages are asked for together)
        if (s < count) {
            begin[s] = find(P);
            from[s] = P;
            if (s + 1 < count) advance<RW>(a, P);
        }
    if (S - 1 < count) spot = find(P);
#pragma unroll
    for (int s = 0; s < S - 1; ++s) {
        if (s < count) copy(begin[s], from[s], s);
        cp_commit();
    }
    ahead = min(S - 1, count);
    put_q();
    int stage = 0, first_t = C.t;
    for (int i = 0; i < count; ++i) {
        cp_wait<S - 2>();
        __syncwarp();
        if (ahead < count) {
            copy(spot, P, stage + S - 1 >= S ? stage - 1 : stage + S - 1);
            if (++ahead < count) { advance<RW>(a, P); spot = find(P); }
        }
        cp_commit();
        TileAt t;
        t.k = ring + stage * 2 * L::BYTES;
        t.v = t.k + L::BYTES;
        if (++stage == S) stage = 0;
        t.j0 = (C.t < C.s.ns ? C.t : C.t + C.s.skip) * RW;
        t.first_pos = C.s.len - C.s.nb;
        t.last_pos = C.s.len - 1;
        t.inner = t.j0 + RW - 1 <= t.first_pos && (a.window <= 0 || t.j0 + RW <= a.sinks || t.j0 > t.last_pos - a.window);
        t.many = C.s.nb > 1;
        const long long head = (long long)C.b * Hkv + C.hr;
        core.tile(a, t, 0, a.scores ? a.scores + head * ROWS * a.score_ld : nullptr, chunks);
        ++C.t;
        const bool last = i + 1 == count, head_end = C.t == C.s.nt;
        if (!last && !head_end) continue;
        // ---- end of the head, or of this warp's share of it (first piece: place 0, one that begins inside the share: place 1)
        const bool cut = first_t != 0 || !head_end;
        const long long place = 2ll * worker + (i + 1 > C.t - first_t ? 1 : 0);
        core.join_lanes();
#pragma unroll
        for (int n = 0; n < Core::N8; ++n)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int m = n * 8 + core.t2 + e;
                if (m >= rows) continue;
                if (cut) {
                    float* dst = a.part_o + (place * ROWS + m) * HD + core.g;
#pragma unroll
                    for (int d = 0; d < HD / 16; ++d) {
                        dst[d * 16] = core.o[d][n][e];
                        dst[d * 16 + 8] = core.o[d][n][e + 2];
                    }
                    if (core.g == 0) a.part_ml[place * ROWS + m] = make_float2(core.m[n][e], core.l[n][e]);
                } else {
                    const int r = m / a.G, hq = C.hr * a.G + m - r * a.G;
                    T* dst = reinterpret_cast<T*>(a.out) + (long long)C.b * a.o_sb + (long long)r * a.o_sr + (long long)hq * a.o_sh + core.g;
                    const float inv = inverse(core.l[n][e] * Prob<T>::SCALE);
#pragma unroll
                    for (int d = 0; d < HD / 16; ++d) {
                        if (d * 16 < a.kv.hd) dst[d * 16] = Num<T>::from(core.o[d][n][e] * inv);
                        if (d * 16 + 8 < a.kv.hd) dst[d * 16 + 8] = Num<T>::from(core.o[d][n][e + 2] * inv);
                    }
                    if (core.g == 0) {
                        const float lse2 = core.m[n][e] + log2f(core.l[n][e]);
                        if (a.lse) a.lse[((long long)C.b * a.R + r) * (Hkv * a.G) + hq] = lse2 * LN2;
                        if (a.weights) a.row_lse2[head * ROWS + m] = lse2;
                    }
                }
            }
        if (last) return;
        C.t = C.s.nt - 1;
        advance<RW>(a, C);
        first_t = 0;
        core.reset();
        read_q();
        put_q();
    }
}

// ---- what the blocks left of heads that were cut, and the weights

struct Pieces {                      // the shares that hold a head's tiles
    int per, s, c0, n;
};
__device__ __forceinline__ Pieces pieces_of(const AttnArgs& a, const Seq& q, int b, int hr) {
    Pieces p;
    p.per = a.plan[0];
    p.s = a.plan[1 + b] + hr * q.nt;
    p.c0 = p.s / p.per;
    p.n = (p.s + q.nt - 1) / p.per - p.c0 + 1;
    return p;
}
__device__ __forceinline__ long long place_of(const Pieces& p, int i) {
    return 2ll * (p.c0 + i) + (i == 0 && p.s > p.c0 * p.per ? 1 : 0);
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
template <typename T, int HD, int UNIT, bool SPLIT, bool WEIGHTS>
__global__ void __launch_bounds__(NT, 8) join_kernel(const AttnArgs a, int n_join, int groups) {
    constexpr int PER = HD / 32;     // columns of a lane
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, HR = a.kv.Hkv * a.RB;
    __shared__ float s_lse[MAX_ROWS_BLOCK];
    __shared__ float s_acc[SPLIT ? 4 : 1][SPLIT ? HD : 1];
    pdl_wait();
    if ((int)blockIdx.x < n_join) {
        // a warp has a row, or (SPLIT) the block has one and its warps a quarter of the pieces each
        const int seg = blockIdx.x / groups, m = SPLIT ? blockIdx.x - seg * groups : (blockIdx.x - seg * groups) * 4 + warp, b = seg / HR, hr = seg - b * HR;
        const Seq q = seq_of<UNIT>(a, b);
        const int h = hr / a.RB, row = (hr - h * a.RB) * a.rows_block + m;
        if (q.nt == 0 || m >= a.rows_block || row >= q.nb * a.G) return;
        const Pieces p = pieces_of(a, q, b, hr);
        if (p.n == 1) return;
        float2 ml;
        float acc[PER];
#pragma unroll
        for (int k = 0; k < PER; ++k) acc[k] = 0.f;
        if (!SPLIT && p.n <= 8) {                         // outputs and statistics are asked for together
            const float2 mine = lane < p.n ? a.part_ml[place_of(p, lane) * a.rows_block + m] : make_float2(-CUDART_INF_F, 0.f);
            float x[8][PER];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float* src = a.part_o + (place_of(p, min(i, p.n - 1)) * a.rows_block + m) * HD + lane * PER;
                if (i < p.n)
#pragma unroll
                    for (int k = 0; k < PER; k += 2) *reinterpret_cast<float2*>(&x[i][k]) = *reinterpret_cast<const float2*>(src + k);
            }
            ml.x = mine.x;
#pragma unroll
            for (int o = 4; o > 0; o >>= 1) ml.x = fmaxf(ml.x, __shfl_xor_sync(0xffffffffu, ml.x, o));
            ml.x = __shfl_sync(0xffffffffu, ml.x, 0);
            const float f = mine.x == ml.x ? 1.f : ex2(mine.x - ml.x);
            ml.y = lane < p.n ? mine.y * f : 0.f;
#pragma unroll
            for (int o = 4; o > 0; o >>= 1) ml.y += __shfl_xor_sync(0xffffffffu, ml.y, o);
            ml.y = __shfl_sync(0xffffffffu, ml.y, 0);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float fi = __shfl_sync(0xffffffffu, f, i);
                if (i < p.n)
#pragma unroll
                    for (int k = 0; k < PER; ++k) acc[k] += fi * x[i][k];
            }
        } else {
            ml = joined(a, p, m, lane);
            const int each = SPLIT ? (p.n + 3) / 4 : p.n, p0 = SPLIT ? warp * each : 0, p1 = min(p0 + each, p.n);
#pragma unroll 8
            for (int i = p0; i < p1; ++i) {
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
        }
        if constexpr (SPLIT) {
#pragma unroll
            for (int k = 0; k < PER; ++k) s_acc[warp][lane * PER + k] = acc[k];
            __syncthreads();
            if (warp > 0) return;
#pragma unroll
            for (int w = 1; w < 4; ++w)
#pragma unroll
                for (int k = 0; k < PER; ++k) acc[k] += s_acc[w][lane * PER + k];
        }
        const int r = row / a.G, hq = h * a.G + row - r * a.G;
        const float inv = inverse(ml.y * Prob<T>::SCALE);
        if (lane * PER < a.kv.hd) {
            uint16_t* dst = a.out + (long long)b * a.o_sb + (long long)r * a.o_sr + (long long)hq * a.o_sh + lane * PER;
#pragma unroll
            for (int k = 0; k < PER; k += 2) *reinterpret_cast<uint32_t*>(dst + k) = Num<T>::pack(acc[k] * inv, acc[k + 1] * inv);
        }
        if (a.lse && lane == 0) a.lse[((long long)b * a.R + r) * (a.kv.Hkv * a.G) + hq] = (ml.x + log2f(ml.y)) * LN2;
        return;
    }
    if constexpr (!WEIGHTS) return;
    const int per_head = (a.max_len + W_KEYS - 1) / W_KEYS, w = blockIdx.x - n_join, bh = w / per_head, b = bh / a.kv.Hkv, h = bh - b * a.kv.Hkv;
    const int k0 = (w - bh * per_head) * W_KEYS;
    const Seq q = seq_of<UNIT>(a, b);
    if (q.nt == 0 || k0 >= q.len) return;
    const int j = k0 + tid * 4;                           // (four neighbouring slots lie in one tile; tiles that no row sees have no scores)
    const bool there = j < q.len && (j / UNIT < q.ns || j / UNIT >= q.ns + q.skip);
    if (!__syncthreads_or(there)) return;
    const int RBL = a.rows_block;
    float* const dst = a.weights + (long long)b * a.w_sb + (long long)h * a.w_sh + j;
    // everything that does not need the sums is asked for before they are known
    float old[4], acc[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int k = 0; k < 4; ++k) old[k] = there && j + k < q.len ? dst[k] : 0.f;
    for (int rb = 0; rb < a.RB; ++rb) {
        const int hr = h * a.RB + rb, rows = min(q.nb * a.G - rb * RBL, RBL);
        if (rows <= 0) break;
        const float* z = a.scores + ((long long)bh * (a.RB * RBL) + rb * RBL) * a.score_ld + j;
        float4 x[8];
#pragma unroll
        for (int m = 0; m < 8; ++m)
            if (there && m < rows) x[m] = *reinterpret_cast<const float4*>(z + m * a.score_ld);
        const Pieces p = pieces_of(a, q, b, hr);
        __syncthreads();
        if (p.n == 1) {
            if (tid < rows) s_lse[tid] = a.row_lse2[((long long)b * HR + hr) * RBL + tid];
        } else if (p.n <= 4 && rows <= 32) {              // (four lanes a row)
            const int m = tid >> 2, i = tid & 3;
            const float2 ml = m < rows && i < p.n ? a.part_ml[place_of(p, i) * RBL + m] : make_float2(-CUDART_INF_F, 0.f);
            float mx = fmaxf(ml.x, __shfl_xor_sync(0xffffffffu, ml.x, 1));
            mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 2));
            float sum = ml.y * (ml.x == mx ? 1.f : ex2(ml.x - mx));
            sum += __shfl_xor_sync(0xffffffffu, sum, 1);
            sum += __shfl_xor_sync(0xffffffffu, sum, 2);
            if (m < rows && i == 0) s_lse[m] = mx + log2f(sum);
        } else {
            for (int m = warp; m < rows; m += 4) {
                const float2 ml = joined(a, p, m, lane);
                if (lane == 0) s_lse[m] = ml.x + log2f(ml.y);
            }
        }
        __syncthreads();
        for (int m0 = 0; m0 < rows; m0 += 8) {
#pragma unroll
            for (int m = 0; m < 8; ++m) {
                if (m0 + m >= rows) break;
                const float lse = s_lse[m0 + m];
                if (lse == -CUDART_INF_F) continue;       // (a row that sees nothing has no scores)
                acc[0] += weight(x[m].x, lse); acc[1] += weight(x[m].y, lse); acc[2] += weight(x[m].z, lse); acc[3] += weight(x[m].w, lse);
            }
#pragma unroll
            for (int m = 0; m < 8; ++m)
                if (there && m0 + 8 + m < rows) x[m] = *reinterpret_cast<const float4*>(z + (m0 + 8 + m) * a.score_ld);
        }
    }
#pragma unroll
    for (int k = 0; k < 4; ++k)
        if (there && j + k < q.len) dst[k] = old[k] + acc[k];
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
    int HD, grid;
    bool narrow;                     // the list is cut over warps
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
    if (!lie_apart(kv->head_dim, {{a.B, a.o_sb}, {a.R, a.o_sr}, {c->n_q_heads, a.o_sh}})) return MTAD_E_INVALID;
    if (c->weights && !lie_apart(a.max_len, {{a.B, c->weights_stride_seq}, {kv->n_kv_heads, c->weights_stride_head}})) return MTAD_E_INVALID;
    if (a.window >= a.max_len) a.window = a.sinks = 0;    // (every slot is inside it)
    a.scale2 = (float)((c->scale != 0.f ? (double)c->scale : 1.0 / sqrt((double)kv->head_dim)) * 1.4426950408889634);
    a.weights = c->weights; a.w_sb = c->weights_stride_seq; a.w_sh = c->weights_stride_head;
    p->HD = kv->head_dim <= 64 ? 64 : kv->head_dim <= 128 ? 128 : 256;
    const int M = a.R * a.G;
    a.rows_block = M <= 8 ? 8 : M <= 16 ? 16 : M <= 32 ? 32 : 64;
    a.RB = (M + a.rows_block - 1) / a.rows_block;
    long long tiles = (a.max_len + TK - 1) / TK;          // of 64 keys
    if (a.window > 0) {
        const long long some = ((long long)a.sinks + TK - 1) / TK + ((long long)a.window + a.R + TK - 2) / TK + 1;
        tiles = some < tiles ? some : tiles;
    }
    const long long heads = (long long)a.B * a.kv.Hkv * a.RB;
    if (heads * std::max(4 * tiles, (long long)MAX_CLUSTER) > 0x7fffffffll ||
        heads * ((a.max_len + W_KEYS - 1) / W_KEYS) + heads * MAX_ROWS_BLOCK > 0x7fffffffll) return MTAD_E_CAPACITY;
    // (workspace sizes may be asked for without a device)
    int sms = 148, dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) sms = 148;
    const long long fill = (long long)sms * (p->HD == 256 ? 1 : 2);
    // A cluster per head where that takes few tiles a block
    int cs = 1;
    while (cs < MAX_CLUSTER && cs < tiles && heads * cs * 2 <= fill) cs *= 2;
    const bool list = (tiles + cs - 1) / cs > (a.rows_block <= 16 ? CLUSTER_TILES : CLUSTER_TILES_WIDE) || (a.weights && a.RB > 1);
    a.cluster = list ? 0 : cs;
    a.even = kv->page_size % 16 == 0;
    a.dense = kv->slot_stride == kv->head_dim ? kv->head_dim : 0;
    p->narrow = list && a.rows_block <= 16;
    p->grid = (int)(list ? std::min(heads * tiles, fill) : heads * cs);
    a.grid = p->narrow ? p->grid * (NT / 32) : p->grid;  // shares
    Carve w;
    p->plan = w.take(list ? sizeof(int) * (a.B + 1) : 0);
    p->part_o = w.take(list ? sizeof(float) * 2 * (size_t)a.grid * a.rows_block * p->HD : 0);
    p->part_ml = w.take(list ? sizeof(float2) * 2 * (size_t)a.grid * a.rows_block : 0);
    a.score_ld = a.weights ? (long long)((a.max_len + TK - 1) / TK) * TK : 0;
    p->row_lse2 = w.take(list && a.weights ? sizeof(float) * heads * a.rows_block : 0);
    p->scores = w.take(a.weights ? sizeof(float) * (size_t)heads * a.rows_block * a.score_ld : 0);
    p->bytes = w.off;
    return MTAD_OK;
}

template <typename T, int HD, int ROWS, bool LIST>
cudaError_t launch_attn(const AttnPlan& p, cudaStream_t st) {
    constexpr int smem = Tile<HD, ROWS>::SMEM + (LIST ? Tile<HD, ROWS>::OBUF : 0);
    const cudaError_t e = ops_smem<attn_kernel<T, HD, ROWS, LIST>>(smem);
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3(p.grid);
    cfg.blockDim = dim3(NT);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute at[2];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    at[1].id = cudaLaunchAttributeClusterDimension;
    at[1].val.clusterDim.x = LIST ? 1 : p.a.cluster;
    at[1].val.clusterDim.y = at[1].val.clusterDim.z = 1;
    cfg.attrs = at;
    cfg.numAttrs = LIST ? 1 : 2;
    return cudaLaunchKernelEx(&cfg, attn_kernel<T, HD, ROWS, LIST>, p.a);
}
template <typename T, int HD, int ROWS>
cudaError_t launch_stream(const AttnPlan& p, cudaStream_t st) {
    constexpr int smem = Ring<HD, ROWS>::SMEM;
    const cudaError_t e = ops_smem<stream_kernel<T, HD, ROWS>>(smem);
    return e != cudaSuccess ? e : launch_pdl(stream_kernel<T, HD, ROWS>, dim3(p.grid), dim3(NT), smem, st, true, p.a);
}
template <typename T, int HD, bool LIST>
cudaError_t launch_rows(const AttnPlan& p, cudaStream_t st) {
    switch (p.a.rows_block) {
        case 8: if constexpr (LIST) return launch_stream<T, HD, 8>(p, st); else return launch_attn<T, HD, 8, LIST>(p, st);
        case 16: if constexpr (LIST) return launch_stream<T, HD, 16>(p, st); else return launch_attn<T, HD, 16, LIST>(p, st);
        case 32: return launch_attn<T, HD, 32, LIST>(p, st);
        default: return launch_attn<T, HD, 64, LIST>(p, st);
    }
}
template <typename T, int HD>
cudaError_t launch_hd(const AttnPlan& p, cudaStream_t st) {
    mtad_ops_count(1);
    if (p.a.cluster) return launch_rows<T, HD, false>(p, st);
    const cudaError_t e = launch_rows<T, HD, true>(p, st);
    if (e != cudaSuccess) return e;
    mtad_ops_count(1);
    // (a head in many pieces, four warps a row / one: 37 pieces 27.1 / 28.6 us a call, 148 pieces 16.1 / 24.5, 1184 pieces 22 / 49; with few, blocks of
    // one row have too little to do)
    const long long heads = (long long)p.a.B * p.a.kv.Hkv * p.a.RB;
    const bool split = p.a.grid / heads >= 12;
    const int rows = std::min(p.a.R * p.a.G, p.a.rows_block), groups = split ? rows : (rows + 3) / 4, join = (int)heads * groups;
    const int add = p.a.weights ? p.a.B * p.a.kv.Hkv * ((p.a.max_len + W_KEYS - 1) / W_KEYS) : 0;
    auto go = [&](auto kernel) { return launch_pdl(kernel, dim3(join + add), dim3(NT), 0, st, true, p.a, join, groups); };
    auto pick = [&](auto unit) {
        constexpr int U = decltype(unit)::value;
        return split ? (add ? go(join_kernel<T, HD, U, true, true>) : go(join_kernel<T, HD, U, true, false>))
                     : (add ? go(join_kernel<T, HD, U, false, true>) : go(join_kernel<T, HD, U, false, false>));
    };
    return p.narrow ? pick(std::integral_constant<int, RW>()) : pick(std::integral_constant<int, TK>());
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
    p.a.plan = reinterpret_cast<int*>(w + p.plan);
    p.a.part_o = reinterpret_cast<float*>(w + p.part_o);
    p.a.part_ml = reinterpret_cast<float2*>(w + p.part_ml);
    p.a.row_lse2 = reinterpret_cast<float*>(w + p.row_lse2);
    p.a.scores = p.a.weights ? reinterpret_cast<float*>(w + p.scores) : nullptr;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    return ops_status(kv->dtype == MTAD_BF16 ? launch_t<__nv_bfloat16>(p, st) : launch_t<__half>(p, st));
}

}  // extern "C"
