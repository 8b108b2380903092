// Attention of one new token per sequence over a paged cache: over all its rows, or over the pages chosen for each KV head
// (page_select_kernel).  As in decode.cuh the work is a stream over K and V that the memory bounds, bf16 caches go through
// warp-level matrix instructions with the fp32 weights in three bf16 pieces and fp32 caches through multiply-adds, and every sum
// has a fixed order.  What differs:
//
// The lengths are on the device and ragged, so the host cannot cut the work.  A pair (sequence, KV head) has its rows in units; the
// units of all pairs of a column of KV heads (heads column, column + columns, ...) in order are one line, which its CTAs (the grid is as
// many as the device holds at once, those of neighbouring columns neighbours) cut into equal shares.  So the CTAs of the columns go
// along the same rows side by side, and what they read of a row at a time is a stretch of memory: with the heads one after the other
// instead one sequence of 128K rows took 91 us, 86 with eight columns.
// A CTA adds the lengths up to find its share, which may start inside a pair, hold several pairs and end inside one.  Pairs that lie
// in one share are written out; of the others every share leaves (accumulator, maximum, sum) in scratch, at most one at its
// start and one at its end, and paged_merge_kernel, one block per share and head, adds up the pairs that begin in its share.
//
// Bound by memory where there is work for the device: one sequence of 128K rows, 8 KV heads of 128, 537 MB in 87 to 94 us a call, from one B200 to
// another, = 5.7 to 6.2 TB/s (88 to 95 % of a copy's rate; 84 in a graph of calls); 16 sequences of 4K to 16K rows 578 MB in 95 to 103 us; 64
// sequences of 1K to 1.5K rows, 331 MB in 63 to 67 us, of which 8 are the two launches, the sum over the lengths and the first look-ups.
//
// A row is found through the table (and the list of chosen pages): the lanes of a warp look up the sixteen rows of a
// chunk one turn before its copies go out (two turns before for the list), so the look-ups are never waited for.  Rows that do not
// exist are not read: their 16-byte pieces are filled with zeros.
#pragma once
#include "decode.cuh"
#include "paged.cuh"

namespace sab {

struct PagedAttnArgs {
    Paged pg;
    const void* q;                                   // [n_seqs][H][D]
    const int* sel;                                  // [n_seqs][Hkv][n_sel], or NULL: all pages
    int n_sel;
    int H, Hkv, G, D;
    int columns;                                     // of KV heads (and their groups), a divisor of Hkv * groups and of the grid
    int groups, group_heads;                         // head groups of a KV head, heads of a group (the last may have fewer)
    bool same_place;                                 // K and V have the same strides
    float c2;                                        // log2(e) / sqrt(D)
    float* part;                                     // [2 x CTAs][group_heads][D + 4]: accumulator, max (log2 units), sum
    int4* jobs;                                      // [CTAs]: first head row, heads, parts (every columns-th CTA from this one on)
    float* out;                                      // [n_seqs][H][D]
    float* lse;                                      // optional [n_seqs][H]
    // rows of sequence s that the queries see through the list (a last page's absent rows count)
    __device__ __forceinline__ int listed_rows(int s) const
    {
        const int rows = pg.rows_of(s);
        return sel ? min(n_sel, pg.by_page.div(rows + pg.page_size - 1)) * pg.page_size : rows;
    }
};

// A CTA's share [u, u_end) of its column's line of units; where it starts: sequence s, `skip` units into the units of that
// sequence's pairs of the column.
struct PgShare {
    long long u, u_end, quota, skip;
    int s;
};

template <int THREADS, int UNIT>
__device__ __forceinline__ PgShare pg_share(const PagedAttnArgs& a, int pairs)
{
    __shared__ long long warp_sum_s[THREADS / 32];
    __shared__ long long skip_s;
    __shared__ int s_s;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int n = a.pg.n_seqs, per = (n + THREADS - 1) / THREADS;
    const int s0 = min(tid * per, n), s1 = min(s0 + per, n);
    auto units = [&](int s) { return max(1, (a.listed_rows(s) + UNIT - 1) / UNIT); };
    long long mine = 0;
    for (int s = s0; s < s1; ++s) mine += units(s);
    long long upto = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const long long x = __shfl_up_sync(0xffffffffu, upto, o);
        if (lane >= o) upto += x;
    }
    if (lane == 31) warp_sum_s[warp] = upto;
    __syncthreads();
    long long total = 0;
#pragma unroll
    for (int w = 0; w < THREADS / 32; ++w) {
        if (w < warp) upto += warp_sum_s[w];
        total += warp_sum_s[w];
    }
    total *= pairs;
    PgShare r;
    const int shares = gridDim.x / a.columns;
    r.quota = (total + shares - 1) / shares;
    r.u = min((long long)(blockIdx.x / a.columns) * r.quota, total);
    r.u_end = min(r.u + r.quota, total);
    long long before = (upto - mine) * pairs;
    if (r.u >= before && r.u < before + mine * pairs)
        for (int s = s0; s < s1; ++s) {
            const long long here = (long long)units(s) * pairs;
            if (r.u < before + here) {
                s_s = s;
                skip_s = r.u - before;
                break;
            }
            before += here;
        }
    __syncthreads();
    r.s = s_s;                                       // (not set where the share is empty, and not used)
    r.skip = skip_s;
    return r;
}

// The segment of pair `pair` of sequence s (of those of the column) from unit w on, of which `left` units are the share's.
struct PgSegment {
    int s, hk, g0, heads;                            // sequence, KV head, first head of the group, heads
    int rows, row0, row1;                            // rows of the pair, and the segment's
    bool first, last;                                // the segment starts (ends) the pair
    long long units;                                 // of the pair
};
template <int UNIT>
__device__ __forceinline__ PgSegment pg_segment(const PagedAttnArgs& a, int s, int pair, int w, long long left)
{
    PgSegment g;
    g.s = s;
    pair = pair * a.columns + (int)blockIdx.x % a.columns;
    g.hk = pair / a.groups;
    const int gi = pair - g.hk * a.groups;
    g.g0 = gi * a.group_heads;
    g.heads = min(a.group_heads, a.G - g.g0);
    g.rows = a.listed_rows(s);
    g.units = max(1, (g.rows + UNIT - 1) / UNIT);
    const long long n = min(g.units - w, left);
    g.first = w == 0;
    g.last = w + n == g.units;
    g.row0 = w * UNIT;
    g.row1 = (int)min((long long)g.rows, (w + n) * UNIT);
    return g;
}

// The share's partial result of a segment: at the start of the share (0) or at its end (1).
__device__ __forceinline__ float* pg_part(const PagedAttnArgs& a, const PgSegment& g, int h)
{
    return a.part + (((size_t)2 * blockIdx.x + (g.first ? 1 : 0)) * a.group_heads + h) * (a.D + 4);
}
__device__ __forceinline__ size_t pg_head(const PagedAttnArgs& a, const PgSegment& g) { return (size_t)g.s * a.H + (size_t)g.hk * a.G + g.g0; }

// Row look-ups of a warp's chunk, one row per lane: page list, then table, then offsets.
struct PgRow {
    int page, slot;
    bool ok;                                         // the row exists (if the page does)
};
struct PgLook {
    const int *table, *sel;
    int rows;                                        // of the segment, absolute end
    int len;                                         // rows of the sequence
};
__device__ __forceinline__ PgLook pg_look(const PagedAttnArgs& a, const PgSegment& g)
{
    PgLook l;
    l.table = a.pg.table + (long long)g.s * a.pg.table_stride;
    l.sel = a.sel ? a.sel + ((size_t)g.s * a.Hkv + g.hk) * a.n_sel : nullptr;
    l.rows = g.row1;
    l.len = a.pg.rows_of(g.s);
    return l;
}
// page of the sequence that row v of the list is in, first half of a look-up.  (Loads are unconditional, and what they say about rows that
// do not exist is ignored when it is used: a branch here would wait for them.)
__device__ __forceinline__ int pg_listed(const PagedAttnArgs& a, const PgLook& l, int v)
{
    const int j = a.pg.by_page.div(max(0, min(v, l.rows - 1)));       // (a sequence without rows has a first entry all the same)
    return l.sel ? l.sel[j] : j;
}
__device__ __forceinline__ PgRow pg_find(const PagedAttnArgs& a, const PgLook& l, int v, int j)
{
    PgRow r;
    r.slot = v - a.pg.by_page.div(v) * a.pg.page_size;
    const bool in = (unsigned)j < (unsigned)a.pg.max_pages;
    r.ok = in && v < l.rows && (long long)j * a.pg.page_size + r.slot < l.len;
    r.page = l.table[in ? j : 0];
    return r;
}

// 16-byte asynchronous copy, or 16 bytes of zeros and nothing read
__device__ __forceinline__ void cp_async16_or_zero(uint32_t dst, const void* src, bool there)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(there ? 16 : 0) : "memory");
}

// A pair's result, or the share's part of it, from the merged sums of a CTA.
__device__ __forceinline__ void pg_emit(const PagedAttnArgs& a, const PgSegment& g, int h, int d, float sum, float m, float l)
{
    if (g.first && g.last) {
        const size_t row = pg_head(a, g) + h;
        a.out[row * a.D + d] = l == 0.f ? 0.f : sum / l;
        if (a.lse && d == 0) a.lse[row] = l == 0.f ? -INFINITY : (m + log2f(l)) * 0.6931471805599453f;
    } else {
        float* dst = pg_part(a, g, h);
        dst[d] = sum;
        if (d == 0) { dst[a.D] = m; dst[a.D + 1] = l; }
    }
}

__device__ __forceinline__ void pg_emit4(const PagedAttnArgs& a, const PgSegment& g, int h, int d, const float4& sum, float m, float l)
{
    if (g.first && g.last) {
        const size_t row = pg_head(a, g) + h;
        float* dst = a.out + row * a.D + d;
        dst[0] = l == 0.f ? 0.f : sum.x / l;
        dst[1] = l == 0.f ? 0.f : sum.y / l;
        dst[2] = l == 0.f ? 0.f : sum.z / l;
        dst[3] = l == 0.f ? 0.f : sum.w / l;
        if (a.lse && d == 0) a.lse[row] = l == 0.f ? -INFINITY : (m + log2f(l)) * 0.6931471805599453f;
    } else {
        float* dst = pg_part(a, g, h);
        *reinterpret_cast<float4*>(dst + d) = sum;
        if (d == 0) *reinterpret_cast<float2*>(dst + a.D) = make_float2(m, l);
    }
}

// ---- bf16 -----------------------------------------------------------------------------------------------
// As decode_mma_kernel (decode.cuh has the reasons): four warps, each with a private ring of 16-row chunks and its own online
// softmax; a unit is 64 rows.  Up to four heads (Q4) go into rows 0-3 of the 16-row A operand and again into rows 4-7: rows 0-3
// then carry the leading pieces of the weights, rows 8-11 the middle and rows 4-7 the last ones, one instruction for all three.
// Otherwise heads come in NS sets of eight: the queries of the first set in rows 0-7, of the second in rows 8-15, one product for both;
// the weights of a set take two instructions, half of the leading pieces in rows 0-7 of either (zeros there would make no numbers
// of infinite values), the middle pieces in rows 8-15 of one and the last ones of the other.
// head_dim is padded to DP with zeros that are not read from memory.
// All 255 registers are used.  Two sets at 128 channels (9 to 16 heads) spill 176 bytes of a thread and read 276 back, one set at 256 channels 112 and
// 104: with four products of weights and values for a pair of sets, that is why the warps' own work and not memory bounds these two.
constexpr int kPaThreads = 128;
constexpr int kPaWarps = kPaThreads / 32;
constexpr int kPaStages = 3;
constexpr int kPaUnit = 16 * kPaWarps;
__host__ __device__ constexpr int pa_ring_bytes(int DP) { return kPaWarps * kPaStages * 2 * 16 * DP * 2; }
// the ring, the sums of the warps for four heads, the queries (a row of heads' channels is 16 bytes longer: eight rows fall into all banks)
__host__ __device__ constexpr int pa_smem(int DP, int heads) { return pa_ring_bytes(DP) + kPaWarps * 4 * DP * (int)sizeof(float) + heads * (DP + 8) * 2; }
static_assert(2 * (pa_smem(128, 16) + 512 + 1024) <= kSmSharedBytes, "two CTAs on an SM");

__device__ __forceinline__ void ldsm_x2(uint32_t addr, uint32_t& r0, uint32_t& r1)
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x2.shared.b16 {%0, %1}, [%2];" : "=r"(r0), "=r"(r1) : "r"(addr) : "memory");
}
// The product alone, nothing added.
__device__ __forceinline__ void mma_bf16_only(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1)
{
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%10, %10, %10, %10};"
                 : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.f));
}

// What a warp keeps of a segment, and a chunk's products.
template <int NS, bool Q4, int DP> struct PaWarp {
    static_assert(!Q4 || NS == 1, "four heads are one set");
    static constexpr int PR = DP / 8;                // 16-byte pieces of a row
    static constexpr int KS = DP / 16;               // k-steps of the logits
    static constexpr int GP = Q4 ? 4 : 8 * NS;       // heads of a group
    static constexpr uint32_t kOp = 16 * DP * 2;     // bytes of a chunk of K or V
    using Queries = __nv_bfloat16 (*)[DP + 8];
    using Sums = float (*)[4][DP];
    static constexpr bool kKeep = KS * NS <= 8;      // the queries stay in registers; more are read from shared memory at every chunk
    uint32_t qa[kKeep ? KS : 1][2 * NS];
    uint32_t q_at;
    float m[NS], l[NS];
    uint64_t acc[NS][DP / 8][2];                     // packed pairs

    __device__ __forceinline__ void clear()
    {
#pragma unroll
        for (int n = 0; n < NS; ++n) {
            m[n] = -INFINITY;
            l[n] = 0.f;
#pragma unroll
            for (int i = 0; i < DP / 8; ++i) acc[n][i][0] = acc[n][i][1] = pack2(0.f, 0.f);
        }
    }
    __device__ __forceinline__ void take_queries(Queries qs, int lane)
    {
        // row of matrix lane / 8: heads 0-7 and, with two sets, 8-15 of the first eight channels of a k-step, then of the others
        const int mat = lane >> 3, row = Q4 ? lane & 3 : NS == 2 ? (lane & 7) + 8 * (mat & 1) : lane & 7;
        q_at = smem_u32(&qs[row][8 * (NS == 2 ? mat >> 1 : mat & 1)]);
        if constexpr (kKeep)
#pragma unroll
            for (int n = 0; n < NS; ++n) {
                const int hh = Q4 ? (lane >> 2) & 3 : 8 * n + (lane >> 2);
#pragma unroll
                for (int ks = 0; ks < KS; ++ks)
#pragma unroll
                    for (int x = 0; x < 2; ++x)
                        qa[ks][2 * n + x] = *reinterpret_cast<const uint32_t*>(&qs[hh][ks * 16 + x * 8 + 2 * (lane & 3)]);
            }
    }
    // Sixteen rows of K and V at ks_base and vs_base, `there`: which of them exist.
    __device__ __forceinline__ void chunk(uint32_t ks_base, uint32_t vs_base, uint32_t there, float c2, int lane)
    {
        const int lr = lane & 7, mat = lane >> 3;
        float c[2][4];
#pragma unroll
        for (int x = 0; x < 2; ++x)
#pragma unroll
            for (int e = 0; e < 4; ++e) c[x][e] = 0.f;
        {
            const int row = lr + 8 * (mat >> 1);
            const uint32_t base = ks_base + (uint32_t)row * PR * 16;
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) {
                uint32_t b[4];
                ldsm_x4(base + (uint32_t)((2 * ks + (mat & 1)) ^ lr) * 16, b);
                uint32_t a0, a1 = 0u, a2, a3 = 0u;
                if constexpr (kKeep) {
                    a0 = qa[ks][0];
                    a2 = qa[ks][1];
                    if constexpr (NS == 2) { a1 = qa[ks][2]; a3 = qa[ks][3]; }
                } else if constexpr (NS == 2) {
                    uint32_t q[4];
                    ldsm_x4(q_at + ks * 32, q);
                    a0 = q[0]; a1 = q[1]; a2 = q[2]; a3 = q[3];
                } else {
                    ldsm_x2(q_at + ks * 32, a0, a2);
                }
                mma_bf16(c[0], a0, a1, a2, a3, b[0], b[1]);
                mma_bf16(c[1], a0, a1, a2, a3, b[2], b[3]);
            }
        }
        // logits of this thread's heads, rows row0, row0 + 1, row0 + 8, row0 + 9 of the chunk
        const uint32_t seen = there >> (2 * (lane & 3));
        uint32_t hi[NS][2], mid[NS][2], lo[NS][2];
#pragma unroll
        for (int n = 0; n < NS; ++n) {
            float x[4];
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int e = 0; e < 2; ++e) x[2 * t + e] = (seen >> (8 * t + e)) & 1 ? c[t][2 * n + e] : -INFINITY;
            const float mx = fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])) * c2;
            if (__any_sync(0xffffffffu, mx > m[n])) {
                float t = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 1));
                t = fmaxf(t, __shfl_xor_sync(0xffffffffu, t, 2));
                const float mn = fmaxf(m[n], t);
                const float sc = m[n] == -INFINITY ? 0.f : exp2f(m[n] - mn);
                m[n] = mn;
                l[n] *= sc;
                const uint64_t sc2 = pack2(sc, sc);
#pragma unroll
                for (int i = 0; i < DP / 8; ++i)
#pragma unroll
                    for (int e = 0; e < 2; ++e) acc[n][i][e] = mul2(acc[n][i][e], sc2);
            }
            const float mr = m[n] == -INFINITY ? 0.f : m[n];
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                const float p0 = exp2f(fmaf(x[2 * t], c2, -mr)), p1 = exp2f(fmaf(x[2 * t + 1], c2, -mr));
                l[n] += p0 + p1;
                constexpr float kShare = Q4 ? 1.f : 0.5f;      // of the leading piece in one instruction
                hi[n][t] = pack_bf16(kShare * p0, kShare * p1);
                const float q0 = fmaf(-1.f / kShare, __uint_as_float(hi[n][t] << 16), p0);
                const float q1 = fmaf(-1.f / kShare, __uint_as_float(hi[n][t] & 0xffff0000u), p1);
                mid[n][t] = pack_bf16(q0, q1);
                lo[n][t] = pack_bf16(q0 - __uint_as_float(mid[n][t] << 16), q1 - __uint_as_float(mid[n][t] & 0xffff0000u));
            }
            if constexpr (Q4) {
#pragma unroll
                for (int t = 0; t < 2; ++t) {
                    hi[n][t] = lane < 16 ? hi[n][t] : lo[n][t];
                    mid[n][t] = lane < 16 ? mid[n][t] : 0u;
                }
            }
        }
        {
            const int row = lr + 8 * (mat & 1);
            const uint32_t base = vs_base + (uint32_t)row * PR * 16;
#pragma unroll
            for (int i = 0; i < DP / 8; i += 2) {
                uint32_t b[4];
                ldsm_x4_trans(base + (uint32_t)((i + (mat >> 1)) ^ lr) * 16, b);
#pragma unroll
                for (int n = 0; n < NS; ++n)
#pragma unroll
                    for (int t = 0; t < 2; ++t) {
                        // (the instruction rounds its sums towards zero: a chunk's go into registers of their own, and are added
                        // up by additions that round to nearest: 128K rows, 896 a warp, were off by 1.6e-6 the other way, by 6.6e-7 so)
                        float o[4];
                        mma_bf16_only(o, hi[n][0], mid[n][0], hi[n][1], mid[n][1], b[2 * t], b[2 * t + 1]);
                        if constexpr (!Q4) mma_bf16(o, hi[n][0], lo[n][0], hi[n][1], lo[n][1], b[2 * t], b[2 * t + 1]);
                        acc[n][i + t][0] = add2(acc[n][i + t][0], pack2(o[0], o[1]));
                        acc[n][i + t][1] = add2(acc[n][i + t][1], pack2(o[2], o[3]));
                    }
            }
        }
    }
    __device__ __forceinline__ void join_lanes()
    {
#pragma unroll
        for (int n = 0; n < NS; ++n) {
            l[n] += __shfl_xor_sync(0xffffffffu, l[n], 1);
            l[n] += __shfl_xor_sync(0xffffffffu, l[n], 2);
        }
    }
    // The warp's sums of heads 4 r .. 4 r + 3, the pieces added.
    __device__ __forceinline__ void put(int r, Sums accs, float (*ms)[4], float (*ls)[4], int warp, int lane) const
    {
        const int n = r / 2;
        const bool mine = lane >> 4 == (r & 1);      // (with four heads, lanes 16 to 31 have copies)
#pragma unroll
        for (int i = 0; i < DP / 8; ++i) {
            float x[2], v[4];
            unpack2(acc[n][i][0], v[0], v[1]);
            unpack2(acc[n][i][1], v[2], v[3]);
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const float less = Q4 ? v[2 + e] + __shfl_down_sync(0xffffffffu, v[e], 16) : v[2 + e];
                // an infinite value times a smaller piece is an infinity of either sign or, where the piece is zero, no
                // number: the leading piece alone says what the weight times the value is
                x[e] = isinf(v[e]) ? v[e] : v[e] + less;
            }
            if (mine) *reinterpret_cast<float2*>(&accs[warp][(lane >> 2) & 3][i * 8 + 2 * (lane & 3)]) = make_float2(x[0], x[1]);
        }
        if (mine && (lane & 3) == 0) { ms[warp][(lane >> 2) & 3] = m[n]; ls[warp][(lane >> 2) & 3] = l[n]; }
    }
};

// The warps' sums of one of four heads, columns d .. d + 3, in their order.
template <int DP>
__device__ __forceinline__ void pa_join(const float (*accs)[4][DP], const float (*ms)[4], const float (*ls)[4], int hs, int d, float4& sum, float& mx, float& lsum)
{
    mx = -INFINITY;
#pragma unroll
    for (int v = 0; v < kPaWarps; ++v) mx = fmaxf(mx, ms[v][hs]);
    sum = make_float4(0.f, 0.f, 0.f, 0.f);
    lsum = 0.f;
#pragma unroll
    for (int v = 0; v < kPaWarps; ++v) {
        if (ls[v][hs] == 0.f) continue;              // (a warp without rows; one whose sum is no number counts)
        const float wt = ms[v][hs] == -INFINITY ? 1.f : exp2f(ms[v][hs] - mx);
        const float4 x = *reinterpret_cast<const float4*>(&accs[v][hs][d]);
        sum.x += x.x * wt; sum.y += x.y * wt; sum.z += x.z * wt; sum.w += x.w * wt;
        lsum += ls[v][hs] * wt;
    }
}

// Copies of a chunk's rows into a warp's ring, found by its lanes (lane r and lane r + 16 have row r); which rows exist, a bit each.
template <int DP>
__device__ __forceinline__ uint32_t pa_copy(const PagedAttnArgs& a, const PgRow& row, const __nv_bfloat16* kb, const __nv_bfloat16* vb, uint32_t dst, int lane)
{
    constexpr int PR = DP / 8;
    const int pc = lane % PR;
    const bool piece_there = pc < a.D / 8, ok = row.ok && a.pg.holds(row.page);
    const long long ko = ok ? (long long)row.page * a.pg.k_page + (long long)row.slot * a.pg.k_row : -1;
    const long long vo = a.same_place ? ko : ok ? (long long)row.page * a.pg.v_page + (long long)row.slot * a.pg.v_row : -1;
#pragma unroll
    for (int i = 0; i < PR / 2; ++i) {
        const int rr = lane / PR + i * (32 / PR);
        const long long k_at = __shfl_sync(0xffffffffu, ko, rr);
        const long long v_at = a.same_place ? k_at : __shfl_sync(0xffffffffu, vo, rr);
        const bool there = k_at >= 0 && piece_there;
        const uint32_t o = dst + (uint32_t)(rr * PR + (pc ^ (rr & 7))) * 16;
        cp_async16_or_zero(o, kb + (there ? k_at + pc * 8 : 0), there);
        cp_async16_or_zero(o + 16 * DP * 2, vb + (there ? v_at + pc * 8 : 0), there);
    }
    return __ballot_sync(0xffffffffu, ok) & 0xffffu;
}

// The queries of a group, asked for by a CTA and put into its shared memory.
template <int GP, int DP> struct PaQueries {
    static constexpr int PR = DP / 8, N = (GP * PR + kPaThreads - 1) / kPaThreads;
    uint4 x[N];
    __device__ __forceinline__ void ask(const PagedAttnArgs& a, size_t head, int heads)
    {
#pragma unroll
        for (int t = 0; t < N; ++t) {
            const int i = threadIdx.x + t * kPaThreads, h = min(i / PR, heads - 1), c = min(i % PR, a.D / 8 - 1);
            x[t] = *reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(a.q) + (head + h) * a.D + c * 8);
        }
    }
    __device__ __forceinline__ void put(__nv_bfloat16 (*qs)[DP + 8], int D) const
    {
#pragma unroll
        for (int t = 0; t < N; ++t) {
            const int i = threadIdx.x + t * kPaThreads;
            if (i < GP * PR) *reinterpret_cast<uint4*>(&qs[i / PR][i % PR * 8]) = i % PR < D / 8 ? x[t] : make_uint4(0, 0, 0, 0);
        }
    }
};

// CTAs on an SM: what shared memory holds.  (Three with 64 channels were no faster: 16 sequences of 4K to 16K rows 63 and 61 us.)
__host__ __device__ constexpr int pa_per_sm(int DP) { return DP == 256 ? 1 : 2; }

template <int NS, bool Q4, int DP>
__global__ void __launch_bounds__(kPaThreads, pa_per_sm(DP))
paged_mma_kernel(const __grid_constant__ PagedAttnArgs a)
{
    using Warp = PaWarp<NS, Q4, DP>;
    constexpr uint32_t kOp = Warp::kOp;
    using bf16 = __nv_bfloat16;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    extern __shared__ __align__(128) uint8_t pa_ring[];
    const typename Warp::Sums accs = reinterpret_cast<typename Warp::Sums>(pa_ring + pa_ring_bytes(DP));
    const typename Warp::Queries qs = reinterpret_cast<typename Warp::Queries>(pa_ring + pa_ring_bytes(DP) + kPaWarps * 4 * DP * sizeof(float));
    __shared__ float ms[kPaWarps][4], ls[kPaWarps][4];
    const uint32_t ring = smem_u32(pa_ring) + warp * kPaStages * 2 * kOp;
    pdl_wait();
    pdl_launch();
    const int pairs = a.Hkv * a.groups / a.columns;  // of a sequence in this CTA's column
    PgShare sh = pg_share<kPaThreads, kPaUnit>(a, pairs);
    if (tid == 0) a.jobs[blockIdx.x] = make_int4(0, 0, 0, 0);
    if (sh.u >= sh.u_end) return;
    int s = sh.s, pair, w;
    {
        const long long units = max(1, (a.listed_rows(s) + kPaUnit - 1) / kPaUnit);
        pair = (int)(sh.skip / units);
        w = (int)(sh.skip - pair * units);
    }
    auto chunks_of = [&](const PgSegment& g) { return ((g.row1 > g.row0 ? (g.row1 - g.row0 + 15) / 16 : 0) - warp + kPaWarps - 1) / kPaWarps; };

    // The copies: a cursor of its own, kPaStages - 1 chunks ahead of the products and over the ends of segments, so that the loads of the
    // next segment are on their way while one is merged.  A chunk's rows are looked up one chunk, their pages two chunks earlier.
    struct {
        long long left;                              // units of the share that are not opened
        int s, pair, w;
        int k, n;                                    // next chunk of this warp in the open segment, and its chunks
        int stage;
    } io = {sh.u_end - sh.u, s, pair, w, 0, 0, 0};
    PgLook look;
    const bf16 *kb, *vb;
    int io_row;                                      // this lane's row of the open segment's chunk 0
    PgRow next;
    int next_j;
    uint32_t there_ring = 0;                         // which rows of the chunks in flight exist, 16 bits each, the newest on top
    static_assert(kPaStages == 3, "two chunks in flight beside the one at hand");
    auto open = [&] {                                // the next segment that has chunks for this warp
        while (io.k == io.n && io.left > 0) {
            const PgSegment g = pg_segment<kPaUnit>(a, io.s, io.pair, io.w, io.left);
            io.left -= min(g.units - io.w, io.left);
            io.w = 0;
            if (++io.pair == pairs) { io.pair = 0; ++io.s; }
            io.k = 0;
            io.n = chunks_of(g);
            if (io.n == 0) continue;
            look = pg_look(a, g);
            kb = static_cast<const bf16*>(a.pg.k) + (size_t)g.hk * a.pg.k_head;
            vb = static_cast<const bf16*>(a.pg.v) + (size_t)g.hk * a.pg.v_head;
            io_row = g.row0 + warp * 16 + (lane & 15);
            const int j = pg_listed(a, look, io_row);
            next_j = pg_listed(a, look, io_row + kPaUnit);
            next = pg_find(a, look, io_row, j);
        }
    };
    auto step = [&] {
        uint32_t there_rows = 0;
        if (io.k < io.n) {
            there_rows = pa_copy<DP>(a, next, kb, vb, ring + (uint32_t)io.stage * 2 * kOp, lane);
            ++io.k;
            next = pg_find(a, look, io_row + io.k * kPaUnit, next_j);
            next_j = pg_listed(a, look, io_row + (io.k + 1) * kPaUnit);
            io.stage = io.stage == kPaStages - 1 ? 0 : io.stage + 1;
            open();                                  // (its look-ups are on their way until the next step)
        }
        there_ring = there_ring >> 16 | there_rows << 16;
        cp_async_commit();
    };
    // The queries of a segment are asked for while the segment before is worked on, and put into shared memory at its end.
    PaQueries<Warp::GP, DP> queries;
    PgSegment g = pg_segment<kPaUnit>(a, s, pair, w, sh.u_end - sh.u);
    queries.ask(a, pg_head(a, g), g.heads);
    int stage = 0;
    open();
    step();
    step();
    queries.put(qs, a.D);
    __syncthreads();
    Warp me;
    while (true) {
        me.take_queries(qs, lane);
        const PgSegment at = g;                      // the segment at hand; g is the next one from here on
        const long long unit = sh.u;
        sh.u += min(g.units - w, sh.u_end - sh.u);
        w = 0;
        if (++pair == pairs) { pair = 0; ++s; }
        const bool more = sh.u < sh.u_end;
        if (more) {
            g = pg_segment<kPaUnit>(a, s, pair, w, sh.u_end - sh.u);
            queries.ask(a, pg_head(a, g), g.heads);
        }
        me.clear();
        const int n_it = chunks_of(at);
        for (int it = 0; it < n_it; ++it) {
            const uint32_t there = there_ring & 0xffffu;         // (of the two chunks in flight, the older one)
            step();
            cp_async_wait<kPaStages - 1>();
            __syncwarp();
            const uint32_t base = ring + (uint32_t)stage * 2 * kOp;
            me.chunk(base, base + kOp, there, a.c2, lane);
            stage = stage == kPaStages - 1 ? 0 : stage + 1;
            __syncwarp();                            // the stage may be refilled
        }
        // The segment is over: the warps are merged, in a fixed order, four heads at a time.
        if (tid == 0 && at.first && !at.last) {
            // the pair goes on in the next shares: the last unit of it is unit `end` of the line
            const long long end = unit + at.units - 1;
            a.jobs[blockIdx.x] = make_int4((int)pg_head(a, at), at.heads, (int)(end / sh.quota) - (int)blockIdx.x / a.columns + 1, 0);
        }
        me.join_lanes();
#pragma unroll
        for (int r = 0; r < Warp::GP / 4; ++r) {
            me.put(r, accs, ms, ls, warp, lane);
            __syncthreads();
            if (r == 0 && more) queries.put(qs, a.D);    // (every warp has taken those of this segment)
            for (int i = tid; i < DP; i += kPaThreads) {
                const int hs = i / (DP / 4), h = 4 * r + hs, d = 4 * (i % (DP / 4));
                if (h >= at.heads || d >= a.D) continue;
                float4 sum;
                float mx, lsum;
                pa_join<DP>(accs, ms, ls, hs, d, sum, mx, lsum);
                pg_emit4(a, at, h, d, sum, mx, lsum);
            }
            __syncthreads();                             // the sums may be written again
        }
        if (!more) break;
    }
    cp_async_wait<0>();
}

// ---- bf16, one launch -------------------------------------------------------------------------------------
// Where a cluster of CTAs has all of a pair, the parts are merged on chip and there is no second launch; and where pages are to be
// chosen (SEL), it chooses them too: every CTA scores a share of the pages, leaves the keys with all CTAs of the cluster, and each
// chooses for itself (the choice costs less than handing it round).  The keys lie where the ring is later.  Bound by latencies one
// behind the other: 16 sequences of 4K to 16K rows, 48 of their 128 to 512 pages of 32 rows, 39 us: scores 4 to 12, choosing 3, the
// first look-up 2, the stream 14, merging 2.
constexpr int kPcMaxCluster = 8;
__host__ __device__ constexpr int pc_keys(int DP) { return pa_ring_bytes(DP) / 4; }      // pages whose keys there is room for
constexpr int kPcMaxList = 1024;                     // chosen pages
__host__ __device__ constexpr int pc_smem(int DP, int heads, int n_sel) { return pa_smem(DP, heads) + n_sel * 4; }
static_assert(2 * (pc_smem(128, 8, kPcMaxList) + 512 + 1024) <= kSmSharedBytes, "two CTAs on an SM");

__device__ __forceinline__ float4 ld_cluster_f4(const void* p, int rank)
{
    float4 v;
    asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(cluster_map(p, rank)) : "memory");
    return v;
}

template <bool Q4, int DP, bool SEL>
__global__ void __launch_bounds__(kPaThreads, 2)
paged_cluster_kernel(const __grid_constant__ PagedAttnArgs a, const __grid_constant__ PageSelectArgs ps, int n_cta)
{
    using Warp = PaWarp<1, Q4, DP>;
    constexpr uint32_t kOp = Warp::kOp;
    constexpr int GP = Warp::GP;
    using bf16 = __nv_bfloat16;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int rank = blockIdx.x, hk = blockIdx.y, s = blockIdx.z;
    extern __shared__ __align__(128) uint8_t pa_ring[];
    const typename Warp::Sums accs = reinterpret_cast<typename Warp::Sums>(pa_ring + pa_ring_bytes(DP));
    const typename Warp::Queries qs = reinterpret_cast<typename Warp::Queries>(pa_ring + pa_ring_bytes(DP) + kPaWarps * 4 * DP * sizeof(float));
    int* list = reinterpret_cast<int*>(pa_ring + pa_smem(DP, GP));
    __shared__ float ms[kPaWarps][4], ls[kPaWarps][4];
    __shared__ __align__(16) float2 cml[GP];         // this CTA's maxima and sums
    const uint32_t ring = smem_u32(pa_ring) + warp * kPaStages * 2 * kOp;
    pdl_wait();
    pdl_launch();
    const int len = a.pg.rows_of(s);
    const size_t head = (size_t)s * a.H + (size_t)hk * a.G;
    PaQueries<GP, DP> queries;
    queries.ask(a, head, a.G);
    int rows = len;
    if constexpr (SEL) {
        const int P = a.pg.by_page.div(len + a.pg.page_size - 1), n = min(ps.n_sel, P);
        int* sel = ps.sel + ((size_t)s * a.Hkv + hk) * ps.n_sel;
        if (P > ps.n_sel) {
            uint32_t* keys = reinterpret_cast<uint32_t*>(pa_ring);
            auto& mem = *reinterpret_cast<ChooseMem<kPaThreads>*>(accs);
            static_assert(sizeof(ChooseMem<kPaThreads>) <= pa_smem(DP, GP) - pa_ring_bytes(DP), "what choosing needs lies where sums and queries are later");
            if (n_cta > 1) cluster_arrive();
            score_pages<bf16, 1, 16>(ps, s, hk, P, (rank * kPaWarps + warp) * 16, n_cta * kPaWarps * 16,
                [&] { if (n_cta > 1) cluster_await(); },           // the others have started: their memory may be written
                [&](int j, uint32_t key) {
                    if (n_cta == 1) {
                        if ((lane & 3) == 0) keys[j] = key;
                        return;
                    }
                    for (int r = lane & 3; r < n_cta; r += 4) st_cluster_u32(keys + j, r, key);
                });
            if (n_cta > 1) cluster_sync();
            else __syncthreads();
            choose_pages<kPaThreads>(keys, P, ps.n_sel, ps.n_first + ps.n_last, mem, [&](int at, int j) {
                list[at] = j;
                if (rank == 0) sel[at] = j;
            });
        } else {
            for (int i = tid; i < ps.n_sel; i += kPaThreads) {
                if (i < P) list[i] = i;
                if (rank == 0) sel[i] = i < P ? i : -1;
            }
        }
        rows = n * a.pg.page_size;
        __syncthreads();                             // the list is there, the keys have been read
    }
    queries.put(qs, a.D);
    const int units = (rows + kPaUnit - 1) / kPaUnit, share = (units + n_cta - 1) / n_cta;
    const int row0 = min(rows, rank * share * kPaUnit), row1 = min(rows, row0 + share * kPaUnit);
    const int n_it = ((row1 - row0 + 15) / 16 - warp + kPaWarps - 1) / kPaWarps;
    const bf16* kb = static_cast<const bf16*>(a.pg.k) + (size_t)hk * a.pg.k_head;
    const bf16* vb = static_cast<const bf16*>(a.pg.v) + (size_t)hk * a.pg.v_head;
    PgLook look;
    look.table = a.pg.table + (long long)s * a.pg.table_stride;
    look.sel = nullptr;
    look.rows = row1;
    look.len = len;
    const int my_row = row0 + warp * 16 + (lane & 15);
    auto find = [&](int it) {                        // row of chunk `it`
        const int v = my_row + it * kPaUnit;
        int j = a.pg.by_page.div(max(0, min(v, row1 - 1)));
        if constexpr (SEL) j = row1 > 0 ? list[j] : -1;
        return pg_find(a, look, v, j);
    };
    uint32_t there_ring = 0;
    PgRow next;
    auto step = [&](int it) {
        uint32_t there_rows = 0;
        if (it < n_it) there_rows = pa_copy<DP>(a, next, kb, vb, ring + (uint32_t)(it % kPaStages) * 2 * kOp, lane);
        next = find(it + 1);
        there_ring = there_ring >> 16 | there_rows << 16;
        cp_async_commit();
    };
    next = find(0);
    step(0);
    step(1);
    __syncthreads();
    Warp me;
    me.take_queries(qs, lane);
    me.clear();
    for (int it = 0; it < n_it; ++it) {
        const uint32_t there = there_ring & 0xffffu;
        step(it + kPaStages - 1);
        cp_async_wait<kPaStages - 1>();
        __syncwarp();
        const uint32_t base = ring + (uint32_t)(it % kPaStages) * 2 * kOp;
        me.chunk(base, base + kOp, there, a.c2, lane);
        __syncwarp();
    }
    cp_async_wait<0>();
    me.join_lanes();
    // ---- merge: the warps (the CTA's sums go where the ring was), then the CTAs
    float (*csum)[DP] = reinterpret_cast<float (*)[DP]>(pa_ring);
    static_assert(GP * DP * (int)sizeof(float) <= pa_ring_bytes(DP), "sums fit in the ring");
#pragma unroll
    for (int r = 0; r < GP / 4; ++r) {
        me.put(r, accs, ms, ls, warp, lane);
        __syncthreads();
        for (int i = tid; i < DP; i += kPaThreads) {
            const int hs = i / (DP / 4), h = 4 * r + hs, d = 4 * (i % (DP / 4));
            float4 sum;
            float mx, lsum;
            pa_join<DP>(accs, ms, ls, hs, d, sum, mx, lsum);
            *reinterpret_cast<float4*>(&csum[h][d]) = sum;
            if (d == 0) cml[h] = make_float2(mx, lsum);
        }
        __syncthreads();
    }
    if (n_cta > 1) cluster_sync();
    for (int i = rank * kPaThreads + tid; i < GP * DP / 4; i += n_cta * kPaThreads) {
        const int h = i / (DP / 4), d = 4 * (i % (DP / 4));
        if (h >= a.G || d >= a.D) continue;
        float M = -INFINITY;
        for (int c = 0; c < n_cta; ++c) M = fmaxf(M, ld_cluster_f32(&cml[h].x, c));
        float4 num = make_float4(0.f, 0.f, 0.f, 0.f);
        float den = 0.f;
#pragma unroll 4
        for (int c = 0; c < n_cta; ++c) {
            const float m = ld_cluster_f32(&cml[h].x, c), l = ld_cluster_f32(&cml[h].y, c);
            const float4 x = ld_cluster_f4(&csum[h][d], c);
            if (l == 0.f) continue;
            const float w = m == -INFINITY ? 1.f : exp2f(m - M);
            num.x += x.x * w; num.y += x.y * w; num.z += x.z * w; num.w += x.w * w;
            den += l * w;
        }
        float* dst = a.out + (head + h) * a.D + d;
        dst[0] = den == 0.f ? 0.f : num.x / den;
        dst[1] = den == 0.f ? 0.f : num.y / den;
        dst[2] = den == 0.f ? 0.f : num.z / den;
        dst[3] = den == 0.f ? 0.f : num.w / den;
        if (a.lse && d == 0) a.lse[head + h] = den == 0.f ? -INFINITY : (M + log2f(den)) * 0.6931471805599453f;
    }
    if (n_cta > 1) cluster_sync();                   // the others may still read this one's sums
}

// ---- fp32 -----------------------------------------------------------------------------------------------
// Multiply-adds.  A warp's chunk is eight rows: for the logits four lanes share a row (lane = 4 row + part, pieces part, part + 4, ...),
// for the weighted values a lane owns columns and the weights go round through shared memory.
constexpr int kPfRows = 8;
constexpr int kPfStages = 3;
constexpr int kPfUnit = kPfRows * kPaWarps;
// Where piece p of row r of a chunk lies: the two rows that eight lanes read at a time for the logits fall into different banks.
__device__ __forceinline__ int pf_piece(int r, int p) { return p ^ ((r & 1) << 2 | r >> 1); }
__host__ __device__ constexpr int pf_smem(int DP) { return kPaWarps * kPfStages * 2 * kPfRows * DP * 4; }

template <int GP, int DP>
__global__ void __launch_bounds__(kPaThreads, DP == 256 ? 1 : 2)
paged_fma_kernel(const __grid_constant__ PagedAttnArgs a)
{
    constexpr int PR = DP / 4;                       // 16-byte pieces of a row
    constexpr uint32_t kOp = kPfRows * DP * 4;
    constexpr int CW = DP / 32;                      // columns of a lane: 2, 4 or 8, in runs of at most four
    constexpr int RUN = CW < 4 ? CW : 4;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    extern __shared__ __align__(128) uint8_t pa_ring[];
    __shared__ __align__(16) float qs[GP][DP];
    __shared__ __align__(16) float ws[kPaWarps][kPfRows][GP];
    __shared__ float ms[kPaWarps][GP], ls[kPaWarps][GP];
    const uint32_t ring = smem_u32(pa_ring) + warp * kPfStages * 2 * kOp;
    const uint8_t* ring_p = pa_ring + warp * kPfStages * 2 * kOp;
    pdl_wait();
    pdl_launch();
    const int pairs = a.Hkv * a.groups / a.columns;  // of a sequence in this CTA's column
    PgShare sh = pg_share<kPaThreads, kPfUnit>(a, pairs);
    if (tid == 0) a.jobs[blockIdx.x] = make_int4(0, 0, 0, 0);
    if (sh.u >= sh.u_end) return;
    int s = sh.s, pair, w;
    {
        const long long units = max(1, (a.listed_rows(s) + kPfUnit - 1) / kPfUnit);
        pair = (int)(sh.skip / units);
        w = (int)(sh.skip - pair * units);
    }
    const int n_pieces = a.D / 4;
    while (sh.u < sh.u_end) {
        const PgSegment g = pg_segment<kPfUnit>(a, s, pair, w, sh.u_end - sh.u);
        const PgLook look = pg_look(a, g);
        const int chunks = g.row1 > g.row0 ? (g.row1 - g.row0 + kPfRows - 1) / kPfRows : 0;
        const int n_it = (chunks - warp + kPaWarps - 1) / kPaWarps;
        const float* kb = static_cast<const float*>(a.pg.k) + (size_t)g.hk * a.pg.k_head;
        const float* vb = static_cast<const float*>(a.pg.v) + (size_t)g.hk * a.pg.v_head;
        auto row_of = [&](int it) { return g.row0 + (it * kPaWarps + warp) * kPfRows + (lane & 7); };
        auto listed = [&](int it) { return pg_listed(a, look, row_of(it)); };
        auto find = [&](int it, int j) { return pg_find(a, look, row_of(it), j); };
        auto issue = [&](int it, const PgRow r) {
            if (it < n_it) {
                const uint32_t dst = ring + (uint32_t)(it % kPfStages) * 2 * kOp;
                const bool ok = r.ok && a.pg.holds(r.page);
                const long long ko = ok ? (long long)r.page * a.pg.k_page + (long long)r.slot * a.pg.k_row : -1;
                const long long vo = ok ? (long long)r.page * a.pg.v_page + (long long)r.slot * a.pg.v_row : -1;
#pragma unroll
                for (int i = 0; i < kPfRows * PR / 32; ++i) {
                    const int id = i * 32 + lane, rr = id / PR, pc = id % PR;
                    const long long k_at = __shfl_sync(0xffffffffu, ko, rr), v_at = __shfl_sync(0xffffffffu, vo, rr);
                    const bool there = k_at >= 0 && pc < n_pieces;
                    const uint32_t o = dst + (uint32_t)(rr * PR + pf_piece(rr, pc)) * 16;
                    cp_async16_or_zero(o, kb + (there ? k_at + pc * 4 : 0), there);
                    cp_async16_or_zero(o + kOp, vb + (there ? v_at + pc * 4 : 0), there);
                }
            }
            cp_async_commit();
        };
        uint32_t there_ring[kPfStages - 1];
        {
            PgRow r[kPfStages - 1];
            int j[kPfStages - 1];
#pragma unroll
            for (int t = 0; t < kPfStages - 1; ++t) j[t] = listed(t);
#pragma unroll
            for (int t = 0; t < kPfStages - 1; ++t) r[t] = find(t, j[t]);
#pragma unroll
            for (int t = 0; t < kPfStages - 1; ++t) {
                there_ring[t] = __ballot_sync(0xffffffffu, r[t].ok && a.pg.holds(r[t].page)) & 0xffu;
                issue(t, r[t]);
            }
        }
        PgRow next = find(kPfStages - 1, listed(kPfStages - 1));
        int next_j = listed(kPfStages);
        for (int i = tid; i < GP * DP; i += kPaThreads) {
            const int h = i / DP, d = i - h * DP;
            qs[h][d] = h < g.heads && d < a.D ? static_cast<const float*>(a.q)[(pg_head(a, g) + h) * a.D + d] * a.c2 : 0.f;
        }
        __syncthreads();
        float m[GP], l[GP], acc[GP][CW];
#pragma unroll
        for (int h = 0; h < GP; ++h) {
            m[h] = -INFINITY;
            l[h] = 0.f;
#pragma unroll
            for (int e = 0; e < CW; ++e) acc[h][e] = 0.f;
        }
        const int row = lane >> 2, part = lane & 3;
        for (int it = 0; it < n_it; ++it) {
            const uint32_t there = there_ring[0];
#pragma unroll
            for (int t = 0; t + 1 < kPfStages - 1; ++t) there_ring[t] = there_ring[t + 1];
            there_ring[kPfStages - 2] = __ballot_sync(0xffffffffu, next.ok && a.pg.holds(next.page)) & 0xffu;
            issue(it + kPfStages - 1, next);
            next = find(it + kPfStages, next_j);
            next_j = listed(it + kPfStages + 1);
            cp_async_wait<kPfStages - 1>();
            __syncwarp();
            const uint8_t* kc = ring_p + (it % kPfStages) * 2 * kOp;
            const uint8_t* vc = kc + kOp;
            float x[GP];
#pragma unroll
            for (int h = 0; h < GP; ++h) x[h] = 0.f;
#pragma unroll 4
            for (int i = 0; i < PR / 4; ++i) {
                const int pc = 4 * i + part;
                const float4 kv = *reinterpret_cast<const float4*>(kc + (row * PR + pf_piece(row, pc)) * 16);
#pragma unroll
                for (int h = 0; h < GP; ++h) {
                    const float4 qv = *reinterpret_cast<const float4*>(&qs[h][pc * 4]);
                    x[h] = fmaf(qv.x, kv.x, fmaf(qv.y, kv.y, fmaf(qv.z, kv.z, fmaf(qv.w, kv.w, x[h]))));
                }
            }
#pragma unroll
            for (int h = 0; h < GP; ++h) {
                x[h] += __shfl_xor_sync(0xffffffffu, x[h], 1);
                x[h] += __shfl_xor_sync(0xffffffffu, x[h], 2);
                if (!((there >> row) & 1)) x[h] = -INFINITY;
                if (__any_sync(0xffffffffu, x[h] > m[h])) {
                    float t = x[h];
#pragma unroll
                    for (int o = 4; o < 32; o <<= 1) t = fmaxf(t, __shfl_xor_sync(0xffffffffu, t, o));
                    const float mn = fmaxf(m[h], t);
                    const float sc = m[h] == -INFINITY ? 0.f : exp2f(m[h] - mn);
                    m[h] = mn;
                    l[h] *= sc;
#pragma unroll
                    for (int e = 0; e < CW; ++e) acc[h][e] *= sc;
                }
                const float p = exp2f(x[h] - (m[h] == -INFINITY ? 0.f : m[h]));
                l[h] += p;                           // (the four lanes of a row hold the same)
                if (part == 0) ws[warp][row][h] = p;
            }
            __syncwarp();
#pragma unroll
            for (int r = 0; r < kPfRows; ++r) {
                float v[CW];
#pragma unroll
                for (int c = 0; c < CW / RUN; ++c) {
                    const int d = (c * 32 + lane) * RUN;         // first column of the run
                    const float* src = reinterpret_cast<const float*>(vc + (r * PR + pf_piece(r, d / 4)) * 16) + (d & 3);
                    if constexpr (RUN == 4) {
                        const float4 t = *reinterpret_cast<const float4*>(src);
                        v[4 * c] = t.x; v[4 * c + 1] = t.y; v[4 * c + 2] = t.z; v[4 * c + 3] = t.w;
                    } else {
                        const float2 t = *reinterpret_cast<const float2*>(src);
                        v[0] = t.x; v[1] = t.y;
                    }
                }
#pragma unroll
                for (int h = 0; h < GP; ++h) {
                    const float p = ws[warp][r][h];
#pragma unroll
                    for (int e = 0; e < CW; ++e) acc[h][e] = fmaf(p, v[e], acc[h][e]);
                }
            }
            __syncwarp();                            // the stage may be refilled, the weights written again
        }
        cp_async_wait<0>();
        __syncthreads();
        float (*accs)[GP][DP] = reinterpret_cast<float (*)[GP][DP]>(pa_ring);
        static_assert(kPaWarps * GP * DP * (int)sizeof(float) <= pf_smem(DP), "accumulators fit in the ring");
#pragma unroll
        for (int h = 0; h < GP; ++h) {
#pragma unroll
            for (int o = 4; o < 32; o <<= 1) l[h] += __shfl_xor_sync(0xffffffffu, l[h], o);
#pragma unroll
            for (int e = 0; e < CW; ++e) accs[warp][h][((e / RUN) * 32 + lane) * RUN + e % RUN] = acc[h][e];
            if (lane == 0) { ms[warp][h] = m[h]; ls[warp][h] = l[h]; }
        }
        __syncthreads();
        for (int i = tid; i < g.heads * a.D; i += kPaThreads) {
            const int h = i / a.D, d = i - h * a.D;
            float mx = -INFINITY;
#pragma unroll
            for (int v = 0; v < kPaWarps; ++v) mx = fmaxf(mx, ms[v][h]);
            float sum = 0.f, lsum = 0.f;
#pragma unroll
            for (int v = 0; v < kPaWarps; ++v) {
                if (ls[v][h] == 0.f) continue;
                const float wt = ms[v][h] == -INFINITY ? 1.f : exp2f(ms[v][h] - mx);
                sum += accs[v][h][d] * wt;
                lsum += ls[v][h] * wt;
            }
            pg_emit(a, g, h, d, sum, mx, lsum);
        }
        if (tid == 0 && g.first && !g.last) {
            const long long end = sh.u + g.units - 1;
            a.jobs[blockIdx.x] = make_int4((int)pg_head(a, g), g.heads, (int)(end / sh.quota) - (int)blockIdx.x / a.columns + 1, 0);
        }
        const long long n = min(g.units - w, sh.u_end - sh.u);
        sh.u += n;
        w = 0;
        if (++pair == pairs) { pair = 0; ++s; }
        __syncthreads();
    }
}

// ---- merging --------------------------------------------------------------------------------------------
// Block (share, head): the pair that begins in the share and goes on in others, its parts in their order.  A thread has four columns and
// every n-th part; it asks for its first parts before the weights are known, which are found meanwhile.
constexpr int kPmThreads = 256;
constexpr int kPmMaxParts = 1024;                    // shares of a call
constexpr int kPmAhead = 5;

__global__ void __launch_bounds__(kPmThreads)
paged_merge_kernel(const __grid_constant__ PagedAttnArgs a)
{
    const int b = blockIdx.x, h = blockIdx.y, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    __shared__ float w_s[kPmMaxParts];
    __shared__ float red[kPmThreads / 32], red_l[kPmThreads / 32];
    __shared__ float4 num_s[kPmThreads];
    pdl_wait();
    pdl_launch();
    const int4 job = a.jobs[b];
    if (h >= job.y) return;
    const int n = job.z, D = a.D, quads = D / 4, slices = kPmThreads / quads, slice = tid / quads, d = 4 * (tid - slice * quads);
    // part i: of the i-th share from this one on, at its end for the first, at its start for the others
    auto part = [&](int i) { return a.part + (((size_t)2 * (b + i * a.columns) + (i == 0 ? 1 : 0)) * a.group_heads + h) * (D + 4); };
    const bool mine = slice < slices;
    float4 x[kPmAhead];
#pragma unroll
    for (int t = 0; t < kPmAhead; ++t) {
        const int i = slice + t * slices;
        x[t] = *reinterpret_cast<const float4*>(part(min(i, n - 1)) + (mine ? d : 0));      // (no branch between the loads)
    }
    float2 ml[(kPmMaxParts + kPmThreads - 1) / kPmThreads];
    float mx = -INFINITY;
#pragma unroll
    for (int t = 0; t < kPmMaxParts / kPmThreads; ++t) {
        const int i = tid + t * kPmThreads;
        ml[t] = make_float2(-INFINITY, 0.f);
        if (i < n) ml[t] = *reinterpret_cast<const float2*>(part(i) + D);
        mx = fmaxf(mx, ml[t].x);
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, o));
    if (lane == 0) red[warp] = mx;
    __syncthreads();
    float M = -INFINITY, l = 0.f;
#pragma unroll
    for (int i = 0; i < kPmThreads / 32; ++i) M = fmaxf(M, red[i]);
#pragma unroll
    for (int t = 0; t < kPmMaxParts / kPmThreads; ++t) {
        // (a part without rows weighs nothing; one whose sum is no number counts)
        const float w = ml[t].y == 0.f ? 0.f : ml[t].x == -INFINITY ? 1.f : exp2f(ml[t].x - M);
        if (tid + t * kPmThreads < n) w_s[tid + t * kPmThreads] = w;
        l += ml[t].y == 0.f ? 0.f : ml[t].y * w;
    }
    l = warp_sum(l);
    if (lane == 0) red_l[warp] = l;
    __syncthreads();
    float4 num = make_float4(0.f, 0.f, 0.f, 0.f);
    auto add = [&](const float4& v, float w) {
        if (w == 0.f) return;                        // (what a part without weight holds does not count)
        num.x += v.x * w; num.y += v.y * w; num.z += v.z * w; num.w += v.w * w;
    };
    if (mine) {
#pragma unroll
        for (int t = 0; t < kPmAhead; ++t)
            if (slice + t * slices < n) add(x[t], w_s[slice + t * slices]);
#pragma unroll 4
        for (int i = slice + kPmAhead * slices; i < n; i += slices) {
            const float4 v = *reinterpret_cast<const float4*>(part(i) + d);
            add(v, w_s[i]);
        }
    }
    num_s[tid] = num;
    __syncthreads();
    if (slice != 0) return;
    float den = 0.f;
#pragma unroll
    for (int i = 0; i < kPmThreads / 32; ++i) den += red_l[i];
    for (int i = 1; i < slices; ++i) {
        const float4 v = num_s[i * quads + tid];
        num.x += v.x; num.y += v.y; num.z += v.z; num.w += v.w;
    }
    const size_t row = (size_t)job.x + h;
    float* out = a.out + row * D + d;
    out[0] = den == 0.f ? 0.f : num.x / den;
    out[1] = den == 0.f ? 0.f : num.y / den;
    out[2] = den == 0.f ? 0.f : num.z / den;
    out[3] = den == 0.f ? 0.f : num.w / den;
    if (a.lse && tid == 0) a.lse[row] = den == 0.f ? -INFINITY : (M + log2f(den)) * 0.6931471805599453f;
}

}  // namespace sab
