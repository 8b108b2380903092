// A paged key-value cache: rows of K and V of a sequence lie in pages of page_size rows, page j of sequence s in page
// table[s][j] of a pool that all sequences share.  This file: rows go into pages, keys and queries rotated on the way
// (paged_append_kernel); which pages of a sequence a new token's queries look at (page_select_kernel).  The attention over the
// pages is in paged_attn.cuh.
//
// Whatever the device arrays say, no access leaves the pool, the table or the token arrays: a row past max_pages * page_size has
// no place, and a page number outside [0, n_pages) is not followed (appending drops the row, attention treats it as absent).
#pragma once
#include "common.cuh"

namespace sab {

constexpr int kPgMaxSeqs = 4096;                     // sequences of a call
constexpr int kPgMaxRows = 1 << 30;                  // rows of a sequence (max_pages * page_size)
constexpr int kPgMaxD = 256;

// n / d for 0 <= n < 2^31 (round-up multiplier of 33 bits, its top one implied).
struct FastDiv {
    uint32_t mul, shift;
    __host__ __device__ __forceinline__ int div(int n) const
    {
#ifdef __CUDA_ARCH__
        const uint32_t high = __umulhi((uint32_t)n, mul);
#else
        const uint32_t high = (uint32_t)(((uint64_t)(uint32_t)n * mul) >> 32);
#endif
        return (int)((high + (uint32_t)n) >> shift);
    }
};
inline FastDiv fast_div(uint32_t d)
{
    FastDiv f;
    f.shift = 0;
    while ((1ull << f.shift) < d) ++f.shift;
    f.mul = (uint32_t)(((1ull << 32) * ((1ull << f.shift) - d)) / d + 1);
    return f;
}

struct Paged {
    void *k, *v;                                     // pools, through the strides below (elements)
    void* bounds;                                    // [n_pages][Hkv][2][D]: smallest and largest value of each channel of the page's keys
    const int* table;                                // [n_seqs][table_stride]
    const int* lens;                                 // [n_seqs]
    long long table_stride, k_page, k_row, k_head, v_page, v_row, v_head;
    int n_seqs, n_pages, page_size, max_pages, max_rows;
    FastDiv by_page;
    __device__ __forceinline__ int rows_of(int s) const { return max(0, min(lens[s], max_rows)); }
    __device__ __forceinline__ bool holds(int page) const { return (unsigned)page < (unsigned)n_pages; }
};

// 16 bytes of a row as fp32.
template <typename T> struct PgVec;
template <> struct PgVec<float> {
    static constexpr int kElems = 4;
    __device__ static void unpack(const uint4& u, float (&x)[4])
    {
        x[0] = __uint_as_float(u.x); x[1] = __uint_as_float(u.y); x[2] = __uint_as_float(u.z); x[3] = __uint_as_float(u.w);
    }
    __device__ static float round(float x) { return x; }
};
template <> struct PgVec<__nv_bfloat16> {
    static constexpr int kElems = 8;
    __device__ static void unpack(const uint4& u, float (&x)[8])
    {
        const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[2 * i] = __uint_as_float(w[i] << 16);
            x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
        }
    }
    __device__ static __nv_bfloat16 round(float x) { return __float2bfloat16_rn(x); }
};

// The smaller (larger) of two values; no number where one of them is none.
__device__ __forceinline__ float min_nan(float a, float b)
{
    float r;
    asm("min.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ float max_nan(float a, float b)
{
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}

// ---- appending ------------------------------------------------------------------------------------------
// New token t of sequence s becomes row r = lens[s] - (cu[s + 1] - t) (lens counts the new rows too).  Key and query channels
// come in pairs (d, d + rd / 2), or (2 i, 2 i + 1) interleaved, and a pair is turned by the angle position * inv_freq[i]:
//   x' = x cos - y sin,  y' = y cos + x sin,
// in fp32, rounded once to the cache's type.  The angle needs more than 32 bits (at position 10^6 an fp32 angle is off by 0.03): as turns,
// position * inv_freq / 2 pi, it is formed modulo one in 64-bit fixed point from the turn per position, a product in double that is off by
// at most 2^-52.3 of itself.  For inv_freq <= 1 (0.16 turns) that is less than the 2^-32 of a turn that the angle is cut to up to position 2^22,
// and 2^-24 at the last one, 2^31 - 1; rounding it to the fp32 argument of the sine adds up to 2^-26.
//
// A CTA has one run of rows of one sequence, at most kApRun of them and aligned, and its KV heads with their query heads.  A warp takes a
// token at a time (where a run has fewer tokens than the CTA warps, several share one): it makes the token's cosines and sines once
// for all heads, and its lanes take neighbouring heads, two pieces of a head each that hold each other's partners, four such loads at
// a time, so that what a warp reads and writes is whole stretches of memory.  The loads of a turn have no branch between them: with one
// (a load that is skipped where a row is missing, in place of an address that is clamped) they went out one after the other, and
// prompts took 113 us where they take 68.  Nothing is shared between warps.
//
// Bounds of a page have one writer, a CTA that has all its new rows: the one that writes them, where a page has no more than
// kApBoundsRun rows or a sequence has one new token; a second launch elsewhere, which reads the keys again (in L2).  Pages of 64 rows
// in the first launch leave 214 CTAs for the 13419 tokens of five prompts: 69 us, two launches 67; 16384 rows into pages of 32 rows, 512
// CTAs: 30 us, two launches 33.  (Both points are of calls that fill the device; the rule goes by the page's rows alone.)
//
// Long calls are bound by memory, every row being read and written once: 13419 tokens of five prompts, 32 + 8 + 8 heads of 128, 332 MB in
// 69 us = 4.8 TB/s (74 % of a copy's rate; without bounds 5.6 TB/s).  With bounds in the same launch a thread has 127 registers, two CTAs an SM,
// rotation or not: 16384 retained rows, 138 MB in 30.6 us = 4.5 TB/s, are 512 CTAs on 296 places, 1.7 turns of them, each with its look-ups ahead of its
// rows.  Without bounds it has the 80 that three CTAs an SM leave, and 36 bytes are spilled.  One token is a chain of latencies, 4 us.
constexpr int kApThreads = 256;
constexpr int kApRun = 16;
constexpr int kApBoundsRun = 32;                            // rows of a page whose bounds the same CTA makes

struct AppendArgs {
    Paged pg;
    const void *q, *k, *v;                           // [n_tokens][heads][D], tokens q_tok, k_tok, v_tok elements apart
    void* q_out;                                     // [n_tokens][H][D]
    long long q_tok, k_tok, v_tok;
    const int* cu;                                   // [n_seqs + 1], or NULL: one token per sequence
    const int* pos;                                  // [n_tokens], or NULL: the row
    const float* inv_freq;                           // [half]
    int half, interleaved, n_tokens;
    int H, Hkv, G, D, heads;                         // heads: KV heads of a CTA
    int run_rows, slots, lane_bits;                  // slots: pairs of pieces of a head, for 2^lane_bits lanes
    FastDiv by_run;
};

// Runs that a call can have at most: a sequence's rows start anywhere in a run.
inline long long append_runs(long long n_tokens, int n_seqs, int run_rows, bool one_each)
{
    if (one_each) return n_seqs;
    const long long seqs = n_seqs < n_tokens ? n_seqs : n_tokens, by_rows = n_tokens / run_rows + 2 * seqs;
    return by_rows < n_tokens ? by_rows : n_tokens;
}

// Pieces of a row: 16 bytes, or fewer where the halves of the rotation are not whole pieces of 16.
template <int BYTES> struct Piece;
template <> struct Piece<16> { using type = uint4; };
template <> struct Piece<8> { using type = uint2; };
template <> struct Piece<4> { using type = uint32_t; };
template <> struct Piece<2> { using type = uint16_t; };

// How the pairs of a rotation lie in a slot: nothing is turned, channel e of a piece with channel e of the other, neighbours of a piece.
enum { kTurnNone = 0, kTurnAcross = 1, kTurnInside = 2 };

template <typename T, int PB> struct ApSlot {
    static constexpr int E = PB / (int)sizeof(T);
    using V = typename Piece<PB>::type;
    int d0, d1, how;                                 // first channels of the pieces; d1 < 0: there is no second
    float c[E], s[E];                                // cosines and sines of the pairs

    __device__ __forceinline__ void init(int slot, const AppendArgs& a)
    {
        // (neighbouring slots have neighbouring pieces: whole sectors go out at a time)
        const int pairs = a.interleaved ? 0 : a.half / E;          // slots that hold a pair of partners
        if (slot < pairs) {
            d0 = slot * E;
            d1 = d0 + a.half;
            how = kTurnAcross;
        } else {
            const int rest = a.slots - pairs;
            d0 = 2 * pairs * E + (slot - pairs) * E;
            d1 = d0 + rest * E < a.D ? d0 + rest * E : -1;
            how = d0 < 2 * a.half ? kTurnInside : kTurnNone;
        }
    }
    // cosines and sines of the slot from those of the token
    __device__ __forceinline__ void angles(const float* cs, const float* sn, const AppendArgs& a)
    {
        if (how == kTurnNone) return;
#pragma unroll
        for (int e = 0; e < E; ++e) {
            // inside: pairs 0 .. E / 2 - 1 are the first piece's, the others the second's
            const int f = how == kTurnAcross ? d0 + e : min(e < E / 2 ? (d0 >> 1) + e : d1 < 0 ? 0 : (d1 >> 1) + e - E / 2, a.half - 1);
            c[e] = cs[f];
            s[e] = sn[f];
        }
    }
    __device__ __forceinline__ void turn(V& u, V& w, const AppendArgs& a) const
    {
        float x[E], y[E];
        if (how == kTurnAcross) {
            unpack(u, x);
            unpack(w, y);
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const float t = x[e] * c[e] - y[e] * s[e];
                y[e] = y[e] * c[e] + x[e] * s[e];
                x[e] = t;
            }
            u = pack(x);
            w = pack(y);
        } else if (how == kTurnInside) {
            if constexpr (E >= 2) {
                unpack(u, x);
                unpack(w, y);
#pragma unroll
                for (int e = 0; e < E; e += 2) {
                    inside(x[e], x[e + 1], c[e / 2], s[e / 2], d0 + e < 2 * a.half);
                    inside(y[e], y[e + 1], c[E / 2 + e / 2], s[E / 2 + e / 2], d1 + e < 2 * a.half);
                }
                u = pack(x);
                w = pack(y);
            }
        }
    }
    __device__ static __forceinline__ void inside(float& x, float& y, float c, float s, bool in)
    {
        const float t = x * c - y * s, z = y * c + x * s;
        x = in ? t : x;
        y = in ? z : y;
    }
    __device__ static __forceinline__ void unpack(const V& v, float (&x)[E])
    {
        const T* p = reinterpret_cast<const T*>(&v);
#pragma unroll
        for (int e = 0; e < E; ++e) x[e] = ld_as_float(p + e);
    }
    __device__ static __forceinline__ V pack(const float (&x)[E])
    {
        V v;
        T* p = reinterpret_cast<T*>(&v);
#pragma unroll
        for (int e = 0; e < E; ++e) p[e] = PgVec<T>::round(x[e]);
        return v;
    }
};

// Smallest and largest values of a piece, packed as the piece is; no number where one is none.
template <typename T> struct ApBounds;
template <> struct ApBounds<float> {
    __device__ static uint32_t least(uint32_t a, uint32_t b) { return __float_as_uint(min_nan(__uint_as_float(a), __uint_as_float(b))); }
    __device__ static uint32_t most(uint32_t a, uint32_t b) { return __float_as_uint(max_nan(__uint_as_float(a), __uint_as_float(b))); }
    static constexpr uint32_t kInf = 0x7f800000u, kNegInf = 0xff800000u;
};
template <> struct ApBounds<__nv_bfloat16> {
    __device__ static uint32_t least(uint32_t a, uint32_t b)
    {
        uint32_t r;
        asm("min.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
        return r;
    }
    __device__ static uint32_t most(uint32_t a, uint32_t b)
    {
        uint32_t r;
        asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
        return r;
    }
    static constexpr uint32_t kInf = 0x7f807f80u, kNegInf = 0xff80ff80u;
};
template <typename T>
__device__ __forceinline__ void widen(uint4 (&b)[2], const uint4& lo, const uint4& hi)
{
    using A = ApBounds<T>;
    b[0] = make_uint4(A::least(b[0].x, lo.x), A::least(b[0].y, lo.y), A::least(b[0].z, lo.z), A::least(b[0].w, lo.w));
    b[1] = make_uint4(A::most(b[1].x, hi.x), A::most(b[1].y, hi.y), A::most(b[1].z, hi.z), A::most(b[1].w, hi.w));
}

// The run of a CTA: rows [ra, rb) of sequence s (none: rb <= ra), which begins at row `first`; its last row is that of token t_end - 1 - (len - rb).
struct ApRun {
    int s, len, t_end, first, ra, rb;
};
__device__ __forceinline__ ApRun append_run(const AppendArgs& a)
{
    __shared__ int run_s, run_j;
    __shared__ int warp_runs[kApThreads / 32];
    const Paged& pg = a.pg;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    // rows [r0, r1) of sequence s are new; its tokens end before t_end
    int r0, r1, t_end;
    auto span = [&](int s) {
        const int len = pg.lens[s];
        int n = 1;
        t_end = s + 1;
        if (a.cu) {
            t_end = max(0, min(a.cu[s + 1], a.n_tokens));
            n = t_end - max(0, min(a.cu[s], a.n_tokens));
        }
        r0 = max(len - max(n, 0), 0);
        r1 = min(len, pg.max_rows);
        return len;
    };
    ApRun run = {(int)blockIdx.x, 0, 0, 0, 0, 0};
    int j = -1;
    if (a.cu) {
        // runs counted over the sequences, a thread taking neighbouring ones
        const int per = (pg.n_seqs + kApThreads - 1) / kApThreads;
        const int s0 = min(tid * per, pg.n_seqs), s1 = min(s0 + per, pg.n_seqs);
        auto runs_of = [&](int i) {
            span(i);
            return r1 > r0 ? a.by_run.div(r1 - 1) - a.by_run.div(r0) + 1 : 0;
        };
        int mine = 0;
        for (int i = s0; i < s1; ++i) mine += runs_of(i);
        int upto = mine;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int x = __shfl_up_sync(0xffffffffu, upto, o);
            if (lane >= o) upto += x;
        }
        if (tid == 0) run_s = -1;
        if (lane == 31) warp_runs[warp] = upto;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < kApThreads / 32; ++w) upto += w < warp ? warp_runs[w] : 0;
        int left = (int)blockIdx.x - (upto - mine);
        if (left >= 0 && left < mine)
            for (int i = s0; i < s1; ++i) {
                const int n = runs_of(i);
                if (left < n) {
                    run_s = i;
                    run_j = a.by_run.div(r0) + left;
                    break;
                }
                left -= n;
            }
        __syncthreads();
        run.s = run_s;
        j = run_j;
        if (run.s < 0) return run;
    }
    run.len = span(run.s);
    if (r1 <= r0) return run;
    run.t_end = t_end;
    run.first = (j < 0 ? a.by_run.div(r0) : j) * a.run_rows;
    run.ra = max(r0, run.first);
    run.rb = (int)min((long long)r1, (long long)run.first + a.run_rows);
    return run;
}

// The bounds of the page whose rows a run is, columns [c0, c0 + n_cols) of 16-byte pieces of its keys: of the rows just written and,
// unless they begin the page, of those before them.
template <typename T>
__device__ __forceinline__ void append_bounds(const AppendArgs& a, const ApRun& run, int c0, int n_cols)
{
    constexpr int E = PgVec<T>::kElems;
    __shared__ uint4 red[2 * kApThreads];
    const Paged& pg = a.pg;
    const int tid = threadIdx.x, page = pg.table[(long long)run.s * pg.table_stride + pg.by_page.div(run.ra)];
    if (!pg.holds(page)) return;
    const int PR = a.D / E, at = run.ra - run.first, n = run.rb - run.ra;
    for (int c = c0; c < c0 + n_cols; c += kApThreads) {
        // a column to a thread, its rows shared where there are fewer columns than threads
        const int cols = min(kApThreads, c0 + n_cols - c), lanes = kApThreads / cols, tl = tid / cols, col = tid - tl * cols;
        const int h = (c + col) / PR, d = (c + col) % PR * E;
        const T* src = static_cast<const T*>(pg.k) + (long long)page * pg.k_page + (long long)at * pg.k_row + (long long)h * pg.k_head + d;
        T* dst = static_cast<T*>(pg.bounds) + (((size_t)page * a.Hkv + h) * 2) * a.D + d;
        uint4 *lo = reinterpret_cast<uint4*>(dst), *hi = reinterpret_cast<uint4*>(dst + a.D);
        uint4 was_lo = {}, was_hi = {};              // what earlier rows left, asked for before the new rows
        if (at > 0) { was_lo = *lo; was_hi = *hi; }
        constexpr uint32_t inf = ApBounds<T>::kInf, neg = ApBounds<T>::kNegInf;
        uint4 b[2] = {make_uint4(inf, inf, inf, inf), make_uint4(neg, neg, neg, neg)};
        if (tl < lanes)
            for (int i = tl; i < n; i += 8 * lanes) {
                uint4 x[8];
#pragma unroll
                for (int t = 0; t < 8; ++t) x[t] = *reinterpret_cast<const uint4*>(src + (long long)min(i + t * lanes, n - 1) * pg.k_row);
#pragma unroll
                for (int t = 0; t < 8; ++t) widen<T>(b, x[t], x[t]);
            }
        red[tid] = b[0];
        red[kApThreads + tid] = b[1];
        __syncthreads();
        if (tl == 0) {
            for (int l = 1; l < lanes; ++l) widen<T>(b, red[l * cols + col], red[kApThreads + l * cols + col]);
            if (at > 0) widen<T>(b, was_lo, was_hi);
            *lo = b[0];
            *hi = b[1];
        }
        __syncthreads();
    }
}

template <typename T, int PB, bool BOUNDS>
__global__ void __launch_bounds__(kApThreads, BOUNDS ? 2 : 3)
paged_append_kernel(const __grid_constant__ AppendArgs a)
{
    using Slot = ApSlot<T, PB>;
    using V = typename Slot::V;
    const Paged& pg = a.pg;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    __shared__ float trig[kApThreads / 32][2][kPgMaxD / 2];
    pdl_wait();
    pdl_launch();

    const ApRun run = append_run(a);
    if (run.rb <= run.ra) return;
    const int ra = run.ra, rb = run.rb;
    const int* table = pg.table + (long long)run.s * pg.table_stride;

    const int h0 = blockIdx.y * a.heads, nk = min(a.heads, a.Hkv - h0), n_rows = (a.q ? 2 + a.G : 2) * nk;
    // warps: `rows` of them on rows of their own, the others share these rows' heads
    constexpr int kWarps = kApThreads / 32;
    int rows = 1;
    while (rows < kWarps && rows < rb - ra) rows *= 2;
    const int beside = 32 >> a.lane_bits;                          // heads that a warp has side by side
    const int from = (warp / rows) * beside, step = (kWarps / rows) * beside, mine = lane >> a.lane_bits;
    float *cs = trig[warp][0], *sn = trig[warp][1];
    for (int r = ra + (warp & (rows - 1)); r < rb; r += rows) {
        const int pj = pg.by_page.div(r), at = r - pj * pg.page_size, t = run.t_end - (run.len - r);
        const int page = table[pj], p = a.pos ? a.pos[t] : r;
        if (!pg.holds(page)) continue;
        const T* ks = static_cast<const T*>(a.k) + (long long)t * a.k_tok + (long long)h0 * a.D;
        const T* vs = static_cast<const T*>(a.v) + (long long)t * a.v_tok + (long long)h0 * a.D;
        const T* qs = static_cast<const T*>(a.q) + (long long)t * a.q_tok + (long long)h0 * a.G * a.D;
        T* kd = static_cast<T*>(pg.k) + (long long)page * pg.k_page + (long long)at * pg.k_row + (long long)h0 * pg.k_head;
        T* vd = static_cast<T*>(pg.v) + (long long)page * pg.v_page + (long long)at * pg.v_row + (long long)h0 * pg.v_head;
        T* qd = static_cast<T*>(a.q_out) + ((long long)t * a.H + (long long)h0 * a.G) * a.D;
        bool made = a.half == 0;                                   // the token's cosines and sines
        for (int slot = lane & ((1 << a.lane_bits) - 1); slot < (a.slots + (1 << a.lane_bits) - 1 >> a.lane_bits) << a.lane_bits; slot += 1 << a.lane_bits) {
            Slot sl;
            sl.init(min(slot, a.slots - 1), a);
            const bool two = sl.d1 >= 0, in = slot < a.slots;
            const int d1 = two ? sl.d1 : sl.d0;
            bool known = false;
            for (int u = from; u < n_rows; u += 4 * step) {
                V x[4], y[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int h = min(u + i * step + mine, n_rows - 1);         // (no branch between the loads)
                    const T* src = h < nk ? ks + h * a.D : h < 2 * nk ? vs + (h - nk) * a.D : qs + (h - 2 * nk) * a.D;
                    x[i] = *reinterpret_cast<const V*>(src + sl.d0);
                    y[i] = *reinterpret_cast<const V*>(src + d1);
                }
                if (!made) {                                       // (while the first loads are on their way)
                    made = true;
                    __syncwarp();
                    for (int f = lane; f < a.half; f += 32) {
                        const double per = (double)a.inv_freq[f] * 0.15915494309189533577;       // 1 / (2 pi): turns from position to position
                        const long long turn = (long long)((per - rint(per)) * 18446744073709551616.0);
                        const int left = (int)(((unsigned long long)turn * (unsigned long long)(long long)p) >> 32);   // turns modulo one, in 2^-32
                        sincospif((float)left * 0x1p-31f, &sn[f], &cs[f]);
                    }
                    __syncwarp();
                }
                if (!known) sl.angles(cs, sn, a);
                known = true;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int h = u + i * step + mine;
                    if (!in || h >= n_rows) continue;
                    T* dst = h < nk ? kd + h * pg.k_head : h < 2 * nk ? vd + (h - nk) * pg.v_head : qd + (h - 2 * nk) * a.D;
                    if (h < nk || h >= 2 * nk) sl.turn(x[i], y[i], a);
                    *reinterpret_cast<V*>(dst + sl.d0) = x[i];
                    if (two) *reinterpret_cast<V*>(dst + d1) = y[i];
                }
            }
        }
    }
    if constexpr (BOUNDS) {
        __syncthreads();                             // the rows are written
        append_bounds<T>(a, run, h0 * (a.D / PgVec<T>::kElems), nk * (a.D / PgVec<T>::kElems));
    }
}

// The bounds of pages of more rows than a CTA of the kernel above writes.
template <typename T>
__global__ void __launch_bounds__(kApThreads)
paged_bounds_kernel(const __grid_constant__ AppendArgs a)
{
    pdl_wait();
    pdl_launch();
    const ApRun run = append_run(a);
    if (run.rb <= run.ra) return;
    const int all = a.Hkv * (a.D / PgVec<T>::kElems), per = (all + gridDim.y - 1) / gridDim.y, c0 = blockIdx.y * per;
    if (c0 < all) append_bounds<T>(a, run, c0, min(per, all - c0));
}

// ---- which pages a token's queries look at --------------------------------------------------------------
// A page's score for a KV head: the largest logit that a key within the page's bounds could have with each of the head's queries,
// added over the queries (the mean over the heads, as in Eq. 3, up to a factor),
//   sum_h sum_d max(q_hd lo_d, q_hd hi_d) = sum_d (sum_h max(q_hd, 0)) hi_d + (sum_h min(q_hd, 0)) lo_d,
// so the queries are added first and a page costs 2 D multiply-adds, whatever the number of heads.  Sums are in double, rounded
// once to fp32: which page comes in at the border then does not hang on the order of a sum.  Ties go to the lower page.
//
// A cluster of CTAs has one (sequence, KV head).  Its warps score several pages at a time (a page's bounds are one row of 4 D bytes in
// bf16, read by the whole warp) and leave the order-preserving integer images of the scores in shared memory.  The n_sel-th largest is
// found by counting into 1024 bins over the range of the keys, then over the range of the bin that it is in, until all of a bin is in
// or its keys are equal.  Two kernels do this: page_select_kernel below, where CTA 0 of the cluster chooses, and
// paged_cluster_kernel (paged_attn.cuh), where every CTA does, for itself.
// The scores are bound by the conversions to double, 16 lanes a cycle on an SM: a page of 128 channels takes an SM 22 cycles, 2048 pages and
// eight KV heads 7 us, with choosing (3 us) and the launch 12.7; reading their bounds, 16.8 MB, is 2.6.
__host__ __device__ constexpr int ps_threads(int NP) { return NP > 2 ? 256 : 512; }      // (registers for eight pages)
constexpr int kPsBinBits = 10, kPsBins = 1 << kPsBinBits;
constexpr int kPsMaxPages = 49152;                                 // keys of a sequence in shared memory (192 KB)
constexpr int kPsMaxCluster = 8;
constexpr uint32_t kKeyForced = 0xffffffffu, kKeyNan = 0xfffffffeu;

struct PageSelectArgs {
    Paged pg;
    const void* q;                                   // [n_seqs][H][D]
    int* sel;                                        // [n_seqs][Hkv][n_sel]: chosen pages of the sequence, ascending, then -1
    int H, Hkv, G, D, n_sel, n_first, n_last;
};

// fp32 as an unsigned integer of the same order, no number above all
__device__ __forceinline__ uint32_t page_key(float x)
{
    if (x != x) return kKeyNan;
    const uint32_t u = __float_as_uint(x == 0.f ? 0.f : x);
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ void st_cluster_u32(const void* p, int rank, uint32_t v)
{
    asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(cluster_map(p, rank)), "r"(v) : "memory");
}
// The halves of cluster_sync: what a thread does between them need not wait for the others.
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_await() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }

// Sums of a warp's values, eight at a time: lane 4 p (p = 0 .. 7) and its three neighbours have the sum of v[p].
__device__ __forceinline__ double sum8(double* v, int lane)
{
#pragma unroll
    for (int o = 16, n = 4; o >= 4; o >>= 1, n >>= 1) {
        const bool up = lane & o;
#pragma unroll
        for (int i = 0; i < n; ++i) {
            const double give = up ? v[i] : v[i + n], keep = up ? v[i + n] : v[i];
            v[i] = keep + __shfl_xor_sync(0xffffffffu, give, o);
        }
    }
    double x = v[0] + __shfl_xor_sync(0xffffffffu, v[0], 2);
    return x + __shfl_xor_sync(0xffffffffu, x, 1);
}

// Scores pages at, at + 1, .. at + NB - 1, then from at + step on, of the P pages of sequence s for KV head hk, by a warp: ready() before the
// first result, then store(page, key), called by the four lanes that hold it.  NP: 16-byte pieces of a page's bounds that a lane has.
template <typename T, int NP, int NB, typename Ready, typename Store>
__device__ __forceinline__ void score_pages(const PageSelectArgs& a, int s, int hk, int P, int at, int step, Ready&& ready, Store&& store)
{
    constexpr int E = PgVec<T>::kElems;
    const Paged& pg = a.pg;
    const int lane = threadIdx.x & 31, pieces = 2 * a.D / E;
    const int* table = pg.table + (long long)s * pg.table_stride;
    auto ask = [&](int b) { return table[min(b + (lane & (NB - 1)), P - 1)]; };
    int next = ask(at);
    // weights of this lane's pieces: the first D elements of a page's bounds are its smallest values
    double w[NP][E];
    const T* q = static_cast<const T*>(a.q) + ((size_t)s * a.H + (size_t)hk * a.G) * a.D;
#pragma unroll
    for (int n = 0; n < NP; ++n) {
#pragma unroll
        for (int e = 0; e < E; ++e) w[n][e] = 0.0;
        const int pc = lane + 32 * n;
        if (pc >= pieces) continue;
        const bool upper = pc * E >= a.D;
        const int d = pc * E - (upper ? a.D : 0);
        for (int h0 = 0; h0 < a.G; h0 += 4) {
            uint4 u[4];
#pragma unroll
            for (int h = 0; h < 4; ++h) u[h] = *reinterpret_cast<const uint4*>(q + (size_t)min(h0 + h, a.G - 1) * a.D + d);
#pragma unroll
            for (int h = 0; h < 4; ++h) {
                float x[E];
                PgVec<T>::unpack(u[h], x);
                if (h0 + h < a.G)
#pragma unroll
                    for (int e = 0; e < E; ++e) w[n][e] += upper ? (x[e] < 0.f ? 0.0 : (double)x[e]) : (x[e] > 0.f ? 0.0 : (double)x[e]);
            }
        }
    }
    const T* bounds = static_cast<const T*>(pg.bounds);
    uint4 x[NB][NP];
    auto load = [&](int page) {
#pragma unroll
        for (int i = 0; i < NB; ++i) {
            // (no branch between the loads: a page that is not there reads page 0, and its score is not used)
            const int id = __shfl_sync(0xffffffffu, page, i);
            const uint4* row = reinterpret_cast<const uint4*>(bounds + ((size_t)(pg.holds(id) ? id : 0) * a.Hkv + hk) * 2 * a.D);
#pragma unroll
            for (int n = 0; n < NP; ++n) x[i][n] = row[min(lane + 32 * n, pieces - 1)];
        }
    };
    bool first = true;
    int page = next;
    next = ask(at + step);
    load(page);
    for (int b = at; b < P; b += step) {
        const uint32_t there = __ballot_sync(0xffffffffu, pg.holds(page));
        double v[NB];
#pragma unroll
        for (int i = 0; i < NB; ++i) {
            v[i] = 0.0;
#pragma unroll
            for (int n = 0; n < NP; ++n) {
                float f[E];
                PgVec<T>::unpack(x[i][n], f);
#pragma unroll
                for (int e = 0; e < E; ++e) v[i] = fma((double)f[e], w[n][e], v[i]);
            }
        }
        page = next;
        next = ask(b + 2 * step);
        load(page);                                                // (on their way while the sums go round)
#pragma unroll
        for (int i0 = 0; i0 < NB; i0 += 8) {
            const double sum = sum8(v + i0, lane);
            if (first) ready();
            first = false;
            const int i = i0 + (lane >> 2), j = b + i;
            if (j < P)
                store(j, j < a.n_first || j >= P - a.n_last ? kKeyForced : (there >> i) & 1 ? page_key((float)sum) : page_key(-INFINITY));
        }
    }
    if (first) ready();
}

// Chooses n_sel of the P keys (n_sel < P, n_forced of them forced), by all THREADS of a CTA: put(place, page), pages ascending.
template <int THREADS> struct ChooseMem {
    int hist[kPsBins];
    int tot[2][THREADS / 32];
    uint32_t ends[2][THREADS / 32];
    int found[3];
};
template <int THREADS, typename Put>
__device__ __forceinline__ void choose_pages(const uint32_t* keys, int P, int n_sel, int n_forced, ChooseMem<THREADS>& mem, Put&& put)
{
    constexpr int kWarps = THREADS / 32;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    // the range of the keys but for the pages that are in anyway
    uint32_t kmin = 0xffffffffu, kmax = 0;
    // (eight keys at a time: their loads do not wait for one another)
    auto each = [&](int from, int to, int step, auto&& f) {
        for (int i = from; i < to; i += 8 * step) {
            uint32_t k[8];
#pragma unroll
            for (int t = 0; t < 8; ++t) k[t] = keys[min(i + t * step, P - 1)];
#pragma unroll
            for (int t = 0; t < 8; ++t)
                if (i + t * step < to) f(k[t], i + t * step);
        }
    };
    each(tid, P, THREADS, [&](uint32_t k, int) {
        kmin = min(kmin, k);
        if (k != kKeyForced) kmax = max(kmax, k);
    });
    kmin = __reduce_min_sync(0xffffffffu, kmin);
    kmax = __reduce_max_sync(0xffffffffu, kmax);
    if (lane == 0) { mem.ends[0][warp] = kmin; mem.ends[1][warp] = kmax; }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kWarps; ++i) { kmin = min(kmin, mem.ends[0][i]); kmax = max(kmax, mem.ends[1][i]); }
    // keys above the range: `above` < n_sel; keys above or in it: at least n_sel
    int above = n_forced, ties = 0;
    if (above == n_sel) kmin = kmax = kKeyNan;
    else while (true) {
        const uint32_t width = kmax - kmin;
        const int shift = max(0, 32 - kPsBinBits - __clz(width | 1u));     // width >> shift < kPsBins
        for (int i = tid; i < kPsBins; i += THREADS) mem.hist[i] = 0;
        __syncthreads();
        each(tid, P, THREADS, [&](uint32_t k, int) {
            if (k >= kmin && k <= kmax) atomicAdd(&mem.hist[(k - kmin) >> shift], 1);
        });
        __syncthreads();
        // some bins a thread, from the top
        constexpr int kPer = kPsBins / THREADS;
        int c[kPer], sum = 0;
#pragma unroll
        for (int i = 0; i < kPer; ++i) sum += c[i] = mem.hist[kPsBins - 1 - (tid * kPer + i)];
        int upto = sum;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int x = __shfl_up_sync(0xffffffffu, upto, o);
            if (lane >= o) upto += x;
        }
        if (lane == 31) mem.tot[0][warp] = upto;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < kWarps; ++i) upto += i < warp ? mem.tot[0][i] : 0;
        int before = above + upto - sum;                           // keys above this thread's bins
        if (before < n_sel && before + sum >= n_sel)
#pragma unroll
            for (int i = 0; i < kPer; ++i) {
                if (before < n_sel && before + c[i] >= n_sel) {
                    mem.found[0] = kPsBins - 1 - (tid * kPer + i);
                    mem.found[1] = before;
                    mem.found[2] = c[i];
                }
                before += c[i];
            }
        __syncthreads();
        const uint32_t low = kmin + ((uint32_t)mem.found[0] << shift);
        above = mem.found[1];
        const int in_bin = mem.found[2];
        ties = n_sel - above;
        kmax = low + min(kmax - low, (1u << shift) - 1u);
        kmin = low;
        if (ties == in_bin) { ties = 0x7fffffff; break; }          // all of the bin is in
        if (shift == 0) break;                                     // its keys are equal: the first `ties` of them are in
        // (every thread has read found and tot before the next pass writes them: two barriers lie between)
    }
    // keys above kmax are in, and the first `ties` from kmin to kmax
    const int per = ((P + THREADS - 1) / THREADS) | 1;             // (odd: a warp's threads read from 32 banks)
    const int j0 = min(tid * per, P), j1 = min(j0 + per, P);
    int n_hi = 0, n_eq = 0;
    each(j0, j1, 1, [&](uint32_t k, int) {
        n_hi += k > kmax;
        n_eq += k >= kmin && k <= kmax;
    });
    int s_hi = n_hi, s_eq = n_eq;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int x = __shfl_up_sync(0xffffffffu, s_hi, o), y = __shfl_up_sync(0xffffffffu, s_eq, o);
        if (lane >= o) { s_hi += x; s_eq += y; }
    }
    __syncthreads();
    if (lane == 31) { mem.tot[0][warp] = s_hi; mem.tot[1][warp] = s_eq; }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kWarps; ++i) {
        s_hi += i < warp ? mem.tot[0][i] : 0;
        s_eq += i < warp ? mem.tot[1][i] : 0;
    }
    int eq = s_eq - n_eq, at = s_hi - n_hi + min(eq, ties);
    each(j0, j1, 1, [&](uint32_t k, int i) {
        if (k > kmax || (k >= kmin && k <= kmax && eq++ < ties)) put(at++, i);
    });
}

template <typename T, int NP>
__global__ void __launch_bounds__(ps_threads(NP))
page_select_kernel(const __grid_constant__ PageSelectArgs a, int n_cta)
{
    constexpr int kPsThreads = ps_threads(NP), kPsWarps = kPsThreads / 32;
    const Paged& pg = a.pg;
    const int tid = threadIdx.x, warp = tid >> 5;
    const int rank = blockIdx.x, pair = blockIdx.y, s = pair / a.Hkv, hk = pair - s * a.Hkv;
    extern __shared__ __align__(16) uint32_t ps_keys[];
    __shared__ ChooseMem<kPsThreads> mem;
    pdl_wait();
    pdl_launch();
    const int rows = pg.rows_of(s), P = pg.by_page.div(rows + pg.page_size - 1);
    int* sel = a.sel + (size_t)pair * a.n_sel;
    if (P <= a.n_sel) {                                            // (the whole cluster: all pages are in)
        for (int i = rank * kPsThreads + tid; i < a.n_sel; i += n_cta * kPsThreads) sel[i] = i < P ? i : -1;
        return;
    }
    if (n_cta > 1) cluster_arrive();
    score_pages<T, NP, 8>(a, s, hk, P, (rank * kPsWarps + warp) * 8, n_cta * kPsWarps * 8,
        [&] { if (n_cta > 1) cluster_await(); },                   // CTA 0 has started: its memory may be written
        [&](int j, uint32_t key) {
            if (tid & 3) return;
            if (n_cta > 1) st_cluster_u32(ps_keys + j, 0, key);
            else ps_keys[j] = key;
        });
    if (n_cta > 1) cluster_sync();
    else __syncthreads();
    if (rank == 0) choose_pages<kPsThreads>(ps_keys, P, a.n_sel, a.n_first + a.n_last, mem, [&](int at, int j) { sel[at] = j; });
}

}  // namespace sab
