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
    __device__ static uint4 pack(const float (&x)[4])
    {
        return make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3]));
    }
    __device__ static float rounded(float x) { return x; }
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
    __device__ static uint4 pack(const float (&x)[8])
    {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const __nv_bfloat162 t = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
            w[i] = *reinterpret_cast<const uint32_t*>(&t);
        }
        return make_uint4(w[0], w[1], w[2], w[3]);
    }
    __device__ static float rounded(float x) { return __bfloat162float(__float2bfloat16_rn(x)); }
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
// in fp32, rounded once to the cache's type.  The angle needs more than 32 bits (at position 10^6 an fp32 angle is off by 0.03): its turns,
// position * inv_freq / 2 pi, are formed in double, and what is left of them after the whole turns is small enough for fp32.
//
// A CTA has one run of rows of one sequence (those of one page where bounds are kept, at most run_rows elsewhere; rows of a run are
// aligned, so that a page's bounds have one writer) and some of the KV heads with their query heads.  It makes the cosines and sines of
// kApTok tokens at a time for all its heads; then a thread owns one 16-byte piece of one head and walks the tokens, so that the
// bounds stay in its registers.  Bound by memory: every row is read and written once.
constexpr int kApThreads = 256;
constexpr int kApTok = 16;

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
    int run_rows;
    FastDiv by_run;
};

// Runs that a call can have at most: a sequence's rows start anywhere in a run.
inline long long append_runs(long long n_tokens, int n_seqs, int run_rows, bool one_each)
{
    if (one_each) return n_seqs;
    const long long seqs = n_seqs < n_tokens ? n_seqs : n_tokens, by_rows = n_tokens / run_rows + 2 * seqs;
    return by_rows < n_tokens ? by_rows : n_tokens;
}

template <typename T>
__device__ __forceinline__ uint4 rotate_piece(const uint4& raw, const T* row, int d0, const AppendArgs& a, const float* cs, const float* sn)
{
    constexpr int E = PgVec<T>::kElems;
    const int rd = 2 * a.half;
    if (d0 >= rd) return raw;
    float x[E], y[E];
    PgVec<T>::unpack(raw, x);
    if (a.interleaved) {
#pragma unroll
        for (int e = 0; e < E; e += 2) {
            const int i = (d0 + e) >> 1;
            const bool in = d0 + e < rd;
            const float c = in ? cs[i] : 1.f, s = in ? sn[i] : 0.f;
            y[e] = in ? x[e] * c - x[e + 1] * s : x[e];
            y[e + 1] = in ? x[e + 1] * c + x[e] * s : x[e + 1];
        }
    } else if (a.half % E == 0) {
        // (a piece lies in one half, and so does its partner)
        const bool upper = d0 >= a.half;
        const int i0 = upper ? d0 - a.half : d0;
        float z[E];
        PgVec<T>::unpack(*reinterpret_cast<const uint4*>(row + (upper ? i0 : d0 + a.half)), z);
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const float c = cs[i0 + e], s = sn[i0 + e];
            y[e] = upper ? x[e] * c + z[e] * s : x[e] * c - z[e] * s;
        }
    } else {
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const int d = d0 + e;
            y[e] = x[e];
            if (d < rd) {
                const bool upper = d >= a.half;
                const int i = upper ? d - a.half : d;
                const float z = ld_as_float(row + (upper ? i : d + a.half));
                y[e] = upper ? x[e] * cs[i] + z * sn[i] : x[e] * cs[i] - z * sn[i];
            }
        }
    }
    return PgVec<T>::pack(y);
}

template <typename T, bool BOUNDS>
__global__ void __launch_bounds__(kApThreads)
paged_append_kernel(const __grid_constant__ AppendArgs a)
{
    constexpr int E = PgVec<T>::kElems;
    const Paged& pg = a.pg;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    __shared__ int run_s, run_j;
    __shared__ int warp_runs[kApThreads / 32];
    __shared__ long long k_at[kApTok], v_at[kApTok];               // where a token's row goes (elements), -1: nowhere
    __shared__ __align__(16) float cs[kApTok][kPgMaxD / 2], sn[kApTok][kPgMaxD / 2];
    __shared__ __align__(16) float red[BOUNDS ? 2 * kApThreads * E : 4];
    pdl_wait();
    pdl_launch();

    // rows [r0, r1) of sequence s are new; its tokens end before t_end
    auto span = [&](int s, int& r0, int& r1, int& t_end) {
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
    int s = blockIdx.x, j = -1, r0, r1, t_end;
    if (a.cu) {
        // the sequence and run of this CTA: runs counted over the sequences, a thread taking neighbouring ones
        const int per = (pg.n_seqs + kApThreads - 1) / kApThreads;
        const int s0 = min(tid * per, pg.n_seqs), s1 = min(s0 + per, pg.n_seqs);
        auto runs_of = [&](int i) {
            span(i, r0, r1, t_end);
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
        for (int w = 0; w < warp; ++w) upto += warp_runs[w];
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
        s = run_s;
        j = run_j;
        if (s < 0) return;
    }
    const int len = span(s, r0, r1, t_end);
    if (r1 <= r0) return;
    if (j < 0) j = a.by_run.div(r0);
    const long long first = (long long)j * a.run_rows;
    const int ra = max(r0, (int)first), rb = (int)min((long long)r1, first + a.run_rows);

    const int h0 = blockIdx.y * a.heads, nk = min(a.heads, a.Hkv - h0);
    const int PR = a.D / E, cols = nk * PR;
    const int lanes = kApThreads / cols;                           // threads that share a piece's tokens (the host keeps cols <= kApThreads)
    const int col = tid % cols, tl = tid / cols;
    const int hk = h0 + col / PR, d0 = (col % PR) * E;
    const T* kg = static_cast<const T*>(a.k) + (size_t)hk * a.D;
    const T* vg = static_cast<const T*>(a.v) + (size_t)hk * a.D;
    T* kp = static_cast<T*>(pg.k) + (size_t)hk * pg.k_head + d0;
    T* vp = static_cast<T*>(pg.v) + (size_t)hk * pg.v_head + d0;
    float lo[E], hi[E];
#pragma unroll
    for (int e = 0; e < E; ++e) { lo[e] = INFINITY; hi[e] = -INFINITY; }

    for (int base = ra; base < rb; base += kApTok) {
        const int nb = min(kApTok, rb - base);
        const int t0 = t_end - (len - base);                       // token of row `base`
        if (base > ra) __syncthreads();
        for (int i = tid; i < nb * a.half; i += kApThreads) {
            const int r = i / a.half, f = i - r * a.half;
            const int p = a.pos ? a.pos[t0 + r] : base + r;
            const double turns = (double)p * ((double)a.inv_freq[f] * 0.15915494309189533577);      // 1 / (2 pi)
            const float left = (float)(turns - rint(turns));
            float sv, cv;
            sincospif(2.f * left, &sv, &cv);
            cs[r][f] = cv;
            sn[r][f] = sv;
        }
        if (tid < nb) {
            const int row = base + tid, pj = pg.by_page.div(row), slot = row - pj * pg.page_size;
            const int page = pg.table[(long long)s * pg.table_stride + pj];
            const bool ok = pg.holds(page);
            k_at[tid] = ok ? (long long)page * pg.k_page + (long long)slot * pg.k_row : -1;
            v_at[tid] = ok ? (long long)page * pg.v_page + (long long)slot * pg.v_row : -1;
        }
        __syncthreads();
        if (tl < lanes) {
#pragma unroll 2
            for (int i = tl; i < nb; i += lanes) {
                if (k_at[i] < 0) continue;
                const T* row = kg + (long long)(t0 + i) * a.k_tok;
                uint4 x = *reinterpret_cast<const uint4*>(row + d0);
                const uint4 y = *reinterpret_cast<const uint4*>(vg + (long long)(t0 + i) * a.v_tok + d0);
                x = rotate_piece<T>(x, row, d0, a, cs[i], sn[i]);
                *reinterpret_cast<uint4*>(kp + k_at[i]) = x;
                *reinterpret_cast<uint4*>(vp + v_at[i]) = y;
                if constexpr (BOUNDS) {
                    float f[E];
                    PgVec<T>::unpack(x, f);
#pragma unroll
                    for (int e = 0; e < E; ++e) { lo[e] = min_nan(lo[e], f[e]); hi[e] = max_nan(hi[e], f[e]); }
                }
            }
        }
        if (a.q) {
            const int qcols = cols * a.G, hq = h0 * a.G;
            for (int i = tid; i < nb * qcols; i += kApThreads) {
                const int r = i / qcols, c = i - r * qcols;
                if (k_at[r] < 0) continue;
                const int h = hq + c / PR, d = (c % PR) * E;
                const T* row = static_cast<const T*>(a.q) + (long long)(t0 + r) * a.q_tok + (size_t)h * a.D;
                const uint4 x = *reinterpret_cast<const uint4*>(row + d);
                *reinterpret_cast<uint4*>(static_cast<T*>(a.q_out) + ((size_t)(t0 + r) * a.H + h) * a.D + d) =
                    rotate_piece<T>(x, row, d, a, cs[r], sn[r]);
            }
        }
    }
    if constexpr (BOUNDS) {
        // the threads that share a piece, then what the page's earlier rows left; rows of this run are all in page j
        const int page = pg.table[(long long)s * pg.table_stride + j];
        if (!pg.holds(page)) return;
        if (tl < lanes)
#pragma unroll
            for (int e = 0; e < E; ++e) { red[e * kApThreads + tid] = lo[e]; red[(E + e) * kApThreads + tid] = hi[e]; }
        __syncthreads();
        if (tl == 0) {
            for (int l = 1; l < lanes; ++l)
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    lo[e] = min_nan(lo[e], red[e * kApThreads + l * cols + col]);
                    hi[e] = max_nan(hi[e], red[(E + e) * kApThreads + l * cols + col]);
                }
            T* b = static_cast<T*>(pg.bounds) + (((size_t)page * a.Hkv + hk) * 2) * a.D + d0;
            if (ra > first) {
                float f[E], g[E];
                PgVec<T>::unpack(*reinterpret_cast<const uint4*>(b), f);
                PgVec<T>::unpack(*reinterpret_cast<const uint4*>(b + a.D), g);
#pragma unroll
                for (int e = 0; e < E; ++e) { lo[e] = min_nan(lo[e], f[e]); hi[e] = max_nan(hi[e], g[e]); }
            }
            *reinterpret_cast<uint4*>(b) = PgVec<T>::pack(lo);
            *reinterpret_cast<uint4*>(b + a.D) = PgVec<T>::pack(hi);
        }
    }
}

// ---- which pages a token's queries look at --------------------------------------------------------------
// A page's score for a KV head: the largest logit that a key within the page's bounds could have with each of the head's queries,
// added over the queries (the mean over the heads, as in Eq. 3, up to a factor),
//   sum_h sum_d max(q_hd lo_d, q_hd hi_d) = sum_d (sum_h max(q_hd, 0)) hi_d + (sum_h min(q_hd, 0)) lo_d,
// so the queries are added first and a page costs 2 D multiply-adds, whatever the number of heads.  Sums are in double, rounded
// once to fp32: which page comes in at the border then does not hang on the order of a sum.  Ties go to the lower page.
//
// A cluster of CTAs has one (sequence, KV head).  Its warps score eight pages at a time (a page's bounds are one row of 4 D bytes in
// bf16, read by the whole warp) and leave the order-preserving integer images of the scores in the shared memory of CTA 0, which
// finds the n_sel-th largest by counting into 1024 bins over the range of the keys, then over the range of the bin that it is
// in, until all of a bin is in or its keys are equal.
constexpr int kPsThreads = 256;
constexpr int kPsWarps = kPsThreads / 32;
constexpr int kPsBins = 1024;
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

// Sums of a warp's values, eight at a time: lane 4 p (p = 0 .. 7) and its three neighbours have the sum of v[p].
__device__ __forceinline__ double sum8(double (&v)[8], int lane)
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

// NP: 16-byte pieces of a page's bounds that a lane has
template <typename T, int NP>
__global__ void __launch_bounds__(kPsThreads)
page_select_kernel(const __grid_constant__ PageSelectArgs a, int n_cta)
{
    constexpr int E = PgVec<T>::kElems;
    const Paged& pg = a.pg;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int rank = blockIdx.x, pair = blockIdx.y, s = pair / a.Hkv, hk = pair - s * a.Hkv;
    extern __shared__ __align__(16) uint32_t ps_keys[];
    __shared__ int hist[kPsBins];
    __shared__ int tot[2][kPsWarps];
    __shared__ uint32_t ends[2][kPsWarps];
    __shared__ int found[3];
    pdl_wait();
    pdl_launch();
    const int rows = pg.rows_of(s), P = pg.by_page.div(rows + pg.page_size - 1);
    int* sel = a.sel + (size_t)pair * a.n_sel;
    if (P <= a.n_sel) {                                            // (the whole cluster: all pages are in)
        for (int i = rank * kPsThreads + tid; i < a.n_sel; i += n_cta * kPsThreads) sel[i] = i < P ? i : -1;
        return;
    }
    // weights of this lane's pieces: the first D elements of a page's bounds are its smallest values
    double w[NP][E];
    const int pieces = 2 * a.D / E;
#pragma unroll
    for (int n = 0; n < NP; ++n)
#pragma unroll
        for (int e = 0; e < E; ++e) w[n][e] = 0.0;
    const T* q = static_cast<const T*>(a.q) + ((size_t)s * a.H + (size_t)hk * a.G) * a.D;
#pragma unroll
    for (int n = 0; n < NP; ++n) {
        const int pc = lane + 32 * n;
        if (pc >= pieces) continue;
        const bool upper = pc * E >= a.D;
        const int d = pc * E - (upper ? a.D : 0);
        for (int h = 0; h < a.G; ++h)
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const float x = ld_as_float(q + (size_t)h * a.D + d + e);
                w[n][e] += upper ? (x < 0.f ? 0.0 : (double)x) : (x > 0.f ? 0.0 : (double)x);
            }
    }
    if (n_cta > 1) cluster_sync();                                 // CTA 0 has started: its memory may be written
    const T* bounds = static_cast<const T*>(pg.bounds);
    const int* table = pg.table + (long long)s * pg.table_stride;
    const int step = n_cta * kPsWarps * 8;
    int next = -1;
    {
        const int j = (rank * kPsWarps + warp) * 8 + (lane & 7);
        if (j < P) next = table[j];
    }
    for (int b = (rank * kPsWarps + warp) * 8; b < P; b += step) {
        const int page = next;
        next = b + step + (lane & 7) < P ? table[b + step + (lane & 7)] : -1;
        double v[8];
        uint4 x[8][NP];
        bool there[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int id = __shfl_sync(0xffffffffu, page, i);
            there[i] = b + i < P && pg.holds(id);
#pragma unroll
            for (int n = 0; n < NP; ++n)
                x[i][n] = there[i] && lane + 32 * n < pieces
                              ? __ldg(reinterpret_cast<const uint4*>(bounds + ((size_t)id * a.Hkv + hk) * 2 * a.D) + lane + 32 * n)
                              : make_uint4(0, 0, 0, 0);
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            v[i] = 0.0;
#pragma unroll
            for (int n = 0; n < NP; ++n) {
                float f[E];
                PgVec<T>::unpack(x[i][n], f);
#pragma unroll
                for (int e = 0; e < E; ++e) v[i] = fma((double)f[e], w[n][e], v[i]);
            }
        }
        const double sum = sum8(v, lane);
        const int i = lane >> 2;
        bool ok = false;
#pragma unroll
        for (int t = 0; t < 8; ++t) ok = t == i ? there[t] : ok;
        const int j = b + i;
        if ((lane & 3) == 0 && j < P) {
            const uint32_t key = j < a.n_first || j >= P - a.n_last ? kKeyForced : ok ? page_key((float)sum) : page_key(-INFINITY);
            if (n_cta > 1) st_cluster_u32(ps_keys + j, 0, key);
            else ps_keys[j] = key;
        }
    }
    if (n_cta > 1) cluster_sync();
    else __syncthreads();
    if (rank != 0) return;

    // the range of the keys
    uint32_t kmin = 0xffffffffu, kmax = 0;
    for (int i = tid; i < P; i += kPsThreads) {
        kmin = min(kmin, ps_keys[i]);
        kmax = max(kmax, ps_keys[i]);
    }
    kmin = __reduce_min_sync(0xffffffffu, kmin);
    kmax = __reduce_max_sync(0xffffffffu, kmax);
    if (lane == 0) { ends[0][warp] = kmin; ends[1][warp] = kmax; }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kPsWarps; ++i) { kmin = min(kmin, ends[0][i]); kmax = max(kmax, ends[1][i]); }
    // keys above the range: `above` < n_sel; keys above or in it: at least n_sel
    int above = 0, ties = 0;
    while (true) {
        const uint32_t width = kmax - kmin;
        const int shift = max(0, 22 - __clz(width | 1u));          // width >> shift < kPsBins
        for (int i = tid; i < kPsBins; i += kPsThreads) hist[i] = 0;
        __syncthreads();
        for (int i = tid; i < P; i += kPsThreads) {
            const uint32_t k = ps_keys[i];
            if (k >= kmin && k <= kmax) atomicAdd(&hist[(k - kmin) >> shift], 1);
        }
        __syncthreads();
        // four bins a thread, from the top
        constexpr int kPer = kPsBins / kPsThreads;
        int c[kPer], sum = 0;
#pragma unroll
        for (int i = 0; i < kPer; ++i) sum += c[i] = hist[kPsBins - 1 - (tid * kPer + i)];
        int upto = sum;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int x = __shfl_up_sync(0xffffffffu, upto, o);
            if (lane >= o) upto += x;
        }
        if (lane == 31) tot[0][warp] = upto;
        __syncthreads();
        for (int i = 0; i < warp; ++i) upto += tot[0][i];
        int before = above + upto - sum;                           // keys above this thread's bins
        if (before < a.n_sel && before + sum >= a.n_sel)
#pragma unroll
            for (int i = 0; i < kPer; ++i) {
                if (before < a.n_sel && before + c[i] >= a.n_sel) {
                    found[0] = kPsBins - 1 - (tid * kPer + i);
                    found[1] = before;
                    found[2] = c[i];
                }
                before += c[i];
            }
        __syncthreads();
        const uint32_t low = kmin + ((uint32_t)found[0] << shift);
        above = found[1];
        const int in_bin = found[2];
        ties = a.n_sel - above;
        kmax = low + min(kmax - low, (1u << shift) - 1u);
        kmin = low;
        if (ties == in_bin) { ties = 0x7fffffff; break; }          // all of the bin is in
        if (shift == 0) break;                                     // its keys are equal: the first `ties` of them are in
        // (every thread has read found and tot before the next pass writes them: two barriers lie between)
    }
    // keys above kmax are in, and the first `ties` from kmin to kmax
    const int per = (P + kPsThreads - 1) / kPsThreads;
    const int j0 = min(tid * per, P), j1 = min(j0 + per, P);
    int n_hi = 0, n_eq = 0;
    for (int i = j0; i < j1; ++i) {
        const uint32_t k = ps_keys[i];
        n_hi += k > kmax;
        n_eq += k >= kmin && k <= kmax;
    }
    int s_hi = n_hi, s_eq = n_eq;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int x = __shfl_up_sync(0xffffffffu, s_hi, o), y = __shfl_up_sync(0xffffffffu, s_eq, o);
        if (lane >= o) { s_hi += x; s_eq += y; }
    }
    __syncthreads();
    if (lane == 31) { tot[0][warp] = s_hi; tot[1][warp] = s_eq; }
    __syncthreads();
    for (int i = 0; i < warp; ++i) { s_hi += tot[0][i]; s_eq += tot[1][i]; }
    int eq = s_eq - n_eq, at = s_hi - n_hi + min(eq, ties);
    for (int i = j0; i < j1; ++i) {
        const uint32_t k = ps_keys[i];
        if (k > kmax || (k >= kmin && eq++ < ties)) sel[at++] = i;
    }
}

}  // namespace sab
