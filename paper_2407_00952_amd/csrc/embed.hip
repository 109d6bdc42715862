// Embedding lookup with scaling, and the gradient of the table.
//
//   out[t] = scale table[tokens[t]],   dtable[v] = scale sum_{t: tokens[t] = v} dout[t]
//
// The lookup is bound by HBM (and by its launch where there are few tokens).  The gradient is formed without floating-point atomics: the
// tokens are sorted, stably, by a radix sort on 8 bits a pass (tokens that are padding sort behind all others), which lists the rows of
// dout that belong to a row of the table in token order; then every row of the table is written once, with its sum or with zero.
// A word of a text is as frequent as the inverse of its rank, so some runs of the list are long: those of more than 64 are summed
// in pieces of 64 positions first, by blocks of their own, and the pieces in order.  Bound by HBM: dout once, the table's
// gradient once.
#include "../../include/slora.h"
#include "common.h"
#include "stream_store.h"

#include <type_traits>

namespace {

constexpr int EB_MAX = 1 << 24;          // tokens, words
constexpr int SORT_THR = 1024, SORT_WAVES = SORT_THR / 64;
// Fewest tokens of a block (a multiple of SORT_THR; up to so many are sorted by one block in one launch), and the most blocks: each adds up the
// counts of all others.  Gradient of 50257 words x 64 with tiles of 1024 / 2048 / 8192 tokens, us: 2048 tokens 33.1 / 31.2 / 31.2,
// 8192 37.9 / 40.7 / 55.7, 65536 48.5 / 50.7 / 73.1; with 32 / 64 / 256 blocks: 262144 tokens 97 / 82 / 78, 4194304 940 / 654 / 452 (and 4
// times the counts in the workspace).
constexpr int SORT_TILE = 2048;
constexpr int SORT_BLOCKS = 64;

constexpr int LONG_RUN = 64;             // positions of a token from which on it is summed in pieces
constexpr int EMBED_ROWS = 8;            // rows of the table a block writes

struct Pair { unsigned key, row; };      // a token and where it stands

__device__ __forceinline__ void load8(const bf16 *p, float (&v)[8])
{
    const bf16x8 t = *(const bf16x8 *)p;
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = bf2f(t[i]);
}
__device__ __forceinline__ void load8(const float *p, float (&v)[8])
{
    const f32x4 a = *(const f32x4 *)p, b = *(const f32x4 *)(p + 4);
#pragma unroll
    for (int i = 0; i < 4; ++i) { v[i] = a[i]; v[4 + i] = b[i]; }
}
template <bool STREAM>
__device__ __forceinline__ void store8(bf16 *p, const float (&v)[8])
{
    bf16x8 t;
#pragma unroll
    for (int i = 0; i < 8; ++i) t[i] = f2bf(v[i]);
    store_result<STREAM>((bf16x8 *)p, t);
}
template <bool STREAM>
__device__ __forceinline__ void store8(float *p, const float (&v)[8])
{
    store_result<STREAM>((f32x4 *)p, f32x4{v[0], v[1], v[2], v[3]});
    store_result<STREAM>((f32x4 *)(p + 4), f32x4{v[4], v[5], v[6], v[7]});
}

// 2^lg threads a row: a wave; for rows of up to 512 bytes as many as hold it 8 columns each (131072 rows of 64, 128 and 256 in bf16: 21.8,
// 21.7 and 32.6 us with a wave each, 6.1, 9.3 and 23.8 so; of 256 in fp32 29 and 36).  (2, 4 and 8 rows to a wave, their loads in
// flight together, take the same time.  65536 rows of 1024 in bf16, 15510 words of 50257: 31 us, 5.4 TB/s with every word that occurs read
// once; in fp32 78 us, 4.2 TB/s.)
template <class E, bool STREAM>
__global__ __launch_bounds__(256) void embed_fwd_kernel(int T, int V, int d, int lg, const int *__restrict__ tokens,
                                                        const E *__restrict__ table, float scale, E *__restrict__ out, size_t ldo)
{
    const int lane = threadIdx.x & ((1 << lg) - 1), t = (int)blockIdx.x * (256 >> lg) + (int)(threadIdx.x >> lg);
    if (t >= T) return;
    const int tok = tokens[t];
    const bool word = tok >= 0 && tok < V;
    const E *src = table + (size_t)(word ? tok : 0) * d;
    for (int col = lane * 8; col < d; col += 8 << lg) {
        float v[8];
        load8(src + col, v);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = word ? v[i] * scale : 0.f;
        store8<STREAM>(out + t * ldo + col, v);
    }
}

template <class E>
void launch_fwd(int T, int V, int d, const int *tokens, const void *table, float scale, void *out, size_t ldo, hipStream_t st)
{
    int lg = 6;
    if (sizeof(E) * d <= 512)
        while (lg > 0 && (8 << (lg - 1)) >= d) --lg;
    const int rows = 256 >> lg;
    const dim3 grid((T + rows - 1) / rows);
    if (stream_results(sizeof(E) * (size_t)d * (T + (T < V ? T : V))))
        hipLaunchKernelGGL((embed_fwd_kernel<E, true>), grid, dim3(256), 0, st, T, V, d, lg, tokens, (const E *)table, scale, (E *)out, ldo);
    else
        hipLaunchKernelGGL((embed_fwd_kernel<E, false>), grid, dim3(256), 0, st, T, V, d, lg, tokens, (const E *)table, scale, (E *)out, ldo);
}

// ---- sort ---------------------------------------------------------------------------------------
// the key of position i: a token, or V for padding; later passes read the pairs of the pass before
template <bool FIRST>
__device__ __forceinline__ Pair pair_at(int i, int V, const int *tokens, const Pair *in)
{
    if (!FIRST) return in[i];
    const int t = tokens[i];
    return Pair{(unsigned)(t >= 0 && t < V ? t : V), (unsigned)i};
}

// passes of 8 bits over keys 0 .. V (V <= 2^24)
__host__ __device__ inline int sort_passes(int V) { return V < 1 << 8 ? 1 : V < 1 << 16 ? 2 : V < 1 << 24 ? 3 : 4; }

// What a pass of the sort reads and writes; counts [block][256]: of the digit at `shift` among a block's `per` positions
struct SortPass {
    int T, V, per, shift;
    const int *tokens; const Pair *in;
    int *counts;
    Pair *out;
};

template <bool FIRST>
__global__ __launch_bounds__(SORT_THR) void sort_count_kernel(SortPass p)
{
    __shared__ int h[256];
    if (threadIdx.x < 256) h[threadIdx.x] = 0;
    __syncthreads();
    const int lo = blockIdx.x * p.per, hi = min(p.T, lo + p.per);
    for (int i = lo + threadIdx.x; i < hi; i += SORT_THR)
        atomicAdd(&h[(pair_at<FIRST>(i, p.V, p.tokens, p.in).key >> p.shift) & 255], 1);     // (integers: any order)
    __syncthreads();
    if (threadIdx.x < 256) p.counts[blockIdx.x * 256 + threadIdx.x] = h[threadIdx.x];
}

struct SortLds { int base[256], wcnt[SORT_WAVES][256], scan[4]; };

// base[digit] = smaller digits everywhere + this digit in the blocks before (total, before: of the thread's digit)
__device__ __forceinline__ void digit_bases(SortLds &l, int total, int before)
{
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    int incl = total;                                    // inclusive prefix over the digits
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const int up = __shfl_up(incl, o, 64);
        if (lane >= o) incl += up;
    }
    if (tid < 256 && lane == 63) l.scan[wave] = incl;
    __syncthreads();
    if (tid < 256) {
        int ex = incl - total;
        for (int w = 0; w < wave; ++w) ex += l.scan[w];
        l.base[tid] = ex + before;
    }
}

// Stable placement of positions lo .. hi - 1 by the digit at p.shift.  A position's place is: base[digit], its digit in the rounds of 1024
// positions before, in the waves before, in the lanes before (the lanes with the same digit by eight ballots).
template <bool FIRST>
__device__ __forceinline__ void place(const SortPass &p, SortLds &l, int lo, int hi)
{
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    for (int r = lo; r < hi; r += SORT_THR) {
        const int i = r + tid;
        const bool on = i < hi;
        Pair t = {0u, 0u};
        if (on) t = pair_at<FIRST>(i, p.V, p.tokens, p.in);
        const int digit = (t.key >> p.shift) & 255;
        unsigned long long peers = __ballot(on);
#pragma unroll
        for (int b = 0; b < 8; ++b) {
            const unsigned long long m = __ballot((digit >> b) & 1);
            peers &= (digit >> b) & 1 ? m : ~m;
        }
        const int rank = __popcll(peers & ((1ull << lane) - 1));
        for (int c = tid; c < SORT_WAVES * 256; c += SORT_THR) (&l.wcnt[0][0])[c] = 0;
        __syncthreads();
        if (on && rank == 0) l.wcnt[wave][digit] = __popcll(peers);
        __syncthreads();
        if (tid < 256) {                                 // the waves' counts become their places
            int at = l.base[tid], n[SORT_WAVES];
#pragma unroll
            for (int w = 0; w < SORT_WAVES; ++w) n[w] = l.wcnt[w][tid];
#pragma unroll
            for (int w = 0; w < SORT_WAVES; ++w) {
                l.wcnt[w][tid] = at;
                at += n[w];
            }
            l.base[tid] = at;
        }
        __syncthreads();
        if (on) p.out[l.wcnt[wave][digit] + rank] = t;
        __syncthreads();
    }
}

template <bool FIRST>
__global__ __launch_bounds__(SORT_THR) void sort_place_kernel(SortPass p)
{
    __shared__ SortLds l;
    // four threads to a digit add up the blocks' counts
    const int digit = threadIdx.x & 255, quarter = threadIdx.x >> 8;
    int total = 0, before = 0;
    for (int b0 = 0; b0 < (int)gridDim.x; b0 += 32) {    // eight loads in flight
        int n[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) n[k] = p.counts[min(b0 + 4 * k + quarter, (int)gridDim.x - 1) * 256 + digit];
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const int b = b0 + 4 * k + quarter;
            total += b < (int)gridDim.x ? n[k] : 0;
            before += b < (int)blockIdx.x ? n[k] : 0;
        }
    }
    l.wcnt[quarter][digit] = total;
    l.wcnt[4 + quarter][digit] = before;
    __syncthreads();
    total = before = 0;
    if (threadIdx.x < 256) {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            total += l.wcnt[k][digit];
            before += l.wcnt[4 + k][digit];
        }
    }
    digit_bases(l, total, before);
    const int lo = blockIdx.x * p.per;
    place<FIRST>(p, l, lo, min(p.T, lo + p.per));
}

// all passes of few positions in one block
__global__ __launch_bounds__(SORT_THR) void sort_block_kernel(int T, int V, const int *__restrict__ tokens, Pair *out, Pair *in)
{
    __shared__ SortLds l;
    __shared__ int h[256];
    for (int shift = 0; shift < 8 * sort_passes(V); shift += 8) {
        if (threadIdx.x < 256) h[threadIdx.x] = 0;
        __syncthreads();
        for (int i = threadIdx.x; i < T; i += SORT_THR) {
            const unsigned key = shift ? in[i].key : pair_at<true>(i, V, tokens, nullptr).key;
            atomicAdd(&h[(key >> shift) & 255], 1);
        }
        __syncthreads();
        digit_bases(l, threadIdx.x < 256 ? h[threadIdx.x] : 0, 0);
        const SortPass p = {T, V, T, shift, tokens, in, nullptr, out};
        if (shift) place<false>(p, l, 0, T);
        else place<true>(p, l, 0, T);
        __syncthreads();                                 // (the block's own stores: its waves share the memory path)
        Pair *t = in; in = out; out = t;
    }
}

// ---- sums -----------------------------------------------------------------------------------------
// how many of the n sorted keys are below v; the whole wave calls it (64 probes a step)
__device__ __forceinline__ int keys_below(const Pair *sorted, int n, unsigned v, int lane)
{
    int lo = 0, hi = n;
    while (lo < hi) {
        const int step = (hi - lo + 63) >> 6, at = lo + lane * step;
        const int c = __popcll(__ballot(at < hi && sorted[min(at, n - 1)].key < v));
        if (c == 0) break;
        hi = min(hi, lo + c * step);
        lo = lo + (c - 1) * step + 1;
    }
    return lo;
}

// columns of a row of dout in fp32: 4 a lane, so that a wave's stores of the gradient are whole lines
__device__ __forceinline__ f32x4 load4(const bf16 *p)
{
    const bf16x4 t = *(const bf16x4 *)p;
    return f32x4{bf2f(t[0]), bf2f(t[1]), bf2f(t[2]), bf2f(t[3])};
}
__device__ __forceinline__ f32x4 load4(const float *p) { return *(const f32x4 *)p; }

template <bool STREAM>
__device__ __forceinline__ void put4(float *o, f32x4 s, float scale, int accumulate)
{
    s = s * scale;
    if (accumulate) s = s + *(const f32x4 *)o;
    store_result<STREAM>((f32x4 *)o, s);
}

// Sum of n rows, in order, of 4 columns; where(i): address of row i.  Up to eight rows in flight.
template <int N, class F>
__device__ __forceinline__ void add_rows(f32x4 &s, int i, F where)
{
    f32x4 t[N];
#pragma unroll
    for (int k = 0; k < N; ++k) t[k] = load4(where(i + k));
#pragma unroll
    for (int k = 0; k < N; ++k) s = s + t[k];
}
template <class F>
__device__ __forceinline__ f32x4 sum_rows(int n, F where)
{
    f32x4 s = {0.f, 0.f, 0.f, 0.f};
    int i = 0;
    for (; i + 8 <= n; i += 8) add_rows<8>(s, i, where);
    if (n & 4) { add_rows<4>(s, i, where); i += 4; }
    if (n & 2) { add_rows<2>(s, i, where); i += 2; }
    if (n & 1) add_rows<1>(s, i, where);
    return s;
}

// The same shared by a block's groups of threads: a group has lanes for 4 columns each and a piece of the rows; sums of the groups in
// order through LDS.  Every thread calls it; the result is right in group 0.
template <class F>
__device__ __forceinline__ f32x4 sum_rows_block(int n, int lanes, f32x4 *red, F where)
{
    const int groups = 256 / lanes, gr = threadIdx.x / lanes, per = (n + groups - 1) / groups;
    const int a = min(gr * per, n), b = gr < groups ? min(a + per, n) : a;
    f32x4 s = sum_rows(b - a, [&](int i) { return where(a + i); });
    __syncthreads();
    red[threadIdx.x] = s;
    __syncthreads();
    if (gr == 0)
        for (int g = 1; g < groups; ++g) s = s + red[g * lanes + threadIdx.x];
    return s;
}

// Long runs (more than LONG_RUN positions of one key).  Piece c is positions 64 c .. 64 c + 63; a long run that touches it covers
// its start or its end, or both, so a piece holds at most two sums: part[c][0] of a long run that covers its start, part[c][1] of one
// that starts inside.  A run reaching 64 positions before (behind) its last (first) one in the piece is long.
struct Piece { int n0, b1; };            // positions of the first sum; first position of the second (64: none)
__device__ __forceinline__ Piece piece_of(const Pair *sorted, int T, int V, int c, int lane)
{
    const int base = c * LONG_RUN, n = min(LONG_RUN, T - base);
    const unsigned key = sorted[base + min(lane, n - 1)].key;
    const unsigned first = __shfl(key, 0, 64), last = __shfl(key, n - 1, 64);
    const int a = __popcll(__ballot(lane < n && key == first));          // positions of the first key
    const int b = n - __popcll(__ballot(lane < n && key == last));       // where the last one starts
    Piece p;
    p.n0 = 0;
    p.b1 = LONG_RUN;
    // (words only: padding, key V, has no row)
    if (first < (unsigned)V) {
        const int back = base + a - 1 - LONG_RUN, on = base + LONG_RUN;
        const bool is_long = (back >= 0 && sorted[back].key == first) || (a == LONG_RUN && on < T && sorted[on].key == first);
        if (is_long) p.n0 = a;
    }
    if (b > 0 && last < (unsigned)V) {
        const int on = base + b + LONG_RUN;
        if (on < T && sorted[on].key == last) p.b1 = b;
    }
    return p;
}

// (The whole gradient of 65536 tokens x 1024, 50257 words, written / added: bf16 112 / 102 us, fp32 141 / 136.)
// Blocks 0 .. pieces - 1 sum the long runs' share of a piece each (waits for memory mostly: they run beside the others' stores); the
// others write EMBED_ROWS rows of the table each, a wave one after the other, and leave the long ones out.
template <class E, bool STREAM>
__global__ __launch_bounds__(256) void embed_sum_kernel(int T, int V, int d, int lanes, int pieces, const Pair *__restrict__ sorted,
                                                        const E *__restrict__ dout, size_t ldd, float scale, int accumulate,
                                                        float *__restrict__ part, float *__restrict__ dtable)
{
    __shared__ f32x4 red[256];
    const int lane = threadIdx.x & 63;
    if ((int)blockIdx.x < pieces) {
        const int c = blockIdx.x, base = c * LONG_RUN, cl = (threadIdx.x % lanes) * 4;
        const Piece p = piece_of(sorted, T, V, c, lane);
#pragma unroll
        for (int w = 0; w < 2; ++w) {
            const int first = w ? base + p.b1 : base, n = w ? max(min(LONG_RUN, T - base) - p.b1, 0) : p.n0;
            if (n == 0) continue;                        // (uniform over the block)
            for (int col = 0; col < d; col += lanes * 4) {
                const int my = min(col + cl, d - 4);
                const f32x4 s = sum_rows_block(n, lanes, red, [&](int i) { return dout + sorted[first + i].row * ldd + my; });
                if ((int)threadIdx.x < lanes && col + cl < d) *(f32x4 *)(part + ((size_t)c * 2 + w) * d + my) = s;
            }
        }
        return;
    }
    const int v0 = ((int)blockIdx.x - pieces) * EMBED_ROWS, v1 = min(v0 + EMBED_ROWS, V);
    int lo = keys_below(sorted, T, v0, lane), window = lo;
    Pair at = sorted[min(lo + lane, T - 1)];             // 64 positions from `window` on
    for (int v = v0; v < v1; ++v) {
        unsigned long long same = __ballot(window + lane < T && at.key == (unsigned)v);
        if ((same >> 63) && window != lo) {              // the run may go on behind the window: one that starts with it
            window = lo;
            at = sorted[min(lo + lane, T - 1)];
            same = __ballot(window + lane < T && at.key == (unsigned)v);
        }
        const int n = __popcll(same);
        const bool is_long = n == 64 && lo + 64 < T && sorted[lo + 64].key == (unsigned)v;
        const int first = __builtin_amdgcn_readfirstlane(lo - window), rows = __builtin_amdgcn_readfirstlane(n);
        const unsigned row = at.row;
        lo = is_long ? keys_below(sorted, T, v + 1, lane) : lo + n;
        if (lo >= window + 64) {
            window = lo;
            at = sorted[min(lo + lane, T - 1)];
        }
        if (is_long || (v & 3) != (int)(threadIdx.x >> 6) || (accumulate && n == 0)) continue;
        for (int c0 = 0; c0 < d; c0 += 1024) {           // 1024 columns of a row at a time, two rows in flight
            f32x4 s[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) s[k] = f32x4{0.f, 0.f, 0.f, 0.f};
            auto add = [&](int i, auto count) {
                f32x4 t[decltype(count)::value][4];
#pragma unroll
                for (int r = 0; r < decltype(count)::value; ++r) {
                    const E *src = dout + (unsigned)__builtin_amdgcn_readlane((int)row, first + i + r) * ldd;
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const int col = c0 + 256 * k + lane * 4;
                        t[r][k] = load4(src + (col < d ? col : 0));
                    }
                }
#pragma unroll
                for (int r = 0; r < decltype(count)::value; ++r)
#pragma unroll
                    for (int k = 0; k < 4; ++k) s[k] = s[k] + t[r][k];
            };
            int i = 0;
            for (; i + 2 <= rows; i += 2) add(i, std::integral_constant<int, 2>());
            if (i < rows) add(i, std::integral_constant<int, 1>());
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int col = c0 + 256 * k + lane * 4;
                if (col < d) put4<STREAM>(dtable + (size_t)v * d + col, s[k], scale, accumulate);
            }
        }
    }
}

// Each block finishes the long run that starts in its piece, if one does
__global__ __launch_bounds__(256) void embed_finish_kernel(int T, int V, int d, int lanes, const Pair *__restrict__ sorted, float scale,
                                                           int accumulate, const float *__restrict__ part, float *__restrict__ dtable)
{
    __shared__ f32x4 red[256];
    const int c = blockIdx.x, lane = threadIdx.x & 63, base = c * LONG_RUN;
    const Piece p = piece_of(sorted, T, V, c, lane);
    int start = -1;
    if (p.b1 < LONG_RUN) start = base + p.b1;
    else if (p.n0 > 0 && (base == 0 || sorted[base - 1].key != sorted[base].key)) start = base;
    if (start < 0) return;
    const unsigned v = sorted[start].key;
    const int end = keys_below(sorted, T, v + 1, lane), n = (end - 1) / LONG_RUN - c + 1;
    const int cl = (threadIdx.x % lanes) * 4, w0 = start > base ? 1 : 0;
    for (int col = 0; col < d; col += lanes * 4) {
        const int my = min(col + cl, d - 4);
        const f32x4 s = sum_rows_block(n, lanes, red, [&](int i) { return part + ((size_t)(c + i) * 2 + (i ? 0 : w0)) * d + my; });
        if ((int)threadIdx.x < lanes && col + cl < d) put4<false>(dtable + (size_t)v * d + my, s, scale, accumulate);
    }
}

struct EmbedWs { size_t counts, a, b, part, total; };

inline size_t al256(size_t v) { return (v + 255) & ~(size_t)255; }
inline int pieces_of(int T) { return (T + LONG_RUN - 1) / LONG_RUN; }
EmbedWs embed_ws(int T, int d)
{
    EmbedWs w;
    w.counts = 0;
    w.a = al256(SORT_BLOCKS * 256 * 4);
    w.b = w.a + al256(sizeof(Pair) * (size_t)T);
    w.part = w.b + al256(sizeof(Pair) * (size_t)T);
    w.total = w.part + (T > LONG_RUN ? al256(8 * (size_t)pieces_of(T) * d) : 0);
    return w;
}

inline bool aligned(const void *p, unsigned n) { return ((uintptr_t)p & (n - 1)) == 0; }
inline bool stride_ok(int64_t ld, int d) { return ld >= d && ld % 8 == 0 && ld < (1ll << 40); }
inline bool embed_sizes_ok(int T, int V, int d)
{
    return T >= 0 && T <= EB_MAX && V > 0 && V <= EB_MAX && d > 0 && d <= 65536 && d % 8 == 0;
}

// sorts (token, position) by token; returns the sorted pairs
const Pair *launch_sort(int T, int V, const int *tokens, char *ws, const EmbedWs &w, hipStream_t st)
{
    Pair *out = (Pair *)(ws + w.a), *in = (Pair *)(ws + w.b);
    const int passes = sort_passes(V);
    if (T <= SORT_TILE) {
        hipLaunchKernelGGL(sort_block_kernel, dim3(1), dim3(SORT_THR), 0, st, T, V, tokens, out, in);
        return passes & 1 ? out : in;
    }
    int per = (T + SORT_BLOCKS - 1) / SORT_BLOCKS;
    per = per < SORT_TILE ? SORT_TILE : (per + SORT_THR - 1) / SORT_THR * SORT_THR;
    const int blocks = (T + per - 1) / per;
    for (int i = 0; i < passes; ++i) {
        const SortPass p = {T, V, per, 8 * i, tokens, in, (int *)(ws + w.counts), out};
        if (i == 0) {
            hipLaunchKernelGGL(sort_count_kernel<true>, dim3(blocks), dim3(SORT_THR), 0, st, p);
            hipLaunchKernelGGL(sort_place_kernel<true>, dim3(blocks), dim3(SORT_THR), 0, st, p);
        } else {
            hipLaunchKernelGGL(sort_count_kernel<false>, dim3(blocks), dim3(SORT_THR), 0, st, p);
            hipLaunchKernelGGL(sort_place_kernel<false>, dim3(blocks), dim3(SORT_THR), 0, st, p);
        }
        Pair *t = in; in = out; out = t;
    }
    return in;
}

template <class E>
void launch_sums(int T, int V, int d, const Pair *sorted, const void *dout, size_t ldd, float scale, int accumulate, float *part,
                 float *dtable, hipStream_t st)
{
    const int lanes = d / 4 < 256 ? d / 4 : 256;         // threads that hold a row's columns, 4 each
    const int pieces = T > LONG_RUN ? pieces_of(T) : 0;  // (no run is long where there are no more positions)
    const size_t moved = sizeof(E) * (size_t)T * d + (accumulate ? 8 * (size_t)d * (T < V ? T : V) : 4 * (size_t)V * d);
    const dim3 grid(pieces + (V + EMBED_ROWS - 1) / EMBED_ROWS);
    if (stream_results(moved))
        hipLaunchKernelGGL((embed_sum_kernel<E, true>), grid, dim3(256), 0, st, T, V, d, lanes, pieces, sorted, (const E *)dout, ldd, scale,
                           accumulate, part, dtable);
    else
        hipLaunchKernelGGL((embed_sum_kernel<E, false>), grid, dim3(256), 0, st, T, V, d, lanes, pieces, sorted, (const E *)dout, ldd, scale,
                           accumulate, part, dtable);
    if (pieces)
        hipLaunchKernelGGL(embed_finish_kernel, dim3(pieces), dim3(256), 0, st, T, V, d, lanes, sorted, scale, accumulate, part, dtable);
}

}  // namespace

extern "C" {

int slora_embed_fwd(int32_t T, int32_t vocab, int32_t d, int32_t dtype, const int32_t *tokens, const void *table,
                    float scale, void *out, int64_t ldo, void *stream)
{
    if (!embed_sizes_ok(T, vocab, d) || (dtype != SLORA_DTYPE_F32 && dtype != SLORA_DTYPE_BF16)) return SLORA_EINVAL;
    if (T == 0) return SLORA_OK;                         // (an empty tensor has no address)
    if (!tokens || !table || !out || !stride_ok(ldo, d)) return SLORA_EINVAL;
    if (!aligned(tokens, 4) || !aligned(table, 16) || !aligned(out, 16)) return SLORA_EINVAL;
    const hipStream_t st = (hipStream_t)stream;
    if (dtype == SLORA_DTYPE_F32) launch_fwd<float>(T, vocab, d, tokens, table, scale, out, (size_t)ldo, st);
    else launch_fwd<bf16>(T, vocab, d, tokens, table, scale, out, (size_t)ldo, st);
    SL_CHECK_LAUNCH("embed_fwd");
    return SLORA_OK;
}

size_t slora_embed_bwd_ws_bytes(int32_t T, int32_t vocab, int32_t d)
{
    return embed_sizes_ok(T, vocab, d) ? embed_ws(T, d).total : 0;
}

int slora_embed_bwd(int32_t T, int32_t vocab, int32_t d, int32_t dtype, const int32_t *tokens, const void *dout,
                    int64_t ldd, float scale, int32_t accumulate, float *dtable, void *ws, size_t ws_bytes, void *stream)
{
    if (!embed_sizes_ok(T, vocab, d) || (dtype != SLORA_DTYPE_F32 && dtype != SLORA_DTYPE_BF16)) return SLORA_EINVAL;
    if (!dtable || !aligned(dtable, 16) || (accumulate & ~1)) return SLORA_EINVAL;
    const hipStream_t st = (hipStream_t)stream;
    if (T == 0) return accumulate ? SLORA_OK : launch_fill_zero(dtable, 4 * (size_t)vocab * d, st);
    if (!tokens || !dout || !ws || !stride_ok(ldd, d)) return SLORA_EINVAL;
    if (!aligned(tokens, 4) || !aligned(dout, 16) || !aligned(ws, 256)) return SLORA_EINVAL;
    if (ws_bytes < embed_ws(T, d).total) return SLORA_ENOSPC;
    const EmbedWs w = embed_ws(T, d);
    const Pair *sorted = launch_sort(T, vocab, tokens, (char *)ws, w, st);
    SL_CHECK_LAUNCH("embed_sort");
    float *part = (float *)((char *)ws + w.part);
    if (dtype == SLORA_DTYPE_F32) launch_sums<float>(T, vocab, d, sorted, dout, (size_t)ldd, scale, accumulate, part, dtable, st);
    else launch_sums<bf16>(T, vocab, d, sorted, dout, (size_t)ldd, scale, accumulate, part, dtable, st);
    SL_CHECK_LAUNCH("embed_sum");
    return SLORA_OK;
}

}  // extern "C"
