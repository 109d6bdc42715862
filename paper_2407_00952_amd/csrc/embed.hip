// Embedding lookup with scaling, and the gradient of the table.
//
//   out[t] = scale table[tokens[t]],   dtable[v] = scale sum_{t: tokens[t] = v} dout[t]
//
// The lookup is bound by HBM (and by its launch where there are few tokens).  The gradient is formed without atomics: the tokens are
// sorted, stably, by a radix sort on 8 bits a pass (tokens that are padding sort behind all others), which lists the rows of dout that
// belong to a row of the table in token order; then every row of the table is written once, with its sum or with zero.  Bound by
// HBM: dout once, the table's gradient once.
#include "../../include/slora.h"
#include "common.h"

namespace {

constexpr int EB_MAX = 1 << 24;          // tokens, words
constexpr int SORT_THR = 1024, SORT_WAVES = SORT_THR / 64;
constexpr int SORT_TILE = 2048;          // fewest tokens of a block (a multiple of SORT_THR)
constexpr int SORT_BLOCKS = 64;          // most blocks: each adds up the counts of those before it

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
__device__ __forceinline__ void store8(bf16 *p, const float (&v)[8])
{
    bf16x8 t;
#pragma unroll
    for (int i = 0; i < 8; ++i) t[i] = f2bf(v[i]);
    *(bf16x8 *)p = t;
}
__device__ __forceinline__ void store8(float *p, const float (&v)[8])
{
    *(f32x4 *)p = f32x4{v[0], v[1], v[2], v[3]};
    *(f32x4 *)(p + 4) = f32x4{v[4], v[5], v[6], v[7]};
}

// one wave a row
template <class E>
__global__ __launch_bounds__(256) void embed_fwd_kernel(int T, int V, int d, const int *__restrict__ tokens,
                                                        const E *__restrict__ table, float scale, E *__restrict__ out, size_t ldo)
{
    const int lane = threadIdx.x & 63, t = blockIdx.x * 4 + (threadIdx.x >> 6);
    if (t >= T) return;
    const int tok = tokens[t];
    const bool word = tok >= 0 && tok < V;
    const E *src = table + (size_t)(word ? tok : 0) * d;
    for (int col = lane * 8; col < d; col += 512) {
        float v[8];
        if (word) load8(src + col, v);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = word ? v[i] * scale : 0.f;
        store8(out + t * ldo + col, v);
    }
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

// counts [block][256] of the digit at `shift` among a block's `per` positions
template <bool FIRST>
__global__ __launch_bounds__(SORT_THR) void sort_count_kernel(int T, int V, int per, int shift, const int *__restrict__ tokens,
                                                              const Pair *__restrict__ in, int *__restrict__ counts)
{
    __shared__ int h[256];
    if (threadIdx.x < 256) h[threadIdx.x] = 0;
    __syncthreads();
    const int lo = blockIdx.x * per, hi = min(T, lo + per);
    for (int i = lo + threadIdx.x; i < hi; i += SORT_THR)
        atomicAdd(&h[(pair_at<FIRST>(i, V, tokens, in).key >> shift) & 255], 1);     // (integers: any order)
    __syncthreads();
    if (threadIdx.x < 256) counts[blockIdx.x * 256 + threadIdx.x] = h[threadIdx.x];
}

// Stable placement by the digit at `shift`.  A position's place is: the smaller digits everywhere, its digit in the blocks before, in
// the rounds of 1024 positions before, in the waves before, in the lanes before (the lanes with the same digit by eight ballots).
template <bool FIRST>
__global__ __launch_bounds__(SORT_THR) void sort_place_kernel(int T, int V, int per, int shift, const int *__restrict__ tokens,
                                                              const Pair *__restrict__ in, const int *__restrict__ counts,
                                                              Pair *__restrict__ out)
{
    __shared__ int base[256], wcnt[SORT_WAVES][256], scan[4];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    int total = 0, before = 0;
    if (tid < 256) {
        for (int b = 0; b < (int)gridDim.x; ++b) {
            const int n = counts[b * 256 + tid];
            total += n;
            before += b < (int)blockIdx.x ? n : 0;
        }
    }
    int incl = total;                                    // inclusive prefix over the digits
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const int up = __shfl_up(incl, o, 64);
        if (lane >= o) incl += up;
    }
    if (tid < 256 && lane == 63) scan[wave] = incl;
    __syncthreads();
    if (tid < 256) {
        int ex = incl - total;
        for (int w = 0; w < wave; ++w) ex += scan[w];
        base[tid] = ex + before;
    }
    const int lo = blockIdx.x * per, hi = min(T, lo + per);
    for (int r = lo; r < hi; r += SORT_THR) {
        const int i = r + tid;
        const bool on = i < hi;
        Pair p = {0u, 0u};
        if (on) p = pair_at<FIRST>(i, V, tokens, in);
        const int digit = (p.key >> shift) & 255;
        unsigned long long peers = __ballot(on);
#pragma unroll
        for (int b = 0; b < 8; ++b) {
            const unsigned long long m = __ballot((digit >> b) & 1);
            peers &= (digit >> b) & 1 ? m : ~m;
        }
        const int rank = __popcll(peers & ((1ull << lane) - 1));
        for (int c = tid; c < SORT_WAVES * 256; c += SORT_THR) (&wcnt[0][0])[c] = 0;
        __syncthreads();
        if (on && rank == 0) wcnt[wave][digit] = __popcll(peers);
        __syncthreads();
        if (tid < 256) {                                 // the waves' counts become their places
            int at = base[tid];
            for (int w = 0; w < SORT_WAVES; ++w) {
                const int n = wcnt[w][tid];
                wcnt[w][tid] = at;
                at += n;
            }
            base[tid] = at;
        }
        __syncthreads();
        if (on) out[wcnt[wave][digit] + rank] = p;
        __syncthreads();
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

// one wave a row of the table
template <class E>
__global__ __launch_bounds__(256) void embed_sum_kernel(int T, int V, int d, const Pair *__restrict__ sorted,
                                                        const E *__restrict__ dout, size_t ldd, float scale, int accumulate,
                                                        float *__restrict__ dtable)
{
    const int lane = threadIdx.x & 63, v = blockIdx.x * 4 + (threadIdx.x >> 6);
    if (v >= V) return;
    const int lo = keys_below(sorted, T, v, lane), hi = keys_below(sorted, T, v + 1, lane);
    if (accumulate && lo == hi) return;
    for (int col = lane * 8; col < d; col += 512) {
        float s[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f}, t[8];
        for (int i = lo; i < hi; ++i) {
            load8(dout + sorted[i].row * ldd + col, t);
#pragma unroll
            for (int j = 0; j < 8; ++j) s[j] += t[j];
        }
        float *o = dtable + (size_t)v * d + col;
#pragma unroll
        for (int j = 0; j < 8; ++j) s[j] *= scale;
        if (accumulate) {
            load8(o, t);
#pragma unroll
            for (int j = 0; j < 8; ++j) s[j] += t[j];
        }
        store8(o, s);
    }
}

struct EmbedWs { size_t counts, a, b, total; };

inline size_t al256(size_t v) { return (v + 255) & ~(size_t)255; }
EmbedWs embed_ws(int T)
{
    EmbedWs w;
    w.counts = 0;
    w.a = al256(SORT_BLOCKS * 256 * 4);
    w.b = w.a + al256(sizeof(Pair) * (size_t)T);
    w.total = w.b + al256(sizeof(Pair) * (size_t)T);
    return w;
}

inline bool aligned(const void *p, unsigned n) { return ((uintptr_t)p & (n - 1)) == 0; }
inline bool stride_ok(int64_t ld, int d) { return ld >= d && ld % 8 == 0 && ld < (1ll << 40); }
inline bool embed_sizes_ok(int T, int V, int d)
{
    return T >= 0 && T <= EB_MAX && V > 0 && V <= EB_MAX && d > 0 && d <= 65536 && d % 8 == 0;
}

// sorts (token, position) by token; returns the sorted pairs
const Pair *launch_sort(int T, int V, const int *tokens, char *ws, hipStream_t st)
{
    const EmbedWs w = embed_ws(T);
    int *counts = (int *)(ws + w.counts);
    Pair *out = (Pair *)(ws + w.a), *in = (Pair *)(ws + w.b);
    int per = (T + SORT_BLOCKS - 1) / SORT_BLOCKS;
    per = per < SORT_TILE ? SORT_TILE : (per + SORT_THR - 1) / SORT_THR * SORT_THR;
    const int blocks = (T + per - 1) / per;
    for (int shift = 0; shift == 0 || (V >> shift) != 0; shift += 8) {
        if (shift == 0) {
            hipLaunchKernelGGL(sort_count_kernel<true>, dim3(blocks), dim3(SORT_THR), 0, st, T, V, per, shift, tokens, nullptr, counts);
            hipLaunchKernelGGL(sort_place_kernel<true>, dim3(blocks), dim3(SORT_THR), 0, st, T, V, per, shift, tokens, nullptr, counts, out);
        } else {
            hipLaunchKernelGGL(sort_count_kernel<false>, dim3(blocks), dim3(SORT_THR), 0, st, T, V, per, shift, nullptr, in, counts);
            hipLaunchKernelGGL(sort_place_kernel<false>, dim3(blocks), dim3(SORT_THR), 0, st, T, V, per, shift, nullptr, in, counts, out);
        }
        Pair *t = in; in = out; out = t;
    }
    return in;
}

}  // namespace

extern "C" {

int slora_embed_fwd(int32_t T, int32_t vocab, int32_t d, int32_t dtype, const int32_t *tokens, const void *table,
                    float scale, void *out, int64_t ldo, void *stream)
{
    if (!embed_sizes_ok(T, vocab, d) || (dtype != SLORA_DTYPE_F32 && dtype != SLORA_DTYPE_BF16)) return SLORA_EINVAL;
    if (!tokens || !table || !out || !stride_ok(ldo, d)) return SLORA_EINVAL;
    if (!aligned(tokens, 4) || !aligned(table, 16) || !aligned(out, 16)) return SLORA_EINVAL;
    if (T == 0) return SLORA_OK;
    const hipStream_t st = (hipStream_t)stream;
    if (dtype == SLORA_DTYPE_F32)
        hipLaunchKernelGGL(embed_fwd_kernel<float>, dim3((T + 3) / 4), dim3(256), 0, st, T, vocab, d, tokens, (const float *)table, scale,
                           (float *)out, (size_t)ldo);
    else
        hipLaunchKernelGGL(embed_fwd_kernel<bf16>, dim3((T + 3) / 4), dim3(256), 0, st, T, vocab, d, tokens, (const bf16 *)table, scale,
                           (bf16 *)out, (size_t)ldo);
    SL_CHECK_LAUNCH("embed_fwd");
    return SLORA_OK;
}

size_t slora_embed_bwd_ws_bytes(int32_t T, int32_t vocab, int32_t d)
{
    return embed_sizes_ok(T, vocab, d) ? embed_ws(T).total : 0;
}

int slora_embed_bwd(int32_t T, int32_t vocab, int32_t d, int32_t dtype, const int32_t *tokens, const void *dout,
                    int64_t ldd, float scale, int32_t accumulate, float *dtable, void *ws, size_t ws_bytes, void *stream)
{
    if (!embed_sizes_ok(T, vocab, d) || (dtype != SLORA_DTYPE_F32 && dtype != SLORA_DTYPE_BF16)) return SLORA_EINVAL;
    if (!tokens || !dout || !dtable || !ws || !stride_ok(ldd, d) || (accumulate & ~1)) return SLORA_EINVAL;
    if (!aligned(tokens, 4) || !aligned(dout, 16) || !aligned(dtable, 16) || !aligned(ws, 256)) return SLORA_EINVAL;
    if (ws_bytes < embed_ws(T).total) return SLORA_ENOSPC;
    const hipStream_t st = (hipStream_t)stream;
    if (T == 0) return accumulate ? SLORA_OK : launch_fill_zero(dtable, 4 * (size_t)vocab * d, st);
    const Pair *sorted = launch_sort(T, vocab, tokens, (char *)ws, st);
    SL_CHECK_LAUNCH("embed_sort");
    if (dtype == SLORA_DTYPE_F32)
        hipLaunchKernelGGL(embed_sum_kernel<float>, dim3((vocab + 3) / 4), dim3(256), 0, st, T, vocab, d, sorted, (const float *)dout,
                           (size_t)ldd, scale, accumulate, dtable);
    else
        hipLaunchKernelGGL(embed_sum_kernel<bf16>, dim3((vocab + 3) / 4), dim3(256), 0, st, T, vocab, d, sorted, (const bf16 *)dout,
                           (size_t)ldd, scale, accumulate, dtable);
    SL_CHECK_LAUNCH("embed_sum");
    return SLORA_OK;
}

}  // extern "C"
