// Root-mean-square norm with the residual's addition, its result in bf16, in MXFP8 or both, and its backward.
//
//   s = x + res,  rho = 1 / sqrt(mean(s^2) + eps),  u = gamma s rho
//   dh = dres + rho (gamma du - h rho m),  m = mean(gamma du h rho),  dgamma = sum_t du h rho
//
// Both are bound by HBM: every tensor is read or written once, a row stays in registers between its sum and its result.  A row of
// up to 2048 columns belongs to one wave (4 rows to a block), of up to 256 or 128 to half or a quarter of one, longer ones to a block
// of 4 or 8 waves.  A lane moves 16 bytes of the
// residual stream at a time: 4 neighbouring columns of it in fp32, 8 in bf16, so that a wave's accesses are whole lines.  Columns past
// the row are loaded from its start instead and counted as zero: no branch stands between the loads of a row.
#include "../../include/slora.h"
#include "common.h"
#include "mx_codec.h"
#include "stream_store.h"

namespace {

constexpr int RN_MAXD = 16384;
constexpr int RN_MAXT = 1 << 23;         // rows: a grid has fewer than 2^32 threads, up to 512 of them a row
constexpr int RN_MAX_PARTS = 512;        // partial sums of dgamma

// RES: 0 no residual, 1 bf16, 2 fp32.  W columns to a piece: what 16 bytes of the residual stream hold (8 where there is none).
template <int RES> struct Row {
    typedef bf16 type;
    typedef bf16x8 piece, piece16;       // of the residual stream, of a bf16 tensor
    static constexpr int W = 8;
};
template <> struct Row<2> {
    typedef float type;
    typedef f32x4 piece;
    typedef bf16x4 piece16;
    static constexpr int W = 4;
};

typedef unsigned u32x2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ float to_f(bf16 v) { return bf2f(v); }
__device__ __forceinline__ float to_f(float v) { return v; }
template <bool STREAM>
__device__ __forceinline__ void put(bf16 *p, const float (&v)[8])
{
    bf16x8 t;
#pragma unroll
    for (int i = 0; i < 8; ++i) t[i] = f2bf(v[i]);
    store_result<STREAM>((bf16x8 *)p, t);
}
template <bool STREAM>
__device__ __forceinline__ void put(bf16 *p, const float (&v)[4])
{
    bf16x4 t;
#pragma unroll
    for (int i = 0; i < 4; ++i) t[i] = f2bf(v[i]);
    store_result<STREAM>((bf16x4 *)p, t);
}
template <bool STREAM>
__device__ __forceinline__ void put(float *p, const float (&v)[4])
{
    store_result<STREAM>((f32x4 *)p, f32x4{v[0], v[1], v[2], v[3]});
}
template <bool STREAM>
__device__ __forceinline__ void put(float *p, const float (&v)[8])
{
    store_result<STREAM>((f32x4 *)p, f32x4{v[0], v[1], v[2], v[3]});
    store_result<STREAM>((f32x4 *)(p + 4), f32x4{v[4], v[5], v[6], v[7]});
}

// The compiler may not know that p is what it was: it unpacks p again where it is used again, instead of keeping the unpacked values
// (registers of half the waves) until then.
template <class P>
__device__ __forceinline__ void forget(P &p)
{
    union { P v; unsigned w[sizeof(P) / 4]; } b;
    b.v = p;
#pragma unroll
    for (unsigned i = 0; i < sizeof(P) / 4; ++i) asm volatile("" : "+v"(b.w[i]));
    p = b.v;
}

// sum over the TPR threads of a row; every thread of the row calls it, of the block where a row has more than a wave
template <int TPR>
__device__ __forceinline__ float row_sum(float v, float *red)
{
    if (TPR < 64) {
#pragma unroll
        for (int o = TPR / 2; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
        return v;
    }
    v = wave_sum(v);
    if (TPR == 64) return v;
    __syncthreads();                     // `red` may still be read from the sum before
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
    __syncthreads();
    float s = red[0];
#pragma unroll
    for (int w = 1; w < TPR / 64; ++w) s += red[w];
    return s;
}

// MXFP8 of W bf16 values a lane, blocks of 32 / W neighbouring lanes; every thread of the row calls it.  (Stored the ordinary way:
// half the bytes of the bf16 result, and what reads them comes next: 71 us against 74, the reader 21 against 24.5.)
template <int W, class P>
__device__ __forceinline__ void mx_put(P o, bool valid, int lane, unsigned char *q_row, unsigned char *s_row, int col)
{
    union { P v; unsigned w[W / 2]; } b;
    b.v = o;
    unsigned mag = 0u;
#pragma unroll
    for (int i = 0; i < W / 2; ++i) mag = max(mag, max(b.w[i] & 0x7FFFu, (b.w[i] >> 16) & 0x7FFFu));
#pragma unroll
    for (int k = 1; k < 32 / W; k <<= 1) mag = max(mag, (unsigned)__shfl_xor((int)mag, k, 64));
    if (!valid) return;
    const int sc = mx_scale_code(mag);
    union { unsigned short h[W / 2]; unsigned w[W / 4]; } q;
#pragma unroll
    for (int i = 0; i < W / 2; ++i) q.h[i] = (unsigned short)mx_encode_pair_bf16(b.w[i] & 0xFFFFu, b.w[i] >> 16, sc);
    if (W == 8) *(u32x2 *)(q_row + col) = u32x2{q.w[0], q.w[W / 4 - 1]};
    else *(unsigned *)(q_row + col) = q.w[0];
    if ((lane & (32 / W - 1)) == 0) s_row[col >> 5] = (unsigned char)sc;
}

// NC times 8 columns a thread, TPR threads a row
template <int RES, int NC, int TPR, bool STREAM>
__global__ __launch_bounds__(TPR < 256 ? 256 : TPR) void rmsnorm_fwd_kernel(
    int T, int d, const bf16 *x, size_t ldx, const typename Row<RES>::type *res, const bf16 *__restrict__ gamma, float eps,
    typename Row<RES>::type *h, bf16 *u, size_t ldu, unsigned char *__restrict__ codes, unsigned char *__restrict__ scales,
    float *__restrict__ rho_out)
{
    typedef typename Row<RES>::piece P;
    typedef typename Row<RES>::piece16 P16;
    constexpr int W = Row<RES>::W, N = NC * 8 / W, RPB = TPR < 256 ? 256 / TPR : 1;
    __shared__ float red[TPR < 64 ? 1 : TPR / 64];
    const int lane = threadIdx.x & 63, rt = threadIdx.x % TPR;
    const int row = blockIdx.x * RPB + threadIdx.x / TPR;
    if (row >= T) return;                // all threads of a row, whole blocks where they share one
    P16 xv[N], g[N];
    P rv[N];
    float s[N][W], q = 0.f;
#pragma unroll
    for (int c = 0; c < N; ++c) {
        const int col = (c * TPR + rt) * W, at = col < d ? col : 0;
        xv[c] = *(const P16 *)(x + row * ldx + at);
        if (RES) rv[c] = *(const P *)(res + (size_t)row * d + at);
    }
#pragma unroll
    for (int c = 0; c < N; ++c) {
        const int col = (c * TPR + rt) * W;
        g[c] = *(const P16 *)(gamma + (col < d ? col : 0));
    }
#pragma unroll
    for (int c = 0; c < N; ++c)
#pragma unroll
        for (int i = 0; i < W; ++i) {
            const float v = RES ? to_f(xv[c][i]) + to_f(rv[c][i]) : to_f(xv[c][i]);
            s[c][i] = (c * TPR + rt) * W < d ? v : 0.f;
            q = fmaf(s[c][i], s[c][i], q);
        }
    const float rho = rsqrtf(row_sum<TPR>(q, red) / (float)d + eps);
    if (rho_out && rt == 0) rho_out[row] = rho;
#pragma unroll
    for (int c = 0; c < N; ++c) {
        const int col = (c * TPR + rt) * W;
        const bool in = col < d;
        if (RES && h && in) put<STREAM>(h + (size_t)row * d + col, s[c]);
        P16 o;
#pragma unroll
        for (int i = 0; i < W; ++i) o[i] = f2bf(s[c][i] * rho * to_f(g[c][i]));
        if (u && in) store_result<STREAM>((P16 *)(u + row * ldu + col), o);
        if (codes) mx_put<W>(o, in, lane, codes + (size_t)row * d, scales + (size_t)row * (d >> 5), col);
    }
}

// Blocks walk the rows with the grid's stride, so that each keeps one partial sum of dgamma in registers; part [blocks][d], or null.  A
// row's tensors stay packed until they are used: registers for more waves.
template <int RES, int NC, int TPR, bool STREAM>
__global__ __launch_bounds__(TPR < 256 ? 256 : TPR) void rmsnorm_bwd_kernel(
    int T, int d, const bf16 *__restrict__ du, size_t lddu, const typename Row<RES>::type *__restrict__ h,
    const float *__restrict__ rho_in, const bf16 *__restrict__ gamma, const typename Row<RES>::type *dres,
    typename Row<RES>::type *dh, bf16 *__restrict__ dx, size_t lddx, float *__restrict__ part)
{
    typedef typename Row<RES>::piece P;
    typedef typename Row<RES>::piece16 P16;
    constexpr int W = Row<RES>::W, N = NC * 8 / W, RPB = TPR < 256 ? 256 / TPR : 1;
    __shared__ float red[TPR < 64 ? 1 : TPR / 64];
    __shared__ float acc[RPB > 1 ? NC * 512 : 1];
    const int rt = threadIdx.x % TPR, sub = threadIdx.x / TPR;
    P16 g[N];
    float dg[N][W];
#pragma unroll
    for (int c = 0; c < N; ++c) {
        const int col = (c * TPR + rt) * W;
        g[c] = *(const P16 *)(gamma + (col < d ? col : 0));
#pragma unroll
        for (int i = 0; i < W; ++i) dg[c][i] = 0.f;
    }
    for (long long r0 = (long long)blockIdx.x * RPB; r0 < T; r0 += (long long)gridDim.x * RPB) {
        const bool on = r0 + sub < T;
        const int row = on ? (int)r0 + sub : T - 1;      // (a row past the end repeats the last one and stores nothing)
        P16 a[N];
        P v[N], r[N];
#pragma unroll
        for (int c = 0; c < N; ++c) {
            const int col = (c * TPR + rt) * W, at = col < d ? col : 0;
            a[c] = *(const P16 *)(du + row * lddu + at);
            v[c] = *(const P *)(h + (size_t)row * d + at);
        }
        const float rho = rho_in[row];
        if (dres) {
#pragma unroll
            for (int c = 0; c < N; ++c) {
                const int col = (c * TPR + rt) * W;
                r[c] = *(const P *)(dres + (size_t)row * d + (col < d ? col : 0));
            }
        } else {
#pragma unroll
            for (int c = 0; c < N; ++c)
#pragma unroll
                for (int i = 0; i < W; ++i) r[c][i] = 0.f;
        }
#pragma unroll
        for (int c = 0; c < N; ++c) forget(g[c]);
        float m = 0.f;
#pragma unroll
        for (int c = 0; c < N; ++c) {
            const bool in = on && (c * TPR + rt) * W < d;
#pragma unroll
            for (int i = 0; i < W; ++i) {
                const float t = in ? to_f(a[c][i]) * (to_f(v[c][i]) * rho) : 0.f;
                dg[c][i] += t;
                m = fmaf(t, to_f(g[c][i]), m);
            }
        }
        m = row_sum<TPR>(m, red) / (float)d;
#pragma unroll
        for (int c = 0; c < N; ++c) {
            forget(g[c]);
            forget(a[c]);
            forget(v[c]);
            forget(r[c]);
        }
#pragma unroll
        for (int c = 0; c < N; ++c) {
            const int col = (c * TPR + rt) * W;
            if (on && col < d) {
                float o[W];
#pragma unroll
                for (int i = 0; i < W; ++i)
                    o[i] = fmaf(rho, fmaf(to_f(a[c][i]), to_f(g[c][i]), -(to_f(v[c][i]) * rho) * m), to_f(r[c][i]));
                if (dh) put<STREAM>(dh + (size_t)row * d + col, o);
                if (dx) put<STREAM>(dx + row * lddx + col, o);
            }
        }
    }
    if (!part) return;
    if (RPB > 1) {                                       // the block's rows one after the other: a fixed order
        for (int w = 0; w < RPB; ++w) {
            if (sub == w) {
#pragma unroll
                for (int c = 0; c < N; ++c)
#pragma unroll
                    for (int i = 0; i < W; ++i) {
                        float *p = acc + (c * TPR + rt) * W + i;
                        *p = w ? *p + dg[c][i] : dg[c][i];
                    }
            }
            __syncthreads();
        }
        for (int col = threadIdx.x; col < d; col += blockDim.x) part[(size_t)blockIdx.x * d + col] = acc[col];
    } else {
#pragma unroll
        for (int c = 0; c < N; ++c)
            if ((c * TPR + rt) * W < d) put<false>(part + (size_t)blockIdx.x * d + (c * TPR + rt) * W, dg[c]);
    }
}

// dgamma = the partial sums in order: 16 columns a block, 64 threads with a 64th of the partial sums each for a column
__global__ __launch_bounds__(1024) void rmsnorm_dgamma_kernel(const float *__restrict__ part, int n, int d, float *__restrict__ dgamma)
{
    __shared__ float red[64][17];
    const int c = threadIdx.x & 15, sub = threadIdx.x >> 4, col = blockIdx.x * 16 + c;
    const int per = (n + 63) / 64, lo = min(sub * per, n), hi = min(lo + per, n);
    float s = 0.f;
    if (col < d) {
        for (int i = lo; i < hi; i += 8) {               // eight loads in flight
            float t[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) t[k] = part[(size_t)min(i + k, hi - 1) * d + col];
#pragma unroll
            for (int k = 0; k < 8; ++k) s += i + k < hi ? t[k] : 0.f;
        }
    }
    red[sub][c] = s;
    __syncthreads();
    if (threadIdx.x < 16 && col < d) {
        s = 0.f;
#pragma unroll
        for (int w = 0; w < 64; ++w) s += red[w][c];
        dgamma[col] = s;
    }
}

// (Narrow rows share a wave: [300000, 128] bf16, backward with dgamma 179 us with a wave each, 64 with a quarter of one; without dgamma 99.5
// and 54.3 = 5.7 TB/s; [33563, 160] with half of one 22.8 and 15.3.)
inline int rows_per_block(int d) { return d <= 128 ? 16 : d <= 256 ? 8 : d <= 2048 ? 4 : 1; }

// Blocks of the backward.  Where dgamma is wanted a block's partial sum costs a write and a read of a row in fp32, and fewer blocks are
// better: [32768, 1024] fp32 with 4096, 1024 and 512 of them 103, 92.5 and 89.6 us, [10001, 5120] bf16 92.9 and 82.9.  Without dgamma every
// row has its own wave: blocks that start one after the other spread reads and writes better than ones that walk in step
// (83.0 us against 87.5, 71.7 against 81.0 = 5.7 TB/s).
inline int bwd_blocks(int T, int d, bool dgamma)
{
    const int blocks = (T + rows_per_block(d) - 1) / rows_per_block(d);
    return dgamma && blocks > RN_MAX_PARTS ? RN_MAX_PARTS : blocks;
}

struct FwdCall {
    int T, d; const bf16 *x; size_t ldx; const void *res; const bf16 *gamma; float eps; void *h; bf16 *u; size_t ldu;
    unsigned char *codes, *scales; float *rho; bool stream; hipStream_t st;
    template <int RES, int NC, int TPR> void go() const { stream ? go_as<RES, NC, TPR, true>() : go_as<RES, NC, TPR, false>(); }
    template <int RES, int NC, int TPR, bool STREAM> void go_as() const
    {
        typedef typename Row<RES>::type R;
        const int rpb = TPR < 256 ? 256 / TPR : 1;
        hipLaunchKernelGGL((rmsnorm_fwd_kernel<RES, NC, TPR, STREAM>), dim3((T + rpb - 1) / rpb), dim3(TPR < 256 ? 256 : TPR), 0, st, T, d, x, ldx,
                           (const R *)res, gamma, eps, (R *)h, u, ldu, codes, scales, rho);
    }
};
struct BwdCall {
    int T, d; const bf16 *du; size_t lddu; const void *h; const float *rho; const bf16 *gamma; const void *dres; void *dh; bf16 *dx;
    size_t lddx; float *part; int blocks; bool stream; hipStream_t st;
    template <int RES, int NC, int TPR> void go() const { stream ? go_as<RES, NC, TPR, true>() : go_as<RES, NC, TPR, false>(); }
    template <int RES, int NC, int TPR, bool STREAM> void go_as() const
    {
        typedef typename Row<RES>::type R;
        hipLaunchKernelGGL((rmsnorm_bwd_kernel<RES, NC, TPR, STREAM>), dim3(blocks), dim3(TPR < 256 ? 256 : TPR), 0, st, T, d, du, lddu, (const R *)h,
                           rho, gamma, (const R *)dres, (R *)dh, dx, lddx, part);
    }
};

// the kernel of a width: as few threads and chunks as hold a row
template <int RES, class Call>
void by_width(const Call &c)
{
    const int d = c.d;
    if (d <= 128) c.template go<RES, 1, 16>();
    else if (d <= 256) c.template go<RES, 1, 32>();
    else if (d <= 512) c.template go<RES, 1, 64>();
    else if (d <= 1024) c.template go<RES, 2, 64>();
    else if (d <= 1536) c.template go<RES, 3, 64>();
    else if (d <= 2048) c.template go<RES, 4, 64>();
    else if (d <= 4096) c.template go<RES, 2, 256>();
    else if (d <= 6144) c.template go<RES, 3, 256>();
    else if (d <= 8192) c.template go<RES, 4, 256>();
    else if (d <= 12288) c.template go<RES, 3, 512>();
    else c.template go<RES, 4, 512>();
}

inline bool aligned(const void *p, unsigned n) { return ((uintptr_t)p & (n - 1)) == 0; }
inline bool stride_ok(int64_t ld, int d) { return ld >= d && ld % 8 == 0 && ld < (1ll << 40); }

}  // namespace

extern "C" {

int slora_rmsnorm_fwd(int32_t T, int32_t d, int32_t res_dtype, const void *x, int64_t ldx, const void *res,
                      const void *gamma, float eps, void *h, void *u, int64_t ldu, void *codes, void *scales,
                      float *rho, void *stream)
{
    if (T < 0 || T >= RN_MAXT || d <= 0 || d > RN_MAXD || d % 8 || !(eps >= 0.f)) return SLORA_EINVAL;
    if (res_dtype != SLORA_DTYPE_F32 && res_dtype != SLORA_DTYPE_BF16) return SLORA_EINVAL;
    if (T == 0) return SLORA_OK;                         // (an empty tensor has no address)
    if (!x || !gamma || (!u && !codes) || !codes != !scales || (h && !res)) return SLORA_EINVAL;
    if (!stride_ok(ldx, d) || (u && !stride_ok(ldu, d)) || (codes && d % 32)) return SLORA_EINVAL;
    if (!aligned(x, 16) || !aligned(res, 16) || !aligned(gamma, 16) || !aligned(h, 16) || !aligned(u, 16) ||
        !aligned(codes, 8) || !aligned(rho, 4))
        return SLORA_EINVAL;
    const size_t e = res_dtype == SLORA_DTYPE_F32 ? 4 : 2;
    const size_t moved = (size_t)T * d * (2 + (res ? e : 0) + (h ? e : 0) + (u ? 2 : 0) + (codes ? 1 : 0));
    const FwdCall c = {T, d, (const bf16 *)x, (size_t)ldx, res, (const bf16 *)gamma, eps, h, (bf16 *)u, (size_t)ldu,
                       (unsigned char *)codes, (unsigned char *)scales, rho, stream_results(moved), (hipStream_t)stream};
    if (!res) by_width<0>(c);
    else if (res_dtype == SLORA_DTYPE_BF16) by_width<1>(c);
    else by_width<2>(c);
    SL_CHECK_LAUNCH("rmsnorm_fwd");
    return SLORA_OK;
}

size_t slora_rmsnorm_bwd_ws_bytes(int32_t T, int32_t d)
{
    if (T < 0 || T >= RN_MAXT || d <= 0 || d > RN_MAXD || d % 8) return 0;
    const size_t n = 4 * (size_t)bwd_blocks(T < 1 ? 1 : T, d, true) * d;
    return (n + 255) & ~(size_t)255;
}

int slora_rmsnorm_bwd(int32_t T, int32_t d, int32_t res_dtype, const void *du, int64_t lddu, const void *h,
                      const float *rho, const void *gamma, const void *dres, void *dh, void *dx, int64_t lddx,
                      float *dgamma, void *ws, size_t ws_bytes, void *stream)
{
    if (T < 0 || T >= RN_MAXT || d <= 0 || d > RN_MAXD || d % 8) return SLORA_EINVAL;
    if (res_dtype != SLORA_DTYPE_F32 && res_dtype != SLORA_DTYPE_BF16) return SLORA_EINVAL;
    if (!aligned(dgamma, 4)) return SLORA_EINVAL;
    if (T == 0) return dgamma ? launch_fill_zero(dgamma, 4 * (size_t)d, (hipStream_t)stream) : SLORA_OK;
    if (!du || !h || !rho || !gamma || (!dh && !dx) || (dgamma && !ws)) return SLORA_EINVAL;
    if (!stride_ok(lddu, d) || (dx && !stride_ok(lddx, d))) return SLORA_EINVAL;
    if (!aligned(du, 16) || !aligned(h, 16) || !aligned(rho, 4) || !aligned(gamma, 16) || !aligned(dres, 16) ||
        !aligned(dh, 16) || !aligned(dx, 16) || (dgamma && !aligned(ws, 256)))
        return SLORA_EINVAL;
    if (dgamma && ws_bytes < slora_rmsnorm_bwd_ws_bytes(T, d)) return SLORA_ENOSPC;
    const hipStream_t st = (hipStream_t)stream;
    float *part = dgamma ? (float *)ws : nullptr;
    const int blocks = bwd_blocks(T, d, dgamma != nullptr);
    const size_t e = res_dtype == SLORA_DTYPE_F32 ? 4 : 2;
    const size_t moved = (size_t)T * d * (2 + e + (dres ? e : 0) + (dh ? e : 0) + (dx ? 2 : 0));
    const BwdCall c = {T, d, (const bf16 *)du, (size_t)lddu, h, rho, (const bf16 *)gamma, dres, dh, (bf16 *)dx, (size_t)lddx, part,
                       blocks, stream_results(moved), st};
    if (res_dtype == SLORA_DTYPE_BF16) by_width<1>(c);
    else by_width<2>(c);
    SL_CHECK_LAUNCH("rmsnorm_bwd");
    if (dgamma) {
        hipLaunchKernelGGL(rmsnorm_dgamma_kernel, dim3((d + 15) / 16), dim3(1024), 0, st, part, blocks, d, dgamma);
        SL_CHECK_LAUNCH("rmsnorm_dgamma");
    }
    return SLORA_OK;
}

}  // extern "C"
