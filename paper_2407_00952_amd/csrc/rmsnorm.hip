// Root-mean-square norm with the residual's addition, its result in bf16, in MXFP8 or both, and its backward.
//
//   s = x + res,  rho = 1 / sqrt(mean(s^2) + eps),  u = gamma s rho
//   dh = dres + rho (gamma du - h rho m),  m = mean(gamma du h rho),  dgamma = sum_t du h rho
//
// Both are bound by HBM: every tensor is read or written once, a row stays in registers between its sum and its result.  A row of
// up to 2048 columns belongs to one wave (4 rows to a block), longer ones to a block of 4 or 8 waves; a lane holds 8 neighbouring
// columns of each chunk of 512, so that bf16 moves 16 bytes a lane and a block of 32 columns of the MXFP8 result is 4 lanes.  Columns
// past the row are loaded from its start instead and counted as zero: no branch stands between the loads of a row.
#include "../../include/slora.h"
#include "common.h"
#include "mx_codec.h"

namespace {

constexpr int RN_MAXD = 16384;
constexpr int RN_MAX_PARTS = 1024;       // partial sums of dgamma

template <int RES> struct ResT { typedef float type; };
template <> struct ResT<1> { typedef bf16 type; };

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
__device__ __forceinline__ bf16x8 pack8(const float (&v)[8])
{
    bf16x8 t;
#pragma unroll
    for (int i = 0; i < 8; ++i) t[i] = f2bf(v[i]);
    return t;
}
__device__ __forceinline__ void store8(bf16 *p, const float (&v)[8]) { *(bf16x8 *)p = pack8(v); }
__device__ __forceinline__ void store8(float *p, const float (&v)[8])
{
    *(f32x4 *)p = f32x4{v[0], v[1], v[2], v[3]};
    *(f32x4 *)(p + 4) = f32x4{v[4], v[5], v[6], v[7]};
}

// sum over the TPR threads of a row; every thread of the block calls it
template <int TPR>
__device__ __forceinline__ float row_sum(float v, float *red)
{
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

// MXFP8 of 8 bf16 values a lane, blocks of 4 neighbouring lanes; every lane of the wave calls it
__device__ __forceinline__ void mx_store8(bf16x8 o, bool valid, int lane, unsigned char *q_row, unsigned char *s_row, int col)
{
    union { bf16x8 v; unsigned w[4]; } b;
    b.v = o;
    unsigned mag = 0u;
#pragma unroll
    for (int i = 0; i < 4; ++i) mag = max(mag, max(b.w[i] & 0x7FFFu, (b.w[i] >> 16) & 0x7FFFu));
    mag = max(mag, (unsigned)__shfl_xor((int)mag, 1, 64));
    mag = max(mag, (unsigned)__shfl_xor((int)mag, 2, 64));
    if (!valid) return;
    const int sc = mx_scale_code(mag);
    unsigned q[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) q[i] = mx_encode_pair_bf16(b.w[i] & 0xFFFFu, b.w[i] >> 16, sc);
    uint2 c;
    c.x = q[0] | (q[1] << 16);
    c.y = q[2] | (q[3] << 16);
    *(uint2 *)(q_row + col) = c;
    if ((lane & 3) == 0) s_row[col >> 5] = (unsigned char)sc;
}

// RES: 0 no residual, 1 bf16, 2 fp32.  NC chunks of 8 columns a thread, TPR threads a row.
template <int RES, int NC, int TPR>
__global__ __launch_bounds__(TPR < 256 ? 256 : TPR) void rmsnorm_fwd_kernel(
    int T, int d, const bf16 *x, size_t ldx, const typename ResT<RES>::type *res, const bf16 *__restrict__ gamma, float eps,
    typename ResT<RES>::type *h, bf16 *u, size_t ldu, unsigned char *__restrict__ codes, unsigned char *__restrict__ scales,
    float *__restrict__ rho_out)
{
    __shared__ float red[TPR / 64];
    constexpr int RPB = TPR < 256 ? 256 / TPR : 1;
    const int lane = threadIdx.x & 63, rt = threadIdx.x % TPR;
    const int row = blockIdx.x * RPB + threadIdx.x / TPR;
    if (row >= T) return;                // whole waves, and whole blocks where they share a row
    float s[NC][8], g[NC][8], q = 0.f;
    bool in[NC];
#pragma unroll
    for (int c = 0; c < NC; ++c) {
        const int col = (c * TPR + rt) * 8;
        in[c] = col < d;
        load8(x + row * ldx + (in[c] ? col : 0), s[c]);
    }
    if (RES) {
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            const int col = (c * TPR + rt) * 8;
            float r[8];
            load8(res + (size_t)row * d + (in[c] ? col : 0), r);
#pragma unroll
            for (int i = 0; i < 8; ++i) s[c][i] += r[i];
        }
    }
#pragma unroll
    for (int c = 0; c < NC; ++c) load8(gamma + (in[c] ? (c * TPR + rt) * 8 : 0), g[c]);
#pragma unroll
    for (int c = 0; c < NC; ++c)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            s[c][i] = in[c] ? s[c][i] : 0.f;
            q = fmaf(s[c][i], s[c][i], q);
        }
    const float rho = rsqrtf(row_sum<TPR>(q, red) / (float)d + eps);
    if (rho_out && rt == 0) rho_out[row] = rho;
#pragma unroll
    for (int c = 0; c < NC; ++c) {
        const int col = (c * TPR + rt) * 8;
        if (RES && h && in[c]) store8(h + (size_t)row * d + col, s[c]);
        float w[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) w[i] = s[c][i] * rho * g[c][i];
        const bf16x8 o = pack8(w);
        if (u && in[c]) *(bf16x8 *)(u + row * ldu + col) = o;
        if (codes) mx_store8(o, in[c], lane, codes + (size_t)row * d, scales + (size_t)row * (d >> 5), col);
    }
}

// Blocks walk the rows with the grid's stride, so that each keeps one partial sum of dgamma in registers; part [blocks][d], or null.
template <int RES, int NC, int TPR>
__global__ __launch_bounds__(TPR < 256 ? 256 : TPR) void rmsnorm_bwd_kernel(
    int T, int d, const bf16 *__restrict__ du, size_t lddu, const typename ResT<RES>::type *__restrict__ h,
    const float *__restrict__ rho_in, const bf16 *__restrict__ gamma, const typename ResT<RES>::type *dres,
    typename ResT<RES>::type *dh, bf16 *__restrict__ dx, size_t lddx, float *__restrict__ part)
{
    constexpr int RPB = TPR < 256 ? 256 / TPR : 1;
    __shared__ float red[TPR / 64];
    __shared__ float acc[RPB > 1 ? NC * 512 : 1];
    const int rt = threadIdx.x % TPR, sub = threadIdx.x / TPR;
    float g[NC][8], dg[NC][8];
    bool in[NC];
#pragma unroll
    for (int c = 0; c < NC; ++c) {
        const int col = (c * TPR + rt) * 8;
        in[c] = col < d;
        load8(gamma + (in[c] ? col : 0), g[c]);
#pragma unroll
        for (int i = 0; i < 8; ++i) dg[c][i] = 0.f;
    }
    for (long long r0 = (long long)blockIdx.x * RPB; r0 < T; r0 += (long long)gridDim.x * RPB) {
        const bool on = r0 + sub < T;
        const int row = on ? (int)r0 + sub : T - 1;      // (a row past the end repeats the last one and stores nothing)
        float v[NC][8], a[NC][8], r[NC][8];
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            const int col = in[c] ? (c * TPR + rt) * 8 : 0;
            load8(du + row * lddu + col, a[c]);
            load8(h + (size_t)row * d + col, v[c]);
        }
        const float rho = rho_in[row];
        if (dres) {
#pragma unroll
            for (int c = 0; c < NC; ++c) load8(dres + (size_t)row * d + (in[c] ? (c * TPR + rt) * 8 : 0), r[c]);
        } else {
#pragma unroll
            for (int c = 0; c < NC; ++c)
#pragma unroll
                for (int i = 0; i < 8; ++i) r[c][i] = 0.f;
        }
        float m = 0.f;
#pragma unroll
        for (int c = 0; c < NC; ++c)
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                v[c][i] *= rho;                          // h rho
                const float t = on && in[c] ? a[c][i] * v[c][i] : 0.f;
                dg[c][i] += t;
                m = fmaf(t, g[c][i], m);
            }
        m = row_sum<TPR>(m, red) / (float)d;
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            const int col = (c * TPR + rt) * 8;
            float o[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) o[i] = fmaf(rho, fmaf(a[c][i], g[c][i], -v[c][i] * m), r[c][i]);
            if (on && in[c]) {
                if (dh) store8(dh + (size_t)row * d + col, o);
                if (dx) store8(dx + row * lddx + col, o);
            }
        }
    }
    if (!part) return;
    if (RPB > 1) {                                       // the block's waves one after the other: a fixed order
        for (int w = 0; w < RPB; ++w) {
            if (sub == w) {
#pragma unroll
                for (int c = 0; c < NC; ++c)
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        float *p = acc + (c * TPR + rt) * 8 + i;
                        *p = w ? *p + dg[c][i] : dg[c][i];
                    }
            }
            __syncthreads();
        }
        for (int col = threadIdx.x; col < d; col += blockDim.x) part[(size_t)blockIdx.x * d + col] = acc[col];
    } else {
#pragma unroll
        for (int c = 0; c < NC; ++c)
            if (in[c]) store8(part + (size_t)blockIdx.x * d + (c * TPR + rt) * 8, dg[c]);
    }
}

// dgamma = the partial sums in order: 64 columns a block, 16 waves with a sixteenth of the partial sums each
__global__ __launch_bounds__(1024) void rmsnorm_dgamma_kernel(const float *__restrict__ part, int n, int d, float *__restrict__ dgamma)
{
    __shared__ float red[16][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, col = blockIdx.x * 64 + lane;
    const int per = (n + 15) / 16;
    float s = 0.f;
    if (col < d)
        for (int i = wave * per; i < min(n, wave * per + per); ++i) s += part[(size_t)i * d + col];
    red[wave][lane] = s;
    __syncthreads();
    if (wave == 0 && col < d) {
        for (int w = 1; w < 16; ++w) s += red[w][lane];
        dgamma[col] = s;
    }
}

inline int threads_per_row(int d) { return d <= 2048 ? 64 : d <= 8192 ? 256 : 512; }
inline int rows_per_block(int d) { return d <= 2048 ? 4 : 1; }

// Blocks of the backward: enough to fill the chip several times over, each with rows enough that its partial sum of dgamma
// (written once, read once) is small beside them
inline int bwd_blocks(int T, int d)
{
    const int blocks = (T + rows_per_block(d) - 1) / rows_per_block(d);
    return blocks < RN_MAX_PARTS ? blocks : RN_MAX_PARTS;
}

struct FwdCall {
    int T, d; const bf16 *x; size_t ldx; const void *res; const bf16 *gamma; float eps; void *h; bf16 *u; size_t ldu;
    unsigned char *codes, *scales; float *rho; hipStream_t st;
    template <int RES, int NC, int TPR> void go() const
    {
        typedef typename ResT<RES>::type R;
        const int rpb = TPR < 256 ? 256 / TPR : 1;
        hipLaunchKernelGGL((rmsnorm_fwd_kernel<RES, NC, TPR>), dim3((T + rpb - 1) / rpb), dim3(TPR < 256 ? 256 : TPR), 0, st, T, d, x, ldx,
                           (const R *)res, gamma, eps, (R *)h, u, ldu, codes, scales, rho);
    }
};
struct BwdCall {
    int T, d; const bf16 *du; size_t lddu; const void *h; const float *rho; const bf16 *gamma; const void *dres; void *dh; bf16 *dx;
    size_t lddx; float *part; int blocks; hipStream_t st;
    template <int RES, int NC, int TPR> void go() const
    {
        typedef typename ResT<RES>::type R;
        hipLaunchKernelGGL((rmsnorm_bwd_kernel<RES, NC, TPR>), dim3(blocks), dim3(TPR < 256 ? 256 : TPR), 0, st, T, d, du, lddu, (const R *)h,
                           rho, gamma, (const R *)dres, (R *)dh, dx, lddx, part);
    }
};

// the kernel of a width: as few threads and chunks as hold a row
template <int RES, class Call>
void by_width(const Call &c)
{
    const int d = c.d;
    if (d <= 512) c.template go<RES, 1, 64>();
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
    if (T < 0 || T > (1 << 28) || d <= 0 || d > RN_MAXD || d % 8 || !(eps >= 0.f)) return SLORA_EINVAL;
    if (res_dtype != SLORA_DTYPE_F32 && res_dtype != SLORA_DTYPE_BF16) return SLORA_EINVAL;
    if (!x || !gamma || (!u && !codes) || !codes != !scales || (h && !res)) return SLORA_EINVAL;
    if (!stride_ok(ldx, d) || (u && !stride_ok(ldu, d)) || (codes && d % 32)) return SLORA_EINVAL;
    if (!aligned(x, 16) || !aligned(res, 16) || !aligned(gamma, 16) || !aligned(h, 16) || !aligned(u, 16) ||
        !aligned(codes, 8) || !aligned(rho, 4))
        return SLORA_EINVAL;
    if (T == 0) return SLORA_OK;
    const FwdCall c = {T, d, (const bf16 *)x, (size_t)ldx, res, (const bf16 *)gamma, eps, h, (bf16 *)u, (size_t)ldu,
                       (unsigned char *)codes, (unsigned char *)scales, rho, (hipStream_t)stream};
    if (!res) by_width<0>(c);
    else if (res_dtype == SLORA_DTYPE_BF16) by_width<1>(c);
    else by_width<2>(c);
    SL_CHECK_LAUNCH("rmsnorm_fwd");
    return SLORA_OK;
}

size_t slora_rmsnorm_bwd_ws_bytes(int32_t T, int32_t d)
{
    if (T < 0 || T > (1 << 28) || d <= 0 || d > RN_MAXD || d % 8) return 0;
    const size_t n = 4 * (size_t)bwd_blocks(T < 1 ? 1 : T, d) * d;
    return (n + 255) & ~(size_t)255;
}

int slora_rmsnorm_bwd(int32_t T, int32_t d, int32_t res_dtype, const void *du, int64_t lddu, const void *h,
                      const float *rho, const void *gamma, const void *dres, void *dh, void *dx, int64_t lddx,
                      float *dgamma, void *ws, size_t ws_bytes, void *stream)
{
    if (T < 0 || T > (1 << 28) || d <= 0 || d > RN_MAXD || d % 8) return SLORA_EINVAL;
    if (res_dtype != SLORA_DTYPE_F32 && res_dtype != SLORA_DTYPE_BF16) return SLORA_EINVAL;
    if (!du || !h || !rho || !gamma || (!dh && !dx) || (dgamma && !ws)) return SLORA_EINVAL;
    if (!stride_ok(lddu, d) || (dx && !stride_ok(lddx, d))) return SLORA_EINVAL;
    if (!aligned(du, 16) || !aligned(h, 16) || !aligned(rho, 4) || !aligned(gamma, 16) || !aligned(dres, 16) ||
        !aligned(dh, 16) || !aligned(dx, 16) || !aligned(dgamma, 4) || (dgamma && !aligned(ws, 256)))
        return SLORA_EINVAL;
    if (dgamma && ws_bytes < slora_rmsnorm_bwd_ws_bytes(T, d)) return SLORA_ENOSPC;
    const hipStream_t st = (hipStream_t)stream;
    float *part = dgamma ? (float *)ws : nullptr;
    const int blocks = T ? bwd_blocks(T, d) : 0;
    if (T) {
        const BwdCall c = {T, d, (const bf16 *)du, (size_t)lddu, h, rho, (const bf16 *)gamma, dres, dh, (bf16 *)dx, (size_t)lddx, part,
                           blocks, st};
        if (res_dtype == SLORA_DTYPE_BF16) by_width<1>(c);
        else by_width<2>(c);
        SL_CHECK_LAUNCH("rmsnorm_bwd");
    }
    if (dgamma) {
        hipLaunchKernelGGL(rmsnorm_dgamma_kernel, dim3((d + 63) / 64), dim3(1024), 0, st, part, blocks, d, dgamma);
        SL_CHECK_LAUNCH("rmsnorm_dgamma");
    }
    return SLORA_OK;
}

}  // extern "C"
