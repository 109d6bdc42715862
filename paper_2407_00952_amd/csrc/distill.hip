// Distillation from a teacher's top logits, with the labels' cross-entropy beside it.
//
//   p = softmax(t / tau) over a row's used entries,  q = softmax(z / tau),  q1 = softmax(z) over the vocabulary
//   loss_t = kd tau^2 sum_j p_j (log p_j - log q[id_j]) + ce (logsumexp(z) - z[label])
//   dz = w_t (kd tau (q - sum_j p_j e_{id_j}) + ce (q1 - e_label))
//
// One block per row.  Rows that the block's registers hold (packed) are read once: maximum, sums of exponentials and gradient from
// there.  Longer ones are read twice: running maximum and sums in one pass, the gradient in a second.  The gradient of every column
// is stored as that of the two softmaxes, then the few columns of the teacher's entries and of the label again.  Bound by HBM: the
// logits once, the gradient once.
//
// A row may start anywhere (a dense [T, 50257] tensor has rows at every alignment): the 16-byte pieces that lie whole in the row
// move as such, the up to 7 elements before the first and behind the last one by themselves.
#include "../../include/slora.h"
#include "common.h"
#include "stream_store.h"

namespace {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

__device__ __forceinline__ float to_f(bf16 v) { return bf2f(v); }
__device__ __forceinline__ float to_f(float v) { return v; }
__device__ __forceinline__ void from_f(bf16 &o, float v) { o = f2bf(v); }
__device__ __forceinline__ void from_f(float &o, float v) { o = v; }

template <class E> struct Piece { typedef bf16x8 type; static constexpr int n = 8; };
template <> struct Piece<float> { typedef f32x4 type; static constexpr int n = 4; };

__device__ __forceinline__ float wave_max(float v)
{
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor(v, o, 64));
    return v;
}

// Sum (or maximum) over the block of values that wave_sum (wave_max) has brought together in each wave; `red` belongs to this call alone.
template <int WAVES> __device__ __forceinline__ void put_wave(float v, float *red)
{
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
}
// a value that is the same in all lanes, in a scalar register
__device__ __forceinline__ float uniform(float v) { return __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(v))); }
template <int WAVES> __device__ __forceinline__ float all_waves(const float *red, bool is_max)
{
    float r = red[0];
#pragma unroll
    for (int i = 1; i < WAVES; ++i) r = is_max ? fmaxf(r, red[i]) : r + red[i];
    return uniform(r);
}

// The compiler may not know that p is what it was: it unpacks p again in the next pass instead of keeping the unpacked values, for
// which there are no registers.
template <class P>
__device__ __forceinline__ void forget(P &p)
{
    union { P v; unsigned w[4]; } b;
    b.v = p;
#pragma unroll
    for (int i = 0; i < 4; ++i) asm volatile("" : "+v"(b.w[i]));
    p = b.v;
}

struct DistillArgs {
    int T, V, k;                             // k 0: no teacher
    size_t ldl, ldd;
    const int *ids; const float *top;
    float tau, kd;
    const int *labels; float ce;             // labels null: no second term
    const float *w;                          // null: 1 / T
    float *loss_tok;
};

// E: type of the logits.  POW: 1 where one softmax serves both terms (tau = 1, or no labels).  Else the second one's exponentials are
// e^((z - M)) = (e^((z - M) / tau))^tau: products for tau = 2 and 4 (POW = tau), exponentials of their own otherwise (POW 0); a vector
// instruction takes 4 cycles, an exponential 16, and the two passes over 50257 columns are 0.43 ms of instructions with products,
// 0.71 with exponentials, beside 0.6 of memory time.  THR threads, each with one of the teacher's entries, hold CH pieces of the row
// each; CH 0: the row is read twice.
// [16384, 50257] bf16, 64 entries and labels, tau 2, a quarter of the rows of weight 0: 971 us with every row read twice and two
// exponentials, 721 with products, 620 with registers too (2.88 GB: 4.7 TB/s, a copy reaches 4.9), 689 with tau 1.5; [2053, 32003] fp32
// 132 -> 103 us.  The loss alone takes 434 us.  Values that spill cost more than anything: at 55 spilled registers 1397 us.
template <class E, int POW, int THR, int CH, bool STREAM>
__global__ __launch_bounds__(THR, 8) void distill_row_kernel(DistillArgs a, const E *logits, E *dlogits)
{
    typedef typename Piece<E>::type P;
    constexpr bool TWO = POW != 1;
    constexpr int N = Piece<E>::n, WAVES = THR / 64, HELD = CH ? CH : 1;
    __shared__ float red_m[WAVES], red_t[WAVES], red_s[WAVES], red_s1[WAVES], red_ts[WAVES], red_kl[WAVES];
    __shared__ __align__(16) int id_s[THR];
    __shared__ float p_s[THR], z_s[THR];     // the teacher's logit, then its probability; the student's logit there
    __shared__ int taught_s, label_hit_s;
    const int tid = threadIdx.x, row = blockIdx.x, V = a.V;
    const float w = a.w ? a.w[row] : 1.0f / (float)a.T;
    const E *z = logits + (size_t)row * a.ldl;
    E *dz = dlogits ? dlogits + (size_t)row * a.ldd : nullptr;
    const int head = min(V, (int)((16 - ((uintptr_t)z & 15)) & 15) / (int)sizeof(E));
    const int pieces = (V - head) / N, tail0 = head + pieces * N;
    const E *zp = z + head;
    // the element by itself of this thread: one before the first piece or behind the last
    const int lone = tid < head ? tid : tid - head < V - tail0 ? tail0 + tid - head : -1;
    if (w == 0.f) {
        if (tid == 0) a.loss_tok[row] = 0.f;
        if (dz) {
            P zeros;
#pragma unroll
            for (int i = 0; i < N; ++i) zeros[i] = (E)0.f;
            const int zhead = min(V, (int)((16 - ((uintptr_t)dz & 15)) & 15) / (int)sizeof(E)), zpieces = (V - zhead) / N;
            for (int c = tid; c < zpieces; c += THR) store_result<STREAM>((P *)(dz + zhead) + c, zeros);
            const int ztail = zhead + zpieces * N;
            if (tid < zhead) dz[tid] = (E)0.f;
            else if (tid - zhead < V - ztail) dz[ztail + tid - zhead] = (E)0.f;
        }
        return;
    }
    const unsigned tid16 = tid * 16u;    // (scalar bases and one offset: no registers for 64-bit addresses)
    P held[HELD];                        // (pieces past the row: masked words, which add nothing)
    if (CH) {
#pragma unroll
        for (int c = 0; c < CH; ++c) {
#pragma unroll
            for (int i = 0; i < N; ++i) held[c][i] = (E)-INFINITY;
            if (tid + c * THR < pieces) held[c] = *(const P *)((const char *)(zp + c * THR * N) + tid16);
        }
    }
    const float lone_v = lone >= 0 ? to_f(z[lone]) : -INFINITY;
    const int label = a.labels ? a.labels[row] : -1;
    const bool labeled = label >= 0 && label < V;
    const float zl = labeled ? uniform(to_f(z[label])) : 0.f;

    // the teacher's entry of this thread: its id, its logit, the student's logit there
    if (tid == 0) taught_s = label_hit_s = 0;
    __syncthreads();
    int id = -1;
    float t = -INFINITY;
    if (tid < a.k) {
        id = a.ids[(size_t)row * a.k + tid];
        t = a.top[(size_t)row * a.k + tid];
        if (id < 0 || id >= V || t == -INFINITY) id = -1;
        if (id >= 0) z_s[tid] = to_f(z[id]);
        p_s[tid] = t;
    }
    id_s[tid] = id;
    if (id >= 0) taught_s = 1;
    if (id >= 0 && id == label) label_hit_s = 1;
    {
        const float tm = wave_max(id >= 0 ? t : -INFINITY);
        put_wave<WAVES>(tm, red_t);
    }
    __syncthreads();
    const bool taught = __builtin_amdgcn_readfirstlane(taught_s) != 0;
    const bool label_left = labeled && __builtin_amdgcn_readfirstlane(label_hit_s) == 0;
    const float tmax = all_waves<WAVES>(red_t, true);
    // the entry's column is stored by the first thread that holds its id: col, or -1; twice: others hold it too
    bool first = id >= 0, twice = false;
    if (__ballot(first) != 0) {
        for (int i = 0; i < a.k; i += 4) {
            const int4 o = *(const int4 *)(id_s + i);
            const bool e0 = o.x == id, e1 = o.y == id, e2 = o.z == id, e3 = o.w == id;
            first = first && !((e0 && i < tid) || (e1 && i + 1 < tid) || (e2 && i + 2 < tid) || (e3 && i + 3 < tid));
            twice = twice || (e0 && i != tid) || (e1 && i + 1 != tid) || (e2 && i + 2 != tid) || (e3 && i + 3 != tid);
        }
    }

    if (!first && id >= 0) id = -2 - id;                 // (an entry, not one that stores)

    // maximum and sums of exponentials
    const float at = kLog2e / a.tau;
    float m = lone_v, s = 0.f, s1 = 0.f;
    auto second = [&](float e, float arg) {              // the second softmax's exponential, from the first one's or from z - M
        return POW == 2 ? e * e : POW == 4 ? (e * e) * (e * e) : __builtin_amdgcn_exp2f(arg * kLog2e);
    };
    auto add = [&](float v, float base) {
        const float e = __builtin_amdgcn_exp2f((v - base) * at);
        s += e;
        if (POW == 2) s1 = fmaf(e, e, s1);
        else if (TWO) s1 += second(e, v - base);
    };
    if (CH) {
#pragma unroll
        for (int c = 0; c < CH; ++c)
#pragma unroll
            for (int i = 0; i < N; ++i) m = fmaxf(m, to_f(held[c][i]));
    } else {
        // the sums relative to the thread's own maximum so far
        if (lone >= 0) add(lone_v, lone_v == -INFINITY ? 0.f : lone_v);
        for (int c = tid; c < pieces; c += THR) {
            const P q = *(const P *)(zp + (size_t)c * N);
            float mx = to_f(q[0]);
#pragma unroll
            for (int i = 1; i < N; ++i) mx = fmaxf(mx, to_f(q[i]));
            if (mx > m) {
                const float f = m - mx;                  // (-inf the first time)
                s *= __builtin_amdgcn_exp2f(f * at);
                if (TWO) s1 *= __builtin_amdgcn_exp2f(f * kLog2e);
                m = mx;
            }
            const float base = m == -INFINITY ? 0.f : m; // (nothing but masked words so far: they add nothing)
#pragma unroll
            for (int i = 0; i < N; ++i) add(to_f(q[i]), base);
        }
    }
    put_wave<WAVES>(wave_max(m), red_m);
    __syncthreads();
    const float M = all_waves<WAVES>(red_m, true);
    if (CH) {
#pragma unroll
        for (int c = 0; c < CH; ++c) forget(held[c]);
        if (lone >= 0) add(lone_v, M);
#pragma unroll
        for (int c = 0; c < CH; ++c) {
#pragma unroll
            for (int i = 0; i < N; ++i) add(to_f(held[c][i]), M);
            if (TWO) asm volatile("" : "+v"(s1));
            asm volatile("" : "+v"(s));                  // (one piece after the other: else the compiler keeps all exponentials for s1)
            __builtin_amdgcn_sched_barrier(0);
        }
#pragma unroll
        for (int c = 0; c < CH; ++c) forget(held[c]);
    } else {
        const float f = m == -INFINITY ? 0.f : m - M;
        s *= __builtin_amdgcn_exp2f(f * at);
        if (TWO) s1 *= __builtin_amdgcn_exp2f(f * kLog2e);
    }
    put_wave<WAVES>(wave_sum(s), red_s);
    if (TWO) put_wave<WAVES>(wave_sum(s1), red_s1);
    put_wave<WAVES>(wave_sum(id != -1 ? __builtin_amdgcn_exp2f((p_s[tid] - tmax) * at) : 0.f), red_ts);
    __syncthreads();
    s = all_waves<WAVES>(red_s, false);
    s1 = TWO ? all_waves<WAVES>(red_s1, false) : s;
    const float log_s = uniform(__builtin_amdgcn_logf(s) * kLn2), log_s1 = TWO ? uniform(__builtin_amdgcn_logf(s1) * kLn2) : log_s;
    const float log_t = uniform(__builtin_amdgcn_logf(all_waves<WAVES>(red_ts, false)) * kLn2);

    // the teacher's probability and the loss
    float kl = 0.f;
    if (id != -1) {
        const float lt = (p_s[tid] - tmax) / a.tau - log_t, lq = (z_s[tid] - M) / a.tau - log_s;
        const float p = __builtin_amdgcn_exp2f(lt * kLog2e);
        if (p != 0.f) kl = p * (lt - lq);
        p_s[tid] = p;
    }
    put_wave<WAVES>(wave_sum(kl), red_kl);
    __syncthreads();                     // (also: whoever reads z elsewhere than in its own pieces has done so; dlogits may be the logits)
    if (tid == 0)
        a.loss_tok[row] = (taught ? a.kd * a.tau * a.tau * all_waves<WAVES>(red_kl, false) : 0.f) +
                          (labeled ? a.ce * ((M - zl) + log_s1) : 0.f);
    if (!dz) return;

    const float g1 = uniform(labeled ? w * a.ce / s1 : 0.f);
    const float g = uniform((taught ? w * a.kd * a.tau / s : 0.f) + (TWO ? 0.f : g1));
    auto grad = [&](float v) {
        const float e = __builtin_amdgcn_exp2f((v - M) * at);
        return POW == 2 ? e * fmaf(g1, e, g) : TWO ? fmaf(g1, second(e, v - M), g * e) : g * e;
    };
    // the gradient's pieces are aligned as the logits' are, or it is stored by elements
    const bool same = (((uintptr_t)dz ^ (uintptr_t)z) & 15) == 0;
    auto put = [&](E *base, unsigned off, P q) {
        P o;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            E e;
            from_f(e, grad(to_f(q[i])));
            o[i] = e;
        }
        E *to = (E *)((char *)base + off);
        if (same) store_result<STREAM>((P *)to, o);
        else
#pragma unroll
            for (int i = 0; i < N; ++i) to[i] = o[i];
    };
    if (CH) {
#pragma unroll
        for (int c = 0; c < CH; ++c)
            if (tid + c * THR < pieces) {
                put(dz + head + c * THR * N, tid16, held[c]);
                __builtin_amdgcn_sched_barrier(0);
            }
    } else {
        for (int c = tid; c < pieces; c += THR) put(dz + head, c * 16u, *(const P *)(zp + c * N));
    }
    if (lone >= 0) from_f(dz[lone], grad(lone_v));
    __syncthreads();
    if (id >= 0) {
        float p = p_s[tid];
        if (twice)                                       // an id given more than once: its probabilities together
            for (int i = tid + 1; i < a.k; ++i) p += id_s[i] == id ? p_s[i] : 0.f;
        from_f(dz[id], grad(z_s[tid]) - w * a.kd * a.tau * p - (labeled && id == label ? w * a.ce : 0.f));
    }
    if (tid == 0 && label_left) from_f(dz[label], grad(zl) - w * a.ce);
}

// loss = sum_t w_t loss_tok[t]: one block, a fixed order, sums in 64 bits
__global__ __launch_bounds__(1024) void distill_mean_kernel(const float *__restrict__ loss_tok, const float *__restrict__ w, int T,
                                                            float *__restrict__ loss)
{
    __shared__ double red[1024];
    double s = 0.0;
    for (int i = threadIdx.x; i < T; i += 1024 * 8) {    // eight rows in flight
        float v[8], wi[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const int at = min(i + k * 1024, T - 1);
            v[k] = loss_tok[at];
            wi[k] = w ? w[at] : 1.0f / (float)T;
        }
#pragma unroll
        for (int k = 0; k < 8; ++k) s += i + k * 1024 < T && wi[k] != 0.f ? (double)wi[k] * (double)v[k] : 0.0;
    }
    red[threadIdx.x] = s;
    __syncthreads();
    for (int o = 512; o > 0; o >>= 1) {
        if (threadIdx.x < o) red[threadIdx.x] += red[threadIdx.x + o];
        __syncthreads();
    }
    if (threadIdx.x == 0) *loss = (float)red[0];
}

// The form of a row: the fewest threads and registers that hold it and the teacher's entries, or none.  Short rows on few threads, most of
// whose 1024 would only wait at the sums: [16384, 8003] bf16 103 us, on 1024 threads 394.  Rows of up to 8 pieces a thread, held / read twice
// (the second time mostly from the caches), gradient and loss alone, us: [16384, 50257] bf16 621 / 721, 434 / 385; [2048, 32003] fp32
// 90 / 104, 57 / 53; [16384, 16003] bf16 458 / 380, 374 / 284.  Longer ones are read twice: 16 pieces would leave one row to a CU instead of two
// ([4096, 70001] bf16 375 / 251, 258 / 125; [4096, 128256] bf16 499 / 420, 312 / 178; [4096, 50257] fp32 351 / 340, 223 / 146).
// [4096, 151936] bf16: 501 us, the loss alone 194.
template <class E, int POW, bool STREAM>
void launch_form(const DistillArgs &a, const E *z, E *dz, hipStream_t st)
{
    const int pieces = a.V / Piece<E>::n;                // (the most: rows that start aligned)
    if (pieces <= 256 * 4 && a.k <= 256)
        hipLaunchKernelGGL((distill_row_kernel<E, POW, 256, 4, STREAM>), dim3(a.T), dim3(256), 0, st, a, z, dz);
    else if (pieces <= 1024 * 8)
        hipLaunchKernelGGL((distill_row_kernel<E, POW, 1024, 8, STREAM>), dim3(a.T), dim3(1024), 0, st, a, z, dz);
    else
        hipLaunchKernelGGL((distill_row_kernel<E, POW, 1024, 0, STREAM>), dim3(a.T), dim3(1024), 0, st, a, z, dz);
}

template <class E, int POW>
void launch_pow(const DistillArgs &a, const E *z, E *dz, hipStream_t st)
{
    if (stream_results(sizeof(E) * (size_t)a.T * a.V * (dz ? 2 : 1))) launch_form<E, POW, true>(a, z, dz, st);
    else launch_form<E, POW, false>(a, z, dz, st);
}

template <class E>
void launch_rows(const DistillArgs &a, const void *logits, void *dlogits, hipStream_t st)
{
    const E *z = (const E *)logits;
    E *dz = (E *)dlogits;
    if (!a.labels || a.tau == 1.0f) launch_pow<E, 1>(a, z, dz, st);
    else if (a.tau == 2.0f) launch_pow<E, 2>(a, z, dz, st);
    else if (a.tau == 4.0f) launch_pow<E, 4>(a, z, dz, st);
    else launch_pow<E, 0>(a, z, dz, st);
}

inline bool aligned(const void *p, unsigned n) { return ((uintptr_t)p & (n - 1)) == 0; }

}  // namespace

extern "C" int slora_distill_loss(int32_t T, int32_t vocab, int32_t dtype, const void *logits, int64_t ldl, int32_t k,
                                  const int32_t *t_ids, const float *t_logits, float tau, float kd, const int32_t *labels,
                                  float ce, const float *row_weight, float *loss_tok, float *loss, void *dlogits,
                                  int64_t ldd, void *stream)
{
    // (a block of up to 1024 threads a row; a grid has fewer than 2^32)
    if (T <= 0 || T >= (1 << 22) || vocab <= 0 || vocab > (1 << 24) || k <= 0 || k > SLORA_MAX_TOP) return SLORA_EINVAL;
    if (dtype != SLORA_DTYPE_F32 && dtype != SLORA_DTYPE_BF16) return SLORA_EINVAL;
    if (!logits || !t_ids || !t_logits || !loss_tok || !loss) return SLORA_EINVAL;
    // (1 / tau and tau^2 are normal fp32 numbers, also with log2(e) beside them)
    if (!(tau >= 1e-15f) || !(tau <= 1e15f) || !(kd >= 0.f) || !(kd <= 1e30f) || !(ce >= 0.f) || !(ce <= 1e30f)) return SLORA_EINVAL;
    // (the loss's factor; 1e30 as fp32 rounds it, and tau = 1e15 with kd = 1, stay within)
    if ((double)kd * tau * tau > 1.0000001e30) return SLORA_EINVAL;
    if (ldl < vocab || ldl >= (1ll << 40) || (dlogits && (ldd < vocab || ldd >= (1ll << 40)))) return SLORA_EINVAL;
    if (dlogits == logits && ldd != ldl) return SLORA_EINVAL;
    const unsigned e = dtype == SLORA_DTYPE_F32 ? 4 : 2;
    if (!aligned(logits, e) || !aligned(dlogits, e) || !aligned(t_ids, 4) || !aligned(t_logits, 4) || !aligned(labels, 4) ||
        !aligned(row_weight, 4) || !aligned(loss_tok, 4) || !aligned(loss, 4))
        return SLORA_EINVAL;
    const hipStream_t st = (hipStream_t)stream;
    // a term of weight 0 takes no part: no entries (and one softmax, that of the logits as they are), no labels
    const bool taught = kd > 0.f;
    const DistillArgs a = {T, vocab, taught ? k : 0, (size_t)ldl, (size_t)ldd, t_ids, t_logits, taught ? tau : 1.0f, kd,
                           ce > 0.f ? labels : nullptr, ce, row_weight, loss_tok};
    if (dtype == SLORA_DTYPE_F32) launch_rows<float>(a, logits, dlogits, st);
    else launch_rows<bf16>(a, logits, dlogits, st);
    SL_CHECK_LAUNCH("distill_row");
    hipLaunchKernelGGL(distill_mean_kernel, dim3(1), dim3(1024), 0, st, loss_tok, row_weight, T, loss);
    SL_CHECK_LAUNCH("distill_mean");
    return SLORA_OK;
}
