// Distillation from a teacher's top logits, with the labels' cross-entropy beside it.
//
//   p = softmax(t / tau) over a row's used entries,  q = softmax(z / tau),  q1 = softmax(z) over the vocabulary
//   loss_t = kd tau^2 sum_j p_j (log p_j - log q[id_j]) + ce (logsumexp(z) - z[label])
//   dz = w_t (kd tau (q - sum_j p_j e_{id_j}) + ce (q1 - e_label))
//
// One block per row: the running maximum and the two sums of exponentials in one pass over the row, the gradient in a second one
// that writes every column, then the few columns of the teacher's entries and of the label again.  Bound by HBM: the
// logits once, the gradient once.
//
// A row may start anywhere (a dense [T, 50257] tensor has rows at every alignment): the 16-byte pieces that lie whole in the row
// move as such, the up to 7 elements before the first and behind the last one by themselves.
#include "../../include/slora.h"
#include "common.h"

namespace {

constexpr int DS_THR = 1024;
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

__device__ __forceinline__ float to_f(bf16 v) { return bf2f(v); }
__device__ __forceinline__ float to_f(float v) { return v; }
__device__ __forceinline__ void from_f(bf16 &o, float v) { o = f2bf(v); }
__device__ __forceinline__ void from_f(float &o, float v) { o = v; }

template <class E> struct Piece { typedef bf16x8 type; static constexpr int n = 8; };
template <> struct Piece<float> { typedef f32x4 type; static constexpr int n = 4; };

template <int THR>
__device__ __forceinline__ float block_max(float v, float *red)
{
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor(v, o, 64));
    __syncthreads();
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
    __syncthreads();
    float r = red[0];
#pragma unroll
    for (int i = 1; i < THR / 64; ++i) r = fmaxf(r, red[i]);
    return r;
}
template <int THR>
__device__ __forceinline__ float block_sum(float v, float *red)
{
    v = wave_sum(v);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
    __syncthreads();
    float r = red[0];
#pragma unroll
    for (int i = 1; i < THR / 64; ++i) r += red[i];
    return r;
}

struct DistillArgs {
    int T, V, k;
    size_t ldl, ldd;
    const int *ids; const float *top;
    float tau, kd;
    const int *labels; float ce;             // labels null: no second term
    const float *w;                          // null: 1 / T
    float *loss_tok;
};

// E: type of the logits.  TWO: the second term is there and tau is not 1 (its softmax needs sums of its own).
template <class E, bool TWO>
__global__ __launch_bounds__(DS_THR) void distill_row_kernel(DistillArgs a, const E *logits, E *dlogits)
{
    typedef typename Piece<E>::type P;
    constexpr int N = Piece<E>::n;
    __shared__ float red[DS_THR / 64];
    __shared__ int id_s[SLORA_MAX_TOP];
    __shared__ float p_s[SLORA_MAX_TOP];
    const int tid = threadIdx.x, row = blockIdx.x, V = a.V;
    const float w = a.w ? a.w[row] : 1.0f / (float)a.T;
    const E *z = logits + (size_t)row * a.ldl;
    E *dz = dlogits ? dlogits + (size_t)row * a.ldd : nullptr;
    const int head = min(V, (int)((16 - ((uintptr_t)z & 15)) & 15) / (int)sizeof(E));
    const int pieces = (V - head) / N, tail0 = head + pieces * N;
    // the element by itself of this thread: one before the first piece or behind the last
    const int lone = tid < head ? tid : tid - head < V - tail0 ? tail0 + tid - head : -1;
    const bool same = dz && (((uintptr_t)dz ^ (uintptr_t)z) & 15) == 0;      // the gradient's pieces are aligned as the logits' are
    if (w == 0.f) {
        if (tid == 0) a.loss_tok[row] = 0.f;
        if (dz) {
            E zero;
            from_f(zero, 0.f);
            for (int c = tid; c < V; c += DS_THR) dz[c] = zero;
        }
        return;
    }
    // the teacher's row
    const int label = a.labels ? a.labels[row] : -1;
    const bool labeled = label >= 0 && label < V;
    float tmax = -INFINITY;
    int any = 0;
    for (int j = tid; j < a.k; j += DS_THR) {
        const int id = a.ids[(size_t)row * a.k + j];
        const float t = a.top[(size_t)row * a.k + j];
        const bool used = id >= 0 && id < V && t != -INFINITY;
        id_s[j] = used ? id : -1;
        p_s[j] = used ? t : 0.f;
        if (used) { tmax = fmaxf(tmax, t); any = 1; }
    }
    const bool taught = __syncthreads_or(any) != 0;
    tmax = block_max<DS_THR>(tmax, red);
    const float at = kLog2e / a.tau;

    // maximum and sums of this thread's elements, the sums relative to its own maximum
    float m = -INFINITY, s = 0.f, s1 = 0.f;
    auto take = [&](const float *v, int n) {
        float mx = v[0];
        for (int i = 1; i < n; ++i) mx = fmaxf(mx, v[i]);
        if (mx > m) {
            const float f = m - mx;                      // -inf the first time
            s *= __builtin_amdgcn_exp2f(f * at);
            if (TWO) s1 *= __builtin_amdgcn_exp2f(f * kLog2e);
            m = mx;
        }
        const float base = m == -INFINITY ? 0.f : m;     // (nothing but masked words so far: they add nothing)
        for (int i = 0; i < n; ++i) {
            s += __builtin_amdgcn_exp2f((v[i] - base) * at);
            if (TWO) s1 += __builtin_amdgcn_exp2f((v[i] - base) * kLog2e);
        }
    };
    for (int c = tid; c < pieces; c += DS_THR) {
        const P t = *(const P *)(z + head + (size_t)c * N);
        float v[N];
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = to_f(t[i]);
        take(v, N);
    }
    float lone_v = -INFINITY;
    if (lone >= 0) {
        lone_v = to_f(z[lone]);
        take(&lone_v, 1);
    }
    const float M = block_max<DS_THR>(m, red);
    const float f = m == -INFINITY ? 0.f : m - M;
    s = block_sum<DS_THR>(s * __builtin_amdgcn_exp2f(f * at), red);
    s1 = TWO ? block_sum<DS_THR>(s1 * __builtin_amdgcn_exp2f(f * kLog2e), red) : s;
    const float log_s = __builtin_amdgcn_logf(s) * kLn2, log_s1 = __builtin_amdgcn_logf(s1) * kLn2;

    // p and the loss; p_s becomes the probability
    float tsum = 0.f;
    for (int j = tid; j < a.k; j += DS_THR) {
        if (id_s[j] >= 0) tsum += __builtin_amdgcn_exp2f((p_s[j] - tmax) * at);
    }
    tsum = block_sum<DS_THR>(tsum, red);
    const float log_t = __builtin_amdgcn_logf(tsum) * kLn2;
    float kl = 0.f;
    for (int j = tid; j < a.k; j += DS_THR) {
        if (id_s[j] < 0) continue;
        const float lt = (p_s[j] - tmax) / a.tau - log_t, p = __builtin_amdgcn_exp2f(lt * kLog2e);
        const float lq = (to_f(z[id_s[j]]) - M) / a.tau - log_s;
        if (p != 0.f) kl += p * (lt - lq);
        p_s[j] = p;
    }
    kl = block_sum<DS_THR>(kl, red);
    const float zl = labeled ? to_f(z[label]) : 0.f;
    if (tid == 0)
        a.loss_tok[row] = (taught ? a.kd * a.tau * a.tau * kl : 0.f) + (labeled ? a.ce * ((M - zl) + log_s1) : 0.f);
    if (!dz) return;

    // gradient: every column from the two softmaxes, then the teacher's and the label's again.  z is read again, so whoever stores
    // over it (dlogits may be the logits) has read it: a thread's own pieces, and the teacher's columns before the barrier.
    const float g = taught ? w * a.kd * a.tau / s : 0.f, g1 = labeled ? w * a.ce / s1 : 0.f;
    auto grad = [&](float v) {
        float r = g * __builtin_amdgcn_exp2f((v - M) * at);
        if (TWO) r += g1 * __builtin_amdgcn_exp2f((v - M) * kLog2e);
        else r += g1 * __builtin_amdgcn_exp2f((v - M) * at);
        return r;
    };
    // columns that are stored again: entry j by the first thread that holds its id, with the sum of its probabilities
    float mine[SLORA_MAX_TOP / DS_THR];
    int col[SLORA_MAX_TOP / DS_THR];
#pragma unroll
    for (int r = 0; r < SLORA_MAX_TOP / DS_THR; ++r) {
        const int j = tid + r * DS_THR;
        col[r] = -1;
        mine[r] = 0.f;
        if (j >= a.k || id_s[j] < 0) continue;
        const int id = id_s[j];
        float p = 0.f;
        bool first = true;
        for (int i = 0; i < a.k; ++i) {
            if (id_s[i] != id) continue;
            if (i < j) { first = false; break; }
            p += p_s[i];
        }
        if (!first) continue;
        col[r] = id;
        mine[r] = grad(to_f(z[id])) - w * a.kd * a.tau * p - (labeled && id == label ? w * a.ce : 0.f);
    }
    bool label_left = labeled;                           // the label is none of the teacher's
    for (int i = 0; i < a.k && label_left; ++i) label_left = id_s[i] != label;
    const float label_v = labeled ? grad(zl) - w * a.ce : 0.f;
    __syncthreads();
    for (int c = tid; c < pieces; c += DS_THR) {
        const P t = *(const P *)(z + head + (size_t)c * N);
        P o;
#pragma unroll
        for (int i = 0; i < N; ++i) { E e; from_f(e, grad(to_f(t[i]))); o[i] = e; }
        E *p = dz + head + (size_t)c * N;
        if (same) *(P *)p = o;
        else
            for (int i = 0; i < N; ++i) p[i] = o[i];
    }
    if (lone >= 0) from_f(dz[lone], grad(lone_v));
    __syncthreads();
#pragma unroll
    for (int r = 0; r < SLORA_MAX_TOP / DS_THR; ++r)
        if (col[r] >= 0) from_f(dz[col[r]], mine[r]);
    if (tid == 0 && label_left) from_f(dz[label], label_v);
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

template <class E>
void launch_rows(const DistillArgs &a, const void *logits, void *dlogits, hipStream_t st)
{
    if (a.labels && a.tau != 1.0f)
        hipLaunchKernelGGL((distill_row_kernel<E, true>), dim3(a.T), dim3(DS_THR), 0, st, a, (const E *)logits, (E *)dlogits);
    else
        hipLaunchKernelGGL((distill_row_kernel<E, false>), dim3(a.T), dim3(DS_THR), 0, st, a, (const E *)logits, (E *)dlogits);
}

inline bool aligned(const void *p, unsigned n) { return ((uintptr_t)p & (n - 1)) == 0; }

}  // namespace

extern "C" int slora_distill_loss(int32_t T, int32_t vocab, int32_t dtype, const void *logits, int64_t ldl, int32_t k,
                                  const int32_t *t_ids, const float *t_logits, float tau, float kd, const int32_t *labels,
                                  float ce, const float *row_weight, float *loss_tok, float *loss, void *dlogits,
                                  int64_t ldd, void *stream)
{
    if (T <= 0 || T > (1 << 24) || vocab <= 0 || vocab > (1 << 24) || k <= 0 || k > SLORA_MAX_TOP) return SLORA_EINVAL;
    if (dtype != SLORA_DTYPE_F32 && dtype != SLORA_DTYPE_BF16) return SLORA_EINVAL;
    if (!logits || !t_ids || !t_logits || !loss_tok || !loss) return SLORA_EINVAL;
    if (!(tau > 0.f) || !(tau <= 1e30f) || !(kd >= 0.f) || !(kd <= 1e30f) || !(ce >= 0.f) || !(ce <= 1e30f)) return SLORA_EINVAL;
    if (ldl < vocab || ldl >= (1ll << 40) || (dlogits && (ldd < vocab || ldd >= (1ll << 40)))) return SLORA_EINVAL;
    if (dlogits == logits && ldd != ldl) return SLORA_EINVAL;
    const unsigned e = dtype == SLORA_DTYPE_F32 ? 4 : 2;
    if (!aligned(logits, e) || !aligned(dlogits, e) || !aligned(t_ids, 4) || !aligned(t_logits, 4) || !aligned(labels, 4) ||
        !aligned(row_weight, 4) || !aligned(loss_tok, 4) || !aligned(loss, 4))
        return SLORA_EINVAL;
    const hipStream_t st = (hipStream_t)stream;
    const DistillArgs a = {T, vocab, k, (size_t)ldl, (size_t)ldd, t_ids, t_logits, tau, kd, ce > 0.f ? labels : nullptr, ce, row_weight,
                           loss_tok};
    if (dtype == SLORA_DTYPE_F32) launch_rows<float>(a, logits, dlogits, st);
    else launch_rows<bf16>(a, logits, dlogits, st);
    SL_CHECK_LAUNCH("distill_row");
    hipLaunchKernelGGL(distill_mean_kernel, dim3(1), dim3(1024), 0, st, loss_tok, row_weight, T, loss);
    SL_CHECK_LAUNCH("distill_mean");
    return SLORA_OK;
}
