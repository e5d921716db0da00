// The training half's losses on logits with their gradients, and the global gradient norm with clipping.
#include "space_device.h"

namespace space {

// ------------------------------------------------------------------------------------------
// rows of logits
// ------------------------------------------------------------------------------------------
// With m = max x, e_i = exp(x_i - m), y the label: O = sum of e_i over i != y, T = O + e_y, logp = (x_y - m) - log T, and
// the gradient of a loss whose slope along logp is c: dx_i = -c e_i / T for i != y, dx_y = c O / T (no difference of nearly
// equal numbers where the label is likely).

template <typename T> __device__ __forceinline__ float load_f32(const T* p);
template <> __device__ __forceinline__ float load_f32<float>(const float* p) { return *p; }
template <> __device__ __forceinline__ float load_f32<uint16_t>(const uint16_t* p) { return bf2f(*p); }
template <typename T> __device__ __forceinline__ void store_f32(T* p, float v);
template <> __device__ __forceinline__ void store_f32<float>(float* p, float v) { *p = v; }
template <> __device__ __forceinline__ void store_f32<uint16_t>(uint16_t* p, float v) { *p = f2bf(v); }

constexpr int kRowThreads = 256;

template <int W>
__device__ __forceinline__ float block_max(float v, float* s) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor(v, o, 64));
    __syncthreads();
    if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = v;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < W; ++w) v = fmaxf(v, s[w]);
    return v;
}
template <int W>
__device__ __forceinline__ double block_sum(double v, double* s) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = v;
    __syncthreads();
    v = 0.0;
#pragma unroll
    for (int w = 0; w < W; ++w) v += s[w];
    return v;
}

struct RowFacts {
    float top;      // m
    double others;  // O
    double total;   // T
    double logp;
};

template <typename T>
__device__ __forceinline__ RowFacts row_facts(const T* __restrict__ x, int vocab, int label) {
    constexpr int W = kRowThreads / 64;
    __shared__ float s_max[W];
    __shared__ double s_sum[W];
    float mx = -INFINITY;
    for (int i = threadIdx.x; i < vocab; i += kRowThreads) mx = fmaxf(mx, load_f32(x + i));
    RowFacts f;
    f.top = block_max<W>(mx, s_max);
    double sum = 0.0;
    for (int i = threadIdx.x; i < vocab; i += kRowThreads)
        if (i != label) sum += exp_below(load_f32(x + i) - f.top);
    f.others = block_sum<W>(sum, s_sum);
    const float d = load_f32(x + label) - f.top;
    f.total = f.others + exp_below(d);
    f.logp = (double)d - (d == 0.f ? log1p(f.others) : log(f.total));
    return f;
}

// d logits of one row: slope = c above, times the caller's scale
template <typename T>
__device__ __forceinline__ void row_gradient(const T* x, T* __restrict__ d, int vocab, int label, float top, float per_e, float at_label) {
    for (int i = threadIdx.x; i < vocab; i += kRowThreads)
        store_f32(d + i, i == label ? at_label : per_e * exp_below(load_f32(x + i) - top));
}
template <typename T>
__device__ __forceinline__ void row_zero(T* __restrict__ d, int vocab) {
    for (int i = threadIdx.x; i < vocab; i += kRowThreads) store_f32(d + i, 0.f);
}

// Whether row `label` counts; one that lies behind the vocabulary is a fault of the caller's.
__device__ __forceinline__ bool row_counts(int label, int vocab) { return label >= 0 && label < vocab; }

template <typename T, int KIND>
__global__ __launch_bounds__(kRowThreads) void loss_rows_kernel(LossLaunch l, PolicyArgs p) {
    const int row = blockIdx.x, label = l.labels[row];
    const T* x = (const T*)l.logits + (size_t)row * l.logits_stride;
    T* d = l.dlogits ? (T*)l.dlogits + (size_t)row * l.dlogits_stride : nullptr;
    if (!row_counts(label, l.vocab)) {
        if (threadIdx.x == 0) {
            l.row_logp[row] = 0.f;
            if (KIND != LOSS_PREF) l.row_loss[row] = 0.f;
            if (KIND == LOSS_POLICY && p.row_kl) p.row_kl[row] = 0.f;
            l.work[row] = f32x4_raw{{0.f, 0.f, 0.f, 0.f}};
            if (label >= 0) atomicAdd(l.faults, 1);
        }
        if (KIND != LOSS_PREF && d) row_zero(d, l.vocab);
        return;
    }
    const RowFacts f = row_facts(x, l.vocab, label);
    if (KIND == LOSS_PREF) {
        if (threadIdx.x == 0) {
            l.row_logp[row] = (float)f.logp;
            l.work[row] = f32x4_raw{{f.top, (float)(1.0 / f.total), (float)(f.others / f.total), 0.f}};
        }
        return;
    }
    double slope = -1.0, term = -f.logp, clipped = 0.0;
    if (KIND == LOSS_POLICY) {
        const double a = p.advantages[row], q = p.old_logp ? exp(f.logp - p.old_logp[row]) : 1.0;
        const double u = q * a, c = fmin(fmax(q, (double)p.lo), (double)p.hi) * a;
        clipped = u > c ? 1.0 : 0.0;
        term = u > c ? -c : -u;
        slope = u > c ? 0.0 : -u;
        double kl = 0.0;
        if (p.ref_logp) {
            const double gap = p.ref_logp[row] - f.logp, em = expm1(gap);
            kl = em - gap;
            if (p.kl_coef != 0.f) {
                term += (double)p.kl_coef * kl;
                slope -= (double)p.kl_coef * em;
            }
        }
        if (p.row_weight) {
            term *= p.row_weight[row];
            slope *= p.row_weight[row];
        }
        if (threadIdx.x == 0 && p.row_kl) p.row_kl[row] = (float)kl;
    }
    if (threadIdx.x == 0) {
        l.row_logp[row] = (float)f.logp;
        l.row_loss[row] = (float)term;
        l.work[row] = f32x4_raw{{(float)clipped, 0.f, 0.f, 0.f}};
    }
    if (!d) return;
    double c = slope;
    if (l.mean) c /= max(*l.n_terms, 1);
    if (l.grad_scale) c *= *l.grad_scale;
    row_gradient(x, d, l.vocab, label, f.top, (float)(-c / f.total), (float)(c * (f.others / f.total)));
}

// How many rows count, for the mean that the rows' gradients need before the rows are done.
__global__ __launch_bounds__(1024) void loss_count_kernel(LossLaunch l) {
    __shared__ double s[16];
    int n = 0;
    for (int r = threadIdx.x; r < l.rows; r += 1024) n += row_counts(l.labels[r], l.vocab);
    const double all = block_sum<16>(n, s);
    if (threadIdx.x == 0) *l.n_terms = (int)all;
}

// The rows' terms added up: each thread its own in row order, then a fixed tree, in 64 bits.
__global__ __launch_bounds__(1024) void loss_sum_kernel(LossLaunch l, int32_t* n_clipped) {
    __shared__ double s[16];
    double sum = 0.0;
    int n = 0, clipped = 0;
    for (int r = threadIdx.x; r < l.rows; r += 1024) {
        sum += l.row_loss[r];
        n += row_counts(l.labels[r], l.vocab);
        if (n_clipped) clipped += l.work[r].v[0] != 0.f;
    }
    sum = block_sum<16>(sum, s);
    const double count = block_sum<16>(n, s);
    const double cut = n_clipped ? block_sum<16>(clipped, s) : 0.0;
    if (threadIdx.x == 0) {
        *l.loss = (float)(l.mean ? sum / fmax(count, 1.0) : sum);
        *l.n_terms = (int)count;
        if (n_clipped) *n_clipped = (int)cut;
    }
}

// The pairs, one to a wave: sums over the rows of their two sequences, their terms, and the slope of every row.
__global__ __launch_bounds__(1024) void pref_pairs_kernel(LossLaunch l, PrefArgs p) {
    __shared__ double s[16];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    double sum = 0.0;
    int n_all = 0;
    for (int pair = wave; pair < p.pairs; pair += 16) {
        int from[2], to[2], n[2];
        double ratio[2];
        bool bad = false;
#pragma unroll
        for (int w = 0; w < 2; ++w) {
            const int a = p.seq_start[2 * pair + w], b = p.seq_start[2 * pair + w + 1];
            from[w] = min(max(a, 0), l.rows);
            to[w] = min(max(b, from[w]), l.rows);
            bad = bad || a != from[w] || b != to[w];
            double t = 0.0;
            int k = 0;
            for (int r = from[w] + lane; r < to[w]; r += 64) {
                t += l.row_logp[r];
                k += row_counts(l.labels[r], l.vocab);
            }
#pragma unroll
            for (int o = 32; o > 0; o >>= 1) {
                t += __shfl_xor(t, o, 64);
                k += __shfl_xor(k, o, 64);
            }
            if (p.average) t /= max(k, 1);
            n[w] = k;
            n_all += k;
            if (lane == 0 && p.seq_logp) p.seq_logp[2 * pair + w] = (float)t;
            ratio[w] = p.ref_logp ? t - p.ref_logp[2 * pair + w] : t;
        }
        if (bad && lane == 0) atomicAdd(l.faults, 1);
        const double z = (double)p.beta * (ratio[0] - ratio[1]) - (double)p.margin, eps = p.smoothing;
        const double tail = log1p(exp(-fabs(z))), low = fmax(-z, 0.0) + tail, high = fmax(z, 0.0) + tail;  // softplus(-z), softplus(z)
        const double term = (eps < 1.0 ? (1.0 - eps) * low : 0.0) + (eps > 0.0 ? eps * high : 0.0);
        if (lane == 0) p.pair_loss[pair] = (float)term;
        sum += term;
        if (!l.dlogits) continue;
        // sigmoid(z) and sigmoid(-z), each without a difference from 1
        const double t = exp(-fabs(z)), big = 1.0 / (1.0 + t), small = t / (1.0 + t);
        double slope = (double)p.beta * (eps * (z >= 0.0 ? big : small) - (1.0 - eps) * (z >= 0.0 ? small : big));
        if (l.mean) slope /= p.pairs;
        if (l.grad_scale) slope *= *l.grad_scale;
#pragma unroll
        for (int w = 0; w < 2; ++w) {
            const double c = (w ? -slope : slope) / (p.average ? max(n[w], 1) : 1);
            for (int r = from[w] + lane; r < to[w]; r += 64) l.work[r].v[3] = (float)c;
        }
    }
    sum = block_sum<16>(lane == 0 ? sum : 0.0, s);
    const double n = block_sum<16>(lane == 0 ? n_all : 0, s);
    if (threadIdx.x == 0) {
        *l.loss = (float)(l.mean ? sum / p.pairs : sum);
        *l.n_terms = (int)n;
    }
}

template <typename T>
__global__ __launch_bounds__(kRowThreads) void pref_gradient_kernel(LossLaunch l) {
    const int row = blockIdx.x, label = l.labels[row];
    T* d = (T*)l.dlogits + (size_t)row * l.dlogits_stride;
    const f32x4_raw f = l.work[row];
    if (!row_counts(label, l.vocab) || f.v[3] == 0.f) return row_zero(d, l.vocab);
    row_gradient((const T*)l.logits + (size_t)row * l.logits_stride, d, l.vocab, label, f.v[0], -f.v[3] * f.v[1], f.v[3] * f.v[2]);
}

template <int KIND>
hipError_t launch_rows(const LossLaunch& l, const PolicyArgs& p, hipStream_t s) {
    if (l.dtype == 0) hipLaunchKernelGGL((loss_rows_kernel<float, KIND>), dim3(l.rows), dim3(kRowThreads), 0, s, l, p);
    else hipLaunchKernelGGL((loss_rows_kernel<uint16_t, KIND>), dim3(l.rows), dim3(kRowThreads), 0, s, l, p);
    return hipGetLastError();
}

template <int KIND>
hipError_t launch_loss(const LossLaunch& l, const PolicyArgs& p, hipStream_t s) {
    if (l.mean && l.dlogits) {
        hipLaunchKernelGGL(loss_count_kernel, dim3(1), dim3(1024), 0, s, l);
        if (hipError_t e = hipGetLastError()) return e;
    }
    if (hipError_t e = launch_rows<KIND>(l, p, s)) return e;
    hipLaunchKernelGGL(loss_sum_kernel, dim3(1), dim3(1024), 0, s, l, p.n_clipped);
    return hipGetLastError();
}

hipError_t launch_sar_grad(const LossLaunch& l, hipStream_t s) { return launch_loss<LOSS_SAR>(l, PolicyArgs{}, s); }
hipError_t launch_policy(const LossLaunch& l, const PolicyArgs& p, hipStream_t s) { return launch_loss<LOSS_POLICY>(l, p, s); }

hipError_t launch_preference(const LossLaunch& l, const PrefArgs& p, hipStream_t s) {
    if (hipError_t e = launch_rows<LOSS_PREF>(l, PolicyArgs{}, s)) return e;
    hipLaunchKernelGGL(pref_pairs_kernel, dim3(1), dim3(1024), 0, s, l, p);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || !l.dlogits) return e;
    if (l.dtype == 0) hipLaunchKernelGGL(pref_gradient_kernel<float>, dim3(l.rows), dim3(kRowThreads), 0, s, l);
    else hipLaunchKernelGGL(pref_gradient_kernel<uint16_t>, dim3(l.rows), dim3(kRowThreads), 0, s, l);
    return hipGetLastError();
}

// ------------------------------------------------------------------------------------------
// gradient norm and clipping
// ------------------------------------------------------------------------------------------
// A launch takes up to kGradList tensors by value (arguments of a kernel: 4 KB at most), so nothing has to be kept on the device; their elements are cut into
// chunks that are dealt out to the workgroups in turn.
constexpr int kGradList = 112, kGradThreads = 256, kGradChunk = 8192;
struct GradList {
    const void* grad[kGradList];
    void* out[kGradList];
    int64_t n[kGradList];
    int64_t first[kGradList + 1];  // chunks in front of a tensor
    uint8_t type[kGradList];       // bit 0: bf16 gradient, bit 1: bf16 output
    int count;
};
static_assert(sizeof(GradList) < 3900, "arguments of a kernel");

__device__ __forceinline__ int grad_tensor_of(const GradList& g, int64_t chunk) {
    int lo = 0, hi = g.count - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (g.first[mid] <= chunk) lo = mid; else hi = mid - 1;
    }
    return lo;
}
__device__ __forceinline__ float grad_load(const void* p, int64_t i, bool bf16) {
    return bf16 ? bf2f(((const uint16_t*)p)[i]) : ((const float*)p)[i];
}

// Squares are exact in 64 bits for both types, and no sum of them leaves the range.
__global__ __launch_bounds__(kGradThreads) void grad_square_kernel(GradList g, double* work, int first_launch) {
    __shared__ double s[kGradThreads / 64];
    double sum = 0.0;
    const int64_t chunks = g.first[g.count];
    for (int64_t c = blockIdx.x; c < chunks; c += gridDim.x) {
        const int t = grad_tensor_of(g, c);
        const int64_t from = (c - g.first[t]) * kGradChunk, to = min(from + kGradChunk, g.n[t]);
        for (int64_t i = from + threadIdx.x; i < to; i += kGradThreads) {
            const double v = grad_load(g.grad[t], i, g.type[t] & 1);
            sum += v * v;
        }
    }
    sum = block_sum<kGradThreads / 64>(sum, s);
    if (threadIdx.x == 0) work[blockIdx.x] = first_launch ? sum : work[blockIdx.x] + sum;
}

__global__ __launch_bounds__(1024) void grad_norm_kernel(const double* work, int parts, float* norm) {
    __shared__ double s[16];
    double sum = 0.0;
    for (int i = threadIdx.x; i < parts; i += 1024) sum += work[i];
    sum = block_sum<16>(sum, s);
    if (threadIdx.x == 0) *norm = (float)sqrt(sum);
}

__global__ __launch_bounds__(kGradThreads) void grad_clip_kernel(GradList g, const float* norm, float max_norm) {
    const float n = *norm;
    const float scale = n > max_norm && n < INFINITY ? max_norm / n : 1.f;
    const int64_t chunks = g.first[g.count];
    for (int64_t c = blockIdx.x; c < chunks; c += gridDim.x) {
        const int t = grad_tensor_of(g, c);
        if (scale == 1.f && g.out[t] == g.grad[t]) continue;
        const int64_t from = (c - g.first[t]) * kGradChunk, to = min(from + kGradChunk, g.n[t]);
        for (int64_t i = from + threadIdx.x; i < to; i += kGradThreads) {
            const float v = grad_load(g.grad[t], i, g.type[t] & 1) * scale;
            if (g.type[t] & 2) ((uint16_t*)g.out[t])[i] = f2bf(v); else ((float*)g.out[t])[i] = v;
        }
    }
}

// Calls launch(list, workgroups, first) for every kGradList tensors that are not empty.
template <typename F>
hipError_t each_grad_list(const GradTensor* t, int n, F launch) {
    GradList g;
    bool first = true;
    for (int i = 0; i < n;) {
        g.count = 0;
        g.first[0] = 0;
        for (; i < n && g.count < kGradList; ++i) {
            if (t[i].n == 0) continue;
            const int c = g.count++;
            g.grad[c] = t[i].grad;
            g.out[c] = t[i].out;
            g.n[c] = t[i].n;
            g.type[c] = (uint8_t)(t[i].dtype | t[i].out_dtype << 1);
            g.first[c + 1] = g.first[c] + (t[i].n + kGradChunk - 1) / kGradChunk;
        }
        if (!g.count) break;
        launch(g, (int)(g.first[g.count] < kGradParts ? g.first[g.count] : kGradParts), first);
        if (hipError_t e = hipGetLastError()) return e;
        first = false;
    }
    return hipSuccess;
}

hipError_t launch_grad_norm(const GradTensor* t, int n, float* norm, double* work, hipStream_t s) {
    int parts = 0;
    // (a later launch adds to the partial sums of an earlier one, so all of them use as many workgroups)
    int64_t most = 0;
    const hipError_t count = each_grad_list(t, n, [&](const GradList& g, int wgs, bool) { most = wgs > most ? wgs : most; });
    if (count != hipSuccess) return count;
    parts = (int)most;
    const hipError_t e = each_grad_list(t, n, [&](const GradList& g, int, bool first) {
        hipLaunchKernelGGL(grad_square_kernel, dim3(parts), dim3(kGradThreads), 0, s, g, work, (int)first);
    });
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(grad_norm_kernel, dim3(1), dim3(1024), 0, s, work, parts, norm);
    return hipGetLastError();
}

hipError_t launch_grad_clip(const GradTensor* t, int n, const float* norm, float max_norm, hipStream_t s) {
    return each_grad_list(t, n, [&](const GradList& g, int wgs, bool) {
        hipLaunchKernelGGL(grad_clip_kernel, dim3(wgs), dim3(kGradThreads), 0, s, g, norm, max_norm);
    });
}

}  // namespace space
