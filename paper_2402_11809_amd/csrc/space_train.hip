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

// 16 bytes of a row, on any whole element (the hardware takes them unaligned)
template <typename T> struct Vec;
template <> struct Vec<float> {
    static constexpr int N = 4;
    typedef float raw __attribute__((ext_vector_type(4), aligned(4)));
    static __device__ __forceinline__ void get(raw q, float* v) {
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = q[e];
    }
    static __device__ __forceinline__ raw put(const float* v) { return raw{v[0], v[1], v[2], v[3]}; }
};
template <> struct Vec<uint16_t> {
    static constexpr int N = 8;
    typedef uint32_t raw __attribute__((ext_vector_type(4), aligned(2)));
    static __device__ __forceinline__ void get(raw q, float* v) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const uint32_t w = q[e];
            v[2 * e] = __uint_as_float(w << 16);
            v[2 * e + 1] = __uint_as_float(w & 0xffff0000u);
        }
    }
    static __device__ __forceinline__ raw put(const float* v) {
        raw q;
#pragma unroll
        for (int e = 0; e < 4; ++e) q[e] = (uint32_t)f2bf(v[2 * e]) | (uint32_t)f2bf(v[2 * e + 1]) << 16;
        return q;
    }
};

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

// KEPT: the ordinary way; else past the caches, for what is read once
template <bool KEPT, typename V>
__device__ __forceinline__ typename V::raw read_vec(const void* p) {
    if (KEPT) return *(const typename V::raw*)p;
    return __builtin_nontemporal_load((const typename V::raw*)p);
}

// Whether row `label` counts; one that lies behind the vocabulary is a fault of the caller's.
__device__ __forceinline__ bool row_counts(int label, int vocab) { return label >= 0 && label < vocab; }

template <typename T, int THREADS>
__device__ __forceinline__ void row_zero(T* __restrict__ d, int vocab) {
    typedef Vec<T> V;
    const float none[V::N] = {};
    for (int i = threadIdx.x * V::N; i < vocab / V::N * V::N; i += THREADS * V::N) __builtin_nontemporal_store(V::put(none), (typename V::raw*)(d + i));
    if ((int)threadIdx.x < vocab % V::N) store_f32(d + vocab / V::N * V::N + threadIdx.x, 0.f);
}

// ---- what the rows add up to: by a launch of its own, or, where a call is small, by the rows' workgroup that ends last.  The last
// one finds out by the caller's arrival count (space_arrivals.h); what it reads of others' rows they store past their XCD's L2.
__device__ __forceinline__ void put(float* p, float v) { __hip_atomic_store(p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
__device__ __forceinline__ float got(const float* p) { return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }

// Whether this workgroup is the last of the launch's.  Thread 0 made the stores that the last one reads.
__device__ __forceinline__ bool arrive(uint32_t* arrived, int* s_last) {
    if (threadIdx.x == 0) {
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        const uint32_t share = arrival_share(gridDim.x, blockIdx.x);
        *s_last = arrival_is_last(__hip_atomic_fetch_add(arrived, share, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT), share);
    }
    __syncthreads();
    return *s_last;
}

// The rows that count, by a whole workgroup (without its sum over the waves): this wave's.
template <int THREADS>
__device__ __forceinline__ int count_rows(const LossLaunch& l) {
    int n = 0;
#pragma unroll 8
    for (int r = threadIdx.x; r < l.rows; r += THREADS) n += row_counts(l.labels[r], l.vocab);
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) n += __shfl_xor(n, o, 64);
    return n;
}

// Loss, counts (SMALL: within the rows' launch): each thread adds its own rows in row order, in 64 bits, then a fixed tree.
template <int THREADS, bool SMALL>
__device__ __forceinline__ void sum_rows(const LossLaunch& l, int32_t* n_clipped) {
    constexpr int W = THREADS / 64;
    __shared__ double s_sum[W];
    __shared__ int2 s_n[W];
    double sum = 0.0;
    int n = 0, cut = 0;
#pragma unroll 8
    for (int r = threadIdx.x; r < l.rows; r += THREADS) {
        sum += SMALL ? got(l.row_loss + r) : l.row_loss[r];
        n += row_counts(l.labels[r], l.vocab);
        if (n_clipped) cut += (SMALL ? got(&l.work[r].v[0]) : l.work[r].v[0]) != 0.f;
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) {
        sum += __shfl_xor(sum, o, 64);
        n += __shfl_xor(n, o, 64);
        cut += __shfl_xor(cut, o, 64);
    }
    if ((threadIdx.x & 63) == 0) {
        s_sum[threadIdx.x >> 6] = sum;
        s_n[threadIdx.x >> 6] = int2{n, cut};
    }
    __syncthreads();
    if (threadIdx.x != 0) return;
    for (int w = 1; w < W; ++w) {
        sum += s_sum[w];
        n += s_n[w].x;
        cut += s_n[w].y;
    }
    *l.loss = (float)(l.mean ? sum / max(n, 1) : sum);
    *l.n_terms = n;
    if (n_clipped) *n_clipped = cut;
}

// ---- the preference loss
// Sequence `seq` by one wave: its rows (clamped to those there are), how many count, and their sum or mean of logp, added in 64 bits as they are
// given out, rounded to 32 bits each (what their own sums of exponentials are off by is more).
struct SeqSum {
    int from, to, n;
    double sum;
    bool fault;
};
__device__ __forceinline__ SeqSum sum_sequence(const LossLaunch& l, const PrefArgs& p, int seq) {
    SeqSum q;
    const int a = p.seq_start[seq], b = p.seq_start[seq + 1];
    q.from = min(max(a, 0), l.rows);
    q.to = min(max(b, q.from), l.rows);
    q.fault = a != q.from || b != q.to;
    q.sum = 0.0;
    q.n = 0;
#pragma unroll 8
    for (int r = q.from + (threadIdx.x & 63); r < q.to; r += 64) {
        q.sum += l.row_logp[r];
        q.n += row_counts(l.labels[r], l.vocab);
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) {
        q.sum += __shfl_xor(q.sum, o, 64);
        q.n += __shfl_xor(q.n, o, 64);
    }
    if (p.average) q.sum /= max(q.n, 1);
    return q;
}
__device__ __forceinline__ double against_reference(const PrefArgs& p, int seq, double sum) { return p.ref_logp ? sum - p.ref_logp[seq] : sum; }

struct PairTerm {
    double term, slope;  // slope: along z, times the caller's factors
};
__device__ __forceinline__ PairTerm pair_term(const LossLaunch& l, const PrefArgs& p, double chosen, double rejected) {
    const double z = (double)p.beta * (chosen - rejected) - (double)p.margin, eps = p.smoothing;
    const double far = exp(-fabs(z)), tail = log1p(far);
    const double low = fmax(-z, 0.0) + tail, high = fmax(z, 0.0) + tail;  // softplus(-z), softplus(z)
    PairTerm t;
    t.term = (eps < 1.0 ? (1.0 - eps) * low : 0.0) + (eps > 0.0 ? eps * high : 0.0);
    // sigmoid(z) and sigmoid(-z), each without a difference from 1
    const double big = 1.0 / (1.0 + far), small = far / (1.0 + far);
    t.slope = (double)p.beta * (eps * (z >= 0.0 ? big : small) - (1.0 - eps) * (z >= 0.0 ? small : big));
    if (l.mean) t.slope /= p.pairs;
    if (l.grad_scale) t.slope *= *l.grad_scale;
    return t;
}
// Of a row of the chosen (which = 0) or the rejected sequence, in which n rows count
__device__ __forceinline__ float row_slope_of(const PrefArgs& p, const PairTerm& t, int which, int n) {
    const double c = p.average ? t.slope / max(n, 1) : t.slope;
    return (float)(which ? -c : c);
}

// Eight pairs to a workgroup of 1024 threads, a sequence to a wave: the pairs' terms and, where WRITE, the slopes of the rows.  A
// workgroup that has all pairs adds them up, too.
constexpr int kPairs = 8;
template <bool WRITE>
__device__ __forceinline__ void join_pairs(const LossLaunch& l, const PrefArgs& p, int first) {
    __shared__ double s_sum[2 * kPairs], s_term[kPairs];
    __shared__ int s_n[2 * kPairs];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, seq = 2 * first + wave;
    const bool mine = seq < 2 * p.pairs;
    SeqSum q;
    if (mine) {
        q = sum_sequence(l, p, seq);
        if (lane == 0) {
            s_sum[wave] = against_reference(p, seq, q.sum);
            s_n[wave] = q.n;
            if (p.seq_logp) p.seq_logp[seq] = (float)q.sum;
            if (q.fault) atomicAdd(l.faults, 1);
        }
    }
    __syncthreads();
    if (mine) {
        const PairTerm t = pair_term(l, p, s_sum[wave & ~1], s_sum[wave | 1]);
        if (lane == 0 && wave % 2 == 0) {
            p.pair_loss[seq / 2] = (float)t.term;
            s_term[wave / 2] = t.term;
        }
        if (WRITE) {
            const float slope = row_slope_of(p, t, wave % 2, q.n);
            for (int r = q.from + lane; r < q.to; r += 64) l.work[r].v[3] = slope;
        }
    }
    if (p.pairs > kPairs) return;
    __syncthreads();  // no others: the loss, too
    if (threadIdx.x != 0) return;
    double sum = 0.0;
    int n = 0;
    for (int k = 0; k < p.pairs; ++k) {
        sum += s_term[k];
        n += s_n[2 * k] + s_n[2 * k + 1];
    }
    *l.loss = (float)(l.mean ? sum / p.pairs : sum);
    *l.n_terms = n;
}

// The loss of many pairs, from their terms, and the rows that count: 1024 threads, a fixed order, 64 bits.
__device__ __forceinline__ void sum_pairs(const LossLaunch& l, const PrefArgs& p) {
    __shared__ double s[16];
    double sum = 0.0, n = 0.0;
    for (int i = threadIdx.x; i < p.pairs; i += 1024) sum += p.pair_loss[i];
    const int from = min(max(p.seq_start[0], 0), l.rows), to = min(max(p.seq_start[2 * p.pairs], 0), l.rows);
#pragma unroll 4
    for (int r = from + threadIdx.x; r < to; r += 1024) n += row_counts(l.labels[r], l.vocab);
    sum = block_sum<16>(sum, s);
    n = block_sum<16>(n, s);
    if (threadIdx.x == 0) {
        *l.loss = (float)(l.mean ? sum / p.pairs : sum);
        *l.n_terms = (int)n;
    }
}

// What a row's label and its other tokens add up to, in the row's own scale (its maximum)
struct RowFacts {
    float top;
    float at_label;  // e_y
    double others;   // O
    double total;    // T
    __device__ __forceinline__ double logp(float x_label) const {
        const float d = x_label - top;
        return (double)d - (d == 0.f ? log1p(others) : log(total));
    }
};

// Joins the waves' maxima and sums (without the label's): one barrier a row.  *factor: from the wave's scale to the row's.
template <int W>
__device__ __forceinline__ RowFacts join_waves(float mx, double sum, float x_label, float* factor, float* s_max, double* s_sum) {
    if ((threadIdx.x & 63) == 0) {
        s_max[threadIdx.x >> 6] = mx;
        s_sum[threadIdx.x >> 6] = sum;
    }
    __syncthreads();
    RowFacts f;
    f.top = x_label;
#pragma unroll
    for (int w = 0; w < W; ++w) f.top = fmaxf(f.top, s_max[w]);
    f.others = 0.0;
#pragma unroll
    for (int w = 0; w < W; ++w) f.others += s_sum[w] * (s_max[w] == -INFINITY ? 0.f : exp_below(s_max[w] - f.top));
    f.at_label = exp_below(x_label - f.top);
    f.total = f.others + f.at_label;
    *factor = mx == -INFINITY ? 0.f : exp_below(mx - f.top);
    return f;
}

template <int W>
__device__ __forceinline__ int sum_of(const int* s) {
    int n = 0;
#pragma unroll
    for (int w = 0; w < W; ++w) n += s[w];
    return n;
}

// v * by, and 0 where `by` is 0 though v is infinite: nothing is contributed, as for every finite v (NaN stays NaN).
__device__ __forceinline__ double times(double v, double by) { return by == 0.0 && isinf(v) ? 0.0 : v * by; }

struct RowSlope {
    double term, slope, kl;
    bool clipped;
};
template <int KIND>
__device__ __forceinline__ RowSlope row_slope(const PolicyArgs& p, int row, double logp) {
    RowSlope s{-logp, -1.0, 0.0, false};
    if (KIND == LOSS_POLICY) {
        // (without old_logp the ratio is logp's to itself: 1, also of a masked token, but no number where logp is none)
        const double a = p.advantages[row], q = p.old_logp ? exp(logp - p.old_logp[row]) : isnan(logp) ? logp : 1.0;
        const double u = times(q, a), c = fmin(fmax(q, (double)p.lo), (double)p.hi) * a;
        s.clipped = u > c;
        s.term = s.clipped ? -c : -u;
        s.slope = s.clipped ? 0.0 : -u;
        if (p.ref_logp) {
            const double gap = p.ref_logp[row] - logp, em = expm1(gap);
            s.kl = em == INFINITY ? em : em - gap;  // (a token that is masked out now)
            if (p.kl_coef != 0.f) {
                s.term += (double)p.kl_coef * s.kl;
                s.slope -= (double)p.kl_coef * em;
            }
        }
        if (p.row_weight) {
            const double w = p.row_weight[row];
            s.term = times(s.term, w);
            s.slope = times(s.slope, w);
        }
    }
    return s;
}

// What a row that does not count leaves behind.
template <typename T, int KIND, int THREADS>
__device__ __forceinline__ void row_left_out(const LossLaunch& l, const PolicyArgs& p, int row, int label, T* d) {
    if (threadIdx.x == 0) {
        put(l.row_logp + row, 0.f);
        if (KIND != LOSS_PREF) put(l.row_loss + row, 0.f);
        if (KIND == LOSS_POLICY && p.row_kl) p.row_kl[row] = 0.f;
        if (KIND == LOSS_POLICY) put(&l.work[row].v[0], 0.f);
        if (label >= 0) atomicAdd(l.faults, 1);
    }
    if (KIND != LOSS_PREF && d) row_zero<T, THREADS>(d, l.vocab);
}

// The row's own outputs, by thread 0.  Returns the slope of the loss along logp.
template <int KIND>
__device__ __forceinline__ double row_outputs(const LossLaunch& l, const PolicyArgs& p, int row, const RowFacts& f, float x_label) {
    const double logp = f.logp(x_label);
    put(l.row_logp + row, (float)logp);
    if (KIND == LOSS_PREF) {  // (behind them stands the row's slope, which join_pairs writes)
        l.work[row].v[0] = f.top;
        l.work[row].v[1] = (float)(1.0 / f.total);
        l.work[row].v[2] = (float)(f.others / f.total);
        return 0.0;
    }
    const RowSlope s = row_slope<KIND>(p, row, logp);
    put(l.row_loss + row, (float)s.term);
    if (KIND == LOSS_POLICY) {
        put(&l.work[row].v[0], s.clipped ? 1.f : 0.f);
        if (p.row_kl) p.row_kl[row] = (float)s.kl;
    }
    return s.slope;
}
// What the gradient of the loss along logp is multiplied with.
__device__ __forceinline__ double slope_factor(const LossLaunch& l, int n) {
    double c = l.mean ? 1.0 / max(n, 1) : 1.0;
    if (l.grad_scale) c *= *l.grad_scale;
    return c;
}
// The slope with everything in it, for all threads; the policy loss has it from thread 0.
template <int KIND>
__device__ __forceinline__ double row_coefficient(const LossLaunch& l, const PolicyArgs& p, int row, const RowFacts& f, float x_label, int n, double* s_slope) {
    if (KIND == LOSS_SAR) return -slope_factor(l, n);
    if (threadIdx.x == 0) *s_slope = row_outputs<KIND>(l, p, row, f, x_label) * slope_factor(l, n);
    __syncthreads();
    return *s_slope;
}

// Behind a row: the last workgroup adds up.
template <int THREADS>
__device__ __forceinline__ void finish_rows(const LossLaunch& l, const PolicyArgs& p) {
    __shared__ int s_last;
    if (arrive(l.arrived, &s_last)) sum_rows<THREADS, true>(l, p.n_clipped);
}

// A row in the registers of one workgroup: read once, written once.  Bound by memory: a row that is read while another one
// of the CU is computed or written, so what counts is that two rows or more share a CU (128 registers a thread, four waves a
// SIMD).  32 elements a thread in short rows, 64 in longer ones.  KEEP: the exponentials take the logits' place, 32 bits each;
// otherwise (bf16 rows that would fill the CU that way) the packed logits stay and the exponential is taken again, without
// exp_below's correction: it is off by |x - max| 2^-24 of itself at most, 5e-6 before it vanishes, against bf16's half step of 4e-3.
// The 64-bit functions of the policy loss' slope do not all fit beside a full row: the bf16 kernels that keep it packed and have the sums
// in them (up to 4096 rows) spill 36 bytes a thread, the fp32 ones of 512 and 1024 threads without them 16 and 12 (policy and finetuning
// loss: 2000 rows of 64000 in bf16 122 and 112 us, in fp32 198 and 193; 1000 of 128000 in bf16 137 and 122; 4200 of 40001 in fp32 276 and 267).
// 5.77 TB/s read and written in fp32 (4096 rows of 32000, 182 us), 5.46 in bf16 (8192 rows, 192 us), where a copy of such
// buffers reaches 4.8 - 4.9; all in one launch of 1024 threads and 32 elements 5.0 and 4.0.  Loads and stores are non-temporal:
// stores 5.1 -> 5.5 TB/s.
template <typename T, int KIND, int THREADS, int NV, bool KEEP, bool SMALL>
__device__ __forceinline__ void row_of_loss(const LossLaunch& l, const PolicyArgs& p) {
    typedef Vec<T> V;
    constexpr int W = THREADS / 64, E = V::N;
    __shared__ float s_max[W];
    __shared__ double s_sum[W], s_slope;
    __shared__ int s_n[W];
    const int row = blockIdx.x, tid = threadIdx.x, label = l.labels[row], vocab = l.vocab;
    const T* x = (const T*)l.logits + (size_t)row * l.logits_stride;
    T* d = l.dlogits ? (T*)l.dlogits + (size_t)row * l.dlogits_stride : nullptr;
    if (!row_counts(label, vocab)) return row_left_out<T, KIND, THREADS>(l, p, row, label, d);
    const float x_label = load_f32(x + label);
    // whole vectors, then the odd elements behind them, one to a thread
    const int whole = vocab / E, odd = whole * E + tid;
    typename V::raw q[NV];
#pragma unroll
    for (int j = 0; j < NV; ++j)
        if (tid + j * THREADS < whole) q[j] = read_vec<KIND == LOSS_PREF, V>(x + (size_t)(tid + j * THREADS) * E);
    float t = odd < vocab && odd != label ? load_f32(x + odd) : -INFINITY;
    float v[KEEP ? NV * E : E], mx = t;
    // vector j as 32-bit numbers, nothing behind the row and nothing at the label, which stands apart
    auto unpack = [&](int j, float* u) {
        if (tid + j * THREADS < whole) {
            V::get(q[j], u);
        } else {
#pragma unroll
            for (int e = 0; e < E; ++e) u[e] = -INFINITY;
        }
        if (tid + j * THREADS == label / E) {
#pragma unroll
            for (int e = 0; e < E; ++e)
                if (e == label % E) u[e] = -INFINITY;
        }
    };
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        if (j * THREADS < whole) {  // (all threads or none)
            float* u = v + (KEEP ? j * E : 0);
            unpack(j, u);
#pragma unroll
            for (int e = 0; e < E; ++e) mx = fmaxf(mx, u[e]);
        }
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) mx = fmaxf(mx, __shfl_xor(mx, o, 64));
    const float base = mx == -INFINITY ? 0.f : mx;
    float part[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        if (j * THREADS < whole) {
            float* u = v + (KEEP ? j * E : 0);
            if (!KEEP) unpack(j, u);
#pragma unroll
            for (int e = 0; e < E; ++e) {
                u[e] = exp_below(u[e] - base);
                part[e % 4] += u[e];
            }
        }
    }
    t = exp_below(t - base);
    double sum = ((double)part[0] + part[1]) + ((double)part[2] + part[3]) + t;
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) sum += __shfl_xor(sum, o, 64);
    // the mean's divisor: counted here in a small call, by a launch in front in a large one
    if (SMALL && KIND != LOSS_PREF && l.mean && d) {
        const int n = count_rows<THREADS>(l);
        if ((tid & 63) == 0) s_n[tid >> 6] = n;
    }
    float factor;
    const RowFacts f = join_waves<W>(mx, sum, x_label, &factor, s_max, s_sum);
    if (KIND == LOSS_PREF || !d) {
        if (tid == 0) row_outputs<KIND>(l, p, row, f, x_label);
        return;
    }
    const int n = !l.mean ? 1 : SMALL ? sum_of<W>(s_n) : *l.n_terms;
    // (what a row's elements are multiplied with is rounded once)
    const double c = row_coefficient<KIND>(l, p, row, f, x_label, n, &s_slope) / f.total;
    const float per_e = (float)(-c * factor), at_label = (float)(c * f.others);
#pragma unroll
    for (int j = 0; j < NV; ++j)
        if (tid + j * THREADS < whole) {
            float g[E];
            float* u = v + (KEEP ? j * E : 0);
            if (!KEEP) {
                V::get(q[j], u);
#pragma unroll
                for (int e = 0; e < E; ++e) u[e] = __builtin_amdgcn_exp2f((u[e] - base) * 1.4426950408889634f);
            }
#pragma unroll
            for (int e = 0; e < E; ++e) g[e] = u[e] * per_e;
            if (tid + j * THREADS == label / E) {
#pragma unroll
                for (int e = 0; e < E; ++e)
                    if (e == label % E) g[e] = at_label;
            }
            __builtin_nontemporal_store(V::put(g), (typename V::raw*)(d + (size_t)(tid + j * THREADS) * E));
        }
    if (odd < vocab) store_f32(d + odd, odd == label ? at_label : t * per_e);
    if (KIND == LOSS_SAR && tid == 0) row_outputs<KIND>(l, p, row, f, x_label);
}

template <typename T, int KIND, int THREADS, int NV, bool KEEP, bool SMALL>
__global__ __launch_bounds__(THREADS, 4) void loss_rows_kernel(LossLaunch l, PolicyArgs p) {
    row_of_loss<T, KIND, THREADS, NV, KEEP, SMALL>(l, p);
    if (SMALL) finish_rows<THREADS>(l, p);
}

// A row that no workgroup's registers hold: once for maximum and sum, once for the gradient.
constexpr int kLongThreads = 1024, kLongVecs = 4;
template <typename T, int THREADS>
__device__ __forceinline__ void long_gradient(const T* x, T* d, int vocab, int label, float top, float per_e, float at_label) {
    typedef Vec<T> V;
    constexpr int E = V::N;
    const int whole = vocab / E, odd = whole * E + threadIdx.x;
    for (int at = threadIdx.x; at < whole; at += THREADS * kLongVecs) {
        typename V::raw q[kLongVecs];
#pragma unroll
        for (int j = 0; j < kLongVecs; ++j)
            if (at + j * THREADS < whole) q[j] = *(const typename V::raw*)(x + (size_t)(at + j * THREADS) * E);
#pragma unroll
        for (int j = 0; j < kLongVecs; ++j) {
            const int i = at + j * THREADS;
            if (i >= whole) break;
            float g[E];
            V::get(q[j], g);
#pragma unroll
            for (int e = 0; e < E; ++e) g[e] = per_e * exp_below(g[e] - top);
            if (i == label / E) {
#pragma unroll
                for (int e = 0; e < E; ++e)
                    if (e == label % E) g[e] = at_label;
            }
            __builtin_nontemporal_store(V::put(g), (typename V::raw*)(d + (size_t)i * E));
        }
    }
    if (odd < vocab) store_f32(d + odd, odd == label ? at_label : per_e * exp_below(load_f32(x + odd) - top));
}

template <typename T, int KIND, bool SMALL>
__device__ __forceinline__ void long_row_of_loss(const LossLaunch& l, const PolicyArgs& p) {
    typedef Vec<T> V;
    constexpr int W = kLongThreads / 64, E = V::N;
    __shared__ float s_max[W];
    __shared__ double s_sum[W], s_slope;
    __shared__ int s_n[W];
    const int row = blockIdx.x, tid = threadIdx.x, label = l.labels[row], vocab = l.vocab;
    const T* x = (const T*)l.logits + (size_t)row * l.logits_stride;
    T* d = l.dlogits ? (T*)l.dlogits + (size_t)row * l.dlogits_stride : nullptr;
    if (!row_counts(label, vocab)) return row_left_out<T, KIND, kLongThreads>(l, p, row, label, d);
    const float x_label = load_f32(x + label);
    const int whole = vocab / E, odd = whole * E + tid;
    float mx = odd < vocab && odd != label ? load_f32(x + odd) : -INFINITY;
    double sum = mx == -INFINITY ? 0.0 : (double)exp_below(mx - mx);
    for (int at = tid; at < whole; at += kLongThreads * kLongVecs) {
        float v[kLongVecs * E];
        float m = mx;
        typename V::raw q[kLongVecs];
#pragma unroll
        for (int j = 0; j < kLongVecs; ++j)
            if (at + j * kLongThreads < whole) q[j] = *(const typename V::raw*)(x + (size_t)(at + j * kLongThreads) * E);
#pragma unroll
        for (int j = 0; j < kLongVecs; ++j) {
            if (at + j * kLongThreads < whole) {
                V::get(q[j], v + j * E);
            } else {
#pragma unroll
                for (int e = 0; e < E; ++e) v[j * E + e] = -INFINITY;
            }
            if (at + j * kLongThreads == label / E) {
#pragma unroll
                for (int e = 0; e < E; ++e)
                    if (e == label % E) v[j * E + e] = -INFINITY;
            }
#pragma unroll
            for (int e = 0; e < E; ++e) m = fmaxf(m, v[j * E + e]);
        }
        const float base = m == -INFINITY ? 0.f : m;
        if (mx != -INFINITY) sum *= exp_below(mx - base);
        mx = m;
        float part[2] = {0.f, 0.f};
#pragma unroll
        for (int i = 0; i < kLongVecs * E; ++i) part[i & 1] += exp_below(v[i] - base);
        sum += (double)part[0] + part[1];
    }
    float top = mx;
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor(top, o, 64));
    if (mx != -INFINITY) sum *= exp_below(mx - top);
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) sum += __shfl_xor(sum, o, 64);
    // the mean's divisor: counted here in a small call, by a launch in front in a large one
    if (SMALL && KIND != LOSS_PREF && l.mean && d) {
        const int n = count_rows<kLongThreads>(l);
        if ((tid & 63) == 0) s_n[tid >> 6] = n;
    }
    float factor;
    const RowFacts f = join_waves<W>(top, sum, x_label, &factor, s_max, s_sum);
    if (KIND == LOSS_PREF || !d) {
        if (tid == 0) row_outputs<KIND>(l, p, row, f, x_label);
        return;
    }
    const int n = !l.mean ? 1 : SMALL ? sum_of<W>(s_n) : *l.n_terms;
    const double c = row_coefficient<KIND>(l, p, row, f, x_label, n, &s_slope) / f.total;
    long_gradient<T, kLongThreads>(x, d, vocab, label, f.top, (float)-c, (float)(c * f.others));
    if (KIND == LOSS_SAR && tid == 0) row_outputs<KIND>(l, p, row, f, x_label);
}

template <typename T, int KIND, bool SMALL>
__global__ __launch_bounds__(kLongThreads) void loss_long_rows_kernel(LossLaunch l, PolicyArgs p) {
    long_row_of_loss<T, KIND, SMALL>(l, p);
    if (SMALL) finish_rows<kLongThreads>(l, p);
}

// How many rows count, for the mean that the rows' gradients need before the rows are done.
__global__ __launch_bounds__(1024) void loss_count_kernel(LossLaunch l) {
    __shared__ int s[16];
    const int n = count_rows<1024>(l);
    if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = n;
    __syncthreads();
    if (threadIdx.x != 0) return;
    int all = 0;
    for (int w = 0; w < 16; ++w) all += s[w];
    *l.n_terms = all;
}
__global__ __launch_bounds__(1024) void loss_sum_kernel(LossLaunch l, int32_t* n_clipped) { sum_rows<1024, false>(l, n_clipped); }
__global__ __launch_bounds__(1024) void pref_pairs_kernel(LossLaunch l, PrefArgs p) {
    if (l.dlogits) {  // rows of no sequence
        const int from = p.seq_start[0], to = p.seq_start[2 * p.pairs];
        for (int r = blockIdx.x * 1024 + threadIdx.x; r < l.rows; r += gridDim.x * 1024)
            if (r < from || r >= to) l.work[r].v[3] = 0.f;
        join_pairs<true>(l, p, blockIdx.x * kPairs);
    } else {
        join_pairs<false>(l, p, blockIdx.x * kPairs);
    }
}
__global__ __launch_bounds__(1024) void pref_sum_kernel(LossLaunch l, PrefArgs p) { sum_pairs(l, p); }

// The gradient of the preference loss, a row to a workgroup.  A row's coefficient is known when its whole pair has been read, so the
// logits are read twice; the last rows first, which the memory-side cache still holds from the first time (6820 rows of 32000 in
// bf16, six in ten counting: the whole call 158 us, first rows first 160; 3000 rows in fp32 127 and 128).  The row's factors are rounded to 32
// bits before their product is: 1.5 units in the last place of a 32-bit gradient, beside the exponential's own.
template <typename T, int THREADS>
__device__ __forceinline__ void pref_row(const LossLaunch& l, int row, int label, float slope) {
    T* d = (T*)l.dlogits + (size_t)row * l.dlogits_stride;
    if (!row_counts(label, l.vocab) || slope == 0.f) return row_zero<T, THREADS>(d, l.vocab);
    const f32x4_raw f = l.work[row];
    long_gradient<T, THREADS>((const T*)l.logits + (size_t)row * l.logits_stride, d, l.vocab, label, f.v[0], -slope * f.v[1], slope * f.v[2]);
}
template <typename T, int THREADS>
__global__ __launch_bounds__(THREADS) void pref_gradient_kernel(LossLaunch l) {
    const int row = l.rows - 1 - blockIdx.x;
    pref_row<T, THREADS>(l, row, l.labels[row], l.work[row].v[3]);
}
// A call of up to kPairs pairs and kPrefSmall rows does without a launch for the pairs: every row's workgroup adds up the two sequences
// itself, a wave each, and one workgroup more writes what the pairs give out (43 rows of 32000 in bf16 13.8 -> 12.6 us; from a
// workgroup per CU on it costs more than the launch: 803 rows of 5003 in fp32 16.7 -> 20.0).
constexpr int kPrefSmall = 256;
template <typename T>
__global__ __launch_bounds__(1024) void pref_small_kernel(LossLaunch l, PrefArgs p) {
    if (blockIdx.x == 0) return join_pairs<false>(l, p, 0);  // (first, as it takes longest)
    __shared__ SeqSum s_seq[2];
    __shared__ float s_slope;
    const int row = l.rows - blockIdx.x, label = l.labels[row], wave = threadIdx.x >> 6;
    int seq = -1;  // the row's sequence: how many begin at or in front of it
    for (int i = 0; i <= 2 * p.pairs; ++i) seq += p.seq_start[i] <= row;
    float slope = 0.f;
    if (row_counts(label, l.vocab) && seq >= 0 && seq < 2 * p.pairs) {  // (all threads)
        if (wave < 2) {
            const SeqSum q = sum_sequence(l, p, (seq & ~1) + wave);
            if ((threadIdx.x & 63) == 0) s_seq[wave] = q;
        }
        __syncthreads();
        if (wave == 0) {
            const PairTerm t = pair_term(l, p, against_reference(p, seq & ~1, s_seq[0].sum), against_reference(p, seq | 1, s_seq[1].sum));
            if (threadIdx.x == 0) s_slope = row_slope_of(p, t, seq & 1, s_seq[seq & 1].n);
        }
        __syncthreads();
        slope = s_slope;
    }
    pref_row<T, 1024>(l, row, label, slope);
}
// (threads: 8000 rows of 2000 in bf16 32 us with 64, 44 with 1024, statistics included; 8000 of 4000 in fp32 73 with 256, 75 with 128; 4000 of
// 12000 in bf16 57.7 with 1024, 60.6 with 256)
template <typename T>
hipError_t launch_pref_gradient(const LossLaunch& l, hipStream_t s) {
    const dim3 grid(l.rows);
    if (l.vocab <= 64 * 32) hipLaunchKernelGGL((pref_gradient_kernel<T, 64>), grid, dim3(64), 0, s, l);
    else if (l.vocab <= 256 * 32) hipLaunchKernelGGL((pref_gradient_kernel<T, 256>), grid, dim3(256), 0, s, l);
    else hipLaunchKernelGGL((pref_gradient_kernel<T, 1024>), grid, dim3(1024), 0, s, l);
    return hipGetLastError();
}

// Threads and elements a thread by the row's length, so that few registers stay empty and two rows or more fit a CU (us, this / next best):
// 6001 rows of 2000 in fp32 64 x 32 17.0, 128 x 16 20.1; of 4000 128 x 32 36.7, 64 x 64 38.9 (bf16 21.0, 20.3); 2000 rows of 5003 128 x 64
// 15.6, 256 x 32 16.5; of 12000 256 x 64 34.8, 512 x 32 36.7 (4000 in bf16 36.6, 42.8); 4096 of 32000 512 x 64 182, 1024 x 32 209; 2000
// of 64000 in fp32 1024 x 64 189, 512 x 128 200, in bf16 packed 512 x 128 98, unpacked 1024 x 64 107; 1000 of 128256 in bf16 packed 1024 x
// 128 115, read twice 139, without gradient 76 and 68: statistics alone are read in pieces from there on.
template <typename T, int KIND, bool SMALL>
hipError_t launch_rows_of(const LossLaunch& l, const PolicyArgs& p, hipStream_t s) {
    constexpr int E = Vec<T>::N;
    const dim3 grid(l.rows);
#define SPACE_ROWS(THREADS, ELEMS, KEEP) \
    hipLaunchKernelGGL((loss_rows_kernel<T, KIND, THREADS, (ELEMS) / E, KEEP, SMALL>), grid, dim3(THREADS), 0, s, l, p)
    if (l.vocab <= 64 * 32) {
        SPACE_ROWS(64, 32, true);
    } else if (l.vocab <= 128 * 32) {
        SPACE_ROWS(128, 32, true);
    } else if (l.vocab <= 128 * 64) {
        SPACE_ROWS(128, 64, true);
    } else if (l.vocab <= 256 * 64) {
        SPACE_ROWS(256, 64, true);
    } else if (l.vocab <= 512 * 64) {
        SPACE_ROWS(512, 64, true);
    } else {
        if constexpr (sizeof(T) == 4) {
            if (l.vocab <= 1024 * 64) {
                SPACE_ROWS(1024, 64, true);
                return hipGetLastError();
            }
        } else {
            if (l.vocab <= 512 * 128) {
                SPACE_ROWS(512, 128, false);
                return hipGetLastError();
            }
            if constexpr (KIND != LOSS_PREF) {
                if (l.vocab <= 1024 * 128) {
                    SPACE_ROWS(1024, 128, false);
                    return hipGetLastError();
                }
            }
        }
        hipLaunchKernelGGL((loss_long_rows_kernel<T, KIND, SMALL>), grid, dim3(kLongThreads), 0, s, l, p);
    }
#undef SPACE_ROWS
    return hipGetLastError();
}
template <int KIND, bool SMALL>
hipError_t launch_rows(const LossLaunch& l, const PolicyArgs& p, hipStream_t s) {
    return l.dtype == 0 ? launch_rows_of<float, KIND, SMALL>(l, p, s) : launch_rows_of<uint16_t, KIND, SMALL>(l, p, s);
}

// Whether the rows' workgroups count and add up themselves.  That saves two launches (one where nothing has to be counted first), 3 -
// 4 us, but every workgroup reads all labels, and adds to one count, 13 ns each: the longer a row takes the less of either shows, so
// the rows may be as many as the square of their bytes allows.  In one launch / apart, mean, all rows counting: 32000 in fp32
// 1000 rows 47.0 / 49.9 us, 2900 134 / 138, 4000 181 / 186 (policy 189 / 185); in bf16 1000 rows 31.3 / 32.1, 2000 58.8 / 55.8,
// 4000 114 / 100; short rows win up to about 200 (of 1000 in fp32: 200 8.2 / 9.0, 500 11.0 / 9.3, 2000 30 / 12).
bool small_call(const LossLaunch& l) {
    const int64_t bytes = min((int64_t)l.vocab * (l.dtype ? 2 : 4), (int64_t)1 << 20);
    return l.rows <= 192 || (l.rows <= 4096 && ((int64_t)l.rows << 22) <= bytes * bytes);
}

template <int KIND>
hipError_t launch_loss(const LossLaunch& l, const PolicyArgs& p, hipStream_t s) {
    if (small_call(l)) return launch_rows<KIND, true>(l, p, s);
    if (l.mean && l.dlogits) {
        hipLaunchKernelGGL(loss_count_kernel, dim3(1), dim3(1024), 0, s, l);
        if (hipError_t e = hipGetLastError()) return e;
    }
    if (hipError_t e = launch_rows<KIND, false>(l, p, s)) return e;
    hipLaunchKernelGGL(loss_sum_kernel, dim3(1), dim3(1024), 0, s, l, p.n_clipped);
    return hipGetLastError();
}

hipError_t launch_sar_grad(const LossLaunch& l, hipStream_t s) { return launch_loss<LOSS_SAR>(l, PolicyArgs{}, s); }
hipError_t launch_policy(const LossLaunch& l, const PolicyArgs& p, hipStream_t s) { return launch_loss<LOSS_POLICY>(l, p, s); }

hipError_t launch_preference(const LossLaunch& l, const PrefArgs& p, hipStream_t s) {
    if (hipError_t e = launch_rows<LOSS_PREF, false>(l, PolicyArgs{}, s)) return e;
    if (l.dlogits && l.rows <= kPrefSmall && p.pairs <= kPairs) {
        const dim3 grid(l.rows + 1);
        if (l.dtype == 0) hipLaunchKernelGGL(pref_small_kernel<float>, grid, dim3(1024), 0, s, l, p);
        else hipLaunchKernelGGL(pref_small_kernel<uint16_t>, grid, dim3(1024), 0, s, l, p);
        return hipGetLastError();
    }
    const int wgs = (p.pairs + kPairs - 1) / kPairs;
    hipLaunchKernelGGL(pref_pairs_kernel, dim3(wgs), dim3(1024), 0, s, l, p);
    if (hipError_t e = hipGetLastError()) return e;
    if (wgs > 1) {
        hipLaunchKernelGGL(pref_sum_kernel, dim3(1), dim3(1024), 0, s, l, p);
        if (hipError_t e = hipGetLastError()) return e;
    }
    if (!l.dlogits) return hipSuccess;
    return l.dtype == 0 ? launch_pref_gradient<float>(l, s) : launch_pref_gradient<uint16_t>(l, s);
}

// ------------------------------------------------------------------------------------------
// gradient norm and clipping
// ------------------------------------------------------------------------------------------
// A launch takes up to kGradList tensors by value (arguments of a kernel: 4 KB at most), so nothing has to be kept on the device; their
// elements are cut into chunks that are dealt out to the workgroups in turn.
constexpr int kGradList = 152, kGradThreads = 256, kGradChunk = kGradThreads * 32, kGradChunks = 1 << 30;
struct GradList {
    const void* grad[kGradList];
    void* out[kGradList];
    int32_t first[kGradList + 1];  // chunks in front of a tensor, up to kGradChunks
    int32_t last[kGradList];       // elements of its last chunk; bit 14: bf16 gradient, bit 15: bf16 output (16 bits would take a vector load)
    int count;
};
static_assert(sizeof(GradList) <= 3700 && kGradChunk < 1 << 14, "arguments of a kernel, elements of a chunk");

__device__ __forceinline__ int grad_tensor_of(const GradList& g, int chunk) {
    int lo = 0, hi = g.count - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (g.first[mid] <= chunk) lo = mid; else hi = mid - 1;
    }
    return lo;
}
__device__ __forceinline__ int chunk_elements(const GradList& g, int t, int chunk) { return chunk + 1 < g.first[t + 1] ? kGradChunk : g.last[t] & 0x3fff; }

// What both passes over the gradients read twice comes from the memory-side cache the second time, if it is small enough: the
// last kGradKept bytes are read in the ordinary way by the norm, and first by the clipping; everything in front of them, which the
// cache would lose again, is read past it.  Norm and clipping of 49 M gradients in fp32 113 -> 87 us against reading past the cache
// throughout, of 435 M 969 -> 936; of the 256 MB of the cache 240 are best (247 MB of gradients: 192 / 224 / 240 / 256 MB 132 /
// 127 / 118 / 118 us, 320 MB: 150 / 147 / 151 / 159).
constexpr int64_t kGradKept = 240ll << 20;
// The squares of n elements of a chunk, this thread's share.  A square is exact in 64 bits for both types, and no sum of them leaves the range.
template <typename T, bool KEPT>
__device__ __forceinline__ double chunk_squares(const T* __restrict__ x, int n) {
    typedef Vec<T> V;
    constexpr int E = V::N, NV = kGradChunk / kGradThreads / E;
    double sum[2] = {0.0, 0.0};
    const int tid = threadIdx.x % kGradThreads, whole = n / E, odd = whole * E + tid;
    typename V::raw q[NV];
#pragma unroll
    for (int j = 0; j < NV; ++j)
        if (tid + j * kGradThreads < whole) q[j] = read_vec<KEPT, V>(x + (tid + j * kGradThreads) * E);
    if (odd < n) {
        const double v = load_f32(x + odd);
        sum[0] = v * v;
    }
#pragma unroll
    for (int j = 0; j < NV; ++j)
        if (tid + j * kGradThreads < whole) {
            float v[E];
            V::get(q[j], v);
#pragma unroll
            for (int e = 0; e < E; ++e) sum[e & 1] = fma((double)v[e], (double)v[e], sum[e & 1]);
        }
    return sum[0] + sum[1];
}

// One chunk after another, dealt out to the workgroups; those from kept_from on stay in the cache.
template <bool KEPT>
__device__ __forceinline__ double list_squares(const GradList& g, int c, int end, int step) {
    double sum = 0.0;
    for (; c < end; c += step) {
        const int t = grad_tensor_of(g, c), n = chunk_elements(g, t, c);
        const int64_t from = (int64_t)(c - g.first[t]) * kGradChunk;
        if (g.last[t] & 0x4000) sum += chunk_squares<uint16_t, KEPT>((const uint16_t*)g.grad[t] + from, n);
        else sum += chunk_squares<float, KEPT>((const float*)g.grad[t] + from, n);
    }
    return sum;
}
template <int THREADS, bool SMALL>
__device__ __forceinline__ void sum_squares(const double* work, int parts, float* norm, double* s) {
    double sum = 0.0;
    for (int i = threadIdx.x; i < parts; i += THREADS) sum += SMALL ? __hip_atomic_load(work + i, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) : work[i];
    sum = block_sum<THREADS / 64>(sum, s);
    if (threadIdx.x == 0) *norm = (float)sqrt(sum);
}
// A workgroup takes CHUNKS chunks at a time, kGradThreads threads each.  LAST: a lone launch of few workgroups, the last of which takes the
// root; else a launch behind them does.
template <int CHUNKS, bool LAST>
__global__ __launch_bounds__(kGradThreads * CHUNKS) void grad_square_kernel(GradList g, int kept_from, double* work, int first_launch, uint32_t* arrived,
                                                                            float* norm) {
    constexpr int THREADS = kGradThreads * CHUNKS;
    __shared__ double s[THREADS / 64];
    __shared__ int s_last;
    // (the same for all threads of a wave)
    const int mine = blockIdx.x * CHUNKS + __builtin_amdgcn_readfirstlane(threadIdx.x / kGradThreads), step = gridDim.x * CHUNKS;
    double sum = list_squares<false>(g, mine, kept_from, step);
    const int turns = max(kept_from - mine + step - 1, 0) / step;  // how many of those these threads had
    sum += list_squares<true>(g, mine + turns * step, g.first[g.count], step);
    sum = block_sum<THREADS / 64>(sum, s);
    if (threadIdx.x == 0) __hip_atomic_store(work + blockIdx.x, first_launch ? sum : work[blockIdx.x] + sum, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    if (LAST && arrive(arrived, &s_last)) sum_squares<THREADS, true>(work, gridDim.x, norm, s);
}
__global__ __launch_bounds__(1024) void grad_norm_kernel(const double* work, int parts, float* norm) {
    __shared__ double s[16];
    sum_squares<1024, false>(work, parts, norm, s);
}

// Four bf16 numbers, which go with four in fp32: neighbouring lanes' stores meet
struct Vec4Bf16 {
    static constexpr int N = 4;
    typedef uint32_t raw __attribute__((ext_vector_type(2), aligned(2)));
    static __device__ __forceinline__ void get(raw q, float* v) {
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const uint32_t w = q[e];
            v[2 * e] = __uint_as_float(w << 16);
            v[2 * e + 1] = __uint_as_float(w & 0xffff0000u);
        }
    }
    static __device__ __forceinline__ raw put(const float* v) {
        raw q;
#pragma unroll
        for (int e = 0; e < 2; ++e) q[e] = (uint32_t)f2bf(v[2 * e]) | (uint32_t)f2bf(v[2 * e + 1]) << 16;
        return q;
    }
};
template <typename T, typename Other> struct VecBeside { typedef Vec<T> type; };
template <> struct VecBeside<uint16_t, float> { typedef Vec4Bf16 type; };

// n elements of a chunk, scaled.  (All loads, then all arithmetic, then all stores: what stands in one condition with a load or a store
// waits for it, one vector after the other: 667 M bf16 gradients into fp32 932 -> 905 us.)
template <bool KEPT, typename T, typename O>
__device__ __forceinline__ void chunk_scale(const T* x, O* y, int n, float scale) {
    typedef typename VecBeside<T, O>::type In;
    typedef typename VecBeside<O, T>::type Out;
    constexpr int E = In::N, NV = kGradChunk / kGradThreads / E;
    static_assert(In::N == Out::N, "as many elements in as out");
    const int tid = threadIdx.x, whole = n / E, odd = whole * E + tid;
    typename In::raw q[NV];
    typename Out::raw r[NV];
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        q[j] = typename In::raw{};
        if (tid + j * kGradThreads < whole) q[j] = read_vec<KEPT, In>(x + (tid + j * kGradThreads) * E);
    }
    if (odd < n) store_f32(y + odd, load_f32(x + odd) * scale);
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        float v[E];
        In::get(q[j], v);
#pragma unroll
        for (int e = 0; e < E; ++e) v[e] *= scale;
        r[j] = Out::put(v);
    }
#pragma unroll
    for (int j = 0; j < NV; ++j)
        if (tid + j * kGradThreads < whole) __builtin_nontemporal_store(r[j], (typename Out::raw*)(y + (tid + j * kGradThreads) * E));
}

template <bool KEPT>
__global__ __launch_bounds__(kGradThreads) void grad_clip_kernel(GradList g, int begin, int end, const float* norm, float max_norm) {
    const float size = *norm;
    const float scale = size > max_norm && size < INFINITY ? max_norm / size : 1.f;
    for (int c = begin + blockIdx.x; c < end; c += gridDim.x) {
        const int t = grad_tensor_of(g, c), n = chunk_elements(g, t, c);
        if (scale == 1.f && g.out[t] == g.grad[t]) continue;
        const int64_t from = (int64_t)(c - g.first[t]) * kGradChunk;
        const void* x = g.grad[t];
        void* y = g.out[t];
        switch (g.last[t] >> 14) {
            case 0: chunk_scale<KEPT>((const float*)x + from, (float*)y + from, n, scale); break;
            case 1: chunk_scale<KEPT>((const uint16_t*)x + from, (float*)y + from, n, scale); break;
            case 2: chunk_scale<KEPT>((const float*)x + from, (uint16_t*)y + from, n, scale); break;
            default: chunk_scale<KEPT>((const uint16_t*)x + from, (uint16_t*)y + from, n, scale); break;
        }
    }
}

int64_t grad_bytes(const GradTensor& t) { return t.n * (t.dtype ? 2 : 4); }

// Calls launch(list, first chunk that is kept) for every kGradList tensors that are not empty (fewer where they have too many chunks).
template <typename F>
hipError_t each_grad_list(const GradTensor* t, int n, F launch) {
    int64_t left = -kGradKept;  // bytes still in front of those that are kept
    for (int i = 0; i < n; ++i) left += grad_bytes(t[i]);
    GradList g;
    for (int i = 0; i < n;) {
        g.count = 0;
        g.first[0] = 0;
        int kept_from = 0;
        for (; i < n && g.count < kGradList; ++i) {
            if (t[i].n == 0) continue;
            const int64_t chunks = (t[i].n + kGradChunk - 1) / kGradChunk;
            if (g.first[g.count] + chunks > kGradChunks) break;  // (a lone tensor has fewer: grad_list)
            const int c = g.count++;
            g.grad[c] = t[i].grad;
            g.out[c] = t[i].out;
            g.last[c] = (int)(t[i].n - (chunks - 1) * kGradChunk) | t[i].dtype << 14 | t[i].out_dtype << 15;
            g.first[c + 1] = g.first[c] + (int)chunks;
            if (left > 0) {
                const int64_t bytes = kGradChunk * (t[i].dtype ? 2 : 4), past = (left + bytes - 1) / bytes;
                kept_from = g.first[c] + (int)(past < chunks ? past : chunks);
            }
            left -= grad_bytes(t[i]);
        }
        if (!g.count) break;
        launch(g, kept_from);
        if (hipError_t e = hipGetLastError()) return e;
    }
    return hipSuccess;
}

int grad_workgroups(int chunks) { return chunks < kGradParts ? chunks : kGradParts; }

// Chunks up to which the last workgroup takes the root itself: one launch less, but each workgroup adds to one count, 14 ns, so from kGradSingle
// on a workgroup takes two chunks at a time (us of norm and clipping in replayed graphs, one / two / a launch behind: 16 chunks 8.1 / 8.3 / 9.0, 48 8.5 / 8.7 /
// 9.2, 96 9.1 / 8.9 / 9.2, 192 10.4 / 9.7 / 9.5, 288 12.1 / 10.4 / 10.0, 384 13.3 / 12.0 / 10.1).  On the GPU alone two and a launch behind
// cross at 170 (behind other work 128 11.3 / 11.6, 192 11.8 / 11.6, 288 12.8 / 12.4, 384 13.8 / 12.7); where the host's launches are waited for, a
// call by itself at 320 (192 23.2 / 24.1, 288 24.1 / 24.4, 320 24.4 / 24.4, 384 25.0 / 24.4) and calls in a row later (320 12.7 / 15.3, 512 14.8 /
// 15.3).  The border is that of a call by itself, in which both count.
constexpr int kGradSingle = 64, kGradSmall = 320;

hipError_t launch_grad_norm(const GradTensor* t, int n, float* norm, double* work, hipStream_t s) {
    uint32_t* arrived = (uint32_t*)work;
    work += 2;
    // a later launch adds to the partial sums of an earlier one, so all of them have as many workgroups
    int chunks = 0, lists = 0, first = 1;
    hipError_t e = each_grad_list(t, n, [&](const GradList& g, int) {
        chunks = max(chunks, g.first[g.count]);
        ++lists;
    });
    if (e != hipSuccess) return e;
    const bool small = lists == 1 && chunks <= kGradSmall;
    const int parts = !small ? grad_workgroups(chunks) : chunks <= kGradSingle ? chunks : (chunks + 1) / 2;
    e = each_grad_list(t, n, [&](const GradList& g, int kept_from) {
        const auto kernel = !small ? grad_square_kernel<1, false> : chunks <= kGradSingle ? grad_square_kernel<1, true> : grad_square_kernel<2, true>;
        hipLaunchKernelGGL(kernel, dim3(parts), dim3(small && chunks > kGradSingle ? 2 * kGradThreads : kGradThreads), 0, s, g, kept_from, work, first, arrived, norm);
        first = 0;
    });
    if (e != hipSuccess || small) return e;
    hipLaunchKernelGGL(grad_norm_kernel, dim3(1), dim3(1024), 0, s, work, parts, norm);
    return hipGetLastError();
}

hipError_t launch_grad_clip(const GradTensor* t, int n, const float* norm, float max_norm, hipStream_t s) {
    const hipError_t e = each_grad_list(t, n, [&](const GradList& g, int kept_from) {
        const int end = g.first[g.count];
        if (kept_from < end) hipLaunchKernelGGL(grad_clip_kernel<true>, dim3(grad_workgroups(end - kept_from)), dim3(kGradThreads), 0, s, g, kept_from, end, norm, max_norm);
    });
    if (e != hipSuccess) return e;
    return each_grad_list(t, n, [&](const GradList& g, int kept_from) {
        if (kept_from > 0) hipLaunchKernelGGL(grad_clip_kernel<false>, dim3(grad_workgroups(kept_from)), dim3(kGradThreads), 0, s, g, 0, kept_from, norm, max_norm);
    });
}

}  // namespace space
