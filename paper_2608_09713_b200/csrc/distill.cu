// Distillation from a teacher's top logits: rows of ids and teacher's logits z (CSR) meet dense rows of a student's logits s.
// With x = s / tau, lse = log sum_v exp(x_v), q_v = exp(x_v - lse), p_t = exp(z_t / tau - L):
//     loss = scale r (sum_t p_t (z_t - s_t) / tau + P (lse - L)),      G_v = scale r / tau (P q_v - sum of the p_t with id v).
//
// Bound by memory: the logits are read once (running maximum and sum, no second pass for the maximum), and the gradient written once; when
// both are asked for, the row is read again for the gradient as soon as its sum is known, while it still lies in L2 (a row is
// 16 KB to 1 MB, those in flight together are far below 126 MB).  A cluster of 1 to 8 CTAs takes a row, so that few rows still use
// many SMs.  exp(x) is computed as 2^(s * log2(e) / tau - ...), one multiply-add and one exponential per logit.
// The gradient is first written for all ids as if they were not the teacher's, then the few of the teacher's are overwritten, from
// logits that were fetched beforehand (so the gradient may overwrite the logits).  An id that occurs more than once is
// written by its first entry, with the sum of its entries in their order: they are found with a hash table in shared memory.  Rows of
// more than TOP entries go through the ids in windows instead.
#include <algorithm>
#include <math_constants.h>

#include "element.cuh"

using namespace spsyrk;

namespace {

constexpr int THREADS = 512;
constexpr int WARPS = THREADS / 32;
constexpr int TOP = 1024;         // teacher's entries of a row that are kept in shared memory
constexpr int TABLE = 2 * TOP;    // slots of the hash table; of a window's ids in rows of more entries
constexpr int SMS = 148;
constexpr int NONE = 0x7fffffff;
constexpr double LOG2E = 1.4426950408889634, LN2 = 0.6931471805599453;

struct Teacher {
    const int32_t* ids;
    const void* z;
    spsyrk_dtype_t dtype;
    const float* lse;
    __device__ __forceinline__ float logit(int64_t t) const {
        return dtype == SPSYRK_F32 ? static_cast<const float*>(z)[t]
               : dtype == SPSYRK_BF16 ? widen(static_cast<const __nv_bfloat16*>(z)[t]) : widen(static_cast<const __half*>(z)[t]);
    }
};

// 2^v; 0 below the range, relative error 2^-22 (the PTX ISA's bound for ex2.approx.ftz.f32)
__device__ __forceinline__ float power_of_two(float v) {
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
    return r;
}

// The sum of 2^(k s) over logits s, k = log2(e) / tau, as sum * 2^at: `most` is the largest logit so far (-infinity if there was
// none) and at = most * k, rounded, is what the exponents are taken relative to: rounding it moves nothing, since the terms, the
// changes of `most` and the logarithm at the end all use the same number.  Logits beyond LARGE, whose products could overflow (rows masked
// with the lowest value throughout), go by (s - most) * k instead.
struct Running {
    float most, sum;
};
constexpr float LARGE = 1e30f;
__device__ __forceinline__ float base_of(float most) { return most == -CUDART_INF_F ? 0.f : most; }  // nothing but -infinity: terms of 0, or NaN
__device__ __forceinline__ float step_down(float from, float to, float k) {  // the factor when `most` goes from one to the other
    if (fabsf(to) < LARGE && fabsf(from) < LARGE) return power_of_two(__fmul_rn(from, k) - __fmul_rn(to, k));
    return power_of_two((from - to) * k);
}
template <int N>
__device__ __forceinline__ void take(Running& r, const float (&s)[N], float k) {
    float top = s[0];
#pragma unroll
    for (int i = 1; i < N; ++i) top = fmaxf(top, s[i]);
    if (top > r.most) {
        r.sum *= step_down(r.most, top, k);  // most = -infinity: times 0
        r.most = top;
    }
    const float b = base_of(r.most), at = __fmul_rn(b, k);
    if (fabsf(b) < LARGE) {
#pragma unroll
        for (int i = 0; i < N; ++i) r.sum += power_of_two(fmaf(s[i], k, -at));
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) r.sum += power_of_two((s[i] - b) * k);
    }
}
__device__ __forceinline__ Running merge(Running a, Running b, float k) {
    const float top = fmaxf(a.most, b.most), to = base_of(top);
    return Running{top, a.sum * step_down(a.most, to, k) + b.sum * step_down(b.most, to, k)};
}

// Sums and maxima over a CTA; every thread gets the result.  `scratch`: WARPS values that nothing else uses meanwhile.
template <typename V, typename Op>
__device__ __forceinline__ V over_cta(V v, V* scratch, Op op) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v = op(v, __shfl_xor_sync(FULL_MASK, v, o));
    __syncthreads();
    if (lane_id() == 0) scratch[threadIdx.x >> 5] = v;
    __syncthreads();
    v = scratch[0];
#pragma unroll
    for (int w = 1; w < WARPS; ++w) v = op(v, scratch[w]);
    return v;
}

// The columns [0, n) of a row in this CTA's share: [v0, v1) in units of W elements from the first 16-byte boundary, and, for the
// first CTA, the `head` elements before it and the elements behind the last unit.
struct Share {
    int64_t head, v0, v1, tail;
};
template <typename T>
__device__ __forceinline__ Share share_of(const T* row, int64_t n, uint32_t rank, uint32_t size) {
    constexpr int W = 16 / (int)sizeof(T);
    Share s;
    s.head = min(n, (int64_t)((0 - reinterpret_cast<uintptr_t>(row)) % 16 / sizeof(T)));
    const int64_t units = (n - s.head) / W, each = (units + size - 1) / size;
    s.v0 = min(units, rank * each);
    s.v1 = min(units, s.v0 + each);
    s.tail = s.head + units * W;
    return s;
}

struct Call {
    Rows rows;
    int64_t n;
    Teacher teacher;
    const float* row_weights;
    float k, inv_tau;   // log2(e) / tau, 1 / tau
    double scale, inv_tau_d;
    int64_t ldl, ldg;
    float *loss, *lse;
    const float* kept;  // the rows' lse of an earlier call (gradient only)
};

// FORWARD: the sum over the row is computed (else it is `kept`); GRAD: the gradient is written.
template <typename T, bool FORWARD, bool GRAD>
__global__ void __launch_bounds__(THREADS, 2) distill_kernel(const Call c, const T* logits, T* grad) {
    constexpr int W = 16 / (int)sizeof(T), U = 4;
    __shared__ int32_t s_id[TOP];
    __shared__ float s_p[TOP], s_at[TOP];  // exp(z / tau - largest), the student's logit
    __shared__ int32_t table[TABLE];
    __shared__ double s_d[WARPS];
    __shared__ float s_f[WARPS];
    __shared__ float2 s_part[WARPS + 1];
    const uint32_t rank = cluster_rank(), size = cluster_size();
    const int64_t row = blockIdx.x / size;
    const int tid = threadIdx.x;
    const T* const s = logits + row * c.ldl;
    T* const g = GRAD ? grad + row * c.ldg : nullptr;
    const float weight = c.row_weights ? c.row_weights[row] : 1.f;
    const int64_t e0 = c.rows.begin(row), entries = max((int64_t)0, c.rows.end(row) - e0);
    const bool few = entries <= TOP;

    // the teacher's row: largest logit, sum of exponentials
    float top = -CUDART_INF_F;
    bool any = false;  // an id of the vocabulary with a logit other than -infinity
    if (weight != 0.f) {
        for (int64_t t = tid; t < entries; t += THREADS) {
            const int32_t id = c.teacher.ids[e0 + t];
            const bool held = id >= 0 && id < c.n;
            const float z = held ? c.teacher.logit(e0 + t) : -CUDART_INF_F;
            any |= z != -CUDART_INF_F;
            top = fmaxf(top, z);
            if (few) {
                s_id[t] = held ? id : -1;
                s_p[t] = z;
                s_at[t] = held ? widen(s[id]) : 0.f;
            }
        }
    }
    const bool live = __syncthreads_or(any);
    const Share mine = share_of(s, c.n, rank, size);
    if (!live) {  // (the same for the whole cluster)
        if (tid == 0 && rank == 0 && FORWARD) {
            if (c.loss) c.loss[row] = 0.f;
            if (c.lse) c.lse[row] = 0.f;
        }
        if (GRAD) {
            const int64_t w0 = rank == 0 ? 0 : mine.head + mine.v0 * W, w1 = mine.head + mine.v1 * W;
            for (int64_t v = w0 + tid; v < w1; v += THREADS) g[v] = narrow<T>(0.f);
            if (rank == 0)
                for (int64_t v = mine.tail + tid; v < c.n; v += THREADS) g[v] = narrow<T>(0.f);
        }
        return;
    }
    top = base_of(over_cta(top, s_f, [](float a, float b) { return fmaxf(a, b); }));
    double total = 0;  // sum of e_t = exp((z_t - top) / tau)
    for (int64_t t = tid; t < entries; t += THREADS) {
        float e = 0.f;
        if (few) {
            if (s_id[t] >= 0) e = expf((s_p[t] - top) * c.inv_tau);
            s_p[t] = e;
        } else {
            const int32_t id = c.teacher.ids[e0 + t];
            if (id >= 0 && id < c.n) e = expf((c.teacher.logit(e0 + t) - top) * c.inv_tau);
        }
        total += (double)e;
    }
    const auto sum = [](double a, double b) { return a + b; };
    total = over_cta(total, s_d, sum);
    // p_t = e_t * unit, mass P
    const double log_unit = c.teacher.lse ? (double)top * c.inv_tau_d - (double)c.teacher.lse[row] : -log(total);
    const double unit = c.teacher.lse ? exp(log_unit) : 1.0 / total;
    const double mass = c.teacher.lse ? total * unit : total / total;  // (1, or NaN)

    Running r{-CUDART_INF_F, 0.f};
    double lse;
    if (FORWARD) {
        for (int64_t v = mine.v0 + tid; v < mine.v1; v += (int64_t)U * THREADS) {
            Vec<T, W> x[U];
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (v + u * THREADS < mine.v1) x[u] = *reinterpret_cast<const Vec<T, W>*>(s + mine.head + (v + u * THREADS) * W);
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (v + u * THREADS >= mine.v1) break;
                float f[W];
#pragma unroll
                for (int i = 0; i < W; ++i) f[i] = widen(x[u].x[i]);
                take<W>(r, f, c.k);
            }
        }
        if (rank == 0) {
            float f[1];
            if (tid < mine.head) {
                f[0] = widen(s[tid]);
                take<1>(r, f, c.k);
            }
            if (mine.tail + tid < c.n) {
                f[0] = widen(s[mine.tail + tid]);
                take<1>(r, f, c.k);
            }
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) r = merge(r, Running{__shfl_xor_sync(FULL_MASK, r.most, o), __shfl_xor_sync(FULL_MASK, r.sum, o)}, c.k);
        if (lane_id() == 0) s_part[tid >> 5] = float2{r.most, r.sum};
        __syncthreads();
        r = Running{s_part[0].x, s_part[0].y};
#pragma unroll
        for (int w = 1; w < WARPS; ++w) r = merge(r, Running{s_part[w].x, s_part[w].y}, c.k);
        if (size > 1) {
            if (tid == 0) s_part[WARPS] = float2{r.most, r.sum};
            cluster_sync();
            const float2 first = load_of_rank(s_part + WARPS, 0);
            r = Running{first.x, first.y};
            for (uint32_t q = 1; q < size; ++q) {
                const float2 other = load_of_rank(s_part + WARPS, q);
                r = merge(r, Running{other.x, other.y}, c.k);
            }
        }
        // log q = (s - b) / tau - rest.  (k is rounded, 1 / tau is not: what the rounding moves b k by is put back.)
        const float b = base_of(r.most);
        const double slip = fabsf(b) < LARGE ? (double)__fmul_rn(b, c.k) - (double)b * (double)c.k : 0.0;
        const double rest = slip * LN2 + log((double)r.sum);
        lse = (double)b * c.inv_tau_d + rest;
        if (rank == 0) {
            double loss = 0;
            for (int64_t t = tid; t < entries; t += THREADS) {
                const int32_t id = few ? s_id[t] : c.teacher.ids[e0 + t];
                if (id < 0 || id >= c.n) continue;
                const float z = c.teacher.logit(e0 + t), at = few ? s_at[t] : widen(s[id]);
                const float e = few ? s_p[t] : expf((z - top) * c.inv_tau);
                if (e != 0.f) loss += (double)e * ((((double)z - (double)top) - ((double)at - (double)b)) * c.inv_tau_d + log_unit + rest);
            }
            loss = over_cta(loss, s_d, sum);
            if (tid == 0) {
                if (c.loss) c.loss[row] = (float)(c.scale * (double)weight * (loss * unit));
                if (c.lse) c.lse[row] = (float)lse;
            }
        }
        if (size > 1) cluster_sync();  // nobody ends, or overwrites logits, before all have read
    } else {
        lse = (double)c.kept[row];
        if (size > 1) cluster_sync();  // nobody overwrites logits before all have fetched the teacher's
    }
    if (!GRAD) return;

    // G_v = a 2^(s k - shift) - (at the teacher's ids) f * (sum of their e_t); what rounding the shift takes away goes into a.  The
    // shift that belongs to a kept lse is that of a logit with q = 1, so that the rounding of k matters to small q only.
    const double factor = c.scale * (double)weight * c.inv_tau_d;
    const float b = FORWARD ? base_of(r.most) : 0.f;
    const bool plain = fabsf(b) < LARGE;
    // a row that was NaN or -infinity throughout is NaN in all places
    const bool sound = FORWARD ? r.sum > 0.f && r.sum < CUDART_INF_F : fabs(lse) < (double)LARGE;
    const double exact = !sound ? (double)CUDART_NAN_F
                         : FORWARD ? (plain ? (double)__fmul_rn(b, c.k) : 0.0) + log2((double)r.sum) : lse / c.inv_tau_d * (double)c.k;
    const float shift = (float)exact;
    const float a = (float)(factor * mass * exp2((double)shift - exact)), f = (float)(factor * unit);
    auto q_of = [&](float x) { return power_of_two(plain ? fmaf(x, c.k, -shift) : (x - b) * c.k - shift); };
    if (few) {
        for (int64_t v = mine.v0 + tid; v < mine.v1; v += (int64_t)U * THREADS) {
            Vec<T, W> x[U];
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (v + u * THREADS < mine.v1) x[u] = *reinterpret_cast<const Vec<T, W>*>(s + mine.head + (v + u * THREADS) * W);
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (v + u * THREADS >= mine.v1) break;
                float y[W];
#pragma unroll
                for (int i = 0; i < W; ++i) y[i] = a * q_of(widen(x[u].x[i]));
                T* const at = g + mine.head + (v + u * THREADS) * W;
                if (reinterpret_cast<uintptr_t>(at) % 16 == 0) {
                    store_narrow<T, W>(at, W, y);
                } else {
#pragma unroll
                    for (int i = 0; i < W; ++i) at[i] = narrow<T>(y[i]);
                }
            }
        }
        if (rank == 0) {
            if (tid < mine.head) g[tid] = narrow<T>(a * q_of(widen(s[tid])));
            if (mine.tail + tid < c.n) g[mine.tail + tid] = narrow<T>(a * q_of(widen(s[mine.tail + tid])));
        }
        // the first entry of every id: slots of the table hold entries, an id's slot its first
        for (int i = tid; i < TABLE; i += THREADS) table[i] = NONE;
        __syncthreads();
        const int count = (int)entries;
        auto slot_of = [](int32_t id) { return (int)(((uint32_t)id * 2654435761u) >> 21); };
        static_assert(TABLE == 1 << 11, "slot_of");
        bool again = false;
        for (int t = tid; t < count; t += THREADS) {
            const int32_t id = s_id[t];
            if (id < 0) continue;
            for (int q = slot_of(id);; q = (q + 1) & (TABLE - 1)) {  // (the table is at most half full)
                const int was = atomicCAS(&table[q], NONE, t);
                if (was == NONE) break;
                if (s_id[was] == id) {
                    atomicMin(&table[q], t);
                    again = true;
                    break;
                }
            }
        }
        again = __syncthreads_or(again);
        const int64_t w0 = rank == 0 ? 0 : mine.head + mine.v0 * W, w1 = mine.head + mine.v1 * W;
        for (int t = tid; t < count; t += THREADS) {
            const int32_t id = s_id[t];
            if (id < 0 || !((id >= w0 && id < w1) || (rank == 0 && id >= mine.tail))) continue;
            float e = s_p[t];
            if (again) {
                int q = slot_of(id);
                while (s_id[table[q]] != id) q = (q + 1) & (TABLE - 1);
                if (table[q] != t) continue;
                for (int o = t + 1; o < count; ++o)
                    if (s_id[o] == id) e += s_p[o];
            }
            g[id] = narrow<T>(fmaf(-e, f, a * q_of(s_at[t])));
        }
        return;
    }
    // Rows of many entries: windows of TABLE ids, in every window the first entry of each id by its place.
    for (int64_t i0 = 0; i0 < c.n; i0 += TABLE) {
        const int64_t i1 = min(i0 + TABLE, c.n);
        if ((i0 / TABLE) % size != rank) continue;
        for (int i = tid; i < TABLE; i += THREADS) table[i] = NONE;
        if (tid == 0) s_id[0] = 0;
        __syncthreads();
        for (int64_t t = tid; t < entries; t += THREADS) {
            const int32_t id = c.teacher.ids[e0 + t];
            if (id < i0 || id >= i1) continue;
            if (atomicMin(&table[id - i0], (int)t) != NONE) s_id[0] = 1;
        }
        __syncthreads();
        const bool again = s_id[0] != 0;
        for (int64_t v = i0 + tid; v < i1; v += THREADS) {
            float y = a * q_of(widen(s[v]));
            const int first = table[v - i0];
            if (first != NONE) {
                float e = 0.f;
                for (int64_t t = first; t < (again ? entries : first + 1); ++t)
                    if (c.teacher.ids[e0 + t] == v) e += expf((c.teacher.logit(e0 + t) - top) * c.inv_tau);
                y = fmaf(-e, f, y);
            }
            g[v] = narrow<T>(y);
        }
        __syncthreads();
    }
}

template <typename T, bool FORWARD, bool GRAD>
spsyrk_status_t launch(const Call& c, const void* logits, void* grad, cudaStream_t st) {
    // as many CTAs per row as two CTAs per SM need, each with at least 8192 logits
    int cluster = 1;
    while (cluster < 8 && c.rows.m * cluster < 2 * SMS && c.n / (2 * cluster) >= 8192) cluster *= 2;
    if (c.rows.m * cluster >= (int64_t(1) << 31)) return SPSYRK_ERR_OVERFLOW;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)(c.rows.m * cluster));
    cfg.blockDim = dim3(THREADS);
    cfg.stream = st;
    cudaLaunchAttribute attr{};
    attr.id = cudaLaunchAttributeClusterDimension;
    attr.val.clusterDim.x = (unsigned)cluster;
    attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    SPSYRK_CUDA_TRY(launch_kernel(cfg, distill_kernel<T, FORWARD, GRAD>, Call(c), static_cast<const T*>(logits), static_cast<T*>(grad)));
    return SPSYRK_OK;
}

bool is_logit(spsyrk_dtype_t t) { return t == SPSYRK_F32 || t == SPSYRK_BF16 || t == SPSYRK_F16; }

spsyrk_status_t distill(int64_t m, int64_t n, int64_t nnz, spsyrk_dtype_t dtype, spsyrk_dtype_t teacher_dtype, const int64_t* d_rowptr,
                        const int32_t* d_ids, const void* d_teacher, const float* d_teacher_lse, const float* d_row_weights, double temperature,
                        double scale, const void* d_logits, int64_t ldl, float* d_loss, float* d_lse, const float* d_kept, bool backward, void* d_grad,
                        int64_t ldg, cudaStream_t st) {
    if (m < 0 || n < 0 || nnz < 0 || !is_logit(dtype) || !is_logit(teacher_dtype)) return SPSYRK_ERR_INVALID_ARG;
    if (!(temperature >= 1e-6 && temperature <= 1e6)) return SPSYRK_ERR_INVALID_ARG;
    constexpr int64_t most = (int64_t(1) << 31) - 1;
    if (m >= most || n >= most || nnz >= most) return SPSYRK_ERR_OVERFLOW;
    if ((nnz > 0 && (!d_ids || !d_teacher)) || (!d_rowptr && (m == 0 ? nnz != 0 : nnz % m != 0))) return SPSYRK_ERR_INVALID_ARG;
    if (ldl < n || (d_grad && ldg < n) || (d_grad && d_grad == d_logits && ldg != ldl)) return SPSYRK_ERR_INVALID_ARG;
    if (m == 0) return SPSYRK_OK;
    if ((n > 0 && (!d_logits || (backward && !d_grad))) || (backward && !d_kept)) return SPSYRK_ERR_INVALID_ARG;
    if (backward && n == 0) return SPSYRK_OK;
    Call c;
    c.rows = Rows{d_rowptr, m, nnz, nnz / m};
    c.n = n;
    c.teacher = Teacher{d_ids, d_teacher, teacher_dtype, d_teacher_lse};
    c.row_weights = d_row_weights;
    c.k = (float)(LOG2E / temperature);
    c.inv_tau = (float)(1.0 / temperature);
    c.inv_tau_d = 1.0 / temperature;
    c.scale = scale;
    c.ldl = ldl;
    c.ldg = ldg;
    c.loss = d_loss;
    c.lse = d_lse;
    c.kept = d_kept;
#define LAUNCH(T) (backward ? launch<T, false, true>(c, d_logits, d_grad, st) \
                   : d_grad ? launch<T, true, true>(c, d_logits, d_grad, st) : launch<T, true, false>(c, d_logits, nullptr, st))
    switch (dtype) {
        case SPSYRK_F32: return LAUNCH(float);
        case SPSYRK_BF16: return LAUNCH(__nv_bfloat16);
        default: return LAUNCH(__half);
    }
#undef LAUNCH
}

}  // namespace

extern "C" spsyrk_status_t spsyrk_distill(int64_t m, int64_t n, int64_t nnz, spsyrk_dtype_t dtype, spsyrk_dtype_t teacher_dtype, const int64_t* d_rowptr,
                                          const int32_t* d_ids, const void* d_teacher, const float* d_teacher_lse, const float* d_row_weights,
                                          double temperature, double scale, const void* d_logits, int64_t ldl, float* d_loss, float* d_lse,
                                          void* d_grad, int64_t ldg, void* cuda_stream) {
    return distill(m, n, nnz, dtype, teacher_dtype, d_rowptr, d_ids, d_teacher, d_teacher_lse, d_row_weights, temperature, scale, d_logits, ldl, d_loss, d_lse,
                   nullptr, false, d_grad, ldg, static_cast<cudaStream_t>(cuda_stream));
}

extern "C" spsyrk_status_t spsyrk_distill_grad(int64_t m, int64_t n, int64_t nnz, spsyrk_dtype_t dtype, spsyrk_dtype_t teacher_dtype,
                                               const int64_t* d_rowptr, const int32_t* d_ids, const void* d_teacher, const float* d_teacher_lse,
                                               const float* d_row_weights, double temperature, double scale, const void* d_logits, int64_t ldl,
                                               const float* d_lse, void* d_grad, int64_t ldg, void* cuda_stream) {
    return distill(m, n, nnz, dtype, teacher_dtype, d_rowptr, d_ids, d_teacher, d_teacher_lse, d_row_weights, temperature, scale, d_logits, ldl, nullptr,
                   nullptr, d_lse, true, d_grad, ldg, static_cast<cudaStream_t>(cuda_stream));
}
