// Distillation from a teacher's top logits: rows of ids and teacher's logits z (CSR) meet dense rows of a student's logits s.
// With x = s / tau, lse = log sum_v exp(x_v), q_v = exp(x_v - lse), p_t = exp(z_t / tau - L):
//     loss = scale r sum_t p_t (log p_t - log q_{id_t}),      G_v = scale r / tau (P q_v - sum of the p_t with id v).
//
// Bound by memory: the logits are read once and the gradient is written once.  A cluster of 1 to 8 CTAs takes a row, each a contiguous
// share of it: a running maximum and sum per thread, joined over the CTA and the cluster, then the gradient, for which the share is read
// again.  It is then still in L2 as long as the shares under way are a fraction of it (888 of 64 KB, 57 MB; with rows of 256 KB a CTA, 76 MB and as
// much of gradients, many went to memory again).  A CTA lives some 13 us, most of them latencies, so what counts is how many bytes are under
// way: six CTAs per SM, and one instruction that asks for the whole share to be brought to L2 before the teacher's entries are looked at
// (422 us without it, 389 with it for 4096 rows of 131072 bfloat16 logits, 2.1 GB; now 373, 88 % of the copy rate).  Kept in shared memory instead
// of L2 only three shares fit an SM (513 us; with CTAs that stay and copy the next row meanwhile 660, whose rows wait for one another).
// exp(x) is computed as 2^(s * log2(e) / tau - ...): a multiply-add and an exponential per logit.  (Instructions for two floats at a time, f32x2,
// are no faster here, and with their operands in register pairs the half-precision gradient that goes by the shift came out with infinities, now and then, in
// warps whose lanes did not all take as many turns of the loop.)
// The gradient is first written for all ids as if they were not the teacher's, then the few of the teacher's are overwritten, from
// logits that were fetched beforehand (so the gradient may overwrite the logits).  An id that occurs more than once is written for one
// of its entries, with the sum of all in their order: they are found with a hash table in shared memory.  Rows of more than
// 1024 entries (ragged rows: of four times the mean) go through the ids in windows instead.
#include <algorithm>
#include <math_constants.h>

#include "element.cuh"

using namespace spsyrk;

namespace {

constexpr int WARPS_PER_SM = 48;
constexpr int TWICE_SHARE = 65536, ONCE_SHARE = 131072;  // bytes of a row that a CTA takes at most, where it reads them twice and once
constexpr int SMALL_SHARE = 49152;                       // up to which CTAs have 128 threads instead of 256
constexpr int ASK_ONCE = 32768;                          // bytes of a share that are asked for at once where it is read once (all but in the widest rows where twice)
constexpr int MOST_TOP = 1024;    // teacher's entries of a row that are kept in shared memory, at most
constexpr int LEAST_TOP = 32;
constexpr int WINDOW = 2048;      // ids of a window in rows of more entries
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
// none) and `at` what the exponents are taken relative to.  As long as most * k is below NEAR in size, `at` is that product, rounded: a term is
// one multiply-add, and rounding `at` moves nothing, since the terms, the changes of `most` and the logarithm at the end all use the
// same number.  Half a step of a larger product would become an exponent of its own (2^7 at 1e9, infinity or 0 from 1.5e9 on): beyond NEAR
// `at` is most * k itself and terms go by (s - most) * k.  slip() is what rounding has moved `at` by.
struct Running {
    float most, sum;
};
constexpr float NEAR = 4096.f;
// A log sum of this size or more is too coarse as a float (half a step 2^-14): what is made from it is made from the logits again.
constexpr float COARSE = 1024.f;
__device__ __forceinline__ float base_of(float most) { return most == -CUDART_INF_F ? 0.f : most; }  // nothing but -infinity: terms of 0, or NaN
__device__ __forceinline__ bool is_near(float most, float k) { return fabsf(__fmul_rn(most, k)) < NEAR; }
__device__ __forceinline__ float slip(float most, float k) {
    const float at = __fmul_rn(most, k);
    return fabsf(at) < NEAR ? -fmaf(most, k, -at) : 0.f;
}
// (ALWAYS: a sum of few terms, the teacher's, whose exponents go by the difference whatever their size.)
template <bool ALWAYS = false>
__device__ __forceinline__ float step_down(float from, float to, float k) {  // the factor when `most` goes from one to the other
    if (ALWAYS) return power_of_two((from - to) * k);
    const float a = __fmul_rn(from, k), b = __fmul_rn(to, k);
    if (fabsf(a) < NEAR && fabsf(b) < NEAR) return power_of_two(a - b);
    return power_of_two((from - to) * k + (slip(from, k) - slip(to, k)));
}
template <bool ALWAYS = false>
__device__ __forceinline__ float term(float s, float base, float k) {
    if (ALWAYS) return power_of_two((s - base) * k);
    const float at = __fmul_rn(base, k);
    return power_of_two(fabsf(at) < NEAR ? fmaf(s, k, -at) : (s - base) * k);
}
template <int N, bool ALWAYS = false>
__device__ __forceinline__ void take(Running& r, const float (&s)[N], float k) {
    float top = s[0];
#pragma unroll
    for (int i = 1; i < N; ++i) top = fmaxf(top, s[i]);
    if (top > r.most) {
        r.sum *= step_down<ALWAYS>(r.most, top, k);  // most = -infinity: times 0
        r.most = top;
    }
    const float b = base_of(r.most);
#pragma unroll
    for (int i = 0; i < N; ++i) r.sum += term<ALWAYS>(s[i], b, k);
}
// Running sums of N lanes (a power of two, the same ones in all groups of N) joined; all lanes get the same bits.
template <int N, bool ALWAYS = false>
__device__ __forceinline__ Running join(Running r, float k) {
    float top;
    asm("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(top) : "f"(r.most));
    r.sum *= step_down<ALWAYS>(r.most, base_of(top), k);  // (0 times 0 for a lane that has nothing; NaN stays NaN)
#pragma unroll
    for (int o = N / 2; o > 0; o >>= 1) r.sum += __shfl_xor_sync(FULL_MASK, r.sum, o);
    return Running{top, r.sum};
}

// 16 bytes of logits as pairs, their largest value, and back
template <typename T> struct Unit;
template <> struct Unit<float> {
    static constexpr int PAIRS = 2;
    static constexpr uint32_t NOTHING = 0xff800000u;  // -infinity
    __device__ static __forceinline__ float2 get(const uint4& u, int i) {
        return i == 0 ? float2{__uint_as_float(u.x), __uint_as_float(u.y)} : float2{__uint_as_float(u.z), __uint_as_float(u.w)};
    }
    template <int U>
    __device__ static __forceinline__ float largest(const uint4 (&u)[U]) {
        float m = __uint_as_float(u[0].x);
#pragma unroll
        for (int i = 0; i < U; ++i) {
            m = fmaxf(fmaxf(m, __uint_as_float(u[i].x)), __uint_as_float(u[i].y));
            m = fmaxf(fmaxf(m, __uint_as_float(u[i].z)), __uint_as_float(u[i].w));
        }
        return m;
    }
    __device__ static __forceinline__ uint4 put(const float2 (&y)[2]) {
        return uint4{__float_as_uint(y[0].x), __float_as_uint(y[0].y), __float_as_uint(y[1].x), __float_as_uint(y[1].y)};
    }
};
__device__ __forceinline__ uint32_t word(const uint4& u, int i) { return i == 0 ? u.x : i == 1 ? u.y : i == 2 ? u.z : u.w; }
template <> struct Unit<__nv_bfloat16> {
    static constexpr int PAIRS = 4;
    static constexpr uint32_t NOTHING = 0xff80ff80u;
    __device__ static __forceinline__ float2 get(const uint4& u, int i) {
        return float2{__uint_as_float(word(u, i) << 16), __uint_as_float(word(u, i) & 0xffff0000u)};
    }
    template <int U>
    __device__ static __forceinline__ float largest(const uint4 (&u)[U]) {
        __nv_bfloat162 m = reinterpret_cast<const __nv_bfloat162&>(u[0].x);
#pragma unroll
        for (int i = 0; i < 4 * U; ++i) {
            const uint32_t w = word(u[i / 4], i % 4);
            m = __hmax2(m, reinterpret_cast<const __nv_bfloat162&>(w));
        }
        return fmaxf(__low2float(m), __high2float(m));
    }
    __device__ static __forceinline__ uint4 put(const float2 (&y)[4]) {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const __nv_bfloat162 b = __float22bfloat162_rn(y[i]);
            w[i] = reinterpret_cast<const uint32_t&>(b);
        }
        return uint4{w[0], w[1], w[2], w[3]};
    }
};
template <> struct Unit<__half> {
    static constexpr int PAIRS = 4;
    static constexpr uint32_t NOTHING = 0xfc00fc00u;
    __device__ static __forceinline__ float2 get(const uint4& u, int i) {
        const uint32_t w = word(u, i);
        return __half22float2(reinterpret_cast<const __half2&>(w));
    }
    template <int U>
    __device__ static __forceinline__ float largest(const uint4 (&u)[U]) {
        __half2 m = reinterpret_cast<const __half2&>(u[0].x);
#pragma unroll
        for (int i = 0; i < 4 * U; ++i) {
            const uint32_t w = word(u[i / 4], i % 4);
            m = __hmax2(m, reinterpret_cast<const __half2&>(w));
        }
        return fmaxf(__low2float(m), __high2float(m));
    }
    __device__ static __forceinline__ uint4 put(const float2 (&y)[4]) {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const __half2 b = __float22half2_rn(y[i]);
            w[i] = reinterpret_cast<const uint32_t&>(b);
        }
        return uint4{w[0], w[1], w[2], w[3]};
    }
};

// U units at a time into a running sum
template <typename T, int U>
__device__ __forceinline__ void take_units(Running& r, const uint4 (&u)[U], float k) {
    constexpr int PAIRS = Unit<T>::PAIRS;
    const float top = Unit<T>::template largest<U>(u);
    if (top > r.most) {
        r.sum *= step_down(r.most, top, k);
        r.most = top;
    }
    const float b = base_of(r.most), at = __fmul_rn(b, k);
    if (fabsf(at) < NEAR) {
        float2 sum[2] = {{r.sum, 0.f}, {0.f, 0.f}};
#pragma unroll
        for (int i = 0; i < U * PAIRS; ++i) {
            const float2 x = Unit<T>::get(u[i / PAIRS], i % PAIRS);
            sum[i & 1].x += power_of_two(fmaf(x.x, k, -at));
            sum[i & 1].y += power_of_two(fmaf(x.y, k, -at));
        }
        r.sum = (sum[0].x + sum[1].x) + (sum[0].y + sum[1].y);
    } else {
#pragma unroll
        for (int i = 0; i < U * PAIRS; ++i) {
            const float2 x = Unit<T>::get(u[i / PAIRS], i % PAIRS);
            r.sum += power_of_two((x.x - b) * k) + power_of_two((x.y - b) * k);
        }
    }
}

// Asks for bytes that will be read soon to be brought to L2; address and number of bytes are multiples of 16.
__device__ __forceinline__ void prefetch(const void* from, int bytes) {
    asm volatile("cp.async.bulk.prefetch.L2.global [%0], %1;" ::"l"(from), "r"(bytes) : "memory");
}

// A row's columns in 16-byte units from its first 16-byte boundary: this CTA has `units` of them from column `first` on, and the
// first CTA also the `head` columns before the boundary and those from `tail` on, behind the last unit.
struct Share {
    int head, units, first, tail;
};
template <typename T>
__device__ __forceinline__ Share share_of(const T* row, int64_t n, uint32_t rank, int log_size) {
    constexpr int W = 16 / (int)sizeof(T);
    Share s;
    s.head = (int)min(n, (int64_t)((0 - reinterpret_cast<uintptr_t>(row)) % 16 / sizeof(T)));
    const int units = (int)((uint32_t)(n - s.head) / W), each = (units + (1 << log_size) - 1) >> log_size, v0 = min(units, (int)rank * each);
    s.units = min(units - v0, each);
    s.first = s.head + v0 * W;
    s.tail = s.head + units * W;
    return s;
}

struct Call {
    Rows rows;
    int64_t n;
    Teacher teacher;
    const float* row_weights;
    float k;                  // log2(e) / tau
    double scale, inv_tau_d;  // 1 / tau
    int64_t ldl, ldg;
    float *loss, *lse;
    const float* kept;  // the rows' lse of an earlier call (gradient only)
    float factor;       // scale / tau
    int log_cluster;    // CTAs of a row
    int top, log_slots; // entries that are kept in shared memory; slots of the hash table, at least twice as many
};

// The gradient of `left` units from `at` on (this thread's: every THREADS-th), but for the teacher's ids: a 2^(s k - shift).  FOLDED: the factor
// is in the shift already (16-bit results whose shift and factor's logarithm are below 400 and 100 in size: half a step of their sum
// is 2^-16 then, the approximate logarithm is off by 2^-22, and half a step of the result is 2^-12 of it or more).
// BY_BASE: a 2^((s - shift) k).
enum Form { FOLDED, BY_SHIFT, BY_BASE };
template <typename T, int THREADS, Form FORM>
__device__ __forceinline__ void write_units(const uint4* at, uint4* to, int left, float k, float shift, float a) {
    constexpr int U = 4, PAIRS = Unit<T>::PAIRS;
    auto of = [&](const uint4& x) {
        float2 y[PAIRS];
#pragma unroll
        for (int q = 0; q < PAIRS; ++q) {
            const float2 s = Unit<T>::get(x, q);
            y[q] = FORM == BY_BASE ? float2{power_of_two((s.x - shift) * k), power_of_two((s.y - shift) * k)}
                                   : float2{power_of_two(fmaf(s.x, k, -shift)), power_of_two(fmaf(s.y, k, -shift))};
            if (FORM != FOLDED) y[q] = float2{a * y[q].x, a * y[q].y};
        }
        return Unit<T>::put(y);
    };
    for (; left >= U * THREADS; left -= U * THREADS, at += U * THREADS, to += U * THREADS) {
        uint4 x[U];
#pragma unroll
        for (int i = 0; i < U; ++i) x[i] = __ldcg(at + i * THREADS);
#pragma unroll
        for (int i = 0; i < U; ++i) __stcs(to + i * THREADS, of(x[i]));
    }
    for (int u = threadIdx.x; u < left; u += THREADS, at += THREADS, to += THREADS) __stcs(to, of(__ldcg(at)));
}

// Loss and lse of a row, by a whole CTA; the teacher's entries are in shared memory (`few`) or are read again.
template <typename T, int THREADS>
__device__ __forceinline__ void write_loss(const Call& c, int64_t row, float weight, int64_t e0, int64_t entries, bool few, const int32_t* s_id,
                                           const float* s_z, const float* s_at, const T* s, Running r, float top, Running teacher) {
    constexpr int WARPS = THREADS / 32;
    __shared__ double s_sum[WARPS][2];
    const float b = base_of(r.most);
    double mass = 0, cross = 0;  // sum of e_t; of e_t tau (log p_t - log q_t), but for the logarithms that all share
    for (int64_t t = threadIdx.x; t < entries; t += THREADS) {
        const int32_t id = few ? s_id[t] : c.teacher.ids[e0 + t];
        if (id < 0 || id >= c.n) continue;
        const float z = few ? s_z[t] : c.teacher.logit(e0 + t), at = few ? s_at[t] : widen(s[id]);
        const float e = term<true>(z, top, c.k);
        if (e == 0.f) continue;
        mass += (double)e;
        cross += (double)e * (((double)z - (double)top) - ((double)at - (double)b));
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        mass += __shfl_xor_sync(FULL_MASK, mass, o);
        cross += __shfl_xor_sync(FULL_MASK, cross, o);
    }
    if (lane_id() == 0) {
        s_sum[threadIdx.x >> 5][0] = mass;
        s_sum[threadIdx.x >> 5][1] = cross;
    }
    __syncthreads();
    if (threadIdx.x != 0) return;
    for (int w = 1; w < WARPS; ++w) {
        mass += s_sum[w][0];
        cross += s_sum[w][1];
    }
    // log p = (z - top) / tau + log_unit, log q = (s - b) / tau - rest; p = e * unit.  (k is rounded, 1 / tau is not: it stands for differences only.)
    const double rest = (double)slip(b, c.k) * LN2 + log((double)r.sum);
    const double log_unit = c.teacher.lse ? (double)top * c.inv_tau_d - (double)c.teacher.lse[row] : -log(mass);
    const double unit = c.teacher.lse ? exp(log_unit) : 1.0 / mass;
    const bool left_out = teacher.sum == 0.f;
    // (p = 0 throughout, under a given norm far above, adds nothing, whatever q is)
    const bool nothing = left_out || (unit == 0.0 && mass < CUDART_INF && r.sum > 0.f && r.sum < CUDART_INF_F);
    if (c.loss) c.loss[row] = nothing ? 0.f : (float)(c.scale * (double)weight * unit * (cross * c.inv_tau_d + mass * (log_unit + rest)));
    if (c.lse) c.lse[row] = left_out ? 0.f : (float)((double)b * c.inv_tau_d + rest);
}

// What the warps of a CTA tell one another: running sums of the student's and of the teacher's row.
struct Joint {
    Running student, teacher;
};

// FORWARD: the sum over the row is computed (else it is `kept`, unless that is too coarse); GRAD: the gradient is written.
template <typename T, int THREADS, bool FORWARD, bool GRAD>
__global__ void __launch_bounds__(THREADS, WARPS_PER_SM * 32 / THREADS) distill_kernel(const Call c, const T* logits, T* grad) {
    constexpr int W = 16 / (int)sizeof(T), U = 4, WARPS = THREADS / 32;
    extern __shared__ int32_t windows[];  // rows of many entries: [WINDOW]; else the teacher's entries
    int32_t* const s_id = windows;  // [top]
    float *const s_z = reinterpret_cast<float*>(s_id + c.top), *const s_at = s_z + c.top;  // [top] the teacher's logit, the student's
    uint16_t* const table = reinterpret_cast<uint16_t*>(s_at + c.top);  // [1 << log_slots]
    __shared__ Joint s_warp[WARPS];
    __shared__ float2 s_cta[8];
    __shared__ int s_again;
    __shared__ uint32_t s_more[MOST_TOP / 32];  // a bit per entry: others have its id too
    __shared__ uint64_t s_arrived;
    const uint32_t rank = cluster_rank(), size = 1u << c.log_cluster;
    const int64_t row = blockIdx.x >> c.log_cluster;
    const int tid = threadIdx.x;
    const T* const s = logits + row * c.ldl;
    T* const g = GRAD ? grad + row * c.ldg : nullptr;
    const float weight = c.row_weights ? c.row_weights[row] : 1.f;
    const int64_t e0 = c.rows.begin(row), entries = max((int64_t)0, c.rows.end(row) - e0);
    const bool few = entries <= c.top;
    const Share mine = share_of(s, c.n, rank, c.log_cluster);
    const bool aligned = !GRAD || reinterpret_cast<uintptr_t>(g + mine.head) % 16 == 0;
    const int last = mine.first + mine.units * W, behind = (int)c.n - mine.tail;  // (columns behind the last unit)
    auto is_mine = [&](int id) { return (id >= mine.first && id < last) || (rank == 0 && (id < mine.head || id >= mine.tail)); };

    auto leave_out = [&] {  // (the same for the whole cluster)
        if (FORWARD && tid == 0 && rank == 0) {
            if (c.loss) c.loss[row] = 0.f;
            if (c.lse) c.lse[row] = 0.f;
        }
        if (GRAD) {
            if (aligned) {
                for (int u = tid; u < mine.units; u += THREADS) *reinterpret_cast<uint4*>(g + mine.first + (int64_t)u * W) = uint4{0, 0, 0, 0};
            } else {
                for (int v = tid; v < last - mine.first; v += THREADS) g[mine.first + v] = narrow<T>(0.f);
            }
            if (rank == 0) {
                if (tid < mine.head) g[tid] = narrow<T>(0.f);
                if (tid < behind) g[mine.tail + tid] = narrow<T>(0.f);
            }
        }
    };
    if (weight == 0.f || entries == 0) {
        leave_out();
        return;
    }

    if (size > 1) {  // (shared memory of a CTA that has not begun is nobody's to write to)
        if (tid == 0) {
            barrier_init(&s_arrived);
            barrier_init_visible();
        }
        cluster_arrive_relaxed();
    }

    if (tid == 0 && (FORWARD || few) && mine.units > 0) prefetch(s + mine.first, min(mine.units * 16, FORWARD && GRAD ? 2 * TWICE_SHARE : ASK_ONCE));

    // the teacher's row
    Running teacher{-CUDART_INF_F, 0.f};
    for (int64_t t = tid; t < entries; t += THREADS) {
        const int32_t id = c.teacher.ids[e0 + t];
        const bool held = id >= 0 && id < c.n;
        const float z[1] = {held ? c.teacher.logit(e0 + t) : -CUDART_INF_F};
        if (few) {
            s_id[t] = held ? id : -1;
            s_z[t] = z[0];
            s_at[t] = held && (rank == 0 || is_mine(id)) ? widen(s[id]) : 0.f;
        }
        take<1, true>(teacher, z, c.k);
    }
    const int slots = 1 << c.log_slots;
    constexpr uint16_t NO_ENTRY = 0xffff;
    if (GRAD && few) {
        for (int i = tid; i < slots; i += THREADS) table[i] = NO_ENTRY;
        if (tid < MOST_TOP / 32) s_more[tid] = 0;
    }

    Running r{-CUDART_INF_F, 0.f};
    const float kept = FORWARD ? 0.f : c.kept[row];
    const bool sums = FORWARD || fabsf(kept) >= COARSE;  // the row's sum is computed
    if (FORWARD) {
        const uint4* at = reinterpret_cast<const uint4*>(s + mine.first) + tid;
        int left = mine.units;
        for (; left >= U * THREADS; left -= U * THREADS, at += U * THREADS) {  // (nothing to look at: half of the instructions beside the arithmetic)
            uint4 x[U];
#pragma unroll
            for (int i = 0; i < U; ++i) x[i] = __ldcg(at + i * THREADS);
            take_units<T, U>(r, x, c.k);
        }
        if (tid < left) {
            uint4 x[U];
#pragma unroll
            for (int i = 0; i < U; ++i) {
                constexpr uint32_t none = Unit<T>::NOTHING;
                x[i] = uint4{none, none, none, none};
                if (tid + i * THREADS < left) x[i] = __ldcg(at + i * THREADS);
            }
            take_units<T, U>(r, x, c.k);
        }
    } else if (sums) {
        for (int u = tid; u < mine.units; u += THREADS) {
            const uint4 x[1] = {__ldcg(reinterpret_cast<const uint4*>(s + mine.first) + u)};
            take_units<T, 1>(r, x, c.k);
        }
    }
    if (sums) {
        if (rank == 0) {
            float f[1];
            if (tid < mine.head) {
                f[0] = widen(s[tid]);
                take<1>(r, f, c.k);
            }
            if (tid < behind) {
                f[0] = widen(s[mine.tail + tid]);
                take<1>(r, f, c.k);
            }
        }
    }
    // joined over the warp, the CTA, the cluster
    if (sums) r = join<32>(r, c.k);
    if ((tid & ~31) < entries) teacher = join<32, true>(teacher, c.k);
    if (lane_id() == 0) s_warp[tid >> 5] = Joint{r, teacher};
    __syncthreads();
    const Joint joint = s_warp[lane_id() & (WARPS - 1)];
    if (sums) r = join<WARPS>(joint.student, c.k);
    teacher = join<WARPS, true>(joint.teacher, c.k);
    if (size > 1) {
        cluster_wait();
        if (tid == 0) barrier_expect(&s_arrived, size * 8);
        if (tid < size) store_to_rank(s_cta + rank, float2{r.most, r.sum}, &s_arrived, tid);
    }

    // meanwhile: an entry for every id of the share; slots of the table hold entries, one of an id's
    const int count = (int)min(entries, (int64_t)c.top);
    uint32_t chosen = 0;  // a bit for each of this thread's entries
    static_assert(MOST_TOP / THREADS <= 32, "bits");
    if (GRAD && few) {
        for (int t = tid, bit = 0; t < count; t += THREADS, ++bit) {
            const int32_t id = s_id[t];
            if (id < 0 || !is_mine(id)) continue;
            for (int q = (int)(((uint32_t)id * 2654435761u) >> (32 - c.log_slots));; q = (q + 1) & (slots - 1)) {  // (multiplicative hashing; at most half full)
                const uint16_t was = atomicCAS(&table[q], NO_ENTRY, (uint16_t)t);
                if (was == NO_ENTRY) {
                    chosen |= 1u << bit;
                    break;
                }
                if (s_id[was] == id) {
                    atomicOr(&s_more[was >> 5], 1u << (was & 31));
                    break;
                }
            }
        }
    }
    // p_t = e_t * unit with e_t as in teacher.sum, mass P
    const float top = base_of(teacher.most);
    float unit = 1.f / teacher.sum;
    if (c.teacher.lse) {  // (the exponent in two parts: rounded as a whole, one of 40 is off by 2e-6)
        const double x = (double)top * c.inv_tau_d - (double)c.teacher.lse[row];
        const float whole = (float)x, rest = isfinite(whole) ? (float)(x - (double)whole) : 0.f;
        unit = expf(whole) * (1.f + rest);
    }
    const float mass = c.teacher.lse ? teacher.sum * unit : 1.f + 0.f * teacher.sum;  // (1, or NaN)
    auto e_of = [&](float z) { return term<true>(z, top, c.k); };

    bool all = true;  // a wait that runs out, which should not happen, is seen in the results: NaN
    if (size > 1) {
        all = barrier_wait(&s_arrived, 0);  // from here on logits may be overwritten: all have fetched the teacher's
            if (sums) {
            const float2 part = s_cta[lane_id() & (size - 1)];
            r = Running{part.x, all ? part.y : CUDART_NAN_F};
            r = size == 2 ? join<2>(r, c.k) : size == 4 ? join<4>(r, c.k) : join<8>(r, c.k);
        }
    }
    if (!few && FORWARD) {  // the loss needs logits that the gradient may overwrite
        if (rank == 0) write_loss<T, THREADS>(c, row, weight, e0, entries, false, s_id, s_z, s_at, s, r, top, teacher);
        if (size > 1) cluster_sync();
    }
    if (teacher.sum == 0.f) {  // no entry with a logit other than -infinity
        leave_out();
        return;
    }
    if (GRAD) {
        // G_v = a 2^(s k - shift) - (at the teacher's ids) f e; a row that was NaN or -infinity throughout is NaN in all places.  The shift that
        // belongs to a kept lse is that of a logit with q = 1, so that the rounding of k matters to small q only; what
        // rounding the shift takes away goes into a (its logarithm is below 2^-14: two terms of the exponential's series are exact to 2^-44).
        const float factor = c.factor * weight, f = factor * unit;
        float a, shift, b = 0.f;
        if (sums) {
            b = base_of(r.most);
            shift = is_near(b, c.k) ? __fmul_rn(b, c.k) : 0.f;
            a = r.sum > 0.f && r.sum < CUDART_INF_F ? factor * mass / r.sum : CUDART_NAN_F;
        } else {
            const double exact = (double)kept / c.inv_tau_d * (double)c.k;
            shift = (float)exact;
            const double slip = ((double)shift - exact) * LN2;
            a = (float)((double)(factor * mass) * (1.0 + slip + 0.5 * slip * slip));
        }
        if (!FORWARD && !all) a = CUDART_NAN_F;
        const bool plain = !sums || is_near(b, c.k);
        auto q_of = [&](float x) { return power_of_two(plain ? fmaf(x, c.k, -shift) : (x - b) * c.k); };
        if (few) {
            const uint4* at = reinterpret_cast<const uint4*>(s + mine.first) + tid;
            int left = mine.units;
            const bool folded = sizeof(T) == 2 && plain && fabsf(shift) < 400.f && a > 0x1p-100f && a < 0x1p100f;
            const float deep = folded ? shift - __log2f(a) : shift;
            auto g_of = [&](float x) { return folded ? power_of_two(fmaf(x, c.k, -deep)) : a * q_of(x); };  // the same wherever the rows lie
            auto write_ends = [&] {
                if (rank != 0) return;
                if (tid < mine.head) g[tid] = narrow<T>(g_of(widen(s[tid])));
                if (tid < behind) g[mine.tail + tid] = narrow<T>(g_of(widen(s[mine.tail + tid])));
            };
            if (!FORWARD) write_ends();  // (before or after: what keeps registers from being spilled in the loops; 1999 rows of 50021 59 us against 65)
            if (aligned) {
                uint4* to = reinterpret_cast<uint4*>(g + mine.first) + tid;
                if (folded) write_units<T, THREADS, FOLDED>(at, to, left, c.k, deep, a);
                else if (plain) write_units<T, THREADS, BY_SHIFT>(at, to, left, c.k, shift, a);
                else write_units<T, THREADS, BY_BASE>(at, to, left, c.k, b, a);
            } else {
                T* const to = g + mine.first;
                for (int u = tid; u < left; u += THREADS, at += THREADS) {
                    const uint4 v = __ldcg(at);
                    const Vec<T, W> x = reinterpret_cast<const Vec<T, W>&>(v);
#pragma unroll
                    for (int q = 0; q < W; ++q) to[(int64_t)u * W + q] = narrow<T>(g_of(widen(x.x[q])));
                }
            }
            if (FORWARD) write_ends();
            __syncthreads();
            for (int t = tid, bit = 0; t < count; t += THREADS, ++bit) {
                if (!(chosen >> bit & 1u)) continue;
                const int32_t id = s_id[t];
                float e = e_of(s_z[t]);
                if (s_more[t >> 5] >> (t & 31) & 1u) {
                    e = 0.f;
                    for (int o = 0; o < count; ++o)
                        if (s_id[o] == id) e += e_of(s_z[o]);
                }
                g[id] = narrow<T>(fmaf(-e, f, a * q_of(s_at[t])));
            }
        } else {
            // Rows of many entries: windows of ids, in every window the first entry of each id by its place.
            int32_t* const firsts = windows;
            for (int64_t i0 = (int64_t)rank * WINDOW; i0 < c.n; i0 += (int64_t)size * WINDOW) {
                const int64_t i1 = min(i0 + WINDOW, c.n);
                __syncthreads();
                for (int i = tid; i < WINDOW; i += THREADS) firsts[i] = NONE;
                if (tid == 0) s_again = 0;
                __syncthreads();
                for (int64_t t = tid; t < entries; t += THREADS) {
                    const int32_t id = c.teacher.ids[e0 + t];
                    if (id < i0 || id >= i1) continue;
                    if (atomicMin(&firsts[id - i0], (int)t) != NONE) s_again = 1;
                }
                __syncthreads();
                const bool again = s_again != 0;
                for (int64_t v = i0 + tid; v < i1; v += THREADS) {
                    float y = a * q_of(widen(s[v]));
                    const int first = firsts[v - i0];
                    if (first != NONE) {
                        float e = 0.f;
                        for (int64_t t = first; t < (again ? entries : first + 1); ++t)
                            if (c.teacher.ids[e0 + t] == v) e += e_of(c.teacher.logit(e0 + t));
                        y = fmaf(-e, f, y);
                    }
                    g[v] = narrow<T>(y);
                }
            }
        }
    }
    if (FORWARD && few && rank == 0) write_loss<T, THREADS>(c, row, weight, e0, entries, true, s_id, s_z, s_at, s, r, top, teacher);
}

template <typename T, int THREADS, bool FORWARD, bool GRAD>
spsyrk_status_t launch_by(Call c, const void* logits, void* grad, cudaStream_t st) {
    constexpr auto kernel = distill_kernel<T, THREADS, FORWARD, GRAD>;
    const int cluster = 1 << c.log_cluster;
    // entries in shared memory: all if every row has as many, else room for four times the mean
    const int64_t entries = c.rows.rowptr ? std::max<int64_t>(128, 4 * (c.rows.nnz / c.rows.m)) : c.rows.k;
    c.top = LEAST_TOP;
    c.log_slots = 6;
    while (c.top < entries && c.top < MOST_TOP) c.top *= 2, ++c.log_slots;
    static_assert(LEAST_TOP == 32, "log_slots");
    const size_t kept = (size_t)c.top * 12 + (GRAD ? (size_t)2 << c.log_slots : 0);
    SPSYRK_CUDA_TRY(allow_shared_memory<kernel>());
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)(c.rows.m * cluster));
    cfg.blockDim = dim3(THREADS);
    cfg.dynamicSmemBytes = std::max<size_t>(kept, GRAD ? WINDOW * 4 : 0);
    cfg.stream = st;
    cudaLaunchAttribute attr{};
    attr.id = cudaLaunchAttributeClusterDimension;
    attr.val.clusterDim.x = (unsigned)cluster;
    attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    SPSYRK_CUDA_TRY(launch_kernel(cfg, kernel, Call(c), static_cast<const T*>(logits), static_cast<T*>(grad)));
    return SPSYRK_OK;
}

template <typename T, bool FORWARD, bool GRAD>
spsyrk_status_t launch(Call c, const void* logits, void* grad, cudaStream_t st) {
    constexpr int W = 16 / (int)sizeof(T);
    const int64_t units = (c.n + W - 1) / W;
    // smaller shares, down to 16 KB, as long as the CTAs do not fill the GPU
    constexpr int64_t MOST = (FORWARD && GRAD ? TWICE_SHARE : ONCE_SHARE) / 16;
    while (c.log_cluster < 3 && (units > MOST << c.log_cluster || (c.rows.m << c.log_cluster < 3 * SMS && units >= int64_t(1024) << c.log_cluster))) ++c.log_cluster;
    if (c.rows.m << c.log_cluster >= int64_t(1) << 31) return SPSYRK_ERR_OVERFLOW;
    // Many short rows: the latencies of a row hide behind more rows, of fewer warps each (8000 rows of 8192 bfloat16 logits 76 us against 86, 4000 of
    // 3001 half-precision ones 37 against 47).
    return (units >> c.log_cluster) * 16 <= SMALL_SHARE && c.rows.m > 6 * SMS ? launch_by<T, 128, FORWARD, GRAD>(c, logits, grad, st) : launch_by<T, 256, FORWARD, GRAD>(c, logits, grad, st);
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
    c.inv_tau_d = 1.0 / temperature;
    c.scale = scale;
    c.factor = (float)(scale / temperature);
    c.log_cluster = 0;
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
