// What the products of CSR rows of ids with dense row-major matrices share: element types, vectors of elements, rows of entries.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "common.cuh"

namespace spsyrk {

// The type sums are held in: double for double, else single precision.
template <typename T> struct Wide { using type = float; };
template <> struct Wide<double> { using type = double; };

__device__ __forceinline__ float widen(float v) { return v; }
__device__ __forceinline__ double widen(double v) { return v; }
__device__ __forceinline__ float widen(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ float widen(__half v) { return __half2float(v); }

// One rounding, to nearest even.
template <typename T, typename A> __device__ __forceinline__ T narrow(A v);
template <> __device__ __forceinline__ float narrow<float, float>(float v) { return v; }
template <> __device__ __forceinline__ double narrow<double, double>(double v) { return v; }
template <> __device__ __forceinline__ __nv_bfloat16 narrow<__nv_bfloat16, float>(float v) { return __float2bfloat16_rn(v); }
template <> __device__ __forceinline__ __half narrow<__half, float>(float v) { return __float2half_rn(v); }

// W elements that are read and written together, 16 bytes at most; their address is a multiple of their size.
template <typename T, int W>
struct alignas(sizeof(T) * W) Vec {
    static_assert(sizeof(T) * W <= 16, "16 bytes");
    T x[W];
};
template <typename T, int V> constexpr int VEC_OF = V * (int)sizeof(T) > 16 ? 16 / (int)sizeof(T) : V;

// the first `left` elements at p as they are, zeros behind them
template <typename T, int V>
__device__ __forceinline__ Vec<T, V> load_raw(const T* __restrict__ p, int64_t left) {
    Vec<T, V> v;
    if (left >= V) {
        v = *reinterpret_cast<const Vec<T, V>*>(p);
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i) v.x[i] = i < left ? p[i] : T(0.f);
    }
    return v;
}
// the first `left` elements at p, widened, zeros behind them
template <typename T, int V>
__device__ __forceinline__ void load_wide(const T* __restrict__ p, int64_t left, typename Wide<T>::type (&x)[V]) {
    constexpr int W = VEC_OF<T, V>;
    if (left >= V) {
#pragma unroll
        for (int k = 0; k < V; k += W) {
            const Vec<T, W> v = *reinterpret_cast<const Vec<T, W>*>(p + k);
#pragma unroll
            for (int i = 0; i < W; ++i) x[k + i] = widen(v.x[i]);
        }
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i) x[i] = i < left ? widen(p[i]) : typename Wide<T>::type(0);
    }
}
template <typename T, int V>
__device__ __forceinline__ void store_narrow(T* __restrict__ p, int64_t left, const typename Wide<T>::type (&x)[V]) {
    constexpr int W = VEC_OF<T, V>;
    if (left >= V) {
#pragma unroll
        for (int k = 0; k < V; k += W) {
            Vec<T, W> v;
#pragma unroll
            for (int i = 0; i < W; ++i) v.x[i] = narrow<T>(x[k + i]);
            *reinterpret_cast<Vec<T, W>*>(p + k) = v;
        }
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i)
            if (i < left) p[i] = narrow<T>(x[i]);
    }
}

inline size_t element_size(spsyrk_dtype_t t) { return t == SPSYRK_F64 ? 8 : t == SPSYRK_BF16 || t == SPSYRK_F16 ? 2 : 4; }
inline bool is_real(spsyrk_dtype_t t) { return t == SPSYRK_F64 || t == SPSYRK_F32 || t == SPSYRK_BF16 || t == SPSYRK_F16; }
// Elements that can be read and written together in every row of a matrix: 16 bytes, or two elements, or one.
inline int together(const void* p, int64_t ld, size_t size) {
    const uint64_t bits = (uint64_t)reinterpret_cast<uintptr_t>(p) | (uint64_t)ld * size;
    return bits % 16 == 0 ? (int)(16 / size) : bits % (2 * size) == 0 ? 2 : 1;
}

// Rows of entries: row pointers, or the same number of entries k in every row.  Row pointers are cut to [0, nnz], so that no
// entry is looked for outside the arrays whatever they hold.
struct Rows {
    const int64_t* rowptr;
    int64_t m, nnz, k;
    __device__ __forceinline__ int64_t begin(int64_t i) const { return rowptr ? max((int64_t)0, min(rowptr[i], nnz)) : i * k; }
    __device__ __forceinline__ int64_t end(int64_t i) const { return rowptr ? max((int64_t)0, min(rowptr[i + 1], nnz)) : (i + 1) * k; }
    // entries before the first row and behind the last one belong to none
    __device__ __forceinline__ bool covered(int64_t e) const { return !rowptr || (e >= rowptr[0] && e < rowptr[m]); }
    // the last row in [lo, hi] that begins at entry e or before
    __device__ __forceinline__ int64_t row_of(int64_t e, int64_t lo, int64_t hi) const {
        if (!rowptr) return e / k;
        while (lo < hi) {
            const int64_t mid = (lo + hi + 1) >> 1;
            if (rowptr[mid] <= e) lo = mid; else hi = mid - 1;
        }
        return lo;
    }
    // the same by a whole warp, among all rows: 32 of them looked at per step
    __device__ __forceinline__ int64_t row_of_by_warp(int64_t e) const {
        int64_t lo = 0, hi = m - 1;
        while (lo < hi) {
            const int64_t step = (hi - lo + 31) / 32, at = lo + (lane_id() + 1) * step;
            const int before = __popc(__ballot_sync(FULL_MASK, at <= hi && rowptr[at] <= e));
            lo += before * step;
            hi = min(hi, lo + step - 1);
        }
        return lo;
    }
};

// Thread-block clusters: this CTA's number, a barrier, and values in another CTA's shared memory.
__device__ __forceinline__ uint32_t cluster_rank() {
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
// (relaxed: says only that this CTA has come so far, and that its barriers in shared memory, made visible, are there)
__device__ __forceinline__ void cluster_arrive_relaxed() { asm volatile("barrier.cluster.arrive.relaxed;" ::: "memory"); }
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait;" ::: "memory"); }
__device__ __forceinline__ void cluster_sync() {
    cluster_arrive();
    cluster_wait();
}
__device__ __forceinline__ uint32_t address_in(const void* mine, uint32_t rank) {
    uint32_t there;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(there) : "r"((uint32_t)__cvta_generic_to_shared(mine)), "r"(rank));
    return there;
}
__device__ __forceinline__ float load_of_rank(const float* mine, uint32_t rank) {
    float v;
    asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(address_in(mine, rank)) : "memory");
    return v;
}
__device__ __forceinline__ double load_of_rank(const double* mine, uint32_t rank) {
    double v;
    asm volatile("ld.shared::cluster.f64 %0, [%1];" : "=d"(v) : "r"(address_in(mine, rank)) : "memory");
    return v;
}

// A barrier in shared memory that counts bytes: every use of it (a phase) ends when `expect` has named the bytes and they have arrived.
__device__ __forceinline__ void barrier_init(uint64_t* bar) {
    asm volatile("mbarrier.init.shared.b64 [%0], 1;" ::"r"((uint32_t)__cvta_generic_to_shared(bar)) : "memory");
}
__device__ __forceinline__ void barrier_init_visible() { asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory"); }
__device__ __forceinline__ void barrier_expect(uint64_t* bar, uint32_t bytes) {
    asm volatile("mbarrier.arrive.expect_tx.shared.b64 _, [%0], %1;" ::"r"((uint32_t)__cvta_generic_to_shared(bar)), "r"(bytes) : "memory");
}
// Waits for the end of a phase; false if the wait ran out.
__device__ __forceinline__ bool barrier_wait(uint64_t* bar, uint32_t parity) {
    const uint32_t at = (uint32_t)__cvta_generic_to_shared(bar);
    for (int polls = 0; polls < (1 << 20); ++polls) {
        uint32_t done;
        asm volatile("{\n.reg .pred p;\nmbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\nselp.u32 %0, 1, 0, p;\n}" : "=r"(done) : "r"(at), "r"(parity) : "memory");
        if (done) return true;
    }
    return false;
}
// v into another CTA's shared memory, where 8 bytes more have then arrived.  Unlike a barrier of the cluster this does not wait for
// what has been stored to global memory before.
__device__ __forceinline__ void store_to_rank(const float2* mine, float2 v, uint64_t* bar, uint32_t rank) {
    asm volatile("st.async.weak.shared::cluster.mbarrier::complete_tx::bytes.v2.f32 [%0], {%1, %2}, [%3];" ::"r"(address_in(mine, rank)), "f"(v.x), "f"(v.y),
                 "r"(address_in(bar, rank))
                 : "memory");
}

}  // namespace spsyrk
