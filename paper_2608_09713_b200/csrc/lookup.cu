// Y = scale * A E for rows of ids A and a dense table E (an embedding lookup, or sums over bags of ids), and the gradient of the
// weights, dw_t = scale * <E[id_t], dY[row of t]>.
//
// Both move every row of E that they name and do two operations per element: bound by memory, or by latency for few rows.
// A group of 1 to 256 lanes holds a row of Y, 16 bytes a lane, and keeps its sum in registers.
#include <algorithm>

#include "element.cuh"

using namespace spsyrk;

namespace {

constexpr int THREADS = 256;
constexpr int SMS = 148;
constexpr int LONG_CLUSTER = 8;
constexpr int LONG_UNITS = 64;  // clusters that look for long rows

// lanes of a group: a power of two that covers the row's vectors, at most a CTA
int group_shift(int64_t vectors) {
    int s = 0;
    while ((int64_t(1) << s) < vectors && s < 8) ++s;
    return s;
}

// One id a row.  A group copies U rows, so that U loads of a lane are under way at a time.
template <typename T, int V, int U>
__global__ void __launch_bounds__(THREADS) lookup_one_kernel(int64_t m, int64_t n, int64_t p, const int32_t* __restrict__ ids,
                                                             const typename Wide<T>::type* __restrict__ weights, typename Wide<T>::type scale,
                                                             const T* __restrict__ e, int64_t lde, T* __restrict__ y, int64_t ldy, int shift) {
    using A = typename Wide<T>::type;
    const int64_t group = (int64_t)blockIdx.x * (THREADS >> shift) + (threadIdx.x >> shift);
    const int64_t groups = (int64_t)gridDim.x * (THREADS >> shift);
    const int lane = threadIdx.x & ((1 << shift) - 1);
    int64_t id[U];
    A w[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int64_t r = group + u * groups;
        id[u] = r < m ? ids[r] : -1;
        w[u] = r < m && weights ? weights[r] * scale : scale;
    }
    for (int64_t c = (int64_t)lane * V; c < p; c += (int64_t)V << shift) {
        A x[U][V];
#pragma unroll
        for (int u = 0; u < U; ++u) load_wide<T, V>(e + (id[u] >= 0 && id[u] < n ? id[u] * lde + c : 0), id[u] >= 0 && id[u] < n ? p - c : 0, x[u]);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int64_t r = group + u * groups;
            if (r >= m) continue;
            if (id[u] >= 0 && id[u] < n) {
#pragma unroll
                for (int i = 0; i < V; ++i) x[u][i] *= w[u];
            }
            store_narrow<T, V>(y + r * ldy + c, p - c, x[u]);
        }
    }
}

// acc += the weighted rows of entries [b, e) at column c, eight rows under way at a time
template <typename T, int V>
__device__ __forceinline__ void add_entries(int64_t b, int64_t e_end, int64_t n, int64_t p, int64_t c, const int32_t* __restrict__ ids,
                                            const typename Wide<T>::type* __restrict__ weights, const T* __restrict__ e, int64_t lde,
                                            typename Wide<T>::type (&acc)[V]) {
    using A = typename Wide<T>::type;
    constexpr int U = V * (int)sizeof(T) >= 16 && sizeof(T) <= 4 ? 8 : 4;
    for (int64_t t = b; t < e_end; t += U) {
        int64_t id[U];
        A w[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            id[u] = t + u < e_end ? ids[t + u] : -1;
            w[u] = weights && t + u < e_end ? weights[t + u] : A(1);
        }
        Vec<T, V> x[U];
        const bool whole = p - c >= V;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (id[u] < 0 || id[u] >= n) continue;
            const T* at = e + id[u] * lde + c;
            if (whole) {
                x[u] = *reinterpret_cast<const Vec<T, V>*>(at);
            } else {
#pragma unroll
                for (int i = 0; i < V; ++i)
                    if (c + i < p) x[u].x[i] = at[i];
            }
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (id[u] < 0 || id[u] >= n) continue;
#pragma unroll
            for (int i = 0; i < V; ++i)
                if (c + i < p) acc[i] += w[u] * widen(x[u].x[i]);
        }
    }
}

// A group per row; rows of more than `longest` entries are left to lookup_long_kernel.
template <typename T, int V>
__global__ void __launch_bounds__(THREADS) lookup_rows_kernel(Rows a, int64_t n, int64_t p, const int32_t* __restrict__ ids,
                                                              const typename Wide<T>::type* __restrict__ weights, typename Wide<T>::type scale,
                                                              const T* __restrict__ e, int64_t lde, T* __restrict__ y, int64_t ldy, int shift,
                                                              int64_t longest) {
    using A = typename Wide<T>::type;
    chain_begin();
    const int64_t row = (int64_t)blockIdx.x * (THREADS >> shift) + (threadIdx.x >> shift);
    const int lane = threadIdx.x & ((1 << shift) - 1);
    if (row < a.m) {
        const int64_t b = a.begin(row), end = a.end(row);
        if (end - b <= longest) {
            for (int64_t c = (int64_t)lane * V; c < p; c += (int64_t)V << shift) {
                A acc[V] = {};
                add_entries<T, V>(b, end, n, p, c, ids, weights, e, lde, acc);
#pragma unroll
                for (int i = 0; i < V; ++i) acc[i] *= scale;
                store_narrow<T, V>(y + row * ldy + c, p - c, acc);
            }
        }
    }
    chain_end();
}

// Rows of more than `longest` entries, one after another by a cluster of eight CTAs: all its groups take a contiguous share of the
// entries, the sums are joined in their order through (distributed) shared memory.  blockIdx.y is a slab of columns.  Cluster u looks
// for long rows among the rows u, u + units, ...; every CTA of it sees the same ones.
template <typename T, int V>
__global__ void __cluster_dims__(LONG_CLUSTER, 1, 1) __launch_bounds__(THREADS)
    lookup_long_kernel(Rows a, int64_t n, int64_t p, const int32_t* __restrict__ ids, const typename Wide<T>::type* __restrict__ weights,
                       typename Wide<T>::type scale, const T* __restrict__ e, int64_t lde, T* __restrict__ y, int64_t ldy, int shift,
                       int64_t longest) {
    using A = typename Wide<T>::type;
    __shared__ A part[THREADS * V];
    __shared__ int64_t found[THREADS];
    __shared__ int count;
    chain_begin();
    const uint32_t rank = cluster_rank();
    const int64_t unit = blockIdx.x / LONG_CLUSTER, units = gridDim.x / LONG_CLUSTER;
    const int lanes = 1 << shift, lane = threadIdx.x & (lanes - 1), groups = THREADS >> shift, group = threadIdx.x >> shift;
    const int64_t c = ((int64_t)blockIdx.y * lanes + lane) * V;
    for (int64_t first = unit; first < a.m; first += units * THREADS) {
        if (threadIdx.x == 0) count = 0;
        __syncthreads();
        const int64_t r = first + (int64_t)threadIdx.x * units;
        const bool is_long = r < a.m && a.end(r) - a.begin(r) > longest;
        // the rows in ascending order: a warp's places follow those of the warps before it
        const unsigned votes = __ballot_sync(FULL_MASK, is_long);
        for (int w = 0; w < THREADS / 32; ++w) {
            if ((int)(threadIdx.x >> 5) == w && votes) {
                if (is_long) found[count + __popc(votes & ((1u << lane_id()) - 1u))] = r;
                __syncwarp();
                if (lane_id() == 0) count += __popc(votes);
            }
            __syncthreads();
        }
        const int rows = count;
        for (int f = 0; f < rows; ++f) {
            const int64_t row = found[f], b = a.begin(row), len = a.end(row) - b;
            const int64_t share = (len + (int64_t)LONG_CLUSTER * groups - 1) / ((int64_t)LONG_CLUSTER * groups);
            const int64_t mine = min(len, (rank * (int64_t)groups + group) * share);
            A acc[V] = {};
            if (c < p) add_entries<T, V>(b + mine, b + min(len, mine + share), n, p, c, ids, weights, e, lde, acc);
#pragma unroll
            for (int i = 0; i < V; ++i) part[i * THREADS + threadIdx.x] = acc[i];
            __syncthreads();
            if (group == 0) {
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    for (int g = 1; g < groups; ++g) acc[i] += part[i * THREADS + g * lanes + lane];
                    part[i * THREADS + lane] = acc[i];
                }
            }
            cluster_sync();
            if (rank == 0 && group == 0 && c < p) {
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    for (uint32_t k = 1; k < LONG_CLUSTER; ++k) acc[i] += load_of_rank(part + i * THREADS + lane, k);
                    acc[i] *= scale;
                }
                store_narrow<T, V>(y + row * ldy + c, p - c, acc);
            }
            cluster_sync();
        }
        __syncthreads();
    }
    chain_end(blockIdx.x == 0 && blockIdx.y == 0);
}

// A CTA takes DW_ENTRIES entries, a group of at most 32 lanes four of them at a time; rows are looked for between the CTA's
// first and last one.
constexpr int DW_EACH = 4;
template <typename T, int V>
__global__ void __launch_bounds__(THREADS) lookup_grad_weights_kernel(Rows a, int64_t n, int64_t p, const int32_t* __restrict__ ids,
                                                                      typename Wide<T>::type scale, const T* __restrict__ e, int64_t lde,
                                                                      const T* __restrict__ dy, int64_t lddy,
                                                                      typename Wide<T>::type* __restrict__ dw, int shift) {
    using A = typename Wide<T>::type;
    __shared__ int64_t span[2];
    const int lanes = 1 << shift, lane = threadIdx.x & (lanes - 1);
    const int64_t here = (int64_t)(THREADS >> shift) * DW_EACH, base = (int64_t)blockIdx.x * here;
    if (a.rowptr) {
        if (threadIdx.x < 2) span[threadIdx.x] = a.row_of(threadIdx.x == 0 ? base : min(base + here, a.nnz) - 1, 0, a.m - 1);
        __syncthreads();
    }
    const int64_t t0 = base + (int64_t)(threadIdx.x >> shift) * DW_EACH;
    const T *row[DW_EACH], *line[DW_EACH];
    A dot[DW_EACH] = {};
#pragma unroll
    for (int u = 0; u < DW_EACH; ++u) {
        const int64_t t = t0 + u, id = t < a.nnz ? ids[t] : -1;
        line[u] = id >= 0 && id < n && a.covered(t) ? e + id * lde : nullptr;
        row[u] = line[u] ? dy + (a.rowptr ? a.row_of(t, span[0], span[1]) : t / a.k) * lddy : nullptr;
    }
    for (int64_t c = (int64_t)lane * V; c < p; c += (int64_t)V << shift) {
        A x[DW_EACH][V], g[DW_EACH][V];
#pragma unroll
        for (int u = 0; u < DW_EACH; ++u) {
            load_wide<T, V>(line[u] ? line[u] + c : e, line[u] ? p - c : 0, x[u]);
            load_wide<T, V>(row[u] ? row[u] + c : dy, row[u] ? p - c : 0, g[u]);
        }
#pragma unroll
        for (int u = 0; u < DW_EACH; ++u)
#pragma unroll
            for (int i = 0; i < V; ++i) dot[u] += x[u][i] * g[u][i];
    }
#pragma unroll
    for (int u = 0; u < DW_EACH; ++u) {
        for (int o = lanes >> 1; o > 0; o >>= 1) dot[u] += __shfl_xor_sync(FULL_MASK, dot[u], o);
        if (lane == 0 && t0 + u < a.nnz) dw[t0 + u] = line[u] ? dot[u] * scale : A(0);
    }
}

template <typename T, int V>
spsyrk_status_t lookup_typed(const Rows& a, int64_t n, int64_t p, const int32_t* ids, const void* weights, double scale, const void* e, int64_t lde,
                             void* y, int64_t ldy, cudaStream_t st) {
    using A = typename Wide<T>::type;
    const A* wv = static_cast<const A*>(weights);
    const T* ev = static_cast<const T*>(e);
    T* yv = static_cast<T*>(y);
    const int shift = group_shift((p + V - 1) / V);
    const int64_t per_cta = THREADS >> shift;
    if (!a.rowptr && a.k == 1) {
        // four rows a group once every SM has its 2048 threads twice over; fewer rows are spread as far as they go
        const bool many = a.m >= 4 * 2 * SMS * 2048 / (1 << shift);
        const int64_t groups = many ? (a.m + 3) / 4 : a.m;
        const unsigned ctas = (unsigned)((groups + per_cta - 1) / per_cta);
        if (many) lookup_one_kernel<T, V, 4><<<ctas, THREADS, 0, st>>>(a.m, n, p, ids, wv, (A)scale, ev, lde, yv, ldy, shift);
        else lookup_one_kernel<T, V, 1><<<ctas, THREADS, 0, st>>>(a.m, n, p, ids, wv, (A)scale, ev, lde, yv, ldy, shift);
        note_launches(1);
        SPSYRK_CUDA_TRY(cudaGetLastError());
        return SPSYRK_OK;
    }
    // A group reads a row eight entries at a time, about a microsecond each; a cluster spends some 3 us on a row beside its loads and
    // 64 of them run at a time.  So few rows go to clusters from 128 entries on, of many only those far above the mean.
    const int64_t longest = a.m <= 4 * LONG_UNITS ? 128 : std::max<int64_t>(512, 4 * (a.nnz / a.m));
    Chain chain{st, true};
    if (a.rowptr || a.k <= longest)
        SPSYRK_CUDA_TRY(chain.launch(true, lookup_rows_kernel<T, V>, (unsigned)((a.m + per_cta - 1) / per_cta), THREADS, 0, a, n, p, ids, wv, (A)scale, ev, lde, yv,
                                     ldy, shift, longest));
    if (a.rowptr ? a.nnz > longest : a.k > longest) {
        const int64_t units = std::min<int64_t>(LONG_UNITS, a.m);
        // slabs of at most 64 lanes, for more CTAs
        const int narrow_shift = std::min(shift, 6);
        const int64_t slabs = (p + ((int64_t)V << narrow_shift) - 1) / ((int64_t)V << narrow_shift);
        cudaLaunchConfig_t cfg{};
        cfg.gridDim = dim3((unsigned)(units * LONG_CLUSTER), (unsigned)slabs);
        cfg.blockDim = dim3(THREADS);
        cfg.stream = st;
        cudaLaunchAttribute attr{};
        attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
        attr.val.programmaticStreamSerializationAllowed = 1;
        cfg.attrs = &attr;
        cfg.numAttrs = chain.first ? 0 : 1;
        SPSYRK_CUDA_TRY(launch_kernel(cfg, lookup_long_kernel<T, V>, a, n, p, ids, wv, (A)scale, ev, lde, yv, ldy, narrow_shift, longest));
    }
    return SPSYRK_OK;
}

template <typename T, int V>
spsyrk_status_t grad_weights_typed(const Rows& a, int64_t n, int64_t p, const int32_t* ids, double scale, const void* e, int64_t lde, const void* dy,
                                   int64_t lddy, void* dw, cudaStream_t st) {
    using A = typename Wide<T>::type;
    const int shift = std::min(group_shift((p + V - 1) / V), 5);
    const int64_t here = (int64_t)(THREADS >> shift) * DW_EACH;
    lookup_grad_weights_kernel<T, V><<<(unsigned)((a.nnz + here - 1) / here), THREADS, 0, st>>>(a, n, p, ids, (A)scale, static_cast<const T*>(e), lde,
                                                                                                static_cast<const T*>(dy), lddy, static_cast<A*>(dw), shift);
    note_launches(1);
    SPSYRK_CUDA_TRY(cudaGetLastError());
    return SPSYRK_OK;
}

// What all calls on rows of ids check alike; *rows receives the rows.
spsyrk_status_t check_rows(int64_t m, int64_t n, int64_t p, int64_t nnz, const int64_t* d_rowptr, const int32_t* d_ids, Rows* rows) {
    if (m < 0 || n < 0 || p < 0 || nnz < 0 || (nnz > 0 && !d_ids)) return SPSYRK_ERR_INVALID_ARG;
    constexpr int64_t most = (int64_t(1) << 31) - 1;
    if (m >= most || n >= most || nnz >= most || p > (int64_t(1) << 22)) return SPSYRK_ERR_OVERFLOW;
    if (!d_rowptr && (m == 0 ? nnz != 0 : nnz % m != 0)) return SPSYRK_ERR_INVALID_ARG;
    *rows = Rows{d_rowptr, m, nnz, m > 0 ? nnz / m : 0};
    return SPSYRK_OK;
}

}  // namespace

// a typed call, 16 bytes at a time if everything is aligned to that
#define SPSYRK_BY_TYPE(dtype, wide, call)                                               \
    switch (dtype) {                                                                    \
        case SPSYRK_F64: return wide ? call(double, 2) : call(double, 1);               \
        case SPSYRK_F32: return wide ? call(float, 4) : call(float, 1);                 \
        case SPSYRK_BF16: return wide ? call(__nv_bfloat16, 8) : call(__nv_bfloat16, 1); \
        default: return wide ? call(__half, 8) : call(__half, 1);                       \
    }

extern "C" spsyrk_status_t spsyrk_lookup(int64_t m, int64_t n, int64_t p, int64_t nnz, spsyrk_dtype_t dtype, const int64_t* d_rowptr,
                                         const int32_t* d_ids, const void* d_weights, double scale, const void* d_e, int64_t lde, void* d_y,
                                         int64_t ldy, void* cuda_stream) {
    Rows a{};
    const spsyrk_status_t s = check_rows(m, n, p, nnz, d_rowptr, d_ids, &a);
    if (s != SPSYRK_OK) return s;
    if (!is_real(dtype) || lde < p || ldy < p) return SPSYRK_ERR_INVALID_ARG;
    if (m == 0 || p == 0) return SPSYRK_OK;
    if (!d_y || (n > 0 && nnz > 0 && !d_e)) return SPSYRK_ERR_INVALID_ARG;
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    const size_t size = element_size(dtype);
    const bool wide = aligned16(d_e, lde, size) && aligned16(d_y, ldy, size);
#define CALL(T, V) (lookup_typed<T, V>(a, n, p, d_ids, d_weights, scale, d_e, lde, d_y, ldy, st))
    SPSYRK_BY_TYPE(dtype, wide, CALL)
#undef CALL
}

extern "C" spsyrk_status_t spsyrk_lookup_grad_weights(int64_t m, int64_t n, int64_t p, int64_t nnz, spsyrk_dtype_t dtype, const int64_t* d_rowptr,
                                                      const int32_t* d_ids, double scale, const void* d_e, int64_t lde, const void* d_dy, int64_t lddy,
                                                      void* d_dw, void* cuda_stream) {
    Rows a{};
    const spsyrk_status_t s = check_rows(m, n, p, nnz, d_rowptr, d_ids, &a);
    if (s != SPSYRK_OK) return s;
    if (!is_real(dtype) || lde < p || lddy < p) return SPSYRK_ERR_INVALID_ARG;
    if (nnz == 0) return SPSYRK_OK;
    if (m == 0 || !d_dw || (n > 0 && p > 0 && (!d_e || !d_dy))) return SPSYRK_ERR_INVALID_ARG;
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    const size_t size = element_size(dtype);
    const bool wide = aligned16(d_e, lde, size) && aligned16(d_dy, lddy, size);
#define CALL(T, V) (grad_weights_typed<T, V>(a, n, p, d_ids, scale, d_e, lde, d_dy, lddy, d_dw, st))
    SPSYRK_BY_TYPE(dtype, wide, CALL)
#undef CALL
}
