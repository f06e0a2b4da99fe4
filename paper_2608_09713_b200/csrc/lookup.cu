// Y = scale * A E for rows of ids A and a dense table E (an embedding lookup, or sums over bags of ids), and the gradient of the
// weights, dw_t = scale * <E[id_t], dY[row of t]>.
//
// Both move every row of E that they name and do two operations per element: bound by memory where rows are wide, by latency for few rows, and
// by latency for sums over many narrow rows (10000 sets of up to 140 rows of 64 floats 52 us, their weights' gradient 60: issue slots half used, 26 and
// 33 % of an SM's warps, L2 at 9 %).
// A group of 1 to 256 lanes holds a row of Y, 16 bytes a lane, and keeps its sum in registers.
#include <algorithm>

#include "element.cuh"

using namespace spsyrk;

namespace {

constexpr int THREADS = 256;
constexpr int SMS = 148;
constexpr int LONG_CLUSTER = 8;
constexpr int LONG_UNITS = 64;  // clusters that look for long rows

// Where rows are gathered entry by entry, two 16-bit elements at a time are slower than one (2500 sets of 40 of 1002 bfloat16 columns 176 us against
// 143, the gradient of their weights 141 against 129); two floats are faster (90 against 150, 100 against 166).
template <typename T, int V> constexpr int BY_ENTRIES = V == 2 && sizeof(T) == 2 ? 1 : V;

// lanes of a group: a power of two that covers the row's vectors, at most a CTA
int group_shift(int64_t vectors) {
    int s = 0;
    while ((int64_t(1) << s) < vectors && s < 8) ++s;
    return s;
}

// One id a row, a group per row.  (Four rows per group, for four loads of a lane under way at a time, took 60 us instead of 47 for 20011 rows
// of 4096 bfloat16: as many CTAs with fewer registers hide more.)
template <typename T, int V>
__global__ void __launch_bounds__(THREADS) lookup_one_kernel(int64_t m, int64_t n, int64_t p, const int32_t* __restrict__ ids,
                                                             const typename Wide<T>::type* __restrict__ weights, typename Wide<T>::type scale,
                                                             const T* __restrict__ e, int64_t lde, T* __restrict__ y, int64_t ldy, int shift) {
    using A = typename Wide<T>::type;
    const int64_t r = (int64_t)blockIdx.x * (THREADS >> shift) + (threadIdx.x >> shift);
    const int lane = threadIdx.x & ((1 << shift) - 1);
    if (r >= m) return;
    const int64_t id = ids[r];
    const bool held = id >= 0 && id < n;
    const A w = held && weights ? weights[r] * scale : scale;
    for (int64_t c = (int64_t)lane * V; c < p; c += (int64_t)V << shift) {
        A x[V] = {};
        if (held) {
            load_wide<T, V>(e + id * lde + c, p - c, x);
#pragma unroll
            for (int i = 0; i < V; ++i) x[i] *= w;
        }
        store_narrow<T, V>(y + r * ldy + c, p - c, x);
    }
}

// acc += the weighted rows of entries [b, end) at column c, UNROLL rows under way at a time.  The lanes of a group (those of it that
// share a warp) fetch an id and a weight each and hand them round; the next ones are under way meanwhile.
// (eight sums a lane leave registers for four rows of 16 bytes at a time, fewer sums for eight)
template <int V> constexpr int UNROLL = V == 8 ? 4 : 8;
template <typename T, int V>
__device__ __forceinline__ void add_entries(int64_t b, int64_t end, int64_t n, int64_t p, int64_t c, const int32_t* __restrict__ ids,
                                            const typename Wide<T>::type* __restrict__ weights, const T* __restrict__ e, int64_t lde, int shift,
                                            typename Wide<T>::type (&acc)[V]) {
    using A = typename Wide<T>::type;
    constexpr int U = UNROLL<V>;
    const int share = 1 << min(shift, 5), lane = threadIdx.x & (share - 1);
    const unsigned mask = share == 32 ? FULL_MASK : ((1u << share) - 1) << (lane_id() & ~(share - 1));
    int32_t next_id = -1;
    A next_w = A(1);
    auto ask = [&](int64_t t) {
        next_id = t + lane < end ? ids[t + lane] : -1;
        if (weights) next_w = t + lane < end ? weights[t + lane] : A(0);
    };
    ask(b);
    for (int64_t t = b; t < end; t += share) {
        const int32_t my_id = next_id >= 0 && next_id < n ? next_id : -1;
        const A my_w = next_w;
        ask(t + share);
        const int count = (int)min((int64_t)share, end - t);
        for (int k = 0; k < count; k += U) {
            int32_t id[U];
            Vec<T, V> x[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                // (a lane beyond the group's gives an id of the group again)
                const int32_t got = __shfl_sync(mask, my_id, k + u, share);
                id[u] = k + u < count ? got : -1;
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (id[u] < 0) continue;
                x[u] = load_raw<T, V>(e + id[u] * lde + c, p - c);
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const A w = weights ? __shfl_sync(mask, my_w, k + u, share) : A(1);
                if (id[u] < 0) continue;
#pragma unroll
                for (int i = 0; i < V; ++i) acc[i] += w * widen(x[u].x[i]);
            }
        }
    }
}

// A group per row; rows of more than `longest` entries are left to lookup_long_kernel.  Few narrow rows: 1 << split groups of a warp share a row,
// each takes a contiguous share of the entries.
template <typename T, int V, bool SHARED>
__global__ void __launch_bounds__(THREADS, 3) lookup_rows_kernel(Rows a, int64_t n, int64_t p, const int32_t* __restrict__ ids,
                                                                 const typename Wide<T>::type* __restrict__ weights, typename Wide<T>::type scale,
                                                                 const T* __restrict__ e, int64_t lde, T* __restrict__ y, int64_t ldy, int shift, int split,
                                                                 int64_t longest) {
    using A = typename Wide<T>::type;
    chain_begin();
    if (!SHARED) split = 0;
    const int all = shift + split;  // at most 5 if split > 0
    const int64_t row = (int64_t)blockIdx.x * (THREADS >> all) + (threadIdx.x >> all);
    const int lane = threadIdx.x & ((1 << shift) - 1), part = (threadIdx.x >> shift) & ((1 << split) - 1);
    const unsigned mask = all >= 5 ? FULL_MASK : ((1u << (1 << all)) - 1) << (lane_id() & ~((1 << all) - 1));
    if (row < a.m) {
        const int64_t begin = a.begin(row), len = a.end(row) - begin;
        if (len <= longest) {
            const int64_t each = (max(len, (int64_t)0) + (1 << split) - 1) >> split, b = begin + min(len, part * each), end = begin + min(len, (part + 1) * each);
            // (all lanes of a group stay together: they hand ids round)
            for (int64_t c0 = 0; c0 < p; c0 += (int64_t)V << shift) {
                const int64_t c = c0 + (int64_t)lane * V;
                A acc[V] = {};
                add_entries<T, V>(b, end, n, p, c, ids, weights, e, lde, shift, acc);
                if (SHARED) {
                    __syncwarp(mask);
                    for (int s = 0; s < split; ++s) {
#pragma unroll
                        for (int i = 0; i < V; ++i) acc[i] += __shfl_xor_sync(mask, acc[i], 1 << (shift + s));
                    }
                }
#pragma unroll
                for (int i = 0; i < V; ++i) acc[i] *= scale;
                if (part == 0 && c < p) store_narrow<T, V>(y + row * ldy + c, p - c, acc);
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
            add_entries<T, V>(b + mine, b + min(len, mine + share), n, p, c, ids, weights, e, lde, shift, acc);
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

// A group of up to 32 lanes takes `each` consecutive entries, DW_EACH of them at a time.  Every lane fetches an id and looks for its
// row (between the CTA's first and last one) and hands them round.  Entries of the same row share the loads of dY.
constexpr int DW_EACH = 8;
template <typename T, int V>
__global__ void __launch_bounds__(THREADS, 3) lookup_grad_weights_kernel(Rows a, int64_t n, int64_t p, const int32_t* __restrict__ ids,
                                                                      typename Wide<T>::type scale, const T* __restrict__ e, int64_t lde,
                                                                      const T* __restrict__ dy, int64_t lddy,
                                                                      typename Wide<T>::type* __restrict__ dw, int shift, int each) {
    using A = typename Wide<T>::type;
    __shared__ int64_t span[2];
    const int lanes = 1 << shift, lane = threadIdx.x & (lanes - 1);
    const unsigned mask = lanes == 32 ? FULL_MASK : ((1u << lanes) - 1) << (lane_id() & ~(lanes - 1));
    const int64_t here = (int64_t)(THREADS >> shift) * each, base = (int64_t)blockIdx.x * here;
    const int64_t t0 = base + (int64_t)(threadIdx.x >> shift) * each, t1 = min(t0 + each, a.nnz);
    int32_t ahead = t0 + lane < t1 ? ids[t0 + lane] : -1;
    if (a.rowptr) {
        if (threadIdx.x < 64) {
            const int64_t r = a.row_of_by_warp(threadIdx.x < 32 ? base : min(base + here, a.nnz) - 1);
            if (lane_id() == 0) span[threadIdx.x >> 5] = r;
        }
        __syncthreads();
    }
    for (int64_t t = t0; t < t1; t += lanes) {
        int32_t my_id = ahead, my_row = 0;
        ahead = t + lanes + lane < t1 ? ids[t + lanes + lane] : -1;
        if (my_id >= n || (my_id >= 0 && !a.covered(t + lane))) my_id = -1;
        if (my_id >= 0) my_row = (int32_t)(a.rowptr ? a.row_of(t + lane, span[0], span[1]) : (t + lane) / a.k);
        for (int k = 0; k < lanes && t + k < t1; k += DW_EACH) {
            int32_t id[DW_EACH], row[DW_EACH];
            A dot[DW_EACH] = {};
            bool same = true;  // all of one row, or padding
            int32_t the_row = -1;
#pragma unroll
            for (int u = 0; u < DW_EACH; ++u) {
                const int32_t got = __shfl_sync(mask, my_id, k + u, lanes);
                row[u] = __shfl_sync(mask, my_row, k + u, lanes);
                id[u] = k + u < lanes ? got : -1;
                if (id[u] >= 0) {
                    same &= the_row < 0 || the_row == row[u];
                    the_row = row[u];
                }
            }
            if (the_row >= 0) {
                for (int64_t c = (int64_t)lane * V; c < p; c += (int64_t)V << shift) {
                    A g[V];
                    if (same) load_wide<T, V>(dy + the_row * lddy + c, p - c, g);
#pragma unroll
                    for (int h = 0; h < DW_EACH; h += DW_EACH / 2) {  // (half of the entries at a time: registers)
                        Vec<T, V> x[DW_EACH / 2];
#pragma unroll
                        for (int u = 0; u < DW_EACH / 2; ++u)
                            if (id[h + u] >= 0) x[u] = load_raw<T, V>(e + id[h + u] * lde + c, p - c);
#pragma unroll
                        for (int u = 0; u < DW_EACH / 2; ++u) {
                            if (!same) load_wide<T, V>(id[h + u] >= 0 ? dy + row[h + u] * lddy + c : dy, id[h + u] >= 0 ? p - c : 0, g);
                            if (id[h + u] < 0) continue;
#pragma unroll
                            for (int i = 0; i < V; ++i) dot[h + u] += widen(x[u].x[i]) * g[i];
                        }
                    }
                }
            }
            // every dot product over the lanes; with eight lanes or more a step halves what a lane holds
            int place = 0;
            if (lanes >= DW_EACH) {
#pragma unroll
                for (int s = 0; s < 5; ++s) {
                    if (1 << s >= lanes) break;
                    const bool upper = lane >> s & 1;
                    const int half = DW_EACH >> (s + 1);
                    if (half > 0) {
#pragma unroll
                        for (int i = 0; i < half; ++i) {
                            const A keep = upper ? dot[i + half] : dot[i], give = upper ? dot[i] : dot[i + half];
                            dot[i] = keep + __shfl_xor_sync(mask, give, 1 << s);
                        }
                        place += upper ? half : 0;
                    } else {
                        dot[0] += __shfl_xor_sync(mask, dot[0], 1 << s);
                    }
                }
                if (lane < DW_EACH && t + k + place < t1) dw[t + k + place] = dot[0] * scale;
            } else {
#pragma unroll
                for (int u = 0; u < DW_EACH; ++u) {
                    for (int o = lanes >> 1; o > 0; o >>= 1) dot[u] += __shfl_xor_sync(mask, dot[u], o);
                    if (lane == 0 && k + u < lanes && t + k + u < t1) dw[t + k + u] = dot[u] * scale;
                }
            }
        }
    }
}

// Rows of one id each.
template <typename T, int V>
spsyrk_status_t lookup_one_typed(const Rows& a, int64_t n, int64_t p, const int32_t* ids, const void* weights, double scale, const void* e, int64_t lde,
                             void* y, int64_t ldy, cudaStream_t st) {
    using A = typename Wide<T>::type;
    const A* wv = static_cast<const A*>(weights);
    const T* ev = static_cast<const T*>(e);
    T* yv = static_cast<T*>(y);
    const int shift = group_shift((p + V - 1) / V);
    const int64_t per_cta = THREADS >> shift;
    lookup_one_kernel<T, V><<<(unsigned)((a.m + per_cta - 1) / per_cta), THREADS, 0, st>>>(a.m, n, p, ids, wv, (A)scale, ev, lde, yv, ldy, shift);
    note_launches(1);
    SPSYRK_CUDA_TRY(cudaGetLastError());
    return SPSYRK_OK;
}

// Rows of any number.
template <typename T, int V>
spsyrk_status_t lookup_rows_typed(const Rows& a, int64_t n, int64_t p, const int32_t* ids, const void* weights, double scale, const void* e, int64_t lde,
                             void* y, int64_t ldy, cudaStream_t st) {
    using A = typename Wide<T>::type;
    const A* wv = static_cast<const A*>(weights);
    const T* ev = static_cast<const T*>(e);
    T* yv = static_cast<T*>(y);
    const int shift = group_shift((p + V - 1) / V);
    // A group reads a row eight entries at a time, about a microsecond each; a cluster spends some 3 us on a row beside its loads and
    // 64 of them run at a time.  So few rows go to clusters from 128 entries on, more rows from 512 on, and of rows that fill the GPU by themselves
    // only those far above the mean.
    const int64_t longest = a.m <= 4 * LONG_UNITS ? 128 : a.m << shift < (int64_t)SMS * 1024 ? 512 : std::max<int64_t>(512, 4 * (a.nnz / a.m));
    Chain chain{st, true};
    if (a.rowptr || a.k <= longest) {
        // rows are shared while they do not fill every SM with threads and have eight entries for everyone
        int split = 0;
        while (shift + split < 5 && a.m << (shift + split) < (int64_t)SMS * 2048 && a.nnz / a.m >= int64_t(16) << split) ++split;
        const int64_t rows = THREADS >> (shift + split);
        const auto kernel = split ? lookup_rows_kernel<T, V, true> : lookup_rows_kernel<T, V, false>;
        SPSYRK_CUDA_TRY(chain.launch(true, kernel, (unsigned)((a.m + rows - 1) / rows), THREADS, 0, a, n, p, ids, wv, (A)scale, ev, lde, yv,
                                     ldy, shift, split, longest));
    }
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
spsyrk_status_t lookup_typed(const Rows& a, int64_t n, int64_t p, const int32_t* ids, const void* weights, double scale, const void* e, int64_t lde,
                             void* y, int64_t ldy, cudaStream_t st) {
    // (two floats at a time copy no faster than one: 20000 rows of 1002 51 us against 45)
    if (!a.rowptr && a.k == 1) return lookup_one_typed<T, V == 2 && sizeof(T) == 4 ? 1 : V>(a, n, p, ids, weights, scale, e, lde, y, ldy, st);
    return lookup_rows_typed<T, BY_ENTRIES<T, V>>(a, n, p, ids, weights, scale, e, lde, y, ldy, st);
}

template <typename T, int V>
spsyrk_status_t grad_weights_typed(const Rows& a, int64_t n, int64_t p, const int32_t* ids, double scale, const void* e, int64_t lde, const void* dy,
                                   int64_t lddy, void* dw, cudaStream_t st) {
    using A = typename Wide<T>::type;
    const int shift = std::min(group_shift((p + V - 1) / V), 5);
    // 32 entries a group if their groups still fill every SM with threads, down to 8 if not
    int each = 32;
    while (each > DW_EACH && (a.nnz / each << shift) < (int64_t)SMS * 2048) each /= 2;
    const int64_t here = (int64_t)(THREADS >> shift) * each;
    lookup_grad_weights_kernel<T, V><<<(unsigned)((a.nnz + here - 1) / here), THREADS, 0, st>>>(a, n, p, ids, (A)scale, static_cast<const T*>(e), lde,
                                                                                                static_cast<const T*>(dy), lddy, static_cast<A*>(dw), shift, each);
    note_launches(1);
    SPSYRK_CUDA_TRY(cudaGetLastError());
    return SPSYRK_OK;
}

// What all calls on rows of ids check alike; *rows receives the rows.
spsyrk_status_t check_rows(int64_t m, int64_t n, int64_t p, int64_t nnz, const int64_t* d_rowptr, const int32_t* d_ids, Rows* rows) {
    if (m < 0 || n < 0 || p < 0 || nnz < 0 || (nnz > 0 && !d_ids)) return SPSYRK_ERR_INVALID_ARG;
    constexpr int64_t most = (int64_t(1) << 31) - 1;
    if (m >= most || n >= most || nnz >= most || p > (int64_t(1) << 21)) return SPSYRK_ERR_OVERFLOW;
    if (!d_rowptr && (m == 0 ? nnz != 0 : nnz % m != 0)) return SPSYRK_ERR_INVALID_ARG;
    *rows = Rows{d_rowptr, m, nnz, m > 0 ? nnz / m : 0};
    return SPSYRK_OK;
}

}  // namespace

// a typed call with as many elements together as all matrices allow (8, 4 or 2 for 2-, 4- and 8-byte elements; 2; 1)
#define SPSYRK_BY_TYPE(dtype, width, call)                                                                                               \
    switch (dtype) {                                                                                                                     \
        case SPSYRK_F64: return width >= 2 ? call(double, 2) : call(double, 1);                                                          \
        case SPSYRK_F32: return width >= 4 ? call(float, 4) : width == 2 ? call(float, 2) : call(float, 1);                              \
        case SPSYRK_BF16: return width >= 8 ? call(__nv_bfloat16, 8) : width == 2 ? call(__nv_bfloat16, 2) : call(__nv_bfloat16, 1);     \
        default: return width >= 8 ? call(__half, 8) : width == 2 ? call(__half, 2) : call(__half, 1);                                   \
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
    const int width = std::min(together(d_e, lde, size), together(d_y, ldy, size));
#define CALL(T, V) (lookup_typed<T, V>(a, n, p, d_ids, d_weights, scale, d_e, lde, d_y, ldy, st))
    SPSYRK_BY_TYPE(dtype, width, CALL)
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
    if (!d_dw || (m > 0 && n > 0 && p > 0 && (!d_e || !d_dy))) return SPSYRK_ERR_INVALID_ARG;
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    const size_t size = element_size(dtype);
    if (m == 0) {  // entries of no row
        SPSYRK_CUDA_TRY(cudaMemsetAsync(d_dw, 0, (size_t)nnz * (dtype == SPSYRK_F64 ? 8 : 4), st));
        return SPSYRK_OK;
    }
    const int width = std::min(together(d_e, lde, size), together(d_dy, lddy, size));
#define CALL(T, V) (grad_weights_typed<T, BY_ENTRIES<T, V>>(a, n, p, d_ids, scale, d_e, lde, d_dy, lddy, d_dw, st))
    SPSYRK_BY_TYPE(dtype, width, CALL)
#undef CALL
}
