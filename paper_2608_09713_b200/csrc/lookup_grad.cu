// dE = scale * A^T dY for rows of ids A: the gradient of an embedding lookup with respect to its table, by sorted ids.
//
// The entries are ordered by id with a stable sort (entries of an id stay in their order), and the ordered list is cut into pieces of
// the same length.  A group of lanes adds up a piece, 16 bytes of dY a lane, run by run (a run = the entries of one id): a run that lies
// inside the piece is written to its row of dE at once, one that crosses the piece's ends leaves its partial sum in the workspace, and
// the partial sums of such a run are added up in their order by a second kernel.  No atomic adds: the same call gives the same bits,
// and an id that every second entry has costs no more than others.  Rows of ids that do not occur are filled with zeros by further
// CTAs, which find them in a bit per id that is set while the ids are read.
// Bound by memory: dY is read once (a row of several ids once per id, through L2), dE written once.
#include <algorithm>

#include "element.cuh"
#include "radix.cuh"

using namespace spsyrk;

namespace {

constexpr size_t ALIGN = 256;
constexpr int THREADS = 256;
constexpr int SMS = 148;
constexpr int64_t FEW = 8192;  // entries that are ranked by comparing all with all instead of sorted by digits
constexpr int MIN_PIECE = 4, MAX_PIECE = 32;

// Entries of a piece: 32 if their groups still fill every SM with threads, fewer if not.  (Lanes of 8 elements, whatever the type: the
// workspace's size depends on it.)
int piece_of(int64_t nnz, int64_t p) {
    int c = MAX_PIECE;
    while (c > MIN_PIECE && nnz / c * ((p + 7) / 8) < (int64_t)SMS * 2048) c /= 2;
    return c;
}

struct GradWs {
    uint32_t *key[2], *row[2];  // ids (n: padding) and rows of the entries, before and after a pass
    void* weight[2];
    uint32_t* present;  // a bit per id
    void* part;         // [pieces][2][p] partial sums: of a run that comes from the piece before, of one that begins here and goes on
    RadixState rs;
    uint32_t* err;
    void* zero;
    size_t zero_bytes;
};

size_t carve(GradWs* w, void* ws, int64_t n, int64_t p, int64_t nnz, bool wide, bool weighted) {
    char* base = static_cast<char*>(ws);
    size_t off = 0;
    auto take = [&](size_t bytes) -> void* {
        off = (off + ALIGN - 1) / ALIGN * ALIGN;
        void* q = base ? base + off : nullptr;
        off += bytes;
        return q;
    };
    const int64_t ne = std::max<int64_t>(nnz, 1), acc = wide ? 8 : 4;
    GradWs t;
    for (int i = 0; i < 2; ++i) {
        t.key[i] = (uint32_t*)take(ne * 4);
        t.row[i] = (uint32_t*)take(ne * 4);
        t.weight[i] = weighted ? take(ne * acc) : nullptr;
    }
    const int piece = piece_of(nnz, p);
    t.part = take((size_t)((ne + piece - 1) / piece) * 2 * p * acc);
    // what has to be zero at the start, in one piece
    const size_t bits = ((size_t)n / 32 + 1) * 4 / 8 * 8 + 8;
    const size_t words = nnz > FEW ? radix_state_words(radix_tiles(nnz), radix_wide(nnz), radix_passes((uint64_t)n)) : 0;
    t.zero_bytes = bits + (1 + RX_MAX_PASSES * RX_BINS + RX_MAX_PASSES + words) * 8;
    t.zero = take(t.zero_bytes);
    char* z = (char*)t.zero;
    t.present = (uint32_t*)z;
    t.err = (uint32_t*)(z + bits);
    t.rs.bins = (unsigned long long*)(z + bits) + 1;
    t.rs.tickets = (uint32_t*)(t.rs.bins + RX_MAX_PASSES * RX_BINS);
    t.rs.words = t.rs.bins + RX_MAX_PASSES * RX_BINS + RX_MAX_PASSES;
    if (w) *w = t;
    return (off + ALIGN - 1) / ALIGN * ALIGN;
}

// Key and row of every entry, a bit per id that occurs and, for the sort, the sizes of all digits.
constexpr int READ_ITEMS = 4;
constexpr int READ_CHUNK = THREADS * READ_ITEMS;
__global__ void __launch_bounds__(THREADS) read_ids_kernel(Rows a, int64_t n, const int32_t* __restrict__ ids, uint32_t* __restrict__ key,
                                                           uint32_t* __restrict__ row, uint32_t* __restrict__ present, int passes,
                                                           unsigned long long* __restrict__ bins) {
    __shared__ int64_t span[2];
    __shared__ uint32_t h[RX_MAX_PASSES][RX_BINS];
    for (int d = threadIdx.x; d < RX_MAX_PASSES * RX_BINS; d += THREADS) (&h[0][0])[d] = 0;
    const int64_t base = (int64_t)blockIdx.x * READ_CHUNK;
    if (a.rowptr && threadIdx.x < 2) span[threadIdx.x] = a.row_of(threadIdx.x == 0 ? base : min(base + READ_CHUNK, a.nnz) - 1, 0, a.m - 1);
    __syncthreads();
#pragma unroll
    for (int i = 0; i < READ_ITEMS; ++i) {
        const int64_t t = base + i * THREADS + threadIdx.x;
        if (t >= a.nnz) continue;
        const int64_t id = ids[t], r = a.rowptr ? a.row_of(t, span[0], span[1]) : t / a.k;
        const bool held = id >= 0 && id < n && a.covered(t);
        const uint32_t k = held ? (uint32_t)id : (uint32_t)n;
        key[t] = k;
        row[t] = (uint32_t)r;
        if (held) atomicOr(present + (k >> 5), 1u << (k & 31));
        for (int q = 0; q < passes; ++q) atomicAdd(&h[q][(k >> (q * RX_BITS)) & (RX_BINS - 1)], 1u);
    }
    __syncthreads();
    for (int d = threadIdx.x; d < passes * RX_BINS; d += THREADS)
        if ((&h[0][0])[d]) atomicAdd(&bins[d], (unsigned long long)(&h[0][0])[d]);
}

// Up to FEW entries: an entry's place in the order is the number of entries with a smaller id, or with the same one before it.  A
// warp counts for four entries at a time.
constexpr int RANK_EACH = 4;
template <typename A>
__global__ void __launch_bounds__(THREADS) rank_kernel(Rows a, int64_t n, const int32_t* __restrict__ ids, const A* __restrict__ weights,
                                                       uint32_t* __restrict__ key, uint32_t* __restrict__ row, A* __restrict__ weight,
                                                       uint32_t* __restrict__ present) {
    const int lane = lane_id();
    const int nnz = (int)a.nnz, t0 = (int)(blockIdx.x * (THREADS / 32) + (threadIdx.x >> 5)) * RANK_EACH;
    const int64_t from = a.rowptr ? a.rowptr[0] : 0, to = a.rowptr ? a.rowptr[a.m] : a.nnz;
    auto key_of = [&](int t) {
        const int64_t id = ids[t];
        return id >= 0 && id < n && t >= from && t < to ? (uint32_t)id : (uint32_t)n;
    };
    uint32_t mine[RANK_EACH];
    int before[RANK_EACH] = {};
#pragma unroll
    for (int u = 0; u < RANK_EACH; ++u) mine[u] = t0 + u < nnz ? key_of(t0 + u) : 0u;
    if (t0 >= nnz) return;
    for (int t = lane; t < nnz; t += 32) {
        const uint32_t k = key_of(t);
#pragma unroll
        for (int u = 0; u < RANK_EACH; ++u) before[u] += k < mine[u] || (k == mine[u] && t < t0 + u);
    }
#pragma unroll
    for (int u = 0; u < RANK_EACH; ++u) {
        const int at = __reduce_add_sync(FULL_MASK, before[u]);
        const int t = t0 + u;
        if (lane != 0 || t >= nnz) continue;
        key[at] = mine[u];
        row[at] = (uint32_t)a.row_of(t, 0, a.m - 1);
        if (weight) weight[at] = weights[t];
        if (mine[u] < (uint32_t)n) atomicOr(present + (mine[u] >> 5), 1u << (mine[u] & 31));
    }
}

template <typename PB>
struct EmitOrdered {
    uint32_t *key, *row;
    PB* weight;
    __device__ __forceinline__ void operator()(int64_t dest, uint32_t k, uint32_t r, PB w) const {
        key[dest] = k;
        row[dest] = r;
        if (weight) weight[dest] = w;
    }
};

template <typename G, typename A, int V>
__device__ __forceinline__ void write_row(G* __restrict__ at, int64_t left, A scale, bool accumulate, A (&x)[V]) {
#pragma unroll
    for (int i = 0; i < V; ++i) x[i] *= scale;
    if (accumulate) {
        A old[V];
        load_wide<G, V>(at, left, old);
#pragma unroll
        for (int i = 0; i < V; ++i) x[i] += old[i];
    }
    store_narrow<G, V>(at, left, x);
}

// CTAs below `piece_ctas` add up pieces; those behind fill the rows of dE without entries, `fill_rows` each.
template <typename T, typename G, int V>
__global__ void __launch_bounds__(THREADS) add_pieces_kernel(int64_t nnz, int64_t n, int64_t p, const uint32_t* __restrict__ key,
                                                             const uint32_t* __restrict__ row, const typename Wide<T>::type* __restrict__ weight,
                                                             typename Wide<T>::type scale, const T* __restrict__ dy, int64_t lddy, G* __restrict__ de,
                                                             int64_t ldde, bool accumulate, typename Wide<T>::type* __restrict__ part, int piece,
                                                             int shift, int64_t slabs, int64_t piece_ctas, const uint32_t* __restrict__ present,
                                                             int64_t fill_rows) {
    using A = typename Wide<T>::type;
    link(key, row, weight, present);
    if ((int64_t)blockIdx.x >= piece_ctas) {
        const int64_t v0 = ((int64_t)blockIdx.x - piece_ctas) * fill_rows, v1 = min(v0 + fill_rows, n);
        // up to a warp per row: elements up to the first 16-byte boundary, 16 bytes a lane, the elements behind
        const int fs = min(5, 32 - __clz((int)min((p * (int64_t)sizeof(G) + 15) / 16, (int64_t)32) - 1));
        const int lane = threadIdx.x & ((1 << fs) - 1);
        for (int64_t v = v0 + (threadIdx.x >> fs); v < v1; v += THREADS >> fs) {
            if (present[v >> 5] >> (v & 31) & 1u) continue;
            G* const at = de + v * ldde;
            const int64_t head = min(p, (int64_t)((0 - reinterpret_cast<uintptr_t>(at)) % 16 / sizeof(G)));
            const int64_t body = (p - head) / (16 / (int)sizeof(G)), tail = head + body * (16 / (int)sizeof(G));
            for (int64_t c = lane; c < head; c += 1 << fs) at[c] = narrow<G>(typename Wide<G>::type(0));
            for (int64_t c = lane; c < body; c += 1 << fs) reinterpret_cast<uint4*>(at + head)[c] = uint4{0, 0, 0, 0};
            for (int64_t c = tail + lane; c < p; c += 1 << fs) at[c] = narrow<G>(typename Wide<G>::type(0));
        }
        return;
    }
    const int lane = threadIdx.x & ((1 << shift) - 1);
    const int64_t item = (int64_t)blockIdx.x * (THREADS >> shift) + (threadIdx.x >> shift);
    const int64_t at_piece = item / slabs, c = ((item - at_piece * slabs) << shift) * V + (int64_t)lane * V;
    const int64_t e0 = at_piece * piece, e1 = min(e0 + piece, nnz);
    if (e0 >= nnz || c >= p) return;
    const uint32_t before = e0 > 0 ? key[e0 - 1] : NO_KEY, behind = e1 < nnz ? key[e1] : NO_KEY;
    A acc[V] = {};
    uint32_t cur = key[e0];
    bool open = cur == before;  // the run comes from the piece before
    auto finish = [&](bool goes_on) {
        if (cur < (uint32_t)n) {
            if (!open && !goes_on) {
                write_row<G, A, V>(de + (int64_t)cur * ldde + c, p - c, scale, accumulate, acc);
            } else {
                A* at = part + (at_piece * 2 + (open ? 0 : 1)) * p + c;
#pragma unroll
                for (int i = 0; i < V; ++i)
                    if (c + i < p) at[i] = acc[i];
            }
        }
#pragma unroll
        for (int i = 0; i < V; ++i) acc[i] = A(0);
    };
    constexpr int U = 4;
    for (int64_t e = e0; e < e1; e += U) {
        uint32_t k[U], r[U];
        A w[U], x[U][V];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const bool on = e + u < e1;
            k[u] = on ? key[e + u] : 0u;
            r[u] = on ? row[e + u] : NO_KEY;
            w[u] = on && weight ? weight[e + u] : A(1);
            if (!on || k[u] >= (uint32_t)n) r[u] = NO_KEY;
        }
#pragma unroll
        for (int u = 0; u < U; ++u) load_wide<T, V>(r[u] != NO_KEY ? dy + (int64_t)r[u] * lddy + c : dy, r[u] != NO_KEY ? p - c : 0, x[u]);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (e + u >= e1) break;
            if (k[u] != cur) {
                finish(false);
                cur = k[u];
                open = false;
            }
            if (r[u] != NO_KEY) {
#pragma unroll
                for (int i = 0; i < V; ++i) acc[i] += w[u] * x[u][i];
            }
        }
    }
    finish(cur == behind);
}

// first entry behind those of id k (the keys ascend)
__device__ __forceinline__ int64_t upper_bound(const uint32_t* __restrict__ key, int64_t lo, int64_t hi, uint32_t k) {
    while (lo < hi) {
        const int64_t mid = (lo + hi) >> 1;
        if (key[mid] <= k) lo = mid + 1; else hi = mid;
    }
    return lo;
}

// The runs that cross pieces: a warp looks at eight pieces for runs that begin there and go on, and adds up the partial sums of a run
// of up to JOIN_SHORT pieces by itself, JOIN_COLS columns per blockIdx.y.  The CTA takes the longer ones, every warp a
// contiguous share of the pieces.
constexpr int JOIN_COLS = 128;
constexpr int JOIN_SHORT = 16;
constexpr int JOIN_WARPS = THREADS / 32;
constexpr int JOIN_EACH = 8;
constexpr int JOIN_PIECES = JOIN_WARPS * JOIN_EACH;  // per CTA
template <typename T, typename G>
__global__ void __launch_bounds__(THREADS) join_kernel(int64_t nnz, int64_t n, int64_t p, const uint32_t* __restrict__ key,
                                                       const typename Wide<T>::type* __restrict__ part, typename Wide<T>::type scale,
                                                       G* __restrict__ de, int64_t ldde, bool accumulate, int piece) {
    using A = typename Wide<T>::type;
    constexpr int EACH = JOIN_COLS / 32;  // columns of a lane
    __shared__ A sums[JOIN_WARPS][JOIN_COLS];
    __shared__ int64_t long_first[JOIN_PIECES], long_count[JOIN_PIECES];
    __shared__ int long_runs;
    link(key, part);
    const int lane = lane_id(), warp = threadIdx.x >> 5;
    if (threadIdx.x == 0) long_runs = 0;
    __syncthreads();
    // pieces that a run begins in and leaves; how many pieces it has
    const int64_t f = (int64_t)blockIdx.x * JOIN_PIECES + warp * JOIN_EACH + lane;
    int64_t count = 0;
    if (lane < JOIN_EACH) {
        const int64_t e0 = f * piece, e1 = min(e0 + piece, nnz);
        if (e1 < nnz) {
            const uint32_t k = key[e1 - 1];
            if (k < (uint32_t)n && key[e1] == k && !(key[e0] == k && e0 > 0 && key[e0 - 1] == k)) count = (upper_bound(key, e1, nnz, k) - 1) / piece - f + 1;
        }
    }
    if (count > JOIN_SHORT) {
        const int at = atomicAdd(&long_runs, 1);  // (the order of the runs does not matter)
        long_first[at] = f;
        long_count[at] = count;
    }
    const int64_t c0 = (int64_t)blockIdx.y * JOIN_COLS + lane;
    auto add = [&](int64_t first, int64_t s0, int64_t s1, A(&acc)[EACH]) {
#pragma unroll 4
        for (int64_t s = s0; s < s1; ++s) {
#pragma unroll
            for (int i = 0; i < EACH; ++i)
                if (c0 + i * 32 < p) acc[i] += part[((first + s) * 2 + (s == 0 ? 1 : 0)) * p + c0 + i * 32];
        }
    };
    auto write = [&](int64_t first, A(&acc)[EACH]) {
        G* const at = de + (int64_t)key[first * piece + piece - 1] * ldde + c0;
#pragma unroll
        for (int i = 0; i < EACH; ++i) {
            A x[1] = {acc[i]};
            if (c0 + i * 32 < p) write_row<G, A, 1>(at + i * 32, 1, scale, accumulate, x);
        }
    };
    for (unsigned runs = __ballot_sync(FULL_MASK, count > 0 && count <= JOIN_SHORT); runs; runs &= runs - 1) {
        const int from = __ffs(runs) - 1;
        const int64_t first = __shfl_sync(FULL_MASK, f, from), pieces = __shfl_sync(FULL_MASK, count, from);
        A acc[EACH] = {};
        add(first, 0, pieces, acc);
        write(first, acc);
    }
    __syncthreads();
    for (int r = 0; r < long_runs; ++r) {
        const int64_t first = long_first[r], pieces = long_count[r], share = (pieces + JOIN_WARPS - 1) / JOIN_WARPS;
        A acc[EACH] = {};
        add(first, min(pieces, warp * share), min(pieces, (warp + 1) * share), acc);
#pragma unroll
        for (int i = 0; i < EACH; ++i) sums[warp][lane + i * 32] = acc[i];
        __syncthreads();
        if (warp == 0) {
            for (int w = 1; w < JOIN_WARPS; ++w) {
#pragma unroll
                for (int i = 0; i < EACH; ++i) acc[i] += sums[w][lane + i * 32];
            }
            write(first, acc);
        }
        __syncthreads();
    }
}

template <typename T, typename G, int V>
spsyrk_status_t add_typed(const GradWs& w, int which, int64_t n, int64_t p, int64_t nnz, bool weighted, double scale, const void* dy, int64_t lddy, void* de,
                          int64_t ldde, bool accumulate, cudaStream_t st) {
    using A = typename Wide<T>::type;
    const int piece = piece_of(nnz, p);
    const int64_t pieces = (nnz + piece - 1) / piece, vectors = (p + V - 1) / V;
    int shift = 0;
    while ((int64_t(1) << shift) < vectors && shift < 8) ++shift;
    const int64_t slabs = (vectors + (int64_t(1) << shift) - 1) >> shift, per_cta = THREADS >> shift;
    const int64_t piece_ctas = (pieces * slabs + per_cta - 1) / per_cta;
    // about 64 KB of dE a CTA
    const int64_t fill_rows = std::max<int64_t>(1, std::min<int64_t>(65536, 65536 / std::max<int64_t>(1, p * (int64_t)sizeof(G))));
    const int64_t fill_ctas = accumulate ? 0 : (n + fill_rows - 1) / fill_rows;
    if (piece_ctas + fill_ctas >= (int64_t(1) << 31)) return SPSYRK_ERR_OVERFLOW;
    const A* weight = weighted ? static_cast<const A*>(w.weight[which]) : nullptr;
    SPSYRK_CUDA_TRY(launch_linked(add_pieces_kernel<T, G, V>, (unsigned)(piece_ctas + fill_ctas), THREADS, 0, st, nnz, n, p, w.key[which], w.row[which], weight,
                                  (A)scale, static_cast<const T*>(dy), lddy, static_cast<G*>(de), ldde, accumulate, static_cast<A*>(w.part), piece, shift,
                                  slabs, piece_ctas, w.present, fill_rows));
    if (pieces > 1) {
        cudaLaunchConfig_t cfg{};
        cfg.gridDim = dim3((unsigned)((pieces + JOIN_PIECES - 1) / JOIN_PIECES), (unsigned)((p + JOIN_COLS - 1) / JOIN_COLS));
        cfg.blockDim = dim3(THREADS);
        cfg.stream = st;
        cudaLaunchAttribute attr{};
        attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
        attr.val.programmaticStreamSerializationAllowed = 1;
        cfg.attrs = &attr;
        cfg.numAttrs = 1;
        SPSYRK_CUDA_TRY(launch_kernel(cfg, join_kernel<T, G>, nnz, n, p, (const uint32_t*)w.key[which], static_cast<const A*>(w.part), (A)scale,
                                      static_cast<G*>(de), ldde, accumulate, piece));
    }
    return SPSYRK_OK;
}

// Orders the entries; *which receives the buffer that they are in.
template <typename A>
spsyrk_status_t order_entries(const GradWs& w, const Rows& a, int64_t n, const int32_t* ids, const void* weights, int* which, cudaStream_t st) {
    SPSYRK_CUDA_TRY(cudaMemsetAsync(w.zero, 0, w.zero_bytes, st));
    const A* wv = static_cast<const A*>(weights);
    if (a.nnz <= FEW) {
        const int64_t each = THREADS / 32 * RANK_EACH;
        rank_kernel<A><<<(unsigned)((a.nnz + each - 1) / each), THREADS, 0, st>>>(a, n, ids, wv, w.key[0], w.row[0], static_cast<A*>(weights ? w.weight[0] : nullptr),
                                                                              w.present);
        note_launches(1);
        SPSYRK_CUDA_TRY(cudaGetLastError());
        *which = 0;
        return SPSYRK_OK;
    }
    const int passes = radix_passes((uint64_t)n);
    read_ids_kernel<<<(unsigned)((a.nnz + READ_CHUNK - 1) / READ_CHUNK), THREADS, 0, st>>>(a, n, ids, w.key[0], w.row[0], w.present, passes, w.rs.bins);
    note_launches(1);
    SPSYRK_CUDA_TRY(cudaGetLastError());
    using PB = typename std::conditional<sizeof(A) == 8, uint64_t, uint32_t>::type;
    for (int q = 0; q < passes; ++q) {
        const int from = q & 1, to = from ^ 1;
        const PB* pb = weights ? reinterpret_cast<const PB*>(q == 0 ? weights : w.weight[from]) : nullptr;
        EmitOrdered<PB> emit{w.key[to], w.row[to], weights ? static_cast<PB*>(w.weight[to]) : nullptr};
        SPSYRK_CUDA_TRY((radix_pass<PB, false>(w.key[from], w.row[from], pb, nullptr, a.nnz, q, w.rs, emit, w.err, st)));
    }
    *which = passes & 1;
    return SPSYRK_OK;
}

}  // namespace

extern "C" spsyrk_status_t spsyrk_lookup_grad(int64_t m, int64_t n, int64_t p, int64_t nnz, spsyrk_dtype_t dtype, spsyrk_dtype_t g_dtype,
                                              const int64_t* d_rowptr, const int32_t* d_ids, const void* d_weights, double scale, const void* d_dy,
                                              int64_t lddy, void* d_de, int64_t ldde, int accumulate, void* d_workspace, size_t* workspace_bytes,
                                              void* cuda_stream) {
    if (!workspace_bytes || m < 0 || n < 0 || p < 0 || nnz < 0 || !is_real(dtype)) return SPSYRK_ERR_INVALID_ARG;
    if (g_dtype != dtype && !(g_dtype == SPSYRK_F32 && dtype != SPSYRK_F64)) return SPSYRK_ERR_INVALID_ARG;
    constexpr int64_t most = (int64_t(1) << 31) - 1;
    if (m >= most || n >= most || nnz >= most || p > (int64_t(1) << 22)) return SPSYRK_ERR_OVERFLOW;
    // (the size with room for weights: a query need not know whether there are any)
    const size_t need = carve(nullptr, nullptr, n, p, nnz, dtype == SPSYRK_F64, true);
    if (!d_workspace) {
        *workspace_bytes = need;
        return SPSYRK_OK;
    }
    if (*workspace_bytes < need) return SPSYRK_ERR_WORKSPACE;
    if (reinterpret_cast<uintptr_t>(d_workspace) % ALIGN) return SPSYRK_ERR_INVALID_ARG;
    if (lddy < p || ldde < p || (nnz > 0 && !d_ids)) return SPSYRK_ERR_INVALID_ARG;
    if (!d_rowptr && (m == 0 ? nnz != 0 : nnz % m != 0)) return SPSYRK_ERR_INVALID_ARG;
    if (n == 0 || p == 0) return SPSYRK_OK;
    if (!d_de || (nnz > 0 && (m == 0 || !d_dy))) return SPSYRK_ERR_INVALID_ARG;
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    const size_t size = element_size(dtype), g_size = element_size(g_dtype);
    if (nnz == 0) {
        if (!accumulate) SPSYRK_CUDA_TRY(cudaMemset2DAsync(d_de, (size_t)ldde * g_size, 0, (size_t)p * g_size, (size_t)n, st));
        return SPSYRK_OK;
    }
    const Rows a{d_rowptr, m, nnz, nnz / m};
    GradWs w;
    carve(&w, d_workspace, n, p, nnz, dtype == SPSYRK_F64, true);
    int which = 0;
    const spsyrk_status_t s = dtype == SPSYRK_F64 ? order_entries<double>(w, a, n, d_ids, d_weights, &which, st)
                                                  : order_entries<float>(w, a, n, d_ids, d_weights, &which, st);
    if (s != SPSYRK_OK) return s;
    const bool wide = aligned16(d_dy, lddy, size) && aligned16(d_de, ldde, g_size);
    const bool weighted = d_weights != nullptr;
#define ADD(T, G, V) add_typed<T, G, V>(w, which, n, p, nnz, weighted, scale, d_dy, lddy, d_de, ldde, accumulate != 0, st)
    switch (dtype) {
        case SPSYRK_F64: return wide ? ADD(double, double, 2) : ADD(double, double, 1);
        case SPSYRK_F32: return wide ? ADD(float, float, 4) : ADD(float, float, 1);
        case SPSYRK_BF16:
            if (g_dtype == SPSYRK_F32) return wide ? ADD(__nv_bfloat16, float, 8) : ADD(__nv_bfloat16, float, 1);
            return wide ? ADD(__nv_bfloat16, __nv_bfloat16, 8) : ADD(__nv_bfloat16, __nv_bfloat16, 1);
        default:
            if (g_dtype == SPSYRK_F32) return wide ? ADD(__half, float, 8) : ADD(__half, float, 1);
            return wide ? ADD(__half, __half, 8) : ADD(__half, __half, 1);
    }
#undef ADD
}
