// dE = scale * A^T dY for rows of ids A: the gradient of an embedding lookup with respect to its table, by sorted ids.
//
// The entries are ordered by id with a stable sort (entries of an id stay in their order), and the ordered list is cut into pieces of
// the same length.  A group of lanes adds up a piece, 16 bytes of dY a lane, run by run (a run = the entries of one id): a run that lies
// inside the piece is written to its row of dE at once, one that crosses the piece's ends leaves its partial sum in the workspace.  The
// partial sums of such runs are joined in their order, 64 pieces at a time, then 64 times 64, until one block holds them all.  No atomic
// adds: the same call gives the same bits, and an id that every tenth entry has costs no more than others (joined by one CTA
// its 5500 pieces of 64 columns took 270 us).  Rows of ids that do not occur are filled with zeros by CTAs that stand among those that
// add up pieces (or rank the ids, if they are few).
// Bound by memory: dY is read once (a row of several ids once per id, through L2), dE written once.
#include <algorithm>
#include <math_constants.h>

#include "element.cuh"
#include "radix.cuh"

using namespace spsyrk;

namespace {

constexpr size_t ALIGN = 256;
constexpr int THREADS = 256;
constexpr int SMS = 148;
// Entries that are ranked by comparing all with all instead of sorted by digits (3800 entries 29 us against 37, 7000 47 against 39 in all).
constexpr int64_t FEW = 6144;
constexpr int MIN_PIECE = 4, MAX_PIECE = 32;

// Entries of a piece: 32 if their groups still fill every SM with threads, fewer if not.  (Lanes of 8 elements, whatever the type: the
// workspace's size depends on it.)
int piece_of(int64_t nnz, int64_t p) {
    int c = MAX_PIECE;
    while (c > MIN_PIECE && nnz / c * ((p + 7) / 8) < (int64_t)SMS * 2048) c /= 2;
    return c;
}

constexpr int JOIN = 64;        // pieces (blocks of pieces) that are joined at a time
constexpr int JOIN_LEVELS = 6;  // 2^31 entries in pieces of MIN_PIECE: 2^29, 2^23, 2^17, 2^11, 2^5, 1

struct GradWs {
    uint32_t *key[2], *row[2];  // ids (n: padding) and rows of the entries, before and after a pass
    void* weight[2];
    uint8_t* present;  // a byte per id: it occurs
    // [pieces][2][p] partial sums: of a run that comes from the piece before, of one that begins here and goes on; then those of blocks of
    // JOIN pieces, of JOIN times JOIN, down to a single one
    void* part[JOIN_LEVELS];
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
    int64_t count = (ne + piece - 1) / piece;
    for (int level = 0; level < JOIN_LEVELS; ++level) {
        t.part[level] = count > 1 ? take((size_t)count * 2 * p * acc) : nullptr;
        count = (count + JOIN - 1) / JOIN;
    }
    // what has to be zero at the start, in one piece
    const size_t marks = nnz > FEW ? ((size_t)n + 7) / 8 * 8 : 0;
    const size_t words = nnz > FEW ? radix_state_words(radix_tiles(nnz), radix_wide(nnz), radix_passes((uint64_t)n)) : 0;
    t.zero_bytes = marks + (1 + RX_MAX_PASSES * RX_BINS + RX_MAX_PASSES + words) * 8;
    t.zero = take(t.zero_bytes);
    char* z = (char*)t.zero;
    t.present = (uint8_t*)z;
    t.err = (uint32_t*)(z + marks);
    t.rs.bins = (unsigned long long*)(z + marks) + 1;
    t.rs.tickets = (uint32_t*)(t.rs.bins + RX_MAX_PASSES * RX_BINS);
    t.rs.words = t.rs.bins + RX_MAX_PASSES * RX_BINS + RX_MAX_PASSES;
    if (w) *w = t;
    return (off + ALIGN - 1) / ALIGN * ALIGN;
}

// Zeros for the rows [v0, v1) of dE without entries.  A warp takes up to 32 rows, every lane looks for one of them whether it has entries.  In
// memory elements up to the first 16-byte boundary, 16 bytes a lane, the elements behind; row by row only where something lies
// between the rows.  (Row by row, narrow rows cost more instructions than bytes: 1.1e6 rows of 144 doubles 262 us.)
struct Fill {
    char* de;
    int64_t row_bytes, used_bytes;  // from row to row; of a row
    int size;                       // of an element
    int64_t rows;                   // a CTA's
    int64_t n;
    template <typename Present>
    __device__ __forceinline__ void rows_of(int64_t v0, int64_t v1, Present present) const {
        const int shift = min(5, 32 - __clz((int)min((used_bytes + 15) / 16, (int64_t)32) - 1));
        const int lanes = 1 << shift, lane = lane_id() & (lanes - 1), warps = blockDim.x >> 5;
        const int each = (int)min((int64_t)32, (v1 - v0 + warps - 1) / warps);
        for (int64_t first = v0 + (int64_t)(threadIdx.x >> 5) * each; first < v1; first += (int64_t)warps * each) {
            const int count = (int)min((int64_t)each, v1 - first);
            const unsigned taken = __ballot_sync(FULL_MASK, lane_id() < count && present(first + lane_id()));
            if (row_bytes == used_bytes) {  // rows without entries that follow one another are one piece of memory
                unsigned free = ~taken & (count == 32 ? FULL_MASK : (1u << count) - 1);
                while (free) {
                    const int begin = __ffs(free) - 1, rows = free >> begin == FULL_MASK ? 32 : __ffs(~(free >> begin)) - 1;
                    zero_bytes(de + (first + begin) * row_bytes, rows * row_bytes);
                    free &= free + (1u << begin);  // (adding at its lowest bit clears the run)
                }
                continue;
            }
            for (int r = lane_id() >> shift; r < count; r += 32 >> shift) {
                if (taken >> r & 1u) continue;
                char* const at = de + (first + r) * row_bytes;
                const int64_t head = min(used_bytes, (int64_t)((0 - reinterpret_cast<uintptr_t>(at)) % 16)), body = (used_bytes - head) / 16;
                const int64_t tail = head + body * 16;
                if (head > 0) zeros(at, head, lane, lanes);
                for (int64_t c = lane; c < body; c += lanes) reinterpret_cast<uint4*>(at + head)[c] = uint4{0, 0, 0, 0};
                if (tail < used_bytes) zeros(at + tail, used_bytes - tail, lane, lanes);
            }
        }
    }
    // by a whole warp; `at` and `bytes` are multiples of an element's size
    __device__ __forceinline__ void zero_bytes(char* at, int64_t bytes) const {
        const int64_t head = min(bytes, (int64_t)((0 - reinterpret_cast<uintptr_t>(at)) % 16));
        if (head > 0) zeros(at, head, lane_id(), 32);
        at += head;
        bytes -= head;
        int64_t units = bytes / 16;
        uint4* to = reinterpret_cast<uint4*>(at) + lane_id();
        for (; units >= 128; units -= 128, to += 128) {
#pragma unroll
            for (int i = 0; i < 4; ++i) to[i * 32] = uint4{0, 0, 0, 0};
        }
        for (int64_t c = lane_id(); c < units; c += 32, to += 32) *to = uint4{0, 0, 0, 0};
        const int64_t tail = bytes & ~int64_t(15);
        if (tail < bytes) zeros(at + tail, bytes - tail, lane_id(), 32);
    }
    __device__ __forceinline__ void zeros(char* at, int64_t bytes, int lane, int lanes) const {
        for (int64_t c = (int64_t)lane * size; c < bytes; c += (int64_t)lanes * size) {
            if (size == 2) *reinterpret_cast<uint16_t*>(at + c) = 0;
            else if (size == 4) *reinterpret_cast<uint32_t*>(at + c) = 0;
            else *reinterpret_cast<uint64_t*>(at + c) = 0;
        }
    }
};

// Key and row of every entry, a mark per id that occurs and the sizes of all digits.
constexpr int READ_ITEMS = 4;
constexpr int READ_CHUNK = THREADS * READ_ITEMS;  // a step of a CTA
constexpr int READ_LOG_MARKS = 11, READ_MARKS = 1 << READ_LOG_MARKS;
__global__ void __launch_bounds__(THREADS) read_ids_kernel(Rows a, int64_t n, const int32_t* __restrict__ ids, uint32_t* __restrict__ key,
                                                           uint32_t* __restrict__ row, uint8_t* __restrict__ present, int passes,
                                                           unsigned long long* __restrict__ bins) {
    __shared__ int64_t span[2];
    __shared__ uint32_t h[RX_MAX_PASSES][RX_BINS];
    __shared__ volatile uint64_t marks[READ_MARKS];  // (written by several threads at a time: one of their words, whole, is what volatile promises)
    for (int d = threadIdx.x; d < RX_MAX_PASSES * RX_BINS; d += THREADS) (&h[0][0])[d] = 0;
    for (int64_t base = (int64_t)blockIdx.x * READ_CHUNK; base < a.nnz; base += (int64_t)gridDim.x * READ_CHUNK) {
        __syncthreads();
        if (a.rowptr && threadIdx.x < 64) {
            const int64_t r = a.row_of_by_warp(threadIdx.x < 32 ? base : min(base + READ_CHUNK, a.nnz) - 1);
            if (lane_id() == 0) span[threadIdx.x >> 5] = r;
        }
        __syncthreads();
        uint32_t k[READ_ITEMS];
#pragma unroll
        for (int i = 0; i < READ_ITEMS; ++i) {
            const int64_t t = base + i * THREADS + threadIdx.x, id = t < a.nnz ? ids[t] : -1;
            k[i] = id >= 0 && id < n && a.covered(t) ? (uint32_t)id : (uint32_t)n;
        }
        // An id is marked by one of the CTA's entries that have it: an id's slot holds one of those whose ids share it.  (Atomic operations
        // on a bit per id, a tenth of 2 million on the same one, took 55 us more, and 25 with this look.)
        auto mark_of = [&](uint32_t id) { return (int)((id * 2654435761u) >> (32 - READ_LOG_MARKS)); };
#pragma unroll
        for (int i = 0; i < READ_ITEMS; ++i) {
            marks[mark_of(k[i])] = (uint64_t)k[i] << 32 | (uint32_t)(i * THREADS + threadIdx.x);
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < READ_ITEMS; ++i) {
            const int64_t t = base + i * THREADS + threadIdx.x;
            if (t >= a.nnz) continue;
            key[t] = k[i];
            row[t] = (uint32_t)(a.rowptr ? a.row_of(t, span[0], span[1]) : t / a.k);
            const uint64_t mark = marks[mark_of(k[i])];
            const bool other = (uint32_t)(mark >> 32) == k[i] && (uint32_t)mark != (uint32_t)(i * THREADS + threadIdx.x);
            if (k[i] < (uint32_t)n && !other) present[k[i]] = 1;
            for (int q = 0; q < passes; ++q) atomicAdd(&h[q][(k[i] >> (q * RX_BITS)) & (RX_BINS - 1)], 1u);
        }
    }
    __syncthreads();
    for (int d = threadIdx.x; d < passes * RX_BINS; d += THREADS)
        if ((&h[0][0])[d]) atomicAdd(&bins[d], (unsigned long long)(&h[0][0])[d]);
}

// Up to FEW entries: an entry's place in the order is the number of entries with a smaller id, or with the same one before it.  All
// keys are fetched to shared memory, and a warp counts for four entries at a time, 128 keys a step.  CTAs behind those of the entries fill rows: they
// look the ids through for those of their rows.
constexpr int RANK_EACH = 4;
constexpr int RANK_HERE = THREADS / 32 * RANK_EACH;  // entries of a CTA
constexpr int FILL_MOST = FEW * 32;                  // rows of a CTA that fills: a bit each in the place of the keys
template <typename A>
__global__ void __launch_bounds__(THREADS) rank_kernel(Rows a, int64_t n, const int32_t* __restrict__ ids, const A* __restrict__ weights,
                                                       uint32_t* __restrict__ key, uint32_t* __restrict__ row, A* __restrict__ weight, int rank_ctas,
                                                       Fill fill) {
    __shared__ __align__(16) uint32_t keys[FEW];
    __shared__ int64_t span[2];
    const int nnz = (int)a.nnz, lane = lane_id();
    const int64_t from = a.rowptr ? a.rowptr[0] : 0, to = a.rowptr ? a.rowptr[a.m] : a.nnz;
    auto key_of = [&](int t) {
        const int64_t id = ids[t];
        return id >= 0 && id < n && t >= from && t < to ? (uint32_t)id : (uint32_t)n;
    };
    if ((int)blockIdx.x >= rank_ctas) {
        const int64_t v0 = ((int64_t)blockIdx.x - rank_ctas) * fill.rows, v1 = min(v0 + fill.rows, n);
        for (int i = threadIdx.x; i < (int)((v1 - v0 + 31) / 32); i += THREADS) keys[i] = 0;
        __syncthreads();
#pragma unroll 8
        for (int t = threadIdx.x; t < nnz; t += THREADS) {
            const int64_t k = key_of(t);
            if (k >= v0 && k < v1) atomicOr(&keys[(k - v0) >> 5], 1u << ((k - v0) & 31));
        }
        __syncthreads();
        fill.rows_of(v0, v1, [&](int64_t v) { return (keys[(v - v0) >> 5] >> ((v - v0) & 31) & 1u) != 0; });
        return;
    }
    const int up = (nnz + 127) / 128 * 128;
#pragma unroll 8
    for (int t = threadIdx.x; t < up; t += THREADS) keys[t] = t < nnz ? key_of(t) : NO_KEY;  // (behind all others)
    const int t0 = (int)(blockIdx.x * (THREADS / 32) + (threadIdx.x >> 5)) * RANK_EACH;
    if (a.rowptr && threadIdx.x < 64) {
        const int64_t here = (int64_t)blockIdx.x * RANK_HERE, r = a.row_of_by_warp(threadIdx.x < 32 ? here : min(here + RANK_HERE, a.nnz) - 1);
        if (lane == 0) span[threadIdx.x >> 5] = r;
    }
    __syncthreads();
    if (t0 >= nnz) return;
    const int64_t my_row = lane < RANK_EACH && t0 + lane < nnz ? a.rowptr ? a.row_of(t0 + lane, span[0], span[1]) : (t0 + lane) / a.k : 0;
    uint32_t mine[RANK_EACH];
    int before[RANK_EACH] = {};
#pragma unroll
    for (int u = 0; u < RANK_EACH; ++u) mine[u] = keys[t0 + u];
    for (int t = lane * 4; t < up; t += 128) {
        const uint4 k = *reinterpret_cast<const uint4*>(keys + t);
#pragma unroll
        for (int u = 0; u < RANK_EACH; ++u) {
            // an entry before counts if its key is not larger, one behind if it is smaller; the entry itself does not
            const int at = t0 + u - t;
            before[u] += (at > 0 ? k.x <= mine[u] : k.x < mine[u]) + (at > 1 ? k.y <= mine[u] : k.y < mine[u]) + (at > 2 ? k.z <= mine[u] : k.z < mine[u]) +
                         (at > 3 ? k.w <= mine[u] : k.w < mine[u]);
        }
    }
#pragma unroll
    for (int u = 0; u < RANK_EACH; ++u) {
        const int at = __reduce_add_sync(FULL_MASK, before[u]);
        if (lane != u || t0 + u >= nnz) continue;
        key[at] = mine[u];
        row[at] = (uint32_t)my_row;
        if (weight) weight[at] = weights[t0 + u];
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

// A group of lanes per piece and slab of columns.  (After a wait among the radix passes that has run out, places of the order hold whatever the
// workspace did: keys are tested anyway, and a row is cut to the last one.)
// (Registers decide: eight sums a lane take four rows at a time and three CTAs per SM, fewer sums two and five; the others cost 5 to 15 %.)
template <typename T, typename G, int V>
__global__ void __launch_bounds__(THREADS, V == 8 ? 3 : 5) add_pieces_kernel(int64_t nnz, uint32_t last_row, int64_t n, int64_t p, const uint32_t* __restrict__ key,
                                                             const uint32_t* __restrict__ row, const typename Wide<T>::type* __restrict__ weight,
                                                             typename Wide<T>::type scale, const T* __restrict__ dy, int64_t lddy, G* __restrict__ de,
                                                             int64_t ldde, bool accumulate, typename Wide<T>::type* __restrict__ part, int piece,
                                                             int shift, int64_t slabs, const uint8_t* __restrict__ present, Fill fill, int fill_ctas) {
    using A = typename Wide<T>::type;
    constexpr int U = V == 8 ? 4 : 2;
    link(key, row, weight, present);
    // CTAs that fill rows stand evenly among the others
    const int64_t filled = (int64_t)blockIdx.x * fill_ctas / gridDim.x;
    if (((int64_t)blockIdx.x + 1) * fill_ctas / gridDim.x != filled) {
        const int64_t v0 = filled * fill.rows;
        fill.rows_of(v0, min(v0 + fill.rows, n), [&](int64_t v) { return present[v] != 0; });
        return;
    }
    const int lane = threadIdx.x & ((1 << shift) - 1);
    const int64_t item = (blockIdx.x - filled) * (THREADS >> shift) + (threadIdx.x >> shift);
    const int64_t at_piece = item / slabs, c = ((item - at_piece * slabs) << shift) * V + (int64_t)lane * V;
    const int64_t e0 = at_piece * piece, e1 = min(e0 + piece, nnz);
    if (e0 >= nnz) return;  // (the whole group)
    // the lanes of a group that share a warp fetch an entry each and hand them round
    const int share = 1 << min(shift, 5), in_share = threadIdx.x & (share - 1);
    const unsigned mask = share == 32 ? FULL_MASK : ((1u << share) - 1) << (lane_id() & ~(share - 1));
    const uint32_t before = e0 > 0 ? key[e0 - 1] : NO_KEY, behind = e1 < nnz ? key[e1] : NO_KEY;
    A acc[V] = {};
    uint32_t cur = key[e0];
    bool open = cur == before;  // the run comes from the piece before
    auto finish = [&](bool goes_on) {
        if (cur < (uint32_t)n && c < p) {
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
    for (int64_t e = e0; e < e1; e += share) {
        const bool on = e + in_share < e1;
        const uint32_t my_key = on ? key[e + in_share] : NO_KEY, my_row = on ? min(row[e + in_share], last_row) : 0u;
        const A my_w = on && weight ? weight[e + in_share] : A(1);
        const int count = (int)min((int64_t)share, e1 - e);
        for (int q = 0; q < count; q += U) {
            uint32_t k[U];
            Vec<T, V> x[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const uint32_t got = __shfl_sync(mask, my_key, q + u, share), r = __shfl_sync(mask, my_row, q + u, share);
                k[u] = q + u < count ? got : NO_KEY;
                if (k[u] < (uint32_t)n) x[u] = load_raw<T, V>(dy + (int64_t)r * lddy + c, p - c);
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const A w = weight ? __shfl_sync(mask, my_w, q + u, share) : A(1);
                if (q + u >= count) continue;
                if (k[u] != cur) {
                    finish(false);
                    cur = k[u];
                    open = false;
                }
                if (k[u] < (uint32_t)n) {
#pragma unroll
                    for (int i = 0; i < V; ++i) acc[i] += w * widen(x[u].x[i]);
                }
            }
        }
    }
    finish(cur == behind);
}

// Joins the partial sums of JOIN pieces (of `piece` entries; blocks of pieces on the later levels): a CTA per block of pieces and
// JOIN_COLS columns.  Every warp joins JOIN_EACH consecutive pieces, and the first warp then what the warps have left, in the same
// way.  What ends inside is written to dE; what crosses the ends is a partial sum of the warp's pieces, of the block.  (A warp that walks all 64
// pieces by itself takes 25 us, most of it waiting for its own instructions.)
constexpr int JOIN_COLS = 64;
constexpr int JOIN_EACH = 8;
static_assert(JOIN == JOIN_EACH * (THREADS / 32), "a warp per JOIN_EACH pieces");

// What joining has to know of JOIN_EACH consecutive pieces from `first` on: a bit each whether its first run comes from before, whether its last
// one goes on, whether it is all one run; and, in lane q, the id of piece q's first entry.
struct Seams {
    unsigned open, on, one;
    uint32_t id;
    __device__ __forceinline__ Seams(const uint32_t* __restrict__ key, int64_t first, int64_t piece, int64_t nnz, int64_t n) {
        const int64_t e0 = (first + lane_id()) * piece, e1 = min(e0 + piece, nnz);
        bool is_open = false, is_on = false, is_one = false;
        id = NO_KEY;
        if (lane_id() < JOIN_EACH && e0 < nnz) {
            id = key[e0];
            const uint32_t last = key[e1 - 1], before = e0 > 0 ? key[e0 - 1] : NO_KEY, behind = e1 < nnz ? key[e1] : NO_KEY;
            is_open = id < (uint32_t)n && before == id;
            is_on = last < (uint32_t)n && behind == last;
            is_one = id == last;
        }
        open = __ballot_sync(FULL_MASK, is_open);
        on = __ballot_sync(FULL_MASK, is_on);
        one = __ballot_sync(FULL_MASK, is_one);
    }
    // get(q, slot, x): the partial sums of piece q (slot 0: of the run from before, 1: of the one that begins there and goes on);
    // write(id, x): a finished sum; leave(slot, x): a partial sum of all these pieces together
    template <typename A, int N, typename Get, typename Write, typename Leave>
    __device__ __forceinline__ void walk(Get get, Write write, Leave leave) const {
        const unsigned begins = on & ~(open & one);  // a run begins in the piece and goes on
        if ((open | begins) == 0) return;
        A x[JOIN_EACH][2][N];
#pragma unroll
        for (int q = 0; q < JOIN_EACH; ++q) {
            if (open >> q & 1) get(q, 0, x[q][0]);
            if (begins >> q & 1) get(q, 1, x[q][1]);
        }
        A acc[N] = {};
        bool from_before = open & 1;
#pragma unroll
        for (int q = 0; q < JOIN_EACH; ++q) {
            if (open >> q & 1) {
#pragma unroll
                for (int i = 0; i < N; ++i) acc[i] += x[q][0][i];
                if (!(one & on & 1u << q)) {  // ends here
                    if (from_before) leave(0, acc);
                    else write(__shfl_sync(FULL_MASK, id, q), acc);
                    from_before = false;
                }
            }
            if (begins >> q & 1) {
#pragma unroll
                for (int i = 0; i < N; ++i) acc[i] = x[q][1][i];
            }
        }
        if (on >> (JOIN_EACH - 1) & 1) leave(from_before ? 0 : 1, acc);
    }
};

template <typename A, typename G>
__global__ void __launch_bounds__(THREADS) join_kernel(int64_t nnz, int64_t n, int64_t p, const uint32_t* __restrict__ key, const A* __restrict__ part,
                                                       A* __restrict__ part_out, A scale, G* __restrict__ de, int64_t ldde, bool accumulate, int64_t piece,
                                                       const uint32_t* __restrict__ err) {
    constexpr int N = JOIN_COLS / 32;
    __shared__ A left[THREADS / 32][2][JOIN_COLS];
    link(key, part);
    const int lane = lane_id(), warp = threadIdx.x >> 5;
    const int64_t c = (int64_t)blockIdx.y * JOIN_COLS + lane, first = (int64_t)blockIdx.x * JOIN + warp * JOIN_EACH;
    auto write = [&](uint32_t id, A(&x)[N]) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            A one[1] = {x[i]};
            if (c + i * 32 < p) write_row<G, A, 1>(de + (int64_t)id * ldde + c + i * 32, 1, scale, accumulate, one);
        }
    };
    const Seams mine(key, first, piece, nnz, n);
    mine.walk<A, N>(
        [&](int q, int slot, A(&x)[N]) {
#pragma unroll
            for (int i = 0; i < N; ++i) x[i] = c + i * 32 < p ? part[((first + q) * 2 + slot) * p + c + i * 32] : A(0);
        },
        write,
        [&](int slot, A(&x)[N]) {
#pragma unroll
            for (int i = 0; i < N; ++i) left[warp][slot][i * 32 + lane] = x[i];
        });
    __syncthreads();
    if (warp > 0) return;
    const Seams all(key, (int64_t)blockIdx.x * (THREADS / 32), piece * JOIN_EACH, nnz, n);
    all.walk<A, N>(
        [&](int q, int slot, A(&x)[N]) {
#pragma unroll
            for (int i = 0; i < N; ++i) x[i] = left[q][slot][i * 32 + lane];
        },
        write,
        [&](int slot, A(&x)[N]) {
#pragma unroll
            for (int i = 0; i < N; ++i)
                if (c + i * 32 < p) part_out[((int64_t)blockIdx.x * 2 + slot) * p + c + i * 32] = x[i];
        });
    if (err && *err) {  // (the last block of all) a wait among the radix passes has run out, which should not happen: what the entries name becomes NaN
        for (int64_t e = 0; e < nnz; ++e)
            for (int i = 0; i < N; ++i)
                if (key[e] < (uint32_t)n && c + i * 32 < p) de[(int64_t)key[e] * ldde + c + i * 32] = narrow<G>(A(CUDART_NAN_F));
    }
}

template <typename T, typename G, int V>
spsyrk_status_t add_typed(const GradWs& w, int which, const uint32_t* err, const Fill& fill, int64_t m, int64_t n, int64_t p, int64_t nnz, bool weighted, double scale, const void* dy, int64_t lddy, void* de,
                          int64_t ldde, bool accumulate, cudaStream_t st) {
    using A = typename Wide<T>::type;
    int64_t piece = piece_of(nnz, p);
    int64_t pieces = (nnz + piece - 1) / piece;
    const int64_t vectors = (p + V - 1) / V;
    int shift = 0;
    while ((int64_t(1) << shift) < vectors && shift < 8) ++shift;
    const int64_t slabs = (vectors + (int64_t(1) << shift) - 1) >> shift, per_cta = THREADS >> shift;
    const int64_t ctas = (pieces * slabs + per_cta - 1) / per_cta;
    const int64_t fill_ctas = fill.rows ? (n + fill.rows - 1) / fill.rows : 0;
    if (ctas + fill_ctas >= (int64_t(1) << 31)) return SPSYRK_ERR_OVERFLOW;
    const uint32_t* const key = w.key[which];
    const A* weight = weighted ? static_cast<const A*>(w.weight[which]) : nullptr;
    SPSYRK_CUDA_TRY(launch_linked(add_pieces_kernel<T, G, V>, (unsigned)(ctas + fill_ctas), THREADS, 0, st, nnz, (uint32_t)(m - 1), n, p, key, w.row[which], weight, (A)scale,
                                  static_cast<const T*>(dy), lddy, static_cast<G*>(de), ldde, accumulate, static_cast<A*>(w.part[0]), (int)piece, shift, slabs, w.present, fill,
                                  (int)fill_ctas));
    for (int level = 0; pieces > 1; ++level) {
        const int64_t blocks = (pieces + JOIN - 1) / JOIN;
        cudaLaunchConfig_t cfg{};
        cfg.gridDim = dim3((unsigned)blocks, (unsigned)((p + JOIN_COLS - 1) / JOIN_COLS));
        cfg.blockDim = dim3(THREADS);
        cfg.stream = st;
        cudaLaunchAttribute attr{};
        attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
        attr.val.programmaticStreamSerializationAllowed = 1;
        cfg.attrs = &attr;
        cfg.numAttrs = 1;
        A* const out = level + 1 < JOIN_LEVELS ? static_cast<A*>(w.part[level + 1]) : nullptr;  // (null where one block holds all: nothing leaves it)
        SPSYRK_CUDA_TRY(launch_kernel(cfg, join_kernel<A, G>, nnz, n, p, key, static_cast<const A*>(w.part[level]), out, (A)scale, static_cast<G*>(de), ldde,
                                      accumulate, piece, blocks == 1 ? err : nullptr));
        piece *= JOIN;
        pieces = blocks;
    }
    return SPSYRK_OK;
}

// Orders the entries; *which receives the buffer that they are in.  Few entries: also fills the rows without any, and sets fill->rows to 0.
template <typename A>
spsyrk_status_t order_entries(const GradWs& w, const Rows& a, int64_t n, const int32_t* ids, const void* weights, Fill* fill, int* which, cudaStream_t st) {
    const A* wv = static_cast<const A*>(weights);
    if (a.nnz <= FEW) {
        const int64_t ctas = (a.nnz + RANK_HERE - 1) / RANK_HERE;
        // (a CTA that fills looks all ids through: few, then)
        if (fill->rows) fill->rows = std::min<int64_t>(FILL_MOST, std::max<int64_t>(fill->rows, (n + SMS * 4 - 1) / (SMS * 4)));
        const int64_t fill_ctas = fill->rows ? (n + fill->rows - 1) / fill->rows : 0;
        rank_kernel<A><<<(unsigned)(ctas + fill_ctas), THREADS, 0, st>>>(a, n, ids, wv, w.key[0], w.row[0], static_cast<A*>(weights ? w.weight[0] : nullptr), (int)ctas,
                                                                         *fill);
        note_launches(1);
        SPSYRK_CUDA_TRY(cudaGetLastError());
        fill->rows = 0;
        *which = 0;
        return SPSYRK_OK;
    }
    SPSYRK_CUDA_TRY(cudaMemsetAsync(w.zero, 0, w.zero_bytes, st));
    const int passes = radix_passes((uint64_t)n);
    read_ids_kernel<<<(unsigned)std::min<int64_t>((a.nnz + READ_CHUNK - 1) / READ_CHUNK, SMS * 4), THREADS, 0, st>>>(a, n, ids, w.key[0], w.row[0], w.present, passes,
                                                                                                               w.rs.bins);
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
    if (m >= most || n >= most || nnz >= most || p > (int64_t(1) << 21)) return SPSYRK_ERR_OVERFLOW;
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
    if (!d_de || (nnz > 0 && m > 0 && !d_dy)) return SPSYRK_ERR_INVALID_ARG;
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    const size_t size = element_size(dtype), g_size = element_size(g_dtype);
    if (nnz == 0 || m == 0) {  // (entries of no row)
        if (!accumulate) SPSYRK_CUDA_TRY(cudaMemset2DAsync(d_de, (size_t)ldde * g_size, 0, (size_t)p * g_size, (size_t)n, st));
        return SPSYRK_OK;
    }
    const Rows a{d_rowptr, m, nnz, nnz / m};
    GradWs w;
    carve(&w, d_workspace, n, p, nnz, dtype == SPSYRK_F64, true);
    // 256 KB of dE a CTA, at most 512 rows
    const int64_t used = p * (int64_t)g_size;
    Fill fill{static_cast<char*>(d_de), ldde * (int64_t)g_size, used, (int)g_size, accumulate ? 0 : std::max<int64_t>(1, std::min<int64_t>(512, (1 << 18) / used)), n};
    // Few entries for a large matrix: all of it is cleared first, at the rate of a copy and a half (the few rows with entries are written twice:
    // 1616 entries of 1.1e6 rows of 144 doubles 260 us otherwise, 215 so).
    if (fill.rows && nnz * 8 <= n && n * used >= int64_t(1) << 28) {
        if (fill.row_bytes == used) SPSYRK_CUDA_TRY(cudaMemsetAsync(d_de, 0, (size_t)(n * used), st));
        else SPSYRK_CUDA_TRY(cudaMemset2DAsync(d_de, (size_t)fill.row_bytes, 0, (size_t)used, (size_t)n, st));
        fill.rows = 0;
    }
    int which = 0;
    const spsyrk_status_t s = dtype == SPSYRK_F64 ? order_entries<double>(w, a, n, d_ids, d_weights, &fill, &which, st)
                                                  : order_entries<float>(w, a, n, d_ids, d_weights, &fill, &which, st);
    if (s != SPSYRK_OK) return s;
    // (8 bfloat16 and 8 floats of a row are 16-byte aligned alike where both are)
    const int of_dy = together(d_dy, lddy, size), of_de = together(d_de, ldde, g_size);
    const bool wide = of_dy == (int)(16 / size) && of_de == (int)(16 / g_size), two = of_dy >= 2 && of_de >= 2;
    const bool weighted = d_weights != nullptr;
#define ADD(T, G, V) add_typed<T, G, V>(w, which, nnz > FEW ? w.err : nullptr, fill, m, n, p, nnz, weighted, scale, d_dy, lddy, d_de, ldde, accumulate != 0, st)
    switch (dtype) {
        case SPSYRK_F64: return wide ? ADD(double, double, 2) : ADD(double, double, 1);
        case SPSYRK_F32: return wide ? ADD(float, float, 4) : two ? ADD(float, float, 2) : ADD(float, float, 1);
        case SPSYRK_BF16:
            if (g_dtype == SPSYRK_F32) return wide ? ADD(__nv_bfloat16, float, 8) : two ? ADD(__nv_bfloat16, float, 2) : ADD(__nv_bfloat16, float, 1);
            return wide ? ADD(__nv_bfloat16, __nv_bfloat16, 8) : two ? ADD(__nv_bfloat16, __nv_bfloat16, 2) : ADD(__nv_bfloat16, __nv_bfloat16, 1);
        default:
            if (g_dtype == SPSYRK_F32) return wide ? ADD(__half, float, 8) : two ? ADD(__half, float, 2) : ADD(__half, float, 1);
            return wide ? ADD(__half, __half, 8) : two ? ADD(__half, __half, 2) : ADD(__half, __half, 1);
    }
#undef ADD
}
