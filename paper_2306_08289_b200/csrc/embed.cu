// Embedding lookup y_t = s E[id_t] and its gradient dE_v (+)= s sum_{t: id_t = v} dy_t.
#include <algorithm>

#include "lm_ops.h"

namespace a2 {

namespace {

constexpr int kThreads = 128;

// Threads that share a row's columns: enough for one vector each, at most a CTA, a power of two.
int group_threads(int64_t width, int vec) {
    int g = 8;
    while (g < kThreads && (int64_t)g * vec < width) g *= 2;
    return g;
}

bool aligned16(const void* p, int64_t pitch, int64_t elem) {
    return reinterpret_cast<uintptr_t>(p) % 16 == 0 && (pitch * elem) % 16 == 0;
}

// ---------------------------------------------------------------------------------------------
// Lookup. Bound by memory: a token's row is read once and written once. A group of threads owns kRows
// tokens, so that every thread has that many loads of 16 bytes in flight. 65,536 ids of 50,003 x 1,024 fp32: 56 us, in which 87 MB are read
// from DRAM and 209 MB written to it (5.3 TB/s): frequent rows are read from L2, and 60 MB of the writes are still there at the end.
// ---------------------------------------------------------------------------------------------
constexpr int kRows = 4;

template <class T, int VEC>
__global__ void __launch_bounds__(kThreads) k_embed(const T* table, int64_t vocab, int64_t width, int64_t table_pitch,
                                                    const int32_t* ids, int64_t n_ids, float scale,
                                                    T* __restrict__ out, int64_t out_pitch, int group) {
    ptx::chained();
    const int lane = threadIdx.x % group;
    const int64_t first = ((int64_t)blockIdx.x * (kThreads / group) + threadIdx.x / group) * kRows;
    int64_t id[kRows];
#pragma unroll
    for (int r = 0; r < kRows; ++r) {
        const int64_t v = first + r < n_ids ? ids[first + r] : -1;
        id[r] = v < vocab ? v : -1;
    }
    for (int64_t c = (int64_t)lane * VEC; c < width; c += (int64_t)group * VEC) {
        Pack<T, VEC> row[kRows];
#pragma unroll
        for (int r = 0; r < kRows; ++r)
            if (id[r] >= 0) row[r] = *reinterpret_cast<const Pack<T, VEC>*>(table + id[r] * table_pitch + c);
#pragma unroll
        for (int r = 0; r < kRows; ++r) {
            if (first + r >= n_ids) break;
            Pack<T, VEC> o;
#pragma unroll
            for (int k = 0; k < VEC; ++k) o.v[k] = narrow<T>(id[r] >= 0 ? widen(row[r].v[k]) * scale : 0.0f);
            *reinterpret_cast<Pack<T, VEC>*>(out + (first + r) * out_pitch + c) = o;
        }
    }
}

template <class T>
cudaError_t embed_typed(const EmbedArgs& a, cudaStream_t s) {
    constexpr int kVec = 16 / sizeof(T);
    const bool wide = a.width % kVec == 0 && aligned16(a.table, a.table_pitch, sizeof(T)) && aligned16(a.out, a.out_pitch, sizeof(T));
    const int group = group_threads(a.width, wide ? kVec : 1);
    const int64_t grid = ceil_div(a.n_ids, (int64_t)(kThreads / group) * kRows);
    auto* table = static_cast<const T*>(a.table);
    auto* out = static_cast<T*>(a.out);
    return launch_chained(wide ? k_embed<T, kVec> : k_embed<T, 1>, dim3((unsigned)grid), kThreads, 0, s, table, a.vocab, a.width, a.table_pitch, a.ids,
                          a.n_ids, a.scale, out, a.out_pitch, group);
}

// ---------------------------------------------------------------------------------------------
// Stable sort of the positions 0 .. n-1 by their id (an id outside the table sorts last, as `vocab`), least
// significant digit first, kDigitBits a pass. Stable and without floating atomics, so the gradient's sums have
// one fixed order: positions ascending.
// ---------------------------------------------------------------------------------------------
constexpr int kDigitBits = 9;
constexpr int kDigits = 1 << kDigitBits;
constexpr int kSortThreads = kDigits;  // thread d of a sorting CTA owns digit d
constexpr int kSortWarps = kSortThreads / 32;
constexpr int kTileItems = 4;                     // items a thread holds
constexpr int kTile = kSortThreads * kTileItems;  // 2048 positions a CTA

struct Pair {
    uint32_t key;
    uint32_t pos;
};

__device__ __forceinline__ uint32_t sort_key(int32_t id, int64_t vocab) {
    return id >= 0 && id < vocab ? (uint32_t)id : (uint32_t)vocab;
}
__device__ __forceinline__ int digit_of(uint32_t key, int pass) { return (key >> (pass * kDigitBits)) & (kDigits - 1); }

// Rank of every item among the tile's items of the same digit, in tile order (warp w holds items
// w * 32 * ITEMS .. , round by round), and the tile's count of digit threadIdx.x. count: [kSortWarps][kDigits].
template <int ITEMS>
__device__ __forceinline__ int tile_ranks(const Pair (&item)[ITEMS], const bool (&live)[ITEMS], int pass, int* count, int (&rank)[ITEMS]) {
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    for (int w = 0; w < kSortWarps; ++w) count[w * kDigits + threadIdx.x] = 0;
    __syncthreads();
    int* mine = count + warp * kDigits;
#pragma unroll
    for (int k = 0; k < ITEMS; ++k) {
        const int d = live[k] ? digit_of(item[k].key, pass) : kDigits + lane;  // an absent item matches none
        const unsigned same = __match_any_sync(0xffffffffu, d);
        int before = 0;
        if (live[k]) before = mine[d];
        __syncwarp();
        rank[k] = before + __popc(same & ((1u << lane) - 1));
        if (live[k] && lane == 31 - __clz(same)) mine[d] = before + __popc(same);
        __syncwarp();
    }
    __syncthreads();
    int total = 0;
#pragma unroll
    for (int w = 0; w < kSortWarps; ++w) {
        const int c = count[w * kDigits + threadIdx.x];
        count[w * kDigits + threadIdx.x] = total;
        total += c;
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < ITEMS; ++k)
        if (live[k]) rank[k] += mine[digit_of(item[k].key, pass)];
    return total;
}

// Exclusive sum over the CTA's kSortThreads threads.
__device__ __forceinline__ int block_exclusive(int v, int* warp_sums) {
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    int inc = v;
#pragma unroll
    for (int o = 1; o < 32; o *= 2) {
        const int up = __shfl_up_sync(0xffffffffu, inc, o);
        if (lane >= o) inc += up;
    }
    if (lane == 31) warp_sums[warp] = inc;
    __syncthreads();
    int base = 0;
    for (int w = 0; w < warp; ++w) base += warp_sums[w];
    __syncthreads();
    return base + inc - v;
}

// Rows [first, last) of a table become zeros: the sort leaves most of the GPU idle, so each of its launches clears kZeroBytes of the
// table in further CTAs, with or without positions (the sums overwrite those); the rest waits for k_segments, which knows which rows
// have none.
struct ZeroFill {
    char* table;
    int64_t first, last, row_bytes, pitch_bytes;
    bool wide;  // 16-byte stores
};
__device__ __forceinline__ void zero_rows(const ZeroFill& z, int64_t cta, int64_t ctas) {
    const int64_t warp = cta * kSortWarps + threadIdx.x / 32, warps = ctas * kSortWarps;
    for (int64_t r = z.first + warp; r < z.last; r += warps) {
        char* row = z.table + r * z.pitch_bytes;
        if (z.wide)
            for (int64_t b = threadIdx.x % 32 * 16; b < z.row_bytes; b += 512) *reinterpret_cast<uint4*>(row + b) = make_uint4(0, 0, 0, 0);
        else
            for (int64_t b = threadIdx.x % 32 * 2; b < z.row_bytes; b += 64) *reinterpret_cast<uint16_t*>(row + b) = 0;
    }
}

// Counts of the first digit, per tile of kTile positions.
__global__ void __launch_bounds__(kSortThreads) k_sort_count(const int32_t* ids, int64_t n, int64_t vocab, int passes, int n_tiles, int* __restrict__ counts,
                                                             const ZeroFill zero) {
    ptx::chained();
    if ((int)blockIdx.x >= n_tiles) return zero_rows(zero, blockIdx.x - n_tiles, gridDim.x - n_tiles);
    __shared__ int c[kDigits];
    c[threadIdx.x] = 0;
    __syncthreads();
    const int64_t first = (int64_t)blockIdx.x * kTile;
    for (int64_t i = first + threadIdx.x; i < min(first + kTile, n); i += kSortThreads) atomicAdd(&c[digit_of(sort_key(ids[i], vocab), 0)], 1);
    __syncthreads();
    for (int p = 0; p < passes; ++p)  // the later passes' counts are added up by the pass before
        counts[((int64_t)p * n_tiles + blockIdx.x) * kDigits + threadIdx.x] = p == 0 ? c[threadIdx.x] : 0;
}

// One pass: every tile adds up where its items go from the counts of all tiles, moves them, and counts the next
// digit of the tiles they land in (integer sums: the order of the atomics does not show).
__global__ void __launch_bounds__(kSortThreads) k_sort_pass(const int32_t* ids, const Pair* in, int64_t n, int64_t vocab,
                                                            int pass, bool last, const int* counts, int n_tiles,
                                                            Pair* __restrict__ out, int* __restrict__ next_counts, const ZeroFill zero) {
    ptx::chained();
    if ((int)blockIdx.x >= n_tiles) return zero_rows(zero, blockIdx.x - n_tiles, gridDim.x - n_tiles);
    __shared__ int count[kSortWarps * kDigits];
    __shared__ int base[kDigits];
    __shared__ int warp_sums[kSortWarps];
    const int64_t first = (int64_t)blockIdx.x * kTile + (threadIdx.x / 32) * 32 * kTileItems + threadIdx.x % 32;
    Pair item[kTileItems];
    bool live[kTileItems];
#pragma unroll
    for (int k = 0; k < kTileItems; ++k) {
        const int64_t i = first + 32 * k;
        live[k] = i < n;
        item[k] = Pair{0, 0};
        if (live[k]) item[k] = in ? in[i] : Pair{sort_key(ids[i], vocab), (uint32_t)i};
    }
    int before = 0, all = 0;
#pragma unroll 8
    for (int t = 0; t < n_tiles; ++t) {
        const int c = counts[(int64_t)t * kDigits + threadIdx.x];
        all += c;
        before += t < (int)blockIdx.x ? c : 0;
    }
    base[threadIdx.x] = block_exclusive(all, warp_sums) + before;
    int rank[kTileItems];
    tile_ranks<kTileItems>(item, live, pass, count, rank);  // its barriers also publish base
#pragma unroll
    for (int k = 0; k < kTileItems; ++k) {
        if (!live[k]) continue;
        const int64_t to = (int64_t)base[digit_of(item[k].key, pass)] + rank[k];
        out[to] = item[k];
        if (!last) atomicAdd(&next_counts[(to / kTile) * kDigits + digit_of(item[k].key, pass + 1)], 1);
    }
}

// ---------------------------------------------------------------------------------------------
// Sums over the sorted positions. A group of threads takes a block of `span` sorted positions and a range of
// columns; an id whose positions all lie in the block is finished there. What an id has in a block that it
// enters or leaves half-way goes to `partial` ([block][2][width]: the id the block begins with, the id it ends
// with), and k_join adds those up, block by block. Bound by memory: 32,768 ids, 50,003 x 1,024 fp32: 56 us, 4.3 TB/s of sums and zeros; with
// 64 registers instead of 90 it is 14 us slower, with 32 positions a block 4 us.
// ---------------------------------------------------------------------------------------------
constexpr int kAhead = 8;  // rows in flight a thread

template <class T, int VEC>
__device__ __forceinline__ void finish_row(T* row, const float (&sum)[VEC], float scale, bool accumulate) {
    Pack<T, VEC> o;
    if (accumulate) o = *reinterpret_cast<Pack<T, VEC>*>(row);
#pragma unroll
    for (int k = 0; k < VEC; ++k) o.v[k] = narrow<T>(accumulate ? widen(o.v[k]) + scale * sum[k] : scale * sum[k]);
    *reinterpret_cast<Pack<T, VEC>*>(row) = o;
}

constexpr int kZeroRows = 64;   // ids a CTA looks through for ones without a position
constexpr unsigned kZeroCtas = 148 * 2;
// About what a launch of the sort has time for (32,768 ids, 50,003 x 1,024 fp32: 96 us with 1 MB, 93 with 16, 98 with 32).
constexpr int64_t kZeroBytes = 16 << 20;

template <class T, int VEC>
__global__ void __launch_bounds__(kThreads) k_segments(const T* grad_out, int64_t grad_pitch, const Pair* sorted, int64_t n,
                                                       int64_t vocab, int64_t width, float scale, bool accumulate, T* __restrict__ table,
                                                       int64_t table_pitch, float* __restrict__ partial, int span, int group, int64_t sum_ctas, int64_t zero_first) {
    ptx::chained();
    const int64_t c = ((int64_t)blockIdx.y * group + threadIdx.x % group) * VEC;
    if ((int64_t)blockIdx.x >= sum_ctas) {  // rows without a position
        __shared__ unsigned char used[kZeroRows];
        const int64_t v0 = zero_first + ((int64_t)blockIdx.x - sum_ctas) * kZeroRows;
        const int64_t v1 = min(v0 + kZeroRows, vocab);
        if (threadIdx.x < v1 - v0) {  // every thread looks one id up
            const uint32_t v = (uint32_t)(v0 + threadIdx.x);
            int64_t a = 0, b = n;
            while (a < b) {
                const int64_t mid = (a + b) / 2;
                if (sorted[mid].key < v) a = mid + 1;
                else b = mid;
            }
            used[threadIdx.x] = a < n && sorted[a].key == v;
        }
        __syncthreads();
        Pack<T, VEC> zero;
#pragma unroll
        for (int k = 0; k < VEC; ++k) zero.v[k] = narrow<T>(0.0f);
        if (c < width)
            for (int64_t v = v0 + threadIdx.x / group; v < v1; v += kThreads / group)
                if (!used[v - v0]) *reinterpret_cast<Pack<T, VEC>*>(table + v * table_pitch + c) = zero;
        return;
    }
    const int64_t block = (int64_t)blockIdx.x * (kThreads / group) + threadIdx.x / group;
    const int64_t p0 = block * span, p1 = min(p0 + span, n);
    if (p0 >= n || c >= width) return;
    const uint32_t head = p0 > 0 ? sorted[p0 - 1].key : 0xffffffffu;  // an id equal to it began in an earlier block
    const uint32_t tail = p1 < n ? sorted[p1].key : 0xffffffffu;      // an id equal to it goes on in the next block
    float sum[VEC] = {};
    uint32_t key = sorted[p0].key;
    auto flush = [&]() {
        if (key >= (uint32_t)vocab) return;  // no token
        const bool enters = key == head, leaves = key == tail;
        if (!enters && !leaves) {
            finish_row<T, VEC>(table + (int64_t)key * table_pitch + c, sum, scale, accumulate);
        } else {
            float* to = partial + (block * 2 + (enters ? 0 : 1)) * width + c;
#pragma unroll
            for (int k = 0; k < VEC; ++k) to[k] = sum[k];
        }
    };
    for (int64_t p = p0; p < p1; p += kAhead) {
        Pair at[kAhead];
        Pack<T, VEC> row[kAhead];
#pragma unroll
        for (int k = 0; k < kAhead; ++k)
            if (p + k < p1) at[k] = sorted[p + k];
#pragma unroll
        for (int k = 0; k < kAhead; ++k)
            if (p + k < p1 && at[k].key < (uint32_t)vocab)
                row[k] = *reinterpret_cast<const Pack<T, VEC>*>(grad_out + (int64_t)at[k].pos * grad_pitch + c);
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            if (p + k >= p1) break;
            if (at[k].key != key) {
                flush();
                key = at[k].key;
#pragma unroll
                for (int e = 0; e < VEC; ++e) sum[e] = 0.0f;
            }
            if (key >= (uint32_t)vocab) continue;
#pragma unroll
            for (int e = 0; e < VEC; ++e) sum[e] += widen(row[k].v[e]);
        }
    }
    flush();
}

// The ids that lie in more than one block: the group of the block where such an id begins adds up its parts in
// block order.
template <class T, int VEC>
__global__ void __launch_bounds__(kThreads) k_join(const Pair* sorted, int64_t n, int64_t vocab, int64_t width, float scale,
                                                   bool accumulate, T* __restrict__ table, int64_t table_pitch,
                                                   const float* partial, int span, int group) {
    ptx::chained();
    const int64_t block = (int64_t)blockIdx.x * (kThreads / group) + threadIdx.x / group;
    const int64_t c = ((int64_t)blockIdx.y * group + threadIdx.x % group) * VEC;
    const int64_t p0 = block * span, p1 = p0 + span;
    if (p1 >= n || c >= width) return;  // the last block's ids end in it
    const uint32_t key = sorted[p1 - 1].key;
    if (key >= (uint32_t)vocab || sorted[p1].key != key) return;  // ends here
    if (p0 > 0 && sorted[p0 - 1].key == key) return;              // began earlier
    // the blocks that begin with this id follow one another; eight loads at a time, first of keys, then of sums
    int64_t end = block + 1;
    for (bool more = true; more;) {
        uint32_t k[8];
#pragma unroll
        for (int a = 0; a < 8; ++a) k[a] = (end + a) * span < n ? sorted[(end + a) * span].key : 0xffffffffu;
#pragma unroll
        for (int a = 0; a < 8; ++a) {
            more = more && k[a] == key;
            end += more;
        }
    }
    float sum[VEC];
#pragma unroll
    for (int k = 0; k < VEC; ++k) sum[k] = partial[(block * 2 + 1) * width + c + k];
#pragma unroll 8
    for (int64_t b = block + 1; b < end; ++b)
#pragma unroll
        for (int k = 0; k < VEC; ++k) sum[k] += partial[b * 2 * width + c + k];
    finish_row<T, VEC>(table + (int64_t)key * table_pitch + c, sum, scale, accumulate);
}

// ---------------------------------------------------------------------------------------------
// Few positions: no sort. A warp takes a position (and a range of columns), looks through all ids for its own, stops if an
// earlier position has it, else adds up the rows of all positions that have it, in order, as it finds them. n * n comparisons, 128
// at a time, are less work than the launches of a sort up to a few thousand positions. Further CTAs write the rows of ids that have
// no position.
// ---------------------------------------------------------------------------------------------
constexpr int64_t kDirectMost = 4096;        // positions
constexpr int64_t kDirectSearch = 60000000;  // comparisons: positions squared times the ranges of columns
constexpr int kDirectThreads = 256;
constexpr int kDirectWarps = kDirectThreads / 32;
constexpr int kFound = 128 + 32;  // positions a warp holds before it adds their rows up: one round of 128 ids, and a remainder

template <class T, int VEC>
__global__ void __launch_bounds__(kDirectThreads, 4) k_direct(const T* grad_out, int64_t grad_pitch, const int32_t* ids, int n,
                                                           int64_t vocab, int64_t width, float scale, bool accumulate, T* __restrict__ table,
                                                           int64_t table_pitch, int64_t sum_ctas) {
    ptx::chained();
    const int tid = threadIdx.x, warp = tid / 32, lane = tid % 32;
    constexpr int64_t kColumns = 32 * VEC;  // columns of a warp
    if ((int64_t)blockIdx.x >= sum_ctas) {        // rows without a position
        __shared__ unsigned char used[kZeroRows];
        const int64_t v0 = ((int64_t)blockIdx.x - sum_ctas) * kZeroRows;
        if (tid < kZeroRows) used[tid] = 0;
        __syncthreads();
#pragma unroll 4
        for (int i = tid; i < n; i += kDirectThreads) {
            const int64_t v = ids[i] - v0;
            if (v >= 0 && v < kZeroRows) used[v] = 1;
        }
        __syncthreads();
        Pack<T, VEC> zero;
#pragma unroll
        for (int k = 0; k < VEC; ++k) zero.v[k] = narrow<T>(0.0f);
        for (int v = warp; v < kZeroRows && v0 + v < vocab; v += kDirectWarps)
            if (!used[v])
                for (int64_t c = (int64_t)lane * VEC; c < width; c += 32 * VEC) *reinterpret_cast<Pack<T, VEC>*>(table + (v0 + v) * table_pitch + c) = zero;
        return;
    }
    __shared__ uint16_t found[kDirectWarps][kFound];
    const int64_t ranges = (width + kColumns - 1) / kColumns;
    const int64_t unit = (int64_t)blockIdx.x * kDirectWarps + warp;
    if (unit >= n * ranges) return;
    const int me = (int)(unit / ranges);
    const int64_t c0 = unit % ranges * kColumns + (int64_t)lane * VEC;
    const int32_t id = ids[me];
    if (id < 0 || id >= vocab) return;
    float sum[VEC] = {};
    int held = 0;
    const bool inside = c0 < width;
    auto add = [&](int from, int count) {  // rows found[from .. from + count), count <= kAhead
        Pack<T, VEC> r[kAhead];
#pragma unroll
        for (int a = 0; a < kAhead; ++a)
            if (a < count && inside) r[a] = *reinterpret_cast<const Pack<T, VEC>*>(grad_out + (int64_t)found[warp][from + a] * grad_pitch + c0);
#pragma unroll
        for (int a = 0; a < kAhead; ++a)
            if (a < count && inside)
#pragma unroll
                for (int e = 0; e < VEC; ++e) sum[e] += widen(r[a].v[e]);
    };
    // earlier positions: any hit, and this warp has nothing to do
    for (int p0 = 0; p0 < me; p0 += 512) {
        bool hit = false;
#pragma unroll
        for (int q = 0; q < 16; ++q) {
            const int p = p0 + q * 32 + lane;
            hit |= p < me && ids[p] == id;
        }
        if (__any_sync(0xffffffffu, hit)) return;
    }
    for (int p0 = me; p0 < n; p0 += 128) {
        unsigned hits[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const int p = p0 + q * 32 + lane;
            hits[q] = __ballot_sync(0xffffffffu, p < n && ids[p] == id);
        }
        if (!(hits[0] | hits[1] | hits[2] | hits[3])) continue;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            if (hits[q] >> lane & 1) found[warp][held + __popc(hits[q] & ((1u << lane) - 1))] = (uint16_t)(p0 + q * 32 + lane);
            held += __popc(hits[q]);
        }
        __syncwarp();
        int done = 0;
        for (; held - done >= kAhead; done += kAhead) add(done, kAhead);
        const uint16_t rest = lane < held - done ? found[warp][done + lane] : (uint16_t)0;
        __syncwarp();
        if (lane < held - done) found[warp][lane] = rest;
        held -= done;
    }
    __syncwarp();
    if (held > 0) add(0, held);
    if (inside) finish_row<T, VEC>(table + (int64_t)id * table_pitch + c0, sum, scale, accumulate);
}

// Columns one thread takes at once: 16 bytes where the rows allow it.
template <class T>
int columns_a_thread(const EmbedGradArgs& a) {
    constexpr int kVec = 16 / sizeof(T);
    return a.width % kVec == 0 && aligned16(a.grad_out, a.grad_out_pitch, sizeof(T)) && aligned16(a.grad_table, a.grad_table_pitch, sizeof(T)) ? kVec : 1;
}
// The two forms cross at 4,000 to 5,000 positions, where no id holds many of them; us, direct / sorted, 512 columns, ids spread over 32,000
// rows, the same with one id in 4 % and in 18 % of the places:
//   bf16  2,000 12 / 32, 13 / 31, 26 / 32; 4,096 23 / 28, 23 / 30, 48 / 38; 5,000 29 / 29, 29 / 32, 54 / 42; 8,192 59 / 32, 59 / 36, 90 / 53
//   fp32  2,000 20 / 33, 20 / 34, 28 / 35; 4,096 39 / 36, 39 / 37, 52 / 42; 5,000 51 / 36, 50 / 38, 70 / 44; 8,192 101 / 37, 99 / 40, 126 / 52
// An id in 18 % of the places is what a small vocabulary has: its warp adds its rows up alone, so there half as many positions go without a
// sort. 4,096 ids of 8,000 x 2,048 (more comparisons than allowed) 72 / 50.
bool is_direct(int64_t n_ids, int64_t vocab, int64_t width, int vec) {
    const int64_t most = vocab >= 4 * n_ids ? kDirectMost : kDirectMost / 2;
    return n_ids <= most && n_ids * n_ids * ceil_div(width, 32 * vec) <= kDirectSearch;
}

int sort_passes(int64_t vocab) {  // keys are 0 .. vocab
    int passes = 1;
    while (passes * kDigitBits < 32 && (vocab >> (passes * kDigitBits)) != 0) ++passes;
    return passes;
}

// Sorted positions one group sums up: small, so that short inputs still fill the GPU.
int segment_span(int64_t n_ids) { return n_ids <= 16384 ? 16 : 64; }

struct GradPlan {
    Pair* sorted;
    Pair* other;
    int* counts;
    float* partial;
    int64_t n_tiles;
    int passes;
};

int64_t grad_layout(int64_t vocab, int64_t width, int64_t n_ids, void* workspace, GradPlan* out) {
    GradPlan p{};
    Carver w(workspace);
    if (is_direct(n_ids, vocab, width, 1)) {  // whatever the alignment
        if (out) *out = p;
        return 0;
    }
    p.passes = sort_passes(vocab);
    p.n_tiles = ceil_div(n_ids, kTile);
    p.sorted = w.take<Pair>(n_ids);
    p.other = w.take<Pair>(n_ids);
    p.counts = w.take<int>(p.passes * p.n_tiles * kDigits);
    p.partial = w.take<float>(ceil_div(n_ids, segment_span(n_ids)) * 2 * width);
    if (out) *out = p;
    return w.used;
}

template <class T, int VEC>
cudaError_t segments_typed(const EmbedGradArgs& a, const GradPlan& p, int64_t zero_first, cudaStream_t s) {
    const int span = segment_span(a.n_ids);
    const int group = group_threads(a.width, VEC);
    const int64_t per_cta = kThreads / group;
    const int64_t blocks = ceil_div(a.n_ids, span);
    const int64_t col_ctas = ceil_div(a.width, (int64_t)group * VEC);
    auto* g = static_cast<const T*>(a.grad_out);
    auto* table = static_cast<T*>(a.grad_table);
    const int64_t sum_ctas = ceil_div(blocks, per_cta);
    const int64_t zero_ctas = a.accumulate ? 0 : ceil_div(a.vocab - zero_first, kZeroRows);
    A2_CUDA_TRY(launch_chained(k_segments<T, VEC>, dim3((unsigned)(sum_ctas + zero_ctas), (unsigned)col_ctas), kThreads, 0, s, g, a.grad_out_pitch, p.sorted,
                           a.n_ids, a.vocab, a.width, a.scale, a.accumulate, table, a.grad_table_pitch, p.partial, span, group, sum_ctas, zero_first));
    return launch_chained(k_join<T, VEC>, dim3((unsigned)sum_ctas, (unsigned)col_ctas), kThreads, 0, s, p.sorted, a.n_ids, a.vocab, a.width, a.scale,
                          a.accumulate, table, a.grad_table_pitch, p.partial, span, group);
}

template <class T, int VEC>
cudaError_t direct_typed(const EmbedGradArgs& a, cudaStream_t s) {
    const int64_t sum_ctas = ceil_div(a.n_ids * ceil_div(a.width, 32 * VEC), kDirectWarps);
    const int64_t ctas = sum_ctas + (a.accumulate ? 0 : ceil_div(a.vocab, kZeroRows));
    if (ctas == 0) return cudaSuccess;
    return launch_chained(k_direct<T, VEC>, dim3((unsigned)ctas), kDirectThreads, 0, s, static_cast<const T*>(a.grad_out), a.grad_out_pitch, a.ids,
                          (int)a.n_ids, a.vocab, a.width, a.scale, a.accumulate, static_cast<T*>(a.grad_table), a.grad_table_pitch, sum_ctas);
}

// Sorts the positions into p.sorted, then sums.
template <class T, int VEC>
cudaError_t sorted_typed(const EmbedGradArgs& a, const GradPlan& p, cudaStream_t s) {
    const int launches = p.passes + 1;
    const unsigned zero_ctas = a.accumulate ? 0 : kZeroCtas;
    const int64_t cleared = std::min(a.vocab, launches * std::max<int64_t>(1, kZeroBytes / (a.width * (int64_t)sizeof(T))));
    auto share = [&](int k) {
        return ZeroFill{static_cast<char*>(a.grad_table), cleared * k / launches, cleared * (k + 1) / launches, a.width * (int64_t)sizeof(T),
                        a.grad_table_pitch * (int64_t)sizeof(T), VEC * sizeof(T) == 16};
    };
    A2_CUDA_TRY(launch_chained(k_sort_count, dim3((unsigned)p.n_tiles + zero_ctas), kSortThreads, 0, s, a.ids, a.n_ids, a.vocab, p.passes, (int)p.n_tiles,
                           p.counts, share(0)));
    // the passes go back and forth between the two buffers and end in p.sorted
    const Pair* from = nullptr;
    for (int pass = 0; pass < p.passes; ++pass) {
        Pair* to = (p.passes - pass) % 2 == 1 ? p.sorted : p.other;
        const int* counts = p.counts + (int64_t)pass * p.n_tiles * kDigits;
        const bool last = pass + 1 == p.passes;
        A2_CUDA_TRY(launch_chained(k_sort_pass, dim3((unsigned)p.n_tiles + zero_ctas), kSortThreads, 0, s, a.ids, from, a.n_ids, a.vocab, pass, last, counts,
                               (int)p.n_tiles, to, last ? nullptr : p.counts + (int64_t)(pass + 1) * p.n_tiles * kDigits, share(pass + 1)));
        from = to;
    }
    return segments_typed<T, VEC>(a, p, cleared, s);
}

template <class T>
cudaError_t grad_typed(const EmbedGradArgs& a, const GradPlan& p, cudaStream_t s) {
    constexpr int kVec = 16 / sizeof(T);
    const int vec = columns_a_thread<T>(a);
    if (is_direct(a.n_ids, a.vocab, a.width, vec)) return vec == kVec ? direct_typed<T, kVec>(a, s) : direct_typed<T, 1>(a, s);
    return vec == kVec ? sorted_typed<T, kVec>(a, p, s) : sorted_typed<T, 1>(a, p, s);
}

}  // namespace

cudaError_t run_embed(const EmbedArgs& a, cudaStream_t s) {
    if (a.n_ids == 0) return cudaSuccess;
    return a.dtype == A2_BF16 ? embed_typed<__nv_bfloat16>(a, s) : embed_typed<float>(a, s);
}

int64_t embed_grad_workspace(int64_t vocab, int64_t width, int64_t n_ids) { return grad_layout(vocab, width, n_ids, nullptr, nullptr); }

cudaError_t run_embed_grad(const EmbedGradArgs& a, void* workspace, cudaStream_t s) {
    GradPlan p;
    grad_layout(a.vocab, a.width, a.n_ids, workspace, &p);
    return a.dtype == A2_BF16 ? grad_typed<__nv_bfloat16>(a, p, s) : grad_typed<float>(a, p, s);
}

}  // namespace a2
