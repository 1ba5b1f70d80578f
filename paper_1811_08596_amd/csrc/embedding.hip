// Embedding lookup and its gradient by sorted tokens.
//
//   out[t] = scale * table[token t]            table_grad[v] = base[v] + scale * sum over {t : token t = v} of out_grad[t]
//
// Both are bound by bytes.  The gradient's rows are summed without atomics: the places are sorted by their token (stable,
// so every token's places stay in order), the sorted list is cut into stretches of equal length, a wave sums the rows of
// one stretch and writes each row of the table whose run of places lies within it; a run that crosses stretches leaves one
// partial sum in each, which a second launch adds in their order.  So the order of every sum follows from the tokens and
// the sizes alone, and a token with most of the places is summed by as many waves as it has stretches.
#include "layers.h"

#include <algorithm>

namespace fftsp {
namespace {

__device__ __forceinline__ uint32_t token_row(const void* tokens, int token_bits, size_t t, uint32_t rows)
{
    const int64_t v = token_bits == 64 ? static_cast<const int64_t*>(tokens)[t] : static_cast<const int32_t*>(tokens)[t];
    return (uint64_t)v < rows ? (uint32_t)v : rows;  // `rows`: none
}

// ---- lookup: `lanes` lanes to a row (a power of two up to 256), V values to a lane at a time ----
// Bound by bytes: 16384 rows of 2048 from fp32 into bf16, 201 MB, take 26.6 us (rows that come again are read from the caches).
// One row of 1024 takes 1.7 us, a launch's end.
template <typename TI, typename TO, int V, bool WHOLE>
__global__ void __launch_bounds__(256) k_embedding(EmbeddingArgs a, uint32_t lanes)
{
    const uint32_t li = threadIdx.x & (lanes - 1u);
    const size_t per = 256u / lanes;
    for (size_t t = blockIdx.x * per + threadIdx.x / lanes; t < a.ntokens; t += gridDim.x * per) {
        const uint32_t row = token_row(a.tokens, a.token_bits, t, (uint32_t)a.rows);
        const bool inside = row < a.rows;
        const TI* src = static_cast<const TI*>(a.source) + (size_t)(inside ? row : 0u) * a.source_stride;
        TO* dst = static_cast<TO*>(a.out) + t * a.out_stride;
        for (uint32_t c = li * V; c < a.width; c += lanes * V) {
            if (WHOLE || c + V <= a.width) {
                Run<TI, V> x{};
                if (inside) x = load_run<TI, V>(src + c);
                Run<TO, V> y;
#pragma unroll
                for (int i = 0; i < V; ++i) y.v[i] = from_float<TO>(inside ? to_float(x.v[i]) * a.scale : 0.f);
                store_run<TO, V>(dst + c, y);
            } else {
                for (uint32_t j = c; j < a.width; ++j) dst[j] = from_float<TO>(inside ? to_float(src[j]) * a.scale : 0.f);
            }
        }
    }
}

// ---- rows that no token has: zeros, or the base's.  Written by workgroups beside those that sort. ----
struct FillArgs {
    const uint8_t* base;  // nullptr: zeros
    uint8_t* out;
    uint64_t chunks;      // of 16 bytes, rounded up, by row
    uint64_t per_row;     // chunks
    uint64_t row_values, stride;
    int bytes;            // of an element
};
template <typename U>
__device__ __forceinline__ void fill_chunk(const FillArgs& f, uint64_t i)
{
    constexpr uint32_t V = 16 / sizeof(U);
    const uint64_t row = f.per_row == f.chunks ? 0 : i / f.per_row, c = (i - row * f.per_row) * V, at = row * f.stride + c;
    U* out = reinterpret_cast<U*>(f.out) + at;
    const U* base = f.base ? reinterpret_cast<const U*>(f.base) + at : nullptr;
    if (c + V <= f.row_values) {
        Run<U, V> x{};
        if (base) x = load_run<U, V>(base);
        store_run<U, V>(out, x);
    } else {
        for (uint64_t j = 0; c + j < f.row_values; ++j) out[j] = base ? base[j] : (U)0;
    }
}
// Chunks [first, end), by `count` workgroups: as a rule one a thread, in the order the workgroups begin in, so that all of them
// together write one stretch at a time, which the memory takes at 6.8 TB/s (400 to 1000 MB; half a million threads that
// go round, 4.5 to 4.9).
constexpr uint32_t kMostFillers = 1u << 21;
__device__ __forceinline__ void fill(const FillArgs& f, uint64_t first, uint64_t end, uint32_t index, uint32_t count)
{
    const uint64_t step = (uint64_t)count * blockDim.x;
    uint64_t i = first + (uint64_t)index * blockDim.x + threadIdx.x;
    if (f.bytes == 4)
        for (; i < end; i += step) fill_chunk<uint32_t>(f, i);
    else
        for (; i < end; i += step) fill_chunk<uint16_t>(f, i);
}

// ---- sorting the places by token: least significant digits first, stable ----
// A wave ranks 64 places at a time: the lanes with its own digit by one ballot per bit, the earlier groups' by a count.
constexpr int kDigitBits = 9, kDigits = 1 << kDigitBits;

__device__ __forceinline__ uint64_t same_digit(uint32_t digit, bool present)
{
    uint64_t m = __ballot(present);
#pragma unroll
    for (int b = 0; b < kDigitBits; ++b) {
        const uint64_t v = __ballot((digit >> b) & 1u);
        m &= (digit >> b) & 1u ? v : ~v;
    }
    return m;
}
// the place of a group's items among those of their digit that the wave has had before; counts them
template <typename U>
__device__ __forceinline__ uint32_t rank_in_wave(U* wave_count, uint32_t digit, bool present, uint32_t lane)
{
    const uint64_t same = same_digit(digit, present), lower = same & ((1ull << lane) - 1ull);
    uint32_t old = 0;
    if (present) old = wave_count[digit];
    // every lane has read before the first of each digit writes: a wave's LDS accesses are done in order, and the fences keep
    // the compiler to it
    __builtin_amdgcn_fence(__ATOMIC_SEQ_CST, "wavefront");
    __builtin_amdgcn_wave_barrier();
    if (present && lower == 0) wave_count[digit] = (U)(old + (uint32_t)__popcll(same));
    __builtin_amdgcn_fence(__ATOMIC_SEQ_CST, "wavefront");
    __builtin_amdgcn_wave_barrier();
    return old + (uint32_t)__popcll(lower);
}
// exclusive sums of one value a thread of the first kDigits threads; `scan`: kDigits / 64 words
__device__ __forceinline__ uint32_t digits_before(uint32_t v, uint32_t* scan)
{
    const uint32_t tid = threadIdx.x, lane = tid & 63u;
    uint32_t sum = v;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const uint32_t u = __shfl_up(sum, d);
        if (lane >= (uint32_t)d) sum += u;
    }
    if (tid < kDigits && lane == 63) scan[tid >> 6] = sum;
    __syncthreads();
    uint32_t before = 0;
    for (uint32_t w = 0; w < kDigits / 64; ++w)
        if (w < tid >> 6) before += scan[w];
    __syncthreads();
    return before + sum - v;
}

struct SortArgs {
    const void* tokens;
    int token_bits;
    uint32_t rows, count, blocks;
    uint2* a;            // (token, place)
    uint2* b;
    uint32_t* counts;    // [passes][blocks][kDigits]
    uint32_t* groups;    // [groups of kGroupBlocks blocks][kDigits] of the pass, or nullptr
    int passes;
    FillArgs fill;
};

// up to kSortOne places: one workgroup, all passes in LDS; the others fill.  8192 places of 64 values take 31 us with their sums, as
// launches of many workgroups (8193) 35.  Its own work hides behind a large table's fill: 50000 x 2048 in fp32 takes 66 us, 6.2 TB/s.
constexpr uint32_t kOneThreads = 1024, kOneWaves = kOneThreads / 64, kOneGroups = 8, kSortOne = kOneThreads * kOneGroups;
__global__ void __launch_bounds__(kOneThreads) k_sort_one(SortArgs s)
{
    __shared__ uint32_t keys[kSortOne];  // 64 KB with the rest: two workgroups to a compute unit
    __shared__ uint16_t places[kSortOne];
    __shared__ uint16_t wave_count[kOneWaves][kDigits];
    __shared__ uint32_t scan[kDigits / 64];
    if (blockIdx.x) {
        fill(s.fill, 0, s.fill.chunks, blockIdx.x - 1, gridDim.x - 1);
        return;
    }
    const uint32_t tid = threadIdx.x, lane = tid & 63u, wave = tid >> 6;
    const uint32_t groups = (s.count + kOneThreads - 1) / kOneThreads;  // of 64 places that a wave has
    uint2 item[kOneGroups];
#pragma unroll
    for (uint32_t g = 0; g < kOneGroups; ++g) {
        if (g >= groups) break;
        const uint32_t i = (wave * groups + g) * 64 + lane;
        item[g] = make_uint2(i < s.count ? token_row(s.tokens, s.token_bits, i, s.rows) : 0xFFFFFFFFu, i);
    }
    for (int pass = 0; pass < s.passes; ++pass) {
        const int shift = pass * kDigitBits;
        for (uint32_t i = tid; i < kOneWaves * kDigits / 2; i += kOneThreads) reinterpret_cast<uint32_t*>(&wave_count[0][0])[i] = 0;
        __syncthreads();
        uint32_t rank[kOneGroups];
#pragma unroll
        for (uint32_t g = 0; g < kOneGroups; ++g) {
            if (g >= groups) break;
            const bool present = (wave * groups + g) * 64 + lane < s.count;
            rank[g] = rank_in_wave(wave_count[wave], (item[g].x >> shift) & (kDigits - 1u), present, lane);
        }
        __syncthreads();
        uint32_t total = 0;
        if (tid < kDigits)
#pragma unroll
            for (uint32_t w = 0; w < kOneWaves; ++w) total += wave_count[w][tid];
        uint32_t sum = digits_before(total, scan);
        if (tid < kDigits)
#pragma unroll
            for (uint32_t w = 0; w < kOneWaves; ++w) {
                const uint32_t c = wave_count[w][tid];
                wave_count[w][tid] = (uint16_t)sum;
                sum += c;
            }
        __syncthreads();
#pragma unroll
        for (uint32_t g = 0; g < kOneGroups; ++g)
            if (g < groups && (wave * groups + g) * 64 + lane < s.count) {
                const uint32_t at = wave_count[wave][(item[g].x >> shift) & (kDigits - 1u)] + rank[g];
                keys[at] = item[g].x;
                places[at] = (uint16_t)item[g].y;
            }
        __syncthreads();
#pragma unroll
        for (uint32_t g = 0; g < kOneGroups; ++g) {
            if (g >= groups) break;
            const uint32_t i = (wave * groups + g) * 64 + lane;
            if (i < s.count) item[g] = make_uint2(keys[i], places[i]);
        }
        __syncthreads();
    }
#pragma unroll
    for (uint32_t g = 0; g < kOneGroups; ++g) {
        if (g >= groups) break;
        const uint32_t i = (wave * groups + g) * 64 + lane;
        if (i < s.count) s.a[i] = item[g];
    }
}

// more places: workgroups of kSortBlock places, a launch a pass behind one that counts; other workgroups fill a share in each
constexpr int kSortThreads = kDigits, kSortWaves = kSortThreads / 64;
constexpr uint32_t kSortBlock = 2048, kGroups = kSortBlock / kSortThreads;

__device__ __forceinline__ bool fill_share(const SortArgs& s, int launch)
{
    if (blockIdx.x < s.blocks) return false;
    const uint64_t launches = (uint64_t)s.passes + 1, first = s.fill.chunks * launch / launches, end = s.fill.chunks * (launch + 1) / launches;
    fill(s.fill, first, end, blockIdx.x - s.blocks, gridDim.x - s.blocks);
    return true;
}

// counts of the first digit, block by block; clears the later passes' counts
__global__ void __launch_bounds__(kSortThreads) k_sort_count(SortArgs s)
{
    __shared__ uint32_t hist[kDigits];
    if (fill_share(s, 0)) return;
    const uint32_t tid = threadIdx.x, at = blockIdx.x * kSortBlock;
    hist[tid] = 0;
    __syncthreads();
#pragma unroll
    for (uint32_t g = 0; g < kGroups; ++g) {
        const uint32_t i = at + g * kSortThreads + tid;
        if (i < s.count) atomicAdd(&hist[token_row(s.tokens, s.token_bits, i, s.rows) & (kDigits - 1u)], 1u);
    }
    __syncthreads();
    s.counts[(size_t)blockIdx.x * kDigits + tid] = hist[tid];
    for (int p = 1; p < s.passes; ++p) s.counts[((size_t)p * s.blocks + blockIdx.x) * kDigits + tid] = 0;
}

// Sums of rows of counts: all of them and the first `mine`
__device__ __forceinline__ void add_rows(const uint32_t* rows, uint32_t count, uint32_t mine, uint32_t* before, uint32_t* total)
{
    uint32_t b = 0;
    for (; b + 16 <= count; b += 16) {
        uint32_t c[16];
#pragma unroll
        for (int u = 0; u < 16; ++u) c[u] = rows[(size_t)(b + u) * kDigits];
#pragma unroll
        for (int u = 0; u < 16; ++u) {
            if (b + u < mine) *before += c[u];
            *total += c[u];
        }
    }
    for (; b < count; ++b) {
        const uint32_t c = rows[(size_t)b * kDigits];
        if (b < mine) *before += c;
        *total += c;
    }
}
// Many blocks: sums of kGroupBlocks blocks' counts each, so that a workgroup reads those of all groups and of its own group's
// blocks, not of all blocks, whose bytes grow as the square of the places.  Two passes over 2^20, 2^22 and 2^24 places take
// 84, 308 and 1169 us, with all blocks' counts in every workgroup 107, 855 and 18331; over 2^19 54 either way.
constexpr uint32_t kGroupBlocks = 64, kManyBlocks = 256;
__global__ void __launch_bounds__(kSortThreads) k_sort_groups(SortArgs s, int pass)
{
    const uint32_t first = blockIdx.x * kGroupBlocks;
    uint32_t before = 0, total = 0;
    add_rows(s.counts + ((size_t)pass * s.blocks + first) * kDigits + threadIdx.x, min(kGroupBlocks, s.blocks - first), 0, &before, &total);
    s.groups[(size_t)blockIdx.x * kDigits + threadIdx.x] = total;
}

// one pass: every workgroup finds where its digits begin from the blocks' counts, and counts the next pass's digits by the
// block that its places go to
__global__ void __launch_bounds__(kSortThreads) k_sort_scatter(SortArgs s, int pass)
{
    __shared__ uint32_t wave_count[kSortWaves][kDigits];
    __shared__ uint32_t scan[kDigits / 64];
    if (fill_share(s, pass + 1)) return;
    const uint32_t tid = threadIdx.x, wave = tid >> 6, lane = tid & 63u;
    const uint2* from = pass & 1 ? s.b : s.a;
    uint2* to = pass & 1 ? s.a : s.b;
    const uint32_t* counts = s.counts + (size_t)pass * s.blocks * kDigits + tid;
    uint32_t* next = pass + 1 < s.passes ? s.counts + (size_t)(pass + 1) * s.blocks * kDigits : nullptr;
    // a wave's share: consecutive groups of 64 places
    uint2 item[kGroups];
#pragma unroll
    for (uint32_t g = 0; g < kGroups; ++g) {
        const uint32_t i = blockIdx.x * kSortBlock + (wave * kGroups + g) * 64 + lane;
        item[g] = make_uint2(0xFFFFFFFFu, i);
        if (i < s.count) item[g] = pass ? from[i] : make_uint2(token_row(s.tokens, s.token_bits, i, s.rows), i);
    }
#pragma unroll
    for (int w = 0; w < kSortWaves; ++w) wave_count[w][tid] = 0;
    uint32_t before = 0, total = 0;
    if (s.groups) {
        const uint32_t group = blockIdx.x / kGroupBlocks;
        uint32_t own = 0;
        add_rows(s.groups + tid, (s.blocks + kGroupBlocks - 1) / kGroupBlocks, group, &before, &total);
        add_rows(counts + (size_t)group * kGroupBlocks * kDigits, blockIdx.x % kGroupBlocks, kGroupBlocks, &before, &own);
    } else {
        add_rows(counts, s.blocks, blockIdx.x, &before, &total);
    }
    uint32_t sum = digits_before(total, scan) + before;  // a barrier within: wave_count is clear
    uint32_t rank[kGroups];
    const int shift = pass * kDigitBits;
#pragma unroll
    for (uint32_t g = 0; g < kGroups; ++g) {
        const bool present = blockIdx.x * kSortBlock + (wave * kGroups + g) * 64 + lane < s.count;
        rank[g] = rank_in_wave(wave_count[wave], (item[g].x >> shift) & (kDigits - 1u), present, lane);
    }
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kSortWaves; ++w) {
        const uint32_t c = wave_count[w][tid];
        wave_count[w][tid] = sum;
        sum += c;
    }
    __syncthreads();
#pragma unroll
    for (uint32_t g = 0; g < kGroups; ++g) {
        const uint32_t i = blockIdx.x * kSortBlock + (wave * kGroups + g) * 64 + lane;
        if (i >= s.count) continue;
        const uint32_t at = wave_count[wave][(item[g].x >> shift) & (kDigits - 1u)] + rank[g];
        to[at] = item[g];
        if (next) atomicAdd(&next[(size_t)(at / kSortBlock) * kDigits + ((item[g].x >> (shift + kDigitBits)) & (kDigits - 1u))], 1u);
    }
}

// nothing to sort
__global__ void __launch_bounds__(256) k_fill(FillArgs f) { fill(f, 0, f.chunks, blockIdx.x, gridDim.x); }

// ---- sums over the sorted places ----
struct SumArgs {
    const uint2* sorted;
    uint32_t count, stretch, stretches;
    uint32_t rows, width;
    const void* source;
    void* out;
    size_t source_stride, out_stride;
    float scale;
    int add;         // the row's present value (the base) is added
    float* partial;  // [stretches][2][width]: what a run that began before the stretch has in it; what a run has that goes on behind it
};

// there: the row's present values, where they are added and all V columns are
template <typename TO, int V>
__device__ __forceinline__ void write_row(const SumArgs& a, uint32_t row, uint32_t c, uint32_t n, const float* acc, const Run<TO, V>& there)
{
    TO* dst = static_cast<TO*>(a.out) + (size_t)row * a.out_stride + c;
    if (n == V) {
        Run<TO, V> y;
#pragma unroll
        for (int i = 0; i < V; ++i) y.v[i] = from_float<TO>(a.add ? to_float(there.v[i]) + acc[i] * a.scale : acc[i] * a.scale);
        store_run<TO, V>(dst, y);
    } else {
#pragma unroll
        for (uint32_t i = 0; i < V; ++i)
            if (i < n) dst[i] = from_float<TO>(a.add ? to_float(dst[i]) + acc[i] * a.scale : acc[i] * a.scale);
    }
}
template <int V>
__device__ __forceinline__ void write_partial(const SumArgs& a, uint32_t stretch, uint32_t which, uint32_t c, uint32_t n, const float* acc)
{
    float* dst = a.partial + ((size_t)stretch * 2 + which) * a.width + c;
    if (n == V) {
        Run<float, V> r;
#pragma unroll
        for (int i = 0; i < V; ++i) r.v[i] = acc[i];
        store_run<float, V>(dst, r);
    } else {
#pragma unroll
        for (uint32_t i = 0; i < V; ++i)
            if (i < n) dst[i] = acc[i];
    }
}

// A wave has a stretch of the sorted places and 64 V columns; kAhead rows are on their way together.  Bound by bytes: 65536 rows
// of 768 bf16, a third of them nobody's, and the rows of a 32000 x 768 fp32 table read and written where they have a token, 38 us.
constexpr uint32_t kAhead = 8;
template <typename TI, typename TO, int V, bool ADD>
__global__ void __launch_bounds__(256) k_sum_stretches(SumArgs a, uint32_t slabs)
{
    const uint32_t wave = __builtin_amdgcn_readfirstlane(blockIdx.x * 4u + (threadIdx.x >> 6)), lane = threadIdx.x & 63u;
    const uint32_t stretch = wave / slabs, slab = wave - stretch * slabs;
    if (stretch >= a.stretches) return;
    const uint32_t c = (slab * 64u + lane) * V;
    const uint32_t n = c >= a.width ? 0u : min((uint32_t)V, a.width - c);
    const uint32_t first = stretch * a.stretch, end = min(a.count, first + a.stretch);
    const TI* src = static_cast<const TI*>(a.source) + c;
    float acc[V];
#pragma unroll
    for (int i = 0; i < V; ++i) acc[i] = 0.f;
    bool head = false;  // the run began before this stretch
    for (uint32_t at = first; at < end; at += 64u) {
        const uint32_t here = min(64u, end - at);
        const uint2 own = a.sorted[at + min(lane, here - 1)];
        const uint32_t behind = at + here < a.count ? a.sorted[at + here].x : a.rows;
        if (at == first) head = first > 0 && a.sorted[first - 1].x == (uint32_t)__builtin_amdgcn_readfirstlane((int)own.x);
        for (uint32_t p = 0; p < here; p += kAhead) {
            Run<TI, V> x[kAhead];
            Run<TO, V> y[ADD ? kAhead : 1];
            uint32_t row[kAhead + 1];
#pragma unroll
            for (uint32_t u = 0; u <= kAhead; ++u)
                row[u] = p + u < here ? (uint32_t)__builtin_amdgcn_readlane((int)own.x, (int)(p + u)) : behind;
#pragma unroll
            for (uint32_t u = 0; u < kAhead; ++u) {
                const uint32_t place = (uint32_t)__builtin_amdgcn_readlane((int)own.y, (int)min(p + u, here - 1));
                const TI* r = src + (size_t)place * a.source_stride;
                if (n == V) {
                    x[u] = load_run<TI, V>(r);
                    // what is in the table's row already, where a run ends
                    if (ADD && p + u < here && row[u] != row[u + 1] && row[u] < a.rows)
                        y[ADD ? u : 0] = load_run<TO, V>(static_cast<const TO*>(a.out) + (size_t)row[u] * a.out_stride + c);
                } else {
#pragma unroll
                    for (uint32_t i = 0; i < V; ++i) x[u].v[i] = i < n ? r[i] : TI{};
                }
            }
#pragma unroll
            for (uint32_t u = 0; u < kAhead; ++u) {
                if (p + u >= here) break;
                if (row[u] >= a.rows) return;  // tokens outside the table are sorted last
#pragma unroll
                for (int i = 0; i < V; ++i) acc[i] += to_float(x[u].v[i]);
                const bool last = at + p + u + 1 == end;
                if (row[u] == row[u + 1] && !last) continue;
                if (head) write_partial<V>(a, stretch, 0, c, n, acc);
                else if (row[u] == row[u + 1]) write_partial<V>(a, stretch, 1, c, n, acc);
                else write_row<TO, V>(a, row[u], c, n, acc, y[ADD ? u : 0]);
#pragma unroll
                for (int i = 0; i < V; ++i) acc[i] = 0.f;
                head = false;
            }
        }
    }
}

// runs that cross stretches: a workgroup per stretch in which one begins and goes on, and per slab of 64 V columns; its
// waves have every fourth part, in order
template <typename TI, typename TO, int V>
__global__ void __launch_bounds__(256) k_join_runs(SumArgs a)
{
    __shared__ float part[3][64 * V];
    const uint32_t stretch = blockIdx.x, lane = threadIdx.x & 63u, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t first = stretch * a.stretch, end = first + a.stretch;
    if (end >= a.count) return;
    const uint32_t run = a.sorted[end].x, inside = a.sorted[end - 1].x, begin = a.sorted[first].x, earlier = first ? a.sorted[first - 1].x : run + 1;
    if (run >= a.rows || inside != run || (begin == run && earlier == run)) return;  // none, or it began earlier
    // the last stretch that the run reaches: 64 of the stretches' first places at a time
    uint32_t last = stretch + 1;
    for (uint32_t s = stretch + 1;; s += 64u) {
        const uint32_t t = s + lane;
        const uint64_t in = __ballot(t < a.stretches && a.sorted[(size_t)t * a.stretch].x == run);
        const uint32_t k = in == ~0ull ? 64u : (uint32_t)__builtin_ctzll(~in);
        if (k) last = s + k - 1;
        if (k < 64) break;
    }
    const uint32_t c = (blockIdx.y * 64u + lane) * V;
    const uint32_t n = c >= a.width ? 0u : min((uint32_t)V, a.width - c);
    float acc[V];
#pragma unroll
    for (int i = 0; i < V; ++i) acc[i] = 0.f;
    for (uint32_t s = stretch + wave; s <= last; s += 4u * 4u) {
        Run<float, V> x[4];
#pragma unroll
        for (uint32_t u = 0; u < 4; ++u) {
            const uint32_t t = min(s + 4u * u, last);
            const float* p = a.partial + ((size_t)t * 2 + (t == stretch ? 1u : 0u)) * a.width + c;
            if (n == V) {
                x[u] = load_run<float, V>(p);
            } else {
#pragma unroll
                for (uint32_t i = 0; i < V; ++i) x[u].v[i] = i < n ? p[i] : 0.f;
            }
        }
#pragma unroll
        for (uint32_t u = 0; u < 4; ++u)
            if (s + 4u * u <= last)
#pragma unroll
                for (int i = 0; i < V; ++i) acc[i] += x[u].v[i];
    }
    if (wave)
#pragma unroll
        for (int i = 0; i < V; ++i) part[wave - 1][lane * V + i] = acc[i];
    __syncthreads();
    if (wave) return;
    for (int w = 0; w < 3; ++w)
#pragma unroll
        for (int i = 0; i < V; ++i) acc[i] += part[w][lane * V + i];
    Run<TO, V> there{};
    if (a.add && n == V) there = load_run<TO, V>(static_cast<const TO*>(a.out) + (size_t)run * a.out_stride + c);
    write_row<TO, V>(a, run, c, n, acc, there);
}

// ---- up to kFew places: no sorting, one launch (700 places, 5003 x 257 in fp32: 10 us; a sort's launches take 21) ----
// A workgroup per place and slab of 64 V columns compares its token with all others; if it is the first with that token, it sums
// the rows of all of them, its waves eight rows at a time in turn.  Other workgroups fill the rows that no token has.
constexpr uint32_t kFew = 2048;           // places
constexpr uint32_t kFewRows = 1u << 18;   // rows whose bits a workgroup holds
constexpr uint64_t kFewBytes = 32 << 20;   // of a table that is filled beside the sums
// workgroups that sum: some 4.5 us a thousand, where sorting takes 21 us and more.  4000 rows, bf16 into fp32: 1000, 2048 and 4096
// workgroups (500, 1024 and 2048 places of 512 values) take 8, 12.5 and 21 us, 8000 (1000 places of 2048) 36 and by sorting 21
constexpr uint64_t kFewGroups = 4096;
struct FewArgs {
    EmbeddingArgs e;  // source: the rows' gradients, out: the table's
    uint32_t slabs, fillers, lanes;
};
template <typename TI, typename TO, int V>
__global__ void __launch_bounds__(256) k_gradient_few(FewArgs f)
{
    const EmbeddingArgs& a = f.e;
    const uint32_t tid = threadIdx.x, lane = tid & 63u, wave = __builtin_amdgcn_readfirstlane(tid >> 6), count = (uint32_t)a.ntokens;
    const TO* base = static_cast<const TO*>(a.base);
    TO* out = static_cast<TO*>(a.out);
    if (blockIdx.x >= count * f.slabs) {
        // rows that have a token, by bit; then rows in turn, `per` to a workgroup, so that all write one stretch at a time
        extern __shared__ uint32_t has[];
        const uint32_t index = blockIdx.x - count * f.slabs, li = tid & (f.lanes - 1u), per = 256u / f.lanes, rows = (uint32_t)a.rows;
        for (uint32_t i = tid; i < (rows + 31u) / 32u; i += 256) has[i] = 0;
        __syncthreads();
        for (uint32_t t = tid; t < count; t += 256) {
            const uint32_t row = token_row(a.tokens, a.token_bits, t, rows);
            if (row < rows) atomicOr(&has[row / 32u], 1u << (row & 31u));
        }
        __syncthreads();
        constexpr uint32_t W = 16 / sizeof(TO);
        for (uint32_t row = index * per + tid / f.lanes; row < rows; row += f.fillers * per) {
            if (has[row / 32u] >> (row & 31u) & 1u) continue;
            for (uint32_t c = li * W; c < a.width; c += f.lanes * W) {
                const uint64_t at = (uint64_t)row * a.out_stride + c;
                if (c + W <= a.width) {
                    Run<TO, W> x{};
                    if (base) x = load_run<TO, W>(base + at);
                    store_run<TO, W>(out + at, x);
                } else {
                    for (uint32_t j = 0; c + j < a.width; ++j) out[at + j] = base ? base[at + j] : TO{};
                }
            }
        }
        return;
    }
    __shared__ uint64_t same[kFew / 64];
    __shared__ uint16_t places[kFew];
    __shared__ float part[3][64 * V];
    const uint32_t place = blockIdx.x / f.slabs, slab = blockIdx.x - place * f.slabs;
    const uint32_t row = token_row(a.tokens, a.token_bits, place, (uint32_t)a.rows);
    if (row >= a.rows) return;
    const uint32_t c = (slab * 64u + lane) * V, n = c >= a.width ? 0u : min((uint32_t)V, a.width - c);
    const uint64_t at = (uint64_t)row * a.out_stride + c;
    Run<TO, V> there{};
    if (base && wave == 0) {
        if (n == V) there = load_run<TO, V>(base + at);
        else
#pragma unroll
            for (uint32_t i = 0; i < V; ++i)
                if (i < n) there.v[i] = base[at + i];
    }
    uint32_t mine = 0;  // which of this lane's places have the token
#pragma unroll
    for (uint32_t k = 0; k < kFew / 256; ++k) {
        const uint32_t t = k * 256 + tid;
        const bool is = t < count && token_row(a.tokens, a.token_bits, t, (uint32_t)a.rows) == row;
        const uint64_t m = __ballot(is);
        if (lane == 0) same[k * 4 + wave] = m;
        mine |= (is ? 1u : 0u) << k;
    }
    __syncthreads();
    uint32_t total = 0, before = 0;  // places of the token; those before this one
#pragma unroll
    for (uint32_t i = 0; i < kFew / 64; ++i) {
        const uint64_t m = same[i];
        before += i * 64 + 64 <= place ? (uint32_t)__popcll(m) : i * 64 <= place ? (uint32_t)__popcll(m & ((1ull << (place & 63u)) - 1ull)) : 0u;
        total += (uint32_t)__popcll(m);
    }
    if (before) return;  // another workgroup's
#pragma unroll
    for (uint32_t k = 0; k < kFew / 256; ++k)
        if (mine >> k & 1u) {
            uint32_t r = (uint32_t)__popcll(same[k * 4 + wave] & ((1ull << lane) - 1ull));
            for (uint32_t i = 0; i < k * 4 + wave; ++i) r += (uint32_t)__popcll(same[i]);
            places[r] = (uint16_t)(k * 256 + tid);
        }
    __syncthreads();
    float acc[V];
#pragma unroll
    for (int i = 0; i < V; ++i) acc[i] = 0.f;
    const TI* src = static_cast<const TI*>(a.source) + c;
    for (uint32_t p = wave * kAhead; p < total; p += 4 * kAhead) {
        Run<TI, V> x[kAhead];
#pragma unroll
        for (uint32_t u = 0; u < kAhead; ++u) {
            const TI* r = src + (size_t)__builtin_amdgcn_readfirstlane(places[min(p + u, total - 1)]) * a.source_stride;
            if (n == V) {
                x[u] = load_run<TI, V>(r);
            } else {
#pragma unroll
                for (uint32_t i = 0; i < V; ++i) x[u].v[i] = i < n ? r[i] : TI{};
            }
        }
#pragma unroll
        for (uint32_t u = 0; u < kAhead; ++u)
            if (p + u < total)
#pragma unroll
                for (int i = 0; i < V; ++i) acc[i] += to_float(x[u].v[i]);
    }
    if (total > kAhead) {
        if (wave)
#pragma unroll
            for (int i = 0; i < V; ++i) part[wave - 1][lane * V + i] = acc[i];
        __syncthreads();
        if (wave == 0)
            for (int w = 0; w < 3; ++w)
#pragma unroll
                for (int i = 0; i < V; ++i) acc[i] += part[w][lane * V + i];
    }
    if (wave) return;
    Run<TO, V> y;
#pragma unroll
    for (int i = 0; i < V; ++i) y.v[i] = from_float<TO>(base ? to_float(there.v[i]) + acc[i] * a.scale : acc[i] * a.scale);
    if (n == V) store_run<TO, V>(out + at, y);
    else
#pragma unroll
        for (uint32_t i = 0; i < V; ++i)
            if (i < n) out[at + i] = y.v[i];
}

int sort_passes(size_t rows)
{
    int bits = 1;
    while (((size_t)1 << bits) <= rows) ++bits;  // rows itself stands for none
    return (bits + kDigitBits - 1) / kDigitBits;
}
uint32_t lanes_for(uint32_t width, uint32_t v)
{
    uint32_t lanes = 1;
    while (lanes < 256 && lanes * v < width) lanes <<= 1;
    return lanes;
}
// values a lane has of a row: 16 bytes of the wider of the two types, so that a wave's accesses to either are whole lines
// (16-bit rows into 32 bits: 5 TB/s; with 8 values, 3.2)
constexpr int values_of(size_t in_bytes, size_t out_bytes) { return in_bytes == 4 || out_bytes == 4 ? 4 : 8; }

struct GradientPlan {
    uint32_t blocks, stretch, stretches;
    int passes;
    size_t a, b, counts, groups, partial, total;
};
GradientPlan gradient_plan(size_t rows, uint32_t width, size_t count)
{
    GradientPlan p{};
    p.passes = sort_passes(rows);
    p.blocks = (uint32_t)((count + kSortBlock - 1) / kSortBlock);
    const size_t slabs = (width + 255u) / 256u;
    p.stretch = 16;
    while (count * slabs / p.stretch > 8192) p.stretch *= 2;
    p.stretches = (uint32_t)((count + p.stretch - 1) / p.stretch);
    size_t off = 0;
    p.a = off;       off = align256(off + count * 8);
    p.b = off;       off = align256(off + count * 8);
    p.counts = off;  off = align256(off + (size_t)p.passes * p.blocks * kDigits * 4);
    p.groups = off;  off = align256(off + (p.blocks > kManyBlocks ? (size_t)(p.blocks + kGroupBlocks - 1) / kGroupBlocks * kDigits * 4 : 0));
    p.partial = off; off = align256(off + (size_t)p.stretches * 2 * width * 4);
    p.total = off;
    return p;
}

}  // namespace

hipError_t launch_embedding(const EmbeddingArgs& a, hipStream_t s)
{
    return with_type(a.source_type, [&](auto ti) {
        return with_type(a.out_type, [&](auto to) {
            using TI = decltype(ti);
            using TO = decltype(to);
            constexpr int V = sizeof(TI) + sizeof(TO) == 8 ? 4 : 8;
            const uint32_t lanes = lanes_for(a.width, V), per = 256u / lanes;
            const dim3 grid((uint32_t)std::min<size_t>((a.ntokens + per - 1) / per, 1u << 20));
            if (a.width % V == 0) FFTSP_LAUNCH("embedding", (k_embedding<TI, TO, V, true>), grid, dim3(256), 0, s, a, lanes);
            else FFTSP_LAUNCH("embedding", (k_embedding<TI, TO, V, false>), grid, dim3(256), 0, s, a, lanes);
            return hipGetLastError();
        });
    });
}

size_t embedding_gradient_workspace(size_t rows, uint32_t width, size_t ntokens)
{
    return gradient_plan(rows, width, ntokens).total;
}

hipError_t launch_embedding_gradient(const EmbeddingArgs& a, uint8_t* ws, hipStream_t s)
{
    FillArgs f{};
    if (a.base != a.out) {
        const bool flat = a.out_stride == a.width;
        f.bytes = type_bytes(a.out_type);
        f.base = static_cast<const uint8_t*>(a.base);
        f.out = static_cast<uint8_t*>(a.out);
        f.row_values = flat ? (uint64_t)a.rows * a.width : a.width;
        f.stride = a.out_stride;
        f.per_row = (f.row_values * f.bytes + 15) / 16;
        f.chunks = f.per_row * (flat ? 1 : a.rows);
    }
    auto fillers = [](uint64_t chunks, uint32_t threads) { return (uint32_t)std::min<uint64_t>((chunks + threads - 1) / threads, kMostFillers); };
    if (a.ntokens == 0) {
        if (f.chunks) FFTSP_LAUNCH("embedding_fill", k_fill, dim3(fillers(f.chunks, 256)), dim3(256), 0, s, f);
        return hipGetLastError();
    }
    const uint32_t in_values = values_of(type_bytes(a.source_type), type_bytes(a.out_type)), few_slabs = (a.width + 64u * in_values - 1u) / (64u * in_values);
    if (a.ntokens <= kFew && a.ntokens * few_slabs <= kFewGroups) {
        // small tables are filled beside the sums, larger ones by a launch before, which writes at the memory's rate
        const bool beside = a.rows <= kFewRows && f.chunks * 16 <= kFewBytes;
        if (f.chunks && !beside) FFTSP_LAUNCH("embedding_fill", k_fill, dim3(fillers(f.chunks, 256)), dim3(256), 0, s, f);
        return with_type(a.source_type, [&](auto ti) {
            return with_type(a.out_type, [&](auto to) {
                using TI = decltype(ti);
                using TO = decltype(to);
                constexpr int V = values_of(sizeof(TI), sizeof(TO));
                FewArgs w{a, few_slabs, 0, lanes_for(a.width, 16 / sizeof(TO))};
                uint32_t lds = 0;
                if (f.chunks && beside) {
                    const uint64_t per = 256u / w.lanes;
                    w.fillers = (uint32_t)std::min<uint64_t>((a.rows + per - 1) / per, 1024);
                    lds = (uint32_t)(a.rows + 31) / 32 * 4;
                }
                FFTSP_LAUNCH("embedding_few", (k_gradient_few<TI, TO, V>), dim3((uint32_t)a.ntokens * few_slabs + w.fillers), dim3(256), lds, s, w);
                return hipGetLastError();
            });
        });
    }
    const GradientPlan p = gradient_plan(a.rows, a.width, a.ntokens);
    SortArgs so{a.tokens, a.token_bits, (uint32_t)a.rows, (uint32_t)a.ntokens, p.blocks, reinterpret_cast<uint2*>(ws + p.a),
                reinterpret_cast<uint2*>(ws + p.b), reinterpret_cast<uint32_t*>(ws + p.counts),
                p.blocks > kManyBlocks ? reinterpret_cast<uint32_t*>(ws + p.groups) : nullptr, p.passes, f};
    const bool one = so.count <= kSortOne;
    if (one) {
        FFTSP_LAUNCH("embedding_sort_one", k_sort_one, dim3(1 + fillers(f.chunks, kOneThreads)), dim3(kOneThreads), 0, s, so);
    } else {
        const dim3 grid(p.blocks + fillers((f.chunks + p.passes) / (p.passes + 1), kSortThreads));
        FFTSP_LAUNCH("embedding_sort_count", k_sort_count, grid, dim3(kSortThreads), 0, s, so);
        for (int i = 0; i < p.passes; ++i) {
            if (so.groups) FFTSP_LAUNCH("embedding_sort_groups", k_sort_groups, dim3((p.blocks + kGroupBlocks - 1) / kGroupBlocks), dim3(kSortThreads), 0, s, so, i);
            FFTSP_LAUNCH("embedding_sort", k_sort_scatter, grid, dim3(kSortThreads), 0, s, so, i);
        }
    }
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    SumArgs m{};
    m.sorted = !one && p.passes & 1 ? so.b : so.a;
    m.count = so.count;
    m.stretch = p.stretch;
    m.stretches = p.stretches;
    m.rows = so.rows;
    m.width = a.width;
    m.source = a.source;
    m.out = a.out;
    m.source_stride = a.source_stride;
    m.out_stride = a.out_stride;
    m.scale = a.scale;
    m.add = a.base != nullptr;
    m.partial = reinterpret_cast<float*>(ws + p.partial);
    return with_type(a.source_type, [&](auto ti) {
        return with_type(a.out_type, [&](auto to) {
            using TI = decltype(ti);
            using TO = decltype(to);
            constexpr int V = values_of(sizeof(TI), sizeof(TO));
            const uint32_t slabs = (a.width + 64u * V - 1u) / (64u * V);
            const uint64_t waves = (uint64_t)p.stretches * slabs;
            const dim3 grid((uint32_t)((waves + 3) / 4));
            if (m.add) FFTSP_LAUNCH("embedding_sum", (k_sum_stretches<TI, TO, V, true>), grid, dim3(256), 0, s, m, slabs);
            else FFTSP_LAUNCH("embedding_sum", (k_sum_stretches<TI, TO, V, false>), grid, dim3(256), 0, s, m, slabs);
            if (p.stretches > 1) FFTSP_LAUNCH("embedding_join", (k_join_runs<TI, TO, V>), dim3(p.stretches, slabs), dim3(256), 0, s, m);
            return hipGetLastError();
        });
    });
}

}  // namespace fftsp
