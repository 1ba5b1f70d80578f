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

// ---- sorting the places by token: least significant digits first, stable ----
// A wave ranks 64 places at a time: the lanes with its own digit by one ballot per bit, the earlier groups' by a count.
constexpr int kDigitBits = 9, kDigits = 1 << kDigitBits;
constexpr int kSortThreads = 1024, kSortWaves = kSortThreads / 64;
constexpr uint32_t kSortBlock = 4096;  // places a workgroup has

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

struct SortArgs {
    const void* tokens;
    int token_bits;
    uint32_t rows, count, blocks;
    uint2* a;            // (token, place)
    uint2* b;
    uint32_t* counts;    // [passes][blocks][kDigits]
    int passes;
};

// counts of the first digit, block by block; clears the later passes' counts
__global__ void __launch_bounds__(kSortThreads) k_sort_count(SortArgs s)
{
    __shared__ uint32_t hist[kDigits];
    for (uint32_t i = threadIdx.x; i < kDigits; i += kSortThreads) hist[i] = 0;
    __syncthreads();
    const uint32_t at = blockIdx.x * kSortBlock;
    for (uint32_t i = threadIdx.x; i < kSortBlock; i += kSortThreads)
        if (at + i < s.count) atomicAdd(&hist[token_row(s.tokens, s.token_bits, at + i, s.rows) & (kDigits - 1u)], 1u);
    __syncthreads();
    for (uint32_t i = threadIdx.x; i < kDigits; i += kSortThreads) {
        s.counts[(size_t)blockIdx.x * kDigits + i] = hist[i];
        for (int p = 1; p < s.passes; ++p) s.counts[((size_t)p * s.blocks + blockIdx.x) * kDigits + i] = 0;
    }
}

// one pass: every workgroup finds where its digits begin from all blocks' counts, and counts the next pass's digits by the
// block that its places go to
__global__ void __launch_bounds__(kSortThreads) k_sort_scatter(SortArgs s, int pass)
{
    __shared__ uint32_t wave_count[kSortWaves][kDigits];
    __shared__ uint32_t base[kDigits];
    __shared__ uint32_t scan[kDigits];
    const uint32_t tid = threadIdx.x, wave = tid >> 6, lane = tid & 63u;
    const uint2* from = pass & 1 ? s.b : s.a;
    uint2* to = pass & 1 ? s.a : s.b;
    const uint32_t* counts = s.counts + (size_t)pass * s.blocks * kDigits;
    uint32_t* next = pass + 1 < s.passes ? s.counts + (size_t)(pass + 1) * s.blocks * kDigits : nullptr;
    for (uint32_t i = tid; i < kSortWaves * kDigits; i += kSortThreads) (&wave_count[0][0])[i] = 0;
    uint32_t before = 0, total = 0;
    if (tid < kDigits)
        for (uint32_t b = 0; b < s.blocks; ++b) {
            const uint32_t c = counts[(size_t)b * kDigits + tid];
            if (b < blockIdx.x) before += c;
            total += c;
        }
    if (tid < kDigits) scan[tid] = total;
    __syncthreads();
    for (uint32_t d = 1; d < kDigits; d <<= 1) {  // inclusive sums
        const uint32_t v = tid < kDigits && tid >= d ? scan[tid - d] : 0;
        __syncthreads();
        if (tid < kDigits) scan[tid] += v;
        __syncthreads();
    }
    if (tid < kDigits) base[tid] = scan[tid] - total + before;
    // a wave's share: consecutive groups of 64 places
    constexpr uint32_t kGroups = kSortBlock / kSortThreads;
    uint2 item[kGroups];
    uint32_t rank[kGroups];
    const int shift = pass * kDigitBits;
#pragma unroll
    for (uint32_t g = 0; g < kGroups; ++g) {
        const uint32_t i = blockIdx.x * kSortBlock + wave * (kGroups * 64) + g * 64 + lane;
        const bool present = i < s.count;
        item[g] = make_uint2(0xFFFFFFFFu, i);
        if (present) item[g] = pass ? from[i] : make_uint2(token_row(s.tokens, s.token_bits, i, s.rows), i);
        const uint32_t digit = (item[g].x >> shift) & (kDigits - 1u);
        const uint64_t same = same_digit(digit, present);
        uint32_t old = 0;
        if (present) {
            old = wave_count[wave][digit];
            rank[g] = old + (uint32_t)__popcll(same & ((1ull << lane) - 1ull));
        }
        // every lane has read before the first of each digit writes: a wave's LDS accesses are done in order, and the fences
        // keep the compiler to it
        __builtin_amdgcn_fence(__ATOMIC_SEQ_CST, "wavefront");
        __builtin_amdgcn_wave_barrier();
        if (present && (same & ((1ull << lane) - 1ull)) == 0) wave_count[wave][digit] = old + (uint32_t)__popcll(same);
        __builtin_amdgcn_fence(__ATOMIC_SEQ_CST, "wavefront");
        __builtin_amdgcn_wave_barrier();
    }
    __syncthreads();
    if (tid < kDigits) {
        uint32_t sum = base[tid];
        for (int w = 0; w < kSortWaves; ++w) {
            const uint32_t c = wave_count[w][tid];
            wave_count[w][tid] = sum;
            sum += c;
        }
    }
    __syncthreads();
#pragma unroll
    for (uint32_t g = 0; g < kGroups; ++g) {
        const uint32_t i = blockIdx.x * kSortBlock + wave * (kGroups * 64) + g * 64 + lane;
        if (i >= s.count) continue;
        const uint32_t at = wave_count[wave][(item[g].x >> shift) & (kDigits - 1u)] + rank[g];
        to[at] = item[g];
        if (next) atomicAdd(&next[(size_t)(at / kSortBlock) * kDigits + ((item[g].x >> (shift + kDigitBits)) & (kDigits - 1u))], 1u);
    }
}

// ---- rows that no token has: zeros, or the base's ----
template <typename T, int V>
__global__ void __launch_bounds__(256) k_fill_rows(const T* base, T* out, size_t rows, uint32_t width, size_t stride, uint32_t lanes)
{
    const uint32_t li = threadIdx.x & (lanes - 1u), per = 256u / lanes;
    for (size_t r = (size_t)blockIdx.x * per + threadIdx.x / lanes; r < rows; r += (size_t)gridDim.x * per)
        for (uint32_t c = li * V; c < width; c += lanes * V) {
            if (c + V <= width) {
                Run<T, V> x{};
                if (base) x = load_run<T, V>(base + r * stride + c);
                store_run<T, V>(out + r * stride + c, x);
            } else {
                for (uint32_t j = c; j < width; ++j) out[r * stride + j] = base ? base[r * stride + j] : from_float<T>(0.f);
            }
        }
}

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

template <typename TI, typename TO, int V>
__device__ __forceinline__ void write_row(const SumArgs& a, uint32_t row, uint32_t c, uint32_t n, const float* acc)
{
    TO* dst = static_cast<TO*>(a.out) + (size_t)row * a.out_stride + c;
    if (n == V) {
        Run<TO, V> y{};
        if (a.add) y = load_run<TO, V>(dst);
#pragma unroll
        for (int i = 0; i < V; ++i) y.v[i] = from_float<TO>(a.add ? to_float(y.v[i]) + acc[i] * a.scale : acc[i] * a.scale);
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
#pragma unroll
    for (uint32_t i = 0; i < V; ++i)
        if (i < n) dst[i] = acc[i];
}

template <typename TI, typename TO, int V>
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
    uint32_t run = a.sorted[first].x;                     // uniform: the run being summed
    bool head = first > 0 && a.sorted[first - 1].x == run;  // it began before this stretch
    for (uint32_t p = first; p < end; ++p) {
        const uint2 it = a.sorted[p];
        if (it.x != run) {
            if (run < a.rows) {
                if (head) write_partial<V>(a, stretch, 0, c, n, acc);
                else write_row<TI, TO, V>(a, run, c, n, acc);
            }
#pragma unroll
            for (int i = 0; i < V; ++i) acc[i] = 0.f;
            run = it.x;
            head = false;
        }
        if (run >= a.rows) return;                        // tokens outside the table are sorted last
        if (n == V) {
            const Run<TI, V> x = load_run<TI, V>(src + (size_t)it.y * a.source_stride);
#pragma unroll
            for (int i = 0; i < V; ++i) acc[i] += to_float(x.v[i]);
        } else {
#pragma unroll
            for (uint32_t i = 0; i < V; ++i)
                if (i < n) acc[i] += to_float(src[(size_t)it.y * a.source_stride + i]);
        }
    }
    if (run >= a.rows) return;
    const bool tail = end < a.count && a.sorted[end].x == run;  // it goes on behind this stretch
    if (head) write_partial<V>(a, stretch, 0, c, n, acc);
    else if (tail) write_partial<V>(a, stretch, 1, c, n, acc);
    else write_row<TI, TO, V>(a, run, c, n, acc);
}

// runs that cross stretches: a workgroup per stretch in which one begins and goes on, and per slab of 64 V columns
template <typename TI, typename TO, int V>
__global__ void __launch_bounds__(1024) k_join_runs(SumArgs a)
{
    __shared__ float part[16][64 * V];
    const uint32_t stretch = blockIdx.x, lane = threadIdx.x & 63u, wave = threadIdx.x >> 6;
    const uint32_t first = stretch * a.stretch, end = first + a.stretch;
    if (end >= a.count) return;
    const uint32_t run = a.sorted[end].x;
    if (run >= a.rows || a.sorted[end - 1].x != run) return;
    if (first > 0 && a.sorted[first].x == run && a.sorted[first - 1].x == run) return;  // it began earlier
    uint32_t last = stretch + 1;  // the last stretch that the run reaches
    while (last + 1 < a.stretches && a.sorted[(last + 1) * a.stretch].x == run) ++last;
    const uint32_t c = (blockIdx.y * 64u + lane) * V;
    const uint32_t n = c >= a.width ? 0u : min((uint32_t)V, a.width - c);
    float acc[V];
#pragma unroll
    for (int i = 0; i < V; ++i) acc[i] = 0.f;
    for (uint32_t s = stretch + wave; s <= last; s += 16u) {
        const float* p = a.partial + ((size_t)s * 2 + (s == stretch ? 1u : 0u)) * a.width + c;
#pragma unroll
        for (uint32_t i = 0; i < V; ++i)
            if (i < n) acc[i] += p[i];
    }
#pragma unroll
    for (int i = 0; i < V; ++i) part[wave][lane * V + i] = acc[i];
    __syncthreads();
    if (wave) return;
    for (int w = 1; w < 16; ++w)
#pragma unroll
        for (int i = 0; i < V; ++i) acc[i] += part[w][lane * V + i];
    write_row<TI, TO, V>(a, run, c, n, acc);
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
// values a lane has of a row of type bytes: 16 bytes
constexpr int values_of(size_t bytes) { return bytes == 4 ? 4 : 8; }

struct GradientPlan {
    uint32_t blocks, stretch, stretches;
    int passes;
    size_t a, b, counts, partial, total;
};
GradientPlan gradient_plan(size_t rows, uint32_t width, size_t count)
{
    GradientPlan p{};
    p.passes = sort_passes(rows);
    p.blocks = (uint32_t)((count + kSortBlock - 1) / kSortBlock);
    const size_t slabs = (width + 511u) / 512u;
    p.stretch = 8;
    while (count * slabs / p.stretch > 8192) p.stretch *= 2;
    p.stretches = (uint32_t)((count + p.stretch - 1) / p.stretch);
    size_t off = 0;
    p.a = off;       off = align256(off + count * 8);
    p.b = off;       off = align256(off + count * 8);
    p.counts = off;  off = align256(off + (size_t)p.passes * p.blocks * kDigits * 4);
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
    hipError_t e = hipSuccess;
    if (a.base != a.out) {
        e = with_type(a.out_type, [&](auto to) {
            using TO = decltype(to);
            constexpr int V = values_of(sizeof(TO));
            const uint32_t lanes = lanes_for(a.width, V), per = 256u / lanes;
            const dim3 grid((uint32_t)std::min<size_t>((a.rows + per - 1) / per, 4096));
            FFTSP_LAUNCH("embedding_fill", (k_fill_rows<TO, V>), grid, dim3(256), 0, s, static_cast<const TO*>(a.base),
                         static_cast<TO*>(a.out), a.rows, a.width, a.out_stride, lanes);
            return hipGetLastError();
        });
        if (e != hipSuccess) return e;
    }
    if (a.ntokens == 0) return hipSuccess;
    const GradientPlan p = gradient_plan(a.rows, a.width, a.ntokens);
    SortArgs so{a.tokens, a.token_bits, (uint32_t)a.rows, (uint32_t)a.ntokens, p.blocks, reinterpret_cast<uint2*>(ws + p.a),
                reinterpret_cast<uint2*>(ws + p.b), reinterpret_cast<uint32_t*>(ws + p.counts), p.passes};
    FFTSP_LAUNCH("embedding_sort_count", k_sort_count, dim3(p.blocks), dim3(kSortThreads), 0, s, so);
    for (int i = 0; i < p.passes; ++i)
        FFTSP_LAUNCH("embedding_sort", k_sort_scatter, dim3(p.blocks), dim3(kSortThreads), 0, s, so, i);
    e = hipGetLastError();
    if (e != hipSuccess) return e;
    SumArgs m{};
    m.sorted = p.passes & 1 ? so.b : so.a;
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
            constexpr int V = values_of(sizeof(TI));
            const uint32_t slabs = (a.width + 64u * V - 1u) / (64u * V);
            const uint64_t waves = (uint64_t)p.stretches * slabs;
            FFTSP_LAUNCH("embedding_sum", (k_sum_stretches<TI, TO, V>), dim3((uint32_t)((waves + 3) / 4)), dim3(256), 0, s, m, slabs);
            if (p.stretches > 1)
                FFTSP_LAUNCH("embedding_join", (k_join_runs<TI, TO, V>), dim3(p.stretches, slabs), dim3(1024), 0, s, m);
            return hipGetLastError();
        });
    });
}

}  // namespace fftsp
