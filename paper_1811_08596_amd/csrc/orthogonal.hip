// Newton-Schulz orthogonalisation of a list of matrices, and the momentum step round it.
//
//   X = U / (|U|_F + eps), n x m with n <= m;   per step  A = X X^T,  P = a I + b A + c A A,  X <- P X;   out = gain X
//
// The products carry the time.  All matrices of a phase of a few steps are polynomials of the phase's first A, so
// they commute, and the steps can be taken on n x n matrices alone: Q <- P Q, A <- P A P, and X <- Q X at the phase's end.
// That is n^2 m for A and 2 n^2 m for Q X once a phase instead of once a step, and four symmetric n x n products (n^3
// each: only tiles on and under the diagonal are computed, and written twice) a step instead of one.  A has an absolute error
// of 2^-24 of its largest eigenvalue, which the small eigenvalues' growth by a^2 a step turns into a relative one: 1e-6 after
// two steps, 3.4445^4 2^-24 = 1e-5 after three, 1e-3 after five.  So a phase has up to two steps where the result is stored in
// 32 bits, up to three where it is rounded to 16.
//
// Products run on binary16 matrix instructions whose inputs carry a binary32 number in two planes: 2^e v = hi + lo, each
// rounded to nearest (v is then 2^-24 v off, or 2^-(25 + e) where v is small), and x y = hi hi + hi lo + lo hi summed in
// binary32; the part left out is under 2^-24 |x| |y|.  Three instructions at sixteen times the binary32 one's rate.  e is up to
// 14 and follows from the coefficients: they bound the singular values of every matrix of the iteration.
//
// Layout: an operand is kept as the instruction reads it, in fragments of 32 rows x 16 columns (of the contracted index),
// 64 lanes x 8 values of hi and then of lo: 2 KB, so that every access from memory to a wave is 1 KB in one piece, goes
// straight into LDS and is read from there without conflicts.  Fragments along the contracted index follow each other.
// X is kept twice, by rows (for X X^T) and by columns (for Q X).  Rows and columns are padded with zeros to whole tiles;
// products of them are zero again, so no kernel asks where a matrix ends but those that read the input or write the output.
#include "layers.h"

#include <algorithm>
#include <atomic>
#include <cmath>
#include <vector>

namespace fftsp {
namespace {

typedef _Float16 half8 __attribute__((ext_vector_type(8)));
typedef _Float16 half4 __attribute__((ext_vector_type(4)));
typedef float float16v __attribute__((ext_vector_type(16)));

constexpr uint32_t kFragBytes = 2048;                   // hi and lo of 32 x 16
constexpr uint32_t kLeastSteps = 8, kMostSlices = 64;   // of a tile: steps that are worth a workgroup of their own; workgroups
constexpr uint32_t kMostParts = 1024;                   // workgroups that sum a matrix's squares

// n x n matrices of the iteration
enum Square { kA, kP, kT, kQ0, kQ1, kSquares };

// Launches of products by what they contract: X X^T, one or two products of n x n by n x n, and n x n by X.
enum Class { kGrams, kSingles, kPairs, kWides, kClasses };
// What the workgroups of a launch do: how many the matrices before each have, by kind of launch.
enum Kind { kNorm, kConvert, kChain, kProducts, kKinds = kProducts + kClasses };

// A matrix as the kernels see it.  Offsets are bytes from the workspace's start.
struct Item {
    uint64_t at, stride;        // first element and distance of rows in the caller's arrays
    uint64_t x[2], xt[2];       // X by rows and by columns, before and after a phase
    uint64_t square, square_bytes;
    uint32_t rows, cols, n, m;  // n = min, m = max
    uint32_t nf, mf;            // fragments along n and along m that there is room for
    uint32_t parts;             // workgroups that sum its squares
    float gain;
    uint32_t chain;             // 1: one workgroup does its phase, 2: X X^T, too
    uint32_t pad;
};
__device__ __forceinline__ bool tall(const Item& it) { return it.rows > it.cols; }
__device__ __forceinline__ uint64_t by_rows(const Item& it, int phase) { return phase & 1 ? it.x[1] : it.x[0]; }
__device__ __forceinline__ uint64_t by_columns(const Item& it, int phase) { return phase & 1 ? it.xt[1] : it.xt[0]; }

constexpr int kItemsPerLaunch = 24;
static_assert(kItemsPerLaunch <= 64, "a lane each");
struct ItemTable {
    Item item[kItemsPerLaunch];
    uint32_t start[kItemsPerLaunch][kKinds];
    uint32_t first, count, total;
};

// starts: [kKinds][matrices]
__device__ __forceinline__ void put_items(const ItemTable& t, Item* items, uint32_t* starts)
{
    const uint32_t i = threadIdx.x;
    if (i < t.count) {
        items[t.first + i] = t.item[i];
        for (int k = 0; k < kKinds; ++k) starts[(size_t)k * t.total + t.first + i] = t.start[i][k];
    }
}
__global__ void k_items(ItemTable t, Item* items, uint32_t* starts) { put_items(t, items, starts); }

// the last matrix whose first workgroup is not behind `wg`, and how far behind it wg is
__device__ __forceinline__ uint32_t find_item(const uint32_t* starts, uint32_t count, uint32_t wg, uint32_t* within)
{
    const uint32_t lane = threadIdx.x & 63u;
    uint32_t found = 0, begin = 0;
    for (uint32_t base = 0; base < count; base += 64) {
        const uint32_t v = base + lane < count ? starts[base + lane] : 0xFFFFFFFFu;
        const uint64_t m = __ballot(v <= wg);
        if (m == 0) break;
        const int top = 63 - __builtin_clzll(m);
        found = base + (uint32_t)top;
        begin = (uint32_t)__builtin_amdgcn_readlane((int)v, top);
        if (top < 63) break;
    }
    *within = wg - begin;
    return (uint32_t)__builtin_amdgcn_readfirstlane((int)found);
}

__device__ __forceinline__ float load_value(const void* p, int type, uint64_t i)
{
    if (type == 0) return static_cast<const float*>(p)[i];
    if (type == 1) return to_float(static_cast<const Bf16*>(p)[i]);
    return to_float(static_cast<const F16*>(p)[i]);
}
// up to four values behind each other
template <typename T>
__device__ __forceinline__ void load_some(const T* p, uint32_t n, float* v)
{
    if (n == 4) {
        const Run<T, 4> r = load_run<T, 4>(p);
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = to_float(r.v[e]);
    } else {
#pragma unroll
        for (uint32_t e = 0; e < 4; ++e) v[e] = e < n ? to_float(p[e]) : 0.f;
    }
}
template <typename T>
__device__ __forceinline__ void store_some(T* p, uint32_t n, const float* v)
{
    if (n == 4) {
        Run<T, 4> r;
#pragma unroll
        for (int e = 0; e < 4; ++e) r.v[e] = from_float<T>(v[e]);
        store_run<T, 4>(p, r);
    } else {
#pragma unroll
        for (uint32_t e = 0; e < 4; ++e)
            if (e < n) p[e] = from_float<T>(v[e]);
    }
}
struct Common {
    const void* in;
    const float* momentum;
    float* momentum_out;
    const void* weights;
    void* out;
    int in_type, out_type, nesterov, step;
    float beta, lr, decay, eps, lift;  // lift: X's planes hold so many times X before the first phase
    uint8_t* ws;
    const Item* items;
    const uint32_t* starts;  // [kKinds][count]
    double* sums;            // [norm workgroups]
    uint8_t* partial;        // parts of tiles that several workgroups share, by workgroup
    uint32_t* arrivals;      // of workgroups at such a tile, by the first one's number; zero between launches
    uint32_t count, most;    // matrices; entries of arrivals
};

// ---- momentum and |U|_F^2 ----
// A workgroup has pieces of kPiece values of a row, or of the whole matrix where its rows follow each other, in turn.
constexpr uint32_t kPiece = 1024;
template <typename T, bool STEP>
__device__ __forceinline__ double norm_part(const Common& c, const Item& it, uint32_t part)
{
    const bool flat = it.stride == it.cols;
    const uint64_t rows = flat ? 1 : it.rows, cols = flat ? (uint64_t)it.rows * it.cols : it.cols;
    const uint32_t across = (uint32_t)((cols + kPiece - 1) / kPiece);
    const uint64_t pieces = rows * across;
    double s = 0.0;
    for (uint64_t p = part; p < pieces; p += it.parts) {
        const uint64_t row = flat ? 0 : p / across, first = (p - row * across) * kPiece + threadIdx.x * 4u;
        if (first >= cols) continue;
        const uint64_t at = it.at + row * it.stride + first;
        const uint32_t n = (uint32_t)min((uint64_t)4, cols - first);
        float u[4];
        load_some<T>(static_cast<const T*>(c.in) + at, n, u);
        if (STEP) {
            float m[4];
            load_some<float>(c.momentum + at, n, m);
#pragma unroll
            for (int e = 0; e < 4; ++e) m[e] = fmaf(c.beta, m[e], u[e]);
            store_some<float>(c.momentum_out + at, n, m);
#pragma unroll
            for (int e = 0; e < 4; ++e) u[e] = c.nesterov ? fmaf(c.beta, m[e], u[e]) : m[e];
        }
#pragma unroll
        for (uint32_t e = 0; e < 4; ++e)
            if (e < n) s += (double)u[e] * (double)u[e];
    }
    return s;
}
template <typename T>
__device__ __forceinline__ double norm_of_type(const Common& c, const Item& it, uint32_t part)
{
    return c.step ? norm_part<T, true>(c, it, part) : norm_part<T, false>(c, it, part);
}
// ARGUMENTS: the whole list is in the launch's arguments, and the first workgroup writes it down for the later launches
template <bool ARGUMENTS>
struct NormTable {
};
template <>
struct NormTable<true> {
    ItemTable t;
};
template <bool ARGUMENTS>
__global__ void __launch_bounds__(256) k_norm(Common c, NormTable<ARGUMENTS> table)
{
    __shared__ double sums[4];
    uint32_t part, id = 0;
    if constexpr (ARGUMENTS) {
        if (blockIdx.x == 0) put_items(table.t, const_cast<Item*>(c.items), const_cast<uint32_t*>(c.starts));
        const uint32_t lane = threadIdx.x & 63u, v = lane < c.count ? table.t.start[lane][kNorm] : 0xFFFFFFFFu;
        id = 63u - (uint32_t)__builtin_clzll(__ballot(v <= blockIdx.x));
        part = blockIdx.x - (uint32_t)__builtin_amdgcn_readlane((int)v, (int)id);
    } else {
        id = find_item(c.starts + (size_t)kNorm * c.count, c.count, blockIdx.x, &part);
    }
    Item it;
    if constexpr (ARGUMENTS) it = table.t.item[id];
    else it = c.items[id];
    for (uint32_t i = blockIdx.x * 256u + threadIdx.x; i < c.most; i += gridDim.x * 256u) c.arrivals[i] = 0;
    double s = c.in_type == 0 ? norm_of_type<float>(c, it, part) : c.in_type == 1 ? norm_of_type<Bf16>(c, it, part) : norm_of_type<F16>(c, it, part);
    for (int d = 32; d; d >>= 1) s += __shfl_xor(s, d);
    if ((threadIdx.x & 63u) == 0) sums[threadIdx.x >> 6] = s;
    __syncthreads();
    if (threadIdx.x == 0) c.sums[blockIdx.x] = (sums[0] + sums[1]) + (sums[2] + sums[3]);
}

__device__ __forceinline__ void split(float v, _Float16* hi, _Float16* lo)
{
    *hi = (_Float16)v;
    *lo = (_Float16)(v - (float)*hi);
}

// ---- U / (|U|_F + eps) as fragments, by rows and by columns: a workgroup per 64 x 64 values ----
// A thread's values: four of rows tid / 16 + 16 q of the caller's array, which are on their way while the norm is added up
template <typename T>
__device__ __forceinline__ void convert_load(const Common& c, const Item& it, uint32_t row, uint32_t col, float (&v)[4][4])
{
    float m[4][4];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        const uint32_t r = row + 16u * q, n = r < it.rows && col < it.cols ? min(4u, it.cols - col) : 0u;
        const uint64_t at = it.at + (uint64_t)r * it.stride + col;
#pragma unroll
        for (int e = 0; e < 4; ++e) v[q][e] = m[q][e] = 0.f;
        if (n) load_some<T>(static_cast<const T*>(c.in) + at, n, v[q]);
        if (n && c.step) load_some<float>(c.momentum_out + at, n, m[q]);
    }
    if (c.step)
#pragma unroll
        for (int q = 0; q < 4; ++q)
#pragma unroll
            for (int e = 0; e < 4; ++e) v[q][e] = c.nesterov ? fmaf(c.beta, m[q][e], v[q][e]) : m[q][e];
}
__global__ void __launch_bounds__(256) k_convert(Common c)
{
    __shared__ float tile[64][65];
    __shared__ double sums[4];
    uint32_t at;
    const uint32_t id = find_item(c.starts + (size_t)kConvert * c.count, c.count, blockIdx.x, &at);
    const Item it = c.items[id];
    const uint32_t first_part = c.starts[(size_t)kNorm * c.count + id];
    const uint32_t tid = threadIdx.x, lane = tid & 63u, wave = tid >> 6;
    // tile (tn, tm) of the iteration's n x m matrix
    const uint32_t across = (it.m + 63u) / 64u, tn = at / across, tm = at - tn * across;
    const bool t = tall(it);
    const uint32_t slow = tid >> 4, fast = (tid & 15u) * 4u;
    const uint32_t row = (t ? tm : tn) * 64u + slow, col = (t ? tn : tm) * 64u + fast;
    float v[4][4];
    if (c.in_type == 0) convert_load<float>(c, it, row, col, v);
    else if (c.in_type == 1) convert_load<Bf16>(c, it, row, col, v);
    else convert_load<F16>(c, it, row, col, v);
    double s = 0.0;
    for (uint32_t i = tid; i < it.parts; i += 256) s += c.sums[first_part + i];
    for (int d = 32; d; d >>= 1) s += __shfl_xor(s, d);
    if (lane == 0) sums[wave] = s;
    __syncthreads();
    const double norm = sqrt((sums[0] + sums[1]) + (sums[2] + sums[3])) + (double)c.eps;
    const double factor = norm > 0.0 ? (double)c.lift / norm : 0.0;
#pragma unroll
    for (int q = 0; q < 4; ++q)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const uint32_t r = slow + 16u * q, k = fast + e;
            tile[t ? k : r][t ? r : k] = (float)((double)v[q][e] * factor);
        }
    __syncthreads();
    // 2 x 4 fragments of each kind, two of each to a wave
    for (uint32_t f = wave; f < 16; f += 4) {
        const bool turned = f >= 8;
        const uint32_t rb = (f >> 2) & 1u, kb = f & 3u;
        half8 hi, lo;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const uint32_t r = rb * 32 + (lane & 31u), k = kb * 16 + (lane >> 5) * 8 + j;
            _Float16 h, l;
            split(turned ? tile[k][r] : tile[r][k], &h, &l);
            hi[j] = h;
            lo[j] = l;
        }
        const uint64_t row = (turned ? tm : tn) * 2u + rb, col = (turned ? tn : tm) * 4u + kb;
        const uint64_t per_row = turned ? it.nf : it.mf;
        uint8_t* dst = c.ws + (turned ? it.xt[0] : it.x[0]) + (row * per_row + col) * kFragBytes + lane * 16u;
        *reinterpret_cast<half8*>(dst) = hi;
        *reinterpret_cast<half8*>(dst + 1024) = lo;
    }
}

// ---- products C = L R^T of fragments ----
// A workgroup of WM x WN waves has a tile of 32 WM BM x 32 WN BN, a wave BM x BN blocks of 32 x 32.
// STAGES steps of 16 along the contracted index are in LDS or on their way there.
template <int WM_, int WN_, int BM_, int BN_, int STAGES_>
struct Shape {
    static constexpr int WM = WM_, WN = WN_, BM = BM_, BN = BN_, STAGES = STAGES_;
    static constexpr int kWaves = WM * WN, kThreads = kWaves * 64;
    static constexpr int kLeft = WM * BM, kRight = WN * BN;             // row blocks of a step
    static constexpr int kPieces = (kLeft + kRight) * 2 / kWaves;       // KB that a wave brings a step
    static constexpr uint32_t kTile = kLeft * 32;
    static constexpr uint32_t kStage = (kLeft + kRight) * kFragBytes;
    static constexpr uint32_t kTurn = 32 * 36 * 4;                      // a wave's part of LDS in the epilogue
    static constexpr uint32_t kLds = std::max(kStage * STAGES, kTurn * kWaves);
    static constexpr uint32_t kTileBytes = kTile * kTile * 4;
    static constexpr bool kSliced = kTile < 256;  // putting down and taking up parts of 256 KB costs more than it gains
    static_assert(kLeft == kRight && (kLeft + kRight) * 2 % kWaves == 0 && kPieces * (STAGES - 2) < 64 && STAGES >= 3, "");
};
using Least = Shape<2, 2, 1, 1, 8>;  // 64 x 64
using Small = Shape<2, 2, 2, 2, 5>;  // 128 x 128, two workgroups to a compute unit, which fill its LDS
using Large = Shape<2, 4, 4, 2, 4>;  // 256 x 256, one
constexpr int kSizes = 3;
constexpr uint32_t kTileOf[kSizes] = {Least::kTile, Small::kTile, Large::kTile}, kTileBytesOf[kSizes] = {Least::kTileBytes, Small::kTileBytes, Large::kTileBytes};
static_assert(Least::kSliced && Small::kSliced && !Large::kSliced, "the last size is not sliced");

template <int N>
__device__ __forceinline__ void arrived()  // all but the wave's last N pieces; then everybody's
{
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(N) : "memory");
}
// 1 KB from src into LDS, 16 bytes a lane
__device__ __forceinline__ void bring_piece(const uint8_t* src, uint32_t lane16, uint32_t lds)
{
    __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)(src + lane16), (__attribute__((address_space(3))) void*)(uintptr_t)lds, 16, 0, 0);
}

template <typename S>
struct Accumulators {
    float16v v[S::BM][S::BN];
};

// acc += sum over `steps` steps; left and right: fragments of the first row block and step, row_bytes to the next row block's.
// A wave's fragments of a step are read from LDS while the step before is multiplied, and those reads and the next pieces from
// memory are issued between the products, two products apart: behind the barrier they would hold up all waves at once (at
// 4096 x 4096 x 4096 in tiles of 256 a step of 1536 cycles of matrix instructions took 2095 that way and takes 1724, in tiles
// of 128 two workgroups' steps 1070 and now 806 of 768; the card then lowers its clock from 1.8 to 1.6 GHz, and 1.33 and 1.20
// PFLOP/s become 1.38 and 1.22).  idle: a wave above the diagonal of a symmetric result, which only helps to bring the pieces.
template <typename S>
__device__ __forceinline__ void multiply(Accumulators<S>& acc, uint8_t* lds, const uint8_t* left, const uint8_t* right, uint64_t left_row,
                                         uint64_t right_row, uint32_t steps, bool idle, uint32_t wave, uint32_t lane)
{
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t*)lds + wave * (S::kPieces * 1024u);
    const uint8_t* src[S::kPieces];
#pragma unroll
    for (int q = 0; q < S::kPieces; ++q) {
        const uint32_t p = wave * S::kPieces + q, rb = p >> 1;
        src[q] = (rb < S::kLeft ? left + rb * left_row : right + (rb - S::kLeft) * right_row) + (p & 1u) * 1024u;
    }
    auto bring = [&](int q, uint32_t slot) {
        bring_piece(src[q], lane * 16u, lds0 + slot * S::kStage + q * 1024u);
        src[q] += kFragBytes;
    };
    for (uint32_t s = 0; s + 1 < S::STAGES && s < steps; ++s)
#pragma unroll
        for (int q = 0; q < S::kPieces; ++q) bring(q, s);
    const uint32_t wi = (wave % S::WM) * S::BM, wj = (wave / S::WM) * S::BN;
    constexpr int kReads = 2 * (S::BM + S::BN), kGroups = 3 * S::BM, kAside = S::kPieces + kReads;
    // fragments of the wave's right blocks, then of its left ones, hi and lo
    auto read = [&](half8 (&f)[kReads], uint32_t slot, int q) {
        const uint32_t rb = q / 2 < S::BN ? S::kLeft + wj + q / 2 : wi + q / 2 - S::BN;
        f[q] = *reinterpret_cast<const half8*>(lds + slot * S::kStage + rb * kFragBytes + (q & 1) * 1024u + lane * 16u);
    };
    uint32_t slot = 0, next = S::STAGES - 1;
    auto step = [&](uint32_t k, half8 (&now)[kReads], half8 (&then)[kReads]) {
        // step k + 1 has to be there; steps k + 2 .. k + STAGES - 2 may still be on their way
        if (k + S::STAGES - 1 <= steps) arrived<(S::STAGES - 3) * S::kPieces>();
        else arrived<0>();
        const bool more = k + S::STAGES - 1 < steps;
        slot = slot + 1 == S::STAGES ? 0 : slot + 1;
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int g = 0; g < kGroups; ++g) {
            const int t = g / S::BM, i = g % S::BM;  // hi lo, lo hi, hi hi
#pragma unroll
            for (int j = 0; j < S::BN; ++j)
                acc.v[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(now[2 * (S::BN + i) + (t == 1)], now[2 * j + (t == 0)], acc.v[i][j], 0, 0, 0);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int q = g * kAside / kGroups; q < (g + 1) * kAside / kGroups; ++q) {
                const int piece = q * S::kPieces / kAside;  // pieces evenly among the reads
                if ((q + 1) * S::kPieces / kAside > piece) {
                    if (more) bring(piece, next);
                } else {
                    read(then, slot, q - piece);
                }
            }
            __builtin_amdgcn_sched_barrier(0);
        }
        next = next + 1 == S::STAGES ? 0 : next + 1;
    };
    if (S::STAGES - 1 <= steps) arrived<(S::STAGES - 2) * S::kPieces>();
    else arrived<0>();
    if (idle) {  // as many barriers as the others have
        for (uint32_t k = 0; k < steps; ++k) {
            if (k + S::STAGES - 1 <= steps) arrived<(S::STAGES - 3) * S::kPieces>();
            else arrived<0>();
            if (k + S::STAGES - 1 < steps)
#pragma unroll
                for (int q = 0; q < S::kPieces; ++q) bring(q, next);
            next = next + 1 == S::STAGES ? 0 : next + 1;
        }
        arrived<0>();
        return;
    }
    half8 f[2][kReads];
#pragma unroll
    for (int q = 0; q < kReads; ++q) read(f[0], 0, q);
    uint32_t k = 0;
    for (; k + 2 <= steps; k += 2) {
        step(k, f[0], f[1]);
        step(k + 1, f[1], f[0]);
    }
    if (k < steps) step(k, f[0], f[1]);
    arrived<0>();  // LDS is free again
}

enum Product { kGram, kPoly, kTimes, kApply, kLast };
__host__ __device__ constexpr bool symmetric(int what) { return what == kGram || what == kPoly || what == kTimes; }

struct ProductArgs {
    Common c;
    float scale[2];              // of the sums, to what the result's planes hold
    float ca, cb;                // kPoly: and ca on the diagonal, cb times A's planes
    int left[2], right[2], out[2];  // Square; a launch of kTimes has one or two products
    int products;
    int phase;                   // X is x[phase & 1]
    int cls;
    uint32_t len;                // steps that a workgroup has at most
    int local;                   // neighbouring workgroups' operands fit an XCD's L2
};

// Of a tile on the diagonal: the wave's blocks are above it, or what is above the diagonal for them is left out
template <typename S>
__device__ __forceinline__ bool above(uint32_t wave) { return wave % S::WM < S::WM / 2 && wave / S::WM >= S::WN / 2; }
template <typename S>
__device__ __forceinline__ bool below(uint32_t wave) { return wave % S::WM >= S::WM / 2 && wave / S::WM < S::WN / 2; }

// The last product's tile to the caller's array, through LDS, so that lanes go along its rows.  The weights of the next blocks
// are on their way while these are written.
template <typename S, typename T>
__device__ __forceinline__ void finish_last(const ProductArgs& g, const Item& it, Accumulators<S>& acc, uint8_t* lds, uint32_t ti, uint32_t tj,
                                            uint32_t wave, uint32_t lane)
{
    const Common& c = g.c;
    const uint32_t wi = (wave % S::WM) * S::BM, wj = (wave / S::WM) * S::BN;
    const uint32_t col = lane & 31u, half = lane >> 5;
    float* turn = reinterpret_cast<float*>(lds + wave * S::kTurn);
    constexpr uint32_t kBlocks = S::kTile / 32u;  // of a tile's side
    const bool t = tall(it), step = c.step != 0;
    const float scale = it.gain * g.scale[0];
    const T* weights = static_cast<const T*>(c.weights);
    T* out = static_cast<T*>(c.out);
    // a lane's four values of row 8 q + lane / 8 of a block: the element, and how many of them there are
    auto place = [&](int i, int j, int q, uint64_t* el) {
        const uint32_t bi = ti * kBlocks + wi + i, bj = tj * kBlocks + wj + j;
        const uint32_t row = (t ? bj : bi) * 32u + q * 8u + (lane >> 3), first = (t ? bi : bj) * 32u + (lane & 7u) * 4u;
        *el = it.at + (uint64_t)row * it.stride + first;
        return row < it.rows && first < it.cols ? min(4u, it.cols - first) : 0u;
    };
    float w[2][S::BN][4][4];
    auto fetch = [&](float (&v)[S::BN][4][4], int i) {
#pragma unroll
        for (int j = 0; j < S::BN; ++j)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                uint64_t el;
                const uint32_t n = place(i, j, q, &el);
                if (n) load_some<T>(weights + el, n, v[j][q]);
            }
    };
    if (step) fetch(w[0], 0);
#pragma unroll
    for (int i = 0; i < S::BM; ++i) {
        if (step && i + 1 < S::BM) fetch(w[(i + 1) & 1], i + 1);
#pragma unroll
        for (int j = 0; j < S::BN; ++j) {
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                const uint32_t r = 8 * (e / 4) + 4 * half + e % 4;
                turn[t ? col * 36u + r : r * 36u + col] = acc.v[i][j][e] * scale;
            }
            __builtin_amdgcn_fence(__ATOMIC_SEQ_CST, "wavefront");
            __builtin_amdgcn_wave_barrier();
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                uint64_t el;
                const uint32_t n = place(i, j, q, &el);
                float v[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] = turn[(q * 8u + (lane >> 3)) * 36u + (lane & 7u) * 4u + e];
                if (n) {
                    if (step)
#pragma unroll
                        for (int e = 0; e < 4; ++e) v[e] = fmaf(-c.lr, v[e], c.decay * w[i & 1][j][q][e]);
                    store_some<T>(out + el, n, v);
                }
            }
            __builtin_amdgcn_fence(__ATOMIC_SEQ_CST, "wavefront");
            __builtin_amdgcn_wave_barrier();
        }
    }
}

// Any other product's tile to fragments, in both orientations.
// lane l has column l % 32 of a block and rows 8 (e / 4) + 4 (l / 32) + e % 4
template <typename S, int WHAT>
__device__ __forceinline__ void finish(const ProductArgs& g, const Item& it, int product, Accumulators<S>& acc, uint8_t* lds, uint32_t ti,
                                       uint32_t tj, uint32_t wave, uint32_t lane)
{
    const Common& c = g.c;
    if constexpr (WHAT == kLast) {
        if (c.out_type == 0) finish_last<S, float>(g, it, acc, lds, ti, tj, wave, lane);
        else if (c.out_type == 1) finish_last<S, Bf16>(g, it, acc, lds, ti, tj, wave, lane);
        else finish_last<S, F16>(g, it, acc, lds, ti, tj, wave, lane);
        return;
    }
    const uint32_t wi = (wave % S::WM) * S::BM, wj = (wave / S::WM) * S::BN;
    const uint32_t col = lane & 31u, half = lane >> 5;
    uint32_t* turn = reinterpret_cast<uint32_t*>(lds + wave * S::kTurn);
    constexpr uint32_t kBlocks = S::kTile / 32u;  // of a tile's side
    if (symmetric(WHAT) && ti == tj && above<S>(wave)) return;
    const int out = g.out[product];
    uint8_t* direct = c.ws + (symmetric(WHAT) ? it.square + out * it.square_bytes : by_columns(it, g.phase + 1));  // rows: C's columns
    uint8_t* turned = c.ws + (symmetric(WHAT) ? it.square + out * it.square_bytes : by_rows(it, g.phase + 1));
    const uint8_t* a = c.ws + it.square + kA * it.square_bytes;
    const uint32_t direct_row = it.nf, turned_row = symmetric(WHAT) ? it.nf : it.mf;
    // four values of a lane in the fragments whose rows are C's columns
    auto place = [&](int i, int j, int q) {
        const uint32_t bi = ti * kBlocks + wi + i, bj = tj * kBlocks + wj + j;
        return ((uint64_t)bj * direct_row + bi * 2u + q / 2) * kFragBytes + (col + 32u * (q & 1)) * 16u + half * 8u;
    };
    half4 ah[2][S::BN][4], al[2][S::BN][4];  // kPoly: A there, the next blocks' on their way while these are written
    auto fetch = [&](int b, int i) {
#pragma unroll
        for (int j = 0; j < S::BN; ++j)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const uint8_t* src = a + place(i, j, q);
                ah[b][j][q] = *reinterpret_cast<const half4*>(src);
                al[b][j][q] = *reinterpret_cast<const half4*>(src + 1024);
            }
    };
    if constexpr (WHAT == kPoly) fetch(0, 0);
#pragma unroll
    for (int i = 0; i < S::BM; ++i) {
        if constexpr (WHAT == kPoly)
            if (i + 1 < S::BM) fetch((i + 1) & 1, i + 1);
#pragma unroll
        for (int j = 0; j < S::BN; ++j) {
            const uint32_t bi = ti * kBlocks + wi + i, bj = tj * kBlocks + wj + j;
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                half4 hi, lo;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    float v = acc.v[i][j][q * 4 + e] * g.scale[product];
                    if constexpr (WHAT == kPoly) {
                        v = fmaf(g.cb, (float)ah[i & 1][j][q][e] + (float)al[i & 1][j][q][e], v);
                        if (bi == bj && col == 8u * q + 4u * half + e) v += g.ca;
                    }
                    _Float16 h, l;
                    split(v, &h, &l);
                    hi[e] = h;
                    lo[e] = l;
                    uint16_t hb, lb;
                    __builtin_memcpy(&hb, &h, 2);
                    __builtin_memcpy(&lb, &l, 2);
                    turn[(8 * q + 4 * half + e) * 36 + col] = (uint32_t)hb | (uint32_t)lb << 16;
                }
                uint8_t* dst = direct + place(i, j, q);
                *reinterpret_cast<half4*>(dst) = hi;
                *reinterpret_cast<half4*>(dst + 1024) = lo;
            }
            __builtin_amdgcn_fence(__ATOMIC_SEQ_CST, "wavefront");
            __builtin_amdgcn_wave_barrier();
            if (!symmetric(WHAT) || ti != tj || below<S>(wave)) {  // the other orientation, hi and lo of a value in one word
#pragma unroll
                for (int kb = 0; kb < 2; ++kb) {
                    uint32_t w[8];
#pragma unroll
                    for (int e = 0; e < 8; ++e) w[e] = turn[col * 36 + kb * 16 + half * 8 + e];
                    uint4 hi, lo;
                    uint32_t* ph = reinterpret_cast<uint32_t*>(&hi);
                    uint32_t* pl = reinterpret_cast<uint32_t*>(&lo);
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        ph[e] = (w[2 * e] & 0xFFFFu) | w[2 * e + 1] << 16;
                        pl[e] = w[2 * e] >> 16 | (w[2 * e + 1] & 0xFFFF0000u);
                    }
                    uint8_t* dst = turned + ((uint64_t)bi * turned_row + bj * 2u + kb) * kFragBytes + lane * 16u;
                    *reinterpret_cast<uint4*>(dst) = hi;
                    *reinterpret_cast<uint4*>(dst + 1024) = lo;
                }
            }
            __builtin_amdgcn_fence(__ATOMIC_SEQ_CST, "wavefront");
            __builtin_amdgcn_wave_barrier();
        }
    }
}

__device__ __forceinline__ uint32_t steps_of(const Item& it, int what) { return ((what == kGram ? it.m : it.n) + 15u) / 16u; }

// acc = the steps first .. first + steps - 1 of a tile
template <typename S, int WHAT>
__device__ __forceinline__ void multiply_tile(const ProductArgs& g, const Item& it, int product, uint32_t ti, uint32_t tj, uint32_t first,
                                              uint32_t steps, Accumulators<S>& acc, uint8_t* lds, uint32_t wave, uint32_t lane)
{
#pragma unroll
    for (int i = 0; i < S::BM; ++i)
#pragma unroll
        for (int j = 0; j < S::BN; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc.v[i][j][e] = 0.f;
    const Common& c = g.c;
    const uint64_t x = by_rows(it, g.phase), xt = by_columns(it, g.phase);
    const uint64_t row = (uint64_t)(WHAT == kGram ? it.mf : it.nf) * kFragBytes;  // bytes of a row block
    const uint64_t l = WHAT == kGram ? x : it.square + g.left[product] * it.square_bytes;
    const uint64_t r = WHAT == kGram ? x : WHAT == kApply || WHAT == kLast ? xt : it.square + g.right[product] * it.square_bytes;
    multiply<S>(acc, lds, c.ws + l + (uint64_t)ti * (S::kTile / 32u) * row + (uint64_t)first * kFragBytes,
                c.ws + r + (uint64_t)tj * (S::kTile / 32u) * row + (uint64_t)first * kFragBytes, row, row, steps,
                symmetric(WHAT) && ti == tj && above<S>(wave), wave, lane);
}

// Memory that workgroups of one launch hand over: device-scope accesses, which pass the caches that are not shared
__device__ __forceinline__ void put(uint64_t* p, float x, float y)
{
    __hip_atomic_store(p, (uint64_t)__float_as_uint(x) | (uint64_t)__float_as_uint(y) << 32, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ float2 take(const uint64_t* p)
{
    const uint64_t v = __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    return make_float2(__uint_as_float((uint32_t)v), __uint_as_float((uint32_t)(v >> 32)));
}

// A workgroup per tile, or per slice of a tile's steps where tiles have more than `len` of them.  Every workgroup of a sliced
// tile writes its part and counts its arrival, and the last to arrive adds the parts in the order of the steps, whoever that
// is.  Nobody waits.
template <typename S, int WHAT>
__global__ void __launch_bounds__(S::kThreads, 2) k_product(ProductArgs g)
{
    extern __shared__ __align__(1024) uint8_t lds[];
    const Common& c = g.c;
    const uint32_t lane = threadIdx.x & 63u, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    // Workgroups go round the eight XCDs.  32 tiles behind each other to each of them in turn where their operands, which they
    // have in common, fit its L2 (eight matrices of 1024 x 1024: 41 us a launch instead of 48); elsewhere all XCDs then read other
    // panels at a time (4096 x 9216: X X^T in 900 us instead of 620).
    uint32_t wg = blockIdx.x;
    if (g.local && (wg | 255u) < gridDim.x) wg = (wg & ~255u) + (wg & 7u) * 32u + (wg >> 3 & 31u);
    uint32_t at, ti, tj;
    const Item it = c.items[find_item(c.starts + (size_t)(kProducts + g.cls) * c.count, c.count, wg, &at)];
    const uint32_t per = steps_of(it, WHAT), slices = !S::kSliced || per <= g.len ? 1u : (per + g.len - 1) / g.len;
    const uint32_t nt = (it.n + S::kTile - 1) / S::kTile;
    uint32_t tiles = nt * (nt + 1) / 2;
    if (!symmetric(WHAT)) tiles = nt * ((it.m + S::kTile - 1) / S::kTile);
    int product = 0;
    if (WHAT == kTimes && at >= tiles * slices) {
        product = 1;
        at -= tiles * slices;
    }
    uint32_t slice = 0, tile = at, first = 0, steps = per;
    if (S::kSliced && slices > 1) {  // workgroups of one slice behind each other
        slice = at / tiles;
        tile = at - slice * tiles;
        first = per * slice / slices;  // per < 2^17, slices <= kMostSlices
        steps = per * (slice + 1) / slices - first;
    }
    if (symmetric(WHAT)) {  // row ti has ti + 1 tiles
        ti = (uint32_t)((sqrtf(8.f * (float)tile + 1.f) - 1.f) * 0.5f);
        while (ti * (ti + 1) / 2 > tile) --ti;
        while ((ti + 1) * (ti + 2) / 2 <= tile) ++ti;
        tj = tile - ti * (ti + 1) / 2;
    } else {
        tj = tile / nt;
        ti = tile - tj * nt;
    }
    ti = __builtin_amdgcn_readfirstlane(ti);
    tj = __builtin_amdgcn_readfirstlane(tj);
    Accumulators<S> acc;
    multiply_tile<S, WHAT>(g, it, product, ti, tj, first, steps, acc, lds, wave, lane);
    if (S::kSliced && slices > 1) {
        const uint32_t wg0 = wg - slice * tiles;
        auto part = [&](uint32_t s) { return reinterpret_cast<uint64_t*>(c.partial + (uint64_t)(wg0 + s * tiles) * S::kTileBytes) + threadIdx.x; };
        uint64_t* dst = part(slice);
#pragma unroll
        for (int i = 0; i < S::BM; ++i)
#pragma unroll
            for (int j = 0; j < S::BN; ++j)
#pragma unroll
                for (int q = 0; q < 8; ++q) put(dst + ((i * S::BN + j) * 8 + q) * S::kThreads, acc.v[i][j][2 * q], acc.v[i][j][2 * q + 1]);
        arrived<0>();  // every wave's stores are where all can see them
        uint32_t* count = c.arrivals + wg0;
        uint32_t* before = reinterpret_cast<uint32_t*>(lds);
        if (threadIdx.x == 0) *before = __hip_atomic_fetch_add(count, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        __syncthreads();
        if (__builtin_amdgcn_readfirstlane(*before) + 1 < slices) return;
        __syncthreads();  // LDS is free again
        if (threadIdx.x == 0) __hip_atomic_store(count, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        for (uint32_t s = 0; s < slices; ++s) {
            const uint64_t* src = part(s);
#pragma unroll
            for (int i = 0; i < S::BM; ++i) {
                float2 v[S::BN][8];  // all on their way before the first is added
#pragma unroll
                for (int j = 0; j < S::BN; ++j)
#pragma unroll
                    for (int q = 0; q < 8; ++q) v[j][q] = take(src + ((i * S::BN + j) * 8 + q) * S::kThreads);
#pragma unroll
                for (int j = 0; j < S::BN; ++j)
#pragma unroll
                    for (int q = 0; q < 8; ++q) {
                        acc.v[i][j][2 * q] = s ? acc.v[i][j][2 * q] + v[j][q].x : v[j][q].x;
                        acc.v[i][j][2 * q + 1] = s ? acc.v[i][j][2 * q + 1] + v[j][q].y : v[j][q].y;
                    }
            }
        }
    }
    finish<S, WHAT>(g, it, product, acc, lds, ti, tj, wave, lane);
}

// ---- a whole phase of a small matrix (n <= 128): one workgroup, A, P and (n <= 96) Q in LDS ----
struct ChainStep {
    float ca, cb, poly, t, q, a;  // as in ProductArgs, for P, P A, P Q and A's
};
struct ChainArgs {
    Common c;
    ChainStep step[kPhaseMost];
    int steps, phase, q;  // q: where the apply looks for Q
    float gram;
};
constexpr int kChainThreads = 512, kChainWaves = 8;
constexpr uint32_t kChainMost = 128, kChainGram = 64, kChainGramSteps = 512;  // n; n and steps of X X^T that the same workgroup does
constexpr uint32_t kChainLds = 128 * 1024;

// fragments of a matrix: row block rb, step kb
struct Plane {
    uint8_t* base;
    uint32_t per_row;
    __device__ uint8_t* frag(uint32_t rb, uint32_t kb) const { return base + ((uint64_t)rb * per_row + kb) * kFragBytes; }
};

// blocks b = w PER + e of the nb x nb ones.  The three terms have sums of their own, so that products do not wait for each
// other, and the fragments of two steps are on their way together.
template <int PER>
__device__ __forceinline__ void chain_product(float16v (&acc)[PER], const Plane& l, const Plane& r, uint32_t nb, uint32_t steps, uint32_t wave, uint32_t lane)
{
    float16v hl[PER], lh[PER];
#pragma unroll
    for (int e = 0; e < PER; ++e)
#pragma unroll
        for (int k = 0; k < 16; ++k) acc[e][k] = hl[e][k] = lh[e][k] = 0.f;
    if (wave * PER >= nb * nb) return;
    for (uint32_t k = 0; k < steps; k += 2) {
        half8 left[2][PER][2], right[2][PER][2];
#pragma unroll
        for (uint32_t u = 0; u < 2; ++u)
#pragma unroll
            for (int e = 0; e < PER; ++e) {
                const uint32_t b = min(wave * PER + e, nb * nb - 1), i = b / nb, j = b - i * nb, kk = min(k + u, steps - 1);
                const uint8_t *pl = l.frag(i, kk) + lane * 16u, *pr = r.frag(j, kk) + lane * 16u;
                left[u][e][0] = *reinterpret_cast<const half8*>(pl);
                left[u][e][1] = *reinterpret_cast<const half8*>(pl + 1024);
                right[u][e][0] = *reinterpret_cast<const half8*>(pr);
                right[u][e][1] = *reinterpret_cast<const half8*>(pr + 1024);
            }
#pragma unroll
        for (uint32_t u = 0; u < 2; ++u) {
            if (k + u >= steps) break;
#pragma unroll
            for (int e = 0; e < PER; ++e) {
                hl[e] = __builtin_amdgcn_mfma_f32_32x32x16_f16(left[u][e][0], right[u][e][1], hl[e], 0, 0, 0);
                lh[e] = __builtin_amdgcn_mfma_f32_32x32x16_f16(left[u][e][1], right[u][e][0], lh[e], 0, 0, 0);
                acc[e] = __builtin_amdgcn_mfma_f32_32x32x16_f16(left[u][e][0], right[u][e][0], acc[e], 0, 0, 0);
            }
        }
    }
#pragma unroll
    for (int e = 0; e < PER; ++e)
#pragma unroll
        for (int k = 0; k < 16; ++k) acc[e][k] += hl[e][k] + lh[e][k];
}
// four values of one column to a matrix's fragments (of its transpose, which it equals)
__device__ __forceinline__ void chain_write(const Plane& to, uint32_t i, uint32_t j, uint32_t q, const float* v, uint32_t lane)
{
    half4 hi, lo;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        _Float16 h, l;
        split(v[e], &h, &l);
        hi[e] = h;
        lo[e] = l;
    }
    uint8_t* dst = to.frag(j, i * 2u + q / 2u) + ((lane & 31u) + 32u * (q & 1u)) * 16u + (lane >> 5) * 8u;
    *reinterpret_cast<half4*>(dst) = hi;
    *reinterpret_cast<half4*>(dst + 1024) = lo;
}
template <int PER>
__device__ __forceinline__ void chain_store(const Plane& to, const float16v (&acc)[PER], float scale, uint32_t nb, uint32_t wave, uint32_t lane)
{
#pragma unroll
    for (int e = 0; e < PER; ++e) {
        const uint32_t b = wave * PER + e;
        if (b >= nb * nb) continue;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            float v[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) v[k] = acc[e][4 * q + k] * scale;
            chain_write(to, b / nb, b % nb, q, v, lane);
        }
    }
}

template <int PER>
__device__ __forceinline__ void chain_steps(const ChainArgs& g, const Item& it, uint8_t* lds, uint32_t nb, uint32_t wave, uint32_t lane)
{
    const uint32_t steps = (it.n + 15u) / 16u, bytes = nb * nb * 2u * kFragBytes;
    const Plane a{lds, 2 * nb}, p{lds + bytes, 2 * nb}, out{g.c.ws + it.square + g.q * it.square_bytes, it.nf};
    const Plane q = nb < 4 ? Plane{lds + 2 * bytes, 2 * nb} : out;
    for (int s = 0; s < g.steps; ++s) {
        const ChainStep& st = g.step[s];
        const bool again = s + 1 < g.steps;
        {
            float16v acc[PER];
            chain_product<PER>(acc, a, a, nb, steps, wave, lane);
#pragma unroll
            for (int e = 0; e < PER; ++e) {
                const uint32_t b = wave * PER + e, i = b / nb, j = b % nb;
                if (b >= nb * nb) continue;
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const uint8_t* src = a.frag(j, i * 2u + k / 2u) + ((lane & 31u) + 32u * (k & 1u)) * 16u + (lane >> 5) * 8u;
                    const half4 ah = *reinterpret_cast<const half4*>(src), al = *reinterpret_cast<const half4*>(src + 1024);
                    float v[4];
#pragma unroll
                    for (int t = 0; t < 4; ++t) {
                        v[t] = fmaf(st.cb, (float)ah[t] + (float)al[t], acc[e][4 * k + t] * st.poly);
                        if (i == j && (lane & 31u) == 8u * k + 4u * (lane >> 5) + t) v[t] += st.ca;
                    }
                    if (again || s) chain_write(p, i, j, k, v, lane);
                    if (s == 0) chain_write(again ? q : out, i, j, k, v, lane);
                }
            }
        }
        __syncthreads();
        float16v t[PER], w[PER];
        if (again) chain_product<PER>(t, p, a, nb, steps, wave, lane);
        if (s) chain_product<PER>(w, p, q, nb, steps, wave, lane);
        __syncthreads();
        if (again) chain_store<PER>(a, t, st.t, nb, wave, lane);  // T in A's place
        if (s) chain_store<PER>(again ? q : out, w, st.q, nb, wave, lane);
        __syncthreads();
        if (again) {
            chain_product<PER>(t, a, p, nb, steps, wave, lane);
            __syncthreads();
            chain_store<PER>(a, t, st.a, nb, wave, lane);
            __syncthreads();
        }
    }
}

// A = X X^T of n <= 32 NB: every wave has an eighth of the steps
template <int NB>
__device__ __forceinline__ void chain_gram(const ChainArgs& g, const Item& it, uint8_t* lds, uint32_t wave, uint32_t lane)
{
    float16v acc[NB][NB];
#pragma unroll
    for (int i = 0; i < NB; ++i)
#pragma unroll
        for (int j = 0; j < NB; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.f;
    const uint32_t steps = (it.m + 15u) / 16u;
    const Plane x{g.c.ws + by_rows(it, g.phase), it.mf};
    constexpr uint32_t kAhead = 6;  // steps whose fragments are on their way together
    for (uint32_t k = wave; k < steps; k += kChainWaves * kAhead) {
        half8 h[kAhead][NB], l[kAhead][NB];
#pragma unroll
        for (uint32_t u = 0; u < kAhead; ++u)
#pragma unroll
            for (int i = 0; i < NB; ++i) {
                const uint8_t* src = x.frag(i, min(k + u * kChainWaves, steps - 1)) + lane * 16u;
                h[u][i] = *reinterpret_cast<const half8*>(src);
                l[u][i] = *reinterpret_cast<const half8*>(src + 1024);
            }
#pragma unroll
        for (uint32_t u = 0; u < kAhead; ++u) {
            if (k + u * kChainWaves >= steps) break;
#pragma unroll
            for (int i = 0; i < NB; ++i)
#pragma unroll
                for (int j = 0; j < NB; ++j) {
                    acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(h[u][i], l[u][j], acc[i][j], 0, 0, 0);
                    acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(l[u][i], h[u][j], acc[i][j], 0, 0, 0);
                    acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(h[u][i], h[u][j], acc[i][j], 0, 0, 0);
                }
        }
    }
    float4* sums = reinterpret_cast<float4*>(lds);  // [wave][block][4][lane]
#pragma unroll
    for (int i = 0; i < NB; ++i)
#pragma unroll
        for (int j = 0; j < NB; ++j)
#pragma unroll
            for (int q = 0; q < 4; ++q)
                sums[((wave * (NB * NB) + i * NB + j) * 4 + q) * 64 + lane] =
                    make_float4(acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]);
    __syncthreads();
    constexpr int kUnits = NB * NB * 4, kEach = (kUnits + kChainWaves - 1) / kChainWaves;
    float v[kEach][4];
#pragma unroll
    for (int u = 0; u < kEach; ++u) {
        const uint32_t unit = wave * kEach + u;
        v[u][0] = v[u][1] = v[u][2] = v[u][3] = 0.f;
        if (unit < kUnits)
            for (int w = 0; w < kChainWaves; ++w) {
                const float4 f = sums[(w * kUnits + unit) * 64 + lane];
                v[u][0] += f.x;
                v[u][1] += f.y;
                v[u][2] += f.z;
                v[u][3] += f.w;
            }
    }
    __syncthreads();
#pragma unroll
    for (int u = 0; u < kEach; ++u) {
        const uint32_t unit = wave * kEach + u, b = unit / 4;
        if (unit >= kUnits) continue;
#pragma unroll
        for (int e = 0; e < 4; ++e) v[u][e] *= g.gram;
        chain_write(Plane{lds, 2 * NB}, b / NB, b % NB, unit % 4, v[u], lane);
    }
    __syncthreads();
}

__global__ void __launch_bounds__(kChainThreads, 2) k_chain(ChainArgs g)
{
    extern __shared__ __align__(1024) uint8_t lds[];
    const Common& c = g.c;
    const uint32_t lane = threadIdx.x & 63u, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    uint32_t at;
    const Item it = c.items[find_item(c.starts + (size_t)kChain * c.count, c.count, blockIdx.x, &at)];
    const uint32_t nb = (it.n + 31u) / 32u;
    if (it.chain == 2) {
        if (nb == 1) chain_gram<1>(g, it, lds, wave, lane);
        else chain_gram<2>(g, it, lds, wave, lane);
    } else {
        const Plane from{c.ws + it.square + kA * it.square_bytes, it.nf};
        for (uint32_t i = threadIdx.x; i < nb * nb * 2u * (kFragBytes / 16u); i += kChainThreads) {
            const uint32_t frag = i / (kFragBytes / 16u), in = i % (kFragBytes / 16u);
            *reinterpret_cast<uint4*>(lds + i * 16u) = *reinterpret_cast<const uint4*>(from.frag(frag / (2 * nb), frag % (2 * nb)) + in * 16u);
        }
        __syncthreads();
    }
    if (nb <= 2) chain_steps<1>(g, it, lds, nb, wave, lane);
    else chain_steps<2>(g, it, lds, nb, wave, lane);
}

// ---- host ----
// How a class of products is launched: the tiles' size, and the steps that a workgroup has at most.
struct Share {
    int size;
    uint32_t len, workgroups;
    double us;   // what it is thought to take
    bool local;  // neighbouring workgroups' operands fit an XCD's L2
};
struct Layout {
    size_t items, starts, sums, arrivals, partial, total;
    uint32_t count[kKinds], most;
    bool fits;  // the counts are within 32 bits
};

// workgroups that sum a matrix's squares: up to kMostParts, with two pieces each or more
uint32_t norm_parts(const MatrixSpan& m)
{
    const uint64_t pieces = m.stride == m.cols ? ((uint64_t)m.rows * m.cols + kPiece - 1) / kPiece : (uint64_t)m.rows * ((m.cols + kPiece - 1) / kPiece);
    return (uint32_t)std::min<uint64_t>(kMostParts, (pieces + 1) / 2);
}
// What a list's matrix has of every class: steps of a tile, and tiles by size.
struct Work {
    uint32_t steps[kClasses];
    uint64_t tiles[kSizes][kClasses];
    int chain;
};
// chains: every matrix of the list is short enough.  Beside longer ones, whose launches there are anyway, the short ones' tiles
// cost nothing, and their chains would hold up the others.
Work work_of(const MatrixSpan& m, bool chains)
{
    Work w{};
    const uint32_t n = std::min(m.rows, m.cols), wide = std::max(m.rows, m.cols), nsteps = (n + 15) / 16, msteps = (wide + 15) / 16;
    w.chain = !chains ? 0 : n <= kChainGram && msteps <= kChainGramSteps ? 2 : 1;
    for (int cls = 0; cls < kClasses; ++cls) w.steps[cls] = cls == kGrams ? msteps : nsteps;
    for (int size = 0; size < kSizes; ++size) {
        const uint64_t t = kTileOf[size], nt = (n + t - 1) / t, mt = (wide + t - 1) / t, half = nt * (nt + 1) / 2;
        w.tiles[size][kGrams] = w.chain == 2 ? 0 : half;
        w.tiles[size][kSingles] = w.chain ? 0 : half;
        w.tiles[size][kPairs] = w.chain ? 0 : 2 * half;
        w.tiles[size][kWides] = nt * mt;
    }
    return w;
}

// What a launch takes, in us: a step of a tile, what a workgroup does before and behind its steps, and for a sliced tile, putting
// a part down and taking one up.  By tile size.
constexpr double kStepUs[kSizes] = {0.12, 0.28, 1.09}, kEndsUs[kSizes] = {3.0, 5.0, 12.0}, kPutUs[kSizes - 1] = {2.0, 3.0}, kTakeUs[kSizes - 1] = {1.0, 2.0};
constexpr uint32_t kUnits = 256;           // compute units
constexpr uint64_t kLocalBytes = 8 << 20;  // of a matrix's operand that a launch goes through
constexpr double kChainUs = 6.0, kChainStepUs = 5.0;

Share share_of(const std::vector<Work>& work, const MatrixSpan* m, int cls, int sizes)
{
    Share best{};
    double least = 0.0;
    uint32_t longest = 0;
    for (const Work& w : work)
        if (w.tiles[0][cls]) longest = std::max(longest, w.steps[cls]);
    for (int size = 0; size < sizes && longest; ++size)
        for (uint32_t slices = 1; slices <= kMostSlices; slices += slices < 4 ? 1 : slices / 2) {  // 1 2 3 4 6 9 13 19 28 42 63
            const uint32_t len = std::max(std::min(kLeastSteps, longest), (longest + slices - 1) / slices);
            double workgroups = 0, steps = 0, sliced = 0;
            for (const Work& w : work) {
                const double tiles = (double)w.tiles[size][cls];
                const uint32_t per = w.steps[cls], s = per <= len ? 1 : (per + len - 1) / len;
                workgroups += tiles * s;
                steps += tiles * per;
                if (s > 1) sliced += tiles * s;
            }
            // every compute unit has as many, or the work is even but for the last one's
            const double one = len * kStepUs[size] + kEndsUs[size];
            double us = std::min(std::ceil(workgroups / kUnits) * one, (steps * kStepUs[size] + workgroups * kEndsUs[size]) / kUnits + one);
            if (sliced > 0) us += std::ceil(sliced / kUnits) * kPutUs[size] + slices * kTakeUs[size];
            if (best.workgroups == 0 || us < least) {
                least = us;
                best = Share{size, len, (uint32_t)std::min(workgroups, 4e9), us, false};
            }
            if (len <= kLeastSteps || size == kSizes - 1) break;
        }
    uint64_t bytes = 0;
    for (size_t i = 0; i < work.size(); ++i)
        if (work[i].tiles[0][cls])
            bytes = std::max(bytes, (uint64_t)std::min(m[i].rows, m[i].cols) * 64u * std::min(work[i].steps[cls], best.len));
    best.local = bytes <= kLocalBytes;
    return best;
}

// Steps of a phase: one (X X^T, P, P X) or several, whichever is thought to take less.  Matrices that are about square have as
// much work either way, and then one has fewer launches; wide ones gain from several.
int phase_steps_of(const Share* share, bool chains, int nsteps, int most)
{
    int best = 1;
    double least = 0.0;
    for (int length = 1; length <= most; ++length) {
        const int phases = (nsteps + length - 1) / length;
        double us = phases * (share[kGrams].us + share[kWides].us);
        for (int p = 0, step = 0; p < phases; ++p) {
            const int steps = (nsteps * (p + 1) + phases - 1) / phases - step;
            step += steps;
            us += steps * share[kSingles].us;  // P
            // the first step's P A, the last one's P Q and every other's two at once; A
            if (steps > 1) us += (steps + 1) * share[kSingles].us + (steps - 2) * share[kPairs].us;
            if (chains) us += kChainUs + steps * kChainStepUs;
        }
        if (length == 1 || us < least) {
            least = us;
            best = length;
        }
    }
    return best;
}

// How a list is taken: everything that its shapes decide.
struct Plan {
    std::vector<Work> work;
    Share share[kClasses];
    uint32_t room;  // rows and columns that there is room for are multiples of this
    int phase_steps;
};
Plan plan_of(const MatrixSpan* m, int count, int nsteps, int most_phase)
{
    Plan p{};
    uint32_t highest = 0;
    for (int i = 0; i < count; ++i) highest = std::max(highest, std::min(m[i].rows, m[i].cols));
    const bool chains = highest <= kChainMost;
    p.work.reserve((size_t)count);
    for (int i = 0; i < count; ++i) p.work.push_back(work_of(m[i], chains));
    const int sizes = highest > Large::kTile ? kSizes : kSizes - 1;
    p.room = kTileOf[sizes - 1];
    for (int cls = 0; cls < kClasses; ++cls) p.share[cls] = share_of(p.work, m, cls, sizes);
    p.phase_steps = phase_steps_of(p.share, chains, nsteps, most_phase);
    return p;
}

// the matrices' places; each(i, item, units of the kinds before it)
template <typename Each>
Layout lay_out(const MatrixSpan* m, int count, const Plan& plan, Each&& each)
{
    Layout l{};
    uint64_t sum[kKinds] = {}, sums = 0;
    for (int i = 0; i < count; ++i) sums += norm_parts(m[i]);
    size_t off = 0;
    l.items = off;  off = align256(off + (size_t)count * sizeof(Item));
    l.starts = off; off = align256(off + (size_t)count * kKinds * 4);
    l.sums = off;   off = align256(off + sums * 8);
    bool sliced[kClasses] = {};
    for (int i = 0; i < count; ++i) {
        const Work& w = plan.work[(size_t)i];
        Item it{};
        it.at = m[i].offset;
        it.stride = m[i].stride;
        it.rows = m[i].rows;
        it.cols = m[i].cols;
        it.n = std::min(it.rows, it.cols);
        it.m = std::max(it.rows, it.cols);
        const uint32_t np = (it.n + plan.room - 1) / plan.room * plan.room, mp = (it.m + plan.room - 1) / plan.room * plan.room;
        it.nf = np / 16;
        it.mf = mp / 16;
        it.gain = m[i].gain;
        it.chain = (uint32_t)w.chain;
        const size_t x = (size_t)np * mp * 4;
        for (int k = 0; k < 2; ++k) {
            it.x[k] = off;  off += x;
            it.xt[k] = off; off += x;
        }
        it.square = off;
        it.square_bytes = (size_t)np * np * 4;
        off += kSquares * it.square_bytes;
        it.parts = norm_parts(m[i]);
        uint64_t units[kKinds] = {};
        units[kNorm] = it.parts;
        units[kConvert] = (uint64_t)((it.n + 63) / 64) * ((it.m + 63) / 64);
        units[kChain] = it.chain != 0;
        for (int cls = 0; cls < kClasses; ++cls) {
            const Share& s = plan.share[cls];
            if (!s.workgroups) continue;
            const uint32_t slices = (w.steps[cls] + s.len - 1) / s.len;
            units[kProducts + cls] = w.tiles[s.size][cls] * slices;
            sliced[cls] = sliced[cls] || (slices > 1 && w.tiles[s.size][cls]);
        }
        each(i, it, l.count);
        for (int k = 0; k < kKinds; ++k) l.count[k] = (uint32_t)(sum[k] += units[k]);
    }
    l.fits = true;
    for (int k = 0; k < kKinds; ++k) l.fits = l.fits && sum[k] < (uint64_t)1 << 22;  // of 512 threads: within a launch's 2^32
    size_t partial = 0;
    for (int cls = 0; cls < kClasses; ++cls) {
        if (!sliced[cls]) continue;
        l.most = std::max(l.most, l.count[kProducts + cls]);
        partial = std::max(partial, (size_t)l.count[kProducts + cls] * kTileBytesOf[plan.share[cls].size]);
    }
    l.arrivals = align256(off);
    l.partial = align256(l.arrivals + (size_t)l.most * 4);
    l.total = l.partial + partial;
    return l;
}

hipError_t allow_lds(const void* kernel, std::atomic<bool> (&ready)[64], uint32_t bytes)
{
    int dev = 0;
    hipError_t e = hipGetDevice(&dev);
    if (e != hipSuccess) return e;
    if (dev < 0 || dev >= 64) return hipErrorInvalidDevice;
    if (!ready[dev]) {
        e = hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
        if (e != hipSuccess) return e;
        ready[dev] = true;
    }
    return hipSuccess;
}

template <typename S, int WHAT>
hipError_t launch_shared(const char* name, const ProductArgs& g, uint32_t workgroups, hipStream_t s)
{
    static std::atomic<bool> ready[64] = {};  // by device
    const hipError_t e = allow_lds(reinterpret_cast<const void*>(&k_product<S, WHAT>), ready, S::kLds);
    if (e != hipSuccess) return e;
    FFTSP_LAUNCH(name, (k_product<S, WHAT>), dim3(workgroups), dim3(S::kThreads), S::kLds, s, g);
    return hipGetLastError();
}
template <int WHAT>
hipError_t launch_product(const char* name, ProductArgs g, const Plan& plan, const Layout& places, hipStream_t s)
{
    g.cls = WHAT == kGram ? kGrams : !symmetric(WHAT) ? kWides : WHAT == kTimes && g.products == 2 ? kPairs : kSingles;
    const Share& share = plan.share[g.cls];
    const uint32_t workgroups = places.count[kProducts + g.cls];
    if (workgroups == 0) return hipSuccess;
    g.len = share.len;
    g.local = share.local;
    switch (share.size) {
        case 0: return launch_shared<Least, WHAT>(name, g, workgroups, s);
        case 1: return launch_shared<Small, WHAT>(name, g, workgroups, s);
        default: return launch_shared<Large, WHAT>(name, g, workgroups, s);
    }
}

// How many times a matrix of singular values up to `bound` its planes hold: a power of two that leaves a factor of two
// below binary16's largest number
float lift_for(double bound)
{
    int e = 14;
    while (e > -20 && std::ldexp(bound, e) > 32768.0) --e;
    return (float)std::ldexp(1.0, e);
}

hipError_t launch_steps(const Common& c, const OrthogonalArgs& a, const StepBounds& b, const Plan& plan, const Layout& places, hipStream_t s)
{
    hipError_t e = hipSuccess;
    int step = 0;
    for (int phase = 0; phase < b.phases && e == hipSuccess; ++phase) {
        const float lx = lift_for(b.x[phase]);
        ChainArgs chain{};
        chain.c = c;
        chain.phase = phase;
        ProductArgs g{};
        g.c = c;
        g.products = 1;
        g.phase = phase;
        g.out[0] = kA;
        float la = lift_for(b.a[step]), lq = 1.f;
        chain.gram = g.scale[0] = la / (lx * lx);
        e = launch_product<kGram>("orthogonal_gram", g, plan, places, s);
        int q = kQ0;
        for (const int first = step; step < b.end[phase] && e == hipSuccess; ++step) {
            ChainStep& st = chain.step[chain.steps++];
            const int p = step == first ? kQ0 : kP;
            const float lp = lift_for(p == kP ? b.p[step] : std::max(b.p[step], b.q[step]));
            g.products = 1;
            st.ca = g.ca = a.coefficients[3 * step] * lp;
            st.cb = g.cb = a.coefficients[3 * step + 1] * lp / la;
            st.poly = g.scale[0] = a.coefficients[3 * step + 2] * (lp / (la * la));
            g.left[0] = g.right[0] = kA;
            g.out[0] = p;
            e = launch_product<kPoly>("orthogonal_poly", g, plan, places, s);
            if (e != hipSuccess) break;
            const bool again = step + 1 < b.end[phase];
            const float lt = lift_for(b.t[step]);
            int k = 0;
            if (again) {  // T = P A
                g.left[k] = p;
                g.right[k] = kA;
                st.t = g.scale[k] = lt / (lp * la);
                g.out[k++] = kT;
            }
            if (p == kP) {  // Q <- P Q
                const float next = lift_for(b.q[step]);
                g.left[k] = kP;
                g.right[k] = q;
                q = q == kQ0 ? kQ1 : kQ0;
                st.q = g.scale[k] = next / (lp * lq);
                lq = next;
                g.out[k++] = q;
            } else {
                lq = lp;
            }
            g.products = k;
            if (k) e = launch_product<kTimes>("orthogonal_times", g, plan, places, s);
            if (again && e == hipSuccess) {  // A <- T P
                const float next = lift_for(b.a[step + 1]);
                g.products = 1;
                g.left[0] = kT;
                g.right[0] = p;
                st.a = g.scale[0] = next / (lt * lp);
                la = next;
                g.out[0] = kA;
                e = launch_product<kTimes>("orthogonal_times", g, plan, places, s);
            }
        }
        if (e == hipSuccess && places.count[kChain]) {
            static std::atomic<bool> ready[64] = {};
            chain.q = q;
            e = allow_lds(reinterpret_cast<const void*>(&k_chain), ready, kChainLds);
            if (e == hipSuccess) FFTSP_LAUNCH("orthogonal_chain", k_chain, dim3(places.count[kChain]), dim3(kChainThreads), kChainLds, s, chain);
        }
        if (e != hipSuccess) break;
        g.left[0] = q;
        if (phase + 1 < b.phases) {
            g.scale[0] = lift_for(b.x[phase + 1]) / (lq * lx);
            e = launch_product<kApply>("orthogonal_apply", g, plan, places, s);
        } else {
            g.scale[0] = 1.f / (lq * lx);
            e = launch_product<kLast>("orthogonal_last", g, plan, places, s);
        }
    }
    return e;
}

}  // namespace

// The singular values of X, A, P, T = P A and the phase's Q, from a grid over those that X can begin with.
bool step_bounds(const float* coefficients, int nsteps, int phase_steps, StepBounds* b)
{
    constexpr int kGrid = 256;
    double x[kGrid + 1], q[kGrid + 1];
    for (int i = 0; i <= kGrid; ++i) x[i] = (double)i / kGrid;
    b->phases = (nsteps + phase_steps - 1) / phase_steps;
    int step = 0;
    for (int phase = 0; phase < b->phases; ++phase) {
        b->end[phase] = (nsteps * (phase + 1) + b->phases - 1) / b->phases;
        b->x[phase] = 0.0;
        for (int i = 0; i <= kGrid; ++i) {
            q[i] = 1.0;
            b->x[phase] = std::max(b->x[phase], std::fabs(x[i]));
        }
        for (; step < b->end[phase]; ++step) {
            const double ca = coefficients[3 * step], cb = coefficients[3 * step + 1], cc = coefficients[3 * step + 2];
            b->a[step] = b->p[step] = b->t[step] = b->q[step] = 0.0;
            for (int i = 0; i <= kGrid; ++i) {
                const double a = x[i] * x[i], p = ca + a * (cb + a * cc);
                q[i] *= p;
                x[i] *= p;
                b->a[step] = std::max(b->a[step], a);
                b->p[step] = std::max(b->p[step], std::fabs(p));
                b->t[step] = std::max(b->t[step], std::fabs(a * p));
                b->q[step] = std::max(b->q[step], std::fabs(q[i]));
            }
            const double most = std::max(std::max(b->a[step], b->p[step]), std::max(b->t[step], b->q[step]));
            if (!(most <= kMostBound)) return false;
        }
    }
    for (int i = 0; i <= kGrid; ++i)
        if (!(std::fabs(x[i]) <= kMostBound)) return false;
    return true;
}

size_t orthogonal_workspace(const MatrixSpan* m, int count)
{
    if (!count) return 0;
    const Layout l = lay_out(m, count, plan_of(m, count, 1, 1), [](int, const Item&, const uint32_t*) {});
    return l.fits ? l.total : 0;
}

hipError_t launch_orthogonal(const OrthogonalArgs& a, const MatrixSpan* m, int count, uint8_t* ws, size_t ws_bytes, bool* fits, bool* enough,
                             hipStream_t s)
{
    const Plan plan = plan_of(m, count, a.nsteps, a.out_type == 0 ? kPhaseMost32 : kPhaseMost);
    const Layout places = lay_out(m, count, plan, [](int, const Item&, const uint32_t*) {});
    StepBounds bounds;
    if (!step_bounds(a.coefficients, a.nsteps, plan.phase_steps, &bounds)) return hipErrorInvalidValue;
    *fits = places.fits;
    *enough = ws_bytes >= places.total;
    if (!*fits || !*enough) return hipSuccess;
    Item* items = reinterpret_cast<Item*>(ws + places.items);
    uint32_t* starts = reinterpret_cast<uint32_t*>(ws + places.starts);
    Common c{};
    c.in = a.in;
    c.in_type = a.in_type;
    c.out = a.out;
    c.out_type = a.out_type;
    c.momentum = a.momentum;
    c.momentum_out = a.momentum_out;
    c.weights = a.weights;
    c.step = a.momentum != nullptr;
    c.nesterov = a.nesterov;
    c.beta = a.beta;
    c.lr = a.lr;
    c.decay = a.decay;
    c.eps = a.eps;
    c.ws = ws;
    c.items = items;
    c.starts = starts;
    c.sums = reinterpret_cast<double*>(ws + places.sums);
    c.partial = ws + places.partial;
    c.arrivals = reinterpret_cast<uint32_t*>(ws + places.arrivals);
    c.count = (uint32_t)count;
    c.most = places.most;
    c.lift = lift_for(bounds.x[0]);
    NormTable<true> list{};
    ItemTable& t = list.t;
    t.total = (uint32_t)count;
    lay_out(m, count, plan, [&](int i, const Item& it, const uint32_t* begun) {
        t.item[t.count] = it;
        for (int k = 0; k < kKinds; ++k) t.start[t.count][k] = begun[k];
        if (++t.count < kItemsPerLaunch && i + 1 < count) return;
        if (count <= kItemsPerLaunch) {
            FFTSP_LAUNCH("orthogonal_norm", k_norm<true>, dim3(places.count[kNorm]), dim3(256), 0, s, c, list);
        } else {
            FFTSP_LAUNCH("orthogonal_list", k_items, dim3(1), dim3(64), 0, s, t, items, starts);
        }
        t.first += t.count;
        t.count = 0;
    });
    if (count > kItemsPerLaunch) FFTSP_LAUNCH("orthogonal_norm", k_norm<false>, dim3(places.count[kNorm]), dim3(256), 0, s, c, NormTable<false>{});
    FFTSP_LAUNCH("orthogonal_convert", k_convert, dim3(places.count[kConvert]), dim3(256), 0, s, c);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    return launch_steps(c, a, bounds, plan, places, s);
}

}  // namespace fftsp
