// Newton-Schulz orthogonalisation of a list of matrices, and the momentum step round it.
//
//   X = U / (|U|_F + eps), n x m with n <= m;   per step  A = X X^T,  P = a I + b A + c A A,  X <- P X;   out = gain X
//
// The products carry the time.  All matrices of a phase of a few steps are polynomials of the phase's first A, so
// they commute, and the steps can be taken on n x n matrices alone: Q <- P Q, A <- P A P, and X <- Q X at the phase's end.
// That is n^2 m for A and 2 n^2 m for Q X once a phase instead of once a step, and four symmetric n x n products (n^3
// each: only tiles on and under the diagonal are computed, and written twice) a step instead of one.  A has an absolute error
// of 2^-24 of its largest eigenvalue, which the small eigenvalues' growth by a^2 a step turns into a relative one: 1e-6 after
// two steps, up to 3.4445^4 2^-24 = 1e-5 after three, 1e-3 after five.  So a phase has up to two steps, and one where short sums
// would end closer (plan_of), whatever type the result is stored in: in 16 bits it is the one in 32, rounded.  Lists of small
// matrices take none of this: k_whole.
//
// Products run on binary16 matrix instructions whose inputs carry a binary32 number in two planes: 2^e v = hi + lo, each
// rounded to nearest, and x y = hi hi + hi lo + lo hi summed in binary32.  For v in [1, 2) hi is up to 2^-11 off, so lo has steps
// of up to 2^-22 and is 2^-23 off: that is v's error relative to it, or 2^-(25 + e) where v is small (binary16's least number).  The
// part left out is up to 2^-22 |x| |y|.  Both have random signs, and a result's error is the sums' roundings as much as theirs.
// Three instructions at sixteen times the binary32 one's rate.  e is 14 where the largest value is a half to two, and
// follows from the coefficients: they bound the singular values of every matrix of the iteration.
//
// Layout: an operand is kept as the instruction reads it, in fragments of 32 rows x 16 columns (of the contracted index),
// 64 lanes x 8 values of hi and then of lo: 2 KB, so that every access from memory to a wave is 1 KB in one piece, goes
// straight into LDS and is read from there without conflicts.  Fragments along the contracted index follow each other.
// X is kept twice, by rows (for X X^T) and by columns (for Q X).  Its rows and columns are zero up to a multiple of 64 (what
// k_convert writes); behind that, to the end of a tile of 128 or 256, is what the workspace held.  Products are contracted over
// whole steps of 16, so within the zeros, which stay zero (P has a on the diagonal there, and meets zeros of A, Q and X), and a row or
// column behind them reaches the same row or column of a product only, which nothing contracts or writes out.  So no kernel
// asks where a matrix ends but those that read the input or write the output, as long as no contraction goes further than that.
#include "layers.h"

#include <algorithm>
#include <atomic>
#include <cmath>
#include <type_traits>
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
enum Kind { kNorm, kConvert, kProducts, kKinds = kProducts + kClasses };

// A matrix as the kernels see it.  Offsets are bytes from the workspace's start.
struct Item {
    uint64_t at, stride;        // first element and distance of rows in the caller's arrays
    uint64_t x[2], xt[2];       // X by rows and by columns, before and after a phase
    uint64_t square, square_bytes;
    uint32_t rows, cols, n, m;  // n = min, m = max
    uint32_t nf, mf;            // fragments along n and along m that there is room for
    uint32_t parts;             // workgroups that sum its squares
    float gain;
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
// STAGES steps of 16 along the contracted index are in LDS or on their way there.  APART: the cross terms have sums of their own.
template <int WM_, int WN_, int BM_, int BN_, int STAGES_, bool APART_ = false>
struct Shape {
    static constexpr bool APART = APART_;
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
using Least = Shape<2, 2, 1, 1, 8, true>;  // 64 x 64
using Small = Shape<2, 2, 2, 2, 5, true>;  // 128 x 128, two workgroups to a compute unit, which fill its LDS
using Large = Shape<2, 4, 4, 2, 4>;        // 256 x 256, one; no registers for sums apart
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
// PFLOP/s become 1.38 and 1.22).  Tiles of 64 and 128 have sums of their own for hi lo and lo hi: each term that is added to
// hi hi's rounds that sum once more, and five steps on 2048 x 2048 end 1.9e-6 off instead of 3.2e-6, for 1 to 3 % more time.
// idle: a wave above the diagonal of a symmetric result, which only helps to bring the pieces.
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
    float16v cross[S::BM][S::BN];
#pragma unroll
    for (int i = 0; i < S::BM; ++i)
#pragma unroll
        for (int j = 0; j < S::BN; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e) cross[i][j][e] = 0.f;
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
            for (int j = 0; j < S::BN; ++j) {
                float16v& sum = S::APART && t < 2 ? cross[i][j] : acc.v[i][j];
                sum = __builtin_amdgcn_mfma_f32_32x32x16_f16(now[2 * (S::BN + i) + (t == 1)], now[2 * j + (t == 0)], sum, 0, 0, 0);
            }
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
    if (S::APART)
#pragma unroll
        for (int i = 0; i < S::BM; ++i)
#pragma unroll
            for (int j = 0; j < S::BN; ++j) acc.v[i][j] += cross[i][j];
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

// ---- small matrices (n <= 64, m <= 768): one workgroup each, everything in one launch, X in registers ----
// A launch that depends on the one before takes 4 us whatever it does, and a step has three of them.  Wave w has the columns
// 32 (w + 8 b) .. + 31 of X as fragments whose rows are those columns (three such blocks are 96 registers of its 256; a fourth
// spills).  The accumulators of P X are X's next fragments, and their products by the identity, which are exact, those of X's
// rows, which go into X X^T at once.  Only X X^T, summed over the waves, A and P are in LDS.  A lane's accumulators hold rows
// 8 (e / 4) + 4 (l / 32) + e % 4 of a block, so that is the order of the contracted index in all fragments here.
// Five steps, 32 bits: 64 x 64 takes 25 us, 64 x 768 60 and as launches of products (64 x 769) 93; 1024 of these 327 and 1774,
// 2048 of 64 x 64 261 and (65 x 65) 1436.  A step of 64 x 576 takes 6.6 us: 50 matrix instructions a block of columns are 3.5
// on a SIMD that has five blocks, and the sum over the waves, A and P, which wait for each other, the rest.
struct WholeStep {
    float gram, ca, cb, poly, apply;  // scales of the sums, and what P has besides, as in ProductArgs
};
struct WholeArgs {
    Common c;
    WholeStep step[kMostSteps];
    int steps;
    const MatrixSpan* items;
};
constexpr uint32_t kWholeHeight = 64, kWholeWidth = 768;  // n and m at most
constexpr int kWholeThreads = 512, kWholeWaves = 8, kWholeBlocks = kWholeWidth / 32 / kWholeWaves;
constexpr uint64_t kWholeExtent = 1 << 29;                 // elements from a matrix's first to its last: byte offsets in 32 bits
constexpr int kWholeItems = 64;  // in a launch's arguments
// in LDS: sums of X X^T by wave, block under the diagonal, quarter of it and lane; A; P
template <int NB>
struct WholeLds {
    static constexpr int kUnits = NB * (NB + 1) / 2 * 4;
    static constexpr uint32_t kPlane = NB * 2 * NB * kFragBytes, kA = kWholeWaves * kUnits * 1024, kP = kA + kPlane, kBytes = kP + kPlane;
};
struct WholeTable {
    MatrixSpan item[kWholeItems];
    uint32_t first, count;
};
__global__ void k_whole_items(WholeTable t, MatrixSpan* items)
{
    if (threadIdx.x < t.count) items[t.first + threadIdx.x] = t.item[threadIdx.x];
}

__device__ __forceinline__ void split8(const float* v, half8* hi, half8* lo)
{
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        _Float16 h, l;
        split(v[e], &h, &l);
        (*hi)[e] = h;
        (*lo)[e] = l;
    }
}
__device__ __forceinline__ float16v zeros()
{
    float16v z;
#pragma unroll
    for (int e = 0; e < 16; ++e) z[e] = 0.f;
    return z;
}
__device__ __forceinline__ float16v product3(half8 lh, half8 ll, half8 rh, half8 rl, float16v acc)
{
    acc = __builtin_amdgcn_mfma_f32_32x32x16_f16(lh, rl, acc, 0, 0, 0);
    acc = __builtin_amdgcn_mfma_f32_32x32x16_f16(ll, rh, acc, 0, 0, 0);
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(lh, rh, acc, 0, 0, 0);
}

// U's values of the wave's columns, as fragments whose rows are the caller's columns: of X by columns where it lies as the
// caller's array does, of X by rows where it is the transpose.  The momentum is written down.  Returns the squares' sum.
// Every access is within the matrix: the places outside read its last row or column, and count as zero.
template <int NB, typename T, bool STEP>
__device__ __forceinline__ double whole_load(const Common& c, const MatrixSpan& it, uint32_t blocks, uint32_t wave, uint32_t lane,
                                             float (&v)[kWholeBlocks][2 * NB][8])
{
    const bool t = it.rows > it.cols;
    const T* in_values = static_cast<const T*>(c.in) + it.offset;
    const float* momentum = c.momentum + it.offset;
    float* momentum_out = c.momentum_out + it.offset;
    const uint32_t stride = (uint32_t)it.stride;
    auto place = [&](int b, int k, int e, uint32_t* at) {
        const uint32_t bj = b * kWholeWaves + wave, o = 8u * (e / 4) + 4u * (lane >> 5) + e % 4;
        const uint32_t row = t ? bj * 32u + (k & 1) * 16u + o : k * 16u + o, col = (t ? k >> 1 : bj) * 32u + (lane & 31u);
        *at = min(row, it.rows - 1) * stride + min(col, it.cols - 1);
        return row < it.rows && col < it.cols;
    };
    float mo[kWholeBlocks][2 * NB][8];
#pragma unroll
    for (int b = 0; b < kWholeBlocks; ++b) {
        const bool some = b * kWholeWaves + wave < blocks;
#pragma unroll
        for (int k = 0; k < 2 * NB; ++k)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                uint32_t at;
                place(b, k, e, &at);
                v[b][k][e] = mo[b][k][e] = 0.f;
                if (some) {
                    v[b][k][e] = to_float(in_values[at]);
                    if (STEP) mo[b][k][e] = momentum[at];
                }
            }
    }
    double s = 0.0;
#pragma unroll
    for (int b = 0; b < kWholeBlocks; ++b) {
        if (b * kWholeWaves + wave >= blocks) break;
#pragma unroll
        for (int k = 0; k < 2 * NB; ++k)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                uint32_t at;
                const bool in = place(b, k, e, &at);
                float u = v[b][k][e];
                if (STEP) {
                    const float m = fmaf(c.beta, mo[b][k][e], u);
                    if (in) momentum_out[at] = m;
                    u = c.nesterov ? fmaf(c.beta, m, u) : m;
                }
                u = in ? u : 0.f;
                s += (double)u * (double)u;
                v[b][k][e] = u;
            }
    }
    return s;
}

template <int NB, typename T>
__device__ __forceinline__ double whole_load_of_type(const Common& c, const MatrixSpan& it, uint32_t blocks, uint32_t wave, uint32_t lane,
                                                     float (&v)[kWholeBlocks][2 * NB][8])
{
    return c.step ? whole_load<NB, T, true>(c, it, blocks, wave, lane, v) : whole_load<NB, T, false>(c, it, blocks, wave, lane, v);
}

// A = scale X X^T from the waves' parts: a unit is a quarter of a block under the diagonal, which is A's both ways round
template <int NB>
__device__ __forceinline__ void whole_sum(uint8_t* lds, float scale, uint32_t parts, uint32_t wave, uint32_t lane)
{
    using L = WholeLds<NB>;
    const float4* sums = reinterpret_cast<const float4*>(lds);
    uint8_t* a = lds + L::kA;
    for (uint32_t unit = wave; unit < L::kUnits; unit += kWholeWaves) {
        float v[4] = {};
        for (uint32_t w = 0; w < parts; ++w) {
            const float4 f = sums[(w * L::kUnits + unit) * 64 + lane];
            v[0] += f.x;
            v[1] += f.y;
            v[2] += f.z;
            v[3] += f.w;
        }
        const uint32_t b = unit / 4, q = unit % 4, i = b ? 1 : 0, j = b == 2 ? 1 : 0;  // blocks (0, 0), (1, 0), (1, 1)
        const uint32_t col = lane & 31u, half = lane >> 5;
        half4 hi, lo;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            _Float16 h, l;
            split(v[e] * scale, &h, &l);
            hi[e] = h;
            lo[e] = l;
        }
        uint8_t* dst = a + (j * 2 * NB + i * 2 + q / 2) * kFragBytes + lane * 16u + (q & 1u) * 8u;
        *reinterpret_cast<half4*>(dst) = hi;
        *reinterpret_cast<half4*>(dst + 1024) = lo;
        if (i == j) continue;
        uint8_t* to = a + (i * 2 * NB + j * 2 + col / 16) * kFragBytes + (8u * q + 4u * half + 32u * (col >> 2 & 1u)) * 16u +
                      ((col >> 3 & 1u) * 4u + (col & 3u)) * 2u;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            *reinterpret_cast<_Float16*>(to + e * 16) = hi[e];
            *reinterpret_cast<_Float16*>(to + e * 16 + 1024) = lo[e];
        }
    }
}

// P = a I + b A + c A A: a wave has a block; the three terms have sums of their own, so that products do not wait for each other
template <int NB>
__device__ __forceinline__ void whole_poly(uint8_t* lds, const WholeStep& st, uint32_t steps, uint32_t wave, uint32_t lane)
{
    using L = WholeLds<NB>;
    if (wave >= NB * NB) return;
    const uint32_t i = wave / NB, j = wave % NB;
    const uint8_t* a = lds + L::kA + lane * 16u;
    float16v sum[3] = {zeros(), zeros(), zeros()};
#pragma unroll
    for (uint32_t k = 0; k < 2 * NB; ++k) {
        if (k >= steps) break;
        const uint8_t *pl = a + (i * 2 * NB + k) * kFragBytes, *pr = a + (j * 2 * NB + k) * kFragBytes;
        const half8 lh = *reinterpret_cast<const half8*>(pl), ll = *reinterpret_cast<const half8*>(pl + 1024);
        const half8 rh = *reinterpret_cast<const half8*>(pr), rl = *reinterpret_cast<const half8*>(pr + 1024);
        sum[0] = __builtin_amdgcn_mfma_f32_32x32x16_f16(lh, rl, sum[0], 0, 0, 0);
        sum[1] = __builtin_amdgcn_mfma_f32_32x32x16_f16(ll, rh, sum[1], 0, 0, 0);
        sum[2] = __builtin_amdgcn_mfma_f32_32x32x16_f16(lh, rh, sum[2], 0, 0, 0);
    }
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const uint32_t at = (j * 2 * NB + i * 2 + k) * kFragBytes;
        const half8 ah = *reinterpret_cast<const half8*>(a + at), al = *reinterpret_cast<const half8*>(a + at + 1024);
        float v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float s = sum[2][8 * k + e] + (sum[0][8 * k + e] + sum[1][8 * k + e]);
            v[e] = fmaf(st.cb, (float)ah[e] + (float)al[e], s * st.poly);
            if (i == j && (lane & 31u) == 16u * k + 8u * (e / 4) + 4u * (lane >> 5) + e % 4) v[e] += st.ca;
        }
        half8 hi, lo;
        split8(v, &hi, &lo);
        uint8_t* dst = lds + L::kP + at + lane * 16u;
        *reinterpret_cast<half8*>(dst) = hi;
        *reinterpret_cast<half8*>(dst + 1024) = lo;
    }
}

// P times a block of columns, or the block's transpose times P
template <int NB, bool TURNED>
__device__ __forceinline__ void whole_times(const uint8_t* p, const half8* xh, const half8* xl, uint32_t steps, float16v (&acc)[NB])
{
#pragma unroll
    for (int i = 0; i < NB; ++i) acc[i] = zeros();
#pragma unroll
    for (uint32_t k = 0; k < 2 * NB; ++k) {
        if (k >= steps) break;
#pragma unroll
        for (int i = 0; i < NB; ++i) {
            const uint8_t* src = p + (i * 2 * NB + k) * kFragBytes;
            const half8 h = *reinterpret_cast<const half8*>(src), l = *reinterpret_cast<const half8*>(src + 1024);
            acc[i] = TURNED ? product3(xh[k], xl[k], h, l, acc[i]) : product3(h, l, xh[k], xl[k], acc[i]);
        }
    }
}
// Fragments of a block's transpose: products by the identity, which are exact
template <int NB>
__device__ __forceinline__ void whole_turn(const half8 (&one)[2], const half8* from, half8* to)
{
#pragma unroll
    for (int i = 0; i < NB; ++i) {
        float16v acc = __builtin_amdgcn_mfma_f32_32x32x16_f16(from[2 * i], one[0], zeros(), 0, 0, 0);
        acc = __builtin_amdgcn_mfma_f32_32x32x16_f16(from[2 * i + 1], one[1], acc, 0, 0, 0);
#pragma unroll
        for (int k = 0; k < 2; ++k)
#pragma unroll
            for (int e = 0; e < 8; ++e) to[2 * i + k][e] = (_Float16)acc[8 * k + e];
    }
}
template <int NB>
__device__ __forceinline__ void whole_split(const float16v (&acc)[NB], float scale, half8* hi, half8* lo)
{
#pragma unroll
    for (int i = 0; i < NB; ++i)
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            float v[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = acc[i][8 * k + e] * scale;
            split8(v, hi + 2 * i + k, lo + 2 * i + k);
        }
}

// a block of the result: accumulators' columns are the caller's
template <int NB, typename T>
__device__ __forceinline__ void whole_store(const Common& c, const MatrixSpan& it, const float16v (&acc)[NB], float scale, uint32_t bj, uint32_t lane)
{
    const bool t = it.rows > it.cols;
#pragma unroll
    for (int i = 0; i < NB; ++i) {
        const uint32_t row = (t ? bj : i) * 32u + 4u * (lane >> 5), col = (t ? i : bj) * 32u + (lane & 31u);
        float w[16];
        if (c.step)
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                const uint32_t r = row + 8u * (e / 4) + e % 4;
                w[e] = r < it.rows && col < it.cols ? to_float(static_cast<const T*>(c.weights)[it.offset + (uint64_t)r * it.stride + col]) : 0.f;
            }
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            const uint32_t r = row + 8u * (e / 4) + e % 4;
            float v = acc[i][e] * scale;
            if (c.step) v = fmaf(-c.lr, v, c.decay * w[e]);
            if (r < it.rows && col < it.cols) static_cast<T*>(c.out)[it.offset + (uint64_t)r * it.stride + col] = from_float<T>(v);
        }
    }
}

template <int NB>
__device__ __forceinline__ void whole(const WholeArgs& w, const MatrixSpan& it, uint8_t* lds, uint32_t wave, uint32_t lane)
{
    using L = WholeLds<NB>;
    const Common& c = w.c;
    const uint32_t steps = (min(it.rows, it.cols) + 15u) / 16u, blocks = (max(it.rows, it.cols) + 31u) / 32u;
    const uint32_t parts = min(blocks, (uint32_t)kWholeWaves);
    half8 xh[kWholeBlocks][2 * NB], xl[kWholeBlocks][2 * NB];
    {
        float v[kWholeBlocks][2 * NB][8];
        double s;
        if (c.in_type == 0) s = whole_load_of_type<NB, float>(c, it, blocks, wave, lane, v);
        else if (c.in_type == 1) s = whole_load_of_type<NB, Bf16>(c, it, blocks, wave, lane, v);
        else s = whole_load_of_type<NB, F16>(c, it, blocks, wave, lane, v);
        for (int d = 32; d; d >>= 1) s += __shfl_xor(s, d);
        double* sums = reinterpret_cast<double*>(lds);
        if (lane == 0) sums[wave] = s;
        __syncthreads();
        double sum = 0.0;
#pragma unroll
        for (int i = 0; i < kWholeWaves; ++i) sum += sums[i];
        __syncthreads();
        const double norm = sqrt(sum) + (double)c.eps;
        const double factor = norm > 0.0 ? (double)c.lift / norm : 0.0;
#pragma unroll
        for (int b = 0; b < kWholeBlocks; ++b)
#pragma unroll
            for (int k = 0; k < 2 * NB; ++k) {
#pragma unroll
                for (int e = 0; e < 8; ++e) v[b][k][e] = (float)((double)v[b][k][e] * factor);
                split8(v[b][k], &xh[b][k], &xl[b][k]);
            }
    }
    const uint8_t* p = lds + L::kP + lane * 16u;
    half8 one[2];
#pragma unroll
    for (int k = 0; k < 2; ++k)
#pragma unroll
        for (int e = 0; e < 8; ++e) one[k][e] = (lane & 31u) == k * 16u + 8u * (e / 4) + 4u * (lane >> 5) + e % 4 ? (_Float16)1.f : (_Float16)0.f;
    if (it.rows > it.cols) {
#pragma unroll
        for (int b = 0; b < kWholeBlocks; ++b) {
            if (b * kWholeWaves + wave >= blocks) break;
            half8 hi[2 * NB], lo[2 * NB];
            whole_turn<NB>(one, xh[b], hi);
            whole_turn<NB>(one, xl[b], lo);
#pragma unroll
            for (int k = 0; k < 2 * NB; ++k) {
                xh[b][k] = hi[k];
                xl[b][k] = lo[k];
            }
        }
    }
    float scale = 1.f;
    for (int s = 0; s < w.steps; ++s) {
        float16v sum[NB * (NB + 1) / 2];
#pragma unroll
        for (int b = 0; b < NB * (NB + 1) / 2; ++b) sum[b] = zeros();
#pragma unroll
        for (int b = 0; b < kWholeBlocks; ++b) {
            if (b * kWholeWaves + wave >= blocks) break;
            if (s) {
                float16v acc[NB];
                whole_times<NB, false>(p, xh[b], xl[b], steps, acc);
                whole_split<NB>(acc, scale, xh[b], xl[b]);
            }
            half8 hi[2 * NB], lo[2 * NB];
            whole_turn<NB>(one, xh[b], hi);
            whole_turn<NB>(one, xl[b], lo);
#pragma unroll
            for (int k = 0; k < 2; ++k)
#pragma unroll
                for (int i = 0, u = 0; i < NB; ++i)
#pragma unroll
                    for (int j = 0; j <= i; ++j, ++u) sum[u] = product3(hi[2 * i + k], lo[2 * i + k], hi[2 * j + k], lo[2 * j + k], sum[u]);
        }
        if (wave < parts) {
            float4* to = reinterpret_cast<float4*>(lds) + wave * L::kUnits * 64 + lane;
#pragma unroll
            for (int u = 0; u < L::kUnits; ++u)
                to[u * 64] = make_float4(sum[u / 4][u % 4 * 4], sum[u / 4][u % 4 * 4 + 1], sum[u / 4][u % 4 * 4 + 2], sum[u / 4][u % 4 * 4 + 3]);
        }
        __syncthreads();
        whole_sum<NB>(lds, w.step[s].gram, parts, wave, lane);
        __syncthreads();
        whole_poly<NB>(lds, w.step[s], steps, wave, lane);
        __syncthreads();
        scale = w.step[s].apply;
    }
    scale *= it.gain;
#pragma unroll
    for (int b = 0; b < kWholeBlocks; ++b) {
        const uint32_t bj = b * kWholeWaves + wave;
        if (bj >= blocks) break;
        float16v acc[NB];
        if (it.rows > it.cols) whole_times<NB, true>(p, xh[b], xl[b], steps, acc);
        else whole_times<NB, false>(p, xh[b], xl[b], steps, acc);
        if (c.out_type == 0) whole_store<NB, float>(c, it, acc, scale, bj, lane);
        else if (c.out_type == 1) whole_store<NB, Bf16>(c, it, acc, scale, bj, lane);
        else whole_store<NB, F16>(c, it, acc, scale, bj, lane);
    }
}
// ARGUMENTS: the whole list is in the launch's arguments
template <bool ARGUMENTS>
__global__ void __launch_bounds__(kWholeThreads, 2) k_whole(WholeArgs w, std::conditional_t<ARGUMENTS, WholeTable, NormTable<false>> table)
{
    extern __shared__ __align__(1024) uint8_t lds[];
    const uint32_t lane = threadIdx.x & 63u, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    MatrixSpan it;
    if constexpr (ARGUMENTS) it = table.item[blockIdx.x];
    else it = w.items[blockIdx.x];
    if (min(it.rows, it.cols) <= 32) whole<1>(w, it, lds, wave, lane);
    else whole<2>(w, it, lds, wave, lane);
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
};
Work work_of(const MatrixSpan& m)
{
    Work w{};
    const uint32_t n = std::min(m.rows, m.cols), wide = std::max(m.rows, m.cols);
    for (int cls = 0; cls < kClasses; ++cls) w.steps[cls] = ((cls == kGrams ? wide : n) + 15) / 16;
    for (int size = 0; size < kSizes; ++size) {
        const uint64_t t = kTileOf[size], nt = (n + t - 1) / t, mt = (wide + t - 1) / t, half = nt * (nt + 1) / 2;
        w.tiles[size][kGrams] = w.tiles[size][kSingles] = half;
        w.tiles[size][kPairs] = 2 * half;
        w.tiles[size][kWides] = nt * mt;
    }
    return w;
}

// What a launch takes, in us: a step of a tile, what a workgroup does before and behind its steps, and for a sliced tile, putting
// a part down and taking one up.  By tile size.
constexpr double kStepUs[kSizes] = {0.12, 0.28, 1.09}, kEndsUs[kSizes] = {3.0, 5.0, 12.0}, kPutUs[kSizes - 1] = {2.0, 3.0}, kTakeUs[kSizes - 1] = {1.0, 2.0};
constexpr uint32_t kUnits = 256;           // compute units
constexpr uint64_t kMostWorkgroups = 1 << 22;  // of a launch, with 512 threads: within 2^32
constexpr uint64_t kLocalBytes = 8 << 20;  // of a matrix's operand that a launch goes through

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
int phase_steps_of(const Share* share, int nsteps, int most)
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
    bool whole;  // all matrices are small: k_whole
    std::vector<Work> work;
    Share share[kClasses];
    uint32_t room;  // rows and columns that there is room for are multiples of this
    int phase_steps;
};
// A phase has two steps only for matrices whose own sums are long enough to be about as far off (n >= kFineHeight; a list's
// others are a part of their own, Parts): with phases of two steps, 128 x 128, 300 x 300, 512 x 512, 1024 x 1024 and 2048 x 2048
// are 1.8, 1.6, 1.8, 1.7 and 1.7e-6 off, with one step's 0.9, 1.0, 1.2, 1.5 and 1.9e-6.  Three would do for no type: with them
// 4.8 % of 8192 x 16384 random numbers' binary16 results are not the nearest to the exact ones (plain binary32 products: 2.9 %,
// two steps: 1.5 %), and of 100 x 8000 with one large singular value 6.8 % (1.2 %, one step: 0.84 %).
constexpr uint32_t kFineHeight = 512;
Plan plan_of(const MatrixSpan* m, int count, int nsteps)
{
    Plan p{};
    uint32_t highest = 0;
    p.whole = true;
    for (int i = 0; i < count; ++i) {
        const uint32_t n = std::min(m[i].rows, m[i].cols), wide = std::max(m[i].rows, m[i].cols);
        highest = std::max(highest, n);
        p.whole = p.whole && n <= kWholeHeight && wide <= kWholeWidth && m[i].rows * m[i].stride <= kWholeExtent;
    }
    const int sizes = highest > Large::kTile ? kSizes : kSizes - 1;
    p.room = kTileOf[sizes - 1];
    p.phase_steps = 1;
    if (p.whole) return p;
    p.work.reserve((size_t)count);
    for (int i = 0; i < count; ++i) p.work.push_back(work_of(m[i]));
    for (int cls = 0; cls < kClasses; ++cls) p.share[cls] = share_of(p.work, m, cls, sizes);
    p.phase_steps = phase_steps_of(p.share, nsteps, highest < kFineHeight ? 1 : kPhaseMost);
    return p;
}

// the matrices' places; each(i, item, units of the kinds before it)
template <typename Each>
Layout lay_out(const MatrixSpan* m, int count, const Plan& plan, Each&& each)
{
    Layout l{};
    if (plan.whole) {
        l.total = align256((size_t)count * sizeof(MatrixSpan));
        l.fits = (uint64_t)count <= kMostWorkgroups;
        return l;
    }
    uint64_t sum[kKinds] = {}, sums = 0;
    for (int i = 0; i < count; ++i) sums += norm_parts(m[i]);
    size_t off = 0;
    l.items = off;  off = align256(off + (size_t)count * sizeof(Item));
    l.starts = off; off = align256(off + (size_t)count * kKinds * 4);
    l.sums = off;   off = align256(off + sums * 8);
    bool sliced[kClasses] = {};
    for (int i = 0; i < count; ++i) {
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
        for (int cls = 0; cls < kClasses; ++cls) {
            const Share& s = plan.share[cls];
            if (!s.workgroups) continue;
            const Work& w = plan.work[(size_t)i];
            const uint32_t slices = (w.steps[cls] + s.len - 1) / s.len;
            units[kProducts + cls] = w.tiles[s.size][cls] * slices;
            sliced[cls] = sliced[cls] || (slices > 1 && w.tiles[s.size][cls]);
        }
        each(i, it, l.count);
        for (int k = 0; k < kKinds; ++k) l.count[k] = (uint32_t)(sum[k] += units[k]);
    }
    l.fits = true;
    for (int k = 0; k < kKinds; ++k) l.fits = l.fits && sum[k] <= kMostWorkgroups;
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
// below binary16's largest number, of four where the bound is a half or less
double lift_for(double bound)
{
    int e = 14;
    while (std::ldexp(bound, e) > 32768.0) --e;
    while (e < 120 && std::ldexp(bound, e + 1) <= 16384.0) ++e;
    return std::ldexp(1.0, e);
}

hipError_t launch_steps(const Common& c, const OrthogonalArgs& a, const StepBounds& b, const Plan& plan, const Layout& places, hipStream_t s)
{
    hipError_t e = hipSuccess;
    int step = 0;
    for (int phase = 0; phase < b.phases && e == hipSuccess; ++phase) {
        const double lx = lift_for(b.x[phase]);
        ProductArgs g{};
        g.c = c;
        g.products = 1;
        g.phase = phase;
        g.out[0] = kA;
        double la = lift_for(b.a[step]), lq = 1.0;
        g.scale[0] = (float)(la / (lx * lx));
        e = launch_product<kGram>("orthogonal_gram", g, plan, places, s);
        int q = kQ0;
        for (const int first = step; step < b.end[phase] && e == hipSuccess; ++step) {
            const int p = step == first ? kQ0 : kP;
            const double lp = lift_for(p == kP ? b.p[step] : std::max(b.p[step], b.q[step]));
            g.products = 1;
            g.ca = (float)(a.coefficients[3 * step] * lp);
            g.cb = (float)(a.coefficients[3 * step + 1] * lp / la);
            g.scale[0] = (float)(a.coefficients[3 * step + 2] * (lp / (la * la)));
            g.left[0] = g.right[0] = kA;
            g.out[0] = p;
            e = launch_product<kPoly>("orthogonal_poly", g, plan, places, s);
            if (e != hipSuccess) break;
            const bool again = step + 1 < b.end[phase];
            const double lt = lift_for(b.t[step]);
            int k = 0;
            if (again) {  // T = P A
                g.left[k] = p;
                g.right[k] = kA;
                g.scale[k] = (float)(lt / (lp * la));
                g.out[k++] = kT;
            }
            if (p == kP) {  // Q <- P Q
                const double next = lift_for(b.q[step]);
                g.left[k] = kP;
                g.right[k] = q;
                q = q == kQ0 ? kQ1 : kQ0;
                g.scale[k] = (float)(next / (lp * lq));
                lq = next;
                g.out[k++] = q;
            } else {
                lq = lp;
            }
            g.products = k;
            if (k) e = launch_product<kTimes>("orthogonal_times", g, plan, places, s);
            if (again && e == hipSuccess) {  // A <- T P
                const double next = lift_for(b.a[step + 1]);
                g.products = 1;
                g.left[0] = kT;
                g.right[0] = p;
                g.scale[0] = (float)(next / (lt * lp));
                la = next;
                g.out[0] = kA;
                e = launch_product<kTimes>("orthogonal_times", g, plan, places, s);
            }
        }
        if (e != hipSuccess) break;
        g.left[0] = q;
        if (phase + 1 < b.phases) {
            g.scale[0] = (float)(lift_for(b.x[phase + 1]) / (lq * lx));
            e = launch_product<kApply>("orthogonal_apply", g, plan, places, s);
        } else {
            g.scale[0] = (float)(1.0 / (lq * lx));
            e = launch_product<kLast>("orthogonal_last", g, plan, places, s);
        }
    }
    return e;
}

template <bool ARGUMENTS, typename Table>
hipError_t launch_whole_list(const WholeArgs& w, const Table& table, int count, hipStream_t s)
{
    static std::atomic<bool> ready[64] = {};
    const hipError_t e = allow_lds(reinterpret_cast<const void*>(&k_whole<ARGUMENTS>), ready, WholeLds<2>::kBytes);
    if (e != hipSuccess) return e;
    FFTSP_LAUNCH("orthogonal_whole", k_whole<ARGUMENTS>, dim3((uint32_t)count), dim3(kWholeThreads), WholeLds<2>::kBytes, s, w, table);
    return hipGetLastError();
}
hipError_t launch_whole(const Common& c, const OrthogonalArgs& a, const StepBounds& b, const MatrixSpan* m, int count, hipStream_t s)
{
    WholeArgs w{};
    w.c = c;
    w.steps = a.nsteps;
    for (int i = 0; i < a.nsteps; ++i) {
        const double lx = lift_for(b.x[i]), la = lift_for(b.a[i]), lp = lift_for(b.p[i]);
        w.step[i] = WholeStep{(float)(la / (lx * lx)), (float)(a.coefficients[3 * i] * lp), (float)(a.coefficients[3 * i + 1] * lp / la),
                              (float)(a.coefficients[3 * i + 2] * (lp / (la * la))), (float)((i + 1 < a.nsteps ? lift_for(b.x[i + 1]) : 1.0) / (lp * lx))};
    }
    WholeTable t{};
    if (count <= kWholeItems) {
        std::copy(m, m + count, t.item);
        return launch_whole_list<true>(w, t, count, s);
    }
    MatrixSpan* items = reinterpret_cast<MatrixSpan*>(c.ws);
    for (int i = 0; i < count; i += kWholeItems) {
        t.first = (uint32_t)i;
        t.count = (uint32_t)std::min(count - i, kWholeItems);
        std::copy(m + i, m + i + t.count, t.item);
        FFTSP_LAUNCH("orthogonal_list", k_whole_items, dim3(1), dim3(kWholeItems), 0, s, t, items);
    }
    w.items = items;
    return launch_whole_list<false>(w, NormTable<false>{}, count, s);
}

// The largest magnitude of f over [0, end], where f's derivative is zero at the roots of d0 + d1 a + d2 a^2
template <typename F>
double largest(F&& f, double d0, double d1, double d2, double end)
{
    double most = std::max(std::fabs(f(0.0)), std::fabs(f(end)));
    const double under = d1 * d1 - 4.0 * d0 * d2;
    if (under < 0.0) return most;
    const double r = -0.5 * (d1 + std::copysign(std::sqrt(under), d1));  // no difference of like numbers
    for (const double at : {r / d2, d0 / r})
        if (at > 0.0 && at < end) most = std::max(most, std::fabs(f(at)));
    return most;
}

}  // namespace

// The singular values of X, A, P, T = P A and the phase's Q.  X's begin anywhere in [0, 1], and a step takes [0, top] to what the
// odd polynomial x p(x^2) reaches there: its largest magnitude is at an end or where the derivative is zero, and so are those
// of p(a) and a p(a) over [0, top^2].  Q's bound is the product of its steps' (the default's is reached, at zero).
bool step_bounds(const float* coefficients, int nsteps, int phase_steps, StepBounds* b)
{
    double top = 1.0;
    b->phases = (nsteps + phase_steps - 1) / phase_steps;
    int step = 0;
    for (int phase = 0; phase < b->phases; ++phase) {
        b->end[phase] = (nsteps * (phase + 1) + b->phases - 1) / b->phases;
        b->x[phase] = top;
        double q = 1.0;
        for (; step < b->end[phase]; ++step) {
            const double ca = coefficients[3 * step], cb = coefficients[3 * step + 1], cc = coefficients[3 * step + 2], end = top * top;
            auto p = [&](double a) { return ca + a * (cb + a * cc); };
            b->a[step] = end;
            b->p[step] = largest(p, cb, 2.0 * cc, 0.0, end);
            b->t[step] = largest([&](double a) { return a * p(a); }, ca, 2.0 * cb, 3.0 * cc, end);
            q *= b->p[step];
            b->q[step] = q;
            top = largest([&](double a) { return std::sqrt(a) * p(a); }, ca, 3.0 * cb, 5.0 * cc, end);
            if (!(std::max(top, q) <= kMostBound)) return false;  // A's are up to its square and T's to its cube
        }
    }
    return true;
}

namespace {

// A list's matrices under kFineHeight and the others: one part behind the other, in the same workspace.  All together,
// ResNet-50's take 1270 us in phases of one step and so 1283, AlexNet's 10.91 ms in phases of two, which leave the lower ones
// further off, and so 11.02.
struct Parts {
    std::vector<MatrixSpan> held;  // where there are both
    const MatrixSpan* m[2];
    int count[2];
    Parts(const MatrixSpan* list, int n)
    {
        auto low = [](const MatrixSpan& x) { return std::min(x.rows, x.cols) < kFineHeight; };
        count[0] = (int)std::count_if(list, list + n, low);
        count[1] = n - count[0];
        m[0] = m[1] = list;
        if (!count[0] || !count[1]) return;
        held.assign(list, list + n);
        std::stable_partition(held.begin(), held.end(), low);
        m[0] = held.data();
        m[1] = held.data() + count[0];
    }
};

hipError_t launch_part(const OrthogonalArgs& a, const MatrixSpan* m, int count, Plan plan, const Layout& places, uint8_t* ws, hipStream_t s)
{
    // what is accepted does not depend on how the list is taken: where a phase's products are too large, phases are shorter
    StepBounds bounds;
    while (!step_bounds(a.coefficients, a.nsteps, plan.phase_steps, &bounds))
        if (--plan.phase_steps == 0) return hipErrorInvalidValue;  // the caller has asked about single steps
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
    c.lift = (float)lift_for(bounds.x[0]);
    if (plan.whole) return launch_whole(c, a, bounds, m, count, s);
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

}  // namespace

size_t orthogonal_workspace(const MatrixSpan* m, int count)
{
    const Parts parts(m, count);
    size_t most = 0;
    for (int i = 0; i < 2; ++i) {
        if (!parts.count[i]) continue;
        const Layout l = lay_out(parts.m[i], parts.count[i], plan_of(parts.m[i], parts.count[i], 1), [](int, const Item&, const uint32_t*) {});
        if (!l.fits) return 0;
        most = std::max(most, l.total);
    }
    return most;
}

hipError_t launch_orthogonal(const OrthogonalArgs& a, const MatrixSpan* m, int count, uint8_t* ws, size_t ws_bytes, bool* fits, bool* enough,
                             hipStream_t s)
{
    const Parts parts(m, count);
    Plan plan[2];
    Layout places[2];
    *fits = *enough = true;
    for (int i = 0; i < 2; ++i) {
        if (!parts.count[i]) continue;
        plan[i] = plan_of(parts.m[i], parts.count[i], a.nsteps);
        places[i] = lay_out(parts.m[i], parts.count[i], plan[i], [](int, const Item&, const uint32_t*) {});
        *fits = *fits && places[i].fits;
        *enough = *enough && ws_bytes >= places[i].total;
    }
    if (!*fits || !*enough) return hipSuccess;
    for (int i = 0; i < 2; ++i) {
        if (!parts.count[i]) continue;
        const hipError_t e = launch_part(a, parts.m[i], parts.count[i], plan[i], places[i], ws, s);
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace fftsp
