// Newton-Schulz orthogonalisation of a list of matrices, and the momentum step round it.
//
//   X = U / (|U|_F + eps), n x m with n <= m;   per step  A = X X^T,  P = a I + b A + c A A,  X <- P X;   out = gain X
//
// The products carry the time: per step n^2 m for A and n^3 for A A, whose results are symmetric, so that only the tiles on
// and under the diagonal are computed and written twice, and 2 n^2 m for P X.  They run on binary16 matrix instructions
// whose inputs carry a binary32 number in two planes: 2^12 v = hi + lo, each rounded to nearest (22 bits and the sign of lo;
// v is 2^-24 v off, or 2^-37 where v is small), and x y = hi hi + hi lo + lo hi summed in binary32; the part left out is under
// 2^-24 |x| |y|.  Three instructions at sixteen times the rate of the binary32 one.
//
// Layout: a matrix that is an operand is kept as the instruction reads it, in fragments of 32 rows x 16 columns (of the
// contracted index), 64 lanes x 8 values of hi and then of lo: 2 KB, so that every access from memory to a wave is 1 KB in one
// piece and LDS is read without conflicts.  Fragments along the contracted index follow each other.  X is kept twice, by rows
// (for X X^T) and by columns (for P X).  Rows and columns are padded with zeros to whole tiles of 128; every product of them is zero
// again, so no kernel asks where a matrix ends, but the one that reads the input and the last one.
#include "layers.h"

#include <algorithm>
#include <cmath>

namespace fftsp {
namespace {

typedef _Float16 half8 __attribute__((ext_vector_type(8)));
typedef _Float16 half4 __attribute__((ext_vector_type(4)));
typedef float float16v __attribute__((ext_vector_type(16)));

constexpr float kLift = 4096.f, kDrop = 1.f / 4096.f;   // planes hold 2^12 times the number
constexpr uint32_t kFragBytes = 2048;                   // hi and lo of 32 x 16
constexpr uint32_t kTileRows = 128;                     // of a product's tile, both ways

// A matrix as the kernels see it.  Offsets of planes are bytes from the workspace's start.
struct Item {
    uint64_t at, stride;        // first element and distance of rows in the caller's arrays
    uint64_t x, xt, y, yt, a, p;
    uint32_t rows, cols, n, m;  // n = min, m = max
    uint32_t nt, mt;            // tiles of 128
    uint32_t tall;              // rows > cols: the iteration has the transposed matrix
    uint32_t parts;             // workgroups that sum its squares
    float gain;
    uint32_t pad;
};
// what a workgroup of a launch does: first workgroup of every matrix, by kind of launch
enum Kind { kNorm, kConvert, kSymmetric, kWide, kKinds };
constexpr int kItemsPerLaunch = 24;
struct ItemTable {
    Item item[kItemsPerLaunch];
    uint32_t start[kItemsPerLaunch][kKinds];
    uint32_t first, count, total;
};

__global__ void k_items(ItemTable t, Item* items, uint32_t* starts)
{
    const uint32_t i = threadIdx.x;
    if (i < t.count) {
        items[t.first + i] = t.item[i];
        for (int k = 0; k < kKinds; ++k) starts[(size_t)k * t.total + t.first + i] = t.start[i][k];
    }
}

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
__device__ __forceinline__ void store_value(void* p, int type, uint64_t i, float v)
{
    if (type == 0) static_cast<float*>(p)[i] = v;
    else if (type == 1) static_cast<Bf16*>(p)[i] = from_float<Bf16>(v);
    else static_cast<F16*>(p)[i] = from_float<F16>(v);
}

struct Common {
    const void* in;
    const float* momentum;
    float* momentum_out;
    const void* weights;
    void* out;
    int in_type, out_type, nesterov, step;
    float beta, lr, decay, eps;
    uint8_t* ws;
    const Item* items;
    const uint32_t* starts;  // [kKinds][count]
    double* parts;           // [norm workgroups]
    uint32_t count;
};

// ---- momentum and |U|_F^2 ----
__global__ void __launch_bounds__(256) k_norm(Common c)
{
    __shared__ double sums[4];
    uint32_t part;
    const Item& it = c.items[find_item(c.starts + (size_t)kNorm * c.count, c.count, blockIdx.x, &part)];
    double s = 0.0;
    // a workgroup has whole rows in turn
    for (uint32_t r = part; r < it.rows; r += it.parts) {
        const uint64_t row = it.at + (uint64_t)r * it.stride;
        for (uint32_t j = threadIdx.x; j < it.cols; j += 256) {
            float u = load_value(c.in, c.in_type, row + j);
            if (c.step) {
                const float m = fmaf(c.beta, c.momentum[row + j], u);
                c.momentum_out[row + j] = m;
                u = c.nesterov ? fmaf(c.beta, m, u) : m;
            }
            s += (double)u * (double)u;
        }
    }
    for (int d = 32; d; d >>= 1) s += __shfl_xor(s, d);
    if ((threadIdx.x & 63u) == 0) sums[threadIdx.x >> 6] = s;
    __syncthreads();
    if (threadIdx.x == 0) c.parts[blockIdx.x] = (sums[0] + sums[1]) + (sums[2] + sums[3]);
}

__device__ __forceinline__ void split(float v, _Float16* hi, _Float16* lo)
{
    *hi = (_Float16)v;
    *lo = (_Float16)(v - (float)*hi);
}

// ---- U / (|U|_F + eps) as fragments, by rows and by columns: a workgroup per 64 x 64 values ----
__global__ void __launch_bounds__(256) k_convert(Common c)
{
    __shared__ float tile[64][65];
    __shared__ double sums[4];
    uint32_t at;
    const uint32_t id = find_item(c.starts + (size_t)kConvert * c.count, c.count, blockIdx.x, &at);
    const Item& it = c.items[id];
    const uint32_t tid = threadIdx.x, lane = tid & 63u, wave = tid >> 6;
    double s = 0.0;
    const uint32_t first_part = c.starts[(size_t)kNorm * c.count + id];
    for (uint32_t i = tid; i < it.parts; i += 256) s += c.parts[first_part + i];
    for (int d = 32; d; d >>= 1) s += __shfl_xor(s, d);
    if (lane == 0) sums[wave] = s;
    __syncthreads();
    const double norm = sqrt((sums[0] + sums[1]) + (sums[2] + sums[3])) + (double)c.eps;
    const double factor = norm > 0.0 ? (double)kLift / norm : 0.0;
    // tile (tn, tm) of the iteration's n x m matrix
    const uint32_t across = it.mt * 2u, tn = at / across, tm = at - tn * across;
    for (uint32_t i = tid; i < 64 * 64; i += 256) {
        // consecutive lanes along the caller's rows
        const uint32_t slow = i >> 6, fast = i & 63u;
        const uint32_t n = tn * 64 + (it.tall ? fast : slow), m = tm * 64 + (it.tall ? slow : fast);
        float v = 0.f;
        if (n < it.n && m < it.m) {
            const uint64_t e = it.at + (it.tall ? (uint64_t)m * it.stride + n : (uint64_t)n * it.stride + m);
            v = load_value(c.in, c.in_type, e);
            if (c.step) {
                const float mo = c.momentum_out[e];
                v = c.nesterov ? fmaf(c.beta, mo, v) : mo;
            }
            v = (float)((double)v * factor);
        }
        tile[it.tall ? fast : slow][it.tall ? slow : fast] = v;
    }
    __syncthreads();
    // 2 x 4 fragments of each kind, two of each to a wave
    for (uint32_t f = wave; f < 16; f += 4) {
        const bool by_columns = f >= 8;
        const uint32_t rb = (f >> 2) & 1u, kb = f & 3u;
        half8 hi, lo;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const uint32_t r = rb * 32 + (lane & 31u), k = kb * 16 + (lane >> 5) * 8 + j;
            _Float16 h, l;
            split(by_columns ? tile[k][r] : tile[r][k], &h, &l);
            hi[j] = h;
            lo[j] = l;
        }
        const uint64_t row = (by_columns ? tm : tn) * 2u + rb, col = (by_columns ? tn : tm) * 4u + kb;
        const uint64_t per_row = (by_columns ? it.nt : it.mt) * 8u;
        uint8_t* dst = c.ws + (by_columns ? it.xt : it.x) + (row * per_row + col) * kFragBytes + lane * 16u;
        *reinterpret_cast<half8*>(dst) = hi;
        *reinterpret_cast<half8*>(dst + 1024) = lo;
    }
}

// ---- products C = L R^T of fragments ----
enum Product { kGram, kPoly, kApply, kLast };

struct ProductArgs {
    Common c;
    float ca, cb, cc;   // the step's coefficients (kPoly)
    int odd;            // X is in y, yt (and x, xt are written)
};

template <int WHAT>
__global__ void __launch_bounds__(256) k_product(ProductArgs g)
{
    constexpr bool SYMMETRIC = WHAT == kGram || WHAT == kPoly;
    __shared__ __align__(16) uint8_t lds[2][2][16384];
    uint32_t at;
    const Common& c = g.c;
    const Item& it = c.items[find_item(c.starts + (size_t)(SYMMETRIC ? kSymmetric : kWide) * c.count, c.count, blockIdx.x, &at)];
    const uint32_t tid = threadIdx.x, lane = tid & 63u, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    uint32_t ti, tj;  // tiles of C's rows and columns
    if (SYMMETRIC) {  // row ti has ti + 1 tiles
        ti = (uint32_t)((sqrtf(8.f * (float)at + 1.f) - 1.f) * 0.5f);
        while (ti * (ti + 1) / 2 > at) --ti;
        while ((ti + 1) * (ti + 2) / 2 <= at) ++ti;
        tj = at - ti * (ti + 1) / 2;
    } else {
        tj = at / it.nt;
        ti = at - tj * it.nt;
    }
    const uint32_t contracted = WHAT == kGram ? it.m : it.n;
    const uint32_t per_row = (WHAT == kGram ? it.mt : it.nt) * 8u;  // fragments along the contracted index
    const uint64_t xs = g.odd ? it.y : it.x, xts = g.odd ? it.yt : it.xt;
    const uint8_t* left = c.ws + (WHAT == kGram ? xs : WHAT == kPoly ? it.a : it.p) + (uint64_t)ti * 4u * per_row * kFragBytes + tid * 16u;
    const uint8_t* right = c.ws + (WHAT == kGram ? xs : WHAT == kPoly ? it.a : xts) + (uint64_t)tj * 4u * per_row * kFragBytes + tid * 16u;
    const uint32_t steps = (contracted + 31u) / 32u;
    const uint64_t block = (uint64_t)per_row * kFragBytes;

    float16v acc[2][2];
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.f;

    uint4 sl[4], sr[4];
    auto fetch = [&](uint32_t k) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            sl[i] = *reinterpret_cast<const uint4*>(left + i * block + (uint64_t)k * (2 * kFragBytes));
            sr[i] = *reinterpret_cast<const uint4*>(right + i * block + (uint64_t)k * (2 * kFragBytes));
        }
    };
    auto stage = [&](uint32_t b) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            *reinterpret_cast<uint4*>(&lds[b][0][i * 4096 + tid * 16]) = sl[i];
            *reinterpret_cast<uint4*>(&lds[b][1][i * 4096 + tid * 16]) = sr[i];
        }
    };
    const uint32_t wi = (wave & 1u) * 2u, wj = (wave >> 1) * 2u;  // the wave's 32-blocks
    fetch(0);
    stage(0);
    __syncthreads();
    for (uint32_t k = 0; k < steps; ++k) {
        const uint32_t b = k & 1u;
        if (k + 1 < steps) fetch(k + 1);
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) {
            half8 lh[2], ll[2], rh[2], rl[2];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const uint8_t* pl = &lds[b][0][(wi + i) * 4096 + kb * kFragBytes + lane * 16];
                const uint8_t* pr = &lds[b][1][(wj + i) * 4096 + kb * kFragBytes + lane * 16];
                lh[i] = *reinterpret_cast<const half8*>(pl);
                ll[i] = *reinterpret_cast<const half8*>(pl + 1024);
                rh[i] = *reinterpret_cast<const half8*>(pr);
                rl[i] = *reinterpret_cast<const half8*>(pr + 1024);
            }
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(lh[i], rl[j], acc[i][j], 0, 0, 0);
                    acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(ll[i], rh[j], acc[i][j], 0, 0, 0);
                    acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(lh[i], rh[j], acc[i][j], 0, 0, 0);
                }
        }
        if (k + 1 < steps) stage(b ^ 1u);
        __syncthreads();
    }

    // lane l has column l % 32 of a block and rows 8 (e / 4) + 4 (l / 32) + e % 4
    const uint32_t col = lane & 31u, half = lane >> 5;
    if (WHAT == kLast) {
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    const uint32_t n = ti * kTileRows + (wi + i) * 32 + 8 * (e / 4) + 4 * half + e % 4;
                    const uint32_t m = tj * kTileRows + (wj + j) * 32 + col;
                    if (n >= it.n || m >= it.m) continue;
                    const uint64_t el = it.at + (it.tall ? (uint64_t)m * it.stride + n : (uint64_t)n * it.stride + m);
                    float v = it.gain * (acc[i][j][e] * (kDrop * kDrop));
                    if (c.step) v = fmaf(-c.lr, v, c.decay * load_value(c.weights, c.out_type, el));
                    store_value(c.out, c.out_type, el, v);
                }
        return;
    }
    // the other orientation goes through LDS, 32 x 32 at a time, hi and lo of a value in one word
    uint32_t* turn = reinterpret_cast<uint32_t*>(&lds[0][0][0]) + wave * (32 * 36);
    uint8_t* direct = c.ws + (WHAT == kGram ? it.a : WHAT == kPoly ? it.p : g.odd ? it.xt : it.yt);  // rows: C's columns
    uint8_t* turned = c.ws + (WHAT == kGram ? it.a : WHAT == kPoly ? it.p : g.odd ? it.x : it.y);
    const uint32_t direct_row = it.nt * 8u, turned_row = (SYMMETRIC ? it.nt : it.mt) * 8u;
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const uint32_t bi = ti * 4u + wi + i, bj = tj * 4u + wj + j;
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                half4 hi, lo;
                const uint64_t frag = (uint64_t)bj * direct_row + bi * 2u + q / 2;
                const uint32_t in_frag = (col + 32u * (q & 1)) * 16u + half * 8u;
                half4 ah, al;
                if (WHAT == kPoly) {
                    const uint8_t* src = c.ws + it.a + frag * kFragBytes + in_frag;
                    ah = *reinterpret_cast<const half4*>(src);
                    al = *reinterpret_cast<const half4*>(src + 1024);
                }
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    float v = acc[i][j][q * 4 + e] * kDrop;
                    if (WHAT == kPoly) {
                        v = fmaf(g.cc, v, g.cb * ((float)ah[e] + (float)al[e]));
                        if (bi == bj && col == 8u * q + 4u * half + e) v += g.ca * kLift;
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
                uint8_t* dst = direct + frag * kFragBytes + in_frag;
                *reinterpret_cast<half4*>(dst) = hi;
                *reinterpret_cast<half4*>(dst + 1024) = lo;
            }
            __builtin_amdgcn_fence(__ATOMIC_SEQ_CST, "wavefront");
            __builtin_amdgcn_wave_barrier();
            if (!SYMMETRIC || ti != tj) {
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

// ---- host ----
struct Layout {
    size_t items, starts, parts, planes, total;
    uint32_t workgroups[kKinds];
};

template <typename Each>
Layout lay_out(const MatrixSpan* m, int count, Each&& each)
{
    Layout l{};
    uint64_t parts = 0;
    for (int i = 0; i < count; ++i) parts += std::min<uint32_t>(m[i].rows, 256);  // at most
    size_t off = 0;
    l.items = off;  off = align256(off + (size_t)count * sizeof(Item));
    l.starts = off; off = align256(off + (size_t)count * kKinds * 4);
    l.parts = off;  off = align256(off + parts * 8);
    l.planes = off;
    for (int i = 0; i < count; ++i) {
        Item it{};
        it.at = m[i].offset;
        it.stride = m[i].stride;
        it.rows = m[i].rows;
        it.cols = m[i].cols;
        it.tall = it.rows > it.cols;
        it.n = std::min(it.rows, it.cols);
        it.m = std::max(it.rows, it.cols);
        it.nt = (it.n + kTileRows - 1) / kTileRows;
        it.mt = (it.m + kTileRows - 1) / kTileRows;
        it.gain = m[i].gain;
        const size_t tile = (size_t)kTileRows * kTileRows * 4, x = (size_t)it.nt * it.mt * tile, a = (size_t)it.nt * it.nt * tile;
        it.x = off;  off += x;
        it.xt = off; off += x;
        it.y = off;  off += x;
        it.yt = off; off += x;
        it.a = off;  off += a;
        it.p = off;  off += a;
        const size_t values = (size_t)it.n * it.m;
        it.parts = (uint32_t)std::min<size_t>(std::min<size_t>(it.rows, 256), (values + 8191) / 8192);
        const uint32_t wgs[kKinds] = {it.parts, it.nt * 2u * it.mt * 2u, it.nt * (it.nt + 1) / 2, it.nt * it.mt};
        each(i, it, l.workgroups);
        for (int k = 0; k < kKinds; ++k) l.workgroups[k] += wgs[k];
    }
    l.total = off;
    return l;
}

}  // namespace

size_t orthogonal_workspace(const MatrixSpan* m, int count)
{
    return lay_out(m, count, [](int, const Item&, const uint32_t*) {}).total;
}

hipError_t launch_orthogonal(const OrthogonalArgs& a, const MatrixSpan* m, int count, uint8_t* ws, hipStream_t s)
{
    const Layout places = lay_out(m, count, [](int, const Item&, const uint32_t*) {});
    Item* items = reinterpret_cast<Item*>(ws + places.items);
    uint32_t* starts = reinterpret_cast<uint32_t*>(ws + places.starts);
    ItemTable t{};
    t.total = (uint32_t)count;
    lay_out(m, count, [&](int i, const Item& it, const uint32_t* begun) {
        t.item[t.count] = it;
        for (int k = 0; k < kKinds; ++k) t.start[t.count][k] = begun[k];
        if (++t.count == kItemsPerLaunch || i + 1 == count) {
            FFTSP_LAUNCH("orthogonal_list", k_items, dim3(1), dim3(64), 0, s, t, items, starts);
            t.first += t.count;
            t.count = 0;
        }
    });
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
    c.parts = reinterpret_cast<double*>(ws + places.parts);
    c.count = (uint32_t)count;
    FFTSP_LAUNCH("orthogonal_norm", k_norm, dim3(places.workgroups[kNorm]), dim3(256), 0, s, c);
    FFTSP_LAUNCH("orthogonal_convert", k_convert, dim3(places.workgroups[kConvert]), dim3(256), 0, s, c);
    for (int i = 0; i < a.nsteps; ++i) {
        const ProductArgs g{c, a.coefficients[3 * i], a.coefficients[3 * i + 1], a.coefficients[3 * i + 2], i & 1};
        FFTSP_LAUNCH("orthogonal_gram", k_product<kGram>, dim3(places.workgroups[kSymmetric]), dim3(256), 0, s, g);
        FFTSP_LAUNCH("orthogonal_poly", k_product<kPoly>, dim3(places.workgroups[kSymmetric]), dim3(256), 0, s, g);
        if (i + 1 < a.nsteps) FFTSP_LAUNCH("orthogonal_apply", k_product<kApply>, dim3(places.workgroups[kWide]), dim3(256), 0, s, g);
        else FFTSP_LAUNCH("orthogonal_last", k_product<kLast>, dim3(places.workgroups[kWide]), dim3(256), 0, s, g);
    }
    return hipGetLastError();
}

}  // namespace fftsp
