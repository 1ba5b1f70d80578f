// What embedding.hip and orthogonal.hip share: element types, and accesses that need only an element's alignment.
#pragma once
#include "internal.h"

#include <hip/hip_bf16.h>

namespace fftsp {

constexpr size_t kMostRows = (size_t)1 << 30;
constexpr uint32_t kMostWidth = 1u << 20;

inline int type_bytes(int type) { return type == 0 ? 4 : type == 1 || type == 2 ? 2 : 0; }

// The ABI's element types as types here; bits of the 16-bit ones are converted by hand where the hardware has no one
// instruction, so that NaN stays NaN and ties go to even.
struct Bf16 {
    uint16_t v;
};
struct F16 {
    _Float16 v;
};
__device__ __forceinline__ float to_float(float x) { return x; }
__device__ __forceinline__ float to_float(Bf16 x) { return __uint_as_float((uint32_t)x.v << 16); }
__device__ __forceinline__ float to_float(F16 x) { return (float)x.v; }
template <typename T>
__device__ __forceinline__ T from_float(float x);
template <>
__device__ __forceinline__ float from_float<float>(float x) { return x; }
template <>
__device__ __forceinline__ Bf16 from_float<Bf16>(float x)
{
    const __bf16 b = (__bf16)x;
    Bf16 r;
    __builtin_memcpy(&r, &b, 2);
    return r;
}
template <>
__device__ __forceinline__ F16 from_float<F16>(float x) { return F16{(_Float16)x}; }

// V elements with an element's alignment: the hardware takes such accesses of up to 16 bytes whole
template <typename T, int V>
struct Run {
    T v[V];
};
template <typename T, int V>
__device__ __forceinline__ Run<T, V> load_run(const T* p)
{
    Run<T, V> r;
    __builtin_memcpy(&r, p, sizeof(r));
    return r;
}
template <typename T, int V>
__device__ __forceinline__ void store_run(T* p, const Run<T, V>& r)
{
    __builtin_memcpy(p, &r, sizeof(r));
}

// f(type) with the type that an ABI code stands for
template <typename F>
inline hipError_t with_type(int type, F&& f)
{
    switch (type) {
        case 0: return f(float{});
        case 1: return f(Bf16{});
        default: return f(F16{});
    }
}

// embedding.hip
struct EmbeddingArgs {
    const void* source;  // the table, or the rows' gradients
    const void* tokens;
    void* out;           // the rows, or the table's gradient
    const void* base;    // gradient: what is added, or nullptr
    size_t rows, ntokens, source_stride, out_stride;
    uint32_t width;
    float scale;
    int source_type, out_type, token_bits;
};
hipError_t launch_embedding(const EmbeddingArgs& a, hipStream_t s);
size_t embedding_gradient_workspace(size_t rows, uint32_t width, size_t ntokens);
hipError_t launch_embedding_gradient(const EmbeddingArgs& a, uint8_t* ws, hipStream_t s);

// orthogonal.hip
constexpr int kPhaseMost = 2;  // steps that are taken on n x n matrices before X is
constexpr int kMostSteps = 16;
constexpr double kMostBound = 4096.0;  // of X's singular values and of a phase's polynomials of them
struct StepBounds {                   // largest singular values: X before each phase; A, P, P A, and the phase's product of P, by step
    int phases, end[kMostSteps];
    double x[kMostSteps], a[kMostSteps], p[kMostSteps], t[kMostSteps], q[kMostSteps];
};
// false: X's or a phase's are larger than kMostBound
bool step_bounds(const float* coefficients, int nsteps, int phase_steps, StepBounds* b);

struct OrthogonalArgs {
    const void* in;        // the matrices, or the gradient
    int in_type;
    void* out;             // their orthogonalised forms, or the new weights
    int out_type;
    // the step's, nullptr without one
    const float* momentum;
    float* momentum_out;
    const void* weights;
    float beta, lr, decay;  // decay: 1 - lr * weight_decay
    int nesterov;
    float eps;
    const float* coefficients;  // host, 3 per step
    int nsteps;
};
struct MatrixSpan {  // fftsp_matrix
    uint64_t offset, stride;
    uint32_t rows, cols;
    float gain;
    uint32_t reserved;
};
size_t orthogonal_workspace(const MatrixSpan* m, int count);
// *fits: the list's counts are within a launch's; *enough: so is the workspace.  Nothing is launched where one is false.
hipError_t launch_orthogonal(const OrthogonalArgs& a, const MatrixSpan* m, int count, uint8_t* ws, size_t ws_bytes, bool* fits, bool* enough,
                             hipStream_t s);

}  // namespace fftsp
