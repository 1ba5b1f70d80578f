// C ABI of the embedding and the orthogonalised update (see include/fftsp.h): argument checks and launches.
#include "../../include/fftsp.h"
#include "layers.h"

#include <algorithm>
#include <cmath>
#include <cstddef>
#include <vector>

using namespace fftsp;

namespace {

static_assert(sizeof(fftsp_matrix) == sizeof(MatrixSpan) && offsetof(fftsp_matrix, stride) == offsetof(MatrixSpan, stride) &&
              offsetof(fftsp_matrix, rows) == offsetof(MatrixSpan, rows) && offsetof(fftsp_matrix, cols) == offsetof(MatrixSpan, cols) &&
              offsetof(fftsp_matrix, gain) == offsetof(MatrixSpan, gain) && offsetof(fftsp_matrix, reserved) == offsetof(MatrixSpan, reserved),
              "one layout");

constexpr size_t kMostStride = (size_t)1 << 40, kMostTokens = (size_t)1 << 30, kMostSorted = (size_t)1 << 24;
constexpr uint64_t kMostElements = (uint64_t)1 << 48;  // from an array's first to its last
constexpr uint32_t kMostShort = 16384, kMostLong = 1u << 20;

bool aligned_to(const void* p, int bytes) { return reinterpret_cast<uintptr_t>(p) % (uintptr_t)bytes == 0; }

struct Span {
    uintptr_t begin, end;
};
Span span_of(const void* p, uint64_t first, uint64_t last, int bytes)  // elements [first, last)
{
    const uintptr_t b = reinterpret_cast<uintptr_t>(p);
    return Span{b + first * (uint64_t)bytes, b + last * (uint64_t)bytes};
}
bool meet(const Span& a, const Span& b) { return a.begin < b.end && b.begin < a.end; }

uint64_t rows_end(size_t rows, uint32_t width, size_t stride) { return rows ? (uint64_t)(rows - 1) * stride + width : 0; }
bool too_far(size_t rows, size_t stride) { return rows > 1 && rows - 1 > kMostElements / stride; }

int check_embedding(const EmbeddingArgs& a, size_t source_rows, size_t out_rows)
{
    const int sb = type_bytes(a.source_type), ob = type_bytes(a.out_type);
    if (!sb || !ob || (a.token_bits != 32 && a.token_bits != 64)) return FFTSP_EINVAL;
    if (a.rows < 1 || a.rows > kMostRows || a.width < 1 || a.width > kMostWidth || a.ntokens > kMostTokens) return FFTSP_EINVAL;
    if (a.source_stride < a.width || a.out_stride < a.width || a.source_stride > kMostStride || a.out_stride > kMostStride)
        return FFTSP_EINVAL;
    if (too_far(source_rows, a.source_stride) || too_far(out_rows, a.out_stride)) return FFTSP_EINVAL;
    if (!std::isfinite(a.scale)) return FFTSP_EINVAL;
    if ((source_rows && !a.source) || (out_rows && !a.out) || (a.ntokens && !a.tokens)) return FFTSP_EINVAL;
    if (!aligned_to(a.source, sb) || !aligned_to(a.out, ob) || !aligned_to(a.base, ob) || !aligned_to(a.tokens, a.token_bits / 8))
        return FFTSP_EINVAL;
    const Span out = span_of(a.out, 0, rows_end(out_rows, a.width, a.out_stride), ob);
    if (meet(out, span_of(a.source, 0, rows_end(source_rows, a.width, a.source_stride), sb)) ||
        meet(out, span_of(a.tokens, 0, a.ntokens, a.token_bits / 8)))
        return FFTSP_EINVAL;
    if (a.base && a.base != a.out && meet(out, span_of(a.base, 0, rows_end(out_rows, a.width, a.out_stride), ob))) return FFTSP_EINVAL;
    return FFTSP_OK;
}

uint64_t matrix_end(const fftsp_matrix& m) { return m.offset + (uint64_t)(m.rows - 1) * m.stride + m.cols; }

// elements that two matrices of a list share
bool share(const fftsp_matrix& a, const fftsp_matrix& b)  // a.offset <= b.offset
{
    if (b.offset >= matrix_end(a)) return false;
    if (a.stride != b.stride) return true;  // could be disjoint all the same: refused
    const uint64_t d = (b.offset - a.offset) % a.stride;
    return !(d >= a.cols && d + b.cols <= a.stride);
}

// *first, *last: the elements of an array that the list reaches
int check_matrices(const fftsp_matrix* m, int count, uint64_t* first, uint64_t* last)
{
    if (count < 0 || (count > 0 && !m)) return FFTSP_EINVAL;
    *first = UINT64_MAX;
    *last = 0;
    for (int i = 0; i < count; ++i) {
        if (m[i].rows < 1 || m[i].cols < 1 || m[i].stride < m[i].cols || m[i].stride > kMostStride || m[i].reserved ||
            m[i].offset > kMostElements || !std::isfinite(m[i].gain))
            return FFTSP_EINVAL;
        if (std::min(m[i].rows, m[i].cols) > kMostShort || std::max(m[i].rows, m[i].cols) > kMostLong) return FFTSP_EUNSUPPORTED;
        *first = std::min<uint64_t>(*first, m[i].offset);
        *last = std::max<uint64_t>(*last, matrix_end(m[i]));
    }
    // in the order of their first elements, each against those that reach behind its own first element
    std::vector<int> order((size_t)count), open;
    for (int i = 0; i < count; ++i) order[(size_t)i] = i;
    std::sort(order.begin(), order.end(), [&](int x, int y) { return m[x].offset < m[y].offset; });
    for (int i : order) {
        open.erase(std::remove_if(open.begin(), open.end(), [&](int j) { return matrix_end(m[j]) <= m[i].offset; }), open.end());
        for (int j : open)
            if (share(m[j], m[i])) return FFTSP_EINVAL;
        open.push_back(i);
    }
    return FFTSP_OK;
}

static_assert(kMostSteps == FFTSP_MAX_STEPS, "one limit");
const float kDefaultSteps[5][3] = {{3.4445f, -4.7750f, 2.0315f}, {3.4445f, -4.7750f, 2.0315f}, {3.4445f, -4.7750f, 2.0315f},
                                   {3.4445f, -4.7750f, 2.0315f}, {3.4445f, -4.7750f, 2.0315f}};

int check_steps(OrthogonalArgs* a, const float* coefficients, int nsteps, float eps)
{
    if (!(eps >= 0.f) || !std::isfinite(eps)) return FFTSP_EINVAL;
    a->eps = eps;
    a->coefficients = coefficients ? coefficients : &kDefaultSteps[0][0];
    a->nsteps = coefficients ? nsteps : 5;
    if (a->nsteps < 1 || a->nsteps > FFTSP_MAX_STEPS) return FFTSP_EINVAL;
    for (int i = 0; i < 3 * a->nsteps; ++i)
        if (!std::isfinite(a->coefficients[i])) return FFTSP_EINVAL;
    StepBounds bounds;
    return step_bounds(a->coefficients, a->nsteps, 1, &bounds) ? FFTSP_OK : FFTSP_EUNSUPPORTED;
}

int run_orthogonal(const OrthogonalArgs& a, const fftsp_matrix* m, int count, void* ws, size_t ws_bytes, fftsp_stream_t stream)
{
    const MatrixSpan* spans = reinterpret_cast<const MatrixSpan*>(m);
    if (!ws || !aligned16(ws)) return FFTSP_EINVAL;
    bool fits = false, enough = false;
    const hipError_t e = launch_orthogonal(a, spans, count, static_cast<uint8_t*>(ws), ws_bytes, &fits, &enough, reinterpret_cast<hipStream_t>(stream));
    if (e != hipSuccess) return FFTSP_EHIP;
    return !fits ? FFTSP_EUNSUPPORTED : !enough ? FFTSP_EWORKSPACE : FFTSP_OK;
}

// no exception leaves an entry point: the host's lists could not be allocated
template <typename F>
int guarded(F&& f)
{
    try {
        return f();
    } catch (...) {
        return FFTSP_EHIP;
    }
}

}  // namespace

extern "C" {

int fftsp_embedding(const void* d_table, int table_type, size_t rows, uint32_t width, size_t table_stride, const void* d_tokens,
                    int token_bits, size_t ntokens, float scale, void* d_out, int out_type, size_t out_stride, fftsp_stream_t stream)
{
    const EmbeddingArgs a{d_table, d_tokens, d_out, nullptr, rows, ntokens, table_stride, out_stride, width, scale, table_type, out_type, token_bits};
    const int rc = check_embedding(a, rows, ntokens);
    if (rc || ntokens == 0) return rc;
    return launch_embedding(a, reinterpret_cast<hipStream_t>(stream)) == hipSuccess ? FFTSP_OK : FFTSP_EHIP;
}

size_t fftsp_workspace_bytes_embedding(size_t rows, uint32_t width, size_t ntokens)
{
    if (rows < 1 || rows > kMostRows || width < 1 || width > kMostWidth || ntokens > kMostSorted) return 0;
    return embedding_gradient_workspace(rows, width, ntokens);
}

int fftsp_embedding_gradient(const void* d_out_grad, int out_type, size_t out_stride, const void* d_tokens, int token_bits, size_t ntokens,
                             float scale, const void* d_base, void* d_table_grad, int table_type, size_t rows, uint32_t width,
                             size_t table_stride, void* d_workspace, size_t workspace_bytes, fftsp_stream_t stream)
{
    const EmbeddingArgs a{d_out_grad, d_tokens, d_table_grad, d_base, rows, ntokens, out_stride, table_stride, width, scale, out_type, table_type, token_bits};
    const int rc = check_embedding(a, ntokens, rows);
    if (rc) return rc;
    if (ntokens > kMostSorted) return FFTSP_EUNSUPPORTED;
    if (ntokens) {
        if (!d_workspace || !aligned16(d_workspace)) return FFTSP_EINVAL;
        if (workspace_bytes < embedding_gradient_workspace(rows, width, ntokens)) return FFTSP_EWORKSPACE;
    }
    return launch_embedding_gradient(a, static_cast<uint8_t*>(d_workspace), reinterpret_cast<hipStream_t>(stream)) == hipSuccess ? FFTSP_OK
                                                                                                                                 : FFTSP_EHIP;
}

size_t fftsp_workspace_bytes_orthogonal(const fftsp_matrix* matrices, int nmat)
{
    size_t bytes = 0;
    guarded([&] {
        uint64_t first, last;
        const int rc = check_matrices(matrices, nmat, &first, &last);
        if (!rc) bytes = orthogonal_workspace(reinterpret_cast<const MatrixSpan*>(matrices), nmat);
        return rc;
    });
    return bytes;
}

int fftsp_orthogonal(const void* d_in, int in_type, void* d_out, int out_type, const fftsp_matrix* matrices, int nmat,
                     const float* coefficients, int nsteps, float eps, void* d_workspace, size_t workspace_bytes, fftsp_stream_t stream)
{
    return guarded([&] {
        OrthogonalArgs a{};
        a.in = d_in;
        a.in_type = in_type;
        a.out = d_out;
        a.out_type = out_type;
        const int ib = type_bytes(in_type), ob = type_bytes(out_type);
        uint64_t first, last;
        int rc = check_matrices(matrices, nmat, &first, &last);
        if (!rc) rc = check_steps(&a, coefficients, nsteps, eps);
        if (rc) return rc;
        if (!ib || !ob) return (int)FFTSP_EINVAL;
        if (nmat == 0) return (int)FFTSP_OK;
        if (!d_in || !d_out || !aligned_to(d_in, ib) || !aligned_to(d_out, ob)) return (int)FFTSP_EINVAL;
        if (!(d_in == d_out && in_type == out_type) && meet(span_of(d_in, first, last, ib), span_of(d_out, first, last, ob))) return (int)FFTSP_EINVAL;
        return run_orthogonal(a, matrices, nmat, d_workspace, workspace_bytes, stream);
    });
}

int fftsp_orthogonal_step(const void* d_grad, int grad_type, const float* d_momentum, float* d_momentum_out, const void* d_weights,
                          void* d_weights_out, int weight_type, const fftsp_matrix* matrices, int nmat, const fftsp_step* step,
                          void* d_workspace, size_t workspace_bytes, fftsp_stream_t stream)
{
    return guarded([&] {
        if (!step) return (int)FFTSP_EINVAL;
        OrthogonalArgs a{};
        a.in = d_grad;
        a.in_type = grad_type;
        a.out = d_weights_out;
        a.out_type = weight_type;
        a.momentum = d_momentum;
        a.momentum_out = d_momentum_out;
        a.weights = d_weights;
        a.beta = step->beta;
        a.lr = step->lr;
        a.decay = (float)(1.0 - (double)step->lr * (double)step->weight_decay);
        a.nesterov = step->nesterov != 0;
        const int gb = type_bytes(grad_type), wb = type_bytes(weight_type);
        uint64_t first, last;
        int rc = check_matrices(matrices, nmat, &first, &last);
        if (!rc) rc = check_steps(&a, step->coefficients, step->nsteps, step->eps);
        if (rc) return rc;
        if (!gb || !wb || !(step->beta >= 0.f && step->beta <= 1.f) || !std::isfinite(step->lr) || !std::isfinite(step->weight_decay) ||
            !std::isfinite(a.decay))
            return (int)FFTSP_EINVAL;
        if (nmat == 0) return (int)FFTSP_OK;
        if (!d_grad || !d_momentum || !d_momentum_out || !d_weights || !d_weights_out || !aligned_to(d_grad, gb) ||
            !aligned_to(d_momentum, 4) || !aligned_to(d_momentum_out, 4) || !aligned_to(d_weights, wb) || !aligned_to(d_weights_out, wb))
            return (int)FFTSP_EINVAL;
        const Span g = span_of(d_grad, first, last, gb), mi = span_of(d_momentum, first, last, 4), mo = span_of(d_momentum_out, first, last, 4),
                   wi = span_of(d_weights, first, last, wb), wo = span_of(d_weights_out, first, last, wb);
        if ((d_momentum != d_momentum_out && meet(mi, mo)) || (d_weights != d_weights_out && meet(wi, wo)) || meet(g, mo) || meet(g, wo) ||
            meet(mi, wo) || meet(mo, wi) || meet(mo, wo))
            return (int)FFTSP_EINVAL;
        return run_orthogonal(a, matrices, nmat, d_workspace, workspace_bytes, stream);
    });
}

}  // extern "C"
