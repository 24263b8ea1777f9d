// Host side of the operators of a sparse layer (include/gcoo.h): argument checks, workspaces and launches.
#include "gcoo_layer.hpp"
#include "gcoo_layer_clip.hpp"
#include "gcoo_layer_values.hpp"

#include <algorithm>
#include <memory>
#include <new>

namespace {

size_t aligned(size_t bytes) { return (bytes + 255) / 256 * 256; }
bool known_type(int type) { return type == GCOO_F32 || type == GCOO_BF16 || type == GCOO_F16; }
bool known_activation(int act) { return act >= GCOO_ACT_NONE && act <= GCOO_ACT_GELU_TANH; }
bool on_elements(const void* p, int type) { return reinterpret_cast<uintptr_t>(p) % gcoo::type_bytes(type) == 0; }
bool on_floats(const void* p) { return reinterpret_cast<uintptr_t>(p) % 4 == 0; }
constexpr int64_t kMaxPitch = 0x3fffffff;

int check_work(const void* work, size_t given, size_t need)
{
    if (need == 0) return GCOO_OK;
    if (given < need) return GCOO_ENOMEM;
    return work && reinterpret_cast<uintptr_t>(work) % 256 == 0 ? GCOO_OK : GCOO_EINVAL;
}
int done(hipError_t e, const char* what) { return e == hipSuccess ? GCOO_OK : gcoo::hip_failed(e, what); }

// ---- the product with its epilogue ----

int check_product(const gcoo::RowsView& A, const void* B, int64_t ldb, int64_t N, const gcoo_epilogue* e, const void* C, int64_t ldc)
{
    if (!e || !known_type(e->type) || !known_activation(e->activation)) return GCOO_EINVAL;
    if (N < 0 || N > INT32_MAX || ldb < N || ldb > kMaxPitch || ldc < N) return GCOO_EINVAL;
    if ((e->residual && e->ldr < N) || (e->Z && e->ldz < N)) return GCOO_EINVAL;
    if (!on_elements(B, e->type) || !on_elements(C, e->type) || !on_elements(e->residual, e->type) || !on_elements(e->Z, e->type) || !on_floats(e->bias)) return GCOO_EINVAL;
    if (N == 0 || A.m == 0) return GCOO_OK;
    if (!C || (A.nnz > 0 && !B)) return GCOO_EINVAL;
    if (e->residual == C && e->residual && e->ldr != ldc) return GCOO_EINVAL;
    if (e->Z == C || C == B || (e->Z && (e->Z == B || e->Z == e->residual))) return GCOO_EINVAL;
    return GCOO_OK;
}

}  // namespace

extern "C" {

size_t gcoo_spdm_epilogue_bytes(const gcoo_matrix* A, const void* B_dev, int64_t ldb, int64_t N, const gcoo_epilogue* e, const void* C_dev, int64_t ldc)
{
    if (!A) return 0;
    const gcoo::RowsView v = gcoo::rows_view(A);
    return check_product(v, B_dev, ldb, N, e, C_dev, ldc) == GCOO_OK && N > 0 && v.m > 0 ? gcoo::product_plan(A, B_dev, ldb, N, e->type).work : 0;
}

int gcoo_spdm_epilogue(const gcoo_matrix* A, const void* B_dev, int64_t ldb, int64_t N, const gcoo_epilogue* e, void* C_dev, int64_t ldc,
                       void* work, size_t work_bytes, void* stream)
{
    if (!A) return GCOO_EINVAL;
    const gcoo::RowsView v = gcoo::rows_view(A);
    int rc = check_product(v, B_dev, ldb, N, e, C_dev, ldc);
    if (rc != GCOO_OK || N == 0 || v.m == 0) return rc;
    const gcoo::ProductPlan plan = gcoo::product_plan(A, B_dev, ldb, N, e->type);
    rc = check_work(work, work_bytes, plan.work);
    if (rc != GCOO_OK) return rc;
    const gcoo::EpilogueArgs args{e->bias, e->residual, e->ldr, e->Z, e->ldz, C_dev, ldc, e->type, e->activation};
    return done(gcoo::launch_product(A, plan, B_dev, ldb, N, args, work, static_cast<hipStream_t>(stream)), "product with its epilogue");
}

size_t gcoo_epilogue_grad_bytes(int64_t m, int64_t N)
{
    if (m < 0 || N < 0 || m > INT32_MAX || N > INT32_MAX) return 0;
    const int32_t parts = gcoo::epilogue_grad_parts(m, N);
    return parts > 1 ? aligned((size_t)parts * (size_t)m * 4) : 0;
}

int gcoo_epilogue_grad(int64_t m, int64_t N, int type, int activation, const void* Z_dev, int64_t ldz, const void* dC_dev, int64_t lddc,
                       void* dZ_dev, int64_t lddz, float* dbias_dev, void* work, size_t work_bytes, void* stream)
{
    if (m < 0 || N < 0 || m > INT32_MAX || N > INT32_MAX || !known_type(type) || !known_activation(activation)) return GCOO_EINVAL;
    if (lddc < N || (dZ_dev && lddz < N) || !on_elements(dC_dev, type) || !on_elements(dZ_dev, type) || !on_floats(dbias_dev)) return GCOO_EINVAL;
    const bool reads_z = activation != GCOO_ACT_NONE;
    if (reads_z && (ldz < N || !on_elements(Z_dev, type))) return GCOO_EINVAL;
    if (m == 0) return GCOO_OK;
    if (N > 0 && (!dC_dev || (reads_z && !Z_dev))) return GCOO_EINVAL;
    if (dZ_dev && ((dZ_dev == dC_dev && lddz != lddc) || (reads_z && dZ_dev == Z_dev && lddz != ldz))) return GCOO_EINVAL;
    const int rc = check_work(work, work_bytes, gcoo_epilogue_grad_bytes(m, N));
    if (rc != GCOO_OK || (!dbias_dev && (!dZ_dev || N == 0))) return rc;
    const gcoo::EpilogueGradArgs a{Z_dev, ldz, dC_dev, lddc, dZ_dev, lddz, dbias_dev, m, N, type, activation};
    return done(gcoo::launch_epilogue_grad(a, static_cast<float*>(work), static_cast<hipStream_t>(stream)), "layer_epilogue_grad launch");
}

}  // extern "C"

namespace {

int check_values(const gcoo::RowsView& A, const void* dZ, int64_t lddz, const void* B, int64_t ldb, int64_t N, int type)
{
    if (!known_type(type) || N < 0 || N > INT32_MAX || lddz < N || ldb < N || lddz > kMaxPitch || ldb > kMaxPitch) return GCOO_EINVAL;
    if (!on_elements(dZ, type) || !on_elements(B, type)) return GCOO_EINVAL;
    return N > 0 && A.nnz > 0 && (!dZ || !B) ? GCOO_EINVAL : GCOO_OK;
}

// Where the tiles of a row begin, then the sums of the parts, then a copy of B.
struct ValuesWork { size_t part, copy, total; };
ValuesWork values_work(const gcoo::RowsView& A, const gcoo::ValuesPlan& p, int type)
{
    ValuesWork w;
    w.part = aligned((size_t)p.starts * 4);
    w.copy = w.part + (p.parts > 1 ? aligned((size_t)p.group * (size_t)A.nnz * 4) : 0);
    w.total = w.copy + aligned((size_t)A.k * (size_t)p.ldw * gcoo::type_bytes(type));
    return w;
}

}  // namespace

extern "C" {

size_t gcoo_spdm_grad_values_bytes(const gcoo_matrix* A, const void* dZ_dev, int64_t lddz, const void* B_dev, int64_t ldb, int64_t N, int type)
{
    if (!A) return 0;
    const gcoo::RowsView v = gcoo::rows_view(A);
    if (check_values(v, dZ_dev, lddz, B_dev, ldb, N, type) != GCOO_OK || v.nnz == 0) return 0;
    return values_work(v, gcoo::values_plan(v.m, v.k, v.nnz, N, type, B_dev, ldb), type).total;
}

int gcoo_spdm_grad_values(const gcoo_matrix* A, const void* dZ_dev, int64_t lddz, const void* B_dev, int64_t ldb, int64_t N, int type,
                          float* dvals_dev, void* work, size_t work_bytes, void* stream)
{
    if (!A) return GCOO_EINVAL;
    const gcoo::RowsView v = gcoo::rows_view(A);
    int rc = check_values(v, dZ_dev, lddz, B_dev, ldb, N, type);
    if (rc != GCOO_OK) return rc;
    if (!on_floats(dvals_dev) || (v.nnz > 0 && !dvals_dev)) return GCOO_EINVAL;
    if (v.nnz == 0) return GCOO_OK;
    const gcoo::ValuesPlan plan = gcoo::values_plan(v.m, v.k, v.nnz, N, type, B_dev, ldb);
    const ValuesWork w = values_work(v, plan, type);
    rc = check_work(work, work_bytes, w.total);
    if (rc != GCOO_OK) return rc;
    const gcoo::GradValuesArgs a{v, dZ_dev, lddz, B_dev, ldb, N, type, dvals_dev};
    char* at = static_cast<char*>(work);
    return done(gcoo::launch_grad_values(a, plan, static_cast<int32_t*>(work), reinterpret_cast<float*>(at + w.part), at + w.copy, static_cast<hipStream_t>(stream)), "gradient of the values");
}

}  // extern "C"

// ---- clipping ----

namespace {

int64_t clip_pieces(int64_t count) { return (count + gcoo::kClipPiece - 1) / gcoo::kClipPiece; }

// The number of pieces of all tensors, or a status.
int64_t check_clip(const gcoo_gradient* list, int64_t tensors)
{
    if (tensors < 0 || tensors > INT32_MAX || (tensors > 0 && !list)) return GCOO_EINVAL;
    int64_t pieces = 0;
    for (int64_t i = 0; i < tensors; ++i) {
        const gcoo_gradient& t = list[i];
        if (!known_type(t.type) || t.count < 0 || t.count > INT64_MAX / 8) return GCOO_EINVAL;
        if (t.count > 0 && (!t.data || !t.out || !on_elements(t.data, t.type) || !on_elements(t.out, t.type))) return GCOO_EINVAL;
        pieces += clip_pieces(t.count);
        if (pieces > INT32_MAX) return GCOO_EINVAL;
    }
    return pieces;
}

// No `out`, and not the norm, overlaps another tensor or its own data, but as data itself: the ranges in the order of their addresses, those that are written marked.
int check_clip_ranges(const gcoo_gradient* list, int64_t tensors, const float* norm)
{
    struct Range { uintptr_t from, to; bool written; };
    std::unique_ptr<Range[]> r(new (std::nothrow) Range[2 * (size_t)tensors + 1]);
    if (!r) return GCOO_ENOMEM;
    const uintptr_t at = reinterpret_cast<uintptr_t>(norm);
    r[0] = {at, at + 4, true};
    size_t n = 1;
    for (int64_t i = 0; i < tensors; ++i) {
        const gcoo_gradient& t = list[i];
        if (t.count == 0) continue;
        const uintptr_t bytes = (uintptr_t)t.count * gcoo::type_bytes(t.type), o = reinterpret_cast<uintptr_t>(t.out), d = reinterpret_cast<uintptr_t>(t.data);
        if (o + bytes < o || d + bytes < d) return GCOO_EINVAL;
        r[n++] = {o, o + bytes, true};
        if (t.out != t.data) r[n++] = {d, d + bytes, false};
    }
    std::sort(r.get(), r.get() + n, [](const Range& a, const Range& b) { return a.from < b.from; });
    uintptr_t end_any = 0, end_written = 0;
    for (size_t i = 0; i < n; ++i) {
        if (r[i].from < end_written || (r[i].written && r[i].from < end_any)) return GCOO_EINVAL;
        end_any = std::max(end_any, r[i].to);
        if (r[i].written) end_written = std::max(end_written, r[i].to);
    }
    return GCOO_OK;
}

// How many launches the tensors are, and how many workgroups each has at the most.
struct ClipLaunches { int64_t launches, wgs; };
ClipLaunches clip_launches(const gcoo_gradient* list, int64_t tensors, int64_t pieces)
{
    int64_t full = 0;
    for (int64_t i = 0; i < tensors; ++i) full += list[i].count > 0;
    const int64_t launches = (full + gcoo::kClipTensors - 1) / gcoo::kClipTensors;
    if (launches <= 1 && pieces <= gcoo::kClipSmallPieces) return {1, 0};                       // by one workgroup
    return {launches, std::max<int64_t>(gcoo::kClipSums / launches, 64)};
}
// f(list of a launch) for the tensors, as many as a launch takes at a time.
template <typename F>
int each_clip_launch(const gcoo_gradient* list, int64_t tensors, int64_t most_wgs, F&& f)
{
    gcoo::ClipList l{};
    for (int64_t i = 0; i <= tensors; ++i) {
        if (l.tensors > 0 && (i == tensors || l.tensors == gcoo::kClipTensors)) {
            l.wgs = (int32_t)std::min<int64_t>(l.pieces, most_wgs);
            const int rc = f(l);
            if (rc != GCOO_OK) return rc;
            l.sum0 += l.wgs;
            l.tensors = l.pieces = 0;
        }
        if (i < tensors && list[i].count > 0) {
            l.t[l.tensors++] = {list[i].data, list[i].out, list[i].count, list[i].type, l.pieces};
            l.pieces += (int32_t)clip_pieces(list[i].count);
        }
    }
    return GCOO_OK;
}
}  // namespace

extern "C" {

size_t gcoo_clip_grad_norm_bytes(const gcoo_gradient* list, int64_t tensors)
{
    const int64_t pieces = check_clip(list, tensors);
    if (pieces <= 0) return 0;
    const ClipLaunches n = clip_launches(list, tensors, pieces);
    return aligned((size_t)(n.launches * n.wgs) * sizeof(double));
}

int gcoo_clip_grad_norm(const gcoo_gradient* list, int64_t tensors, float max_norm, float* norm_dev, void* work, size_t work_bytes, void* stream)
{
    const int64_t pieces = check_clip(list, tensors);
    if (pieces < 0) return (int)pieces;
    if (!norm_dev || !on_floats(norm_dev) || !(max_norm >= 0.0f)) return GCOO_EINVAL;
    int rc = check_clip_ranges(list, tensors, norm_dev);
    if (rc == GCOO_OK) rc = check_work(work, work_bytes, gcoo_clip_grad_norm_bytes(list, tensors));
    if (rc != GCOO_OK) return rc;
    hipStream_t s = static_cast<hipStream_t>(stream);
    double* sums = static_cast<double*>(work);
    if (pieces == 0) return done(gcoo::launch_clip_small(gcoo::ClipList{}, max_norm, norm_dev, s), "clip_small launch");
    const int64_t most = clip_launches(list, tensors, pieces).wgs;
    if (most == 0) return each_clip_launch(list, tensors, 0, [&](const gcoo::ClipList& l) { return done(gcoo::launch_clip_small(l, max_norm, norm_dev, s), "clip_small launch"); });
    int32_t sums_all = 0;
    rc = each_clip_launch(list, tensors, most, [&](const gcoo::ClipList& l) {
        sums_all = l.sum0 + l.wgs;
        return done(gcoo::launch_clip_sum(l, sums, s), "clip_sum launch");
    });
    if (rc != GCOO_OK) return rc;
    return each_clip_launch(list, tensors, most, [&](const gcoo::ClipList& l) {
        return done(gcoo::launch_clip_scale(l, sums, sums_all, max_norm, l.sum0 == 0 ? norm_dev : nullptr, s), "clip_scale launch");
    });
}

}  // extern "C"
