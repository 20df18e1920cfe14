// C ABI of the operators on learned tables and layers: the checks of their
// arguments.  Declarations and contracts: include/sqn.h.
#include <math.h>

#include "learn.h"
#include "numeric.h"
#include "sqn_internal.h"

namespace {

using sqn::element_size;
using sqn::fail;

constexpr int64_t kMaxRows = (int64_t{1} << 31) - 1;
constexpr int64_t kMaxCols = int64_t{1} << 20;
constexpr int64_t kMaxIndices = int64_t{1} << 30;      // of a gradient: a launch's threads
constexpr int64_t kMaxTiles = int64_t{1} << 23;        // of a product: the same
constexpr int32_t kMaxSide = 32768;
constexpr int32_t kMaxBatch = 65535;
constexpr int64_t kMaxStride = int64_t{1} << 40;
constexpr int32_t kMaxSteps = 64;

bool valid_dtype(int32_t dt) { return dt == SQN_F32 || dt == SQN_F16 || dt == SQN_BF16; }

// Whether the process sees more than one device: of one, nothing lies on
// another, and the queries below (0.5 us of a lookup's 8.8 us call) are left out.
bool several_devices()
{
    static const bool several = [] {
        int count = 0;
        if (hipGetDeviceCount(&count) == hipSuccess)
            return count > 1;
        (void)hipGetLastError();
        return false;
    }();
    return several;
}

// The memory is there, and the current device's own: a launch goes to that
// device, and nothing orders it with another's streams.
sqn_status check_memory(const void* p, size_t bytes, const char* what)
{
    const sqn_status s = sqn::check_device_range(p, bytes, what);
    if (s != SQN_OK || !several_devices())
        return s;
    int current = 0, device = 0;
    if (hipGetDevice(&current) != hipSuccess)
        return fail(SQN_ERR_DEVICE, "hipGetDevice failed");
    if (hipPointerGetAttribute(&device, HIP_POINTER_ATTRIBUTE_DEVICE_ORDINAL, const_cast<void*>(p)) != hipSuccess) {
        (void)hipGetLastError();
        return fail(SQN_ERR_INVALID_ARG, "%s (%p): its device is not known", what, p);
    }
    if (device != current)
        return fail(SQN_ERR_INVALID_ARG, "%s lives on device %d, current device is %d", what, device, current);
    return SQN_OK;
}

sqn_status check_stream(void* stream)
{
    if (!stream || stream == hipStreamPerThread || !several_devices())
        return SQN_OK;                // those two are the current device's
    int current = 0;
    hipDevice_t device = 0;
    if (hipGetDevice(&current) != hipSuccess)
        return fail(SQN_ERR_DEVICE, "hipGetDevice failed");
    if (hipStreamGetDevice(static_cast<hipStream_t>(stream), &device) != hipSuccess) {
        (void)hipGetLastError();
        return fail(SQN_ERR_INVALID_ARG, "stream (%p): its device is not known", stream);
    }
    if (device != current)
        return fail(SQN_ERR_INVALID_ARG, "stream belongs to device %d, current device is %d", static_cast<int>(device),
                    current);
    return SQN_OK;
}

// The matrix's description, then that its memory is there.
sqn_status check_matrix(const sqn_matrix* x, bool written, const char* what)
{
    if (!x)
        return fail(SQN_ERR_INVALID_ARG, "%s is NULL", what);
    if (!valid_dtype(x->dtype))
        return fail(SQN_ERR_INVALID_ARG, "%s: dtype must be SQN_F32, SQN_F16 or SQN_BF16", what);
    if (x->reserved != 0)
        return fail(SQN_ERR_INVALID_ARG, "%s: reserved must be 0", what);
    if (x->rows < 0 || x->rows > kMaxRows || x->cols < 1 || x->cols > kMaxCols)
        return fail(SQN_ERR_INVALID_ARG, "%s: %lld x %lld outside [0, 2^31) x [1, 2^20]", what,
                    static_cast<long long>(x->rows), static_cast<long long>(x->cols));
    if (x->row_stride < (written ? x->cols : 0) || x->row_stride > kMaxStride)
        return fail(SQN_ERR_INVALID_ARG, "%s: row stride %lld for %lld columns", what,
                    static_cast<long long>(x->row_stride), static_cast<long long>(x->cols));
    if (x->rows == 0)
        return SQN_OK;
    const unsigned __int128 bytes
        = (static_cast<unsigned __int128>(x->rows - 1) * x->row_stride + x->cols) * element_size(x->dtype);
    if (bytes >> 63)
        return fail(SQN_ERR_INVALID_ARG, "%s spans more than 2^63 bytes", what);
    if (reinterpret_cast<uintptr_t>(x->data) % element_size(x->dtype))
        return fail(SQN_ERR_INVALID_ARG, "%s (%p) is not aligned to its elements", what, x->data);
    return check_memory(x->data, static_cast<size_t>(bytes), what);
}

sqn_status check_ids(const void* ids, int32_t type, int64_t n)
{
    if (type != SQN_I32 && type != SQN_I64)
        return fail(SQN_ERR_INVALID_ARG, "ids_type must be SQN_I32 or SQN_I64");
    if (n == 0)
        return SQN_OK;
    const size_t size = type == SQN_I64 ? 8 : 4;
    if (reinterpret_cast<uintptr_t>(ids) % size)
        return fail(SQN_ERR_INVALID_ARG, "ids (%p) is not aligned to its elements", ids);
    return check_memory(ids, static_cast<size_t>(n) * size, "ids");
}

sqn_status check_workspace(const void* workspace, size_t bytes, size_t need)
{
    if (need == 0)
        return SQN_OK;
    if (bytes < need)
        return fail(SQN_ERR_INVALID_ARG, "workspace of %zu bytes, %zu are needed", bytes, need);
    if (reinterpret_cast<uintptr_t>(workspace) % 256)
        return fail(SQN_ERR_INVALID_ARG, "workspace (%p) is not aligned to 256 bytes", workspace);
    return check_memory(workspace, need, "workspace");
}

// The batch's description and the elements it spans.
sqn_status check_batch(const sqn_batch* x, const char* what)
{
    if (!x)
        return fail(SQN_ERR_INVALID_ARG, "%s is NULL", what);
    if (!valid_dtype(x->dtype))
        return fail(SQN_ERR_INVALID_ARG, "%s: dtype must be SQN_F32, SQN_F16 or SQN_BF16", what);
    if (x->batch < 0 || x->batch > kMaxBatch || x->rows < 1 || x->rows > kMaxSide || x->cols < 1 || x->cols > kMaxSide)
        return fail(SQN_ERR_INVALID_ARG, "%s: %d of %d x %d outside [0, 65535] of [1, 32768]^2", what, x->batch, x->rows,
                    x->cols);
    const int64_t strides[3] = {x->batch_stride, x->row_stride, x->col_stride};
    for (int64_t s : strides)
        if (s < 0 || s > kMaxStride)
            return fail(SQN_ERR_INVALID_ARG, "%s: stride %lld outside [0, 2^40]", what, static_cast<long long>(s));
    if (x->batch == 0)
        return SQN_OK;
    const unsigned __int128 bytes
        = (static_cast<unsigned __int128>(x->batch - 1) * x->batch_stride
           + static_cast<unsigned __int128>(x->rows - 1) * x->row_stride
           + static_cast<unsigned __int128>(x->cols - 1) * x->col_stride + 1) * element_size(x->dtype);
    if (bytes >> 63)
        return fail(SQN_ERR_INVALID_ARG, "%s spans more than 2^63 bytes", what);
    if (reinterpret_cast<uintptr_t>(x->data) % element_size(x->dtype))
        return fail(SQN_ERR_INVALID_ARG, "%s (%p) is not aligned to its elements", what, x->data);
    return check_memory(x->data, static_cast<size_t>(bytes), what);
}

// No two elements of a written batch at one place: each axis, from the one
// with the smallest stride on, starts past all that lies within it.
bool elements_apart(const sqn_batch* x)
{
    int64_t size[3] = {x->batch, x->rows, x->cols};
    int64_t stride[3] = {x->batch_stride, x->row_stride, x->col_stride};
    int64_t span = 1;
    for (int done = 0; done < 3; ++done) {
        int k = -1;
        for (int r = 0; r < 3; ++r)
            if (size[r] > 1 && (k < 0 || stride[r] < stride[k]))
                k = r;
        if (k < 0)
            return true;
        if (stride[k] < span)
            return false;
        span += (size[k] - 1) * stride[k];
        size[k] = 1;
    }
    return true;
}

// Most that |a s + b s^3 + c s^5| reaches for s in [0, most].
double reached(double a, double b, double c, double most)
{
    auto p = [&](double s) { return fabs(s * (a + s * s * (b + s * s * c))); };
    double top = p(most);
    auto at = [&](double t) {      // a zero of a + 3 b t + 5 c t^2, t = s^2
        if (t > 0.0 && t < most * most)
            top = fmax(top, p(sqrt(t)));
    };
    if (c != 0.0) {
        const double disc = 9.0 * b * b - 20.0 * a * c;
        if (disc >= 0.0) {
            at((-3.0 * b + sqrt(disc)) / (10.0 * c));
            at((-3.0 * b - sqrt(disc)) / (10.0 * c));
        }
    } else if (b != 0.0) {
        at(-a / (3.0 * b));
    }
    return top;
}

// Whether X, A and b A + c A A stay in the range that their binary16 factors
// are scaled for, whatever the matrix.
sqn_status check_coefficients(const float k[3], int32_t steps)
{
    if (!k)
        return fail(SQN_ERR_INVALID_ARG, "coefficients is NULL");
    for (int r = 0; r < 3; ++r)
        if (!isfinite(k[r]))
            return fail(SQN_ERR_INVALID_ARG, "coefficients[%d] is not finite", r);
    double most = 1.0;
    for (int32_t s = 0; s < steps; ++s) {
        const double t = most * most;
        double middle = fabs(k[1] * t + k[2] * t * t);
        if (k[2] != 0.0f) {
            const double top = -static_cast<double>(k[1]) / (2.0 * k[2]);
            if (top > 0.0 && top < t)
                middle = fmax(middle, fabs(k[1] * top + k[2] * top * top));
        }
        if (middle > 16.0)
            return fail(SQN_ERR_INVALID_ARG, "coefficients (%g, %g, %g): b s^2 + c s^4 reaches %g (16 at most)",
                        static_cast<double>(k[0]), static_cast<double>(k[1]), static_cast<double>(k[2]), middle);
        const double next = reached(k[0], k[1], k[2], most);
        if (next > 2.0)
            return fail(SQN_ERR_INVALID_ARG, "coefficients (%g, %g, %g): a singular value may reach %g (2 at most)",
                        static_cast<double>(k[0]), static_cast<double>(k[1]), static_cast<double>(k[2]), next);
        most = fmax(most, next);
    }
    return SQN_OK;
}

sqn_status check_quantised(const sqn_quantised* x, const char* what)
{
    if (!x)
        return fail(SQN_ERR_INVALID_ARG, "%s is NULL", what);
    if (x->rows < 0 || x->rows > kMaxRows || x->cols < 1 || x->cols > kMaxCols)
        return fail(SQN_ERR_INVALID_ARG, "%s: %lld x %lld outside [0, 2^31) x [1, 2^20]", what,
                    static_cast<long long>(x->rows), static_cast<long long>(x->cols));
    if (x->rows == 0)
        return SQN_OK;
    if (reinterpret_cast<uintptr_t>(x->codes) % 16)
        return fail(SQN_ERR_INVALID_ARG, "%s: codes (%p) are not aligned to 16 bytes", what, x->codes);
    const size_t blocks = static_cast<size_t>(x->rows) * sqn::quant_blocks(x->cols);
    sqn_status s = check_memory(x->codes, 16 * blocks, what);
    if (s != SQN_OK)
        return s;
    return check_memory(x->scales, blocks, what);
}

// Everything of a product but its first factor, [points][cols].
sqn_status check_layer(int64_t points, int64_t cols, const sqn_quantised* w, const float* bias, int32_t relu,
                       const sqn_matrix* out)
{
    sqn_status s = check_quantised(w, "w");
    if (s != SQN_OK)
        return s;
    if ((s = check_matrix(out, true, "out")) != SQN_OK)
        return s;
    if (cols != w->cols)
        return fail(SQN_ERR_INVALID_ARG, "x has %lld columns, w %lld", static_cast<long long>(cols),
                    static_cast<long long>(w->cols));
    if (w->rows < 1)
        return fail(SQN_ERR_INVALID_ARG, "w has no rows");
    if (out->rows != points || out->cols != w->rows)
        return fail(SQN_ERR_INVALID_ARG, "out is %lld x %lld, the product %lld x %lld", static_cast<long long>(out->rows),
                    static_cast<long long>(out->cols), static_cast<long long>(points), static_cast<long long>(w->rows));
    if (relu != 0 && relu != 1)
        return fail(SQN_ERR_INVALID_ARG, "relu must be 0 or 1");
    if (((points + 63) / 64) * ((w->rows + 63) / 64) > kMaxTiles)
        return fail(SQN_ERR_UNSUPPORTED, "a product of %lld x %lld has more than 2^23 tiles of 64 x 64",
                    static_cast<long long>(points), static_cast<long long>(w->rows));
    if (bias) {
        if (reinterpret_cast<uintptr_t>(bias) % 4)
            return fail(SQN_ERR_INVALID_ARG, "bias (%p) is not aligned to its elements", static_cast<const void*>(bias));
        return check_memory(bias, static_cast<size_t>(w->rows) * 4, "bias");
    }
    return SQN_OK;
}

bool valid_layer(int64_t points, int64_t units, int64_t cols)
{
    return points >= 0 && points <= kMaxRows && units >= 1 && units <= kMaxRows && cols >= 1 && cols <= kMaxCols;
}

sqn_status launched(hipError_t e, const char* what)
{
    return e == hipSuccess ? SQN_OK : fail(SQN_ERR_DEVICE, "%s launch failed: %s", what, hipGetErrorString(e));
}

}  // namespace

extern "C" {

sqn_status sqn_lookup(const sqn_matrix* table, const void* ids, int32_t ids_type, float scale, const sqn_matrix* out,
                      void* stream)
{
    sqn_status s = check_stream(stream);
    if (s != SQN_OK)
        return s;
    if ((s = check_matrix(table, false, "table")) != SQN_OK)
        return s;
    if ((s = check_matrix(out, true, "out")) != SQN_OK)
        return s;
    if (out->dtype != table->dtype || out->cols != table->cols)
        return fail(SQN_ERR_INVALID_ARG, "out must have the table's dtype and columns");
    if ((s = check_ids(ids, ids_type, out->rows)) != SQN_OK)
        return s;
    if (out->rows == 0)
        return SQN_OK;
    return launched(sqn::launch_lookup(*table, ids, ids_type == SQN_I64, scale, *out, static_cast<hipStream_t>(stream)),
                    "lookup");
}

size_t sqn_lookup_gradient_workspace(int64_t n_ids, int64_t rows, int64_t cols)
{
    if (n_ids < 0 || n_ids > kMaxIndices || rows < 1 || rows > kMaxRows || cols < 1 || cols > kMaxCols)
        return 0;
    return sqn::lookup_gradient_bytes(n_ids, rows, cols);
}

sqn_status sqn_lookup_gradient(const sqn_matrix* grad, const void* ids, int32_t ids_type, float scale,
                               int32_t accumulate, const sqn_matrix* table_grad, void* workspace, size_t workspace_bytes,
                               void* stream)
{
    sqn_status s = check_stream(stream);
    if (s != SQN_OK)
        return s;
    if ((s = check_matrix(grad, false, "grad")) != SQN_OK)
        return s;
    if ((s = check_matrix(table_grad, true, "table_grad")) != SQN_OK)
        return s;
    if (grad->rows > kMaxIndices)
        return fail(SQN_ERR_INVALID_ARG, "%lld indices, at most 2^30", static_cast<long long>(grad->rows));
    if (table_grad->rows < 1 || table_grad->cols != grad->cols)
        return fail(SQN_ERR_INVALID_ARG, "table_grad must have a row and the gradient's columns");
    if (accumulate != 0 && accumulate != 1)
        return fail(SQN_ERR_INVALID_ARG, "accumulate must be 0 or 1");
    if ((s = check_ids(ids, ids_type, grad->rows)) != SQN_OK)
        return s;
    if ((s = check_workspace(workspace, workspace_bytes,
                             sqn::lookup_gradient_bytes(grad->rows, table_grad->rows, grad->cols))) != SQN_OK)
        return s;
    return launched(sqn::launch_lookup_gradient(*grad, ids, ids_type == SQN_I64, scale, accumulate != 0, *table_grad,
                                                workspace, static_cast<hipStream_t>(stream)),
                    "lookup gradient");
}

size_t sqn_orthogonalise_workspace(int32_t batch, int32_t rows, int32_t cols, int32_t out_dtype)
{
    if (batch < 1 || batch > kMaxBatch || rows < 1 || rows > kMaxSide || cols < 1 || cols > kMaxSide
        || !valid_dtype(out_dtype))
        return 0;
    return sqn::orthogonalise_bytes(batch, rows, cols, out_dtype);
}

sqn_status sqn_orthogonalise(const sqn_batch* updates, int32_t steps, const float coefficients[3], float eps,
                             const sqn_batch* out, void* workspace, size_t workspace_bytes, void* stream)
{
    if (steps < 0 || steps > kMaxSteps)
        return fail(SQN_ERR_INVALID_ARG, "steps = %d outside [0, 64]", steps);
    if (!isfinite(eps) || eps < 0.0f)
        return fail(SQN_ERR_INVALID_ARG, "eps must be finite and >= 0");
    sqn_status s = check_coefficients(coefficients, steps);
    if (s != SQN_OK)
        return s;
    if ((s = check_stream(stream)) != SQN_OK)
        return s;
    if ((s = check_batch(updates, "updates")) != SQN_OK)
        return s;
    if ((s = check_batch(out, "out")) != SQN_OK)
        return s;
    if (out->batch != updates->batch || out->rows != updates->rows || out->cols != updates->cols)
        return fail(SQN_ERR_INVALID_ARG, "out is %d of %d x %d, the updates %d of %d x %d", out->batch, out->rows,
                    out->cols, updates->batch, updates->rows, updates->cols);
    if (!elements_apart(out))
        return fail(SQN_ERR_INVALID_ARG, "out: two elements at one place");
    if (updates->batch == 0)
        return SQN_OK;
    if ((s = check_workspace(workspace, workspace_bytes,
                             sqn::orthogonalise_bytes(updates->batch, updates->rows, updates->cols, out->dtype)))
        != SQN_OK)
        return s;
    return launched(sqn::launch_orthogonalise(*updates, steps, coefficients, eps, *out, workspace,
                                              static_cast<hipStream_t>(stream)),
                    "orthogonalise");
}

sqn_status sqn_quantise(const sqn_matrix* x, const sqn_quantised* out, void* stream)
{
    sqn_status s = check_stream(stream);
    if (s != SQN_OK)
        return s;
    if ((s = check_matrix(x, false, "x")) != SQN_OK)
        return s;
    if ((s = check_quantised(out, "out")) != SQN_OK)
        return s;
    if (out->rows != x->rows || out->cols != x->cols)
        return fail(SQN_ERR_INVALID_ARG, "out must have x's rows and columns");
    if (x->rows == 0)
        return SQN_OK;
    return launched(sqn::launch_quantise(*x, *out, static_cast<hipStream_t>(stream)), "quantise");
}

sqn_status sqn_quantised_values(const sqn_quantised* x, const sqn_matrix* out, void* stream)
{
    sqn_status s = check_stream(stream);
    if (s != SQN_OK)
        return s;
    if ((s = check_quantised(x, "x")) != SQN_OK)
        return s;
    if ((s = check_matrix(out, true, "out")) != SQN_OK)
        return s;
    if (out->rows != x->rows || out->cols != x->cols)
        return fail(SQN_ERR_INVALID_ARG, "out must have x's rows and columns");
    if (x->rows == 0)
        return SQN_OK;
    return launched(sqn::launch_quantised_values(*x, *out, static_cast<hipStream_t>(stream)), "values");
}

size_t sqn_quantised_product_workspace(int64_t points, int64_t units, int64_t cols)
{
    if (!valid_layer(points, units, cols))
        return 0;
    return sqn::quantised_product_bytes(points, units, cols);
}

sqn_status sqn_quantised_product(const sqn_quantised* x, const sqn_quantised* w, const float* bias, int32_t relu,
                                 const sqn_matrix* out, void* workspace, size_t workspace_bytes, void* stream)
{
    sqn_status s = check_stream(stream);
    if (s != SQN_OK)
        return s;
    if ((s = check_quantised(x, "x")) != SQN_OK)
        return s;
    if ((s = check_layer(x->rows, x->cols, w, bias, relu, out)) != SQN_OK)
        return s;
    if (x->rows == 0)
        return SQN_OK;
    if ((s = check_workspace(workspace, workspace_bytes, sqn::quantised_product_bytes(x->rows, w->rows, x->cols)))
        != SQN_OK)
        return s;
    return launched(sqn::launch_quantised_product(*x, *w, bias, relu != 0, *out, workspace,
                                                  static_cast<hipStream_t>(stream)),
                    "product");
}

size_t sqn_quantised_layer_workspace(int64_t points, int64_t units, int64_t cols)
{
    if (!valid_layer(points, units, cols))
        return 0;
    return sqn::quantised_layer_bytes(points, units, cols);
}

sqn_status sqn_quantised_layer(const sqn_matrix* x, const sqn_quantised* w, const float* bias, int32_t relu,
                               const sqn_matrix* out, void* workspace, size_t workspace_bytes, void* stream)
{
    sqn_status s = check_stream(stream);
    if (s != SQN_OK)
        return s;
    if ((s = check_matrix(x, false, "x")) != SQN_OK)
        return s;
    if ((s = check_layer(x->rows, x->cols, w, bias, relu, out)) != SQN_OK)
        return s;
    if (x->rows == 0)
        return SQN_OK;
    if ((s = check_workspace(workspace, workspace_bytes, sqn::quantised_layer_bytes(x->rows, w->rows, x->cols)))
        != SQN_OK)
        return s;
    return launched(sqn::launch_quantised_layer(*x, *w, bias, relu != 0, *out, workspace,
                                                static_cast<hipStream_t>(stream)),
                    "layer");
}

}  // extern "C"
