// C ABI of the operators for networks on decoded batches (include/rinr_nn.h): checks, plans, launches.
#include "rinr_nn_common.hip.h"
#include "rinr_nn_gemm.hip.h"
#include "rinr_nn_rows.hip.h"

#include <algorithm>
#include <cmath>

using namespace rinr_nn;

namespace {

inline bool hip_fail(hipError_t e) { return e != hipSuccess; }
#define NN_HIP(call) do { if (hip_fail(call)) return RINR_E_HIP; } while (0)
inline int launched() { return hip_fail(hipGetLastError()) ? RINR_E_HIP : RINR_OK; }

constexpr int kCUs = 256;
constexpr int64_t kMaxRows = INT32_MAX;

inline bool is_float_type(int t) { return t == RINR_T_BF16 || t == RINR_T_F16 || t == RINR_T_F32; }
inline size_t size_of(int t) { return t == RINR_T_F32 ? 4 : 2; }
inline int64_t round_up(int64_t v, int64_t to) { return (v + to - 1) / to * to; }
inline int64_t div_up(int64_t v, int64_t by) { return (v + by - 1) / by; }
inline bool past_l2(int64_t rows, int64_t cols, int type) { return rows * cols * (int64_t)size_of(type) > kPastL2; }
inline bool aligned(const void *p, size_t to) { return ((uintptr_t)p & (to - 1)) == 0; }

// A matrix of `rows` x `cols` that has to be there: pointers, type, stride, alignment
int check_mat(const void *p, int64_t ld, const uint8_t *scales, int type, int64_t cols) {
    if (!p) return RINR_E_NULL;
    if (type == RINR_T_PACKED8) {
        if (!scales) return RINR_E_NULL;
        if (ld % kBlock8 || ld < cols) return RINR_E_ARG;
        return aligned(p, 16) ? RINR_OK : RINR_E_ALIGN;
    }
    if (ld < cols) return RINR_E_ARG;
    return aligned(p, size_of(type)) ? RINR_OK : RINR_E_ALIGN;
}
// Whether two matrices of rows of `a_row`, `b_row` bytes share memory: their spans do, and rows equally far apart do not lie beside each other
bool overlap(const void *a, int64_t a_rows, int64_t a_row, int64_t a_ld, const void *b, int64_t b_rows, int64_t b_row, int64_t b_ld) {
    const uintptr_t pa = (uintptr_t)a, pb = (uintptr_t)b;
    if (pa + (uintptr_t)((a_rows - 1) * a_ld + a_row) <= pb || pb + (uintptr_t)((b_rows - 1) * b_ld + b_row) <= pa) return false;
    if (a_ld != b_ld) return true;
    const int64_t on = pb >= pa ? (int64_t)((pb - pa) % (uintptr_t)a_ld) : (a_ld - (int64_t)((pa - pb) % (uintptr_t)a_ld)) % a_ld;    // b's rows begin there in a's
    return on < a_row || on + b_row > a_ld;
}
#define NN_CHECK(call) do { const int rc_ = (call); if (rc_) return rc_; } while (0)

bool good_act(int act, float w0) { return act >= RINR_ACT_NONE && act <= RINR_ACT_SINE && (act != RINR_ACT_SINE || (w0 - w0 == 0.0f)); }

// ---- products ------------------------------------------------------------------------------------------------------------------------

typedef void (*gemm_fn)(const GemmArgs);
// slots: workgroups at once; us of a k tile and of a workgroup's start and end where one has a CU, and where all slots are taken
struct Kernel {
    gemm_fn fn;
    int lds, tile_p, tile_q, threads, k_tile, slots;
    float k_us, own_us, full_k_us, full_own_us;
};
enum { kForward = 0, kGradX = 1, kGradW = 2 };

template <class S> Kernel kernel_of(gemm_fn fn, int slots, float k_us, float own_us, float full_k_us, float full_own_us) {
    return {fn, S::LDS, S::WIDE_P, S::WIDE_Q, S::THREADS, S::BK, slots, k_us, own_us, full_k_us, full_own_us};
}
template <class E, class S, int MODE> gemm_fn wide_fn(int what) {
    return what == kForward ? wide_kernel<E, S, MODE, false, MODE, false> : what == kGradX ? wide_kernel<E, S, MODE, true, MODE, false> : wide_kernel<E, S, MODE, true, MODE, true>;
}
typedef WideShape<256, 256, 8, 4> Wide;
typedef WideShape<256, 128, 4, 4> Half;                                          // through registers, which the wide one has none to spare for
typedef WideShape<128, 128, 4, 4> Mid;
Kernel float_of(int what) {
    const gemm_fn fn = what == kForward ? gemm_kernel<false, false> : what == kGradX ? gemm_kernel<true, false> : gemm_kernel<true, true>;
    return {fn, kTileLds, kTile, kTile, kTileThreads, kTileK, 2 * kCUs, 1.45f, 6.7f, 2.85f, 6.7f};
}
// Few rows: 16 to 64 of a workgroup, as few as give no more workgroups than CUs (64 x 1024 -> 1000: 16 rows each 5.9 us, all 64 of them 7.8)
template <class T, class E, int PARTS> Kernel few_of(int64_t rows, int64_t columns, bool packed) {
    constexpr int kOwn = PARTS == 1 ? kSame : kFloat;
    const int64_t across = div_up(columns, kFewColumns);
    int each = 16;
    while (each < 64 && each < rows && across * div_up(rows, each) > kCUs) each *= 2;
    gemm_fn fn;
    if (each == 16) fn = packed ? few_kernel<T, E, PARTS, kOwn, kPacked, 1> : few_kernel<T, E, PARTS, kOwn, kOwn, 1>;
    else if (each == 32) fn = packed ? few_kernel<T, E, PARTS, kOwn, kPacked, 2> : few_kernel<T, E, PARTS, kOwn, kOwn, 2>;
    else fn = packed ? few_kernel<T, E, PARTS, kOwn, kPacked, 4> : few_kernel<T, E, PARTS, kOwn, kOwn, 4>;
    return {fn, 0, kFewColumns, each, kFewWaves * 64, kFewBlock, 2 * kCUs, 0.0f, 0.0f, 0.0f, 0.0f};
}
// Whether offsets in a tile fit 31 bits; whether rows begin on 4 bytes, as what goes straight from memory to LDS has to; whether groups of 8 values
// can be read at all
bool near(const Side &s) { return s.ld <= (1 << 21); }
bool direct(const Side &s) { return aligned(s.p, 4) && s.ld % 2 == 0; }
bool tiny(const Side &s, int64_t rows, int64_t cols) { return (rows - 1) * s.ld + cols < 8; }

// How a product is carried out: its kernel, tiles, and how many workgroups share the k of one tile
struct Plan {
    Kernel kernel;
    int tiles_p, tiles_q, k_tiles, shares, k_share;
    bool join;                                                                   // the result goes through memory as sums, one for each share
    bool tiny;
};
Plan plan_with(const Kernel &kn, int64_t np, int64_t nq, int64_t k, int64_t shares) {
    Plan p = {kn, (int)div_up(np, kn.tile_p), (int)div_up(nq, kn.tile_q), (int)div_up(k, kn.k_tile), 1, 1, false, false};
    p.k_share = (int)div_up(p.k_tiles, std::max<int64_t>(1, std::min<int64_t>(shares, p.k_tiles)));
    p.shares = (int)div_up(p.k_tiles, p.k_share);
    p.join = p.shares > 1;
    return p;
}
// Modelled time: rounds of workgroups, and what joining shares costs (a second kernel; the sums, written and read).  The figures are fits to
// measured calls of 65 to 32768 rows and 64 to 4096 columns, within a fifth of most: 4096 rows, 1024 -> 1024, whole 14.8 us, in two shares 25.7;
// 512 rows, 2048 -> 2048, whole 26, in four shares 19.3; 8192 rows, 256 -> 256, whole 7.6, in two shares 20.
double modelled_us(const Plan &p, int64_t np, int64_t nq) {
    const double n = (double)p.tiles_p * p.tiles_q * p.shares, k = p.k_share;
    const Kernel &kn = p.kernel;
    const double run = n <= kCUs ? k * kn.k_us + kn.own_us : std::ceil(n / kn.slots) * (k * kn.full_k_us + kn.full_own_us);
    return run + (p.join ? 3.5 + 0.15 * p.shares + (double)p.shares * (double)np * (double)nq * 8.0 / 6e6 : 0.0);
}
Plan cheapest(const Kernel *kernels, int n, int64_t np, int64_t nq, int64_t k) {
    Plan best = plan_with(kernels[0], np, nq, k, 1);
    double least = modelled_us(best, np, nq);
    for (int i = 0; i < n; ++i)
        for (int64_t shares = i ? 1 : 2; shares <= 128; shares += shares < 8 ? 1 : shares / 4) {
            const Plan p = plan_with(kernels[i], np, nq, k, shares);
            if (shares > 1 && (int64_t)p.tiles_p * p.tiles_q * p.shares > kernels[i].slots) break;
            const double us = modelled_us(p, np, nq);
            if (us < least) least = us, best = p;
        }
    return best;
}
template <class E> Plan plan_16(int what, const Side &P, const Side &Q, int64_t K) {
    if (!near(P) || !near(Q)) {
        const Kernel far = kernel_of<Mid>(wide_fn<E, Mid, kFar>(what), 2 * kCUs, 2.0f, 5.0f, 2.0f, 6.0f);
        return cheapest(&far, 1, P.n, Q.n, K);
    }
    if (direct(P) && direct(Q)) {
        const Kernel k[2] = {kernel_of<Mid>(wide_fn<E, Mid, kAsync>(what), 2 * kCUs, 0.65f, 5.0f, 1.25f, 6.0f),
                             kernel_of<Wide>(wide_fn<E, Wide, kAsync>(what), kCUs, 1.6f, 11.0f, 1.6f, 11.0f)};
        return cheapest(k, 2, P.n, Q.n, K);
    }
    const Kernel k[2] = {kernel_of<Mid>(wide_fn<E, Mid, kSame>(what), 2 * kCUs, 1.2f, 5.0f, 1.5f, 6.0f),
                         kernel_of<Half>(wide_fn<E, Half, kSame>(what), kCUs, 1.8f, 9.0f, 1.8f, 9.0f)};
    return cheapest(k, 2, P.n, Q.n, K);
}
// x_packed: the product's x is packed, which only few rows' kernels take; in_blocks: a packed z is written
// Beyond 64 rows tiles are faster for large weights (65 rows, 1024 -> 4096: 10.3 us, as few rows 12.4; 4096 -> 1024 12.1 and 14.0; packed x 15 and 22) and slower for small
// ones (256 -> 256: 6.7 and 3.7; 1024 -> 1000: 10.2 and 6.0)
constexpr int64_t kFewRows = 64;
Plan plan_of(int dtype, int what, bool x_packed, bool in_blocks, const Side &P, const Side &Q, int64_t K) {
    const bool kp = what != kForward, kq = what == kGradW;
    if (tiny(P, kp ? K : P.n, kp ? P.n : K) || (!x_packed && tiny(Q, kq ? K : Q.n, kq ? Q.n : K))) {
        Plan p = {};
        p.tiny = true;
        return p;
    }
    if (what == kForward && Q.n <= kFewRows) {
        const Kernel k = dtype == RINR_T_BF16 ? few_of<bf16, bf16, 1>(Q.n, P.n, x_packed) : dtype == RINR_T_F16 ? few_of<f16, f16, 1>(Q.n, P.n, x_packed) : few_of<float, bf16, 3>(Q.n, P.n, x_packed);
        Plan p = plan_with(k, P.n, Q.n, K, 1);
        // a workgroup reads 128 KB of weights in the time of a second kernel: longer k, in few columns, is shared
        p = plan_with(k, P.n, Q.n, K, std::min<int64_t>(kCUs / std::max(1, p.tiles_p * p.tiles_q), p.k_tiles / 64));
        p.join = in_blocks || p.shares > 1;                                      // 16 columns of a workgroup are half a block: join_kernel packs
        if (k.tile_q == 64 && dtype != RINR_T_F32 && !x_packed) {                // 64 rows a workgroup read 1.8 TB/s of weights, 16 rows 4.8
            const Plan m = dtype == RINR_T_BF16 ? plan_16<bf16>(what, P, Q, K) : plan_16<f16>(what, P, Q, K);
            if (modelled_us(m, P.n, Q.n) < 4.0 + (double)P.n * (double)K * 2.0 / 1.8e6) return m;
        }
        return p;
    }
    switch (dtype) {
        case RINR_T_BF16: return plan_16<bf16>(what, P, Q, K);
        case RINR_T_F16: return plan_16<f16>(what, P, Q, K);
        default: {
            const Kernel k = float_of(what);
            return cheapest(&k, 1, P.n, Q.n, K);
        }
    }
}
size_t part_bytes(const Plan &p, int64_t np, int64_t nq) { return p.join ? (size_t)p.shares * (size_t)np * (size_t)nq * 4 : 0; }

template <class T> void launch_join(const float *part, const Plan &p, int64_t nq, int64_t np, const Epilogue &e, hipStream_t st) {
    const int64_t groups = div_up(np, kBlock8) * 4 * nq;
    hipLaunchKernelGGL(join_kernel<T>, dim3((uint32_t)div_up(groups, 256)), dim3(256), 0, st, part, p.shares, nq, np, e);
}

template <class T> void launch_tiny(int what, bool x_packed, const GemmArgs &a, hipStream_t st) {
    const int64_t tasks = div_up(a.P.n, kBlock8) * 4 * a.Q.n;
    hipLaunchKernelGGL(tiny_kernel<T>, grid_of(div_up(tasks, 256)), dim3(256), 0, st, a, tasks, what != kForward, what == kGradW, x_packed && what == kGradW,
                       x_packed && what == kForward);
}
#define NN_BY_TYPE(dtype, call, ...) \
    switch (dtype) { \
        case RINR_T_BF16: call<bf16>(__VA_ARGS__); break; \
        case RINR_T_F16: call<f16>(__VA_ARGS__); break; \
        default: call<float>(__VA_ARGS__); \
    }

// One product; `part` has room for part_bytes of its plan.
int product(int dtype, int what, bool x_packed, const Plan &p, const Side &P, const Side &Q, int64_t K, const Epilogue &e, float *part, hipStream_t st) {
    const Kernel &k = p.kernel;
    const GemmArgs a = {P, Q, K, p.tiles_p, p.tiles_q, p.k_tiles, p.k_share, p.join ? part : nullptr, !near(P) || !near(Q), e};
    if (p.tiny) {
        NN_BY_TYPE(dtype, launch_tiny, what, x_packed, a, st);
        return launched();
    }
    if (k.lds > 65536) NN_HIP(hipFuncSetAttribute((const void *)k.fn, hipFuncAttributeMaxDynamicSharedMemorySize, k.lds));
    hipLaunchKernelGGL(k.fn, dim3((uint32_t)(p.tiles_p * p.tiles_q), (uint32_t)p.shares), dim3((uint32_t)k.threads), (uint32_t)k.lds, st, a);
    if (p.join) NN_BY_TYPE(dtype, launch_join, part, p, Q.n, P.n, e, st);
    return launched();
}

bool good_sizes(int64_t rows, int64_t n_in, int64_t n_out) {
    return rows >= 0 && rows <= kMaxRows && n_in >= 1 && n_in <= RINR_NN_MAX_FEATURES && n_out >= 1 && n_out <= RINR_NN_MAX_FEATURES &&
           div_up(rows, kTile) * div_up(std::max(n_in, n_out), kTile) * kTileThreads <= UINT32_MAX;      // threads of a launch
}

int check_linear(const rinr_linear_args *a) {
    if (!a) return RINR_E_NULL;
    if (!good_sizes(a->rows, a->n_in, a->n_out) || !is_float_type(a->dtype) || !good_act(a->act, a->w0) || a->reserved) return RINR_E_ARG;
    if (a->x_type != a->dtype && a->x_type != RINR_T_PACKED8) return RINR_E_ARG;
    if (a->z_type != RINR_T_NONE && a->z_type != a->dtype && a->z_type != RINR_T_PACKED8) return RINR_E_ARG;
    if (a->rows == 0) return RINR_OK;
    NN_CHECK(check_mat(a->x, a->ld_x, a->x_scales, a->x_type, a->n_in));
    NN_CHECK(check_mat(a->w, a->ld_w, nullptr, a->dtype, a->n_in));
    NN_CHECK(check_mat(a->y, a->ld_y, nullptr, a->dtype, a->n_out));
    if (a->z_type != RINR_T_NONE) NN_CHECK(check_mat(a->z, a->ld_z, a->z_scales, a->z_type, a->n_out));
    if (a->residual) NN_CHECK(check_mat(a->residual, a->ld_residual, nullptr, a->dtype, a->n_out));
    return aligned(a->bias, 4) ? RINR_OK : RINR_E_ALIGN;
}

// Workgroups read x and w while others write: y and z lie apart from both.  The residual is read where y is written, by the same thread.
int check_linear_apart(const rinr_linear_args *a) {
    const int64_t el = (int64_t)size_of(a->dtype), x_el = a->x_type == RINR_T_PACKED8 ? 1 : el, z_el = a->z_type == RINR_T_PACKED8 ? 1 : el;
    const auto touches = [&](const void *p, int64_t el_p, int64_t ld) {
        return overlap(p, a->rows, a->n_out * el_p, ld * el_p, a->x, a->rows, a->n_in * x_el, a->ld_x * x_el) ||
               overlap(p, a->rows, a->n_out * el_p, ld * el_p, a->w, a->n_out, a->n_in * el, a->ld_w * el);
    };
    if (touches(a->y, el, a->ld_y) || (a->z_type != RINR_T_NONE && touches(a->z, z_el, a->ld_z))) return RINR_E_ARG;
    const bool in_place = a->residual == a->y && (a->ld_residual == a->ld_y || a->rows == 1);
    return a->residual && !in_place && overlap(a->y, a->rows, a->n_out * el, a->ld_y * el, a->residual, a->rows, a->n_out * el, a->ld_residual * el) ? RINR_E_ARG : RINR_OK;
}

int check_linear_grad(const rinr_linear_grad_args *a) {
    if (!a) return RINR_E_NULL;
    if (!good_sizes(a->rows, a->n_in, a->n_out) || !is_float_type(a->dtype) || !good_act(a->act, a->w0) || !good_act(a->x_act, a->w0)) return RINR_E_ARG;
    if (a->x_type != a->dtype && a->x_type != RINR_T_PACKED8) return RINR_E_ARG;
    const bool has_act = a->act != RINR_ACT_NONE;
    if (has_act ? a->z_type != a->dtype && a->z_type != RINR_T_PACKED8 : a->z_type != RINR_T_NONE) return RINR_E_ARG;
    if (a->dx) NN_CHECK(check_mat(a->dx, a->ld_dx, nullptr, a->dtype, a->n_in));
    if (a->dw) NN_CHECK(check_mat(a->dw, a->ld_dw, nullptr, a->dtype, a->n_in));
    if (!aligned(a->dbias, 4)) return RINR_E_ALIGN;
    if (a->rows == 0) return RINR_OK;
    if (a->dx || a->dw || a->dbias) NN_CHECK(check_mat(a->dy, a->ld_dy, nullptr, a->dtype, a->n_out));
    if (a->dx) NN_CHECK(check_mat(a->w, a->ld_w, nullptr, a->dtype, a->n_in));
    if (a->dw || (a->dx && a->x_act != RINR_ACT_NONE)) NN_CHECK(check_mat(a->x, a->ld_x, a->x_scales, a->x_type, a->n_in));
    if (has_act && (a->dx || a->dw || a->dbias)) NN_CHECK(check_mat(a->z, a->ld_z, a->z_scales, a->z_type, a->n_out));
    return RINR_OK;
}

// Where things lie in the workspace of a backward pass (dz, the layer's input where it is not kept as it is, and partial sums, which the
// kernels use one after the other), and its two products.  dz and x_act(x) are rounded to the operands' type, because matrix instructions of 16 bits take them so:
// either one makes dw's error at most sqrt 2 of that of rounding dw alone.  Both together would make it sqrt 3, so x_act(x) is then taken in two parts: the product
// runs over twice the rows, dz twice and the parts one below the other (2000 x 500 -> 300: 1.65 of a rounding, and 1.41 in two parts).
struct GradPlan {
    int64_t ld_dz, ld_xa, sum_chunks, rows_each, dw_rows;
    size_t xa, part, bytes;
    Side dx_p, dx_q, dw_p, dw_q;
    Plan dx, dw;
};
GradPlan grad_plan(const rinr_linear_grad_args *a, char *ws) {
    GradPlan g = {};
    const size_t el = size_of(a->dtype);
    size_t part = 0;
    Side dz = {a->dy, a->ld_dy, 0, nullptr}, x = {a->x, a->ld_x, a->n_in, a->x_scales};
    const bool packed = a->x_type == RINR_T_PACKED8;
    g.dw_rows = a->rows * (a->dw && a->act != RINR_ACT_NONE && a->x_act != RINR_ACT_NONE && a->dtype != RINR_T_F32 ? 2 : 1);
    if (a->act != RINR_ACT_NONE && (a->dx || a->dw)) {
        g.ld_dz = round_up(a->n_out, 64);
        g.xa = (size_t)round_up((int64_t)((size_t)g.dw_rows * (size_t)g.ld_dz * el), 256);
        dz = {ws, g.ld_dz, 0, nullptr};
    }
    g.part = g.xa;
    if (a->dw && (packed || a->x_act != RINR_ACT_NONE)) {
        g.ld_xa = round_up(a->n_in, 64);
        g.part += (size_t)round_up((int64_t)((size_t)g.dw_rows * (size_t)g.ld_xa * el), 256);
        x = {ws + g.xa, g.ld_xa, a->n_in, nullptr};
    }
    const int64_t across = div_up(g.ld_dz ? g.ld_dz : a->n_out, 256);
    g.sum_chunks = std::max<int64_t>(1, std::min<int64_t>(div_up(a->rows, 8), 8 * kCUs / across));
    g.rows_each = round_up(div_up(a->rows, g.sum_chunks), 8);
    g.sum_chunks = div_up(a->rows, g.rows_each);
    if (a->dbias) part = (size_t)g.sum_chunks * (size_t)a->n_out * 4;
    if (a->dx) {
        g.dx_p = {a->w, a->ld_w, a->n_in, nullptr};
        g.dx_q = dz;
        g.dx_q.n = a->rows;
        g.dx = plan_of(a->dtype, kGradX, false, false, g.dx_p, g.dx_q, a->n_out);
        part = std::max(part, part_bytes(g.dx, a->n_in, a->rows));
    }
    if (a->dw) {
        g.dw_p = x;
        g.dw_q = dz;
        g.dw_q.n = a->n_out;
        g.dw = plan_of(a->dtype, kGradW, false, false, g.dw_p, g.dw_q, g.dw_rows);
        part = std::max(part, part_bytes(g.dw, a->n_in, a->n_out));
    }
    g.bytes = g.part + (size_t)round_up((int64_t)part, 256);
    return g;
}

template <class T> void launch_slope(const SlopeArgs &s, int64_t across, int64_t chunks, hipStream_t st) {
    hipLaunchKernelGGL(slope_kernel<T>, dim3((uint32_t)across, (uint32_t)chunks), dim3(256), 0, st, s);
}
void launch_sum_parts(const float *part, int64_t n, int64_t cols, float *out, hipStream_t st) {
    hipLaunchKernelGGL(sum_parts_kernel, dim3((uint32_t)div_up(cols, 32)), dim3(1024), 0, st, part, n, cols, out);
}
template <class T, bool LOW> void launch_unpack(int64_t rows, int64_t cols, const void *codes, int64_t ld, const uint8_t *scales, const Act &act, void *x, int64_t ld_x, hipStream_t st) {
    hipLaunchKernelGGL((unpack_kernel<T, LOW>), grid_of(div_up(rows * div_up(cols, 8), 256)), dim3(256), 0, st, rows, (int)cols, (const int8_t *)codes, ld, scales, act, (T *)x,
                       ld_x, rows * cols * (int64_t)sizeof(T) > kPastL2);
}
template <class T> void launch_values(int64_t rows, int64_t cols, const void *codes, int64_t ld, const uint8_t *scales, const Act &act, void *x, int64_t ld_x, hipStream_t st) {
    launch_unpack<T, false>(rows, cols, codes, ld, scales, act, x, ld_x, st);
}
template <class T> void launch_pack(int64_t rows, int64_t cols, const void *x, int64_t ld_x, void *codes, int64_t ld, uint8_t *scales, hipStream_t st) {
    hipLaunchKernelGGL(pack_kernel<T>, grid_of(div_up(rows * div_up(cols, kBlock8) * 4, 256)), dim3(256), 0, st, rows, (int)cols, (const T *)x, ld_x, (int8_t *)codes, ld, scales, rows * cols > kPastL2);
}
template <class T, bool LOW> void launch_act_parts(int64_t rows, int64_t cols, const void *z, int64_t ld, const uint8_t *scales, bool packed, const Act &act, void *x, int64_t ld_x,
                                                   hipStream_t st) {
    if (packed) launch_unpack<T, LOW>(rows, cols, z, ld, scales, act, x, ld_x, st);
    else hipLaunchKernelGGL((act_kernel<T, LOW>), grid_of(div_up(rows * div_up(cols, 8), 256)), dim3(256), 0, st, rows, (int)cols, (const T *)z, ld, act, (T *)x, ld_x,
                            rows * cols * (int64_t)sizeof(T) > kPastL2);
}
// two_parts: of 16-bit types only
template <class T> void launch_act(int64_t rows, int64_t cols, const void *z, int64_t ld, const uint8_t *scales, bool packed, const Act &act, void *x, int64_t ld_x, bool two_parts,
                                   hipStream_t st) {
    if (sizeof(T) == 2 && two_parts) launch_act_parts<T, sizeof(T) == 2>(rows, cols, z, ld, scales, packed, act, x, ld_x, st);
    else launch_act_parts<T, false>(rows, cols, z, ld, scales, packed, act, x, ld_x, st);
}

// ---- norms ---------------------------------------------------------------------------------------------------------------------------

int64_t norm_slots(int64_t cols) { return cols <= 1024 ? 4 : 1; }                // rows of a workgroup
// At most 4 workgroups a CU (2 of the largest), each with as many rows as the others but the last
int64_t norm_grad_blocks(int64_t rows, int64_t cols) {
    const int64_t groups = div_up(rows, norm_slots(cols)), most = (cols <= 8192 ? 4 : 2) * kCUs;
    return std::max<int64_t>(1, div_up(groups, std::max<int64_t>(1, div_up(groups, most))));
}

template <class T, bool PACKED> void launch_norm(const NormArgs &a, hipStream_t st) {
    const dim3 grid = grid_of(div_up(a.rows, norm_slots(a.cols)));
    if (a.cols <= 512) hipLaunchKernelGGL((norm_kernel<T, 64, 1, PACKED>), grid, dim3(256), 0, st, a);
    else if (a.cols <= 1024) hipLaunchKernelGGL((norm_kernel<T, 64, 2, PACKED>), grid, dim3(256), 0, st, a);
    else if (a.cols <= 4096) hipLaunchKernelGGL((norm_kernel<T, 256, 2, PACKED>), grid, dim3(256), 0, st, a);
    else if (a.cols <= 8192) hipLaunchKernelGGL((norm_kernel<T, 256, 4, PACKED>), grid, dim3(256), 0, st, a);
    else hipLaunchKernelGGL((norm_kernel<T, 1024, 4, PACKED>), grid, dim3(1024), 0, st, a);
}
template <class T> void launch_norm_grad(const NormGradArgs &a, hipStream_t st) {
    const uint32_t grid = (uint32_t)norm_grad_blocks(a.rows, a.cols);
    if (a.cols <= 512) hipLaunchKernelGGL((norm_grad_kernel<T, 64, 1>), dim3(grid), dim3(256), 0, st, a);
    else if (a.cols <= 1024) hipLaunchKernelGGL((norm_grad_kernel<T, 64, 2>), dim3(grid), dim3(256), 0, st, a);
    else if (a.cols <= 4096) hipLaunchKernelGGL((norm_grad_kernel<T, 256, 2>), dim3(grid), dim3(256), 0, st, a);
    else if (a.cols <= 8192) hipLaunchKernelGGL((norm_grad_kernel<T, 256, 4>), dim3(grid), dim3(256), 0, st, a);
    else hipLaunchKernelGGL((norm_grad_kernel<T, 1024, 4>), dim3(grid), dim3(1024), 0, st, a);
}

int check_rows(int64_t rows, int64_t cols, int dtype) {
    return rows >= 0 && rows <= kMaxRows && cols >= 1 && is_float_type(dtype) ? RINR_OK : RINR_E_ARG;
}

}  // namespace

namespace {
// A forward pass's product and workspace: x as dtype where it is packed and the rows are not few (unpacked once, not by every tile: in the large
// tiles' kernels that took more registers than there are, 454 us against 280 and 22 for 32768 rows of 1024 to 4096), and sums.
struct LinearPlan {
    Side P, Q;
    Plan plan;
    bool packed;
    int64_t ld_x;
    size_t x, bytes;
};
LinearPlan linear_plan(const rinr_linear_args *a, char *ws) {
    LinearPlan l = {{a->w, a->ld_w, a->n_out, nullptr}, {a->x, a->ld_x, a->rows, a->x_scales}, {}, a->x_type == RINR_T_PACKED8, 0, 0, 0};
    if (l.packed && a->rows > kFewRows) {
        l.packed = false;
        l.ld_x = round_up(a->n_in, 64);
        l.x = (size_t)round_up((int64_t)((size_t)a->rows * (size_t)l.ld_x * size_of(a->dtype)), 256);
        l.Q = {ws, l.ld_x, a->rows, nullptr};
    }
    l.plan = plan_of(a->dtype, kForward, l.packed, a->z_type == RINR_T_PACKED8, l.P, l.Q, a->n_in);
    l.bytes = l.x + part_bytes(l.plan, a->n_out, a->rows);
    return l;
}
}  // namespace

extern "C" size_t rinr_linear_workspace_bytes(const rinr_linear_args *a) { return check_linear(a) || a->rows == 0 ? 0 : linear_plan(a, nullptr).bytes; }

extern "C" int rinr_linear(const rinr_linear_args *a, void *workspace, size_t workspace_bytes, void *stream) {
    NN_CHECK(check_linear(a));
    if (a->rows == 0) return RINR_OK;
    NN_CHECK(check_linear_apart(a));
    const LinearPlan l = linear_plan(a, (char *)workspace);
    if (l.bytes && !workspace) return RINR_E_NULL;
    if (workspace_bytes < l.bytes) return RINR_E_SIZE;
    if (l.bytes && !aligned(workspace, 16)) return RINR_E_ALIGN;
    float *const part = (float *)((char *)workspace + l.x);
    if (l.ld_x) NN_BY_TYPE(a->dtype, launch_act, a->rows, a->n_in, a->x, a->ld_x, a->x_scales, true, make_act(RINR_ACT_NONE, 0.0f), workspace, l.ld_x, false, (hipStream_t)stream);
    Epilogue e = {};
    e.bias = a->bias;
    e.residual = a->residual;
    e.ld_residual = a->ld_residual;
    e.y = a->y;
    e.ld_y = a->ld_y;
    if (a->z_type != RINR_T_NONE) {
        e.z = a->z;
        e.ld_z = a->ld_z;
        e.z_scales = a->z_scales;
        e.z_packed = a->z_type == RINR_T_PACKED8;
    }
    e.act = make_act(a->act, a->w0);
    e.past = past_l2(a->rows, a->n_out, a->dtype);
    return product(a->dtype, kForward, l.packed, l.plan, l.P, l.Q, a->n_in, e, part, (hipStream_t)stream);
}

extern "C" size_t rinr_linear_backward_workspace_bytes(const rinr_linear_grad_args *a) {
    return check_linear_grad(a) || a->rows == 0 ? 0 : grad_plan(a, nullptr).bytes;
}

extern "C" int rinr_linear_backward(const rinr_linear_grad_args *a, void *workspace, size_t workspace_bytes, void *stream) {
    NN_CHECK(check_linear_grad(a));
    hipStream_t st = (hipStream_t)stream;
    const size_t el = size_of(a->dtype);
    if (!a->dw && !a->dbias && (!a->dx || a->rows == 0)) return RINR_OK;
    if (a->rows == 0) {                                                          // sums over nothing
        if (a->dw) hipLaunchKernelGGL(clear_kernel, dim3((uint32_t)a->n_out), dim3(256), 0, st, (char *)a->dw, a->ld_dw * (int64_t)el, a->n_in * (int64_t)el);
        if (a->dbias) hipLaunchKernelGGL(clear_kernel, dim3(1), dim3(256), 0, st, (char *)a->dbias, (int64_t)0, a->n_out * 4);
        return launched();
    }
    char *const ws = (char *)workspace;
    const GradPlan g = grad_plan(a, ws);
    if (g.bytes && !workspace) return RINR_E_NULL;
    if (workspace_bytes < g.bytes) return RINR_E_SIZE;
    if (!aligned(workspace, 16)) return RINR_E_ALIGN;
    float *const part = (float *)(ws + g.part);
    const bool x_packed = a->x_type == RINR_T_PACKED8;
    if (g.ld_dz || a->dbias) {
        const SlopeArgs s = {a->rows, a->n_out, g.rows_each, a->dy, a->z, a->z_scales, g.ld_dz ? ws : nullptr, a->dbias ? part : nullptr,
                             a->ld_dy, a->ld_z, g.ld_dz, g.ld_dz ? g.ld_dz : a->n_out, a->z_type == RINR_T_PACKED8,
                             past_l2(a->rows, a->n_out, a->dtype), g.dw_rows > a->rows, make_act(a->act, a->w0)};
        NN_BY_TYPE(a->dtype, launch_slope, s, div_up(s.cols_dz, 256), g.sum_chunks, st);
        if (a->dbias) launch_sum_parts(part, g.sum_chunks, a->n_out, a->dbias, st);
    }
    if (a->dx) {
        Epilogue e = {};
        e.y = a->dx;
        e.ld_y = a->ld_dx;
        e.past = past_l2(a->rows, a->n_in, a->dtype);
        if (a->x_act != RINR_ACT_NONE) {
            e.slope = a->x;
            e.ld_slope = a->ld_x;
            e.slope_scales = a->x_scales;
            e.slope_packed = x_packed;
            e.slope_act = make_act(a->x_act, a->w0);
        }
        NN_CHECK(product(a->dtype, kGradX, false, g.dx, g.dx_p, g.dx_q, a->n_out, e, part, st));
    }
    if (a->dw) {
        if (g.ld_xa) NN_BY_TYPE(a->dtype, launch_act, a->rows, a->n_in, a->x, a->ld_x, a->x_scales, x_packed, make_act(a->x_act, a->w0), ws + g.xa, g.ld_xa, g.dw_rows > a->rows,
                               st);
        Epilogue e = {};
        e.y = a->dw;
        e.ld_y = a->ld_dw;
        e.past = past_l2(a->n_out, a->n_in, a->dtype);
        NN_CHECK(product(a->dtype, kGradW, false, g.dw, g.dw_p, g.dw_q, g.dw_rows, e, part, st));
    }
    return launched();
}

extern "C" int rinr_rms_norm(const rinr_norm_args *a, void *stream) {
    if (!a) return RINR_E_NULL;
    NN_CHECK(check_rows(a->rows, a->cols, a->dtype));
    if ((a->y_type != a->dtype && a->y_type != RINR_T_PACKED8) || !(a->eps > 0.0f) || !(a->eps - a->eps == 0.0f) || a->reserved) return RINR_E_ARG;
    if (a->cols > RINR_NN_MAX_COLS) return RINR_E_UNSUPPORTED;
    if (a->rows == 0) return RINR_OK;
    NN_CHECK(check_mat(a->x, a->ld_x, nullptr, a->dtype, a->cols));
    NN_CHECK(check_mat(a->y, a->ld_y, a->y_scales, a->y_type, a->cols));
    if (a->residual) NN_CHECK(check_mat(a->residual, a->ld_residual, nullptr, a->dtype, a->cols));
    if (a->h && a->residual) NN_CHECK(check_mat(a->h, a->ld_h, nullptr, a->dtype, a->cols));
    if (!a->gain) return RINR_E_NULL;
    if (!aligned(a->gain, 4)) return RINR_E_ALIGN;
    const NormArgs n = {a->rows, (int)a->cols, a->eps, a->x, a->residual, a->gain, a->y, a->residual ? a->h : nullptr, a->y_scales, a->ld_x, a->ld_residual, a->ld_y, a->ld_h,
                        past_l2(a->rows, a->cols, a->dtype)};
    hipStream_t st = (hipStream_t)stream;
    const bool packed = a->y_type == RINR_T_PACKED8;
    switch (a->dtype) {
        case RINR_T_BF16: packed ? launch_norm<bf16, true>(n, st) : launch_norm<bf16, false>(n, st); break;
        case RINR_T_F16: packed ? launch_norm<f16, true>(n, st) : launch_norm<f16, false>(n, st); break;
        default: packed ? launch_norm<float, true>(n, st) : launch_norm<float, false>(n, st);
    }
    return launched();
}

extern "C" size_t rinr_rms_norm_backward_workspace_bytes(int64_t rows, int64_t cols) {
    if (rows < 1 || rows > kMaxRows || cols < 1 || cols > RINR_NN_MAX_COLS) return 0;
    return (size_t)norm_grad_blocks(rows, cols) * (size_t)cols * 4;
}

extern "C" int rinr_rms_norm_backward(const rinr_norm_grad_args *a, void *workspace, size_t workspace_bytes, void *stream) {
    if (!a) return RINR_E_NULL;
    NN_CHECK(check_rows(a->rows, a->cols, a->dtype));
    if (!(a->eps > 0.0f) || !(a->eps - a->eps == 0.0f)) return RINR_E_ARG;
    if (a->cols > RINR_NN_MAX_COLS) return RINR_E_UNSUPPORTED;
    if (!aligned(a->dgain, 4) || !aligned(a->gain, 4)) return RINR_E_ALIGN;
    hipStream_t st = (hipStream_t)stream;
    if (a->rows == 0) {
        if (!a->dgain) return RINR_OK;
        hipLaunchKernelGGL(clear_kernel, dim3(1), dim3(256), 0, st, (char *)a->dgain, (int64_t)0, a->cols * 4);
        return launched();
    }
    NN_CHECK(check_mat(a->dy, a->ld_dy, nullptr, a->dtype, a->cols));
    NN_CHECK(check_mat(a->h, a->ld_h, nullptr, a->dtype, a->cols));
    NN_CHECK(check_mat(a->dh, a->ld_dh, nullptr, a->dtype, a->cols));
    if (a->dres) NN_CHECK(check_mat(a->dres, a->ld_dres, nullptr, a->dtype, a->cols));
    if (!a->gain) return RINR_E_NULL;
    if (a->dgain) {
        if (!workspace) return RINR_E_NULL;
        if (workspace_bytes < rinr_rms_norm_backward_workspace_bytes(a->rows, a->cols)) return RINR_E_SIZE;
        if (!aligned(workspace, 16)) return RINR_E_ALIGN;
    }
    const NormGradArgs n = {a->rows, (int)a->cols, a->eps, a->dy, a->h, a->dres, a->gain, a->dh, a->dgain ? (float *)workspace : nullptr, a->ld_dy, a->ld_h, a->ld_dres, a->ld_dh,
                            past_l2(a->rows, a->cols, a->dtype)};
    NN_BY_TYPE(a->dtype, launch_norm_grad, n, st);
    if (a->dgain) launch_sum_parts((const float *)workspace, norm_grad_blocks(a->rows, a->cols), a->cols, a->dgain, st);
    return launched();
}

extern "C" int rinr_pack8(int64_t rows, int64_t cols, const void *x, int64_t ld_x, int32_t dtype, void *codes, int64_t ld, uint8_t *scales, void *stream) {
    NN_CHECK(check_rows(rows, cols, dtype));
    if (cols > INT32_MAX - 64) return RINR_E_UNSUPPORTED;
    if (rows == 0) return RINR_OK;
    NN_CHECK(check_mat(x, ld_x, nullptr, dtype, cols));
    NN_CHECK(check_mat(codes, ld, scales, RINR_T_PACKED8, cols));
    if (div_up(rows * div_up(cols, kBlock8) * 4, 256) > INT32_MAX) return RINR_E_UNSUPPORTED;
    NN_BY_TYPE(dtype, launch_pack, rows, cols, x, ld_x, codes, ld, scales, (hipStream_t)stream);
    return launched();
}

extern "C" int rinr_unpack8(int64_t rows, int64_t cols, const void *codes, int64_t ld, const uint8_t *scales, int32_t act, float w0, void *x, int64_t ld_x, int32_t dtype,
                            void *stream) {
    NN_CHECK(check_rows(rows, cols, dtype));
    if (!good_act(act, w0)) return RINR_E_ARG;
    if (cols > INT32_MAX - 64) return RINR_E_UNSUPPORTED;
    if (rows == 0) return RINR_OK;
    NN_CHECK(check_mat(codes, ld, scales, RINR_T_PACKED8, cols));
    NN_CHECK(check_mat(x, ld_x, nullptr, dtype, cols));
    if (div_up(rows * div_up(cols, 8), 256) > INT32_MAX) return RINR_E_UNSUPPORTED;
    NN_BY_TYPE(dtype, launch_values, rows, cols, codes, ld, scales, make_act(act, w0), x, ld_x, (hipStream_t)stream);
    return launched();
}
