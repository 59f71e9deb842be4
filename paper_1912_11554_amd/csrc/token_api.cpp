// C ABI of the token-model operators: argument checks, the layout of the
// workspace, and the order of the launches.  Nothing here allocates, copies or
// waits; no C++ exception crosses this boundary.
#include <hip/hip_runtime.h>

#include "../../include/nuts_token.h"
#include "handle.h"
#include "token.h"

using namespace nuts::token;

namespace {

constexpr int64_t kMaxSize = (int64_t)1 << 31;
constexpr int64_t kMaxStride = (int64_t)1 << 23;  // a tile's byte offsets are 32 bits
// Compute units the plans are made for (a workspace's size is a function of
// the call's arguments alone).
constexpr int kUnits = 256;

// Refusals: the first one's message stays (h may be null: a workspace query).
struct Check {
    nuts_handle* h;
    int code = NUTS_OK;
    template <typename... A>
    void refuse(int c, const char* fmt, A... a)
    {
        if (code != NUTS_OK) return;
        code = c;
        if (h) fail(h, c, fmt, a...);
    }
    bool on_device(const void* p) const
    {
        hipPointerAttribute_t attr;
        if (hipPointerGetAttributes(&attr, p) != hipSuccess) {
            (void)hipGetLastError();  // clear the sticky "invalid value" of unknown host memory
            return false;
        }
        return (attr.type == hipMemoryTypeDevice && attr.device == h->device) || attr.type == hipMemoryTypeManaged;
    }
    void type(int dtype)
    {
        if (dtype != NUTS_F32 && dtype != NUTS_BF16) refuse(NUTS_EINVAL, "dtype must be NUTS_F32 or NUTS_BF16 (got %d)", dtype);
    }
    void act(int a)
    {
        if (a < NUTS_ACT_NONE || a > NUTS_ACT_GELU) refuse(NUTS_EINVAL, "unknown activation %d", a);
    }
    void size(const char* name, int64_t n, int64_t below = kMaxSize)
    {
        if (n < 0 || n >= below)
            refuse(NUTS_EINVAL, "%s must be in [0, %lld) (got %lld)", name, (long long)below, (long long)n);
    }
    void scale(double s)
    {
        // (the kernels take it in fp32)
        const double size = s < 0.0 ? -s : s;
        if (!(size == 0.0 || (size >= 0x1p-126 && size <= (double)__FLT_MAX__)))
            refuse(NUTS_EINVAL, "scale must be zero or a finite, normal fp32 value (got %g)", s);
    }
    // A buffer of `elems` elements of `bytes` each; needed unless it is empty.
    void buffer(const char* name, const void* p, int64_t elems, size_t bytes, bool needed = true)
    {
        if (code != NUTS_OK || (!p && !needed) || elems == 0) return;
        if (!p) return refuse(NUTS_EINVAL, "%s is NULL", name);
        if ((uintptr_t)p % bytes) return refuse(NUTS_EINVAL, "%s is not aligned to its %zu-byte elements", name, bytes);
        if (h && !on_device(p)) refuse(NUTS_EINVAL, "%s must be memory of device %d", name, h->device);
    }
    void matrix(const char* name, const void* p, int64_t rows, int64_t cols, int64_t ld, size_t bytes, bool needed = true,
                int64_t max_ld = kMaxStride)
    {
        if (code != NUTS_OK || (!p && !needed)) return;
        if (rows > 0 && cols > 0) {
            if (ld < cols)
                return refuse(NUTS_EINVAL, "%s: row stride %lld is less than the row's %lld elements", name,
                              (long long)ld, (long long)cols);
            if (ld >= max_ld)
                return refuse(NUTS_EUNSUPPORTED, "%s: row stride %lld is not below %lld", name, (long long)ld,
                              (long long)max_ld);
        }
        buffer(name, p, rows * cols, bytes, needed);
    }
    void space(const void* workspace, int64_t given, int64_t need)
    {
        if (code != NUTS_OK || need == 0) return;
        if (given < need)
            return refuse(NUTS_EINVAL, "workspace: %lld bytes are needed, %lld given", (long long)need, (long long)given);
        if (!workspace || (uintptr_t)workspace % 16)
            return refuse(NUTS_EINVAL, "workspace must be 16-byte aligned device memory");
        if (h && !on_device(workspace)) refuse(NUTS_EINVAL, "workspace must be memory of device %d", h->device);
    }
};

// Consecutive pieces of the workspace; without a base, their sizes only.
struct Space {
    char* base;
    int64_t bytes = 0;
    void* take(int64_t n)
    {
        void* p = base ? base + bytes : nullptr;
        bytes += up(n, 256);
        return p;
    }
};

// Whether a matrix of rows of C elements can be copied to LDS as it lies.
bool direct(const void* p, int64_t C, int64_t ld, int dtype)
{
    return dtype == NUTS_BF16 && C % 8 == 0 && ld % 8 == 0 && (uintptr_t)p % 16 == 0;
}

bool too_many_tiles(int64_t M, int64_t N) { return ((M + 63) / 64) * ((N + 31) / 32) >= (int64_t)1 << 24; }

// ---------------------------------------------------------------------------
// z = x w^T (and x w2^T)
struct Forward {
    int dtype;
    bool gated;
    int64_t M, N, K;
    const void* x;
    int64_t ldx;
    const void* w;
    int64_t ldw;
    const void* w2;
    int64_t ldw2;
    Epilogue epi;
};
// Lays out and (with a stream to run on) enqueues.
hipError_t forward(const Forward& f, Space& space, bool run, hipStream_t stream)
{
    if (f.M == 0 || f.N == 0) return hipSuccess;
    if (few_rows(f.M, f.N, f.K)) {
        if (!run) return hipSuccess;
        FewRows p{f.gated, f.M, f.N, f.K, f.x, f.ldx, f.w, f.ldw, f.w2, f.ldw2, f.epi};
        return launch_few_rows(p, stream);
    }
    Product p{};
    p.M = f.M;
    p.N = f.N;
    p.K = f.K;
    p.dtype = f.dtype;
    p.staged = !direct(f.x, f.K, f.ldx, f.dtype) || !direct(f.w, f.K, f.ldw, f.dtype) ||
               (f.gated && !direct(f.w2, f.K, f.ldw2, f.dtype));
    p.gated = f.gated;
    p.sets = p.nterms = 1;
    p.terms[0][0] = {f.x, f.w, f.w2, f.ldx, f.ldw, f.ldw2};
    p.epi[0] = f.epi;
    float* partials = (float*)space.take((int64_t)product_workspace(p, kUnits));
    return run ? launch_product(p, partials, kUnits, stream) : hipSuccess;
}

// dx and dw (and dw2) for dz (and dz2)
struct Backward {
    int dtype, act;
    bool rounded;  // bf16: dz in one part
    int64_t M, N, K;
    const void* dy;
    int64_t lddy;
    const void* x;
    int64_t ldx;
    const void* w;
    int64_t ldw;
    const void* w2;
    int64_t ldw2;
    bool gated;
    const float* pre;
    void* dx;
    int64_t lddx;
    void *dw, *dw2;
    int64_t lddw, lddw2;
    void* dbias;
};
// A bf16 dz rounded once adds as much error to its products as their own rounding
// does (2.3e-3 of their norm in all, where one rounding leaves 1.7e-3).  So it is kept
// in two bf16 matrices (16 bits), twice the products, unless the caller asks for one
// (linear layer and gated block, one part and two, us: 128 x 1024 x 1024 22 and 23, 24
// and 28; 1024^3 28 and 45, 40 and 61; 8192 x 2048 x 8192 540 and 944, 958 and 1801).
const void* part_of(const void* dz, int part, int64_t rest)
{
    return dz ? (const char*)dz + (part ? rest * 2 : 0) : nullptr;
}
hipError_t backward(const Backward& b, Space& space, bool run, hipStream_t stream)
{
    // dz: dy itself, or written by the pass over dy and pre
    const bool own = !b.gated && b.act == NUTS_ACT_NONE, products = b.dx || b.dw;
    const void *dz = b.dy, *du = nullptr;
    int64_t ldz = b.lddy, rest = 0;
    if (products && !own) {
        ldz = up(b.N, 8);
        if (b.dtype == NUTS_BF16 && !b.rounded) rest = b.M * ldz;
        dz = space.take((b.M * ldz + rest) * (int64_t)type_bytes(b.dtype));
        if (b.gated) du = space.take((b.M * ldz + rest) * (int64_t)type_bytes(b.dtype));
    }
    Slope s{b.M, b.N, b.dy, b.lddy, own ? nullptr : b.pre, b.act, b.dtype, b.gated, nullptr, nullptr, rest, ldz, b.dbias,
            nullptr};
    if (products && !own) {
        s.dz = (void*)dz;
        s.dz2 = (void*)du;
    }
    if (b.dbias) s.sums = (float*)space.take((int64_t)slope_sums_bytes(b.M, b.N));
    if (run && (b.dbias || s.dz)) {
        const hipError_t e = launch_slope(s, stream);
        if (e != hipSuccess) return e;
    }
    Product p{};
    p.dtype = b.dtype;
    p.b_rows = true;
    p.epi[0].dtype = p.epi[1].dtype = b.dtype;
    const bool dz_direct = direct(dz, b.N, ldz, b.dtype);
    const int parts = rest ? 2 : 1;
    if (b.dx && b.M > 0 && b.K > 0) {
        p.M = b.M;
        p.N = b.K;
        p.K = b.N;
        p.staged = !dz_direct || !direct(b.w, b.K, b.ldw, b.dtype) || (b.gated && !direct(b.w2, b.K, b.ldw2, b.dtype));
        p.sets = 1;
        p.nterms = 0;
        p.small_terms = (parts - 1) * (b.gated ? 2 : 1);
        for (int part = parts - 1; part >= 0; --part) {
            p.terms[0][p.nterms++] = {part_of(dz, part, rest), b.w, nullptr, ldz, b.ldw, 0};
            if (b.gated) p.terms[0][p.nterms++] = {part_of(du, part, rest), b.w2, nullptr, ldz, b.ldw2, 0};
        }
        p.epi[0].out = b.dx;
        p.epi[0].ldo = b.lddx;
        float* partials = (float*)space.take((int64_t)product_workspace(p, kUnits));
        if (run) {
            const hipError_t e = launch_product(p, partials, kUnits, stream);
            if (e != hipSuccess) return e;
        }
    }
    if (b.dw && b.N > 0 && b.K > 0) {
        p.M = b.N;
        p.N = b.K;
        p.K = b.M;
        p.staged = !dz_direct || !direct(b.x, b.K, b.ldx, b.dtype);
        p.a_rows = true;
        p.nterms = parts;
        p.small_terms = parts - 1;
        p.sets = b.gated ? 2 : 1;
        for (int t = 0; t < parts; ++t) {
            p.terms[0][t] = {part_of(dz, parts - 1 - t, rest), b.x, nullptr, ldz, b.ldx, 0};
            p.terms[1][t] = {part_of(du, parts - 1 - t, rest), b.x, nullptr, ldz, b.ldx, 0};
        }
        p.epi[0].out = b.dw;
        p.epi[0].ldo = b.lddw;
        p.epi[1].out = b.dw2;
        p.epi[1].ldo = b.lddw2;
        float* partials = (float*)space.take((int64_t)product_workspace(p, kUnits));
        if (run) return launch_product(p, partials, kUnits, stream);
    }
    return hipSuccess;
}

Forward linear_forward(const nuts_linear_args& a)
{
    Forward f{a.dtype, false, a.M, a.N, a.K, a.x, a.ldx, a.w, a.ldw, nullptr, 0, {}};
    f.epi = {a.y, a.ldy, a.bias, a.residual, a.residual ? a.ldr : 0, a.pre, a.act, a.dtype};
    return f;
}
Forward gated_forward(const nuts_gated_args& a)
{
    Forward f{a.dtype, true, a.M, a.F, a.K, a.x, a.ldx, a.wg, a.ldwg, a.wu, a.ldwu, {}};
    f.epi = {a.y, a.ldy, nullptr, nullptr, 0, a.pre, a.act, a.dtype};
    return f;
}
// The activation of a gradient's arguments.
int act_of(int act) { return act & ~NUTS_ROUND_DZ; }

Backward linear_backward(const nuts_linear_grad_args& a)
{
    return {a.dtype, act_of(a.act), (a.act & NUTS_ROUND_DZ) != 0, a.M, a.N, a.K, a.dy, a.lddy, a.x, a.ldx, a.w, a.ldw, nullptr, 0, false, a.pre,
            a.dx, a.lddx, a.dw, nullptr, a.lddw, 0, a.dbias};
}
Backward gated_backward(const nuts_gated_grad_args& a)
{
    return {a.dtype, act_of(a.act), (a.act & NUTS_ROUND_DZ) != 0, a.M, a.F, a.K, a.dy, a.lddy, a.x, a.ldx, a.wg, a.ldwg, a.wu, a.ldwu, true, a.pre,
            a.dx, a.lddx, a.dwg, a.dwu, a.lddwg, a.lddwu, nullptr};
}

void check_sizes(Check& c, int dtype, int act, int64_t M, int64_t N, int64_t K, const char* n)
{
    c.type(dtype);
    c.act(act);
    c.size("M", M);
    c.size(n, N);
    c.size("K", K);
    if (c.code == NUTS_OK && (too_many_tiles(M, N) || too_many_tiles(M, K) || too_many_tiles(N, K)))
        c.refuse(NUTS_EUNSUPPORTED, "M = %lld, %s = %lld, K = %lld: a product has too many tiles", (long long)M, n,
                 (long long)N, (long long)K);
}
int check(Check& c, const nuts_linear_args& a)
{
    check_sizes(c, a.dtype, a.act, a.M, a.N, a.K, "N");
    const size_t b = type_bytes(a.dtype);
    if (c.code == NUTS_OK && a.N > 0) {
        c.matrix("x", a.x, a.M, a.K, a.ldx, b);
        if (a.M > 0) c.matrix("w", a.w, a.N, a.K, a.ldw, b);
        c.buffer("bias", a.bias, a.N, b, false);
        c.matrix("residual", a.residual, a.M, a.N, a.ldr, b, false);
        c.matrix("y", a.y, a.M, a.N, a.ldy, b);
        c.buffer("pre", a.pre, a.M * a.N, 4, false);
    }
    return c.code;
}
int check(Check& c, const nuts_gated_args& a)
{
    check_sizes(c, a.dtype, a.act, a.M, a.F, a.K, "F");
    const size_t b = type_bytes(a.dtype);
    if (c.code == NUTS_OK && a.F > 0) {
        c.matrix("x", a.x, a.M, a.K, a.ldx, b);
        if (a.M > 0) {
            c.matrix("wg", a.wg, a.F, a.K, a.ldwg, b);
            c.matrix("wu", a.wu, a.F, a.K, a.ldwu, b);
        }
        c.matrix("y", a.y, a.M, a.F, a.ldy, b);
        c.buffer("pre", a.pre, a.M * a.F, 4, false);
    }
    return c.code;
}
int check(Check& c, const nuts_linear_grad_args& a)
{
    check_sizes(c, a.dtype, act_of(a.act), a.M, a.N, a.K, "N");
    const size_t b = type_bytes(a.dtype);
    if (c.code == NUTS_OK) {
        c.matrix("dy", a.dy, a.M, a.N, a.lddy, b);
        if (act_of(a.act) != NUTS_ACT_NONE) c.buffer("pre", a.pre, a.M * a.N, 4);
        if (a.dw) c.matrix("x", a.x, a.M, a.K, a.ldx, b);
        if (a.dx) c.matrix("w", a.w, a.N, a.K, a.ldw, b);
        c.matrix("dx", a.dx, a.M, a.K, a.lddx, b, false);
        c.matrix("dw", a.dw, a.N, a.K, a.lddw, b, false);
        c.buffer("dbias", a.dbias, a.N, b, false);
    }
    return c.code;
}
int check(Check& c, const nuts_gated_grad_args& a)
{
    check_sizes(c, a.dtype, act_of(a.act), a.M, a.F, a.K, "F");
    const size_t b = type_bytes(a.dtype);
    if (c.code == NUTS_OK) {
        if ((a.dwg == nullptr) != (a.dwu == nullptr) && a.F > 0 && a.K > 0)
            c.refuse(NUTS_EINVAL, "dwg and dwu are given together or not at all");
        c.matrix("dy", a.dy, a.M, a.F, a.lddy, b);
        c.buffer("pre", a.pre, a.M * a.F, 4);
        if (a.dwg) c.matrix("x", a.x, a.M, a.K, a.ldx, b);
        if (a.dx) {
            c.matrix("wg", a.wg, a.F, a.K, a.ldwg, b);
            c.matrix("wu", a.wu, a.F, a.K, a.ldwu, b);
        }
        c.matrix("dx", a.dx, a.M, a.K, a.lddx, b, false);
        c.matrix("dwg", a.dwg, a.F, a.K, a.lddwg, b, false);
        c.matrix("dwu", a.dwu, a.F, a.K, a.lddwu, b, false);
    }
    return c.code;
}
int check(Check& c, const nuts_embedding_args& a)
{
    c.type(a.dtype);
    c.size("N", a.N);
    c.size("V", a.V);
    c.size("D", a.D);
    c.scale(a.scale);
    const size_t b = type_bytes(a.dtype);
    if (c.code == NUTS_OK && a.D > 0 && a.N > 0) {
        c.buffer("ids", a.ids, a.N, 8);
        c.matrix("table", a.table, a.V, a.D, a.ld_table, b, true, kMaxSize);
        c.matrix("out", a.out, a.N, a.D, a.ld_out, b, true, kMaxSize);
    }
    return c.code;
}
int check(Check& c, const nuts_embedding_grad_args& a)
{
    c.type(a.dtype);
    c.size("N", a.N, ((int64_t)1 << 26) + 1);
    c.size("V", a.V, (int64_t)1 << 30);
    c.size("D", a.D);
    c.scale(a.scale);
    const size_t b = type_bytes(a.dtype);
    if (c.code == NUTS_OK && a.D > 0 && a.V > 0) {
        c.buffer("ids", a.ids, a.N, 8);
        c.matrix("dout", a.dout, a.N, a.D, a.ld_dout, b, true, kMaxSize);
        c.matrix("dtable", a.dtable, a.V, a.D, a.ld_dtable, b, true, kMaxSize);
    }
    return c.code;
}
int check(Check& c, const nuts_categorical_args& a)
{
    c.type(a.dtype);
    c.size("M", a.M);
    c.size("V", a.V);
    c.scale(a.scale);
    const size_t b = type_bytes(a.dtype);
    if (c.code == NUTS_OK) {
        c.matrix("logits", a.logits, a.M, a.V, a.ld_logits, b, true, kMaxSize);
        c.buffer("targets", a.targets, a.M, 8);
        c.buffer("nll", a.nll, a.M, 4);
        c.buffer("total", a.total, 1, 8, false);
        c.matrix("dlogits", a.dlogits, a.M, a.V, a.ld_dlogits, b, false, kMaxSize);
    }
    return c.code;
}

// Common frame of the entry points: arguments, then `enqueue`.
template <typename Args, typename F>
int enter(nuts_handle* h, const Args* a, F enqueue)
{
    if (!h) return NUTS_EINVAL;
    h->err.clear();
    if (!a) return fail(h, NUTS_EINVAL, "the arguments are NULL");
    Check c{h};
    if (check(c, *a) != NUTS_OK) return c.code;
    int current = -1;
    if (hipGetDevice(&current) == hipSuccess && current == h->device) return enqueue(c);
    DeviceScope ds(h->device);
    return enqueue(c);
}

template <typename Args, typename Make, typename Go>
int64_t query(const Args* a, Make make, Go go)
{
    if (!a) return NUTS_EINVAL;
    Check c{nullptr};
    if (check(c, *a) != NUTS_OK) return c.code;
    Space s{nullptr};
    (void)go(make(*a), s, false, nullptr);
    return s.bytes;
}
template <typename Args, typename Make, typename Go>
int run_products(nuts_handle* h, const Args* a, void* workspace, int64_t workspace_bytes, void* hip_stream, Make make,
                 Go go)
{
    return enter(h, a, [&](Check& c) -> int {
        const auto f = make(*a);
        Space need{nullptr};
        (void)go(f, need, false, nullptr);
        c.space(workspace, workspace_bytes, need.bytes);
        if (c.code != NUTS_OK) return c.code;
        Space s{(char*)workspace};
        HIP_TRY(h, go(f, s, true, (hipStream_t)hip_stream));
        return NUTS_OK;
    });
}

}  // namespace

extern "C" {

int nuts_embedding(nuts_handle* h, const nuts_embedding_args* a, void* hip_stream)
{
    return enter(h, a, [&](Check&) -> int {
        HIP_TRY(h, launch_embedding(*a, (hipStream_t)hip_stream));
        return NUTS_OK;
    });
}

int64_t nuts_embedding_grad_workspace(const nuts_embedding_grad_args* a)
{
    if (!a) return NUTS_EINVAL;
    Check c{nullptr};
    if (check(c, *a) != NUTS_OK) return c.code;
    return (int64_t)embedding_grad_workspace(*a);
}

int nuts_embedding_grad(nuts_handle* h, const nuts_embedding_grad_args* a, void* workspace, int64_t workspace_bytes,
                    void* hip_stream)
{
    return enter(h, a, [&](Check& c) -> int {
        c.space(workspace, workspace_bytes, (int64_t)embedding_grad_workspace(*a));
        if (c.code != NUTS_OK) return c.code;
        HIP_TRY(h, launch_embedding_grad(*a, workspace, (hipStream_t)hip_stream));
        return NUTS_OK;
    });
}

int64_t nuts_linear_workspace(const nuts_linear_args* a) { return query(a, linear_forward, forward); }
int nuts_linear(nuts_handle* h, const nuts_linear_args* a, void* workspace, int64_t workspace_bytes,
                    void* hip_stream)
{
    return run_products(h, a, workspace, workspace_bytes, hip_stream, linear_forward, forward);
}

int64_t nuts_linear_grad_workspace(const nuts_linear_grad_args* a) { return query(a, linear_backward, backward); }
int nuts_linear_grad(nuts_handle* h, const nuts_linear_grad_args* a, void* workspace, int64_t workspace_bytes,
                    void* hip_stream)
{
    return run_products(h, a, workspace, workspace_bytes, hip_stream, linear_backward, backward);
}

int64_t nuts_gated_workspace(const nuts_gated_args* a) { return query(a, gated_forward, forward); }
int nuts_gated(nuts_handle* h, const nuts_gated_args* a, void* workspace, int64_t workspace_bytes,
                    void* hip_stream)
{
    return run_products(h, a, workspace, workspace_bytes, hip_stream, gated_forward, forward);
}

int64_t nuts_gated_grad_workspace(const nuts_gated_grad_args* a) { return query(a, gated_backward, backward); }
int nuts_gated_grad(nuts_handle* h, const nuts_gated_grad_args* a, void* workspace, int64_t workspace_bytes,
                    void* hip_stream)
{
    return run_products(h, a, workspace, workspace_bytes, hip_stream, gated_backward, backward);
}

int nuts_categorical(nuts_handle* h, const nuts_categorical_args* a, void* hip_stream)
{
    return enter(h, a, [&](Check&) -> int {
        HIP_TRY(h, launch_categorical(*a, (hipStream_t)hip_stream));
        return NUTS_OK;
    });
}

}  // extern "C"
