// extern "C" boundary of libf3m: argument checks, error translation, introspection.
#include <algorithm>
#include <cmath>
#include <cstring>
#include <new>

#include "attend.h"
#include "plan.h"

namespace {

thread_local std::string g_last_error;

f3m_status set_error(f3m_status st, const std::string &msg) {
    g_last_error = msg;
    return st;
}

template <class F>
f3m_status guarded(F &&f) {
    try {
        f();
        return F3M_OK;
    } catch (const f3m::Error &e) {
        return set_error(e.status, e.msg);
    } catch (const std::bad_alloc &) {
        return set_error(F3M_ERR_OOM, "host allocation failed");
    } catch (const std::exception &e) {
        return set_error(F3M_ERR_HIP, e.what());
    } catch (...) {
        return set_error(F3M_ERR_HIP, "unknown failure");
    }
}

bool finite_pos(float v) { return std::isfinite(v) && v > 0.f; }

f3m_status check_problem(const float *X, int64_t n, int D, float lengthscale) {
    if (n < 0) return set_error(F3M_ERR_INVALID_ARG, "n must be >= 0");
    if (D < 1 || D > F3M_MAX_DIM) return set_error(F3M_ERR_INVALID_ARG, "D must be in [1,7]");
    if (!finite_pos(lengthscale)) return set_error(F3M_ERR_INVALID_ARG, "lengthscale must be finite and > 0");
    if (n > 0 && !X) return set_error(F3M_ERR_INVALID_ARG, "X is null");
    if (n >= ((int64_t)1 << 31)) return set_error(F3M_ERR_UNSUPPORTED, "n must be below 2^31");
    return F3M_OK;
}

// false for a plan with no targets or no sources: it holds no tables
bool built(const f3m_plan_t *plan) { return plan->n > 0 && plan->ns() > 0; }

// milliseconds between two marks of a product (stages without a launch share one)
hipError_t elapsed(float *ms, hipEvent_t from, hipEvent_t to) {
    *ms = 0.f;
    return from == to ? hipSuccess : hipEventElapsedTime(ms, from, to);
}

template <class T>
void copy_to_host(T *dst, const T *src, size_t count) {
    if (count == 0) return;
    F3M_HIP(hipMemcpy(dst, src, count * sizeof(T), hipMemcpyDeviceToHost));
}

// ---- attention ----

// the stride of one row alone means nothing and may be any number: the kernels compute with strides below 2^22
f3m::Rows rows_of(const f3m_rows &r, int64_t rows, int dim) { return {(char *)r.data, rows > 1 ? r.row : dim, r.head}; }

// `paged`: k, v, k_offsets and total_k are not read
f3m_status check_attention(const f3m_attention_args *p, bool paged = false) {
    if (!p) return set_error(F3M_ERR_INVALID_ARG, "args is null");
    if (p->dtype != F3M_BF16 && p->dtype != F3M_F16) return set_error(F3M_ERR_INVALID_ARG, "dtype must be F3M_BF16 or F3M_F16");
    if (p->heads < 1 || p->kv_heads < 1 || p->heads % p->kv_heads) return set_error(F3M_ERR_INVALID_ARG, "heads must be a positive multiple of kv_heads");
    if (p->head_dim < 8 || p->head_dim % 8) return set_error(F3M_ERR_INVALID_ARG, "head_dim must be a positive multiple of 8");
    if (p->head_dim > 128) return set_error(F3M_ERR_UNSUPPORTED, "head_dim above 128 is not supported");
    if (p->batch < 0 || p->max_q < 0 || p->max_k < 0 || p->total_q < 0 || p->total_k < 0)
        return set_error(F3M_ERR_INVALID_ARG, "batch, max_q, max_k, total_q and total_k must be >= 0");
    if (p->window < 0 || p->sinks < 0) return set_error(F3M_ERR_INVALID_ARG, "window and sinks must be >= 0");
    if (p->window && !p->causal) return set_error(F3M_ERR_INVALID_ARG, "a window needs causal order");
    if (p->sinks && !p->window) return set_error(F3M_ERR_INVALID_ARG, "sinks need a window");
    if (!finite_pos(p->scale)) return set_error(F3M_ERR_INVALID_ARG, "scale must be finite and > 0");
    if (!paged && (!p->q_offsets != !p->k_offsets)) return set_error(F3M_ERR_INVALID_ARG, "q_offsets and k_offsets are given both or neither");
    if (!p->q_offsets && p->batch != 1) return set_error(F3M_ERR_INVALID_ARG, "without offsets batch is 1");
    constexpr int64_t most = ((int64_t)1 << 31) - 65536;   // indices of a tile past the last row stay ints
    if (p->total_q >= most || p->total_k >= most || (int64_t)p->max_q * (p->heads / p->kv_heads) >= most ||
        (int64_t)p->batch * p->kv_heads >= ((int64_t)1 << 24))
        return set_error(F3M_ERR_UNSUPPORTED, "rows (times heads to a key head) must stay below 2^31 - 65536, batch * kv_heads below 2^24");
    return F3M_OK;
}

f3m_status check_rows(const f3m_rows &r, int64_t rows, const char *name) {
    if (!r.data) return set_error(F3M_ERR_INVALID_ARG, std::string(name) + " is null");
    if ((uintptr_t)r.data % 16 || r.row % 8 || r.head % 8 || r.row < 0 || r.head < 0)
        return set_error(F3M_ERR_INVALID_ARG, std::string(name) + ": data must be 16-byte aligned, strides multiples of 8 values and >= 0");
    if (rows > 1 && r.row >= 1 << 22) return set_error(F3M_ERR_UNSUPPORTED, std::string(name) + ": rows 2^22 values apart or more are not supported");
    return F3M_OK;
}

// results do not overlap themselves: one stride steps over all that the other spans
f3m_status check_result(const f3m_rows *r, int dim, int64_t rows, int heads, const char *name) {
    if (!r) return set_error(F3M_ERR_INVALID_ARG, std::string(name) + " is null");
    f3m_status st = check_rows(*r, rows, name);
    if (st != F3M_OK) return st;
    const bool by_row = (heads == 1 || r->head >= dim) && (rows == 1 || r->row >= (heads - 1) * (heads == 1 ? 0 : r->head) + dim);
    const bool by_head = (rows == 1 || r->row >= dim) && (heads == 1 || r->head >= (rows - 1) * (rows == 1 ? 0 : r->row) + dim);
    if (!by_row && !by_head) return set_error(F3M_ERR_INVALID_ARG, std::string(name) + ": rows that are written must not overlap");
    return F3M_OK;
}

f3m_status check_workspace(const void *p, int64_t bytes, int64_t needed) {
    if (needed > 0 && !p) return set_error(F3M_ERR_INVALID_ARG, "workspace is null");
    if (bytes < needed) return set_error(F3M_ERR_INVALID_ARG, "workspace is too small");
    if ((uintptr_t)p % 16) return set_error(F3M_ERR_INVALID_ARG, "workspace must be 16-byte aligned");
    return F3M_OK;
}

f3m_status check_cache(const f3m_cache *c) {
    if (!c) return set_error(F3M_ERR_INVALID_ARG, "cache is null");
    if (c->held != F3M_BF16 && c->held != F3M_F16 && c->held != F3M_E4M3) return set_error(F3M_ERR_INVALID_ARG, "held must be F3M_BF16, F3M_F16 or F3M_E4M3");
    if (c->kv_heads < 1 || c->head_dim < 8 || c->head_dim % 8) return set_error(F3M_ERR_INVALID_ARG, "kv_heads must be positive, head_dim a positive multiple of 8");
    if (c->held == F3M_E4M3 && c->head_dim % 16) return set_error(F3M_ERR_UNSUPPORTED, "8-bit caches need a head_dim that is a multiple of 16");
    if (c->head_dim > 128) return set_error(F3M_ERR_UNSUPPORTED, "head_dim above 128 is not supported");
    if (c->page_size < 8 || c->page_size > 1024 || (c->page_size & (c->page_size - 1)))
        return set_error(F3M_ERR_INVALID_ARG, "page_size must be a power of two from 8 to 1024");
    if ((int64_t)c->kv_heads * c->page_size >= (int64_t)1 << 31) return set_error(F3M_ERR_UNSUPPORTED, "kv_heads * page_size must be below 2^31");
    if (c->pages < 0 || c->pages >= ((int64_t)1 << 40) / c->page_size) return set_error(F3M_ERR_INVALID_ARG, "pages * page_size must be in [0, 2^40)");
    if (c->pages > 0) {
        if (!c->k || !c->v) return set_error(F3M_ERR_INVALID_ARG, "k or v of the cache is null");
        if ((uintptr_t)c->k % 16 || (uintptr_t)c->v % 16) return set_error(F3M_ERR_INVALID_ARG, "the cache's data must be 16-byte aligned");
        if (c->held == F3M_E4M3 && (!c->k_exp || !c->v_exp)) return set_error(F3M_ERR_INVALID_ARG, "an 8-bit cache needs k_exp and v_exp");
        if (c->held == F3M_E4M3 && ((uintptr_t)c->k_exp % 4 || (uintptr_t)c->v_exp % 4))
            return set_error(F3M_ERR_INVALID_ARG, "k_exp and v_exp must be 4-byte aligned");
    }
    return F3M_OK;
}

f3m_status check_cache_rows(const f3m_cache *c, int dtype, const f3m_rows *k, const f3m_rows *v, const int64_t *slots, int64_t tokens) {
    f3m_status st = check_cache(c);
    if (st != F3M_OK) return st;
    if (dtype != F3M_BF16 && dtype != F3M_F16) return set_error(F3M_ERR_INVALID_ARG, "dtype must be F3M_BF16 or F3M_F16");
    if (c->held != F3M_E4M3 && c->held != dtype) return set_error(F3M_ERR_INVALID_ARG, "a 16-bit cache holds the type of the rows");
    if (tokens < 0) return set_error(F3M_ERR_INVALID_ARG, "tokens must be >= 0");
    if (tokens == 0) return F3M_OK;
    if (!k || !v || !slots) return set_error(F3M_ERR_INVALID_ARG, "k, v or slots is null");
    st = check_rows(*k, tokens, "k");
    return st != F3M_OK ? st : check_rows(*v, tokens, "v");
}

f3m::AttendArgs attend_args(const f3m_attention_args &p) {
    f3m::AttendArgs a = {};
    a.batch = p.batch;
    a.heads = p.heads;
    a.kv_heads = p.kv_heads;
    a.group = p.heads / p.kv_heads;
    a.dim = p.head_dim;
    a.causal = p.causal != 0;
    a.window = p.window;
    a.sinks = p.window ? std::min(p.sinks, INT32_MAX - 65536) : 0;   // more keys than a sequence has; rounded up to tiles it stays an int
    a.scale = p.scale;
    a.total_q = p.total_q;
    a.total_k = p.total_k;
    a.max_q = (int)std::min<int64_t>(p.max_q, p.total_q);
    a.max_k = p.max_k;
    a.q_offsets = p.q_offsets;
    a.k_offsets = p.k_offsets;
    a.q = rows_of(p.q, p.total_q, p.head_dim);
    a.k = rows_of(p.k, p.total_k, p.head_dim);
    a.v = rows_of(p.v, p.total_k, p.head_dim);
    a.groups = p.batch * p.kv_heads;
    return a;
}

}  // namespace

extern "C" const char *f3m_last_error(void) { return g_last_error.c_str(); }

// plan for one point set (Y == nullptr) or for targets X and sources Y
static f3m_status make_plan(const float *X, int64_t n, const float *Y, int64_t ny, bool two_sets, int D,
                            float lengthscale, int interp_nodes, float eta, const f3m_options *opt, void *stream,
                            f3m_plan_t **plan_out) {
    if (!plan_out) return set_error(F3M_ERR_INVALID_ARG, "plan_out is null");
    *plan_out = nullptr;
    f3m_status st = check_problem(X, n, D, lengthscale);
    if (st != F3M_OK) return st;
    if (two_sets) {
        if (ny < 0) return set_error(F3M_ERR_INVALID_ARG, "ny must be >= 0");
        if (ny > 0 && !Y) return set_error(F3M_ERR_INVALID_ARG, "Y is null");
        if (ny >= ((int64_t)1 << 31)) return set_error(F3M_ERR_UNSUPPORTED, "ny must be below 2^31");
    }
    if (interp_nodes < 2) return set_error(F3M_ERR_INVALID_ARG, "interp_nodes must be >= 2");
    if (!finite_pos(eta)) return set_error(F3M_ERR_INVALID_ARG, "eta (far-field distance ratio) must be finite and > 0");
    if (opt && (opt->leaf_max < 0 || opt->max_depth < 0))
        return set_error(F3M_ERR_INVALID_ARG, "negative option value");
    if (opt && opt->small_field < 0) return set_error(F3M_ERR_INVALID_ARG, "small_field must be >= 0");
    if (opt && opt->route_min_points < 0) return set_error(F3M_ERR_INVALID_ARG, "route_min_points must be >= 0");
    if (opt && !(std::isfinite(opt->eta_smooth) && opt->eta_smooth >= 0.f))
        return set_error(F3M_ERR_INVALID_ARG, "eta_smooth must be finite and >= 0");
    if (interp_nodes > 8) return set_error(F3M_ERR_UNSUPPORTED, "interp_nodes above 8 is not supported");
    double r = std::pow((double)interp_nodes, (double)D);
    if (r > (double)f3m::MAX_NODES) return set_error(F3M_ERR_UNSUPPORTED, "interp_nodes^D exceeds the node cap of 4096");
    if ((double)eta > 1.0e4) return set_error(F3M_ERR_INVALID_ARG, "eta is unreasonably large");

    f3m_plan_s *P = nullptr;
    st = guarded([&] {
        P = new f3m_plan_s();
        P->n = n;
        P->D = D;
        P->p = interp_nodes;
        P->r = (int)std::lround(r);
        P->gamma = lengthscale;
        P->theta = eta;
        P->T = (int)std::ceil((double)eta * (double)eta);
        P->Lq = f3m::quant_depth(D);
        P->leaf_max = (opt && opt->leaf_max > 0) ? opt->leaf_max : 128;
        P->max_depth = opt ? opt->max_depth : 0;
        P->force_all_near = opt ? (opt->force_all_near != 0) : 0;
        P->no_overlap = opt ? (opt->overlap == 0) : 1;
        P->eta_smooth = opt ? opt->eta_smooth : 0.f;
        P->adaptive_far = opt ? (opt->adaptive_far != 0) : 0;
        P->rho = opt ? opt->small_field : 0;
        P->route_given = opt && opt->route_min_points > 0;
        P->route_min_n = P->route_given ? opt->route_min_points : ((int64_t)1 << 24);
        F3M_HIP(hipGetDevice(&P->device));
        if (two_sets) {
            P->src.reset(new f3m_source());
            P->src->n = ny;
        }
        // with no targets there is nothing to compute, with no sources the product is zero
        if (n > 0 && (!two_sets || ny > 0)) {
            f3m::ReleaseScope scope((hipStream_t)stream);
            f3m::build_plan(*P, X, two_sets ? Y : nullptr, (hipStream_t)stream);
        }
    });
    if (st != F3M_OK) {
        delete P;
        (void)hipGetLastError();
        return st;
    }
    *plan_out = P;
    return F3M_OK;
}

extern "C" {

f3m_status f3m_plan_ex(const float *X, int64_t n, int D, float lengthscale, int interp_nodes, float eta,
                       const f3m_options *opt, void *stream, f3m_plan_t **plan_out) {
    return make_plan(X, n, nullptr, 0, false, D, lengthscale, interp_nodes, eta, opt, stream, plan_out);
}

f3m_status f3m_plan_xy(const float *X, int64_t nx, const float *Y, int64_t ny, int D, float lengthscale,
                       int interp_nodes, float eta, const f3m_options *opt, void *stream, f3m_plan_t **plan_out) {
    return make_plan(X, nx, Y, ny, true, D, lengthscale, interp_nodes, eta, opt, stream, plan_out);
}

f3m_status f3m_plan(const float *X, int64_t n, int D, float lengthscale, int interp_nodes, float eta, void *stream,
                    f3m_plan_t **plan_out) {
    return f3m_plan_ex(X, n, D, lengthscale, interp_nodes, eta, nullptr, stream, plan_out);
}

f3m_status f3m_kmvm(f3m_plan_t *plan, const float *b, float *y, void *stream) {
    if (!plan) return set_error(F3M_ERR_INVALID_ARG, "plan is null");
    if (plan->n == 0) return F3M_OK;
    if (!y) return set_error(F3M_ERR_INVALID_ARG, "y is null");
    if (plan->ns() == 0) return guarded([&] { f3m::run_zero(y, plan->n, (hipStream_t)stream); });   // no sources
    if (!b) return set_error(F3M_ERR_INVALID_ARG, "b is null");
    if (b == y) return set_error(F3M_ERR_INVALID_ARG, "b and y must not overlap");
    return guarded([&] { f3m::run_kmvm(*plan, b, y, (hipStream_t)stream); });
}

f3m_status f3m_kmvm_multi(f3m_plan_t *plan, const float *B, int64_t ldb, float *Y, int64_t ldy, int m, void *stream) {
    if (!plan) return set_error(F3M_ERR_INVALID_ARG, "plan is null");
    if (m < 0) return set_error(F3M_ERR_INVALID_ARG, "m must be >= 0");
    if (m == 0 || plan->n == 0) return F3M_OK;
    if (!Y) return set_error(F3M_ERR_INVALID_ARG, "Y is null");
    if (ldy < plan->n) return set_error(F3M_ERR_INVALID_ARG, "ldy must be at least the number of targets");
    if (plan->ns() == 0)
        return guarded([&] { for (int j = 0; j < m; ++j) f3m::run_zero(Y + (int64_t)j * ldy, plan->n, (hipStream_t)stream); });
    if (!B) return set_error(F3M_ERR_INVALID_ARG, "B is null");
    if (ldb < plan->ns()) return set_error(F3M_ERR_INVALID_ARG, "ldb must be at least the number of sources");
    if (B == Y) return set_error(F3M_ERR_INVALID_ARG, "B and Y must not overlap");
    return guarded([&] { f3m::run_kmvm_multi(*plan, B, ldb, Y, ldy, m, (hipStream_t)stream); });
}

f3m_status direct_kmvm(const float *X, int64_t n, int D, float lengthscale, const float *b, float *y, void *stream) {
    f3m_status st = check_problem(X, n, D, lengthscale);
    if (st != F3M_OK) return st;
    if (n == 0) return F3M_OK;
    if (!b || !y) return set_error(F3M_ERR_INVALID_ARG, "b or y is null");
    if (b == y) return set_error(F3M_ERR_INVALID_ARG, "b and y must not overlap");
    return guarded([&] { f3m::run_direct(X, n, X, n, D, lengthscale, b, y, (hipStream_t)stream); });
}

f3m_status direct_kmvm_xy(const float *X, int64_t nx, const float *Y, int64_t ny, int D, float lengthscale,
                          const float *b, float *y, void *stream) {
    f3m_status st = check_problem(X, nx, D, lengthscale);
    if (st != F3M_OK) return st;
    st = check_problem(Y, ny, D, lengthscale);
    if (st != F3M_OK) return st;
    if (nx == 0) return F3M_OK;
    if (!y) return set_error(F3M_ERR_INVALID_ARG, "y is null");
    if (ny == 0) return guarded([&] { f3m::run_zero(y, nx, (hipStream_t)stream); });
    if (!b) return set_error(F3M_ERR_INVALID_ARG, "b is null");
    if (b == y) return set_error(F3M_ERR_INVALID_ARG, "b and y must not overlap");
    return guarded([&] { f3m::run_direct(X, nx, Y, ny, D, lengthscale, b, y, (hipStream_t)stream); });
}

f3m_status direct_kmvm_rows_f64(const float *X, int64_t n, int D, float lengthscale, const float *b,
                                const int64_t *rows, int64_t m, double *y64, void *stream) {
    f3m_status st = check_problem(X, n, D, lengthscale);
    if (st != F3M_OK) return st;
    if (m < 0) return set_error(F3M_ERR_INVALID_ARG, "m must be >= 0");
    if (m == 0) return F3M_OK;
    if (n == 0) return set_error(F3M_ERR_INVALID_ARG, "rows requested of an empty problem");
    if (!b || !rows || !y64) return set_error(F3M_ERR_INVALID_ARG, "b, rows or y64 is null");
    return guarded([&] { f3m::run_direct_rows_f64(X, X, n, D, lengthscale, b, rows, m, y64, (hipStream_t)stream); });
}

f3m_status direct_kmvm_rows_f64_static(const float *X, int64_t n, int D, float lengthscale, const float *b,
                                       const int64_t *rows, int64_t m, double *y64, void *stream) {
    f3m_status st = check_problem(X, n, D, lengthscale);
    if (st != F3M_OK) return st;
    if (m < 0) return set_error(F3M_ERR_INVALID_ARG, "m must be >= 0");
    if (m == 0) return F3M_OK;
    if (n == 0) return set_error(F3M_ERR_INVALID_ARG, "rows requested of an empty problem");
    if (!b || !rows || !y64) return set_error(F3M_ERR_INVALID_ARG, "b, rows or y64 is null");
    return guarded([&] { f3m::run_direct_rows_f64_static(X, n, D, lengthscale, b, rows, m, y64, (hipStream_t)stream); });
}

f3m_status direct_kmvm_xy_rows_f64(const float *X, int64_t nx, const float *Y, int64_t ny, int D, float lengthscale,
                                   const float *b, const int64_t *rows, int64_t m, double *y64, void *stream) {
    f3m_status st = check_problem(X, nx, D, lengthscale);
    if (st != F3M_OK) return st;
    st = check_problem(Y, ny, D, lengthscale);
    if (st != F3M_OK) return st;
    if (m < 0) return set_error(F3M_ERR_INVALID_ARG, "m must be >= 0");
    if (m == 0) return F3M_OK;
    if (nx == 0) return set_error(F3M_ERR_INVALID_ARG, "rows requested of an empty set of targets");
    if (!rows || !y64) return set_error(F3M_ERR_INVALID_ARG, "rows or y64 is null");
    if (ny == 0) return guarded([&] { F3M_HIP(hipMemsetAsync(y64, 0, sizeof(double) * (size_t)m, (hipStream_t)stream)); });
    if (!b) return set_error(F3M_ERR_INVALID_ARG, "b is null");
    return guarded([&] { f3m::run_direct_rows_f64(X, Y, ny, D, lengthscale, b, rows, m, y64, (hipStream_t)stream); });
}

f3m_status f3m_cg_solve(f3m_plan_t *plan, float lambda, const float *b, float *x, int max_iter, float tol,
                        int *iters_host, float *history_host, void *stream) {
    if (iters_host) *iters_host = 0;
    if (!plan) return set_error(F3M_ERR_INVALID_ARG, "plan is null");
    if (plan->src) return set_error(F3M_ERR_INVALID_ARG, "f3m_cg_solve needs a one-set plan (a square operator)");
    if (!(std::isfinite(lambda) && lambda >= 0.f)) return set_error(F3M_ERR_INVALID_ARG, "lambda must be finite and >= 0");
    if (max_iter < 0) return set_error(F3M_ERR_INVALID_ARG, "max_iter must be >= 0");
    if (!(std::isfinite(tol) && tol >= 0.f)) return set_error(F3M_ERR_INVALID_ARG, "tol must be finite and >= 0");
    if (plan->n == 0) return F3M_OK;
    if (!b || !x) return set_error(F3M_ERR_INVALID_ARG, "b or x is null");
    if (b == x) return set_error(F3M_ERR_INVALID_ARG, "b and x must not overlap");
    return guarded([&] { f3m::run_cg(*plan, lambda, b, x, max_iter, tol, iters_host, history_host, (hipStream_t)stream); });
}

int64_t f3m_attention_workspace(const f3m_attention_args *args) {
    f3m_status st = check_attention(args, true);   // also asked for calls over a cache
    return st != F3M_OK ? -(int64_t)st : f3m::attend_workspace(attend_args(*args), args->max_k);
}

int64_t f3m_attention_grad_workspace(const f3m_attention_args *args) {
    f3m_status st = check_attention(args);
    return st != F3M_OK ? -(int64_t)st : f3m::attend_grad_workspace(attend_args(*args), args->max_k);
}

f3m_status f3m_attention(const f3m_attention_args *args, const f3m_rows *out, float *lse, void *workspace, int64_t workspace_bytes,
                         void *stream) {
    f3m_status st = check_attention(args);
    if (st == F3M_OK && args->total_q > 0) {
        st = check_rows(args->q, args->total_q, "q");
        if (st == F3M_OK && args->total_k > 0) st = check_rows(args->k, args->total_k, "k");
        if (st == F3M_OK && args->total_k > 0) st = check_rows(args->v, args->total_k, "v");
        if (st == F3M_OK) st = check_result(out, args->head_dim, args->total_q, args->heads, "out");
        if (st == F3M_OK && !lse) st = set_error(F3M_ERR_INVALID_ARG, "lse is null");
    }
    if (st != F3M_OK || args->total_q == 0 || args->batch == 0) return st;
    f3m::AttendArgs a = attend_args(*args);
    st = check_workspace(workspace, workspace_bytes, f3m::attend_workspace(a, args->max_k));
    if (st != F3M_OK) return st;
    a.out = rows_of(*out, args->total_q, args->head_dim);
    a.lse = lse;
    return guarded([&] { f3m::run_attend(a, args->max_k, args->dtype == F3M_F16, false, workspace, (hipStream_t)stream); });
}

f3m_status f3m_attention_grad(const f3m_attention_args *args, const f3m_rows *dout, const f3m_rows *out, const float *lse,
                              const f3m_rows *dq, const f3m_rows *dk, const f3m_rows *dv, void *workspace, int64_t workspace_bytes,
                              void *stream) {
    f3m_status st = check_attention(args);
    if (st != F3M_OK || args->batch == 0) return st;
    if (args->total_q > 0) {
        if (!dout || !out || !lse) return set_error(F3M_ERR_INVALID_ARG, "dout, out or lse is null");
        st = check_rows(args->q, args->total_q, "q");
        if (st == F3M_OK) st = check_rows(*dout, args->total_q, "dout");
        if (st == F3M_OK) st = check_rows(*out, args->total_q, "out");
        if (st == F3M_OK) st = check_result(dq, args->head_dim, args->total_q, args->heads, "dq");
    }
    if (st == F3M_OK && args->total_k > 0) {
        st = check_rows(args->k, args->total_k, "k");
        if (st == F3M_OK) st = check_rows(args->v, args->total_k, "v");
        if (st == F3M_OK) st = check_result(dk, args->head_dim, args->total_k, args->kv_heads, "dk");
        if (st == F3M_OK) st = check_result(dv, args->head_dim, args->total_k, args->kv_heads, "dv");
    }
    if (st != F3M_OK) return st;
    f3m::AttendArgs a = attend_args(*args);
    st = check_workspace(workspace, workspace_bytes, f3m::attend_grad_workspace(a, args->max_k));
    if (st != F3M_OK) return st;
    if (args->total_q > 0) {
        a.dout = rows_of(*dout, args->total_q, args->head_dim);
        a.out = rows_of(*out, args->total_q, args->head_dim);
        a.lse = const_cast<float *>(lse);
        a.dq = rows_of(*dq, args->total_q, args->head_dim);
    }
    if (args->total_k > 0) {
        a.dk = rows_of(*dk, args->total_k, args->head_dim);
        a.dv = rows_of(*dv, args->total_k, args->head_dim);
    }
    return guarded([&] { f3m::run_attend_grad(a, args->max_k, args->dtype == F3M_F16, workspace, (hipStream_t)stream); });
}

f3m_status f3m_cache_write(const f3m_cache *cache, int dtype, const f3m_rows *k, const f3m_rows *v, const int64_t *slots, int64_t tokens,
                           void *stream) {
    f3m_status st = check_cache_rows(cache, dtype, k, v, slots, tokens);
    if (st != F3M_OK || tokens == 0) return st;
    return guarded([&] { f3m::run_cache_rows(*cache, dtype == F3M_F16, slots, tokens, *k, *v, true, (hipStream_t)stream); });
}

f3m_status f3m_cache_read(const f3m_cache *cache, int dtype, const f3m_rows *k, const f3m_rows *v, const int64_t *slots, int64_t tokens,
                          void *stream) {
    f3m_status st = check_cache_rows(cache, dtype, k, v, slots, tokens);
    if (st != F3M_OK || tokens == 0) return st;
    st = check_result(k, cache->head_dim, tokens, cache->kv_heads, "k");
    if (st == F3M_OK) st = check_result(v, cache->head_dim, tokens, cache->kv_heads, "v");
    if (st != F3M_OK) return st;
    return guarded([&] { f3m::run_cache_rows(*cache, dtype == F3M_F16, slots, tokens, *k, *v, false, (hipStream_t)stream); });
}

f3m_status f3m_cache_attention(const f3m_cache *cache, const f3m_attention_args *args, const int32_t *table, int64_t table_row,
                               int32_t table_cols, const int32_t *lengths, const f3m_rows *out, float *lse, void *workspace,
                               int64_t workspace_bytes, void *stream) {
    f3m_status st = check_attention(args, true);
    if (st == F3M_OK) st = check_cache(cache);
    if (st != F3M_OK) return st;
    if (cache->kv_heads != args->kv_heads || cache->head_dim != args->head_dim)
        return set_error(F3M_ERR_INVALID_ARG, "the cache has another number of heads or another head_dim");
    if (cache->held != F3M_E4M3 && cache->held != args->dtype)
        return set_error(F3M_ERR_INVALID_ARG, "a 16-bit cache holds the type of q");
    if (table_cols < 0 || table_row < table_cols) return set_error(F3M_ERR_INVALID_ARG, "table_row must be >= table_cols >= 0");
    if ((int64_t)table_cols * cache->page_size >= ((int64_t)1 << 31) - 65536)
        return set_error(F3M_ERR_UNSUPPORTED, "table_cols * page_size must be below 2^31 - 65536");
    if (args->total_q == 0 || args->batch == 0) return F3M_OK;
    if (!lengths || (table_cols > 0 && !table)) return set_error(F3M_ERR_INVALID_ARG, "table or lengths is null");
    st = check_rows(args->q, args->total_q, "q");
    if (st == F3M_OK) st = check_result(out, args->head_dim, args->total_q, args->heads, "out");
    if (st != F3M_OK) return st;
    if (!lse) return set_error(F3M_ERR_INVALID_ARG, "lse is null");
    f3m::AttendArgs a = attend_args(*args);
    st = check_workspace(workspace, workspace_bytes, f3m::attend_workspace(a, args->max_k));
    if (st != F3M_OK) return st;
    a.out = rows_of(*out, args->total_q, args->head_dim);
    a.lse = lse;
    a.k = {(char *)cache->k, 0, 0};
    a.v = {(char *)cache->v, 0, 0};
    a.k_exp = cache->k_exp;
    a.v_exp = cache->v_exp;
    a.table = table_cols > 0 && cache->pages > 0 ? table : (const int32_t *)lengths;   // no page: every length is cut to 0
    a.table_row = table_row;
    a.table_cols = cache->pages > 0 ? table_cols : 0;
    a.pages = cache->pages;
    a.page_shift = __builtin_ctz((unsigned)cache->page_size);
    a.lengths = lengths;
    return guarded([&] { f3m::run_attend(a, args->max_k, args->dtype == F3M_F16, cache->held == F3M_E4M3, workspace, (hipStream_t)stream); });
}

int64_t f3m_trim_memory(void) {
    int64_t freed = 0;
    (void)guarded([&] { freed = (int64_t)f3m::pool_trim(); });
    return freed;
}

void f3m_destroy(f3m_plan_t *plan) {
    if (!plan) return;
    (void)hipDeviceSynchronize();
    f3m::ReleaseScope idle;   // one wait for all of its buffers
    delete plan;
}

f3m_status f3m_plan_info(const f3m_plan_t *plan, f3m_info *out) {
    if (!plan || !out) return set_error(F3M_ERR_INVALID_ARG, "null argument");
    if (plan->n > 0 && plan->ns() > 0 && !plan->have_far_point_pairs) {
        // cached on first use; the plan is logically unchanged
        f3m_status st = guarded([&] { f3m::compute_far_point_pairs(*const_cast<f3m_plan_t *>(plan)); });
        if (st != F3M_OK) return st;
    }
    std::memset(out, 0, sizeof(*out));
    out->n = plan->n;
    out->D = plan->D;
    out->interp_nodes = plan->p;
    out->nodes_per_box = plan->r;
    out->depth = plan->L;
    out->quant_depth = plan->Lq;
    out->far_threshold = plan->T;
    out->edge = plan->E;
    out->scale = plan->scale;
    for (int d = 0; d < F3M_MAX_DIM; ++d) out->alpha[d] = plan->alpha[d];
    for (int l = 0; l <= plan->L && built(plan); ++l) {
        out->nboxes[l] = plan->lev[l].nb;
        out->max_box[l] = plan->lev[l].max_box;
        out->near_pairs[l] = plan->lev[l].near_sz;
        out->far_pairs[l] = plan->lev[l].far_sz;
    }
    for (int l = 0; l <= plan->L && built(plan); ++l) out->far_point_pairs[l] = plan->lev[l].far_point_pairs;
    out->near_point_pairs = plan->near_point_pairs;
    out->smooth_depth = plan->smooth_depth;
    for (int l = 0; l <= plan->L && built(plan); ++l) {
        out->small_pairs[l] = plan->lev[l].small_sz;
        out->small_point_pairs[l] = plan->lev[l].small_point_pairs;
    }
    for (int l = 0; l <= F3M_MAX_LEVELS; ++l) out->level_nodes[l] = (l >= 1 && l <= plan->L) ? plan->lev[l].p : 0;
    out->device_bytes = plan->bytes;
    return F3M_OK;
}

f3m_status f3m_plan_product_info(const f3m_plan_t *plan, f3m_product_info *out) {
    if (!plan || !out) return set_error(F3M_ERR_INVALID_ARG, "null argument");
    std::memset(out, 0, sizeof(*out));
    out->near_depth = plan->near_depth;
    for (int l = 1; l <= plan->L && built(plan); ++l) out->far_points[l] = plan->lev[l].far_points ? 1 : 0;
    return F3M_OK;
}

int f3m_plan_near_weighted(const f3m_plan_t *plan) { return plan ? plan->near_weighted : 0; }

f3m_status f3m_plan_get_perm(const f3m_plan_t *plan, uint32_t *perm_host) {
    if (!plan || !perm_host) return set_error(F3M_ERR_INVALID_ARG, "null argument");
    return guarded([&] { copy_to_host(perm_host, plan->perm.p, built(plan) ? (size_t)plan->n : 0); });
}

f3m_status f3m_plan_get_point_keys(const f3m_plan_t *plan, uint32_t *keys_host) {
    if (!plan || !keys_host) return set_error(F3M_ERR_INVALID_ARG, "null argument");
    return guarded([&] { copy_to_host(keys_host, plan->keys.p, built(plan) ? (size_t)plan->n : 0); });
}

f3m_status f3m_plan_get_boxes(const f3m_plan_t *plan, int level, uint32_t *keys_host, uint32_t *starts_host) {
    if (!plan || !keys_host || !starts_host) return set_error(F3M_ERR_INVALID_ARG, "null argument");
    if (!built(plan) || level < 0 || level > plan->L) return set_error(F3M_ERR_INVALID_ARG, "level out of range");
    return guarded([&] {
        const f3m_level &lv = plan->lev[level];
        copy_to_host(keys_host, lv.key.p, (size_t)lv.nb);
        copy_to_host(starts_host, lv.start.p, (size_t)lv.nb + 1);
    });
}

f3m_status f3m_plan_source_info(const f3m_plan_t *plan, f3m_source_info *out) {
    if (!plan || !out) return set_error(F3M_ERR_INVALID_ARG, "null argument");
    std::memset(out, 0, sizeof(*out));
    out->n = plan->ns();
    out->two_sets = plan->src ? 1 : 0;
    for (int d = 0; d < F3M_MAX_DIM; ++d) out->alpha[d] = plan->salpha()[d];
    for (int l = 0; l <= plan->L && built(plan); ++l) {
        out->nboxes[l] = plan->slev(l).nb;
        out->max_box[l] = plan->slev(l).max_box;
    }
    return F3M_OK;
}

f3m_status f3m_plan_get_source_perm(const f3m_plan_t *plan, uint32_t *perm_host) {
    if (!plan || !perm_host) return set_error(F3M_ERR_INVALID_ARG, "null argument");
    return guarded([&] { copy_to_host(perm_host, plan->sperm(), built(plan) ? (size_t)plan->ns() : 0); });
}

f3m_status f3m_plan_get_source_boxes(const f3m_plan_t *plan, int level, uint32_t *keys_host, uint32_t *starts_host) {
    if (!plan || !keys_host || !starts_host) return set_error(F3M_ERR_INVALID_ARG, "null argument");
    if (!built(plan) || level < 0 || level > plan->L) return set_error(F3M_ERR_INVALID_ARG, "level out of range");
    return guarded([&] {
        const f3m_level &lv = plan->slev(level);
        copy_to_host(keys_host, lv.key.p, (size_t)lv.nb);
        copy_to_host(starts_host, lv.start.p, (size_t)lv.nb + 1);
    });
}

f3m_status f3m_plan_get_list(const f3m_plan_t *plan, int level, int kind, uint64_t *row_ptr_host, uint32_t *cols_host) {
    if (!plan || !row_ptr_host || !cols_host) return set_error(F3M_ERR_INVALID_ARG, "null argument");
    if (!built(plan) || level < 0 || level > plan->L) return set_error(F3M_ERR_INVALID_ARG, "level out of range");
    if (kind < 0 || kind > 2) return set_error(F3M_ERR_INVALID_ARG, "kind must be 0 (near), 1 (far) or 2 (small field)");
    return guarded([&] {
        const f3m_level &lv = plan->lev[level];
        if (kind == 2) {
            if (lv.small_ptr.p) {
                copy_to_host(row_ptr_host, lv.small_ptr.p, (size_t)lv.nb + 1);
                copy_to_host(cols_host, lv.small_col.p, (size_t)lv.small_sz);
            } else {
                std::memset(row_ptr_host, 0, sizeof(uint64_t) * ((size_t)lv.nb + 1));
            }
            return;
        }
        copy_to_host(row_ptr_host, kind ? lv.far_ptr.p : lv.near_ptr.p, (size_t)lv.nb + 1);
        if (kind && (lv.far_implicit || lv.far_points)) {
            // this depth keeps only the lengths of its far rows
            f3m::DevBuf<uint32_t> cols;
            cols.alloc((size_t)lv.far_sz);
            f3m::materialize_far(*plan, level, cols.p, nullptr);
            copy_to_host(cols_host, cols.p, (size_t)lv.far_sz);
        } else {
            copy_to_host(cols_host, kind ? lv.far_col.p : lv.near_col.p, (size_t)(kind ? lv.far_sz : lv.near_sz));
        }
    });
}

f3m_status f3m_stage_times(f3m_plan_t *plan, f3m_times *out) {
    if (!plan || !out) return set_error(F3M_ERR_INVALID_ARG, "null argument");
    return guarded([&] {
        f3m_times t = plan->times;
        if (plan->have_kmvm_times) {
            F3M_HIP(hipEventSynchronize(plan->t_end));
            F3M_HIP(elapsed(&t.permute_in, plan->t_begin, plan->t_in));
            F3M_HIP(hipEventSynchronize(plan->t_p2p1));
            F3M_HIP(elapsed(&t.p2p, plan->t_p2p0, plan->t_p2p1));
            F3M_HIP(elapsed(&t.permute_out, plan->t_out, plan->t_end));
            F3M_HIP(elapsed(&t.kmvm_total, plan->t_begin, plan->t_end));
            t.p2m = t.m2l = t.l2p = 0.f;
            for (int l = 1; l <= plan->L; ++l) {
                if (plan->lev[l].far_sz == 0 || plan->far_events.size() < (size_t)(l + 1) * 6) continue;
                hipEvent_t *ev = &plan->far_events[(size_t)l * 6];
                if (!ev[5]) continue;
                float ms = 0.f;
                F3M_HIP(elapsed(&ms, ev[0], ev[1])); t.p2m += ms;
                F3M_HIP(elapsed(&ms, ev[2], ev[3])); t.m2l += ms;
                F3M_HIP(elapsed(&ms, ev[4], ev[5])); t.l2p += ms;
            }
            float wait = 0.f;
            F3M_HIP(elapsed(&wait, plan->t_wait0, plan->t_wait1));
            t.l2p = std::max(0.f, t.l2p - wait);
        }
        *out = t;
    });
}

f3m_status f3m_level_times(f3m_plan_t *plan, int level, float *ms_host) {
    if (!plan || !ms_host) return set_error(F3M_ERR_INVALID_ARG, "null argument");
    if (!built(plan) || level < 0 || level > plan->L) return set_error(F3M_ERR_INVALID_ARG, "level out of range");
    return guarded([&] {
        ms_host[0] = ms_host[1] = ms_host[2] = 0.f;
        if (!plan->have_kmvm_times || plan->lev[level].far_sz == 0 || plan->far_events.size() < (size_t)(level + 1) * 6)
            return;
        hipEvent_t *ev = &plan->far_events[(size_t)level * 6];
        if (!ev[5]) return;
        F3M_HIP(hipEventSynchronize(plan->t_end));
        for (int k = 0; k < 3; ++k) F3M_HIP(elapsed(&ms_host[k], ev[2 * k], ev[2 * k + 1]));
        if (level == plan->tree_lmax) {
            float wait = 0.f;
            F3M_HIP(elapsed(&wait, plan->t_wait0, plan->t_wait1));
            ms_host[2] = std::max(0.f, ms_host[2] - wait);
        }
    });
}

}  // extern "C"
