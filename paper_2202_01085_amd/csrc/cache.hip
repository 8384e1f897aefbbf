// Paged cache of keys and values: rows written to slots, read back.
//
// 8-bit codes: a row (token, key head) of D values gets one exponent e, the least with max|x| <= 448 2^e over its finite values
// (448: the largest e4m3 number), and the codes e4m3(x 2^-e).  A power of two as the scale makes scaling exact both ways: the
// only rounding is that to e4m3, at most half a step, 2^-4 of a value (2^-10 2^e of the small ones).  One exponent byte to 8 .. 128
// codes.  Infinities and NaN become NaN, the one such code that e4m3 has.
//
// For few tokens bound by the launch: 64 tokens 3 us each.  32768 tokens of 8 heads of 128: written in 56 us, 3.6 TB/s, and read in 39, 5.2 TB/s,
// where a copy reaches 6.2: vector issue takes 0.74 and 0.56 of the cycles, a good part of it the 64-bit division that finds a row's token.  One
// kernel for K and V, 8 values to a lane, a row's lanes share its maximum.
#include "attend.h"

namespace f3m {

namespace {

constexpr int NT = 256;

struct CacheArgs {
    char *k, *v;              // pages: (pages, kv_heads, page_size, dim)
    uint8_t *k_exp, *v_exp;   // (pages, kv_heads, page_size)
    int kv_heads, dim, page_shift;
    int64_t slots, tokens;
    const int64_t *slot;
    Rows rk, rv;
};

// row of the cache for a slot and head, -1 if there is none
__device__ __forceinline__ int64_t cache_row(const CacheArgs &a, int64_t slot, int head) {
    if (slot < 0 || slot >= a.slots) return -1;
    return (((slot >> a.page_shift) * a.kv_heads + head) << a.page_shift) + (slot & ((1 << a.page_shift) - 1));
}

// LANES lanes to a row; rows of K, then rows of V
template <class T, int LANES, bool E8> __global__ __launch_bounds__(NT) void write_rows(CacheArgs a) {
    const int64_t at = (int64_t)blockIdx.x * (NT / LANES) + threadIdx.x / LANES, rows = a.tokens * a.kv_heads;
    if (at >= 2 * rows) return;
    const bool second = at >= rows;
    const int64_t row = second ? at - rows : at, token = row / a.kv_heads;
    const int head = (int)(row % a.kv_heads), x = threadIdx.x % LANES * 8;
    const int64_t to = cache_row(a, a.slot[token], head);
    const Rows &from = second ? a.rv : a.rk;
    char *pages = second ? a.v : a.k;
    const bool in = to >= 0 && x < a.dim;
    s16x8 w = {};
    if (in) w = *(const s16x8 *)(from.p + 2 * (token * from.row + (int64_t)head * from.head + x));
    if (!E8) {
        if (in) *(s16x8 *)(pages + 2 * (to * a.dim + x)) = w;
        return;
    }
    float f[8], most = 0.f;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        f[j] = T::up((uint16_t)w[j]);
        const bool finite = (w[j] & T::nonfinite) != T::nonfinite;
        most = fmaxf(most, finite ? fabsf(f[j]) : 0.f);
    }
#pragma unroll
    for (int by = LANES / 2; by > 0; by >>= 1) most = fmaxf(most, __shfl_xor(most, by));
    int e = 0;
    const float m = frexpf(most, &e);
    const int byte = most == 0.f ? 127 : min(max(e - 9 + (m > 0.875f) + 127, 1), 254);
    const float inv = __builtin_bit_cast(float, (uint32_t)(254 - byte) << 23);
    if (!in) return;
    uint32_t lo = 0, hi = 0;
    lo = __builtin_amdgcn_cvt_pk_fp8_f32(f[0] * inv, f[1] * inv, lo, false);
    lo = __builtin_amdgcn_cvt_pk_fp8_f32(f[2] * inv, f[3] * inv, lo, true);
    hi = __builtin_amdgcn_cvt_pk_fp8_f32(f[4] * inv, f[5] * inv, hi, false);
    hi = __builtin_amdgcn_cvt_pk_fp8_f32(f[6] * inv, f[7] * inv, hi, true);
    *(u32x2 *)(pages + to * a.dim + x) = (u32x2){lo, hi};
    if (x == 0) (second ? a.v_exp : a.k_exp)[to] = (uint8_t)byte;
}

template <class T, int LANES, bool E8> __global__ __launch_bounds__(NT) void read_rows(CacheArgs a) {
    const int64_t at = (int64_t)blockIdx.x * (NT / LANES) + threadIdx.x / LANES, rows = a.tokens * a.kv_heads;
    if (at >= 2 * rows) return;
    const bool second = at >= rows;
    const int64_t row = second ? at - rows : at, token = row / a.kv_heads;
    const int head = (int)(row % a.kv_heads), x = threadIdx.x % LANES * 8;
    if (x >= a.dim) return;
    const int64_t from = cache_row(a, a.slot[token], head);
    const char *pages = second ? a.v : a.k;
    u32x4 w = {0, 0, 0, 0};
    if (from >= 0) {
        if (E8) {
            const u32x2 c = *(const u32x2 *)(pages + from * a.dim + x);
            const float scale = __builtin_bit_cast(float, (uint32_t)(second ? a.v_exp : a.k_exp)[from] << 23);
            w = (u32x4){T::template codes<false>(c[0], scale), T::template codes<true>(c[0], scale),
                        T::template codes<false>(c[1], scale), T::template codes<true>(c[1], scale)};
        } else {
            w = *(const u32x4 *)(pages + 2 * (from * a.dim + x));
        }
    }
    const Rows &to = second ? a.rv : a.rk;
    *(u32x4 *)(to.p + 2 * (token * to.row + (int64_t)head * to.head + x)) = w;
}

template <class T, int LANES, bool E8> void launch(const CacheArgs &a, bool write, hipStream_t st) {
    const int64_t blocks = cdiv(2 * a.tokens * a.kv_heads, NT / LANES);
    if (blocks > (1 << 24) - 1) fail(F3M_ERR_UNSUPPORTED, "cache: too many rows for one call (2^24 blocks of 16)");
    if (write) write_rows<T, LANES, E8><<<dim3((uint32_t)blocks), NT, 0, st>>>(a);
    else read_rows<T, LANES, E8><<<dim3((uint32_t)blocks), NT, 0, st>>>(a);
    F3M_HIP(hipGetLastError());
}

template <class T, bool E8> void launch_dim(const CacheArgs &a, bool write, hipStream_t st) {
    if (a.dim <= 32) launch<T, 4, E8>(a, write, st);
    else if (a.dim <= 64) launch<T, 8, E8>(a, write, st);
    else launch<T, 16, E8>(a, write, st);
}

}  // namespace

void run_cache_rows(const f3m_cache &c, bool f16, const int64_t *slot, int64_t tokens, const f3m_rows &k, const f3m_rows &v, bool write,
                    hipStream_t st) {
    CacheArgs a;
    a.k = (char *)c.k;
    a.v = (char *)c.v;
    a.k_exp = c.k_exp;
    a.v_exp = c.v_exp;
    a.kv_heads = c.kv_heads;
    a.dim = c.head_dim;
    a.page_shift = __builtin_ctz(c.page_size);
    a.slots = c.pages << a.page_shift;
    a.tokens = tokens;
    a.slot = slot;
    a.rk = {(char *)k.data, k.row, k.head};
    a.rv = {(char *)v.data, v.row, v.head};
    const bool e8 = c.held == F3M_E4M3;
    if (f16) e8 ? launch_dim<F16, true>(a, write, st) : launch_dim<F16, false>(a, write, st);
    else e8 ? launch_dim<Bf16, true>(a, write, st) : launch_dim<Bf16, false>(a, write, st);
}

}  // namespace f3m
