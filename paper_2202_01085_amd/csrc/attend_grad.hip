// Row-normalised products (attention): gradients.  With P_ij the weights, L_i the logarithms of their sums, delta_i = dO_i.O_i:
//   dV_j = sum_i P_ij dO_i    dS_ij = P_ij (dO_i.v_j - delta_i)    dQ_i = scale sum_j dS_ij k_j    dK_j = scale sum_i dS_ij q_i
// P is made again from q, k and L.  Two kernels, one that keeps rows and goes over keys (dQ) and one that keeps keys and goes over
// the rows of all heads that share them (dK, dV): seven products a pair where one kernel would need five, but each gradient is
// summed in one place and one order, without atomics, so that results repeat bit for bit.
//
// P and dS are rounded to the inputs' type for the matrix cores.  fp16: P is held times 2^12; dS, whose size follows the loss, times
// a power of two per kept row or key that goes down when a larger one comes, so both keep 11 bits.
#include "attend.h"

#include <algorithm>

namespace f3m {

namespace {

constexpr int NT = 256;

// stat = (log2 of the row's sum, or +inf for an empty row, so that its weights are 0; dO.O): 16 lanes to a row, 8 values each
template <class T> __global__ __launch_bounds__(NT) void row_stats(AttendArgs a) {
    const int64_t row = (int64_t)blockIdx.x * 16 + threadIdx.x / 16, all = a.total_q * a.heads;
    const int x = threadIdx.x % 16 * 8;
    float sum = 0.f;
    const int64_t token = row / a.heads;
    const int head = (int)(row % a.heads);
    if (row < all && x < a.dim) {
        const s16x8 g = *(const s16x8 *)(a.dout.p + 2 * (token * a.dout.row + (int64_t)head * a.dout.head + x));
        const s16x8 o = *(const s16x8 *)(a.out.p + 2 * (token * a.out.row + (int64_t)head * a.out.head + x));
#pragma unroll
        for (int j = 0; j < 8; ++j) sum += T::up((uint16_t)g[j]) * T::up((uint16_t)o[j]);
    }
#pragma unroll
    for (int by = 8; by > 0; by >>= 1) sum += __shfl_xor(sum, by);
    if (row < all && x == 0) {
        const float l = a.lse[row];
        const bool empty = l == NO_KEY;
        // a row whose dO or O is not finite makes what it adds to its keys NaN (also where tiles are cleaned)
        a.stat[row] = make_float2(empty ? __builtin_inff() : l * LOG2E + (sum - sum), empty ? 0.f : sum);
    }
}

// a power of two per lane that dS is divided by (fp16): raised, and what is summed so far lowered, when a larger dS comes
struct Unit {
    float u;   // dS / u is at most 2^15
    template <class T, int DB> __device__ __forceinline__ void fit(f32x16 &ds, f32x16 (&acc)[DB]) {
        if (!T::narrow) return;
        float most = 0.f;
#pragma unroll
        for (int i = 0; i < 16; ++i) most = fmaxf(most, fabsf(ds[i]));
        most = both_halves_max(most);
        if (__any(most > u * 32768.f)) {
            // 2^(exponent of most - 14): most / unit is below 2^15
            const float unit = fmaxf(u, __builtin_bit_cast(float, __builtin_bit_cast(uint32_t, most) & 0x7f800000u) * 0x1p-14f);
            const float by = u / unit;
            u = unit;
#pragma unroll
            for (int db = 0; db < DB; ++db)
#pragma unroll
                for (int i = 0; i < 16; ++i) acc[db][i] *= by;
        }
        const float inv = 1.f / u;
#pragma unroll
        for (int i = 0; i < 16; ++i) ds[i] *= inv;
    }
};
constexpr float LEAST_UNIT = 0x1p-100f;

// a tile of N rows of DP values from two tensors, on its way from memory to LDS
template <class T, int DP, int N> struct Pair {
    static constexpr int PIECES = DP / 8, COUNT = (N * PIECES + NT - 1) / NT;
    static constexpr bool ALL = N * PIECES % NT == 0;
    u32x4 x[COUNT], y[COUNT];
    template <class At> __device__ void load(const Rows &p, const Rows &q, int dim, int tid, At &&at) {   // at(row): (row of the tensors, head)
#pragma unroll
        for (int c = 0; c < COUNT; ++c) {
            const int i = tid + NT * c, row = i / PIECES, piece = i % PIECES;
            if (!ALL && row >= N) break;
            const int2 w = at(row);
            x[c] = load_piece<DP>(p.p, (int64_t)w.x * p.row + (int64_t)w.y * p.head, piece, dim);
            y[c] = load_piece<DP>(q.p, (int64_t)w.x * q.row + (int64_t)w.y * q.head, piece, dim);
        }
    }
    __device__ void clean(bool second) {
#pragma unroll
        for (int c = 0; c < COUNT; ++c) {
            x[c] = cleaned<T>(x[c]);
            if (second) y[c] = cleaned<T>(y[c]);
        }
    }
    __device__ void store(short *tx, short *ty, int tid) const {
#pragma unroll
        for (int c = 0; c < COUNT; ++c) {
            const int i = tid + NT * c, row = i / PIECES, piece = i % PIECES;
            if (!ALL && row >= N) break;
            *(u32x4 *)(tx + tile_at<DP>(row, piece)) = x[c];
            *(u32x4 *)(ty + tile_at<DP>(row, piece)) = y[c];
        }
    }
};

// dQ: 128 rows of one group to a block, 32 to a wave, tiles of 64 keys through LDS, as the forward kernel
template <class T, int DP> __global__ __launch_bounds__(NT, 2) void grad_rows(AttendArgs a) {
    constexpr int KS = DP / 16, DB = DP / 32, KT = 64;
    __shared__ __attribute__((aligned(16))) short tile[2][2][KT * DP];
    const Item it = block_of(a, blockIdx.x);
    if (it.group >= a.groups) return;
    const int b = it.group / a.kv_heads, hk = it.group % a.kv_heads;
    const Sequence s = sequence_of(a, b);
    const int rows = min(s.nq, a.max_q) * a.group, r0 = it.tile * 128;
    if (r0 >= rows) return;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const Limits first = limits_of(a, s, r0 / a.group), last = limits_of(a, s, min(r0 + 127, rows - 1) / a.group);
    const Tiles tiles = tiles_of<KT>(first, last, a.sinks);

    const int w0 = r0 + 32 * wave, row = min(w0 + (lane & 31), rows - 1), token = row / a.group, head = hk * a.group + row % a.group;
    const bool valid = w0 + (lane & 31) < rows, idle = w0 >= rows;
    const Limits mine = limits_of(a, s, token);
    const Limits wfirst = limits_of(a, s, min(w0, rows - 1) / a.group), wlast = limits_of(a, s, min(w0 + 31, rows - 1) / a.group);
    const float c = a.scale * LOG2E;
    const float2 stat = a.stat[(int64_t)(s.q0 + token) * a.heads + head];

    s16x8 q[KS], g[KS];
    f32x16 acc[DB];
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
        q[ks] = __builtin_bit_cast(s16x8, load_piece<DP>(a.q.p, (int64_t)(s.q0 + token) * a.q.row + (int64_t)head * a.q.head, 2 * ks + (lane >> 5), a.dim));
        g[ks] = __builtin_bit_cast(s16x8, load_piece<DP>(a.dout.p, (int64_t)(s.q0 + token) * a.dout.row + (int64_t)head * a.dout.head, 2 * ks + (lane >> 5), a.dim));
    }
#pragma unroll
    for (int db = 0; db < DB; ++db) acc[db] = (f32x16)0.f;
    Unit unit{LEAST_UNIT};

    auto block = [&](const short *kt, const short *vt, int kb, int key0, bool edge) {
        f32x16 p = (f32x16)0.f, d = (f32x16)0.f;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
            p = T::mma(frag_r<DP>(kt, 32 * kb, ks, lane), q[ks], p);
            d = T::mma(frag_r<DP>(vt, 32 * kb, ks, lane), g[ks], d);
        }
#pragma unroll
        for (int i = 0; i < 16; ++i) d[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(p[i], c, -stat.x)) * (d[i] - stat.y);
        if (edge) {
#pragma unroll
            for (int i = 0; i < 16; ++i) d[i] = sees(mine, a.sinks, key0 + 32 * kb + c_row(i, lane)) ? d[i] : 0.f;
        }
        unit.fit<T, DB>(d, acc);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const s16x8 w = as_operand<T>(d, h);
#pragma unroll
            for (int db = 0; db < DB; ++db) acc[db] = T::mma(frag_t<DP>(kt, 32 * kb + 16 * h, db, lane), w, acc[db]);
        }
    };

    if (tiles.count > 0) {
        Pair<T, DP, KT> next;
        // k is cleaned in tiles that the mask cuts for some row of the block: rows that see an infinity or NaN of k have such an lse
        auto whole = [&](int key0) { return key0 + KT <= first.hi && (key0 >= last.lo || key0 + KT <= a.sinks); };
        auto fetch = [&](int t) {
            const int key0 = tiles[t] * KT;
            next.load(a.k, a.v, a.dim, tid, [&](int r) { return make_int2(s.k0 + min(key0 + r, s.nk - 1), hk); });
        };
        auto keep = [&](int t, int buf) {
            if (!whole(tiles[t] * KT)) next.clean(false);
            next.store(tile[buf][0], tile[buf][1], tid);
        };
        fetch(0);
        keep(0, 0);
        __syncthreads();
        for (int n = 0; n < tiles.count; ++n) {
            const int buf = n & 1, key0 = tiles[n] * KT;
            if (n + 1 < tiles.count) fetch(n + 1);
            const bool none = idle || key0 >= wlast.hi || (key0 + KT <= wfirst.lo && key0 >= a.sinks);
            const bool full = key0 + KT <= wfirst.hi && (key0 >= wlast.lo || key0 + KT <= a.sinks);
            if (!none) {
                block(tile[buf][0], tile[buf][1], 0, key0, !full);
                block(tile[buf][0], tile[buf][1], 1, key0, !full);
            }
            if (n + 1 < tiles.count) keep(n + 1, buf ^ 1);
            __syncthreads();
        }
    }
    const float by = T::narrow ? a.scale * unit.u : a.scale;
    store_rows<T, DB>(acc, by, a.dq.p, (int64_t)(s.q0 + token) * a.dq.row + (int64_t)head * a.dq.head, a.dim, valid, lane);
}

// dK, dV: 128 keys of one group to a block, 32 to a wave with their k and v in registers; tiles of 32 rows of q and dO through LDS
template <class T, int DP> __global__ __launch_bounds__(NT, DP == 128 ? 1 : 2) void grad_keys(AttendArgs a) {
    constexpr int KS = DP / 16, DB = DP / 32, RT = 32;
    constexpr float LIFT = T::narrow ? 12.f : 0.f;
    __shared__ __attribute__((aligned(16))) short tile[2][2][RT * DP];
    __shared__ __attribute__((aligned(16))) float lse2[2][RT], delta[2][RT];
    __shared__ __attribute__((aligned(16))) int pos[2][RT];
    const Item it = block_of(a, blockIdx.x);
    if (it.group >= a.groups) return;
    const int b = it.group / a.kv_heads, hk = it.group % a.kv_heads;
    const Sequence s = sequence_of(a, b);
    const int k0 = (a.tiles - 1 - it.tile) * 128;   // the first keys have most rows
    if (k0 >= s.nk) return;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int off = s.nk - s.nq, nq = min(s.nq, a.max_q);   // position of token 0

    // tokens that see keys of [from, to): one interval, as keys of the sinks stay visible to all later tokens
    auto tokens = [&](int from, int to) {
        int lo = 0, hi = nq;
        if (a.causal) {
            lo = min(max(from - off, 0), nq);
            if (a.window && from >= a.sinks) hi = max(lo, (int)min((int64_t)nq, (int64_t)to - 1 + a.window - off));
        }
        return make_int2(lo, hi);
    };
    const int2 span = tokens(k0, min(k0 + 128, s.nk));
    const int row0 = span.x * a.group, row1 = span.y * a.group;

    const int w0 = k0 + 32 * wave, key = w0 + (lane & 31), kept = min(key, s.nk - 1);
    const bool valid = key < s.nk, idle = w0 >= s.nk;
    // positions [plo, phi) see this lane's key
    const int plo = a.causal ? key : INT32_MIN;
    const int64_t phi = !valid ? INT64_MIN : a.causal && a.window && key >= a.sinks ? (int64_t)key + a.window : INT64_MAX;
    const int wl = min(w0 + 31, s.nk - 1);
    const float c = a.scale * LOG2E;

    s16x8 k[KS], v[KS];
    f32x16 dk[DB], dv[DB];
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
        k[ks] = __builtin_bit_cast(s16x8, load_piece<DP>(a.k.p, (int64_t)(s.k0 + kept) * a.k.row + (int64_t)hk * a.k.head, 2 * ks + (lane >> 5), a.dim));
        v[ks] = __builtin_bit_cast(s16x8, load_piece<DP>(a.v.p, (int64_t)(s.k0 + kept) * a.v.row + (int64_t)hk * a.v.head, 2 * ks + (lane >> 5), a.dim));
    }
#pragma unroll
    for (int db = 0; db < DB; ++db) { dk[db] = (f32x16)0.f; dv[db] = (f32x16)0.f; }
    Unit unit{LEAST_UNIT};

    auto block = [&](int buf, int left, bool edge) {   // `left` rows of the tile exist
        const short *qt = tile[buf][0], *gt = tile[buf][1];
        f32x16 p = (f32x16)0.f, d = (f32x16)0.f;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
            p = T::mma(frag_r<DP>(qt, 0, ks, lane), k[ks], p);
            d = T::mma(frag_r<DP>(gt, 0, ks, lane), v[ks], d);
        }
#pragma unroll
        for (int i4 = 0; i4 < 4; ++i4) {
            const int r = c_row(4 * i4, lane);
            const float4 l = *(const float4 *)&lse2[buf][r], e = *(const float4 *)&delta[buf][r];
            const float ls[4] = {l.x, l.y, l.z, l.w}, de[4] = {e.x, e.y, e.z, e.w};
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int i = 4 * i4 + j;
                p[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(p[i], c, LIFT - ls[j]));
                d[i] = p[i] * (d[i] - de[j]);
            }
        }
        if (edge) {
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const int r = c_row(i, lane), at = pos[buf][r];
                const bool ok = r < left && at >= plo && at < phi;
                p[i] = ok ? p[i] : 0.f;
                d[i] = ok ? d[i] : 0.f;
            }
        }
        unit.fit<T, DB>(d, dk);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const s16x8 w = as_operand<T>(p, h), u = as_operand<T>(d, h);
#pragma unroll
            for (int db = 0; db < DB; ++db) {
                dv[db] = T::mma(frag_t<DP>(gt, 16 * h, db, lane), w, dv[db]);
                dk[db] = T::mma(frag_t<DP>(qt, 16 * h, db, lane), u, dk[db]);
            }
        }
    };

    if (row0 < row1) {
        Pair<T, DP, RT> next;
        float2 st = make_float2(0.f, 0.f);
        int at = 0;
        auto fetch = [&](int r0) {
            next.load(a.q, a.dout, a.dim, tid, [&](int r) {
                const int x = min(r0 + r, row1 - 1);
                return make_int2(s.q0 + x / a.group, hk * a.group + x % a.group);
            });
            if (tid < RT) {
                const int x = min(r0 + tid, row1 - 1);
                st = a.stat[(int64_t)(s.q0 + x / a.group) * a.heads + hk * a.group + x % a.group];
                at = x / a.group + off;
            }
        };
        // positions of a tile's first and last row; q and dO are cleaned in tiles that the mask cuts for some key of the block (rows with
        // an infinity or NaN have such a stat)
        auto place = [&](int r0) { return make_int2(r0 / a.group + off, min(r0 + RT - 1, row1 - 1) / a.group + off); };
        auto seen_by_all = [&](int2 at, int64_t from, int64_t to) {
            return !a.causal || (at.x >= to - 1 && (!a.window || at.y < from + a.window || to <= a.sinks));
        };
        auto keep = [&](int r0, int buf) {
            if (!(k0 + 128 <= s.nk && r0 + RT <= row1 && seen_by_all(place(r0), k0, k0 + 128))) next.clean(true);
            next.store(tile[buf][0], tile[buf][1], tid);
            if (tid < RT) { lse2[buf][tid] = st.x; delta[buf][tid] = st.y; pos[buf][tid] = at; }
        };
        fetch(row0);
        keep(row0, 0);
        __syncthreads();
        int buf = 0;
        for (int r0 = row0; r0 < row1; r0 += RT, buf ^= 1) {
            if (r0 + RT < row1) fetch(r0 + RT);
            const int2 at = place(r0);
            const bool none = idle || (a.causal && (at.y < w0 || (a.window && w0 >= a.sinks && at.x >= (int64_t)wl + a.window)));
            const bool full = w0 + 32 <= s.nk && r0 + RT <= row1 && seen_by_all(at, w0, w0 + 32);
            if (!none) block(buf, row1 - r0, !full);
            if (r0 + RT < row1) keep(r0 + RT, buf ^ 1);
            __syncthreads();
        }
    }
    const int64_t to = s.k0 + kept;
    store_rows<T, DB>(dv, T::narrow ? 0x1p-12f : 1.f, a.dv.p, to * a.dv.row + (int64_t)hk * a.dv.head, a.dim, valid, lane);
    store_rows<T, DB>(dk, T::narrow ? a.scale * 0x1p-12f * unit.u : a.scale, a.dk.p, to * a.dk.row + (int64_t)hk * a.dk.head, a.dim, valid, lane);
}

template <class T, int DP> void launch(AttendArgs a, int64_t max_k, hipStream_t st) {
    if (a.max_q && a.total_q) {
        row_stats<T><<<dim3((uint32_t)cdiv(a.total_q * a.heads, 16)), NT, 0, st>>>(a);
        F3M_HIP(hipGetLastError());
        a.tiles = (int)cdiv((int64_t)a.max_q * a.group, 128);
        const int64_t blocks = attend_blocks(a, a.tiles);
        grad_rows<T, DP><<<dim3((uint32_t)blocks), NT, 0, st>>>(a);
        F3M_HIP(hipGetLastError());
    }
    if (max_k && a.total_k) {
        a.tiles = (int)cdiv(max_k, 128);
        const int64_t blocks = attend_blocks(a, a.tiles);
        grad_keys<T, DP><<<dim3((uint32_t)blocks), NT, 0, st>>>(a);
        F3M_HIP(hipGetLastError());
    }
}

}  // namespace

int64_t attend_grad_workspace(const AttendArgs &a) { return a.total_q * a.heads * (int64_t)sizeof(float2); }

void run_attend_grad(AttendArgs a, int64_t max_k, bool f16, void *workspace, hipStream_t st) {
    if (!a.groups) return;
    a.stat = (float2 *)workspace;
    a.parts = 1;
    if (a.dim <= 32) f16 ? launch<F16, 32>(a, max_k, st) : launch<Bf16, 32>(a, max_k, st);
    else if (a.dim <= 64) f16 ? launch<F16, 64>(a, max_k, st) : launch<Bf16, 64>(a, max_k, st);
    else f16 ? launch<F16, 128>(a, max_k, st) : launch<Bf16, 128>(a, max_k, st);
}

}  // namespace f3m
