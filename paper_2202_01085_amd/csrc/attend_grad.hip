// Row-normalised products (attention): gradients.  With P_ij the weights, L_i the logarithms of their sums, delta_i = dO_i.O_i:
//   dV_j = sum_i P_ij dO_i    dS_ij = P_ij (dO_i.v_j - delta_i)    dQ_i = scale sum_j dS_ij k_j    dK_j = scale sum_i dS_ij q_i
// P is made again from q, k and L.  Two kernels, one that keeps rows and goes over keys (dQ) and one that keeps keys and goes over
// the rows of all heads that share them (dK, dV): seven products a pair where one kernel would need five, but each gradient is
// summed in one place and one order, without atomics, so that results repeat bit for bit.
//
// P and dS are rounded to the inputs' type for the matrix cores.  fp16: P is held times 2^12; dS, whose size follows the loss, times
// a power of two per kept row or key that goes down when a larger one comes, so both keep 11 bits.
//
// No unit is full: a SIMD has one to two waves, whose products, exponentials and LDS reads (one operand of each product, v too in grad_keys at
// head sizes above 64) wait for one another.  Shares of a launch's cycles, matrix cores / vector issue / LDS:
//   4 x 2048 tokens with causal order, 16 heads of 128, 4 key heads: rows 122 us 0.40 / 0.24 / 0.20, keys 173 us 0.36 / 0.21 / 0.28, sums of parts 9
//   8192 tokens in a window of 1024, heads of 64:                    rows 71 us 0.31 / 0.34 / 0.16, keys 118 us 0.24 / 0.23 / 0.18, sums of parts 13
// (three products a pair in the rows, four in the keys: 0.85 and 0.8 PFLOP/s in the first case).
#include "attend.h"

#include <algorithm>

namespace f3m {

namespace {

constexpr int NT = 256;

// log2 of the factor that grad_keys holds weights with
template <class T> constexpr float LIFT = T::narrow ? 12.f : 0.f;

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

// Parts of a tile of `count` steps: `chunk` each, the last one what is left
__device__ __forceinline__ int parts_of(int count, int chunk, int most) { return min(max(count - 1, 0) / chunk + 1, most); }

// Where the parts' sums lie: by a number of the tile (of 128 rows, `rows` to a token, or keys) among those of all sequences of a key head.  The
// tiles of sequence b, whose first token is `first`, are numbered from rows first / 128 + b on: the next sequence's start as many further as
// b has tiles, or more.  Where that makes more numbers than there are tiles of the longest sequence times sequences, those are counted instead.
__device__ __forceinline__ int64_t tile_slot(const AttendArgs &a, int b, int64_t first, int rows) {
    return a.packed ? first * rows / 128 + b : (int64_t)b * a.tiles;
}
// The sequence that a number belongs to, if to any: the last that starts at or before it
__device__ __forceinline__ int slot_sequence(const AttendArgs &a, int slot, const int *offsets, int64_t total, int rows) {
    if (!a.packed) return slot / a.tiles;
    int lo = 0, hi = a.batch - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) / 2;
        if (tile_slot(a, mid, min(max((int64_t)offsets[mid], (int64_t)0), total), rows) <= slot) lo = mid;
        else hi = mid - 1;
    }
    return lo;
}

// dQ: 128 rows of one group to a block, 32 to a wave, tiles of 64 keys through LDS, as the forward kernel.  Few row tiles are cut into parts
// along the keys (cut_rows), whose fp32 sums join_rows adds up.  It also leaves each row's
// stat for grad_keys: -log2 of its sum (+ LIFT), or -inf for an empty row, so that its weights are 0, and -dO.O.
template <class T, int DP> __global__ __launch_bounds__(NT, 2) void grad_rows(AttendArgs a) {
    constexpr int KS = DP / 16, DB = DP / 32, KT = 64;
    __shared__ __attribute__((aligned(1024))) short tile[2][2][KT * DP];
    const Item it = block_of(a, blockIdx.x);
    if (it.group >= a.groups) return;
    const int b = it.group / a.kv_heads, hk = it.group % a.kv_heads;
    const Sequence s = sequence_of(a, b);
    const int rows = min(s.nq, a.max_q) * a.group, r0 = it.tile * 128;
    if (r0 >= rows) return;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const Limits first = limits_of(a, s, r0 / a.group), last = limits_of(a, s, min(r0 + 127, rows - 1) / a.group);
    const Tiles tiles = tiles_of<KT>(first, last, a.sinks);
    const int parts = parts_of(tiles.count, a.chunk, a.parts);
    if (it.part >= parts) return;
    const int begin = it.part * a.chunk, end = it.part + 1 < parts ? begin + a.chunk : tiles.count;

    const int w0 = r0 + 32 * wave, row = min(w0 + (lane & 31), rows - 1), token = row / a.group, head = hk * a.group + row % a.group;
    const bool valid = w0 + (lane & 31) < rows, idle = w0 >= rows;
    const Limits mine = limits_of(a, s, token);
    const Limits wfirst = limits_of(a, s, min(w0, rows - 1) / a.group), wlast = limits_of(a, s, min(w0 + 31, rows - 1) / a.group);
    const float c = a.scale * LOG2E;
    s16x8 q[KS], g[KS];
    f32x16 acc[DB];
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
        q[ks] = __builtin_bit_cast(s16x8, load_piece<DP>(a.q.p, (int64_t)(s.q0 + token) * a.q.row + (int64_t)head * a.q.head, 2 * ks + (lane >> 5), a.dim));
        g[ks] = __builtin_bit_cast(s16x8, load_piece<DP>(a.dout.p, (int64_t)(s.q0 + token) * a.dout.row + (int64_t)head * a.dout.head, 2 * ks + (lane >> 5), a.dim));
    }
    float less, delta = 0.f;
    {
        s16x8 o[KS];
#pragma unroll
        for (int ks = 0; ks < KS; ++ks)
            o[ks] = __builtin_bit_cast(s16x8, load_piece<DP>(a.out.p, (int64_t)(s.q0 + token) * a.out.row + (int64_t)head * a.out.head, 2 * ks + (lane >> 5), a.dim));
        const float l = a.lse[(int64_t)(s.q0 + token) * a.heads + head];
#pragma unroll
        for (int ks = 0; ks < KS; ++ks)
#pragma unroll
            for (int j = 0; j < 8; ++j) delta -= T::up((uint16_t)g[ks][j]) * T::up((uint16_t)o[ks][j]);
        delta = both_halves_sum(delta);
        const bool empty = l == NO_KEY;
        // a row whose dO or O is not finite makes what it adds to its keys NaN (also where tiles are cleaned)
        less = empty ? NO_KEY : -l * LOG2E + (delta - delta);
        if (empty) delta = 0.f;
    }
    Unit unit{LEAST_UNIT};
    LaneReads<DP> at;
    at.start(lane);
    Tile2<T, DP, KT> src;
    src.start(a.k.p + 2 * ((int64_t)s.k0 * a.k.row + (int64_t)hk * a.k.head), a.k.row, a.v.p + 2 * ((int64_t)s.k0 * a.v.row + (int64_t)hk * a.v.head), a.v.row, a.dim, wave, lane);
    auto fetch = [&](int t, int buf) { src.issue(tiles[t] * KT, s.nk, a.dim, tile[buf][0], tile[buf][1], wave); };
    // p = scores, d = dP - `from` of 32 keys of a tile
    auto scores = [&](uint32_t kt, uint32_t vt, int kb, float from, f32x16 &p, f32x16 &d) {
        p = (f32x16)0.f;
        d = (f32x16)from;
        __builtin_amdgcn_s_setprio(1);      // the matrix cores to the wave that is at the scores, arithmetic to the other of the SIMD
        products<2 * KS, 4>([&](int i) { return at.row(i % 2 ? vt : kt, 32 * kb, i / 2); },
                            [&](int i, s16x8 x) {
                                if (i % 2) d = T::mma(x, g[i / 2], d);
                                else p = T::mma(x, q[i / 2], p);
                            });
        __builtin_amdgcn_s_setprio(0);
    };

    // Rows that see few keys have large results, whose rounding in dO.O would be as large an error as that of dS: where two tiles are all
    // there is, dO.O is summed from the weights instead, sum_j P_ij dP_ij.
    if (tiles.count > 0 && tiles.count <= 2) {
        for (int n = 0; n < tiles.count; ++n) fetch(n, n);
        registers_loaded();
        __syncthreads();
        float sum = 0.f;
        for (int x = 0; x < 2 * tiles.count; ++x) {
            f32x16 p, d;
            scores(lds_address(tile[x / 2][0]), lds_address(tile[x / 2][1]), x % 2, 0.f, p, d);
            const uint32_t bits = (uint32_t)seen_bits(mine, a.sinks, tiles[x / 2] * KT + 32 * (x % 2)) >> (4 * (lane >> 5));
#pragma unroll
            for (int i = 0; i < 16; ++i) sum += pick(bits, c_row(i, 0), __builtin_amdgcn_exp2f(__builtin_fmaf(p[i], c, less)) * d[i], 0.f);
        }
        delta = -both_halves_sum(sum);
        __syncthreads();
    }
    if (it.part == 0 && valid && lane < 32) {
        const int64_t x = (int64_t)head * a.total_q + s.q0 + token;
        a.stat[x] = less + LIFT<T>;
        a.stat[x + (int64_t)a.heads * a.total_q] = delta;
    }

    auto block = [&](uint32_t kt, uint32_t vt, int kb, int key0, bool edge) {
        f32x16 p, d;
        scores(kt, vt, kb, delta, p, d);     // dP starts from -dO.O
#pragma unroll
        for (int i = 0; i < 16; ++i) d[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(p[i], c, less)) * d[i];
        if (edge) {
            const uint32_t bits = (uint32_t)seen_bits(mine, a.sinks, key0 + 32 * kb) >> (4 * (lane >> 5));
#pragma unroll
            for (int i = 0; i < 16; ++i) d[i] = pick(bits, c_row(i, 0), d[i], 0.f);
        }
        unit.fit<T, DB>(d, acc);
        const s16x8 w[2] = {as_operand<T>(d, 0), as_operand<T>(d, 1)};
        products<2 * DB, 2>([&](int i) { return at.column(kt, 32 * kb + 16 * (i / DB), i % DB); }, [&](int i, s16x8 x) { acc[i % DB] = T::mma(x, w[i / DB], acc[i % DB]); });
    };

    // Tiles that the mask cuts are cleaned of infinities and NaN in k only when some shows in the results (rows that see one have such an
    // lse, and are NaN either way)
    auto pass = [&](bool careful) {
#pragma unroll
        for (int db = 0; db < DB; ++db) acc[db] = (f32x16)0.f;
        unit.u = LEAST_UNIT;
        if (begin >= end) return;
        // waits for the loads of tile t
        auto take = [&](int t, int buf) {
            arrived();
            __syncthreads();
            const int key0 = tiles[t] * KT;
            if (!careful || (key0 + KT <= first.hi && (key0 >= last.lo || key0 + KT <= a.sinks))) return;
            clean_tile<T, DP, KT>(tile[buf][0], tid);
            __syncthreads();
        };
        fetch(begin, begin & 1);
        registers_loaded();
        take(begin, begin & 1);
        for (int n = begin; n < end; ++n) {
            const int buf = n & 1, key0 = tiles[n] * KT;
            if (n + 1 < end) fetch(n + 1, buf ^ 1);
            const bool none = idle || key0 >= wlast.hi || (key0 + KT <= wfirst.lo && key0 >= a.sinks);
            const bool full = key0 + KT <= wfirst.hi && (key0 >= wlast.lo || key0 + KT <= a.sinks);
            if (!none) {
                block(lds_address(tile[buf][0]), lds_address(tile[buf][1]), 0, key0, !full);
                block(lds_address(tile[buf][0]), lds_address(tile[buf][1]), 1, key0, !full);
            }
            if (n + 1 < end) take(n + 1, buf ^ 1);
        }
    };
    pass(false);
    bool finite = true;
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int i = 0; i < 16; ++i) finite &= fabsf(acc[db][i]) < __builtin_inff();
    if (__syncthreads_or(!finite)) pass(true);
    const float by = T::narrow ? a.scale * unit.u : a.scale;
    if (parts > 1) {     // fp32 sums of this part, for join_rows
        if (!valid) return;
        const int64_t at_part = ((tile_slot(a, b, s.q0, a.group) + it.tile) * a.kv_heads + hk) * a.parts + it.part;
        float *to_part = a.part_out + (at_part * 128 + 32 * wave + (lane & 31)) * a.dim;
#pragma unroll
        for (int db = 0; db < DB; ++db)
#pragma unroll
            for (int i = 0; i < 16; i += 4) {
                const int x = 32 * db + c_row(i, lane);
                if (x < a.dim) *(float4 *)(to_part + x) = make_float4(acc[db][i] * by, acc[db][i + 1] * by, acc[db][i + 2] * by, acc[db][i + 3] * by);
            }
        return;
    }
    store_rows<T, DB>(acc, by, a.dq.p, (int64_t)(s.q0 + token) * a.dq.row + (int64_t)head * a.dq.head, a.dim, valid, lane);
}

// the parts of the row tiles that were cut, summed in their order: a block to 8 rows of a tile, 32 lanes to a row, 4 values each
template <class T> __global__ __launch_bounds__(NT) void join_rows(AttendArgs a) {
    const int in = blockIdx.x % 16 * 8 + threadIdx.x / 32, x = threadIdx.x % 32 * 4, hk = blockIdx.x / 16 % a.kv_heads, slot = blockIdx.x / (16 * a.kv_heads);
    const int b = slot_sequence(a, slot, a.q_offsets, a.total_q, a.group);
    const Sequence s = sequence_of(a, b);
    const int at_tile = (int)(slot - tile_slot(a, b, s.q0, a.group)), rows = min(s.nq, a.max_q) * a.group;
    if (at_tile < 0 || (int64_t)at_tile * 128 + in >= rows || x >= a.dim) return;
    const int r0 = at_tile * 128;
    const int parts = parts_of(tiles_of<64>(limits_of(a, s, r0 / a.group), limits_of(a, s, min(r0 + 127, rows - 1) / a.group), a.sinks).count, a.chunk, a.parts);
    if (parts == 1) return;
    const float *from = a.part_out + (((int64_t)slot * a.kv_heads + hk) * a.parts * 128 + in) * a.dim + x;
    float4 q = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int p = 0; p < parts; ++p, from += (int64_t)128 * a.dim) {
        const float4 y = *(const float4 *)from;
        q.x += y.x; q.y += y.y; q.z += y.z; q.w += y.w;
    }
    const int token = (r0 + in) / a.group, head = hk * a.group + (r0 + in) % a.group;
    *(u32x2 *)(a.dq.p + 2 * ((int64_t)(s.q0 + token) * a.dq.row + (int64_t)head * a.dq.head + x)) = (u32x2){T::pack(q.x, q.y), T::pack(q.z, q.w)};
}

// A block of grad_keys: 128 keys of a group and the row tiles that see them, RT tokens of one head each: the heads of the group for the
// last tokens, then for those before, so that the blocks of a group, which with causal order all see the last tokens, read the same rows
// at the same time.
constexpr int RT = 64;
struct KeyTile {
    int lo, hi, count;    // tokens [lo, hi), row tiles of all heads
};
// tokens that see keys of [from, to) are one interval: keys of the sinks stay visible to all later tokens
__device__ __forceinline__ KeyTile key_tile(const AttendArgs &a, const Sequence &s, int from, int to) {
    const int off = s.nk - s.nq, nq = min(s.nq, a.max_q);
    KeyTile t;
    t.lo = 0;
    t.hi = nq;
    if (a.causal) {
        t.lo = min(max(from - off, 0), nq);
        if (a.window && from >= a.sinks) t.hi = max(t.lo, (int)min((int64_t)nq, (int64_t)to - 1 + a.window - off));
    }
    t.count = (t.hi - t.lo + RT - 1) / RT * a.group;
    return t;
}

// row tiles of a part of a key tile, and how many parts it has
__device__ __forceinline__ int key_chunk(const AttendArgs &a, int at_tile) { return at_tile < a.sink_tiles ? a.sink_chunk : a.chunk; }
__device__ __forceinline__ int key_parts(const AttendArgs &a, int at_tile, int count) {
    return parts_of(count, key_chunk(a, at_tile), at_tile < a.sink_tiles ? a.sink_parts : a.usual);
}
// Where the sums of part 0 of a key tile lie (dk of its 128 keys, dv of them behind those), and how much further those of the
// next part.  Tiles of sinks, which have parts by the length of their sequence, lie apart.  Sequence b has at most ceil(T group / chunk) of them,
// T the row tiles of a head, which do not reach past the next sequence's start: T <= end / RT - first / RT + 1.
struct KeySums {
    float *at;
    int64_t next;
};
__device__ __forceinline__ KeySums key_sums(const AttendArgs &a, const Sequence &s, int b, int hk, int at_tile) {
    const int64_t tile = (int64_t)256 * a.dim;
    if (at_tile < a.sink_tiles) {
        const int64_t slot = a.sink_packed ? ((int64_t)(s.q0 / RT) + b) * a.group / a.sink_chunk + b : (int64_t)b * a.sink_parts;
        return {a.sink_out + ((slot * a.sink_tiles + at_tile) * a.kv_heads + hk) * tile, (int64_t)a.sink_tiles * a.kv_heads * tile};
    }
    return {a.part_out + ((tile_slot(a, b, s.k0, 1) + at_tile) * a.kv_heads + hk) * a.usual * tile, tile};
}

// dK, dV: 32 keys to a wave, whose sums stay in registers; tiles of q and dO come through a ring in LDS, two or more under way while one
// is worked on.  Head sizes above 64: the sums alone are 128 registers, so that two waves to a SIMD, which the exponentials of one
// need to run under the products of the other, leave room for k only and v stays in LDS.  There a block has eight waves, two to the same
// keys, each with half of a tile's rows; their sums are added at the end.  Below, a wave takes all 64 rows of a tile.
template <class T, int DP> __global__ __launch_bounds__(DP == 128 ? 512 : 256, 2) void grad_keys(AttendArgs a) {
    constexpr int KS = DP / 16, DB = DP / 32, HALVES = DP == 128 ? 2 : 1, SUB = 2 / HALVES, WAVES = 4 * HALVES, THREADS = 64 * WAVES;
    constexpr bool V_LDS = DP == 128;
    constexpr int AHEAD = 2, RING = AHEAD + 1, SLOT = 2 * RT * DP;
    using Src = Tile2<T, DP, RT, WAVES>;
    __shared__ __attribute__((aligned(1024))) short lds[RING * SLOT + (V_LDS ? 128 * DP : 0)];
    __shared__ __attribute__((aligned(256))) float stat[RING][2][WAVES][2][32];   // a copy to a wave, so that all waves have the same loads under way
    short *const vt = lds + RING * SLOT;
    Item it = block_of(a, blockIdx.x);
    if (it.group >= a.groups) return;
    const int b = it.group / a.kv_heads, hk = it.group % a.kv_heads;
    const Sequence s = sequence_of(a, b);
    // the first keys have most rows: their tiles come first.  Items past the usual parts of all tiles are the sinks' other parts
    int at_tile = a.tiles - 1 - it.tile;
    if (it.part >= a.usual) {
        const int x = (it.part - a.usual) * a.tiles + at_tile, more = a.parts - a.usual;
        at_tile = x / more;
        it.part = a.usual + x % more;
        if (at_tile >= a.sink_tiles) return;
    }
    const int k0 = at_tile * 128;
    const int nk = min(s.nk, a.max_k);                               // keys whose gradients are asked for
    if (k0 >= nk) return;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), kw = wave & 3, half = wave >> 2;
    const int off = s.nk - s.nq;                                     // position of token 0
    const KeyTile t = key_tile(a, s, k0, min(k0 + 128, nk));
    const int parts = key_parts(a, at_tile, t.count);
    if (it.part >= parts) return;
    const int chunk = key_chunk(a, at_tile), begin = it.part * chunk, end = it.part + 1 < parts ? begin + chunk : t.count;

    const int w0 = k0 + 32 * kw, key = w0 + (lane & 31), kept = min(key, nk - 1);
    const bool valid = key < nk, idle = w0 >= nk;
    // tokens [from, to) see this lane's key
    const int from = !valid ? t.hi : a.causal ? max(key - off, 0) : 0;
    const int to = a.causal && a.window && key >= a.sinks ? (int)min((int64_t)t.hi, (int64_t)key + a.window - off) : t.hi;
    const KeyTile mine = key_tile(a, s, w0, min(w0 + 32, nk));     // of the wave: it has nothing to do elsewhere
    // tokens [all.x, all.y) see all keys x .. y - 1
    auto seen_by_all = [&](int x, int y) {
        if (y > nk) return make_int2(0, 0);
        if (!a.causal) return make_int2(0, t.hi);
        return make_int2(y - 1 - off, a.window && y > a.sinks ? (int)min((int64_t)t.hi, (int64_t)x + a.window - off) : t.hi);
    };
    const int2 all_block = seen_by_all(k0, k0 + 128), all_wave = seen_by_all(w0, w0 + 32);
    const float c = a.scale * LOG2E;

    s16x8 k[KS], v[V_LDS ? 1 : KS];
    f32x16 dk[DB], dv[DB];
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
        k[ks] = __builtin_bit_cast(s16x8, load_piece<DP>(a.k.p, (int64_t)(s.k0 + kept) * a.k.row + (int64_t)hk * a.k.head, 2 * ks + (lane >> 5), a.dim));
        if (!V_LDS) v[V_LDS ? 0 : ks] = __builtin_bit_cast(s16x8, load_piece<DP>(a.v.p, (int64_t)(s.k0 + kept) * a.v.row + (int64_t)hk * a.v.head, 2 * ks + (lane >> 5), a.dim));
    }
    if (V_LDS)
        for (int at = tid; at < 128 * (DP / 8); at += THREADS) {
            const int r = at / (DP / 8), piece = at % (DP / 8);
            *(u32x4 *)(vt + tile_at<DP>(r, piece)) = load_piece<DP>(a.v.p, (int64_t)(s.k0 + min(k0 + r, nk - 1)) * a.v.row + (int64_t)hk * a.v.head, piece, a.dim);
        }
#pragma unroll
    for (int db = 0; db < DB; ++db) { dk[db] = (f32x16)0.f; dv[db] = (f32x16)0.f; }
    Unit unit{LEAST_UNIT};
    LaneReads<DP> at;
    at.start(lane);

    // the next tile to load: tokens ft .. of head fh; the last tiles of tokens end at t.hi, the first may begin before t.lo
    Src src;
    src.start(nullptr, a.q.row, nullptr, a.dout.row, a.dim, wave, lane);
    int fh = begin % a.group, ft = t.hi - (begin / a.group + 1) * RT, fetched = begin;
    const char *const q_base = a.q.p + 2 * ((int64_t)s.q0 * a.q.row + (int64_t)hk * a.group * a.q.head);
    const char *const g_base = a.dout.p + 2 * ((int64_t)s.q0 * a.dout.row + (int64_t)hk * a.group * a.dout.head);
    const float *const stats = a.stat + ((int64_t)(lane < 32 ? 0 : a.heads) + hk * a.group) * a.total_q + s.q0;
    // past the end the last tile is loaded again, which keeps the count of loads under way
    auto fetch = [&](int slot) {
        src.base[0] = q_base + 2 * fh * a.q.head;
        src.base[1] = g_base + 2 * fh * a.dout.head;
        const int from = max(ft, 0);                   // a tile that would begin before the sequence begins with it
        src.issue(from, t.hi, a.dim, lds + slot * SLOT, lds + slot * SLOT + RT * DP, wave);
#pragma unroll
        for (int h = 0; h < 2; ++h)
            word_to_lds(stats + (int64_t)fh * a.total_q + min(from + 32 * h + (lane & 31), t.hi - 1), lds_address((const short *)stat[slot][h][wave]));
        if (++fetched < end && ++fh == a.group) {
            fh = 0;
            ft -= RT;
        }
    };
    constexpr int LOADS = 2 * Src::COUNT + 2;    // of a wave to a tile
    static_assert(Src::STEP <= RT, "every wave has rows of a tile to load");
    // waits for the loads of a tile, the AHEAD - 1 tiles after it stay under way; where the mask cuts it for the block, q and dO are cleaned
    // if some row has an odd value: such rows have an odd stat, but for rows that see nothing (-inf)
    auto take = [&](int t0, int slot) {
        arrived<(AHEAD - 1) * LOADS>();
        __syncthreads();
        if (t0 >= all_block.x && t0 + RT <= all_block.y) return;
        const float x = stat[slot][0][wave][lane >> 5][lane & 31], y = stat[slot][1][wave][lane >> 5][lane & 31];
        if (!__any(!(fabsf(x) < __builtin_inff() && fabsf(y) < __builtin_inff()))) return;
        clean_tile<T, DP, RT, THREADS>(lds + slot * SLOT, tid);
        clean_tile<T, DP, RT, THREADS>(lds + slot * SLOT + RT * DP, tid);
        __syncthreads();
    };

    if (begin < end) {
        int t0 = max(ft, 0), tt = ft, th = fh, slot = 0;
        for (int x = 0; x < AHEAD; ++x) fetch(x);
        registers_loaded();
        take(t0, 0);
        for (int n = begin; n < end; ++n) {
            fetch(slot == 0 ? RING - 1 : slot - 1);       // the slot of the tile before
            const int x0 = t0 + 32 * half;
            if (!idle && x0 < mine.hi && x0 + 32 * SUB > mine.lo) {
                f32x16 p[SUB], d[SUB];
#pragma unroll
                for (int y = 0; y < SUB; ++y) {
                    p[y] = (f32x16)0.f;
#pragma unroll
                    for (int i4 = 0; i4 < 4; ++i4) {      // dP starts from -dO.O
                        const float4 e = *(const float4 *)&stat[slot][half + y][wave][1][c_row(4 * i4, lane)];
                        d[y][4 * i4] = e.x; d[y][4 * i4 + 1] = e.y; d[y][4 * i4 + 2] = e.z; d[y][4 * i4 + 3] = e.w;
                    }
                }
                const uint32_t qt = lds_address(lds) + 2 * (slot * SLOT + half * 32 * DP), gt = qt + 2 * RT * DP;
                __builtin_amdgcn_s_setprio(1);
                s16x8 vk[KS];
                if (V_LDS) {      // dP first, with v read ahead too, then S
                    products<2 * KS, 4>([&](int i) { return i % 2 ? at.row(gt, 0, i / 2) : at.row(lds_address(vt), 32 * kw, i / 2); },
                                        [&](int i, s16x8 x) {
                                            if (i % 2) d[0] = T::mma(x, vk[i / 2], d[0]);
                                            else vk[i / 2] = x;
                                        });
                    products<KS, 4>([&](int i) { return at.row(qt, 0, i); }, [&](int i, s16x8 x) { p[0] = T::mma(x, k[i], p[0]); });
                } else {
                    products<2 * SUB * KS, 4>([&](int i) { return at.row(i % 2 ? gt : qt, 32 * (i / 2 % SUB), i / 2 / SUB); },
                                              [&](int i, s16x8 x) {
                                                  const int y = i / 2 % SUB, ks = i / 2 / SUB;
                                                  if (i % 2) d[y] = T::mma(x, v[V_LDS ? 0 : ks], d[y]);
                                                  else p[y] = T::mma(x, k[ks], p[y]);
                                              });
                }
                __builtin_amdgcn_s_setprio(0);
#pragma unroll
                for (int y = 0; y < SUB; ++y)
#pragma unroll
                    for (int i4 = 0; i4 < 4; ++i4) {
                        const float4 l = *(const float4 *)&stat[slot][half + y][wave][0][c_row(4 * i4, lane)];
                        const float ls[4] = {l.x, l.y, l.z, l.w};
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            const int i = 4 * i4 + j;
                            p[y][i] = __builtin_amdgcn_exp2f(__builtin_fmaf(p[y][i], c, ls[j]));
                            d[y][i] *= p[y][i];
                        }
                    }
                // tokens of this tile that count: a tile cut short at the front repeats tokens of the one after it
                const int last = min(to, tt + RT), least = max(from, t0);
                if (x0 < all_wave.x || x0 + 32 * SUB > all_wave.y || t0 != tt) {
#pragma unroll
                    for (int y = 0; y < SUB; ++y) {
                        const uint32_t bits = (uint32_t)(below(last - x0 - 32 * y) & ~below(least - x0 - 32 * y)) >> (4 * (lane >> 5));
#pragma unroll
                        for (int i = 0; i < 16; ++i) {
                            p[y][i] = pick(bits, c_row(i, 0), p[y][i], 0.f);
                            d[y][i] = pick(bits, c_row(i, 0), d[y][i], 0.f);
                        }
                    }
                }
#pragma unroll
                for (int y = 0; y < SUB; ++y) {
                    unit.fit<T, DB>(d[y], dk);
                    const s16x8 pw[2] = {as_operand<T>(p[y], 0), as_operand<T>(p[y], 1)}, dw[2] = {as_operand<T>(d[y], 0), as_operand<T>(d[y], 1)};
                    products<4 * DB, 2>([&](int i) { return at.column(i % 2 ? qt : gt, 32 * y + 16 * (i / 2 / DB), i / 2 % DB); },
                                        [&](int i, s16x8 x) {
                                            const int h = i / 2 / DB, db = i / 2 % DB;
                                            if (i % 2) dk[db] = T::mma(x, dw[h], dk[db]);
                                            else dv[db] = T::mma(x, pw[h], dv[db]);
                                        });
                }
            }
            if (++th == a.group) {
                th = 0;
                tt -= RT;
                t0 = max(tt, 0);
            }
            slot = slot + 1 < RING ? slot + 1 : 0;
            if (n + 1 < end) take(t0, slot);
        }
        arrived();      // nothing may come into LDS later: it is used otherwise
    }
    const float v_by = T::narrow ? 0x1p-12f : 1.f, k_by = T::narrow ? a.scale * 0x1p-12f * unit.u : a.scale;
#pragma unroll
    for (int db = 0; db < DB; ++db) {
        dk[db] *= k_by;
        dv[db] *= v_by;
    }
    if (HALVES == 2) {
        float *const sums = (float *)lds + kw * 64 * DB * 16 + lane;
#pragma unroll
        for (int w = 0; w < 2; ++w) {
            __syncthreads();
            f32x16 (&x)[DB] = w ? dv : dk;
            if (half == 1) {
#pragma unroll
                for (int db = 0; db < DB; ++db)
#pragma unroll
                    for (int i = 0; i < 16; ++i) sums[64 * (16 * db + i)] = x[db][i];
            }
            __syncthreads();
            if (half == 0) {
#pragma unroll
                for (int db = 0; db < DB; ++db)
#pragma unroll
                    for (int i = 0; i < 16; ++i) x[db][i] += sums[64 * (16 * db + i)];
            }
        }
        if (half == 1) return;
    }
    const int64_t row = s.k0 + kept;
    if (parts > 1) {     // fp32 sums of this part, for join_keys
        const KeySums sums = key_sums(a, s, b, hk, at_tile);
        float *to_part = sums.at + it.part * sums.next + (32 * kw + (lane & 31)) * a.dim;
#pragma unroll
        for (int db = 0; db < DB; ++db)
#pragma unroll
            for (int i = 0; i < 16; i += 4) {
                const int x = 32 * db + c_row(i, lane);
                if (x >= a.dim) continue;
                *(float4 *)(to_part + x) = make_float4(dk[db][i], dk[db][i + 1], dk[db][i + 2], dk[db][i + 3]);
                *(float4 *)(to_part + 128 * a.dim + x) = make_float4(dv[db][i], dv[db][i + 1], dv[db][i + 2], dv[db][i + 3]);
            }
        return;
    }
    store_rows<T, DB>(dv, 1.f, a.dv.p, row * a.dv.row + (int64_t)hk * a.dv.head, a.dim, valid, lane);
    store_rows<T, DB>(dk, 1.f, a.dk.p, row * a.dk.row + (int64_t)hk * a.dk.head, a.dim, valid, lane);
}

// the parts of the key tiles that were cut, summed in their order: a block to 8 keys of a tile, 32 lanes to a key, 4 values each
template <class T> __global__ __launch_bounds__(NT) void join_keys(AttendArgs a) {
    const int in = blockIdx.x % 16 * 8 + threadIdx.x / 32, x = threadIdx.x % 32 * 4, hk = blockIdx.x / 16 % a.kv_heads, slot = blockIdx.x / (16 * a.kv_heads);
    const bool all = a.usual > 1;      // else only tiles of sinks are cut, and the grid has no others
    const int b = all ? slot_sequence(a, slot, a.k_offsets, a.total_k, 1) : slot / a.sink_tiles;
    const Sequence s = sequence_of(a, b);
    const int at_tile = all ? (int)(slot - tile_slot(a, b, s.k0, 1)) : slot % a.sink_tiles;
    const int nk = min(s.nk, a.max_k);
    if (at_tile < 0 || (int64_t)at_tile * 128 + in >= nk || x >= a.dim) return;
    const int k0 = at_tile * 128;
    const KeyTile t = key_tile(a, s, k0, min(k0 + 128, nk));
    const int parts = key_parts(a, at_tile, t.count);
    if (parts == 1) return;
    const KeySums sums = key_sums(a, s, b, hk, at_tile);
    const float *from = sums.at + in * a.dim + x;
    float4 k = make_float4(0.f, 0.f, 0.f, 0.f), v = k;
    for (int p = 0; p < parts; ++p, from += sums.next) {
        const float4 y = *(const float4 *)from, z = *(const float4 *)(from + 128 * a.dim);
        k.x += y.x; k.y += y.y; k.z += y.z; k.w += y.w;
        v.x += z.x; v.y += z.y; v.z += z.z; v.w += z.w;
    }
    const int64_t row = s.k0 + k0 + in;
    *(u32x2 *)(a.dk.p + 2 * (row * a.dk.row + (int64_t)hk * a.dk.head + x)) = (u32x2){T::pack(k.x, k.y), T::pack(k.z, k.w)};
    *(u32x2 *)(a.dv.p + 2 * (row * a.dv.row + (int64_t)hk * a.dv.head + x)) = (u32x2){T::pack(v.x, v.y), T::pack(v.z, v.w)};
}

// tiles of 128 `rows`, `tiles` in the longest sequence, and their numbers (tile_slot)
void number(AttendArgs &a, int64_t tiles, int64_t rows) {
    const int64_t close = rows / 128 + a.batch, wide = tiles * a.batch;
    a.tiles = (int)tiles;
    a.packed = close < wide;
    a.slots = std::min(close, wide);
}

// floats of the sums of parts of row tiles, and of key tiles without sinks and with
int64_t row_sums(const AttendArgs &a) { return a.parts > 1 ? a.slots * a.kv_heads * a.parts * 128 * a.dim : 0; }
int64_t usual_sums(const AttendArgs &a) { return a.usual > 1 ? a.slots * a.kv_heads * a.usual * 256 * a.dim : 0; }
int64_t sink_sums(const AttendArgs &a) { return a.sink_slots * a.sink_tiles * a.kv_heads * 256 * a.dim; }

// How grad_keys is cut.  A block has a CU to itself at head sizes above 64, half of one below: 256 or 512 places.  Blocks go to the XCDs in
// turn, whatever their length, so that a little more than one round of them takes as long as two.
// With a window, without order or with few tokens after many keys, tiles are about equally long (`usual`) but those of the sinks, which
// all later tokens see and which are always cut to the others' size.  There the parts are those of the shortest time, counted in steps (a row tile
// with a key tile; 2 us, 1 us up to a head size of 64): rounds of parts, each of them `ends` steps longer for its beginning and end, and the
// join, (512 + n) / 128 us for n parts, up to 64 (512 + n) / 100 (512 parts at 128: 8.6 us).  All gradients, in us, by parts:
//   8192 tokens, 16 heads, 4 key heads, window 1024      64: 167 whole, 157 in 2, 171 in 3, 165 in 4;  128: 263, 278, 295, 316
//   the same at 64 with four sinks                       236, 216, 194, 197, in 6 206
//   2000 tokens over 4000 keys, 4 heads, no order        64: 79, 70, 70, 68, in 6 75;  128: 107, 100, 117, 117
//   512 new tokens after 7488, 8 heads, 2 key heads      64: 81, 71, 69, 68, in 6 78;  128: 106, 99, 118, 117
// The rule takes 2, 1, 3, 4, 2, 4, 2.  It counts all of a batch as long as the longest: four of up to 4099, window 1024, four sinks 518, 494 in 2.
// Else lengths fall to nothing along the keys, and p parts of the longest tile make (p + 1) / 2 to a tile: as many as fill 88 % of one
// round or, if that is fewer than three, two, whose second ones are what others lack.  All gradients of 6709 tokens, 4 heads, one key
// head: 692 us whole, 397 in 2 parts, 249 in 4, 202 in 6, 232 in 8; of 4 x 2048, 16 heads, 4 key heads: 322, 286 in 2, 296 in 3, 326 in 4.
// The sums of parts without sinks are those of at most four rounds of blocks, 134 MB.  Tiles of sinks have parts by the rows that see them: where
// these would be more than eight rounds (268 MB), which takes hundreds of sinks or sequences, their parts get longer.
void cut_keys(AttendArgs &a, int64_t max_k) {
    const int64_t tiles = cdiv(max_k, 128), all = all_tiles(a, tiles, a.total_k), places = a.dim > 64 ? 256 : 512, ends = a.dim > 64 ? 12 : 4;
    const int64_t longest = std::max<int64_t>(1, cdiv(a.max_q, RT) * a.group);
    const int64_t usual = a.window ? std::min(longest, (cdiv((int64_t)a.window + 128, RT) + 1) * a.group) : longest;
    const int64_t sinks = usual < longest ? std::min(tiles, cdiv(a.sinks, 128)) : 0;
    int64_t parts = 1;
    if (usual < longest || !a.causal || 2 * (int64_t)a.max_q < max_k) {
        double least = 1e30;
        for (int64_t p = 1; p <= 64 && (p == 1 || all * p <= 4 * places); ++p) {
            const int64_t chunk = cdiv(usual, p), more = sinks * a.groups * std::max<int64_t>(0, cdiv(longest, chunk) - p);
            const double joined = p > 1 && !sinks ? (512.0 + (double)(all * p)) / (a.dim > 64 ? 256.0 : 100.0) : 0.0;
            const double time = (double)(cdiv(all * p + more, places) * (chunk + ends)) + joined;
            if (time < least) {
                least = time;
                parts = p;
            }
        }
    } else {
        parts = std::min<int64_t>((44 * places / 25 - all) / all, 64);
        if (parts < 3) parts = all <= places && usual >= 32 ? 2 : 1;
        parts = std::max<int64_t>(1, std::min(parts, usual / 2));
    }
    const int64_t chunk = cdiv(usual, parts);
    number(a, tiles, a.total_k);
    a.chunk = (int)chunk;
    a.usual = (int)cdiv(usual, chunk);
    a.sink_tiles = (int)sinks;
    a.sink_chunk = (int)longest;
    a.sink_slots = 0;
    const int64_t room = 8 * places / std::max<int64_t>(1, sinks * a.kv_heads), rows = (a.total_q / RT + a.batch) * a.group;
    for (const bool packed : {false, true}) {        // the least chunk with no more numbers than there is room for, and of two the fewer numbers
        const int64_t each = packed ? room - a.batch : room / a.batch;
        if (sinks == 0 || each < 1) continue;
        const int64_t least = std::max(chunk, packed ? rows / (each + 1) + 1 : cdiv(longest, each));
        const int64_t slots = packed ? rows / least + a.batch : a.batch * cdiv(longest, least);
        if (least >= longest || least > a.sink_chunk || (least == a.sink_chunk && slots >= a.sink_slots)) continue;
        a.sink_chunk = (int)least;
        a.sink_packed = packed;
        a.sink_slots = slots;
    }
    a.sink_parts = (int)cdiv(longest, a.sink_chunk);
    a.parts = std::max(a.usual, a.sink_parts);
}

// How grad_rows is cut, at two blocks to a CU: parts of 10 key tiles or more fill the 512 places, where the row tiles do not; of tiles whose
// lengths rise along the rows it takes twice as many.  One head over 6709 tokens, 53 row tiles: 150 us whole, 36 + 8 for the sums in
// 14 parts; four heads, 210: 158 whole, 90 + 9 in 3.  Shorter parts cost as much as they save (4 x 1024 tokens, 16 key tiles, 256 row
// tiles: all gradients 49 us whole, 61 in two parts).
void cut_rows(AttendArgs &a, int64_t max_k) {
    number(a, cdiv((int64_t)a.max_q * a.group, 128), a.total_q * a.group);
    const int64_t longest = std::max<int64_t>(1, cdiv(max_k, 64)), items = all_tiles(a, a.tiles, a.total_q * a.group);
    const int64_t most = a.window ? std::min(longest, cdiv((int64_t)a.window + cdiv(128, a.group), 64) + 1 + cdiv(a.sinks, 64)) : longest;
    const bool even = most < longest || !a.causal || 2 * (int64_t)a.max_q < max_k;
    const int64_t parts = std::min({(even ? 511 : 1023) / items, most / 10, (int64_t)64});
    a.chunk = (int)cdiv(most, std::max<int64_t>(1, parts));
    a.parts = (int)cdiv(most, a.chunk);
}

// items of a group: the usual parts of all tiles, the other parts of the sinks' tiles (in rows of `tiles`, as block_of counts)
int64_t key_items(const AttendArgs &a) {
    return (int64_t)a.tiles * (a.usual + cdiv((int64_t)a.sink_tiles * (a.parts - a.usual), a.tiles));
}

int64_t stat_floats(const AttendArgs &a) { return cdiv(2 * a.total_q * a.heads, 64) * 64; }

template <class T, int DP> void launch(AttendArgs a, int64_t max_k, hipStream_t st) {
    AttendArgs keys = a;                       // what cannot be launched is refused before anything is
    int64_t key_blocks = 0, row_joins = 0, key_joins = 0;
    cut_rows(a, max_k);
    const int64_t row_blocks = attend_blocks(a, (int64_t)a.tiles * a.parts);
    if (a.parts > 1) row_joins = a.slots * a.kv_heads * 16;
    if (max_k && a.total_k) {
        cut_keys(keys, max_k);
        key_blocks = attend_blocks(keys, key_items(keys));
        keys.sink_out = keys.part_out + usual_sums(keys);
        // tiles of sinks are no more than a grid has room for, cut or not
        const int64_t sink_joins = (int64_t)keys.groups * keys.sink_tiles * 16;
        key_joins = keys.usual > 1 ? keys.slots * a.kv_heads * 16 : keys.sink_parts > 1 ? sink_joins : 0;
        if (sink_joins >= 1 << 24) fail(F3M_ERR_UNSUPPORTED, "attention: too many sequences for one call's gradients");
    }
    if (a.max_q && a.total_q) {
        grad_rows<T, DP><<<dim3((uint32_t)row_blocks), NT, 0, st>>>(a);
        F3M_HIP(hipGetLastError());
        if (row_joins) {
            join_rows<T><<<dim3((uint32_t)row_joins), NT, 0, st>>>(a);
            F3M_HIP(hipGetLastError());
        }
    }
    if (key_blocks) {
        grad_keys<T, DP><<<dim3((uint32_t)key_blocks), DP == 128 ? 512 : 256, 0, st>>>(keys);
        F3M_HIP(hipGetLastError());
        if (key_joins) {
            join_keys<T><<<dim3((uint32_t)key_joins), NT, 0, st>>>(keys);
            F3M_HIP(hipGetLastError());
        }
    }
}

}  // namespace

int64_t attend_grad_workspace(AttendArgs a, int64_t max_k) {
    int64_t floats = 0;                    // of the parts of either kernel, one after the other
    if (a.groups && a.max_q && a.total_q) {
        cut_rows(a, max_k);
        floats = row_sums(a);
    }
    if (a.groups && max_k && a.total_k) {
        cut_keys(a, max_k);
        floats = std::max(floats, usual_sums(a) + sink_sums(a));
    }
    return (stat_floats(a) + floats) * (int64_t)sizeof(float);
}

void run_attend_grad(AttendArgs a, int64_t max_k, bool f16, void *workspace, hipStream_t st) {
    if (!a.groups) return;
    a.stat = (float *)workspace;
    a.part_out = a.stat + stat_floats(a);
    if (a.dim <= 32) f16 ? launch<F16, 32>(a, max_k, st) : launch<Bf16, 32>(a, max_k, st);
    else if (a.dim <= 64) f16 ? launch<F16, 64>(a, max_k, st) : launch<Bf16, 64>(a, max_k, st);
    else f16 ? launch<F16, 128>(a, max_k, st) : launch<Bf16, 128>(a, max_k, st);
}

}  // namespace f3m
