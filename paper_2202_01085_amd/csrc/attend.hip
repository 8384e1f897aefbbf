// Row-normalised products (attention), forward: o_i = sum_j w_ij v_j, w_ij = exp(scale q_i.k_j) / (its sum over the visible j).
//
// Rows of a work item are (token, query head) pairs that share a key head, 32 to a wave.  A wave keeps its rows' q and o in
// registers and goes over the keys once, with the running maximum m and sum l of each row (one row to a lane pair): a block of
// scores S^T = K Q^T, weights exp2(c s - c m), o^T = o^T exp2(c m_old - c m) + V^T w^T.  m moves only when a score is above it by
// 2^8 or more, so o is rarely rescaled; weights stay below 2^8 and their sums in fp32 (fp16 weights are held times 2^7, so that
// they keep 11 bits down to 2^-21 of the largest).  The weights are rounded to the inputs' type for the matrix cores.
#include "attend.h"

#include <algorithm>

namespace f3m {

namespace {

constexpr int NT = 256;       // four waves
constexpr int KT = 64;        // keys of a tile
constexpr float GROW = 8.f;   // log2 of how far a score may lie above m

// A tile of K and V from an 8-bit cache on its way from memory to LDS, where it lies as 16-bit values: 16 codes to a thread's piece.  Page
// numbers are looked up a tile before.
template <class T, int DP> struct Codes {
    static constexpr int PIECES = DP / 16, COUNT = (KT * PIECES + NT - 1) / NT;
    static constexpr bool ALL = KT * PIECES % NT == 0;
    u32x4 k[COUNT], v[COUNT];
    uint8_t ke[COUNT], ve[COUNT];
    int pages[COUNT], all;         // of the thread's rows; of row `lane` of the tile

    __device__ void look(const AttendArgs &a, const Sequence &s, int b, int key0, int tid) {
        const int *const table = a.table + (int64_t)b * a.table_row;
#pragma unroll
        for (int c = 0; c < COUNT; ++c) pages[c] = table[min(key0 + (tid + NT * c) / PIECES % KT, s.nk - 1) >> a.page_shift];
        all = table[min(key0 + (tid & 63), s.nk - 1) >> a.page_shift];
    }
    // bits of the rows that lie in pages of the cache
    __device__ uint64_t good(const AttendArgs &a) const { return __ballot(all >= 0 && all < a.pages); }
    __device__ void load(const AttendArgs &a, const Sequence &s, int hk, int key0, int tid) {
#pragma unroll
        for (int c = 0; c < COUNT; ++c) {
            const int at = tid + NT * c, row = at / PIECES, piece = at % PIECES;
            if (!ALL && row >= KT) break;
            const int j = min(key0 + row, s.nk - 1), page = pages[c] >= 0 && pages[c] < a.pages ? pages[c] : 0;
            const uint64_t x = (uint64_t)(uint32_t)page * (uint32_t)(a.kv_heads << a.page_shift) + (uint32_t)((hk << a.page_shift) + (j & ((1 << a.page_shift) - 1)));
            const uint64_t y = x * (uint32_t)a.dim + (piece * 16 < a.dim ? piece * 16 : 0);   // past the head: q is 0 there, and o is not kept
            k[c] = *(const u32x4 *)(a.k.p + y);
            v[c] = *(const u32x4 *)(a.v.p + y);
            ke[c] = a.k_exp[x];
            ve[c] = a.v_exp[x];
        }
    }
    static __device__ bool put(short *tile, int row, int piece, u32x4 x, uint8_t e, bool clean) {
        const float scale = __builtin_bit_cast(float, (uint32_t)e << 23);
        bool odd = false;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            u32x4 w = {T::template codes<false>(x[2 * h], scale), T::template codes<true>(x[2 * h], scale),
                       T::template codes<false>(x[2 * h + 1], scale), T::template codes<true>(x[2 * h + 1], scale)};
            if (clean && any_odd<T>(w)) {
                w = cleaned<T>(w);
                odd = true;
            }
            *(u32x4 *)(tile + tile_at<DP>(row, 2 * piece + h)) = w;
        }
        return odd;
    }
    // to LDS; with `clean`, infinities and NaN of v become 0 and the rows that had one come back as bits (a wave's)
    __device__ uint64_t store(short *kt, short *vt, int tid, bool clean) const {
        uint64_t odd = 0;
#pragma unroll
        for (int c = 0; c < COUNT; ++c) {
            const int at = tid + NT * c, row = at / PIECES, piece = at % PIECES;
            if (!ALL && row >= KT) break;
            put(kt, row, piece, k[c], ke[c], false);
            if (put(vt, row, piece, v[c], ve[c], clean)) odd |= 1ull << row;
        }
        if (!clean || !__any(odd != 0)) return 0;
#pragma unroll 1
        for (int by = 32; by > 0; by >>= 1) odd |= __shfl_xor((unsigned long long)odd, by);
        return odd;
    }
};

// which rows of a tile lie in pages of the cache (bit r: row key0 + r), for lanes r of one wave
__device__ __forceinline__ uint64_t good_pages(const AttendArgs &a, const Sequence &s, int b, int key0, int lane) {
    if (!a.table) return ~0ull;
    const int j = min(key0 + lane, s.nk - 1);
    const int page = a.table[(int64_t)b * a.table_row + (j >> a.page_shift)];
    return __ballot(page >= 0 && page < a.pages);
}

// What a wave carries from tile to tile, for its 32 rows
template <class T, int DP> struct Rows32 {
    static constexpr int KS = DP / 16, DB = DP / 32;
    static constexpr float LIFT = T::narrow ? 7.f : 0.f;   // log2 of the factor that weights are held with
    s16x8 q[KS];
    f32x16 o[DB];
    float m, l;     // largest score so far as used, sum of the weights (of this lane's half of the keys) times 2^LIFT
    float spoil;    // 0, or NaN once the row (in this lane's half) has seen an odd v

    __device__ void start(const AttendArgs &a, const char *base, int64_t at, int lane) {
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) q[ks] = __builtin_bit_cast(s16x8, load_piece<DP>(base, at, 2 * ks + (lane >> 5), a.dim));
#pragma unroll
        for (int db = 0; db < DB; ++db) o[db] = (f32x16)0.f;
        m = NO_KEY;
        l = 0.f;
        spoil = 0.f;
    }

    // NB blocks of 32 keys from key0 on: read_k(base, ks) is the A operand of k from row `base` on, v lies in LDS at vt, all of it or (half
    // given) 16 rows at a time, which half(h) puts there.  edge: the mask cuts the tile for some row, or `good` (rows in pages of the cache) says
    // something.  Returns the bits of the keys that the row sees.
    // An exponent is s c - m c + LIFT in one operation, whose second product is rounded, by up to 2^-25 of it, the same for all weights of a row.
    // From 2^20 on that is not small any more, and from 2^31 on it would leave the range of exp2: with FAR m is taken off first in
    // such rows; the others' results are the same bits either way.
    struct Whole {};
    template <int NB, bool FAR, class ReadK, class Half = Whole>
    __device__ __forceinline__ uint64_t step(const LaneReads<DP> &at, ReadK &&read_k, uint32_t vt, int key0, bool edge, uint64_t good, const Limits &mine, int sinks,
                                             float c, int lane, Half &&half = Whole{}) {
        constexpr bool HALVES = !std::is_same<typename std::decay<Half>::type, Whole>::value;
        uint64_t seen = ~0ull;
        f32x16 s[NB];
#pragma unroll
        for (int kb = 0; kb < NB; ++kb) s[kb] = (f32x16)0.f;
        // key blocks in turn: two chains of products
        __builtin_amdgcn_s_setprio(1);      // the matrix cores to the wave that is at the scores, arithmetic to the other of the SIMD
        products<NB * KS, 4>([&](int i) { return read_k(32 * (i % NB), i / NB); }, [&](int i, s16x8 x) { s[i % NB] = T::mma(x, q[i / NB], s[i % NB]); });
        __builtin_amdgcn_s_setprio(0);
        if (edge) {
            seen = seen_bits(mine, sinks, key0) & good;
            const uint64_t bits = seen >> (4 * (lane >> 5));
#pragma unroll
            for (int kb = 0; kb < NB; ++kb)
#pragma unroll
                for (int i = 0; i < 16; ++i) s[kb][i] = pick((uint32_t)(bits >> (32 * kb)), c_row(i, 0), s[kb][i], NO_KEY);
        }
        float top = s[0][0];
#pragma unroll
        for (int kb = 0; kb < NB; ++kb)
#pragma unroll
            for (int i = 0; i < 16; ++i) top = fmaxf(top, s[kb][i]);
        top = both_halves_max(top);
        if (__any((top - m) * c > GROW)) {       // m = -inf: the difference is inf, or NaN while nothing is visible
            const float now = fmaxf(m, top), by = m == now ? 1.f : __builtin_amdgcn_exp2f((m - now) * c);
            m = now;
            l *= by;
#pragma unroll
            for (int db = 0; db < DB; ++db)
#pragma unroll
                for (int i = 0; i < 16; ++i) o[db][i] *= by;
        }
        const bool far = FAR && m != NO_KEY && !near(c);
        const float off = far ? m : 0.f, base = m == NO_KEY ? 0.f : far ? LIFT : LIFT - m * c;
        float sums[2];
        auto weigh = [&](int kb, int from, int to) {
#pragma unroll
            for (int i = from; i < to; ++i) {
                s[kb][i] = __builtin_amdgcn_exp2f(__builtin_fmaf(FAR ? s[kb][i] - off : s[kb][i], c, base));
                sums[i % 2] = i < 2 ? s[kb][i] : sums[i % 2] + s[kb][i];
            }
            if (to == 16) l += sums[0] + sums[1];
        };
        weigh(0, 0, 16);
#pragma unroll
        for (int kb = 0; kb < NB; ++kb) {
            const s16x8 w[2] = {as_operand<T>(s[kb], 0), as_operand<T>(s[kb], 1)};
            if constexpr (HALVES) {
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    half(h);
                    products<DB, 2>([&](int i) { return at.column(vt, 0, i); }, [&](int i, s16x8 x) { o[i] = T::mma(x, w[h], o[i]); });
                }
                continue;
            }
            // the exponentials of the next block run under the products of this one
            products<2 * DB, 2>([&](int i) { return at.column(vt, 32 * kb + 16 * (i / DB), i % DB); },
                                [&](int i, s16x8 x) {
                                    o[i % DB] = T::mma(x, w[i / DB], o[i % DB]);
                                    if (kb + 1 < NB) weigh(kb + 1 < NB ? kb + 1 : 0, 16 * i / (2 * DB), 16 * (i + 1) / (2 * DB));
                                });
        }
        return seen;
    }
    __device__ bool near(float c) const { return m == NO_KEY || fabsf(m * c) <= 0x1p20f; }
    __device__ bool finite() const {
        bool all = true;
#pragma unroll
        for (int db = 0; db < DB; ++db)
#pragma unroll
            for (int i = 0; i < 16; ++i) all &= fabsf(o[db][i]) < __builtin_inff();
        return all;
    }
    // the logarithm of the row's sum, in natural units
    __device__ float lse(float all, float c) const { return all > 0.f ? (m * c - LIFT + __builtin_amdgcn_logf(all)) * LN2 : all == all ? NO_KEY : all; }
};

// Tiles of K and V straight to LDS, from rows of a tensor or from pages of a 16-bit cache
template <class T, int DP> struct Direct : Tile2<T, DP, KT> {
    using Base = Tile2<T, DP, KT>;
    int pages[Base::COUNT];    // of the next tile's rows

    __device__ void start(const AttendArgs &a, const Sequence &s, int hk, int wave, int lane) {
        if (a.table) Base::start(a.k.p, 0, a.v.p, 0, a.dim, wave, lane);
        else Base::start(a.k.p + 2 * ((int64_t)s.k0 * a.k.row + (int64_t)hk * a.k.head), a.k.row, a.v.p + 2 * ((int64_t)s.k0 * a.v.row + (int64_t)hk * a.v.head), a.v.row, a.dim, wave, lane);
    }
    __device__ void look(const AttendArgs &a, const Sequence &s, int b, int key0) {
        if (!a.table) return;
#pragma unroll
        for (int c = 0; c < Base::COUNT; ++c) {
            const int j = min(key0 + this->row + Base::STEP * c, s.nk - 1), page = a.table[(int64_t)b * a.table_row + (j >> a.page_shift)];
            pages[c] = page >= 0 && page < a.pages ? page : 0;
        }
    }
    __device__ void issue(const AttendArgs &a, const Sequence &s, int hk, int key0, const short *kt, const short *vt, int wave) const {
        if (!a.table) {
            Base::issue(key0, s.nk, a.dim, kt, vt, wave);
            return;
        }
#pragma unroll
        for (int c = 0; c < Base::COUNT; ++c) {
            const int j = min(key0 + this->row + Base::STEP * c, s.nk - 1), piece = this->piece * 8 < a.dim ? this->piece * 8 : 0;
            const int64_t at = 2 * (((((int64_t)pages[c] * a.kv_heads + hk) << a.page_shift) + (j & ((1 << a.page_shift) - 1))) * a.dim + piece);
            to_lds(a.k.p + at, lds_address(kt) + wave * 1024 + 4096 * c);
            to_lds(a.v.p + at, lds_address(vt) + wave * 1024 + 4096 * c);
        }
    }
};

// Many rows: a work item is 128 rows of one group, the four waves share tiles of 64 keys, two in LDS in turn.  Two blocks to a CU (three at a
// head size of 64), so that one's exponentials run under the other's products.  No unit is full: matrix cores and vector issue (the
// exponentials, one for 2 D multiply-adds, their sums, the mask) overlap in part only and fill about the whole time between them, at a clock that
// the power limit holds below 2.4 GHz.  Shares of a launch's cycles, matrix cores / vector issue / LDS:
//   16384 tokens with causal order, 8 heads of 128       502 to 536 us from card to card, 1.03 to 1.10 PFLOP/s    0.53 / 0.41 / 0.27 at 1.6 to 1.8 GHz
//   10007 rows over 20000 keys, 4 heads of 64, fp16      270 us and 26 for the join, 0.76 PFLOP/s               0.38 / 0.58 / 0.19 at 1.9
//   window of 1024, four texts of up to 4099, 16 heads   136 to 141 us; one wave to a SIMD, where two fit          0.23 / 0.23 / 0.11 at 2.2
//   1021 new tokens after up to 15000 in 8 bits, window 4096   157 to 166 us; each block converts the codes     0.35 / 0.42 / 0.36 at 2.1
// (a library's product of 16384^3 reaches 1.33 to 1.35 PFLOP/s on these cards).  Tried without gain: two blocks of 32 rows to a wave, the
// products of one tile under the exponentials of another in one wave, eight waves in two groups in turn.
template <class T, int DP, bool E8> __global__ __launch_bounds__(NT, DP == 128 ? 2 : 3) void attend_many(AttendArgs a) {
    using Row = Rows32<T, DP>;
    constexpr int ROWS = 128;
    __shared__ __attribute__((aligned(1024))) short tile[2][2][KT * DP];
    __shared__ uint64_t good_rows[2], odd_rows[2][4];
    const Item it = block_of(a, blockIdx.x);
    if (it.group >= a.groups) return;
    const int b = it.group / a.kv_heads, hk = it.group % a.kv_heads;
    const Sequence s = sequence_of(a, b);
    const int rows = min(s.nq, a.max_q) * a.group, r0 = it.tile * ROWS;
    if (r0 >= rows) return;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);

    const Limits first = limits_of(a, s, r0 / a.group), last = limits_of(a, s, min(r0 + ROWS - 1, rows - 1) / a.group);
    const Tiles tiles = tiles_of<KT>(first, last, a.sinks);
    int n = it.part * a.chunk, end = tiles.count;
    if (a.parts > 1) end = min(end, n + a.chunk);

    const int w0 = r0 + 32 * wave, row = min(w0 + (lane & 31), rows - 1), token = row / a.group, head = hk * a.group + row % a.group;
    const bool valid = w0 + (lane & 31) < rows;
    const Limits mine = limits_of(a, s, token);
    const Limits wfirst = limits_of(a, s, min(w0, rows - 1) / a.group), wlast = limits_of(a, s, min(w0 + 31, rows - 1) / a.group);
    const bool idle = w0 >= rows;
    const float c = a.scale * LOG2E;
    auto whole = [&](int key0) { return key0 + KT <= first.hi && (key0 >= last.lo || key0 + KT <= a.sinks); };

    LaneReads<DP> at;
    at.start(lane);
    Row r;
    const int begin = n;
    // Tiles that the mask cuts are not cleaned of infinities and NaN in v at first: if none shows in the results, there was none that
    // mattered.  Else all is done again with care, and so it is where scores are too large for the shorter exponents.
    auto pass = [&](auto with_care) {
        constexpr bool careful = decltype(with_care)::value;
        n = begin;
        r.start(a, a.q.p, (int64_t)(s.q0 + token) * a.q.row + (int64_t)head * a.q.head, lane);
        auto step = [&](int buf, int key0, uint64_t ok, uint64_t odd) {
            const bool none = idle || key0 >= wlast.hi || (key0 + KT <= wfirst.lo && key0 >= a.sinks);
            const bool full = key0 + KT <= wfirst.hi && (key0 >= wlast.lo || key0 + KT <= a.sinks) && ok == ~0ull && odd == 0;
            const uint32_t kt = lds_address(tile[buf][0]);
            if (none) return;
            const uint64_t seen = r.template step<2, careful>(at, [&](int base, int ks) { return at.row(kt, base, ks); }, lds_address(tile[buf][1]), key0, !full, ok, mine, a.sinks, c, lane);
            if (seen & odd) r.spoil = __builtin_nanf("");
        };
        if (n >= end) return;
        if constexpr (E8) {
            Codes<T, DP> next;
            uint64_t good = 0;
            auto fetch = [&](int t) {             // its pages are looked up; those of the tile after it follow
                next.load(a, s, hk, tiles[t] * KT, tid);
                good = next.good(a);
                if (t + 1 < end) next.look(a, s, b, tiles[t + 1] * KT, tid);
            };
            auto keep = [&](int t, int buf) {
                const uint64_t odd = next.store(tile[buf][0], tile[buf][1], tid, careful && (!whole(tiles[t] * KT) || good != ~0ull));
                if (careful && lane == 0) odd_rows[buf][wave] = odd;
                if (tid == 0) good_rows[buf] = good;
            };
            next.look(a, s, b, tiles[n] * KT, tid);
            fetch(n);
            keep(n, n & 1);
            registers_loaded();
            __syncthreads();
            for (; n < end; ++n) {
                const int buf = n & 1;
                if (n + 1 < end) fetch(n + 1);
                step(buf, tiles[n] * KT, good_rows[buf], careful ? odd_rows[buf][0] | odd_rows[buf][1] | odd_rows[buf][2] | odd_rows[buf][3] : 0);
                if (n + 1 < end) keep(n + 1, buf ^ 1);
                __syncthreads();
            }
        } else {
            Direct<T, DP> src;
            src.start(a, s, hk, wave, lane);
            uint64_t ok = 0, next_ok = 0;
            auto fetch = [&](int t, int buf) {             // its pages are looked up; those of the tile after it follow
                src.issue(a, s, hk, tiles[t] * KT, tile[buf][0], tile[buf][1], wave);
                next_ok = good_pages(a, s, b, tiles[t] * KT, lane);
                if (t + 1 < end) src.look(a, s, b, tiles[t + 1] * KT);
            };
            // waits for the loads of tile t
            auto take = [&](int t, int buf) -> uint64_t {
                arrived();
                __syncthreads();
                ok = next_ok;
                if (!careful || (whole(tiles[t] * KT) && ok == ~0ull)) return 0;
                const uint64_t odd = clean_tile<T, DP, KT>(tile[buf][1], tid);
                if (lane == 0) odd_rows[buf][wave] = odd;
                __syncthreads();
                return odd_rows[buf][0] | odd_rows[buf][1] | odd_rows[buf][2] | odd_rows[buf][3];
            };
            src.look(a, s, b, tiles[n] * KT);
            fetch(n, n & 1);
            registers_loaded();
            uint64_t odd = take(n, n & 1);
            for (; n < end; ++n) {
                const int buf = n & 1;
                if (n + 1 < end) fetch(n + 1, buf ^ 1);
                step(buf, tiles[n] * KT, ok, odd);
                if (n + 1 < end) odd = take(n + 1, buf ^ 1);
            }
        }
    };
    pass(std::false_type{});
    if (__syncthreads_or(!r.near(c) || !r.finite())) pass(std::true_type{});
    const float all = both_halves_sum(r.l), by = both_halves_sum(r.spoil) + (all > 0.f ? 1.f / all : all == all ? 0.f : all);
    const int64_t at_row = (int64_t)(s.q0 + token) * a.heads + head;
    if (a.parts > 1) {
        const int64_t at = (int64_t)it.part * a.total_q * a.heads + at_row;
        if (valid) {
            if (lane < 32) a.part_lse[at] = r.lse(all, c);
#pragma unroll
            for (int db = 0; db < Row::DB; ++db)
#pragma unroll
                for (int i = 0; i < 16; i += 4) {
                    const int d = 32 * db + c_row(i, lane);
                    if (d < a.dim) *(float4 *)(a.part_out + at * a.dim + d) = make_float4(r.o[db][i] * by, r.o[db][i + 1] * by, r.o[db][i + 2] * by, r.o[db][i + 3] * by);
                }
        }
        return;
    }
    if (valid && lane < 32) a.lse[at_row] = r.lse(all, c);
    store_rows<T, Row::DB>(r.o, by, a.out.p, (int64_t)(s.q0 + token) * a.out.row + (int64_t)head * a.out.head, a.dim, valid, lane);
}

// Few rows (single tokens, short chunks): a work item is 32 rows and a part of the keys; each of the four waves takes every fourth
// tile of 32 keys through a ring in LDS of its own, and the four results are joined at the end.  Bound by the reading of K and V: one token after
// 131071 in 16 bits: 102 us with the join, 5.3 TB/s where a copy, reading and writing, reaches 6.2; a token each of 64 sequences of up to 8192, 8
// key heads of 128 in 8 bits: 136 us, 4.4 TB/s, since the sequences differ in length and the parts are cut by the longest.
constexpr int PAGES_MAX = 1024;   // page numbers of a work item

template <class T, int DP, bool E8> __global__ __launch_bounds__(NT, E8 ? 2 : 1) void attend_few(AttendArgs a) {
    using Row = Rows32<T, DP>;
    constexpr int N = 32, BYTES = E8 ? 1 : 2, PIECES = DP * BYTES / 16, RPI = 64 / PIECES, COUNT = N / RPI;   // pieces of a row, rows to an instruction
    constexpr int RING = 2, TILE = N * DP * BYTES, SLOT = 2 * TILE + (E8 ? 256 : 0), LOADS = 2 * COUNT + (E8 ? 1 : 0), OF_WAVE = RING * SLOT;
    __shared__ __attribute__((aligned(1024))) char lds[4 * OF_WAVE];
    __shared__ int pages[PAGES_MAX];
    __shared__ float joined[4][2][32];
    const Item it = block_of(a, blockIdx.x);
    if (it.group >= a.groups) return;
    const int b = it.group / a.kv_heads, hk = it.group % a.kv_heads;
    const Sequence s = sequence_of(a, b);
    const int rows = min(s.nq, a.max_q) * a.group, r0 = it.tile * 32;
    if (r0 >= rows) return;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const Limits first = limits_of(a, s, r0 / a.group), last = limits_of(a, s, min(r0 + 31, rows - 1) / a.group);
    const Tiles tiles = tiles_of<N>(first, last, a.sinks);
    const int begin = it.part * a.chunk, end = min(tiles.count, begin + a.chunk);   // also of one part: pages[] holds no more
    const int row = min(r0 + (lane & 31), rows - 1), token = row / a.group, head = hk * a.group + row % a.group;
    const bool valid = r0 + (lane & 31) < rows;
    const int64_t at_row = (int64_t)(s.q0 + token) * a.heads + head;
    if (begin >= tiles.count && it.part > 0) {   // nothing here: the part counts as empty
        if (wave == 0 && lane < 32 && valid) a.part_lse[(int64_t)it.part * a.total_q * a.heads + at_row] = NO_KEY;
        return;
    }
    const Limits mine = limits_of(a, s, token);
    const float c = a.scale * LOG2E;

    LaneReads<DP> at;
    at.start(lane);
    Row r;
    r.start(a, a.q.p, (int64_t)(s.q0 + token) * a.q.row + (int64_t)head * a.q.head, lane);
    // the page of rows u * sub .. of tile begin + i is pages[i * subs + u]; -1: none
    const int shift = min(a.page_shift, 5), subs = 32 >> shift;
    if (a.table) {
        for (int x = tid; x < (end - begin) * subs; x += NT) {
            const int j = min(tiles[begin + x / subs] * N + (x % subs << shift), s.nk - 1), page = a.table[(int64_t)b * a.table_row + (j >> a.page_shift)];
            pages[x] = page >= 0 && page < a.pages ? page : -1;
        }
        __syncthreads();
    }
    registers_loaded();

    // the exchange of 16-byte pieces of a tile of codes: rows of one piece spread over all banks
    auto swap = [](int x) { return E8 ? (DP == 128 ? (x >> 1) & 7 : DP == 64 ? (x >> 2) & 3 : (x >> 3) & 1) : piece_swap<DP>(x); };
    const uint32_t ring = lds_address((const short *)lds) + wave * OF_WAVE;
    auto fetch = [&](int n, int slot) {
        const int key0 = tiles[n] * N;
        const uint32_t to = ring + slot * SLOT;
#pragma unroll
        for (int x = 0; x < COUNT; ++x) {
            const int in = x * RPI + lane / PIECES, j = min(key0 + in, s.nk - 1), y = 16 * ((lane % PIECES) ^ swap(in)), piece = y < BYTES * a.dim ? y : 0;
            int64_t k, v;
            if (a.table) {
                const int page = max(pages[(n - begin) * subs + (in >> shift)], 0);
                k = v = BYTES * ((((int64_t)page * a.kv_heads + hk) << a.page_shift) + (j & ((1 << a.page_shift) - 1))) * a.dim + piece;
            } else {
                k = BYTES * ((int64_t)(s.k0 + j) * a.k.row + (int64_t)hk * a.k.head) + piece;
                v = BYTES * ((int64_t)(s.k0 + j) * a.v.row + (int64_t)hk * a.v.head) + piece;
            }
            to_lds(a.k.p + k, to + 1024 * x);
            to_lds(a.v.p + v, to + TILE + 1024 * x);
        }
        if (E8) {   // four exponents to a lane: of k, then of v; pages hold multiples of 8 rows
            const int in = 4 * (lane & 7), j = min(key0 + in, (s.nk - 1) & ~3), page = max(pages[(n - begin) * subs + (in >> shift)], 0);
            const int64_t x = (((int64_t)page * a.kv_heads + hk) << a.page_shift) + (j & ((1 << a.page_shift) - 1));
            word_to_lds((const float *)((lane & 8 ? a.v_exp : a.k_exp) + x), to + 2 * TILE);
        }
    };
    int n = begin + wave;
    if (n < end) {
        const int final = n + (end - 1 - n) / 4 * 4;      // the wave's last tile: loaded again past the end, which keeps the count of loads
        for (int x = 0; x < RING; ++x) fetch(min(n + 4 * x, final), x);
        for (int slot = 0; n < end; n += 4, slot = slot + 1 < RING ? slot + 1 : 0) {
            const int key0 = tiles[n] * N;
            const uint32_t kt = ring + slot * SLOT, vt = kt + TILE;
            uint64_t good = ~0ull;
            if (a.table) good = __ballot(pages[(n - begin) * subs + ((lane & 31) >> shift)] >= 0);
            const bool whole = key0 + N <= first.hi && (key0 >= last.lo || key0 + N <= a.sinks) && good == ~0ull;
            arrived<(RING - 1) * LOADS>();
            uint64_t odd = 0, seen;
            using lds_piece = __attribute__((address_space(3))) u32x4;
            if constexpr (E8) {
                using lds_byte = __attribute__((address_space(3))) const uint8_t;
                using lds_codes = __attribute__((address_space(3))) const u32x2;
                const float scale = __builtin_bit_cast(float, (uint32_t)*(lds_byte *)(uintptr_t)(kt + 2 * TILE + (lane & 31)) << 23);
                const uint32_t from = kt + (lane & 31) * DP + 16 * swap(lane & 31) + 8 * (lane >> 5);
                auto read_k = [&](int, int ks) {
                    const u32x2 w = *(lds_codes *)(uintptr_t)(from ^ (16 * ks));
                    return __builtin_bit_cast(s16x8, (u32x4){T::template codes<false>(w[0], scale), T::template codes<true>(w[0], scale),
                                                            T::template codes<false>(w[1], scale), T::template codes<true>(w[1], scale)});
                };
                // 16 rows of v as 16-bit values, for transposing reads, where k was: k is not needed any more
                auto half = [&](int h) {
                    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");   // LDS does a wave's accesses in their order: nothing to wait for
#pragma unroll
                    for (int x = 0; x < COUNT; ++x) {
                        const int in = x * RPI + lane / PIECES, piece = (lane % PIECES) ^ swap(in);
                        if (COUNT > 1 ? x * RPI / 16 != h : in / 16 != h) continue;
                        const u32x4 w = *(lds_piece *)(uintptr_t)(vt + 1024 * x + 16 * lane);
                        const float by = __builtin_bit_cast(float, (uint32_t)*(lds_byte *)(uintptr_t)(kt + 2 * TILE + 32 + in) << 23);
#pragma unroll
                        for (int z = 0; z < 2; ++z) {
                            u32x4 y = {T::template codes<false>(w[2 * z], by), T::template codes<true>(w[2 * z], by),
                                       T::template codes<false>(w[2 * z + 1], by), T::template codes<true>(w[2 * z + 1], by)};
                            if (!whole && any_odd<T>(y)) {
                                y = cleaned<T>(y);
                                odd |= 1ull << in;
                            }
                            *(lds_piece *)(uintptr_t)(kt + 2 * tile_at<DP>(in & 15, 2 * piece + z)) = y;
                        }
                    }
                    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
                };
                seen = r.template step<1, true>(at, read_k, kt, key0, !whole, good, mine, a.sinks, c, lane, half);
            } else {
                if (!whole) {
#pragma unroll 2
                    for (int x = 0; x < COUNT; ++x) {
                        lds_piece *const p = (lds_piece *)(uintptr_t)(vt + 1024 * x + 16 * lane);
                        const u32x4 w = *p;
                        if (any_odd<T>(w)) {
                            *p = cleaned<T>(w);
                            odd |= 1ull << (x * RPI + lane / PIECES);
                        }
                    }
                }
                __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
                seen = r.template step<1, true>(at, [&](int base, int ks) { return at.row(kt, base, ks); }, vt, key0, !whole, good, mine, a.sinks, c, lane);
            }
            if (!whole && __any(odd != 0)) {
#pragma unroll 1
                for (int by = 32; by > 0; by >>= 1) odd |= __shfl_xor((unsigned long long)odd, by);
                if (seen & odd) r.spoil = __builtin_nanf("");
            }
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            fetch(min(n + 4 * RING, final), slot);
        }
        arrived();      // LDS is used otherwise from here on
    }
    // join: every wave's o in the common unit, summed over the waves from LDS
    const float all = both_halves_sum(r.l);
    if (lane < 32) { joined[wave][0][lane] = r.m; joined[wave][1][lane] = all; }
    __syncthreads();
    float top = NO_KEY, sum = 0.f;
#pragma unroll
    for (int w = 0; w < 4; ++w) top = fmaxf(top, joined[w][0][lane & 31]);
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        const float m = joined[w][0][lane & 31];
        sum += m == NO_KEY && joined[w][1][lane & 31] == 0.f ? 0.f : joined[w][1][lane & 31] * __builtin_amdgcn_exp2f((m - top) * c);
    }
    const float spoil = both_halves_sum(r.spoil);
    const float unit = all == 0.f ? 0.f : __builtin_amdgcn_exp2f((r.m - top) * c), by = spoil + (sum > 0.f ? unit / sum : sum == sum ? 0.f : sum);
    r.m = top;
    static_assert(OF_WAVE >= 4 * 32 * DP, "room for 32 x DP values of fp32");
    float *mine_o = (float *)(lds + wave * OF_WAVE);
#pragma unroll
    for (int db = 0; db < Row::DB; ++db)
#pragma unroll
        for (int i = 0; i < 16; i += 4) {
            const int d4 = (32 * db + c_row(i, lane)) >> 2;
            *(float4 *)(mine_o + (lane & 31) * DP + (((d4 ^ (lane & 7)) << 2))) = make_float4(r.o[db][i] * by, r.o[db][i + 1] * by, r.o[db][i + 2] * by, r.o[db][i + 3] * by);
        }
    if (wave == 0 && lane < 32 && valid) {
        const float y = r.lse(sum, c);
        if (a.parts > 1) a.part_lse[(int64_t)it.part * a.total_q * a.heads + at_row] = y;
        else a.lse[at_row] = y;
    }
    __syncthreads();
    for (int at = tid; at < 32 * (DP / 8); at += NT) {
        const int x = at / (DP / 8), d = at % (DP / 8) * 8;
        if (r0 + x >= rows || d >= a.dim) continue;
        float y[8];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            float4 t = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                const float4 u = *(const float4 *)((const float *)(lds + w * OF_WAVE) + x * DP + ((((d >> 2) + h) ^ (x & 7)) << 2));
                t.x += u.x; t.y += u.y; t.z += u.z; t.w += u.w;
            }
            y[4 * h] = t.x; y[4 * h + 1] = t.y; y[4 * h + 2] = t.z; y[4 * h + 3] = t.w;
        }
        const int tk = (r0 + x) / a.group, hd = hk * a.group + (r0 + x) % a.group;
        if (a.parts > 1) {
            float *to = a.part_out + (((int64_t)it.part * a.total_q + s.q0 + tk) * a.heads + hd) * a.dim + d;
            *(float4 *)to = make_float4(y[0], y[1], y[2], y[3]);
            *(float4 *)(to + 4) = make_float4(y[4], y[5], y[6], y[7]);
        } else {
            *(u32x4 *)(a.out.p + 2 * ((int64_t)(s.q0 + tk) * a.out.row + (int64_t)hd * a.out.head + d)) =
                (u32x4){T::pack(y[0], y[1]), T::pack(y[2], y[3]), T::pack(y[4], y[5]), T::pack(y[6], y[7])};
        }
    }
}

// whether a row of q and its results belongs to some sequence (and to its first max_q tokens): others have no parts and are left alone
__device__ __forceinline__ bool in_sequence(const AttendArgs &a, int64_t token) {
    if (!a.q_offsets) return token < a.max_q;
    int lo = 0, hi = a.batch;      // the last offset not above the token
    while (lo < hi) {
        const int mid = (lo + hi) / 2;
        if (a.q_offsets[mid + 1] <= token) lo = mid + 1;
        else hi = mid;
    }
    const int64_t first = max(lo < a.batch ? a.q_offsets[lo] : 0, 0);      // as sequence_of cuts it
    return lo < a.batch && token >= first && token - first < a.max_q;
}
template <class T> __device__ __forceinline__ void store_joined(const AttendArgs &a, int64_t row, int x, float top, float sum, float4 o) {
    const float by = sum > 0.f ? 1.f / sum : sum == sum ? 0.f : sum;
    if (x == 0) a.lse[row] = sum > 0.f ? top + __builtin_amdgcn_logf(sum) * LN2 : sum == sum ? NO_KEY : sum;
    if (x < a.dim)
        *(u32x2 *)(a.out.p + 2 * (row / a.heads * a.out.row + row % a.heads * a.out.head + x)) = (u32x2){T::pack(o.x * by, o.y * by), T::pack(o.z * by, o.w * by)};
}

// The parts of each row joined: 32 lanes to a row, four dimensions each, part after part.  Bound by reading them: 40028 rows of 64, 4 to 6
// parts: 14 to 27 us
template <class T> __global__ __launch_bounds__(NT) void join_few(AttendArgs a) {
    const int64_t row = (int64_t)blockIdx.x * 8 + threadIdx.x / 32, all = a.total_q * a.heads;
    if (row >= all || !in_sequence(a, row / a.heads)) return;
    const int x = threadIdx.x % 32 * 4;
    float top = NO_KEY, sum = 0.f;
    for (int p = 0; p < a.parts; ++p) top = fmaxf(top, a.part_lse[p * all + row]);
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int p = 0; p < a.parts; ++p) {
        const float l = a.part_lse[p * all + row];
        if (l == NO_KEY) continue;
        const float w = __builtin_amdgcn_exp2f((l - top) * LOG2E);
        sum += w;
        if (x < a.dim) {
            const float4 u = *(const float4 *)(a.part_out + (p * all + row) * a.dim + x);
            o.x += w * u.x; o.y += w * u.y; o.z += w * u.z; o.w += w * u.w;
        }
    }
    store_joined<T>(a, row, x, top, sum, o);
}

// The same for many parts, a block to a row: the parts' weights by all threads, then every eighth part to 32 lanes
template <class T> __global__ __launch_bounds__(NT) void join_many(AttendArgs a) {
    __shared__ float weight[NT], most[4], sums[4];
    __shared__ float4 partial[8][32];
    const int64_t row = blockIdx.x, all = a.total_q * a.heads;
    const int tid = threadIdx.x, x = tid % 32 * 4;
    if (!in_sequence(a, row / a.heads)) return;
    float top = NO_KEY;
    for (int p = tid; p < a.parts; p += NT) top = fmaxf(top, a.part_lse[p * all + row]);
#pragma unroll
    for (int by = 32; by > 0; by >>= 1) top = fmaxf(top, __shfl_xor(top, by));
    if (tid % 64 == 0) most[tid / 64] = top;
    __syncthreads();
    top = fmaxf(fmaxf(most[0], most[1]), fmaxf(most[2], most[3]));
    float sum = 0.f;
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int p0 = 0; p0 < a.parts; p0 += NT) {
        const float l = p0 + tid < a.parts ? a.part_lse[(p0 + tid) * all + row] : NO_KEY, w = l == NO_KEY ? 0.f : __builtin_amdgcn_exp2f((l - top) * LOG2E);
        sum += w;
        __syncthreads();
        weight[tid] = l == NO_KEY ? -1.f : w;          // -1: nothing was written for this part
        __syncthreads();
        if (x < a.dim)
#pragma unroll 4
            for (int p = tid / 32; p < min(NT, a.parts - p0); p += 8) {
                const float v = weight[p];
                if (v == -1.f) continue;
                const float4 u = *(const float4 *)(a.part_out + ((p0 + p) * all + row) * a.dim + x);
                o.x += v * u.x; o.y += v * u.y; o.z += v * u.z; o.w += v * u.w;
            }
    }
#pragma unroll
    for (int by = 32; by > 0; by >>= 1) sum += __shfl_xor(sum, by);
    if (tid % 64 == 0) sums[tid / 64] = sum;
    partial[tid / 32][tid % 32] = o;
    __syncthreads();
    if (tid >= 32) return;
#pragma unroll
    for (int p = 1; p < 8; ++p) {
        const float4 u = partial[p][tid];
        o.x += u.x; o.y += u.y; o.z += u.z; o.w += u.w;
    }
    store_joined<T>(a, row, x, top, (sums[0] + sums[1]) + (sums[2] + sums[3]), o);
}

// key tiles of `per` rows that a work item of `rows` (token, head) rows may see at most
int64_t most_tiles(const AttendArgs &a, int64_t max_k, int rows, int per) {
    int64_t t = cdiv(max_k, per);
    if (a.window) t = std::min(t, cdiv(rows, a.group) / per + a.window / per + 4 + cdiv(a.sinks, per));
    return std::max<int64_t>(t, 1);
}

template <class T, int DP, bool E8> void launch(const AttendArgs &a, bool few, int64_t blocks, hipStream_t st) {
    if (few) attend_few<T, DP, E8><<<dim3((uint32_t)blocks), NT, 0, st>>>(a);
    else attend_many<T, DP, E8><<<dim3((uint32_t)blocks), NT, 0, st>>>(a);
    F3M_HIP(hipGetLastError());
    if (a.parts > 1) {
        const int64_t all = a.total_q * a.heads;
        if (a.parts > 8 && all < 4096) join_many<T><<<dim3((uint32_t)all), NT, 0, st>>>(a);
        else join_few<T><<<dim3((uint32_t)cdiv(all, 8)), NT, 0, st>>>(a);
        F3M_HIP(hipGetLastError());
    }
}

// Head sizes in between run as the next of these: zeros in LDS and registers, and as many products.  At 80 and 96, as 128, that is 16 where 10 and
// 12 would hold the values.
template <class T> void launch_dim(const AttendArgs &a, bool e8, bool few, int64_t blocks, hipStream_t st) {
    if (a.dim <= 32) e8 ? launch<T, 32, true>(a, few, blocks, st) : launch<T, 32, false>(a, few, blocks, st);
    else if (a.dim <= 64) e8 ? launch<T, 64, true>(a, few, blocks, st) : launch<T, 64, false>(a, few, blocks, st);
    else e8 ? launch<T, 128, true>(a, few, blocks, st) : launch<T, 128, false>(a, few, blocks, st);
}

// Up to 32 rows to a key head go to attend_few, one tile of its rows (a token each of 64 sequences of up to 8192, 4 heads to a key head, 8-bit
// cache: 146 us, 206 in attend_many; of one of 32768: 27 and 31; of 16 of 4096 each: 44 and 40), more to attend_many (64 rows of 16 sequences
// of 4096: 52 us, 75 in attend_few; of one of 32768: 38 and 42).  A long key axis is
// cut into parts where the rows alone make too few blocks.
// attend_few: one block to a CU at a time (two with 8-bit codes), whose waves keep 64 KB or more under way; as many parts as fill one round of
// them (one token after 131071 in 16 bits, 8 key heads: 112 us in 8 parts, 102 in 32, 109 in 64, 119 in 128; 16 sequences of 4096 in 8
// bits: 55 us whole, 35 in 4 parts, 44 in 8).  Where that leaves one, three in 8 bits from 4096 keys on, since sequences differ in length (64
// of up to 8192: 153 us whole, 137 in 3; all as long as the longest: 203 and 213; 64 of up to 1000: 28 and 43), in 16 bits it stays
// (24 of up to 6000: 87 and 84; all as long: 106 and 132; 64 of up to 8192: 249 and 234).
// Up to 512 keys the second launch costs more than it saves.
// attend_many: two blocks to a CU (three up to a head size of 64).  Where causal order makes the rows' lengths rise along the sequence, as many
// parts as fill 88 % of those places, p parts of the longest being about (p + 1) / 2 to a tile (4096 tokens, 8 heads, one key head: 84 us
// whole, 71 in 2 parts, 64 in 3, 80 in 4); else the least time, counted in items: rounds of parts, and for each part that falls to a place
// 0.02, its beginning, its end and its share of the join (twice 500 new tokens after 7500, 8 heads, 2 key heads: 183 us whole, 67 in 4
// parts, 63 in 8, 75 in 16).  Parts have 8 or 10 tiles or more, since shorter
// ones cost as much as they save (4 x 1024 tokens, 8 heads of 64, no order: 21 us whole, 33 in two parts).
bool split(AttendArgs &a, int64_t max_k, bool e8) {
    const bool few = (int64_t)a.max_q * a.group <= 32;
    const int per = few ? 32 : KT, rows = few ? 32 : 128;
    a.tiles = (int)cdiv((int64_t)a.max_q * a.group, rows);
    const int64_t most = most_tiles(a, max_k, rows, per);
    if (few) {
        int64_t parts = (e8 ? 512 : 256) / ((int64_t)a.tiles * a.groups);
        if (parts <= 1) parts = e8 && most >= 128 ? 3 : 1;
        a.chunk = (int)std::min(most > 16 ? std::max<int64_t>(cdiv(most, parts), 4) : most, (int64_t)PAGES_MAX / 4);
    } else {
        const int64_t places = a.dim > 64 ? 512 : 768, items = all_tiles(a, a.tiles, a.total_q * a.group);
        int64_t parts = 1;
        if (a.causal && most == cdiv(max_k, per) && 2 * (int64_t)a.max_q >= max_k) {
            parts = std::min((44 * places / 25 - items / 2) / items, most / 8);
        } else if (items < places) {
            double least = 1e30;
            for (int64_t rounds = 0; rounds <= 6; ++rounds) {   // as many parts as fill them; 0: one part
                const int64_t p = rounds ? rounds * places / items : 1;
                const double cost = (double)cdiv(items * p, places) / (double)p + 0.02 * (double)p * (double)items / (double)places;
                if (cost < least) {
                    least = cost;
                    parts = p;
                }
            }
            parts = std::min(parts, most / 10);
        }
        a.chunk = (int)cdiv(most, std::max<int64_t>(1, parts));
    }
    a.parts = (int)cdiv(most, a.chunk);
    return few;
}

}  // namespace

int64_t attend_workspace(AttendArgs a, int64_t max_k) {
    if (!a.max_q || !a.total_q || !a.groups) return 0;
    int64_t parts = 1;           // of either kind of cache: the caller does not say
    for (const bool e8 : {false, true}) {
        split(a, max_k, e8);
        parts = std::max<int64_t>(parts, a.parts);
    }
    return parts > 1 ? parts * a.total_q * a.heads * (a.dim + 1) * (int64_t)sizeof(float) : 0;
}

void run_attend(AttendArgs a, int64_t max_k, bool f16, bool e8, void *workspace, hipStream_t st) {
    if (!a.max_q || !a.total_q || !a.groups) return;
    const bool few = split(a, max_k, e8);
    a.part_out = (float *)workspace;
    a.part_lse = a.part_out ? a.part_out + (int64_t)a.parts * a.total_q * a.heads * a.dim : nullptr;
    const int64_t blocks = attend_blocks(a, (int64_t)a.tiles * a.parts);
    if (a.parts > 1 && cdiv(a.total_q * a.heads, 8) >= 1 << 24) fail(F3M_ERR_UNSUPPORTED, "attention: too many rows to join parts of in one call (2^27)");
    f16 ? launch_dim<F16>(a, e8, few, blocks, st) : launch_dim<Bf16>(a, e8, few, blocks, st);
}

// sets a.pinned; blocks of a launch with `items` to a group
int64_t attend_blocks(AttendArgs &a, int64_t items) {
    a.pinned = a.groups % 8 == 0 || a.groups >= 64;
    const int64_t blocks = (a.pinned ? cdiv(a.groups, 8) * 8 : a.groups) * items;
    if (blocks > (1 << 24) - 1) fail(F3M_ERR_UNSUPPORTED, "attention: too many work items for one call (2^24)");
    return blocks;
}

}  // namespace f3m
