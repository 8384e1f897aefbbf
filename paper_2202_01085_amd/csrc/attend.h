// Row-normalised products (attention): what the kernels of attend.hip, attend_grad.hip and cache.hip share.
//
// Every product of a 32 x 32 block runs on v_mfma_f32_32x32x16 (fp32 sums).  Lane l of a wave has the operand values
//   A[l % 32][8 (l / 32) + j],  B[8 (l / 32) + j][l % 32],  j = 0..7
// and the results C[(i % 4) + 8 (i / 4) + 4 (l / 32)][l % 32], i = 0..15.  So a block of results whose columns stay (queries,
// say) is the B operand of the next product as it lies in the registers, if that product takes its 16 summands in the order
//   slot (l / 32, j)  <->  row 4 (l / 32) + j % 4 + 8 (j / 4)
// and its A operand is read in the same order: two transposing LDS reads of four rows each (column).  No value crosses lanes.
#pragma once
#include "common.h"

#include <algorithm>

namespace f3m {

// one tensor of rows x heads x head_dim, strides in values
struct Rows {
    char *p;
    int64_t row, head;
};

struct AttendArgs {
    int batch, heads, kv_heads, group, dim;   // group = heads / kv_heads
    int causal, window, sinks;
    float scale;
    int64_t total_q, total_k;
    int max_q, max_k;
    const int *q_offsets, *k_offsets;         // null: one sequence
    Rows q, k, v, out;
    float *lse;                               // (rows of q, heads)
    // keys in pages (attention over a cache): pages of page_size rows, all heads of a page behind one another
    const int *table, *lengths;               // table null: rows of k and v
    int64_t table_row, pages;
    int table_cols, page_shift;
    const uint8_t *k_exp, *v_exp;             // 8-bit codes: exponent bytes of the rows
    // the launch
    int tiles, groups, pinned, chunk;         // row tiles of the longest sequence, batch * kv_heads, see block_of, key tiles of a part
    int parts;                                // parts of the key axis; above 1 the results go to part_out, part_lse
    float *part_out, *part_lse;               // (parts, rows of q, heads, dim) and (parts, rows of q, heads); gradients: see tile_slot
    // gradient
    Rows dout, dq, dk, dv;
    float *stat;                              // (2, heads, rows of q): -log2 of the row's sum (-inf: empty row), -dO.O
    int usual;                                // parts of key tiles without sinks, chunk row tiles each; `parts` is the most of any
    int sink_tiles, sink_chunk, sink_parts;   // the first key tiles of a sequence, with sinks; row tiles of a part of theirs; the most parts of one
    int packed, sink_packed;                  // how the parts' sums are numbered, see tile_slot and key_sums
    int64_t slots, sink_slots;                // numbers of a key head
    float *sink_out;                          // sums of the sinks' tiles: (sink_slots, sink_tiles, kv_heads, 2, 128, dim)
};

using s16x4 = __attribute__((ext_vector_type(4))) short;
using s16x8 = __attribute__((ext_vector_type(8))) short;
using f32x16 = __attribute__((ext_vector_type(16))) float;
using f32x2 = __attribute__((ext_vector_type(2))) float;
using u32x4 = __attribute__((ext_vector_type(4))) uint32_t;
using u32x2 = __attribute__((ext_vector_type(2))) uint32_t;
using bf16x8 = __attribute__((ext_vector_type(8))) __bf16;
using bf16x2 = __attribute__((ext_vector_type(2))) __bf16;
using f16x8 = __attribute__((ext_vector_type(8))) _Float16;
using f16x2 = __attribute__((ext_vector_type(2))) _Float16;

constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;
constexpr float NO_KEY = -__builtin_inff();

struct Bf16 {
    static constexpr bool narrow = false;          // fp32's range of exponents: no value needs scaling
    static constexpr int nonfinite = 0x7f80;
    static __device__ f32x16 mma(s16x8 a, s16x8 b, f32x16 c) {
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
    }
    static __device__ uint32_t pack(float x, float y) {
        return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2){x, y}, bf16x2));
    }
    static __device__ float up(uint16_t x) { return __builtin_bit_cast(float, (uint32_t)x << 16); }
    // two of the four e4m3 codes of w, times scale (a power of two): exact
    template <bool HIGH> static __device__ uint32_t codes(uint32_t w, float scale) {
        return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, HIGH));
    }
};

struct F16 {
    static constexpr bool narrow = true;
    static constexpr int nonfinite = 0x7c00;
    static __device__ f32x16 mma(s16x8 a, s16x8 b, f32x16 c) {
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
    }
    static __device__ uint32_t pack(float x, float y) {
        return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2){x, y}, f16x2));
    }
    static __device__ float up(uint16_t x) { return (float)__builtin_bit_cast(_Float16, x); }
    template <bool HIGH> static __device__ uint32_t codes(uint32_t w, float scale) {
        return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, scale, HIGH));
    }
};

// tiles of 128 rows of all groups: `tiles` in the longest sequence, at most as many as all rows make
inline int64_t all_tiles(const AttendArgs &a, int64_t tiles, int64_t rows) {
    return std::max<int64_t>(1, std::min(tiles * a.groups, (rows / 128 + a.batch) * a.kv_heads));
}

// attend.hip, attend_grad.hip: the launches, and the bytes of workspace that they need
int64_t attend_workspace(AttendArgs a, int64_t max_k);
void run_attend(AttendArgs a, int64_t max_k, bool f16, bool e8, void *workspace, hipStream_t st);
int64_t attend_blocks(AttendArgs &a, int64_t items);
int64_t attend_grad_workspace(AttendArgs a, int64_t max_k);
void run_attend_grad(AttendArgs a, int64_t max_k, bool f16, void *workspace, hipStream_t st);
// cache.hip
void run_cache_rows(const f3m_cache &c, bool f16, const int64_t *slot, int64_t tokens, const f3m_rows &k, const f3m_rows &v, bool write,
                    hipStream_t st);

// ---- tiles in LDS: rows of DP values, their 16-byte pieces exchanged so that what a read takes at once lies in different banks: 16 rows at
// one piece (row), four rows at four neighbouring pieces (column) ----
template <int DP> __device__ __forceinline__ int piece_swap(int r) {
    if (DP == 128) return ((r & 3) << 2) | ((r >> 2) & 3);
    if (DP == 64) return ((r & 2) << 1) | ((r >> 2) & 3);
    return (r >> 2) & 3;   // 32
}
template <int DP> __device__ __forceinline__ int tile_at(int r, int piece) {   // in values
    return r * DP + ((piece ^ piece_swap<DP>(r)) << 3);
}
using lds_short = __attribute__((address_space(3))) short;
using lds_s16x4 = __attribute__((address_space(3))) s16x4;
using lds_s16x8 = __attribute__((address_space(3))) s16x8;
__device__ __forceinline__ uint32_t lds_address(const short *p) { return (uint32_t)(uintptr_t)(const lds_short *)p; }

// Where a lane reads operands of a tile.  Exchanged pieces make the addresses of other pieces exclusive ors, and rows 32 (or 16) further have
// the same exchange, so they are offsets that the instruction holds: one register to a tile, one operation to a piece.
template <int DP> struct LaneReads {
    uint32_t r, t;       // bytes from the tile's start (aligned to a row of pieces) for row() and column()
    __device__ void start(int lane) {
        r = 2 * tile_at<DP>(lane & 31, lane >> 5);
        const int i = lane & 15;
        t = 2 * (tile_at<DP>(4 * (lane >> 5) + (i >> 2), 2 * ((lane >> 4) & 1) + ((i & 3) >> 1)) + ((i & 1) << 2));
    }
    // A operand whose rows are rows base .. base + 31 of the tile (base a multiple of 32): dimensions 16 ks .. 16 ks + 15
    __device__ s16x8 row(uint32_t tile, int base, int ks) const {
        return *(const lds_s16x8 *)(uintptr_t)(((tile + r) ^ (32 * ks)) + 2 * DP * base);
    }
    // A operand whose rows are dimensions 32 db .. 32 db + 31 and whose summands are rows base .. base + 15 (base a multiple of 16) of the
    // tile, in the order above: four rows to a read, transposed on the way
    __device__ s16x8 column(uint32_t tile, int base, int db) const {
        constexpr uint32_t EIGHT = 32;   // what the exchange of a row 8 further adds
        const s16x4 x = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(uintptr_t)(((tile + t) ^ (64 * db)) + 2 * DP * base));
        const s16x4 y = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(uintptr_t)(((tile + t) ^ (64 * db) ^ EIGHT) + 2 * DP * (base + 8)));
        return __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7);
    }
};
// Products whose operands come from LDS, read AHEAD of their use: read(i) gives the operand of product i, use(i, operand) makes it.  The
// order is fixed for the scheduler, which would otherwise read each operand just before its product and wait; arithmetic may move across.
__device__ __forceinline__ void keep_order() { __builtin_amdgcn_sched_barrier(0x406); }   // vector and scalar arithmetic may cross
template <int COUNT, int AHEAD, class Read, class Use> __device__ __forceinline__ void products(Read &&read, Use &&use) {
    s16x8 x[AHEAD];
#pragma unroll
    for (int i = 0; i < AHEAD && i < COUNT; ++i) x[i] = read(i);
    keep_order();
#pragma unroll
    for (int i = 0; i < COUNT; ++i) {
        use(i, x[i % AHEAD]);
        if (i + AHEAD < COUNT) x[i % AHEAD] = read(i + AHEAD);
        keep_order();
    }
}

// row of result i of a lane
__device__ __forceinline__ int c_row(int i, int lane) { return (i & 3) + 8 * (i >> 2) + 4 * (lane >> 5); }

__device__ __forceinline__ float both_halves_max(float x) {
    auto r = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(uint32_t, x), __builtin_bit_cast(uint32_t, x), false, false);
    return fmaxf(__builtin_bit_cast(float, (uint32_t)r[0]), __builtin_bit_cast(float, (uint32_t)r[1]));
}
__device__ __forceinline__ float both_halves_sum(float x) {
    auto r = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(uint32_t, x), __builtin_bit_cast(uint32_t, x), false, false);
    return __builtin_bit_cast(float, (uint32_t)r[0]) + __builtin_bit_cast(float, (uint32_t)r[1]);
}

// results 8 s .. 8 s + 7 of a block as a B operand
template <class T> __device__ __forceinline__ s16x8 as_operand(const f32x16 &c, int s) {
    u32x4 w;
#pragma unroll
    for (int j = 0; j < 4; ++j) w[j] = T::pack(c[8 * s + 2 * j], c[8 * s + 2 * j + 1]);
    return __builtin_bit_cast(s16x8, w);
}

// Infinities and NaN in a row that is hidden from some columns must not reach those (0 * NaN = NaN in the product): where the mask
// cuts a tile, operands are cleaned of them, and what they do to the columns that see them is put right otherwise.
template <class T> __device__ __forceinline__ bool any_odd(u32x4 w) {
    bool odd = false;
#pragma unroll
    for (int j = 0; j < 4; ++j)
        odd |= (w[j] & (uint32_t)T::nonfinite) == (uint32_t)T::nonfinite || (w[j] >> 16 & (uint32_t)T::nonfinite) == (uint32_t)T::nonfinite;
    return odd;
}
template <class T> __device__ __forceinline__ u32x4 cleaned(u32x4 w) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        if ((w[j] & (uint32_t)T::nonfinite) == (uint32_t)T::nonfinite) w[j] &= 0xffff0000u;
        if ((w[j] >> 16 & (uint32_t)T::nonfinite) == (uint32_t)T::nonfinite) w[j] &= 0xffffu;
    }
    return w;
}

// ---- sequences ----
struct Sequence {
    int q0, nq, k0, nk;
};
// offsets outside the tensors, or that fall, give shorter or empty sequences and never an access out of range
__device__ __forceinline__ Sequence sequence_of(const AttendArgs &a, int b) {
    Sequence s;
    int64_t q0 = 0, q1 = a.total_q, k0 = 0, k1 = a.total_k;
    if (a.q_offsets) {
        q0 = min(max((int64_t)a.q_offsets[b], (int64_t)0), a.total_q);
        q1 = min(max((int64_t)a.q_offsets[b + 1], q0), a.total_q);
    }
    if (a.table) {
        k0 = 0;
        k1 = min(max((int64_t)a.lengths[b], (int64_t)0), (int64_t)a.table_cols << a.page_shift);
    } else if (a.k_offsets) {
        k0 = min(max((int64_t)a.k_offsets[b], (int64_t)0), a.total_k);
        k1 = min(max((int64_t)a.k_offsets[b + 1], k0), a.total_k);
    }
    s.q0 = (int)q0; s.nq = (int)(q1 - q0); s.k0 = (int)k0; s.nk = (int)(k1 - k0);
    return s;
}

// keys [lo, hi) and the first `sinks` below hi are visible to a token of the sequence
struct Limits {
    int lo, hi;
};
__device__ __forceinline__ Limits limits_of(const AttendArgs &a, const Sequence &s, int token) {
    if (!a.causal) return {0, s.nk};
    const int pos = s.nk - s.nq + token;
    return {a.window && pos >= a.window ? pos - a.window + 1 : 0, pos + 1};
}

// bits of the keys of a tile (bit r: key0 + r) that a row sees
__device__ __forceinline__ uint64_t below(int n) { return n >= 64 ? ~0ull : n <= 0 ? 0ull : (1ull << n) - 1; }
__device__ __forceinline__ uint64_t seen_bits(const Limits &m, int sinks, int key0) {
    return below(m.hi - key0) & (~below(m.lo - key0) | below(sinks - key0));
}
// x where bit `at` of the word is set, else y
__device__ __forceinline__ float pick(uint32_t bits, int at, float x, float y) {
    const uint32_t t = (uint32_t)((int32_t)(bits << (31 - at)) >> 31);
    return __builtin_bit_cast(float, (t & __builtin_bit_cast(uint32_t, x)) | (~t & __builtin_bit_cast(uint32_t, y)));
}

// key tiles of N rows that rows with limits from `first` to `last` see: the tiles of the sinks, then those of the window
struct Tiles {
    int sink, main0, count;   // tile n is n below sink, else main0 + n - sink
    __device__ int operator[](int n) const { return n < sink ? n : main0 + n - sink; }
};
template <int N> __device__ __forceinline__ Tiles tiles_of(const Limits &first, const Limits &last, int sinks) {
    const int end = last.hi > 0 ? (last.hi + N - 1) / N : 0, from = min(first.lo / N, end);
    Tiles t;
    t.sink = min(from, (sinks + N - 1) / N);
    t.main0 = from;
    t.count = t.sink + end - from;
    return t;
}

// Work item of a block.  Blocks go round the 8 XCDs in turn, each with its own L2.  Pinned: all blocks of a group (sequence and key
// head, which read the same keys) are on one XCD; without, groups are too few or would leave XCDs idle.  In both, the row tiles
// come last to first over all groups: with causal order the long ones start first.
struct Item {
    int group, tile, part;
};
__device__ __forceinline__ Item block_of(const AttendArgs &a, uint32_t at) {
    Item w;
    uint32_t rest;
    if (a.pinned) {
        const uint32_t g8 = (uint32_t)(a.groups + 7) >> 3, j = at >> 3;
        w.group = (int)((j % g8) * 8 + (at & 7));
        rest = j / g8;
    } else {
        w.group = (int)(at % (uint32_t)a.groups);
        rest = at / (uint32_t)a.groups;
    }
    w.tile = a.tiles - 1 - (int)(rest % (uint32_t)a.tiles);
    w.part = (int)(rest / (uint32_t)a.tiles);
    return w;
}

// ---- tiles straight from memory to LDS ----
// 16 bytes to a lane, 1 KB to an instruction, in the order of LDS: lane i's bytes go to `lds` + 16 i.  So which piece of which row a lane
// reads follows from where it has to lie (tile_at).  Written out, because the compiler, which cannot tell the tiles apart, would wait
// for the loads before every transposing read of another tile; nothing comes back in registers, and arrived() waits for them.
__device__ __forceinline__ u32x4 buffer_of(const char *p, int bytes) {   // reads past `bytes` give zeros
    const uint64_t at = (uint64_t)p;
    return (u32x4){(uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)at), (uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)(at >> 32)),
                   (uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)bytes), 0x00020000u};
}
constexpr uint32_t NOWHERE = 0x80000000u;   // an offset past every buffer, also with the rows of a tile (64 x 2^23 bytes) added to it
// What the hardware asks for and the compiler sees to in its own code, but not inside an asm: a wait state between the write of m0 and the load
// that reads it; five between a vector instruction that writes a scalar register (a v_readfirstlane for the buffer, which the compiler may
// put right before) and a memory instruction that reads it: s_mov is one, s_nop 3 four.
__device__ __forceinline__ void to_lds(u32x4 buffer, uint32_t lane_offset, uint32_t lds) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 3\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(__builtin_amdgcn_readfirstlane(lds)), "v"(lane_offset),
                 "s"(buffer) : "memory");
}
__device__ __forceinline__ void to_lds(const char *p, uint32_t lds) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(__builtin_amdgcn_readfirstlane(lds)), "v"(p) : "memory");
}
__device__ __forceinline__ void word_to_lds(const float *p, uint32_t lds) {   // 4 bytes to a lane
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, off" ::"s"(__builtin_amdgcn_readfirstlane(lds)), "v"(p) : "memory");
}
// waits until at most LEFT of the wave's loads are under way (they arrive in the order of their issue)
template <int LEFT = 0> __device__ __forceinline__ void arrived() { asm volatile("s_waitcnt vmcnt(%0)" ::"i"(LEFT) : "memory"); }
// Waits for loads that came back in registers, where the compiler sees it: it would otherwise wait at their first use inside a loop, and
// there for all loads under way, the next tiles' too
__device__ __forceinline__ void registers_loaded() { __builtin_amdgcn_s_waitcnt(0x0f70); }   // vmcnt(0)

// Tiles of N rows from two tensors (keys and values, say) with fixed strides, for a block of WAVES waves
template <class T, int DP, int N, int WAVES = 4> struct Tile2 {
    static constexpr int PIECES = DP / 8, RPI = 64 / PIECES, STEP = WAVES * RPI, COUNT = (N + STEP - 1) / STEP;   // rows to an instruction, of all waves
    uint32_t off[2];           // the lane's bytes within the wave's first instruction
    int row, piece;            // the lane's row there, its piece
    const char *base[2];       // row 0
    int stride[2];             // bytes between rows, below 2^23

    __device__ void start(const char *x, int64_t xrow, const char *y, int64_t yrow, int dim, int wave, int lane) {
        row = wave * RPI + lane / PIECES;
        piece = (lane % PIECES) ^ piece_swap<DP>(row);
        base[0] = x;
        base[1] = y;
        stride[0] = 2 * (int)xrow;
        stride[1] = 2 * (int)yrow;
#pragma unroll
        for (int w = 0; w < 2; ++w)                        // zeros where the tile is wider than the head
            off[w] = piece * 8 >= dim ? NOWHERE : (uint32_t)(row * stride[w] + piece * 16);
    }
    // rows from row0 on of one tensor; rows from `end` on give zeros
    template <int W> __device__ void issue_one(int row0, int end, int dim, const short *tile, int wave) const {
        if (N < STEP && wave * RPI >= N) return;
        const char *const at = base[W] + (int64_t)row0 * stride[W];
        const int bytes = (min(end - row0, N) - 1) * stride[W] + 2 * dim;
        const uint32_t lds = lds_address(tile) + wave * 1024;
        const u32x4 buffer = buffer_of(at, bytes);
        // the whole offset in the lane's register: that is what is checked against the buffer's bytes
#pragma unroll
        for (int c = 0; c < COUNT; ++c) to_lds(buffer, off[W] + (uint32_t)(STEP * c * stride[W]), lds + 1024 * WAVES * c);
    }
    __device__ void issue(int row0, int end, int dim, const short *tx, const short *ty, int wave) const {
        issue_one<0>(row0, end, dim, tx, wave);
        issue_one<1>(row0, end, dim, ty, wave);
    }
};
// infinities and NaN of a tile become 0; bits of the rows that had one (a wave's)
template <class T, int DP, int N, int THREADS = 256> __device__ __forceinline__ uint64_t clean_tile(short *tile, int tid) {
    constexpr int PIECES = DP / 8;
    uint64_t odd = 0;
#pragma unroll
    for (int at = tid; at < N * PIECES; at += THREADS) {
        const u32x4 w = *(const u32x4 *)(tile + 8 * at);
        if (any_odd<T>(w)) {
            *(u32x4 *)(tile + 8 * at) = cleaned<T>(w);
            odd |= 1ull << (at / PIECES);
        }
    }
    if (!__any(odd != 0)) return 0;
#pragma unroll 1
    for (int by = 32; by > 0; by >>= 1) odd |= __shfl_xor((unsigned long long)odd, by);
    return odd;
}

// 16 bytes of zeros where the tile is wider than the head
template <int DP> __device__ __forceinline__ u32x4 load_piece(const char *base, int64_t at, int piece, int dim) {
    if (piece * 8 >= dim) return (u32x4){0, 0, 0, 0};
    return *(const u32x4 *)(base + 2 * (at + piece * 8));
}

// a row of results (C layout, columns are rows of the tensor) to 16-bit values: halves exchange four values so that each lane
// stores 16 bytes; `scale` is the lane's
template <class T, int DB>
__device__ __forceinline__ void store_rows(const f32x16 (&acc)[DB], float scale, char *base, int64_t at, int dim, bool valid, int lane) {
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            uint32_t w[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) w[j] = T::pack(acc[db][8 * s + 2 * j] * scale, acc[db][8 * s + 2 * j + 1] * scale);
            auto x = __builtin_amdgcn_permlane32_swap(w[0], w[2], false, false);
            auto y = __builtin_amdgcn_permlane32_swap(w[1], w[3], false, false);
            const int d = 32 * db + 16 * s + 8 * (lane >> 5);
            if (valid && d < dim) *(u32x4 *)(base + 2 * (at + d)) = (u32x4){(uint32_t)x[0], (uint32_t)y[0], (uint32_t)x[1], (uint32_t)y[1]};
        }
}

}  // namespace f3m
