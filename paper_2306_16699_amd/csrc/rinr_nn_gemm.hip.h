// Matrix products with their epilogues.  Every product is  out[q][p] = sum_k P(p, k) Q(q, k),  q the rows of the result and p its
// columns: forward P = w, Q = x; gradient of x P = w (k its rows), Q = dz; gradient of w P = x, Q = dz (k the rows of both).
#ifndef RINR_NN_GEMM_HIP_H
#define RINR_NN_GEMM_HIP_H

#include "rinr_nn_common.hip.h"

#include <algorithm>
#include <type_traits>

namespace rinr_nn {

typedef __attribute__((address_space(3))) char lds_char;
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;

__device__ __forceinline__ f32x4 mfma(vec8<bf16> a, vec8<bf16> b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ f32x4 mfma(vec8<f16> a, vec8<f16> b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }

// What an operand is kept as: the matrix instructions' own type, 32 bits (taken as three bf16 parts), or packed
enum { kSame = 0, kFloat = 1, kPacked = 2 };

struct Side {
    const void *p;
    int64_t ld, n;                                                               // n: extent along p or q
    const uint8_t *scales;
};

struct Epilogue {
    const float *bias;
    const void *residual, *slope;                                                // slope: the result is multiplied by act'(slope)
    void *y, *z;
    const uint8_t *slope_scales;
    uint8_t *z_scales;
    int64_t ld_residual, ld_slope, ld_y, ld_z;
    Act act, slope_act;
    bool past;                                                                   // results go past the L2s
    bool z_packed, slope_packed;                                                 // z_packed: there is a z, and it is packed
};

struct GemmArgs {
    Side P, Q;
    int64_t K;
    int tiles_p, tiles_q, k_tiles, k_share;                                      // k_share: k tiles of one workgroup; gridDim.y of them cover k_tiles
    float *part;                                                                 // [gridDim.y][Q.n][P.n] where k is shared, else NULL
    bool far;                                                                    // rows too far apart for offsets in 32 bits
    Epilogue e;
};

// Eight neighbouring columns (from p on, `have` of them exist) of row q: bias, what is kept, activation, residual, slope.  Four neighbouring lanes
// have a block of 32 columns, all of them here with q and p of their own; `there`: the row exists.  What memory has to give comes first (Inputs).
template <class T> struct Inputs {
    T r[8];
    Kept<T> z;
    __device__ __forceinline__ void load(const Epilogue &e, bool there, int64_t q, int64_t p, int have) {
        if (!there || have <= 0) return;
        if (e.residual) load_raw(((const T *)e.residual + q * e.ld_residual + p), have, r, e.past);
        if (e.slope) z.load(e.slope, e.slope_scales, e.ld_slope, e.slope_packed, q, p, have);
    }
};
__device__ __forceinline__ void bias_of(const Epilogue &e, int64_t p, int have, float (&b)[8]) {
#pragma unroll
    for (int i = 0; i < 8; ++i) b[i] = 0.0f;
    if (e.bias) load_n<float, 8>(e.bias + p, have, b);
}
template <class T> __device__ __forceinline__ void finish(const Epilogue &e, const Inputs<T> &in, const float (&b)[8], bool there, int64_t q, int64_t p, int have, float (&v)[8]) {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] += b[i];
    if (e.z_packed) {
        if (have < 8) {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = i < have ? v[i] : 0.0f;
        }
        if (there) store_packed((int8_t *)e.z, e.z_scales, q, e.ld_z, p, p + have, v, e.past);
    }
    if (!there || have <= 0) return;
    if (e.z && !e.z_packed) store_n<T, 8>((T *)e.z + q * e.ld_z + p, have, v, e.past);
    act_all<T>(v, e.act);
    if (e.residual) {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] += (float)in.r[i];
    }
    if (e.slope) {
        float z[8];
        in.z.get(e.slope_packed, z);
        slope_all<T>(v, z, e.slope_act);
    }
    store_n<T, 8>((T *)e.y + q * e.ld_y + p, have, v, e.past);
}

// ---- operands in LDS and in registers ----------------------------------------------------------------------------------------------------

// One operand's tile in LDS, 16-byte groups of 8 values.  Rows of k (K_ROWS: the matrix has k as its rows): [k][WIDE], read by the
// transposing LDS read; else [WIDE][k].  Groups are exchanged within a row such that the 16 rows (or 4 x 4 rows of k) that one read takes lie in
// different banks.
template <int BK, bool K_ROWS, int WIDE> struct Tile {
    static constexpr int GROUPS = K_ROWS ? WIDE / 8 : BK / 8;                    // groups of a row
    static constexpr int ROWS = K_ROWS ? BK : WIDE;
    static constexpr int ALL = ROWS * GROUPS;
    __device__ static __forceinline__ int place(int row, int group) {            // of a group, in groups
        if (K_ROWS) return row * GROUPS + (group ^ (((row & 3) | ((row >> 1) & 4)) << 1));
        return row * GROUPS + (group ^ ((GROUPS == 8 ? row / 2 : -(row / 4)) & (GROUPS - 1)));
    }
    // The operand of a 16x16x32 step: lane l has row `at + 16 i + l % 16`, k = 32 step + 8 (l / 16) ... + 7.  `from`: what depends on the lane and
    // `at` (a multiple of 64 for i below 4, of 128 for i below 8), in bytes; i and step are constants.
    __device__ static __forceinline__ int from(int at, int lane) {
        if (K_ROWS) {
            // 16 lanes read 4 rows of k x 16 columns and get them transposed: lane i the 4 k of column i; lane 4 r + c supplies columns 4 c.. of row r
            const int k = (lane >> 4) * 8 + ((lane & 15) >> 2), c = at + (lane & 3) * 4;
            return (place(k, c >> 3) * 8 + (c & 7)) * 2;
        }
        return place(at + (lane & 15), lane >> 4) * 16;
    }
    template <class E> __device__ static __forceinline__ vec8<E> read(const E *tile, int from, int i, int step) {
        const char *const t = (const char *)tile;
        if (K_ROWS) {                                                            // 16 columns are 2 groups; the exchange is of bits 1 to 3 of a group's number
            const int at = from ^ (i << 5);
            union { s16x4 h[2]; vec8<E> v; } r;
            r.h[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(t + at + step * 32 * GROUPS * 16));
            r.h[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(t + at + (step * 32 + 4) * GROUPS * 16));
            return r.v;
        }
        // step * 4 groups on: the bit of 4 is exchanged by rows too
        return *(const vec8<E> *)(t + (GROUPS == 8 ? from ^ (step * 64) : from) + i * 16 * GROUPS * 16);
    }
};

// 8 values of an operand on the way from memory to LDS or to a matrix step.  load: part of them may lie behind an end, whole: none does (at an
// offset in bytes); split: PARTS operands that add up to them, 0 for what lies behind an end (FIX: after load).
// Nothing is read outside the matrix (whose rows, end to end, span at least 8 values) and nothing is waited for in load: a group that reaches behind the matrix's
// last value is read from 8 values before that, and put right in split; over the end of another row it reads into the next one.  (With such values read one
// by one, 16 groups of a thread waited for one after the other: 4 us a k tile.)
constexpr int kWholeGroup = 8 << 4;                                              // 16 kept + moved: the first `kept` values, `moved` places on, are the group's
template <class T> __device__ __forceinline__ int load_group(const Side &s, int64_t row, int64_t rows, int64_t col, int64_t cols, void *v) {
    const int64_t r = row < rows ? row : rows - 1, at = r * s.ld + col, last = (rows - 1) * s.ld + cols - 8, from = at < last ? at : last;
    __builtin_memcpy(v, (const T *)s.p + from, sizeof(T) * 8);
    const int64_t moved = at - from, kept = row < rows ? cols - col : 0;
    return (int)(moved < 8 ? moved : 8) | (int)(kept < 0 ? 0 : (kept < 8 ? kept : 8)) << 4;
}
// N words of 8 values: WORDS each
template <int N> __device__ __forceinline__ void fix_group(uint32_t (&d)[N], int fix) {
    const int moved = fix & 15, kept = fix >> 4;
#pragma unroll
    for (int step = N; step >= N / 4; step /= 2)                                 // 8, 4 and 2 values of 16 bits, 8, 4, 2 of 32
        if (moved & (8 * step / N)) {
#pragma unroll
            for (int i = 0; i < N; ++i) d[i] = i + step < N ? d[i + step] : 0u;
        }
    if (moved & 1) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const uint32_t up = i + 1 < N ? d[i + 1] : 0u;
            d[i] = N == 8 ? up : __builtin_amdgcn_alignbit(up, d[i], 16);
        }
    }
#pragma unroll
    for (int i = 0; i < N; ++i) {
        if (N == 8) d[i] = i < kept ? d[i] : 0u;
        else d[i] = 2 * i + 1 < kept ? d[i] : (2 * i < kept ? d[i] & 0xffffu : 0u);
    }
}
template <class E, int SRC> struct Group;
template <class E> struct Group<E, kSame> {
    static constexpr int BYTES = 2;
    uint32_t d[4];
    int fix;
    __device__ __forceinline__ void load(const Side &s, int64_t row, int64_t rows, int64_t col, int64_t cols) { fix = load_group<E>(s, row, rows, col, cols, d); }
    __device__ __forceinline__ void whole(const char *p, uint32_t at, const uint8_t * = nullptr) {
        __builtin_memcpy(d, p + at, 16);
        fix = kWholeGroup;
    }
    template <int PARTS, bool FIX> __device__ __forceinline__ void split(vec8<E> (&o)[PARTS]) {
        static_assert(PARTS == 1, "");
        if (FIX && fix != kWholeGroup) fix_group(d, fix);
        __builtin_memcpy(&o[0], d, 16);
    }
};
template <class E> struct Group<E, kPacked> {
    static constexpr int BYTES = 1;
    uint32_t w[2], byte;
    bool there;
    __device__ __forceinline__ void whole(const char *p, uint32_t at, const uint8_t *scales) {
        __builtin_memcpy(w, p + at, 8);
        byte = scales[at / kBlock8];                                             // p is a block's beginning, ld a multiple of 32
        there = true;
    }
    __device__ __forceinline__ void load(const Side &s, int64_t row, int64_t rows, int64_t col, int64_t cols) {
        const int64_t end = (cols + kBlock8 - 1) / kBlock8 * kBlock8;            // whole blocks are there, zeros behind the last column
        there = row < rows && col < end;
        const int64_t r = row < rows ? row : rows - 1, c = col < end ? col : end - 8;
        __builtin_memcpy(w, (const int8_t *)s.p + r * s.ld + c, 8);
        byte = s.scales[r * (s.ld / kBlock8) + c / kBlock8];
    }
    template <int PARTS, bool FIX> __device__ __forceinline__ void split(vec8<E> (&o)[PARTS]) {
        const float sc = scale_of(there ? byte : 0u);
        float f[8];
        values_of(there ? w[0] : 0u, sc, f);
        values_of(there ? w[1] : 0u, sc, f + 4);
        in_range<E>(there ? byte : 0u, f);
#pragma unroll
        for (int i = 0; i < 8; ++i) o[0][i] = (E)f[i];
#pragma unroll
        for (int n = 1; n < PARTS; ++n) o[n] = vec8<E>{};                        // 7 bits: the first part is all of it
    }
};
template <class E> struct Group<E, kFloat> {
    static constexpr int BYTES = 4;
    uint32_t d[8];
    int fix;
    __device__ __forceinline__ void load(const Side &s, int64_t row, int64_t rows, int64_t col, int64_t cols) { fix = load_group<float>(s, row, rows, col, cols, d); }
    __device__ __forceinline__ void whole(const char *p, uint32_t at, const uint8_t * = nullptr) {
        __builtin_memcpy(d, p + at, 32);
        fix = kWholeGroup;
    }
    // x = hi + mid + lo exactly, each the first 8 significant bits of what is left (of an infinity or a NaN a NaN is left)
    template <int PARTS, bool FIX> __device__ __forceinline__ void split(vec8<E> (&o)[PARTS]) {
        static_assert(PARTS == 3, "");
        if (FIX && fix != kWholeGroup) fix_group(d, fix);
        uint32_t part[3][4];
#pragma unroll
        for (int i = 0; i < 8; i += 2) {
            uint32_t b[3][2];
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                b[0][j] = d[i + j];
                const float r1 = __uint_as_float(b[0][j]) - __uint_as_float(b[0][j] & 0xffff0000u);
                b[1][j] = __float_as_uint(r1);
                b[2][j] = __float_as_uint(r1 - __uint_as_float(b[1][j] & 0xffff0000u));
            }
#pragma unroll
            for (int n = 0; n < 3; ++n) part[n][i / 2] = __builtin_amdgcn_perm(b[n][1], b[n][0], 0x07060302u);
        }
#pragma unroll
        for (int n = 0; n < 3; ++n) __builtin_memcpy(&o[n], part[n], 16);
    }
};
template <class E, int PARTS, bool FIX, class G> __device__ __forceinline__ void put_group(G &g, E *tile, int place, int apart) {
    vec8<E> o[PARTS];
    g.template split<PARTS, FIX>(o);
#pragma unroll
    for (int n = 0; n < PARTS; ++n) *(vec8<E> *)(tile + n * apart + place * 8) = o[n];
}
// a b, of operands in parts, added to c; small terms first
template <class E> __device__ __forceinline__ f32x4 product_of(const vec8<E> (&a)[1], const vec8<E> (&b)[1], f32x4 c) { return mfma(a[0], b[0], c); }
template <class E> __device__ __forceinline__ f32x4 product_of(const vec8<E> (&a)[3], const vec8<E> (&b)[3], f32x4 c) {
    c = mfma(a[2], b[0], c);
    c = mfma(a[0], b[2], c);
    c = mfma(a[1], b[1], c);
    c = mfma(a[1], b[0], c);
    c = mfma(a[0], b[1], c);
    return mfma(a[0], b[0], c);
}

template <int NI, int AT_ONCE> constexpr int pass_floats() { return NI * AT_ONCE * 256; }    // LDS of a wavefront's results on their way out
constexpr int kTile = 128, kTileThreads = 256, kTileK = 32, kTileLds = std::max(2 * 3 * kTile * kTileK * 2, 4 * pass_floats<4, 4>() * 4);

// Workgroups are handed to the 8 XCDs in turn; each XCD takes a run of neighbouring tiles, so that its L2 holds what they share.  Within the
// run 8 rows of tiles are walked column by column.
__device__ __forceinline__ void tile_of(int id, int tiles_p, int tiles_q, int &tp, int &tq) {
    const int n = tiles_p * tiles_q, each = n / 8, more = n % 8, xcd = id % 8, at = id / 8;
    const int i = xcd * each + (xcd < more ? xcd : more) + at;
    const int band = i / (8 * tiles_p), in = i - band * 8 * tiles_p, high = tiles_q - band * 8 < 8 ? tiles_q - band * 8 : 8;
    tq = band * 8 + in % high;
    tp = in / high;
}

// What a wavefront holds of the result, NI x NJ steps of 16 columns (from p0, a multiple of 32) x 16 rows (from q0): lane l the rows l % 16 and, of each
// step's columns, the four from 4 (l / 16) on.  It goes through LDS of the wavefront's own, AT_ONCE steps of rows at a time, so that a lane then has 8
// neighbouring columns, and memory is read and written in runs of whole rows.  16-byte groups are exchanged within a row by its number: what 16 lanes
// write at once lies in different banks.
template <class T, int NI, int NJ, int AT_ONCE> __device__ __forceinline__ void write_tile(const GemmArgs &a, int64_t p0, int64_t q0, int lane, float *lds, const f32x4 (&acc)[NI][NJ]) {
    constexpr int COLS = NI * 16, LANES = COLS / 8, ROWS = 64 / LANES;
    static_assert(NI >= 4, "16 groups of a row");
    const int col = lane % LANES * 8;
    const int64_t p = p0 + col;
    const int have = (int)(a.P.n - p < 8 ? a.P.n - p : 8);
    float bias[8];
    bias_of(a.e, p, have, bias);
#pragma unroll
    for (int j0 = 0; j0 < NJ; j0 += AT_ONCE) {
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int j = 0; j < AT_ONCE; ++j)
#pragma unroll
            for (int i = 0; i < NI; ++i) {
                const int row = j * 16 + (lane & 15);
                *(f32x4 *)(lds + row * COLS + ((i * 4 + (lane >> 4)) ^ (row & 15)) * 4) = acc[i][j0 + j];
            }
        __builtin_amdgcn_wave_barrier();                                         // a wavefront's LDS accesses are carried out in order
        constexpr int AHEAD = 4;                                                 // rows whose inputs are under way together
        static_assert(AT_ONCE * 16 % (ROWS * AHEAD) == 0, "");
#pragma unroll 1
        for (int r0 = 0; r0 < AT_ONCE * 16; r0 += ROWS * AHEAD) {
            Inputs<T> in[AHEAD];
            if (a.e.residual || a.e.slope) {
#pragma unroll
                for (int u = 0; u < AHEAD; ++u) {
                    const int64_t q = q0 + j0 * 16 + r0 + u * ROWS + lane / LANES;
                    in[u].load(a.e, q < a.Q.n, q, p, have);
                }
            }
#pragma unroll
            for (int u = 0; u < AHEAD; ++u) {
                const int row = r0 + u * ROWS + lane / LANES;
                const f32x4 lo = *(const f32x4 *)(lds + row * COLS + ((col / 4) ^ (row & 15)) * 4), hi = *(const f32x4 *)(lds + row * COLS + ((col / 4 + 1) ^ (row & 15)) * 4);
                float v[8] = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
                const int64_t q = q0 + j0 * 16 + row;
                if (a.part) {
                    if (q < a.Q.n) store_n<float, 8>(a.part + ((int64_t)blockIdx.y * a.Q.n + q) * a.P.n + p, have, v);
                } else {
                    finish<T>(a.e, in[u], bias, q < a.Q.n, q, p, have, v);
                }
            }
        }
    }
}

// ---- operands on their way to LDS ------------------------------------------------------------------------------------------------------

// 16 bytes a lane from base + at straight to LDS, a wavefront's 1024 bytes in a row.  Written as one block so that the compiler, which cannot tell
// the LDS buffers apart, does not wait for it before it reads another one: barrier_with does.  What it writes, m0 and LDS, is named: nothing is kept in m0 and no access of
// LDS is moved across it.
typedef int i32x4 __attribute__((ext_vector_type(4)));
__device__ __forceinline__ void direct_16(const i32x4 base, uint32_t at, uint32_t lds_at) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(lds_at), "v"(at), "s"(base) : "m0", "memory");
}
// A barrier behind all but the last N of this wavefront's loads and all of its LDS accesses
template <int N> __device__ __forceinline__ void barrier_with() { asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(N) : "memory"); }

// One side's way from memory to LDS.  kAsync: straight, where rows begin on 4 bytes; the exchange of groups is then made in the addresses that are
// read.  Rows (groups of columns, where k is rows) behind the matrix's end repeat its last: what they give is not stored.  The last k tile, where it is
// not whole, and other matrices go through registers (kSame, kFloat; kFar: rows too far apart for offsets in 32 bits).
enum { kAsync = 3, kFar = 4 };
template <class E, int MODE, bool K_ROWS, int WIDE, int BK, int THREADS> struct Feed {
    typedef Tile<BK, K_ROWS, WIDE> TT;
    static constexpr int NG = WIDE * BK / 8 / THREADS;
        static constexpr int DIRECT = MODE == kAsync ? NG : 0;                       // loads under way for each k tile
    typedef Group<E, MODE == kFloat ? kFloat : kSame> G;
    static constexpr int PARTS = MODE == kFloat ? 3 : 1;
    uint32_t at[NG];                                                             // byte offsets of this lane's groups from the tile's first element

    __device__ __forceinline__ void begin(const Side &s, int64_t n0) {
#pragma unroll
        for (int i = 0; i < NG; ++i) {
            const int place = i * THREADS + threadIdx.x, row = place / TT::GROUPS;
            int group = place % TT::GROUPS;
            if (MODE == kAsync) group = TT::place(row, group) % TT::GROUPS;      // the exchange is its own inverse
            int64_t col = group * 8, r = row;
            if (K_ROWS) {
                const int64_t last = (s.n - 1) / 8 * 8 - n0;
                col = col < last ? col : last;
            } else {
                const int64_t last = s.n - 1 - n0;
                r = r < last ? r : last;
            }
            at[i] = (uint32_t)(r * s.ld + col) * (uint32_t)G::BYTES;
        }
    }
    // k tiles that can be read without looking at each group: whole ones, and where a row's last group reaches over its end, without the last rows, from
    // which that would be over the matrix's
    __device__ static __forceinline__ int whole_tiles(const Side &s, int64_t K) {
        if (MODE == kFar) return 0;
        const int64_t over = K_ROWS ? (s.n + 7) / 8 * 8 - s.n : 0, rows = over ? (over + s.ld - 1) / s.ld : 0;
        return K > rows ? (int)((K - rows) / BK) : 0;
    }
    __device__ __forceinline__ void whole(G (&g)[NG], const Side &s, int64_t n0, int kt) const {
        const int64_t k0 = (int64_t)kt * BK, row = K_ROWS ? k0 : n0, col = K_ROWS ? n0 : k0;
        const char *const p = (const char *)s.p + (row * s.ld + col) * G::BYTES;
#pragma unroll
        for (int i = 0; i < NG; ++i) g[i].whole(p, at[i]);
    }
    // A whole k tile on its way to `tile`, a piece at a time
    struct Way {
        i32x4 from;
        uint32_t to;
    };
    __device__ __forceinline__ Way way(const Side &s, int64_t n0, int kt, E *tile) const {
        const int64_t k0 = (int64_t)kt * BK;
        const uintptr_t base = (uintptr_t)((const E *)s.p + (K_ROWS ? k0 * s.ld + n0 : n0 * s.ld + k0));
        return {{__builtin_amdgcn_readfirstlane((int)base), __builtin_amdgcn_readfirstlane((int)(base >> 32) & 0xffff), 0x7fffffff, 0x00020000},
                (uint32_t)__builtin_amdgcn_readfirstlane((int)((uint32_t)(uintptr_t)(lds_char *)tile + (threadIdx.x >> 6) * 1024u))};
    }
    __device__ __forceinline__ void piece(const Way &w, int i) const { direct_16(w.from, at[i], w.to + i * THREADS * 16u); }
    __device__ __forceinline__ void load(G (&g)[NG], const Side &s, int64_t n0, int kt, E *tile) const {
        if (MODE != kAsync) {
            whole(g, s, n0, kt);
        } else {
            const Way w = way(s, n0, kt, tile);
#pragma unroll
            for (int i = 0; i < NG; ++i) piece(w, i);
        }
    }
    __device__ __forceinline__ void store(G (&g)[NG], E *tile) const {
        if (MODE != kAsync) put<false>(g, tile);
    }
    __device__ static __forceinline__ void guarded(G (&g)[NG], const Side &s, int64_t n0, int64_t K, int kt) {
        const int64_t k0 = (int64_t)kt * BK;
#pragma unroll
        for (int i = 0; i < NG; ++i) {
            const int place = i * THREADS + threadIdx.x, row = place / TT::GROUPS, col = place % TT::GROUPS * 8;
            if (K_ROWS) g[i].load(s, k0 + row, K, n0 + col, s.n);
            else g[i].load(s, n0 + row, s.n, k0 + col, K);
        }
    }
    template <bool FIX> __device__ static __forceinline__ void put(G (&g)[NG], E *tile) {
#pragma unroll
        for (int i = 0; i < NG; ++i) {
            const int place = i * THREADS + threadIdx.x;
            put_group<E, PARTS, FIX>(g[i], tile, TT::place(place / TT::GROUPS, place % TT::GROUPS), WIDE * BK);
        }
    }
};

// ---- tiles of 128 x 128 for 32-bit operands ----------------------------------------------------------------------------------------------

// Each operand as three bf16 parts.  4 wavefronts of 64 x 64, k staged through registers into one LDS buffer, so that two workgroups share a CU: what the
// next k tile needs is under way while this one's matrix steps run.  (Two buffers, one workgroup a CU and the split between the matrix steps: 50176 x
// 256 x 256 in 94 us, not 59.)  That product takes 55 us, with a sine: 784 tiles on 512 places are 1.53 rounds that cost two, and by its counters matrix pipes are 35 % busy,
// vector instructions (split, addresses, sine) 44 %, LDS 10 %: the two workgroups of a CU overlap little of these phases.
template <bool KP, bool KQ> __global__ __launch_bounds__(kTileThreads) __attribute__((amdgpu_waves_per_eu(2, 2))) void gemm_kernel(const GemmArgs a) {
    typedef bf16 E;
    constexpr int BK = kTileK, PARTS = 3, PLANE = kTile * BK, SIDE = PLANE * PARTS;
    typedef Feed<E, kFloat, KP, kTile, BK, kTileThreads> FP;
    typedef Feed<E, kFloat, KQ, kTile, BK, kTileThreads> FQ;
    typedef typename FP::TT TP;
    typedef typename FQ::TT TQ;
    extern __shared__ char lds[];
    E *const base = (E *)lds;
    int tp, tq;
    tile_of(blockIdx.x, a.tiles_p, a.tiles_q, tp, tq);
    const int64_t p0 = (int64_t)tp * kTile, q0 = (int64_t)tq * kTile;
    const int k_from = blockIdx.y * a.k_share, k_to = k_from + a.k_share < a.k_tiles ? k_from + a.k_share : a.k_tiles;
    const int whole = a.far ? 0 : std::min(FP::whole_tiles(a.P, a.K), FQ::whole_tiles(a.Q, a.K));
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, wp = (wave & 1) * 64, wq = (wave >> 1) * 64;
    const int from_p = TP::from(wp, lane), from_q = TQ::from(wq, lane);
    FP fp;
    FQ fq;
    fp.begin(a.P, p0);
    fq.begin(a.Q, q0);
    typename FP::G gp[FP::NG];
    typename FQ::G gq[FQ::NG];

    auto load = [&](int kt) {
        if (kt < whole) {
            fp.whole(gp, a.P, p0, kt);
            fq.whole(gq, a.Q, q0, kt);
        } else {
            FP::guarded(gp, a.P, p0, a.K, kt);
            FQ::guarded(gq, a.Q, q0, a.K, kt);
        }
    };
    auto store = [&](int kt) {
        if (kt < whole) {
            FP::template put<false>(gp, base);
            FQ::template put<false>(gq, base + SIDE);
        } else {
            FP::template put<true>(gp, base);
            FQ::template put<true>(gq, base + SIDE);
        }
    };

    f32x4 acc[4][4] = {};
    load(k_from);
    store(k_from);
    for (int kt = k_from; kt < k_to; ++kt) {
        __syncthreads();                                                         // this tile is in LDS
        const bool more = kt + 1 < k_to;
        if (more) load(kt + 1);
#pragma unroll
        for (int s = 0; s < BK / 32; ++s) {
            vec8<E> vp[4][PARTS], vq[4][PARTS];
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int n = 0; n < PARTS; ++n) {
                    vp[i][n] = TP::template read<E>(base + n * PLANE, from_p, i, s);
                    vq[i][n] = TQ::template read<E>(base + SIDE + n * PLANE, from_q, i, s);
                }
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) acc[i][j] = product_of<E>(vp[i], vq[j], acc[i][j]);
        }
        __syncthreads();                                                         // it has been read
        if (more) store(kt + 1);
    }
    write_tile<float, 4, 4, 4>(a, p0 + wp, q0 + wq, lane, (float *)lds + wave * pass_floats<4, 4>(), acc);
}

// ---- large tiles for 16-bit operands ---------------------------------------------------------------------------------------------------

// WIDE_P columns x WIDE_Q rows of the result, a wavefront NI x NJ steps of 16 x 16 of them, two buffers of 64 values of k.
template <int WIDE_P_, int WIDE_Q_, int NI_, int NJ_> struct WideShape {
    static constexpr int WIDE_P = WIDE_P_, WIDE_Q = WIDE_Q_, NI = NI_, NJ = NJ_, BK = 64;
    static constexpr int WAVES_P = WIDE_P / (NI * 16), WAVES = WAVES_P * (WIDE_Q / (NJ * 16)), THREADS = WAVES * 64;
    static constexpr int STAGE = (WIDE_P + WIDE_Q) * BK;                         // values
    static constexpr int AT_ONCE = 2;                                            // steps of rows that the epilogue takes at a time
    static constexpr int OUT = pass_floats<NI, AT_ONCE>();
    static constexpr int LDS = std::max(2 * STAGE * 2, WAVES * OUT * 4);
};

// A k tile is two steps of 32.  The first step's matrix instructions run while the second's operands are read from LDS.  Then the tile's buffer is
// done with: a barrier in the middle of the second step, behind which the next tile is there, its first operands are read, and the one after it is
// sent for into the freed buffer; so matrix instructions go on across the tiles' bounds.  Reads and requests come one or two at a time between matrix
// instructions: memory and LDS take an instruction of a wavefront only so often, and what waits for them holds up what is behind it.
// 256 x 256 tiles are what L2 and LDS bandwidth allow (each value from LDS is used by 64 or 128 others, each from L2 by 256); 8 wavefronts, two a SIMD,
// hide each other's waits.  Bound by the matrix pipe in the loop (66 % busy at 4096 values of k, at the card's power limit) and by what a tile's start and
// results take, 9 to 11 us that nothing overlaps: 32768 rows in bf16, 4096 -> 4096 784 us (1403 TFLOP/s, 1.39 us a k tile), 1024 -> 4096 248 (1108), with GELU 299, and z
// in 8 bits 329.
template <class E, class S, int MP, bool KP, int MQ, bool KQ> __global__ __launch_bounds__(S::THREADS) __attribute__((amdgpu_waves_per_eu(2, 2))) void wide_kernel(const GemmArgs a) {
    constexpr int BK = S::BK, NI = S::NI, NJ = S::NJ;
    static_assert(NI >= NJ, "");
    typedef Feed<E, MP, KP, S::WIDE_P, BK, S::THREADS> FP;
    typedef Feed<E, MQ, KQ, S::WIDE_Q, BK, S::THREADS> FQ;
    typedef typename FP::TT TP;
    typedef typename FQ::TT TQ;
    constexpr int SIDE = S::WIDE_P * BK;
    extern __shared__ char lds[];
    E *const base = (E *)lds;
    int tp, tq;
    tile_of(blockIdx.x, a.tiles_p, a.tiles_q, tp, tq);
    const int64_t p0 = (int64_t)tp * S::WIDE_P, q0 = (int64_t)tq * S::WIDE_Q;
    const int k_from = blockIdx.y * a.k_share, k_to = k_from + a.k_share < a.k_tiles ? k_from + a.k_share : a.k_tiles;
    const int whole = std::min({FP::whole_tiles(a.P, a.K), FQ::whole_tiles(a.Q, a.K), k_to});
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, wp = wave % S::WAVES_P * (NI * 16), wq = wave / S::WAVES_P * (NJ * 16);
    FP fp;
    FQ fq;
    fp.begin(a.P, p0);
    fq.begin(a.Q, q0);
    const int from_p = TP::from(wp, lane), from_q = TQ::from(wq, lane);
    f32x4 acc[NI][NJ] = {};
    vec8<E> vp[2][NI], vq[2][NJ];
    auto read = [&](const E *tile, int step, int i) {                            // the i-th operands of a step
        if (i < NJ) vq[step][i] = TQ::template read<E>(tile + SIDE, from_q, i, step);
        vp[step][i] = TP::template read<E>(tile, from_p, i, step);
    };
    auto steps = [&](int step, int i) {
#pragma unroll
        for (int j = 0; j < NJ; ++j) acc[i][j] = mfma(vp[step][i], vq[step][j], acc[i][j]);
    };
    if (k_from < whole) {
        {
            typename FP::G gp[FP::NG];
            typename FQ::G gq[FQ::NG];
            fp.load(gp, a.P, p0, k_from, base);
            fq.load(gq, a.Q, q0, k_from, base + SIDE);
            fp.store(gp, base);
            fq.store(gq, base + SIDE);
            barrier_with<0>();
            if (k_from + 1 < whole) {
                fp.load(gp, a.P, p0, k_from + 1, base + S::STAGE);
                fq.load(gq, a.Q, q0, k_from + 1, base + S::STAGE + SIDE);
                fp.store(gp, base + S::STAGE);
                fq.store(gq, base + S::STAGE + SIDE);
            }
        }
#pragma unroll
        for (int j = 0; j < NJ; ++j) vq[0][j] = TQ::template read<E>(base + SIDE, from_q, j, 0);
#pragma unroll
        for (int i = 0; i < NI; ++i) vp[0][i] = TP::template read<E>(base, from_p, i, 0);
        int kt = k_from;
        // next: there is another whole tile; more: and one after that
        auto turn = [&](auto next, auto more) {
            E *const tile = base + ((kt - k_from) & 1) * S::STAGE, *const other = base + ((kt - k_from + 1) & 1) * S::STAGE;
            typename FP::G gp[FP::NG];
            typename FQ::G gq[FQ::NG];
            if (more) {
                if (MP != kAsync) fp.whole(gp, a.P, p0, kt + 2);
                if (MQ != kAsync) fq.whole(gq, a.Q, q0, kt + 2);
            }
#pragma unroll
            for (int i = 0; i < NI; ++i) {
                __builtin_amdgcn_sched_barrier(0);
                read(tile, 1, i);
                steps(0, i);
            }
            constexpr int BAR = NI / 4, SLOTS = NI - BAR, READS = SLOTS - 1, ALL = FP::DIRECT + FQ::DIRECT;
            const typename FP::Way way_p = fp.way(a.P, p0, kt + 2, tile);
            const typename FQ::Way way_q = fq.way(a.Q, q0, kt + 2, tile + SIDE);
#pragma unroll
            for (int i = 0; i < NI; ++i) {
                __builtin_amdgcn_sched_barrier(0);
                if (next && i == BAR) barrier_with<0>();
                if (more && i >= BAR) {
#pragma unroll
                    for (int n = (i - BAR) * ALL / SLOTS; n < (i - BAR + 1) * ALL / SLOTS; ++n) {
                        if (n < FP::DIRECT) fp.piece(way_p, n);
                        else fq.piece(way_q, n - FP::DIRECT);
                    }
                }
                if (next && i >= BAR && i < BAR + READS) {
#pragma unroll
                    for (int n = (i - BAR) * NI / READS; n < (i - BAR + 1) * NI / READS; ++n) read(other, 0, n);
                }
                steps(1, i);
            }
            __builtin_amdgcn_sched_barrier(0);
            if (more) {
                fp.store(gp, tile);
                fq.store(gq, tile + SIDE);
            }
            ++kt;
        };
        while (kt + 2 < whole) turn(std::true_type(), std::true_type());
        if (kt + 1 < whole) turn(std::true_type(), std::false_type());
        turn(std::false_type(), std::false_type());
    }
    __syncthreads();
    for (int kt = whole > k_from ? whole : k_from; kt < k_to; ++kt) {            // k tiles that are not whole
        typename FP::G gp[FP::NG];
        typename FQ::G gq[FQ::NG];
        FP::guarded(gp, a.P, p0, a.K, kt);
        FQ::guarded(gq, a.Q, q0, a.K, kt);
        FP::template put<true>(gp, base);
        FQ::template put<true>(gq, base + SIDE);
        __syncthreads();
#pragma unroll
        for (int step = 0; step < 2; ++step) {
#pragma unroll
            for (int i = 0; i < NI; ++i) read(base, step, i);
#pragma unroll
            for (int i = 0; i < NI; ++i) steps(step, i);
        }
        __syncthreads();
    }
    write_tile<E, NI, NJ, S::AT_ONCE>(a, p0 + wp, q0 + wq, lane, (float *)lds + wave * S::OUT, acc);
}

// ---- few rows ----------------------------------------------------------------------------------------------------------------------------

// 16 NJ rows of the result against 16 columns a workgroup, both operands with k side by side and straight from memory to the matrix steps: the
// weights are read once (by each 16 NJ rows), by the whole GPU at once, and that is what the time goes to.  8 wavefronts share k in blocks of 64 (a lane
// has 16 neighbouring values of it, so that 4 lanes read 128 bytes of a row) and add up through LDS.  Bound by a launch and two latencies (1 x 1024 ->
// 4096 in bf16 4.4 us, 64 x 1024 -> 1000 5.1), for large weights by memory: 16 x 4096 -> 4096 10.8 us, 3.1 TB/s.
constexpr int kFewWaves = 8, kFewBlock = 64, kFewColumns = 16;
template <class T, class E, int PARTS, int SP, int SQ, int NJ> __global__ __launch_bounds__(kFewWaves * 64) void few_kernel(const GemmArgs a) {
    constexpr int AHEAD = NJ * PARTS <= 3 ? 4 : NJ * PARTS <= 6 ? 2 : 1, LD = 20;                              // blocks whose loads are under way together; a row of sums in LDS
    __shared__ float sums[kFewWaves][NJ * 16 * LD];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t p0 = (int64_t)(blockIdx.x % a.tiles_p) * kFewColumns, q0 = (int64_t)(blockIdx.x / a.tiles_p) * (NJ * 16);
    const int from = blockIdx.y * a.k_share, to = from + a.k_share < a.k_tiles ? from + a.k_share : a.k_tiles;
    f32x4 acc[NJ] = {};
    // Whole blocks: offsets from the tile's first row, which rows behind the end share with the last
    typedef Group<E, SP> GP;
    typedef Group<E, SQ> GQ;
    const int whole = a.far ? 0 : (int)(a.K / kFewBlock), k_lane = (lane >> 4) * 16;
    const int64_t last_p = a.P.n - 1 - p0, last_q = a.Q.n - 1 - q0;
    const uint32_t at_p = (uint32_t)(((lane & 15) < last_p ? (lane & 15) : last_p) * a.P.ld + k_lane) * GP::BYTES;
    uint32_t at_q[NJ];
#pragma unroll
    for (int j = 0; j < NJ; ++j) at_q[j] = (uint32_t)((j * 16 + (lane & 15) < last_q ? j * 16 + (lane & 15) : last_q) * a.Q.ld + k_lane) * GQ::BYTES;
    for (int b = from + wave; b < to; b += kFewWaves * AHEAD) {
        GP gp[AHEAD][2];
        GQ gq[AHEAD][2][NJ];
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
            const int block = b + u * kFewWaves;
            if (block < whole && block < to) {
                const int64_t k0 = (int64_t)block * kFewBlock;
                const char *const pp = (const char *)a.P.p + (p0 * a.P.ld + k0) * GP::BYTES, *const pq = (const char *)a.Q.p + (q0 * a.Q.ld + k0) * GQ::BYTES;
                const uint8_t *const sq = SQ == kPacked ? a.Q.scales + (q0 * a.Q.ld + k0) / kBlock8 : nullptr;
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    gp[u][h].whole(pp, at_p + h * 8 * GP::BYTES, nullptr);
#pragma unroll
                    for (int j = 0; j < NJ; ++j) gq[u][h][j].whole(pq, at_q[j] + h * 8 * GQ::BYTES, sq);
                }
            } else if (block < to) {
                const int64_t k = (int64_t)block * kFewBlock + k_lane;
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    gp[u][h].load(a.P, p0 + (lane & 15), a.P.n, k + h * 8, a.K);
#pragma unroll
                    for (int j = 0; j < NJ; ++j) gq[u][h][j].load(a.Q, q0 + j * 16 + (lane & 15), a.Q.n, k + h * 8, a.K);
                }
            }
        }
#pragma unroll
        for (int u = 0; u < AHEAD; ++u)
            if (b + u * kFewWaves < to) {
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    vec8<E> vp[PARTS], vq[PARTS];
                    gp[u][h].template split<PARTS, true>(vp);
#pragma unroll
                    for (int j = 0; j < NJ; ++j) {
                        gq[u][h][j].template split<PARTS, true>(vq);
                        acc[j] = product_of<E>(vp, vq, acc[j]);
                    }
                }
            }
    }
#pragma unroll
    for (int j = 0; j < NJ; ++j) *(f32x4 *)&sums[wave][(j * 16 + (lane & 15)) * LD + (lane >> 4) * 4] = acc[j];
    __syncthreads();
    const int row = threadIdx.x >> 1, col = (threadIdx.x & 1) * 8;
    const int64_t q = q0 + row, p = p0 + col;
    const int have = (int)(a.P.n - p < 8 ? a.P.n - p : 8);
    if (row >= NJ * 16 || q >= a.Q.n || have <= 0) return;
    float v[8] = {};
#pragma unroll
    for (int w = 0; w < kFewWaves; ++w)
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] += sums[w][row * LD + col + i];
    if (a.part) store_n<float, 8>(a.part + ((int64_t)blockIdx.y * a.Q.n + q) * a.P.n + p, have, v);
    else {
        float bias[8];
        Inputs<T> in;
        bias_of(a.e, p, have, bias);
        in.load(a.e, true, q, p, have);
        finish<T>(a.e, in, bias, true, q, p, have, v);
    }
}

// ---- operands of fewer than 8 values ------------------------------------------------------------------------------------------------------

// k is below 8 then: 8 columns of a row a thread, value by value.  Bound by what the results take to write.
template <class T> struct TinySide {
    const Side &s;
    bool k_rows, packed;
    __device__ __forceinline__ float at(int64_t n, int64_t k) const {
        const int64_t row = k_rows ? k : n, col = k_rows ? n : k;
        if (!packed) return (float)((const T *)s.p)[row * s.ld + col];
        const uint32_t byte = s.scales[row * (s.ld / kBlock8) + col / kBlock8];
        float v[1] = {(float)((const int8_t *)s.p)[row * s.ld + col] * scale_of(byte)};
        in_range<T>(byte, v);
        return v[0];
    }
};
template <class T> __global__ __launch_bounds__(256) void tiny_kernel(const GemmArgs a, int64_t tasks, bool kp, bool kq, bool p_packed, bool q_packed) {
    const int64_t per_row = (a.P.n + kBlock8 - 1) / kBlock8 * 4, at = block_of() * 256 + threadIdx.x;
    if (at >= tasks) return;                                                     // of all 4 threads of a block
    const int64_t q = at / per_row, p = (at - q * per_row) * 8;
    const int have = (int)(a.P.n - p < 8 ? a.P.n - p : 8);
    const TinySide<T> P{a.P, kp, p_packed}, Q{a.Q, kq, q_packed};
    float v[8] = {}, bias[8];
    for (int64_t k = 0; k < a.K; ++k) {
        const float x = Q.at(q, k);
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < have) v[i] = __builtin_fmaf(P.at(p + i, k), x, v[i]);
    }
    Inputs<T> in;
    bias_of(a.e, p, have, bias);
    in.load(a.e, true, q, p, have);
    finish<T>(a.e, in, bias, true, q, p, have, v);
}

// What shares of k add up to, in their order: 8 columns a thread.  Bound by memory and a launch: 512 x 2048 in four shares 4 us.
template <class T> __global__ __launch_bounds__(256) void join_kernel(const float *part, int shares, int64_t nq, int64_t np, const Epilogue e) {
    const int64_t per_row = (np + kBlock8 - 1) / kBlock8 * 4;
    const int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const int64_t q = at / per_row, p = (at - q * per_row) * 8;
    if (q >= nq) return;                                                         // of all 4 threads of a block
    const int have = (int)(np - p < 8 ? np - p : 8);
    float v[8] = {};
    for (int s0 = 0; s0 < shares; s0 += 4) {                                     // four shares' loads are under way together
        float o[4][8];
#pragma unroll
        for (int u = 0; u < 4; ++u) load_n<float, 8>(part + ((int64_t)(s0 + u < shares ? s0 + u : s0) * nq + q) * np + p, s0 + u < shares ? have : 0, o[u]);
#pragma unroll
        for (int u = 0; u < 4; ++u)
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] += o[u][i];
    }
    float bias[8];
    Inputs<T> in;
    bias_of(e, p, have, bias);
    in.load(e, true, q, p, have);
    finish<T>(e, in, bias, true, q, p, have, v);
}

}  // namespace rinr_nn
#endif
