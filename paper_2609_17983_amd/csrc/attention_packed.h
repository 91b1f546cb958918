#pragma once
// Grouped-query attention of a set of rows over packed caches (packed.h).
//
// A query row at position p sees slots 0 .. p of its document (p = -1: none; its
// output is zero).  The rows of a document times the G = Hq/Hkv query heads of a kv
// head are the columns of the products, 16 to a matrix tile, so a single token
// brings G columns to one tile.
//
// A code is an integer that bf16 holds exactly (in 4 bits 16 + code, whose bits are
// the code's under a fixed exponent; in 8 bits the code), so the products run on
// the bf16 matrix units over the codes themselves.  With a key's values m + s c per
// group of 64 dimensions,
//   q . k = sum over groups of s (Q . C) + m sum(Q),
// one accumulator per group, which starts at -16 sum(Q) in 4 bits to take the codes'
// offset out.  For the output, p v = (p s) c + p m: the scale multiplies the
// probability on its way into the operand, and p m (with the offset: p (m - 16 s))
// is a sum per group and column, added to the output once, at the end.  fp32 models
// take the codes less half their range (c - 8, c - 128) and the groups' middles
// m + 8 s, m + 128 s: the products then have no common part to cancel, which cost
// two bits (an output's error against 64 bits 1.8e-6; so 0.3e-6 to 0.6e-6, the same
// attention in plain fp32 0.4e-6 to 0.9e-6).  Nothing is dequantised, scores and sums are
// fp32.  Matrix operands that are not codes go in as bf16 pieces, an MFMA each: a bf16
// query is one, a compensated pair two, an fp32 query three (all 24 bits); p s is two
// (16 bits, of the largest term: outputs of 2^-11 of their terms are off by 3e-3) with
// bf16 models and three with fp32 ones.
//
// Scores are computed transposed (keys by columns), so that a lane owns one column
// and its probabilities are the second product's operand as they stand.  The packed
// layout holds the codes in the order of that operand: every load of the key loop is
// one contiguous piece per wavefront, straight into registers, and no LDS or barrier
// is in the loop.  A block's keys are loaded again as soon as the scores have used
// them, its values after the output product.  Softmax runs in the exp2 domain; a
// column's running maximum is raised only when a score exceeds it by 2^8, so the
// cross-lane maximum is rare, and the sums are reduced once, at the end.
//
// Few columns (the next token of a document has G) leave a tile's lanes idle in the
// softmax, whose work is the larger part.  With at most 16 / CL columns the tile
// holds them CL times, and of CL key tiles each copy takes one: the scores of a lane
// are those of its copy's keys, and in the operand of the output product a copy's
// probabilities are zero for the other tiles' keys.  The copies are columns of their
// own, with their own maximum and sum, and are joined at the end.
//
// A block of threads takes (document, column group, kv head, key range): cw
// wavefronts hold a 16-column tile each, and the wavefronts of a tile take alternate
// key blocks and join their states through LDS.  Key ranges that are split over
// blocks of threads leave partials (O, m, l) that a combine kernel joins.
//
// bf16 models with many columns take attention_packed_rows.hip instead.
#include <math.h>

#include <type_traits>

#include "packed.h"

namespace kvr {

namespace {

typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
typedef __attribute__((ext_vector_type(2))) float f32x2;

__device__ __forceinline__ float pk_max4(float v) {
    unsigned u = __float_as_uint(v);
    const auto a = __builtin_amdgcn_permlane16_swap(u, u, false, false);
    v = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
    u = __float_as_uint(v);
    const auto b = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
// Sum over the four lanes l, l^16, l^32, l^48 that hold one column.
__device__ __forceinline__ float pk_sum4(float v) {
    unsigned u = __float_as_uint(v);
    const auto a = __builtin_amdgcn_permlane16_swap(u, u, false, false);
    v = __uint_as_float(a[0]) + __uint_as_float(a[1]);
    u = __float_as_uint(v);
    const auto b = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}

// v of the lane N further on in the 16 lanes of a row (with CL copies of 16 / CL
// columns: of the same column in another copy).
template <int N>
__device__ __forceinline__ float pk_ror(float v) {
    return __uint_as_float(__builtin_amdgcn_mov_dpp(__float_as_uint(v), 0x120 + N, 0xf, 0xf, true));
}

// The least and the largest value over a tile's 16 columns, for the whole wavefront.
__device__ __forceinline__ void pk_minmax16(int *least, int *top) {
    int lo = *least, hi = *top;
#define KVR_STEP(N)                                                            \
    lo = min(lo, __builtin_amdgcn_mov_dpp(lo, 0x120 + N, 0xf, 0xf, true));     \
    hi = max(hi, __builtin_amdgcn_mov_dpp(hi, 0x120 + N, 0xf, 0xf, true));
    KVR_STEP(8) KVR_STEP(4) KVR_STEP(2) KVR_STEP(1)
#undef KVR_STEP
    *least = __builtin_amdgcn_readfirstlane(lo);
    *top = __builtin_amdgcn_readfirstlane(hi);
}

// Weight of a partial state with maximum m in one with maximum `all`.  A state
// without a maximum is empty (zeros) or saw scores of NaN only, which stay.
__device__ __forceinline__ float pk_weight(float m, float all) {
    return m == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m - all);
}

// One 32-key block of a plane as a lane loads it.
template <int HP, int BITS>
struct PackedBlock {
    static constexpr int W = HP * BITS / 256;  // 16-byte units of a lane's codes: 1 (64 wide, 4 bits) .. 4
    static_assert(64 * W * 16 == pk_code_bytes(HP, BITS), "a lane's share of a block");
    u32x4 codes[W];
    // keys: [16-position tile][KS * BITS / 4 words]; values: [KS * BITS / 2 words]
    __device__ __forceinline__ uint32_t word(int i) const { return codes[i >> 2][i & 3]; }
    __device__ __forceinline__ void load_keys(const char *b, int lane) {
        constexpr int TB = pk_code_bytes(HP, BITS) / 2;  // bytes of a 16-position tile
        if constexpr (W == 1) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const uint2 u = *reinterpret_cast<const uint2 *>(b + h * TB + lane * 8);
                codes[0][2 * h] = u.x;
                codes[0][2 * h + 1] = u.y;
            }
        } else {
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int i = 0; i < W / 2; ++i)
                    codes[h * (W / 2) + i] = *reinterpret_cast<const u32x4 *>(b + h * TB + (lane * (W / 2) + i) * 16);
        }
    }
    __device__ __forceinline__ void load_values(const char *b, int lane) {
#pragma unroll
        for (int i = 0; i < W; ++i) codes[i] = *reinterpret_cast<const u32x4 *>(b + (lane * W + i) * 16);
    }
};

// Scale and offset words of positions 16 half + 4 g4 .. +3 of a block, groups side by
// side.
template <int HP, int BITS>
__device__ __forceinline__ void pk_params(u32x4 par[HP / PK_GROUP], const char *plane, int b, int half, int g4) {
    constexpr int GS = HP / PK_GROUP;
    const char *p = plane + (size_t)b * pk_block_bytes(HP, BITS) + pk_code_bytes(HP, BITS) + (16 * half + 4 * g4) * GS * 4;
#pragma unroll
    for (int i = 0; i < GS; ++i) par[i] = reinterpret_cast<const u32x4 *>(p)[i];
}
template <int GS>
__device__ __forceinline__ uint32_t pk_param(const u32x4 par[GS], int i, int g) {
    return par[(i * GS + g) >> 2][(i * GS + g) & 3];
}

__device__ __forceinline__ bf16x8 pk_operand(uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
    return __builtin_bit_cast(bf16x8, u32x4{a, b, c, d});
}
// Two integers 0..255 as fp32, to a pair of bf16 (exact).
__device__ __forceinline__ uint32_t pk_pair(float lo, float hi) {
    return __builtin_amdgcn_perm(__float_as_uint(hi), __float_as_uint(lo), 0x07060302u);
}
__device__ __forceinline__ bf16x8 pk_bytes(uint32_t a, uint32_t b) {
    return pk_operand(pk_pair((float)(a & 0xffu), (float)((a >> 8) & 0xffu)), pk_pair((float)((a >> 16) & 0xffu), (float)(a >> 24)),
                      pk_pair((float)(b & 0xffu), (float)((b >> 8) & 0xffu)), pk_pair((float)((b >> 16) & 0xffu), (float)(b >> 24)));
}
// (x & mask) | bits in one instruction (the compiler makes two of it, with literals).
__device__ __forceinline__ uint32_t pk_and_or(uint32_t x, uint32_t mask, uint32_t bits) {
    uint32_t r;
    asm("v_and_or_b32 %0, %1, %2, %3" : "=v"(r) : "v"(x), "s"(mask), "v"(bits));
    return r;
}
// 16 + code for the eight dimensions of a key word.
__device__ __forceinline__ bf16x8 pk_key4(uint32_t w) {
    constexpr uint32_t M = 0x00780078u, B = 0x41804180u;
    return pk_operand(pk_and_or(w << 3, M, B), pk_and_or(w >> 1, M, B), pk_and_or(w >> 5, M, B), pk_and_or(w >> 9, M, B));
}
// 16 + code for the four positions each of two value words, of their low (nib 0) or
// high dimension.
__device__ __forceinline__ bf16x8 pk_value4(uint32_t a, uint32_t b, int nib) {
    constexpr uint32_t M = 0x78787878u, B = 0x80808080u, X = 0x41414141u;
    const uint32_t x = pk_and_or(nib ? a >> 1 : a << 3, M, B), y = pk_and_or(nib ? b >> 1 : b << 3, M, B);
    return pk_operand(__builtin_amdgcn_perm(X, x, 0x04010400u), __builtin_amdgcn_perm(X, x, 0x04030402u),
                      __builtin_amdgcn_perm(X, y, 0x04010400u), __builtin_amdgcn_perm(X, y, 0x04030402u));
}

// Each half of a pair of bf16 less x (exact for integers below 256).
__device__ __forceinline__ uint32_t pk_less(uint32_t u, float x) {
    return pk_pair(__uint_as_float(u << 16) - x, __uint_as_float(u & 0xffff0000u) - x);
}
__device__ __forceinline__ bf16x8 pk_less(bf16x8 v, float x) {
    const u32x4 u = __builtin_bit_cast(u32x4, v);
    return pk_operand(pk_less(u[0], x), pk_less(u[1], x), pk_less(u[2], x), pk_less(u[3], x));
}

// Eight values to NP bf16 pieces that add up to them (to 8 NP bits).
template <int NP>
__device__ __forceinline__ void pk_pieces(const float v[8], bf16x8 p[NP]) {
    u32x4 u[NP];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        f32x2 f = {v[2 * q], v[2 * q + 1]};
#pragma unroll
        for (int x = 0; x < NP; ++x) {
            const bf16x2 h = __builtin_convertvector(f, bf16x2);
            u[x][q] = __builtin_bit_cast(unsigned int, h);
            if (x + 1 < NP) f -= __builtin_convertvector(h, f32x2);
        }
    }
#pragma unroll
    for (int x = 0; x < NP; ++x) p[x] = __builtin_bit_cast(bf16x8, u[x]);
}

template <int NP>
__device__ __forceinline__ void pk_pieces4(const float v[4], uint32_t p[NP][2]) {
#pragma unroll
    for (int q = 0; q < 2; ++q) {
        f32x2 f = {v[2 * q], v[2 * q + 1]};
#pragma unroll
        for (int x = 0; x < NP; ++x) {
            const bf16x2 h = __builtin_convertvector(f, bf16x2);
            p[x][q] = __builtin_bit_cast(uint32_t, h);
            if (x + 1 < NP) f -= __builtin_convertvector(h, f32x2);
        }
    }
}

// n <= 4 values at columns c.. of row r.
template <typename T>
__device__ __forceinline__ void pk_store(const PackedAttnArgs &a, int64_t r, int c, int n, bool vec, f32x4 y) {
    T *o = (T *)a.out, *lo = (T *)a.out_lo;
    const size_t off = a.o_perm ? perm_offset((int)r, c, (int)a.out_stride) : (size_t)(r * a.out_stride + c);
    if (vec && n == 4) {
        if constexpr (sizeof(T) == 4) {
            *reinterpret_cast<f32x4 *>(o + off) = y;
        } else {
            uint32_t h[2], l[2];
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                const f32x2 x = {y[2 * q], y[2 * q + 1]};
                const bf16x2 b = __builtin_convertvector(x, bf16x2);
                h[q] = __builtin_bit_cast(unsigned int, b);
                l[q] = __builtin_bit_cast(unsigned int, __builtin_convertvector(x - __builtin_convertvector(b, f32x2), bf16x2));
            }
            *reinterpret_cast<uint2 *>(o + off) = make_uint2(h[0], h[1]);
            if (lo) *reinterpret_cast<uint2 *>(lo + off) = make_uint2(l[0], l[1]);
        }
        return;
    }
    for (int e = 0; e < n; ++e)
        store_operand(o, lo, a.o_perm ? perm_offset((int)r, c + e, (int)a.out_stride) : off + e, y[e]);
}

// A lane's part of the query operand: dimensions 32 s + 8 g4 .. +8 of one row and head
// (zeros behind hd), as QP bf16 pieces, and their sums by group.
template <typename T, int HP, int QP>
__device__ __forceinline__ void pk_query(const PackedAttnArgs &a, int64_t row, int head, int g4, int q_vec,
                                         bf16x8 qv[QP][HP / 32], float qsum[HP / PK_GROUP]) {
    constexpr int KS = HP / 32;
    const size_t q0 = (size_t)(row * a.q_stride) + head * a.hd;
    const T *q = (const T *)a.q + q0;
#pragma unroll
    for (int g = 0; g < HP / PK_GROUP; ++g) qsum[g] = 0.f;
    if constexpr (QP <= 2) {
        u32x4 u[QP][KS];
        if (q_vec) {  // hd is a multiple of 8
#pragma unroll
            for (int x = 0; x < QP; ++x)
#pragma unroll
                for (int s = 0; s < KS; ++s)
                    u[x][s] = *reinterpret_cast<const u32x4 *>((x ? (const T *)a.q_lo + q0 : q) + min(32 * s + 8 * g4, a.hd - 8));
#pragma unroll
            for (int x = 0; x < QP; ++x)
#pragma unroll
                for (int s = 0; s < KS; ++s)
                    if (32 * s + 8 * g4 >= a.hd) u[x][s] = u32x4{0, 0, 0, 0};
        } else {
#pragma unroll
            for (int x = 0; x < QP; ++x)
#pragma unroll
                for (int s = 0; s < KS; ++s) {
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const int d = 32 * s + 8 * g4 + 2 * j;  // (hd is even)
                        const T *p = (x ? (const T *)a.q_lo + q0 : q) + min(d, a.hd - 2);
                        u[x][s][j] = d < a.hd ? (uint32_t)p[0] | ((uint32_t)p[1] << 16) : 0;
                    }
                }
        }
#pragma unroll
        for (int x = 0; x < QP; ++x)
#pragma unroll
            for (int s = 0; s < KS; ++s) {
                qv[x][s] = __builtin_bit_cast(bf16x8, u[x][s]);
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    qsum[s / 2] += __uint_as_float(u[x][s][j] << 16) + __uint_as_float(u[x][s][j] & 0xffff0000u);
            }
    } else {
        float v[KS][8];
#pragma unroll
        for (int s = 0; s < KS; ++s)
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (!q_vec) v[s][j] = (float)q[min(32 * s + 8 * g4 + j, a.hd - 1)];
        if (q_vec) {
#pragma unroll
            for (int s = 0; s < KS; ++s)
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    const f32x4 u = *reinterpret_cast<const f32x4 *>(q + min(32 * s + 8 * g4, a.hd - 8) + 4 * k);
#pragma unroll
                    for (int j = 0; j < 4; ++j) v[s][4 * k + j] = u[j];
                }
        }
#pragma unroll
        for (int s = 0; s < KS; ++s) {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                if (32 * s + 8 * g4 + j >= a.hd) v[s][j] = 0.f;
                qsum[s / 2] += v[s][j];
            }
            bf16x8 p[QP];
            pk_pieces<QP>(v[s], p);
#pragma unroll
            for (int x = 0; x < QP; ++x) qv[x][s] = p[x];
        }
    }
}

// T: the model's type.  QP: bf16 pieces of a query; CL: copies of the columns in a
// tile; N: words of the table.
template <typename T, int HP, int BITS, int QP, int CL, int N>
__global__ __launch_bounds__(64 * PK_WAVES_MAX) void attention_packed_kernel(PackedAttnArgs a, PackedWords<N> t) {
    constexpr int KS = HP / 32, GS = HP / PK_GROUP, DT = HP / 16;
    constexpr int PP = sizeof(T) == 4 ? 3 : 2;  // bf16 pieces of a probability times a scale
    constexpr bool CENTRED = sizeof(T) == 4;
    constexpr float RAW = BITS == 4 ? 16.f : 0.f;                      // a loaded code's offset
    constexpr float OFF = !CENTRED ? RAW : BITS == 4 ? -8.f : -128.f;  // the operand's
    constexpr int BB = pk_block_bytes(HP, BITS);
    constexpr int STATE = DT * 256 + 128;  // floats of a wavefront's state: O, then m and l
    constexpr int CC_LOG = CL == 4 ? 2 : CL == 2 ? 3 : 4;
    // a step takes SB blocks of keys: TT key tiles, H of them for each copy
    constexpr int SB = CL == 4 ? 2 : 1, TT = 2 * SB, H = TT / CL, CC = 16 / CL;
    extern __shared__ float merge[];

    const int lane = threadIdx.x & 63, g4 = lane >> 4, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int copy = (lane & 15) / CC, col = (lane & 15) % CC;
    // kv heads first: the longest items of all of them start before the shorter ones
    const int kvh = blockIdx.x;
    const PackedEntry e = pk_entry(t, a.n_docs, PKE_ITEM0, blockIdx.y);
    const int nsplit = e.splits, item = (int)blockIdx.y - e.item0;
    const int cw = 1 << a.cw_log, cols_log = CC_LOG + a.cw_log, cols = 1 << cols_log;
    const int kw = 1 << (a.waves_log - a.cw_log), wk = w >> a.cw_log, wc = w & (cw - 1);
    const int G = a.G, ncols_doc = e.rows * G;
    // column groups from the last one down: later rows see more keys
    const int ncg = (ncols_doc + cols - 1) >> cols_log;
    const int down = nsplit == 1 ? item : ncg == 1 ? 0 : item / nsplit, split = item - down * nsplit, cg = ncg - 1 - down;
    // the first blocks' loads wait for nothing else
    const size_t plane = (size_t)e.blocks * BB;
    const char *kp = e.packed + ((size_t)a.layer * 2 * a.Hkv + kvh) * plane;
    const char *vp = kp + a.Hkv * plane;
    const int last = e.blocks - 1;
    PackedBlock<HP, BITS> kb[SB], vb[SB];
    u32x4 kpar[H][GS], vpar[H][GS];  // of this lane's keys
    // Blocks b .. b + SB - 1; an odd document's last step loads its last block twice.
    auto load_keys = [&](int b) {
#pragma unroll
        for (int x = 0; x < SB; ++x) kb[x].load_keys(kp + (size_t)min(b + x, last) * BB, lane);
#pragma unroll
        for (int h = 0; h < H; ++h) pk_params<HP, BITS>(kpar[h], kp, min(b + (h * CL + copy) / 2, last), (h * CL + copy) & 1, g4);
    };
    auto load_values = [&](int b) {
#pragma unroll
        for (int x = 0; x < SB; ++x) vb[x].load_values(vp + (size_t)min(b + x, last) * BB, lane);
#pragma unroll
        for (int h = 0; h < H; ++h) pk_params<HP, BITS>(vpar[h], vp, min(b + (h * CL + copy) / 2, last), (h * CL + copy) & 1, g4);
    };
    const int b0 = split * (a.range / PK_BLOCK) + wk * SB;
    load_keys(min(b0, last));
    load_values(min(b0, last));
    const int row0 = e.row0;

    // this lane's column: its row, head and number of visible keys
    const int column = cg * cols + wc * CC + col;
    const bool valid = column < ncols_doc;
    const int row = valid ? column / G : 0, head = kvh * G + (valid ? column - row * G : 0);
    const int limit = valid ? min(pk_position(t, e, row, a.rows) + 1, e.keys) : 0;
    bf16x8 qv[QP][KS];
    float qsum[GS];
    pk_query<T, HP, QP>(a, row0 + row, head, g4, a.q_vec, qv, qsum);
    int top = limit, least = valid ? limit : 0x7fffffff;
#pragma unroll
    for (int g = 0; g < GS; ++g) qsum[g] = pk_sum4(qsum[g]);
    // the wavefront's last visible key, and the keys that all its columns see
    pk_minmax16(&least, &top);
    const int b1 = (min(top, (split + 1) * a.range) + PK_BLOCK - 1) / PK_BLOCK;
    // Steps that begin before it need no mask.  With copies there are few values to mask:
    // one loop for all (5 % of its instructions are the masks), half the code.
    const int b_full = CL > 1 ? 0 : min(b1, least / PK_BLOCK) - (SB - 1);

    f32x4 o[DT];
    float m = -INFINITY, l = 0.f, z[GS];
#pragma unroll
    for (int d = 0; d < DT; ++d) o[d] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int g = 0; g < GS; ++g) z[g] = 0.f;
    const float sc = a.scale;
    uint32_t mine[CL];  // all ones for this lane's copy
#pragma unroll
    for (int c = 0; c < CL; ++c) mine[c] = copy == c ? 0xffffffffu : 0u;

    // one step; masked: a column may not see all of its keys
    auto step = [&](int b, auto masked_) {
        constexpr bool MASKED = decltype(masked_)::value;
        const bool more = b + kw * SB < b1;
        const int key0 = b * PK_BLOCK + 16 * copy + 4 * g4;  // this lane's keys: key0 + 16 CL h + i
        f32x4 s[H];
#pragma unroll
        for (int h = 0; h < H; ++h) {
            f32x4 acc[GS];
#pragma unroll
            for (int c = 0; c < CL; ++c) {
                const int tile = h * CL + c;
                f32x4 one[GS];
#pragma unroll
                for (int g = 0; g < GS; ++g) {
                    const float i = CENTRED ? 0.f : -OFF * qsum[g];
                    one[g] = f32x4{i, i, i, i};
                }
#pragma unroll
                for (int st = 0; st < KS; ++st) {
                    const PackedBlock<HP, BITS> &k = kb[tile >> 1];
                    const int i = (tile & 1) * KS + st;
                    bf16x8 ka = BITS == 4 ? pk_key4(k.word(i)) : pk_bytes(k.word(2 * i), k.word(2 * i + 1));
                    if (CENTRED) ka = pk_less(ka, RAW - OFF);
#pragma unroll
                    for (int x = 0; x < QP; ++x)
                        one[st / 2] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ka, qv[x][st], one[st / 2], 0, 0, 0);
                }
#pragma unroll
                for (int g = 0; g < GS; ++g)
#pragma unroll
                    for (int i = 0; i < 4; ++i) acc[g][i] = c == 0 || copy == c ? one[g][i] : acc[g][i];
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                float v = 0.f;
#pragma unroll
                for (int g = 0; g < GS; ++g) {
                    const uint32_t u = pk_param<GS>(kpar[h], i, g);
                    const float sk = __uint_as_float(u << 16), mk = __uint_as_float(u & 0xffff0000u);
                    v = fmaf(CENTRED ? mk - OFF * sk : mk, qsum[g], fmaf(sk, acc[g][i], v));
                }
                s[h][i] = MASKED && key0 + 16 * CL * h + i >= limit ? -INFINITY : v;
            }
        }
        // what uses a block's words stands before the next one's loads: no copies of registers
#pragma unroll
        for (int h = 0; h < H; ++h) asm volatile("" : "+v"(s[h]));
        if (more) load_keys(b + kw * SB);
        // the columns' probabilities, in place
        float mx = -INFINITY;
#pragma unroll
        for (int h = 0; h < H; ++h)
#pragma unroll
            for (int i = 0; i < 4; ++i) mx = fmaxf(mx, s[h][i]);
        mx *= sc;
        if (__any(mx > m + 8.f)) {
            const float mnew = fmaxf(m, pk_max4(mx));
            const float corr = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - mnew);
            m = mnew;
            l *= corr;
#pragma unroll
            for (int g = 0; g < GS; ++g) z[g] *= corr;
#pragma unroll
            for (int d = 0; d < DT; ++d) o[d] *= corr;
        }
        const float mu = m == -INFINITY ? 0.f : m;
#pragma unroll
        for (int h = 0; h < H; ++h)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float p = __builtin_amdgcn_exp2f(fmaf(s[h][i], sc, -mu));
                s[h][i] = p;
                l += p;
            }
#pragma unroll
        for (int g = 0; g < GS; ++g) {
            uint32_t pw[H][PP][2];  // the pieces of four probabilities times scales
#pragma unroll
            for (int h = 0; h < H; ++h) {
                float sv[4], mv[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const uint32_t u = pk_param<GS>(vpar[h], i, g);
                    sv[i] = __uint_as_float(u << 16);
                    mv[i] = fmaf(-OFF, sv[i], __uint_as_float(u & 0xffff0000u));
                }
                float v[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    // slots that a column does not see may hold anything, a scale of NaN too
                    const bool hide = MASKED && key0 + 16 * CL * h + i >= limit;
                    v[i] = s[h][i] * (hide ? 0.f : sv[i]);
                    z[g] = fmaf(s[h][i], hide ? 0.f : mv[i], z[g]);
                }
                pk_pieces4<PP>(v, pw[h]);
            }
#pragma unroll
            for (int x = 0; x < SB; ++x) {
                // slots 0..3 of the operand are the block's first tile's keys, 4..7 the second's
                bf16x8 pb[PP];
#pragma unroll
                for (int q = 0; q < PP; ++q) {
                    uint32_t u[4];
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const int tile = 2 * x + k / 2;
                        u[k] = pw[tile / CL][q][k & 1];
                        if (CL > 1) u[k] &= mine[tile % CL];
                    }
                    pb[q] = pk_operand(u[0], u[1], u[2], u[3]);
                }
#pragma unroll
                for (int q = 0; q < 4; ++q) {  // 16-dimension tiles of the group
                    const int d = 4 * g + q;
                    bf16x8 va = BITS == 4 ? pk_value4(vb[x].word((d >> 1) * 2), vb[x].word((d >> 1) * 2 + 1), d & 1)
                                          : pk_bytes(vb[x].word(d * 2), vb[x].word(d * 2 + 1));
                    if (CENTRED) va = pk_less(va, RAW - OFF);
#pragma unroll
                    for (int y = 0; y < PP; ++y)
                        o[d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(va, pb[y], o[d], 0, 0, 0);
                }
            }
        }
#pragma unroll
        for (int g = 0; g < GS; ++g) asm volatile("" : "+v"(z[g]));
        if (more) load_values(b + kw * SB);
    };
    int b = b0;
    if constexpr (CL == 1) {
#pragma unroll 1
        for (; b < b_full; b += kw * SB) step(b, std::false_type{});
    }
#pragma unroll 1
    for (; b < b1; b += kw * SB) step(b, std::true_type{});

    l = pk_sum4(l);
#pragma unroll
    for (int g = 0; g < GS; ++g) {
        const float y = pk_sum4(z[g]);
#pragma unroll
        for (int q = 0; q < 4; ++q) o[4 * g + q] += y;
    }
    if constexpr (CL > 1) {  // the copies of a column
        float all = fmaxf(m, pk_ror<CC>(m));
        if (CL == 4) all = fmaxf(all, pk_ror<8>(all));
        const float f = pk_weight(m, all);
        m = all;
        auto join = [&](float v) {
            v *= f;
            v += pk_ror<CC>(v);
            return CL == 4 ? v + pk_ror<8>(v) : v;
        };
        l = join(l);
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
            for (int i = 0; i < 4; ++i) o[d][i] = join(o[d][i]);
    }
    // Lane: one column, dimensions 16 d + 4 g4 + i.  The wavefronts of a tile hand their
    // states to each other through LDS, and wavefront wk finishes the dimension tiles wk,
    // wk + kw, ..
    float *const own = merge + (size_t)(wk * cw + wc) * STATE;
#pragma unroll
    for (int d = 0; d < DT; ++d) reinterpret_cast<f32x4 *>(own)[d * 64 + lane] = o[d];
    reinterpret_cast<f32x2 *>(own + DT * 256)[lane] = f32x2{m, l};
    __syncthreads();
    if (!valid || copy > 0) return;
    const float *const first = merge + (size_t)wc * STATE;
    const int next = cw * STATE;  // from a wavefront of the tile to the next
    float all = -INFINITY, sum = 0.f, f[PK_WAVES_MAX], ls[PK_WAVES_MAX];
#pragma unroll
    for (int k = 0; k < PK_WAVES_MAX; ++k) {
        const f32x2 ml = k < kw ? reinterpret_cast<const f32x2 *>(first + k * next + DT * 256)[lane] : f32x2{-INFINITY, 0.f};
        f[k] = ml[0];
        ls[k] = ml[1];
    }
#pragma unroll
    for (int k = 0; k < PK_WAVES_MAX; ++k) all = fmaxf(all, f[k]);
#pragma unroll
    for (int k = 0; k < PK_WAVES_MAX; ++k) {
        f[k] = pk_weight(f[k], all);
        sum += ls[k] * f[k];
    }
    const float inv = sum == 0.f ? 0.f : 1.0f / sum;
    float *part = a.part + (((size_t)(e.part0 + cg * nsplit + split) * a.Hkv + kvh) * cols + wc * CC + col) * (HP + 4);
#pragma unroll 1
    for (int d = wk; d < DT; d += kw) {
        f32x4 y = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int k = 0; k < PK_WAVES_MAX; ++k)
            if (k < kw) y += reinterpret_cast<const f32x4 *>(first + k * next)[d * 64 + lane] * f[k];
        const int dim = 16 * d + 4 * g4;
        if (nsplit > 1) *reinterpret_cast<f32x4 *>(part + dim) = y;
        else if (dim < a.hd) pk_store<T>(a, row0 + row, head * a.hd + dim, min(4, a.hd - dim), a.o_vec, y * inv);
    }
    if (nsplit > 1 && g4 == 0 && wk == 0) {
        part[HP] = all;
        part[HP + 1] = sum;
    }
}

inline int pk_log(int x) { return 31 - __builtin_clz(x); }  // of a power of two

// The arguments with what the launchers add.  Query and output rows can be moved in
// vectors where every row's pieces are aligned (16 bytes; bf16 outputs 8).
inline PackedAttnArgs pk_complete(bool bf16, PackedShape sh, PackedAttnArgs a) {
    const size_t es = bf16 ? 2 : 4;
    auto aligned = [](const void *p, size_t n) { return ((uintptr_t)p & (n - 1)) == 0; };
    a.q_vec = a.hd % 8 == 0 && a.q_stride % (16 / es) == 0 && aligned(a.q, 16) && aligned(a.q_lo, 16);
    a.o_vec = a.hd % 4 == 0 && a.out_stride % 4 == 0 && aligned(a.out, 4 * es) && aligned(a.out_lo, 4 * es);
    a.G = a.Hkv > 0 ? a.Hq / a.Hkv : 1;
    a.scale = 1.4426950408889634f / sqrtf((float)a.hd);
    a.waves_log = pk_log(sh.waves);
    a.cw_log = pk_log(sh.cw);
    return a;
}

template <typename T, int HP, int BITS, int QP, int CL>
hipError_t pk_launch(const PackedTable &t, const PackedAttnArgs &a, PackedShape sh, hipStream_t s, int *resident) {
    const uint32_t lds = (uint32_t)sh.waves * (HP / 16 * 256 + 128) * 4;  // the wavefronts' states
    static std::atomic<int> known[2];
    if (resident) return pk_resident(attention_packed_kernel<T, HP, BITS, QP, CL, PK_WORDS>, sh.waves, lds, known, resident);
    pk_with_words(t, a.n_docs, [&](const auto &words) {
        constexpr int N = sizeof(words) / 4;
        kvr_launch((attention_packed_kernel<T, HP, BITS, QP, CL, N>), dim3(a.Hkv, a.n_items), dim3(64 * sh.waves), lds, s, a, words);
    });
    return hipGetLastError();
}

template <typename T, int HP, int BITS, int QP>
hipError_t pk_launch_copies(const PackedTable &t, const PackedAttnArgs &a, PackedShape sh, hipStream_t s, int *resident) {
    if (sh.copies == 4) return pk_launch<T, HP, BITS, QP, 4>(t, a, sh, s, resident);
    if (sh.copies == 2) return pk_launch<T, HP, BITS, QP, 2>(t, a, sh, s, resident);
    return pk_launch<T, HP, BITS, QP, 1>(t, a, sh, s, resident);
}

template <int HP, int BITS>
hipError_t pk_launch_bits(bool bf16, PackedShape sh, const PackedTable &t, const PackedAttnArgs &a, hipStream_t s, int *resident) {
    if (!bf16) return pk_launch_copies<float, HP, BITS, 3>(t, a, sh, s, resident);
    return a.q_lo ? pk_launch_copies<bf16_t, HP, BITS, 2>(t, a, sh, s, resident)
                  : pk_launch_copies<bf16_t, HP, BITS, 1>(t, a, sh, s, resident);
}

template <int HP>
hipError_t pk_launch_width(bool bf16, int bits, PackedShape sh, const PackedTable &t, const PackedAttnArgs &a, hipStream_t s,
                           int *resident) {
    return bits == 4 ? pk_launch_bits<HP, 4>(bf16, sh, t, a, s, resident) : pk_launch_bits<HP, 8>(bf16, sh, t, a, s, resident);
}

}  // namespace

}  // namespace kvr
