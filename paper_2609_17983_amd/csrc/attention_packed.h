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
// two bits (an output's error against 64 bits 1.8e-6, in plain fp32 0.7e-6).  Nothing is
// dequantised, and the scores and outputs keep 32 bits.  Matrix operands that are
// not codes go in as bf16 pieces, an MFMA each: a bf16 query is one, a compensated
// pair two, an fp32 query three (all 24 bits); p s is two (16 bits) with bf16 models
// and three with fp32 ones.
//
// Scores are computed transposed (keys by columns), so that a lane owns one column
// and its probabilities are the second product's operand as they stand.  The packed
// layout holds the codes in the order of that operand: every load of the key loop is
// one contiguous piece per wavefront, straight into registers, and no LDS or barrier
// is in the loop.  Softmax runs in the exp2 domain; a column's running maximum is
// raised only when a score exceeds it by 2^8, so the cross-lane maximum is rare, and
// the sums are reduced once, at the end.
//
// A block of four wavefronts takes (document, column group, kv head, key range):
// cw wavefronts hold nt 16-column tiles each, and the 4 / cw wavefronts of a tile
// take alternate 32-key blocks and merge their states through LDS.  Key ranges that
// are split over blocks leave partials (O, m, l) that a combine kernel joins.
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

// Weight of a partial state with maximum m in one with maximum `all`.  A state
// without a maximum is empty (zeros) or saw scores of NaN only, which stay.
__device__ __forceinline__ float pk_weight(float m, float all) {
    return m == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m - all);
}

// One 32-key block of a plane as a lane loads it.
template <int HP, int BITS>
struct PackedBlock {
    static constexpr int KS = HP / 32, GS = HP / PK_GROUP;
    static constexpr int W = HP * BITS / 256;  // 16-byte units of a lane's codes: 1 (64 wide, 4 bits) .. 4
    static_assert(64 * W * 16 == pk_code_bytes(HP, BITS), "a lane's share of a block");
    u32x4 codes[W];
    u32x4 par[2][GS];  // scale and offset words of positions 16h + 4g .. +3, groups side by side
    // keys: [16-position tile][KS * BITS / 4 words]; values: [KS * BITS / 2 words]
    __device__ __forceinline__ uint32_t word(int i) const { return codes[i >> 2][i & 3]; }
    __device__ __forceinline__ uint32_t param(int h, int e, int g) const {
        const int i = e * GS + g;
        return par[h][i >> 2][i & 3];
    }
    __device__ __forceinline__ void load_params(const char *b, int g4) {
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int i = 0; i < GS; ++i)
                par[h][i] = *reinterpret_cast<const u32x4 *>(b + pk_code_bytes(HP, BITS) + ((16 * h + 4 * g4) * GS + 4 * i) * 4);
    }
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
        load_params(b, lane >> 4);
    }
    __device__ __forceinline__ void load_values(const char *b, int lane) {
#pragma unroll
        for (int i = 0; i < W; ++i) codes[i] = *reinterpret_cast<const u32x4 *>(b + (lane * W + i) * 16);
        load_params(b, lane >> 4);
    }
};

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
// 16 + code for the eight dimensions of a key word.
__device__ __forceinline__ bf16x8 pk_key4(uint32_t w) {
    constexpr uint32_t M = 0x00780078u, B = 0x41804180u;
    return pk_operand(((w << 3) & M) | B, ((w >> 1) & M) | B, ((w >> 5) & M) | B, ((w >> 9) & M) | B);
}
// 16 + code for the four positions each of two value words, of their low (nib 0) or
// high dimension.
__device__ __forceinline__ bf16x8 pk_value4(uint32_t a, uint32_t b, int nib) {
    constexpr uint32_t M = 0x78787878u, B = 0x80808080u, X = 0x41414141u;
    const uint32_t x = ((nib ? a >> 1 : a << 3) & M) | B, y = ((nib ? b >> 1 : b << 3) & M) | B;
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

// T: the model's type.  QP: bf16 pieces of a query; NT: column tiles of a wavefront.
template <typename T, int HP, int BITS, int QP, int NT>
__global__ __launch_bounds__(64 * PK_ATT_WAVES, 2) void attention_packed_kernel(PackedTable t, PackedAttnArgs a, int cw,
                                                                               int q_vec, int o_vec) {
    constexpr int KS = HP / 32, GS = HP / PK_GROUP, DT = HP / 16;
    constexpr int PP = sizeof(T) == 4 ? 3 : 2;  // bf16 pieces of a probability times a scale
    constexpr bool CENTRED = sizeof(T) == 4;
    constexpr float RAW = BITS == 4 ? 16.f : 0.f;                              // a loaded code's offset
    constexpr float OFF = !CENTRED ? RAW : BITS == 4 ? -8.f : -128.f;  // the operand's
    constexpr int BB = pk_block_bytes(HP, BITS);
    constexpr int ST = DT * 4 + 2;  // a lane's state per tile: O, m, l
    extern __shared__ float merge[];

    const int lane = threadIdx.x & 63, g4 = lane >> 4, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int kvh = blockIdx.y;
    const uint32_t *e = t.w + pk_find(t, a.n_docs, PKE_ITEM0, blockIdx.x) * PK_ENTRY;
    const int nsplit = e[PKE_SPLITS], item = blockIdx.x - (int)e[PKE_ITEM0];
    const int cols = 16 * NT * cw;
    const int kw = PK_ATT_WAVES / cw, wk = w / cw, wc = w - wk * cw;
    const int split = nsplit == 1 ? 0 : item % nsplit;
    // the first key block's loads wait for nothing else
    const size_t plane = (size_t)e[PKE_BLOCKS] * BB;
    const char *kp = pk_pointer(e) + ((size_t)a.layer * 2 * a.Hkv + kvh) * plane;
    const char *vp = kp + a.Hkv * plane;
    const int b0 = split * (a.range / PK_BLOCK) + wk;
    PackedBlock<HP, BITS> kb, vb;
    {
        const size_t first = (size_t)min(b0, (int)e[PKE_BLOCKS] - 1) * BB;
        kb.load_keys(kp + first, lane);
        vb.load_values(vp + first, lane);
    }
    const int G = a.Hq / a.Hkv, ncols_doc = (int)e[PKE_ROWS] * G;
    // column groups from the last one down: later rows see more keys
    const int ncg = (ncols_doc + cols - 1) / cols;
    const int cg = ncg - 1 - (nsplit == 1 ? item : item / nsplit);
    const int row0 = e[PKE_ROW0];

    // this lane's columns: their row, head and number of visible keys
    int limit[NT], row[NT], head[NT];
    bf16x8 qv[NT][QP][KS];
    float qsum[NT][GS];
    int top = 0, least = 0x7fffffff;
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        const int c = cg * cols + (wc * NT + n) * 16 + (lane & 15);
        const bool valid = c < ncols_doc;
        row[n] = valid ? c / G : 0;
        head[n] = kvh * G + (valid ? c - row[n] * G : 0);
        limit[n] = valid ? min(pk_position(t, e, row[n], a.rows) + 1, (int)e[PKE_KEYS]) : 0;
        top = max(top, limit[n]);
        if (valid) least = min(least, limit[n]);
        const size_t q0 = (size_t)(row0 + row[n]) * a.q_stride + head[n] * a.hd;
        row[n] = valid ? row[n] : -1;
        const T *q = (const T *)a.q + q0;
#pragma unroll
        for (int g = 0; g < GS; ++g) qsum[n][g] = 0.f;
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
                        u[x][s] = u32x4{0, 0, 0, 0};
                        for (int j = 0; j < 8; ++j) {
                            const int d = 32 * s + 8 * g4 + j;
                            const uint32_t v = d < a.hd ? (uint32_t)(x ? (const T *)a.q_lo + q0 : q)[d] : 0;
#pragma unroll
                            for (int k = 0; k < 4; ++k)
                                if (k == j >> 1) u[x][s][k] |= v << (16 * (j & 1));
                        }
                    }
            }
#pragma unroll
            for (int x = 0; x < QP; ++x)
#pragma unroll
                for (int s = 0; s < KS; ++s) {
                    qv[n][x][s] = __builtin_bit_cast(bf16x8, u[x][s]);
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        qsum[n][s / 2] += __uint_as_float(u[x][s][j] << 16) + __uint_as_float(u[x][s][j] & 0xffff0000u);
                }
        } else {
            float v[KS][8];
#pragma unroll
            for (int s = 0; s < KS; ++s)
#pragma unroll
                for (int j = 0; j < 8; ++j) v[s][j] = (float)q[min(32 * s + 8 * g4 + j, a.hd - 1)];
#pragma unroll
            for (int s = 0; s < KS; ++s) {
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    if (32 * s + 8 * g4 + j >= a.hd) v[s][j] = 0.f;
                    qsum[n][s / 2] += v[s][j];
                }
                bf16x8 p[QP];
                pk_pieces<QP>(v[s], p);
#pragma unroll
                for (int x = 0; x < QP; ++x) qv[n][x][s] = p[x];
            }
        }
#pragma unroll
        for (int g = 0; g < GS; ++g) qsum[n][g] = pk_sum4(qsum[n][g]);
    }
    // the wavefront's last visible key, and the keys that all its columns see
#pragma unroll
    for (int o = 1; o < 16; o *= 2) {
        top = max(top, __shfl_xor(top, o, 64));
        least = min(least, __shfl_xor(least, o, 64));
    }
    top = __builtin_amdgcn_readfirstlane(top);
    least = __builtin_amdgcn_readfirstlane(least);
    const int b1 = (min(top, (split + 1) * a.range) + PK_BLOCK - 1) / PK_BLOCK;
    const int b_full = min(b1, least / PK_BLOCK);  // blocks before it need no mask

    f32x4 o[NT][DT];
    float m[NT], l[NT], z[NT][GS];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
#pragma unroll
        for (int d = 0; d < DT; ++d) o[n][d] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int g = 0; g < GS; ++g) z[n][g] = 0.f;
        m[n] = -INFINITY;
        l[n] = 0.f;
    }
    const float sc = 1.4426950408889634f / sqrtf((float)a.hd);

    // one block of keys; masked: a column may not see all of them
    auto step = [&](int b, auto masked_) {
        constexpr bool MASKED = decltype(masked_)::value;
        const PackedBlock<HP, BITS> kc = kb, vc = vb;
        if (b + kw < b1) {
            kb.load_keys(kp + (size_t)(b + kw) * BB, lane);
            vb.load_values(vp + (size_t)(b + kw) * BB, lane);
        }
        const int key0 = b * PK_BLOCK + 4 * g4;  // this lane's keys: key0 + 16 h + i
        f32x4 s[NT][2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            f32x4 acc[NT][GS];
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int g = 0; g < GS; ++g) {
                    const float i = CENTRED ? 0.f : -OFF * qsum[n][g];
                    acc[n][g] = f32x4{i, i, i, i};
                }
#pragma unroll
            for (int st = 0; st < KS; ++st) {
                bf16x8 ka = BITS == 4 ? pk_key4(kc.word(h * KS + st))
                                      : pk_bytes(kc.word((h * KS + st) * 2), kc.word((h * KS + st) * 2 + 1));
                if (CENTRED) ka = pk_less(ka, RAW - OFF);
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int x = 0; x < QP; ++x)
                        acc[n][st / 2] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ka, qv[n][x][st], acc[n][st / 2], 0, 0, 0);
            }
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    float v = 0.f;
#pragma unroll
                    for (int g = 0; g < GS; ++g) {
                        const uint32_t u = kc.param(h, i, g);
                        const float sk = __uint_as_float(u << 16), mk = __uint_as_float(u & 0xffff0000u);
                        v = fmaf(CENTRED ? mk - OFF * sk : mk, qsum[n][g], fmaf(sk, acc[n][g][i], v));
                    }
                    s[n][h][i] = MASKED && key0 + 16 * h + i >= limit[n] ? -INFINITY : v;
                }
        }
        // the columns' probabilities, in place
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            float mx = -INFINITY;
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int i = 0; i < 4; ++i) mx = fmaxf(mx, s[n][h][i]);
            mx *= sc;
            if (__any(mx > m[n] + 8.f)) {
                const float mnew = fmaxf(m[n], pk_max4(mx));
                const float corr = m[n] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m[n] - mnew);
                m[n] = mnew;
                l[n] *= corr;
#pragma unroll
                for (int g = 0; g < GS; ++g) z[n][g] *= corr;
#pragma unroll
                for (int d = 0; d < DT; ++d) o[n][d] *= corr;
            }
            const float mu = m[n] == -INFINITY ? 0.f : m[n];
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float p = __builtin_amdgcn_exp2f(fmaf(s[n][h][i], sc, -mu));
                    s[n][h][i] = p;
                    l[n] += p;
                }
        }
#pragma unroll
        for (int g = 0; g < GS; ++g) {
            bf16x8 pb[NT][PP];
            float v[NT][8];
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const uint32_t u = vc.param(h, i, g);
                    const float sv = __uint_as_float(u << 16), mv = fmaf(-OFF, sv, __uint_as_float(u & 0xffff0000u));
#pragma unroll
                    for (int n = 0; n < NT; ++n) {
                        // slots that a column does not see may hold anything, a scale of NaN too
                        const bool hide = MASKED && key0 + 16 * h + i >= limit[n];
                        v[n][4 * h + i] = s[n][h][i] * (hide ? 0.f : sv);
                        z[n][g] = fmaf(s[n][h][i], hide ? 0.f : mv, z[n][g]);
                    }
                }
#pragma unroll
            for (int n = 0; n < NT; ++n) pk_pieces<PP>(v[n], pb[n]);
#pragma unroll
            for (int q = 0; q < 4; ++q) {  // 16-dimension tiles of the group
                const int d = 4 * g + q;
                bf16x8 va = BITS == 4 ? pk_value4(vc.word((d >> 1) * 2), vc.word((d >> 1) * 2 + 1), d & 1)
                                      : pk_bytes(vc.word(d * 2), vc.word(d * 2 + 1));
                if (CENTRED) va = pk_less(va, RAW - OFF);
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int x = 0; x < PP; ++x)
                        o[n][d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(va, pb[n][x], o[n][d], 0, 0, 0);
            }
        }
    };
    int b = b0;
#pragma unroll 1
    for (; b < b_full; b += kw) step(b, std::false_type{});
#pragma unroll 1
    for (; b < b1; b += kw) step(b, std::true_type{});
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        l[n] = pk_sum4(l[n]);
#pragma unroll
        for (int g = 0; g < GS; ++g) {
            const float y = pk_sum4(z[n][g]);
#pragma unroll
            for (int q = 0; q < 4; ++q) o[n][4 * g + q] += y;
        }
    }
    // the wavefronts of a tile, merged into the first one
    if (kw > 1) {
        if (wk > 0) {
            float *p = merge + (size_t)((wk - 1) * cw + wc) * NT * ST * 64 + lane;
#pragma unroll
            for (int n = 0; n < NT; ++n) {
#pragma unroll
                for (int d = 0; d < DT; ++d)
#pragma unroll
                    for (int i = 0; i < 4; ++i) p[(n * ST + d * 4 + i) * 64] = o[n][d][i];
                p[(n * ST + DT * 4) * 64] = m[n];
                p[(n * ST + DT * 4 + 1) * 64] = l[n];
            }
        }
        __syncthreads();
        if (wk > 0) return;
#pragma unroll 1
        for (int k = 1; k < kw; ++k) {
            const float *p = merge + (size_t)((k - 1) * cw + wc) * NT * ST * 64 + lane;
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                const float m1 = p[(n * ST + DT * 4) * 64], l1 = p[(n * ST + DT * 4 + 1) * 64];
                const float mn = fmaxf(m[n], m1);
                const float a0 = pk_weight(m[n], mn), a1 = pk_weight(m1, mn);
                m[n] = mn;
                l[n] = l[n] * a0 + l1 * a1;
#pragma unroll
                for (int d = 0; d < DT; ++d)
#pragma unroll
                    for (int i = 0; i < 4; ++i) o[n][d][i] = o[n][d][i] * a0 + p[(n * ST + d * 4 + i) * 64] * a1;
            }
        }
    }
    // lane: column lane%16, dimensions 16 d + 4 g4 + i
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        if (row[n] < 0) continue;
        if (nsplit == 1) {
            const float inv = l[n] == 0.f ? 0.f : 1.0f / l[n];
#pragma unroll
            for (int d = 0; d < DT; ++d) {
                const int c = 16 * d + 4 * g4;
                if (c < a.hd)
                    pk_store<T>(a, row0 + row[n], head[n] * a.hd + c, min(4, a.hd - c), o_vec, o[n][d] * inv);
            }
        } else {
            const int c = (wc * NT + n) * 16 + (lane & 15);
            float *p = a.part + (((size_t)((int)e[PKE_PART0] + cg * nsplit + split) * a.Hkv + kvh) * cols + c) * (HP + 4);
#pragma unroll
            for (int d = 0; d < DT; ++d) *reinterpret_cast<f32x4 *>(p + 16 * d + 4 * g4) = o[n][d];
            if (g4 == 0) {
                p[HP] = m[n];
                p[HP + 1] = l[n];
            }
        }
    }
}

template <typename T, int HP, int BITS, int QP, int NT>
hipError_t pk_launch(const PackedTable &t, const PackedAttnArgs &a, int cw, bool q_vec, bool o_vec, hipStream_t s) {
    const int kw = PK_ATT_WAVES / cw;
    const uint32_t lds = (uint32_t)(kw - 1) * cw * NT * (HP / 4 + 2) * 64 * 4;
    kvr_launch((attention_packed_kernel<T, HP, BITS, QP, NT>), dim3(a.n_items, a.Hkv), dim3(64 * PK_ATT_WAVES), lds, s, t, a,
               cw, (int)q_vec, (int)o_vec);
    return hipGetLastError();
}

template <int HP, int BITS>
hipError_t pk_launch_bits(bool bf16, PackedShape sh, const PackedTable &t, const PackedAttnArgs &a, bool q_vec, bool o_vec,
                          hipStream_t s) {
    if (!bf16) return pk_launch<float, HP, BITS, 3, 1>(t, a, sh.cw, q_vec, o_vec, s);
    return a.q_lo ? pk_launch<bf16_t, HP, BITS, 2, 1>(t, a, sh.cw, q_vec, o_vec, s)
                  : pk_launch<bf16_t, HP, BITS, 1, 1>(t, a, sh.cw, q_vec, o_vec, s);
}

template <int HP>
hipError_t pk_launch_width(bool bf16, int bits, PackedShape sh, const PackedTable &t, const PackedAttnArgs &a, hipStream_t s) {
    const size_t es = bf16 ? 2 : 4;
    auto aligned = [](const void *p, size_t n) { return ((uintptr_t)p & (n - 1)) == 0; };
    const bool q_vec = bf16 && a.hd % 8 == 0 && a.q_stride % 8 == 0 && aligned(a.q, 16) && aligned(a.q_lo, 16);
    const bool o_vec = a.hd % 4 == 0 && a.out_stride % 4 == 0 && aligned(a.out, 4 * es) && aligned(a.out_lo, 4 * es);
    return bits == 4 ? pk_launch_bits<HP, 4>(bf16, sh, t, a, q_vec, o_vec, s)
                     : pk_launch_bits<HP, 8>(bf16, sh, t, a, q_vec, o_vec, s);
}

}  // namespace

}  // namespace kvr
