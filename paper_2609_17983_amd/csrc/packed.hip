// Writing and reading packed caches.
//
// A row is one position's keys or values of one head.  For each 64 of its
// dimensions: offset = the smallest value rounded down to bf16, scale = (largest -
// offset) / (2^bits - 1) rounded up to bf16, code = (x - offset) / scale to the
// nearest integer; the row stands for offset + scale * code.  The offset and the
// scale are rounded outwards so that no value is cut off.  The difference, the
// product with 1 / (2^bits - 1) and the product with 1 / scale are single fp32
// operations, which makes the codes reproducible bit for bit.  A group that holds a
// value that is not finite, or whose range overflows, stands for NaN throughout.
#include <math.h>

#include <algorithm>

#include "packed.h"

namespace kvr {

namespace {

typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
typedef __attribute__((ext_vector_type(2))) float f32x2;

// x of another lane of the 16 in a row, by a DPP control.
template <int CTRL>
__device__ __forceinline__ uint32_t row_lane(uint32_t x) {
    return __builtin_amdgcn_mov_dpp(x, CTRL, 0xf, 0xf, true);
}
constexpr int ROR = 0x120;                                    // + n: the lane n further on
constexpr int XOR1 = 0xb1, XOR2 = 0x4e, HALF_MIRROR = 0x141;  // of four lanes; 7 - l of eight
// Smallest and largest value of a wavefront, for all of its lanes (of NaN they may be
// anything).
__device__ __forceinline__ void wave_minmax(float *lo, float *hi) {
    auto with = [&](uint32_t l, uint32_t h) {
        *lo = fminf(*lo, __uint_as_float(l));
        *hi = fmaxf(*hi, __uint_as_float(h));
    };
    auto l = [&] { return __float_as_uint(*lo); };
    auto h = [&] { return __float_as_uint(*hi); };
    with(row_lane<ROR + 8>(l()), row_lane<ROR + 8>(h()));
    with(row_lane<ROR + 4>(l()), row_lane<ROR + 4>(h()));
    with(row_lane<ROR + 2>(l()), row_lane<ROR + 2>(h()));
    with(row_lane<ROR + 1>(l()), row_lane<ROR + 1>(h()));
    // the four rows: each swap leaves a lane's own value and the other row's
    const auto l16 = __builtin_amdgcn_permlane16_swap(l(), l(), false, false);
    const auto h16 = __builtin_amdgcn_permlane16_swap(h(), h(), false, false);
    *lo = __uint_as_float(l16[0]);
    *hi = __uint_as_float(h16[0]);
    with(l16[1], h16[1]);
    const auto l32 = __builtin_amdgcn_permlane32_swap(l(), l(), false, false);
    const auto h32 = __builtin_amdgcn_permlane32_swap(h(), h(), false, false);
    *lo = __uint_as_float(l32[0]);
    *hi = __uint_as_float(h32[0]);
    with(l32[1], h32[1]);
}

// Scale and offset of a group of values within [lo, hi] (not `good`, or lo or hi not
// finite: one of them is not), and the reciprocal that its codes are made with.
template <int BITS>
__device__ __forceinline__ uint32_t group_word(float lo, float hi, bool good, float *off, float *inv) {
    const uint32_t u = __float_as_uint(lo);
    uint32_t m = u & 0xffff0000u;
    if ((int)u < 0 && m != u) m += 0x10000u;
    *off = __uint_as_float(m);
    const float t = hi - *off;
    const float w = t * (1.0f / (float)((1 << BITS) - 1));
    uint32_t s = (__float_as_uint(w) + 0xffffu) & 0xffff0000u;
    if (s < 0x00800000u) s = 0x00800000u;  // the smallest normal number
    if (!(t > 0.f)) s = 0;
    if (!good || !(t < INFINITY) || s >= 0x7f800000u) {
        *off = 0.f;
        *inv = 0.f;
        return 0x7fc00000u;  // NaN, scale 0
    }
    *inv = s ? 1.0f / __uint_as_float(s) : 0.f;
    return m | (s >> 16);
}
// The code of x as a whole float.  It is within [0, 2^bits - 1] by itself: off <= x,
// and 1 / inv is at least (hi - off) / (2^bits - 1) to within a few 2^-24.
__device__ __forceinline__ float code_of(float x, float off, float inv) { return rintf((x - off) * inv); }
// A whole float below 2^23 as the low bits of a word.
__device__ __forceinline__ uint32_t low_bits(float c) { return __float_as_uint(c + 8388608.f); }

// A wavefront writes one row: lane l holds dimensions l (x[0]) and, in rows held 128
// wide, 64 + l (x[1]); dimensions from hd on are not read.  `block`: the position's
// block of the plane.
template <int HP, int BITS>
__device__ __forceinline__ void write_row(const float x[2], int hd, bool value, char *block, int r) {
    constexpr int GS = HP / PK_GROUP;
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int g = 0; g < GS; ++g) {
        const int d = g * PK_GROUP + lane;
        const bool real = d < hd;
        const bool good = __ballot(real && !isfinite(x[g])) == 0;
        float lo = real ? x[g] : INFINITY, hi = real ? x[g] : -INFINITY, off, inv;
        wave_minmax(&lo, &hi);
        const uint32_t word = group_word<BITS>(lo, hi, good, &off, &inv);
        uint32_t c = real && inv != 0.f ? (uint32_t)code_of(x[g], off, inv) : 0;
        int bit;
        if (value) {
            const int at = pk_value_byte(HP, BITS, r, d, &bit);
            if (BITS == 4) {  // with the next 16 lanes' codes
                const auto rows = __builtin_amdgcn_permlane16_swap(c, c, false, false);
                c = rows[0] | rows[1] << 4;
            }
            if (BITS == 8 || !(lane & 16)) block[at] = (char)c;
        } else {
            // the lanes of a word put their codes together
            const int at = pk_key_byte(HP, BITS, r, d, &bit);
            c <<= 8 * (at & 3) + bit;
            c |= row_lane<XOR1>(c);
            c |= row_lane<XOR2>(c);
            if (BITS == 4) c |= row_lane<HALF_MIRROR>(c);
            if ((lane & (32 / BITS - 1)) == 0) *reinterpret_cast<uint32_t *>(block + (at & ~3)) = c;
        }
        if (lane == 0) *reinterpret_cast<uint32_t *>(block + pk_code_bytes(HP, BITS) + (r * GS + g) * 4) = word;
    }
}

// One wavefront per (row, plane): fresh rows of one layer.  Bound by its start and one
// round of loads: 64 rows of 8 heads 3.8 us, 528 rows of 4 heads 5.2 us (4.2 and 5.4 with
// exchanges between lanes through LDS).
template <typename T, int HP, int BITS, int N>
__global__ __launch_bounds__(256) void packed_append_kernel(PackedWords<N> t, int n_docs, const T *k, const T *v,
                                                            int64_t stride, int layer, int Hkv, int hd) {
    const int lane = threadIdx.x & 63, plane = blockIdx.y * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t *first = t.w;
    const int row = (int)first[PKE_ROW0] + blockIdx.x;
    const uint32_t *e = t.w + pk_find(t, n_docs, PKE_ROW0, row) * PK_ENTRY;
    if (plane >= 2 * Hkv) return;
    const bool value = plane >= Hkv;
    const T *src = (value ? v : k) + (size_t)row * stride + (plane - (value ? Hkv : 0)) * hd;
    const float x[2] = {lane < hd ? to_f32(src[lane]) : 0.f, 64 + lane < hd ? to_f32(src[64 + lane]) : 0.f};
    const int p = pk_position(t, e, row - (int)e[PKE_ROW0]);
    constexpr int BB = pk_block_bytes(HP, BITS);
    char *base = pk_pointer(e) + (((size_t)layer * 2 * Hkv + plane) * e[PKE_BLOCKS] + p / PK_BLOCK) * BB;
    write_row<HP, BITS>(x, hd, value, base, p % PK_BLOCK);
}

// ---- whole blocks
//
// A block of threads takes a unit: the listed positions (`mask`) of one 32-position
// block of a plane; with rows held 64 wide it takes two.  HP / 16 lanes share a row,
// lane j dimensions 32 (j/2) + 8 (j%2) .. +8 and the eight 16 further on, so that
// the two halves of a value byte are in one lane and a key word is one lane's.  The
// packed block is put together (or taken apart) in LDS and moves to and from memory
// in one contiguous piece; where only some positions are listed, their words and
// bytes move one by one and the others are not touched.  Bound by memory: 32 layers of 8
// heads, 5000 positions, 4 bits (839 MB) 159 us packed and 139 us read back, 5.3 and
// 6.0 TB/s (a large copy 4.9; the packed cache is partly in the last-level cache).  With
// loads that wait for each other and masks for partial rows it was 192 and 178; by one
// row a wavefront, straight to memory, the two took 1960 us.
struct PackedUnit {
    char *block;     // the packed block
    size_t row;      // index of the block's first position among the cache's rows
    const uint32_t *e;
    uint32_t mask;
};
template <int N>
__device__ __forceinline__ PackedUnit pk_unit(const PackedWords<N> &t, int n_docs, int unit, int plane, int block_bytes) {
    PackedUnit u;
    u.e = t.w + pk_find(t, n_docs, PKC_UNIT0, unit) * PK_ENTRY;
    const int i = unit - (int)u.e[PKC_UNIT0];
    int b;
    if (u.e[PKE_REF] == PK_RUN) {
        const int p0 = u.e[PKE_POS], p1 = p0 + (int)u.e[PKC_RUN];
        b = p0 / PK_BLOCK + i;
        const int lo = max(p0 - b * PK_BLOCK, 0), hi = min(p1 - b * PK_BLOCK, PK_BLOCK);
        u.mask = (0xffffffffu >> (32 - (hi - lo))) << lo;
    } else {
        b = t.w[N - u.e[PKE_REF] + 2 * i];
        u.mask = t.w[N - u.e[PKE_REF] + 2 * i + 1];
    }
    u.block = pk_pointer(u.e) + ((size_t)plane * u.e[PKE_BLOCKS] + b) * block_bytes;
    u.row = (size_t)plane * u.e[PKC_NCAP] + (size_t)b * PK_BLOCK;
    return u;
}

// The eight values from dimension d on and the eight 16 further, zeros behind hd; vec: hd
// is a multiple of 8 (rows are then 16-byte aligned).
__device__ __forceinline__ void pk_load16(const float *p, int d, int hd, bool vec, float x[2][8]) {
    if (vec) {
        f32x4 v[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) v[q] = *reinterpret_cast<const f32x4 *>(p + min(d + 16 * (q >> 1), hd - 8) + 4 * (q & 1));
#pragma unroll
        for (int q = 0; q < 4; ++q)
#pragma unroll
            for (int i = 0; i < 4; ++i) x[q >> 1][4 * (q & 1) + i] = d + 16 * (q >> 1) < hd ? v[q][i] : 0.f;
    } else {
#pragma unroll
        for (int i = 0; i < 16; ++i) x[i >> 3][i & 7] = d + i + (i & 8) < hd ? p[d + i + (i & 8)] : 0.f;
    }
}
__device__ __forceinline__ void pk_load16(const bf16_t *p, int d, int hd, bool vec, float x[2][8]) {
    if (vec) {
        u32x4 v[2];
#pragma unroll
        for (int q = 0; q < 2; ++q) v[q] = *reinterpret_cast<const u32x4 *>(p + min(d + 16 * q, hd - 8));
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            const u32x4 u = d + 16 * q < hd ? v[q] : u32x4{0, 0, 0, 0};
#pragma unroll
            for (int i = 0; i < 8; ++i) x[q][i] = __uint_as_float(i & 1 ? u[i >> 1] & 0xffff0000u : u[i >> 1] << 16);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 16; ++i) x[i >> 3][i & 7] = d + i + (i & 8) < hd ? bf16_to_f32(p[d + i + (i & 8)]) : 0.f;
    }
}
__device__ __forceinline__ void pk_store8(float *p, int d, int hd, bool vec, const float *x) {
    if (vec && d < hd) {
#pragma unroll
        for (int q = 0; q < 2; ++q)
            *reinterpret_cast<f32x4 *>(p + d + 4 * q) = f32x4{x[4 * q], x[4 * q + 1], x[4 * q + 2], x[4 * q + 3]};
    } else if (!vec) {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (d + i < hd) p[d + i] = x[i];
    }
}
__device__ __forceinline__ void pk_store8(bf16_t *p, int d, int hd, bool vec, const float *x) {
    if (vec && d < hd) {
        u32x4 v;
#pragma unroll
        for (int q = 0; q < 4; ++q)
            v[q] = __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{x[2 * q], x[2 * q + 1]}, bf16x2));
        // a line leaves in one instruction and is not read again here: past the caches
        // (28 layers of 4-bit codes, 4 heads, 5000 positions: 84 -> 56 us a call, 52 now, 7.0 TB/s)
        __builtin_nontemporal_store(v, reinterpret_cast<u32x4 *>(p + d));
    } else if (!vec) {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (d + i < hd) p[d + i] = f32_to_bf16(x[i]);
    }
}

// FULL: hd is HP.
template <typename T, int HP, int BITS, bool UNPACK, bool FULL, int N>
__global__ __launch_bounds__(256) void packed_copy_kernel(PackedWords<N> t, int n_docs, int n_units, int head_dim, int Hkv, int plane0) {
    const int hd = FULL ? HP : head_dim;
    constexpr int GS = HP / PK_GROUP, BB = pk_block_bytes(HP, BITS), CB = pk_code_bytes(HP, BITS);
    constexpr int TPR = HP / 16, TPU = PK_BLOCK * TPR, NU = 256 / TPU;  // lanes of a row, of a unit; units
    __shared__ __attribute__((aligned(16))) char lds[NU][BB];
    const int sub = __builtin_amdgcn_readfirstlane(threadIdx.x / TPU), lt = threadIdx.x % TPU;
    const int r = lt / TPR, j = lt % TPR, d0 = 32 * (j >> 1) + 8 * (j & 1);
    const int unit = min((int)blockIdx.x * NU + sub, n_units - 1);  // a last odd one is done twice, alike
    const int plane = plane0 + blockIdx.y;
    const PackedUnit u = pk_unit(t, n_docs, unit, plane, BB);
    const bool value = plane / Hkv & 1, vec = FULL || hd % 8 == 0, mine = u.mask >> r & 1;
    T *row = (T *)pk_pointer(u.e + PKC_CACHE) + (u.row + r) * hd;
    char *b = lds[sub];
    uint32_t *words = reinterpret_cast<uint32_t *>(b);
    uint32_t *par = reinterpret_cast<uint32_t *>(b + CB) + r * GS + j / 4;  // four lanes to a group
    if constexpr (UNPACK) {
        // slots that no call wrote are not used, though their block is loaded
        for (int i = lt; i < BB / 16; i += TPU)
            reinterpret_cast<u32x4 *>(b)[i] = reinterpret_cast<const u32x4 *>(u.block)[i];
        __syncthreads();
        if (!mine) return;
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            // here a lane takes the eight dimensions 8 j + q HP / 2, so that a store instruction
            // writes whole lines
            const int d1 = q * (HP / 2) + 8 * j;
            const uint32_t w = *reinterpret_cast<const uint32_t *>(b + CB + (r * GS + d1 / PK_GROUP) * 4);
            const float off = __uint_as_float(w & 0xffff0000u), s = __uint_as_float(w << 16);
            float x[8];
            auto element = [&](int i, uint32_t c) {
                x[i] = fmaf(s, (float)(c & ((1u << BITS) - 1)), off);  // (the product is exact: 8 significant bits each)
            };
            int bit;
            if (value) {
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const int at = pk_value_byte(HP, BITS, r, d1 + i, &bit);
                    element(i, (uint32_t)(uint8_t)b[at] >> bit);
                }
            } else {
                const uint32_t *const k = words + (pk_key_byte(HP, BITS, r, d1, &bit) >> 2);
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    element(i, BITS == 8 ? k[i >> 2] >> (8 * (i & 3)) : k[0] >> (16 * (i & 1) + 4 * (i >> 1)));
            }
            pk_store8(row, d1, hd, vec, x);
        }
    } else {
        float x[2][8];
#pragma unroll
        for (int i = 0; i < 16; ++i) x[i >> 3][i & 7] = 0.f;
        if (mine) pk_load16(row, d0, hd, vec, x);
        // the reductions keep a NaN (v_minimum3 / v_maximum3)
        float lo = INFINITY, hi = -INFINITY;
#pragma unroll
        for (int q = 0; q < 2; ++q)
            if (vec ? d0 + 16 * q < hd : true) {
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (vec || d0 + 16 * q + i < hd) {
                        lo = __builtin_elementwise_minimum(lo, x[q][i]);
                        hi = __builtin_elementwise_maximum(hi, x[q][i]);
                    }
            }
#pragma unroll
        for (int o = 1; o < 4; o *= 2) {
            lo = __builtin_elementwise_minimum(lo, __shfl_xor(lo, o, 64));
            hi = __builtin_elementwise_maximum(hi, __shfl_xor(hi, o, 64));
        }
        float off, inv;
        const uint32_t word = group_word<BITS>(lo, hi, true, &off, &inv);
        if ((j & 3) == 0) *par = word;
        float c[2][8];
#pragma unroll
        for (int q = 0; q < 2; ++q)
#pragma unroll
            for (int i = 0; i < 8; ++i) c[q][i] = code_of(x[q][i], off, inv);
        if (hd != HP) {
#pragma unroll
            for (int q = 0; q < 2; ++q)
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (d0 + 16 * q + i >= hd) c[q][i] = 0.f;
        }
        if (inv == 0.f) {  // one value, or NaN
#pragma unroll
            for (int q = 0; q < 2; ++q)
#pragma unroll
                for (int i = 0; i < 8; ++i) c[q][i] = 0.f;
        }
        // codes are put together as floats, which hold 16 bits of them exactly
        if (value) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                int bit;
                if constexpr (BITS == 4) {
                    b[pk_value_byte(HP, BITS, r, d0 + i, &bit)] = (char)low_bits(c[0][i] + 16.f * c[1][i]);
                } else {
#pragma unroll
                    for (int q = 0; q < 2; ++q) b[pk_value_byte(HP, BITS, r, d0 + 16 * q + i, &bit)] = (char)low_bits(c[q][i]);
                }
            }
        } else {
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                int bit;
                uint32_t *w = words + (pk_key_byte(HP, BITS, r, d0 + 16 * q, &bit) >> 2);
                // halves of a word: 4 bits, even and odd dimensions; 8 bits, pairs
                if constexpr (BITS == 4) {
                    uint32_t h[2];
#pragma unroll
                    for (int k = 0; k < 2; ++k)
                        h[k] = low_bits(c[q][k] + 16.f * c[q][2 + k] + 256.f * c[q][4 + k] + 4096.f * c[q][6 + k]);
                    w[0] = __builtin_amdgcn_perm(h[1], h[0], 0x05040100u);
                } else {
#pragma unroll
                    for (int k = 0; k < 2; ++k)
                        w[k] = __builtin_amdgcn_perm(low_bits(c[q][4 * k + 2] + 256.f * c[q][4 * k + 3]),
                                                     low_bits(c[q][4 * k] + 256.f * c[q][4 * k + 1]), 0x05040100u);
                }
            }
        }
        __syncthreads();
        if (u.mask == 0xffffffffu) {
            for (int i = lt; i < BB / 16; i += TPU)
                reinterpret_cast<u32x4 *>(u.block)[i] = reinterpret_cast<const u32x4 *>(b)[i];
            return;
        }
        uint32_t *out = reinterpret_cast<uint32_t *>(u.block);
        for (int i = lt; i < BB / 4; i += TPU) {
            int at = i;  // word of a code
            uint32_t m = 1;
            if (i >= CB / 4) {
                m = u.mask >> ((i - CB / 4) / GS) & 1;
            } else if (!value) {
                at /= (HP / 32) * (BITS / 4);  // [tile][lane group][position]
                m = u.mask >> ((at >> 6) * 16 + (at & 15)) & 1;
            } else {
                const int h = i & 1, g = i / ((HP / 32) * (BITS / 4) * 2) / 16;  // [position group][dimension]
                m = u.mask >> (16 * h + 4 * g) & 15;
                if (m != 15) {
#pragma unroll
                    for (int k = 0; k < 4; ++k)
                        if (m >> k & 1) u.block[4 * i + k] = b[4 * i + k];
                    continue;
                }
            }
            if (m) out[i] = words[i];
        }
    }
}

// One wavefront per (row, head): the sum of the projection's K slices, bias, the
// rotation, then the query operand or a packed row.
template <typename T, int HP, int BITS>
__global__ __launch_bounds__(256) void rope_pack_kernel(const float *qkv, int nsplit, int R, const T *bq, const T *bk,
                                                        const T *bv, const RowInfo *rows, const DocInfo *docs, int layer,
                                                        int Hq, int Hkv, int hd, const float *rcos, const float *rsin,
                                                        T *Q, T *Q_lo) {
    const int r = blockIdx.x, lane = threadIdx.x & 63;
    const int j = blockIdx.y * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);  // query, key, value heads
    if (j >= Hq + 2 * Hkv) return;
    const int N = (Hq + 2 * Hkv) * hd, half = hd >> 1;
    const T *bias = j < Hq ? bq : j < Hq + Hkv ? bk : bv;
    const int b0 = (j < Hq ? j : j < Hq + Hkv ? j - Hq : j - Hq - Hkv) * hd;
    auto load = [&](int d) {
        float s = qkv[(size_t)r * N + j * hd + d];
        for (int q = 1; q < nsplit; ++q) s += qkv[((size_t)q * R + r) * N + j * hd + d];
        return bias ? s + to_f32(bias[b0 + d]) : s;
    };
    const RowInfo ri = rows[r];
    float x[2] = {0.f, 0.f};
#pragma unroll
    for (int g = 0; g < HP / PK_GROUP; ++g) {
        const int d = g * PK_GROUP + lane;
        if (d >= hd) continue;
        const float a = load(d);
        if (j >= Hq + Hkv) {
            x[g] = a;
            continue;
        }
        const bool low = d < half;
        const float b = load(low ? d + half : d - half);
        const int i = low ? d : d - half;
        const float c = rcos[(size_t)ri.pos * half + i], s = rsin[(size_t)ri.pos * half + i];
        x[g] = low ? a * c - b * s : a * c + b * s;
        if (j < Hq) store_operand(Q, Q_lo, (size_t)r * Hq * hd + j * hd + d, x[g]);
    }
    if (j < Hq) return;
    const DocInfo dc = docs[ri.doc];
    constexpr int BB = pk_block_bytes(HP, BITS);
    char *block = (char *)dc.cache + (((size_t)layer * 2 * Hkv + (j - Hq)) * pk_blocks(dc.n_cap) + ri.pos / PK_BLOCK) * BB;
    write_row<HP, BITS>(x, hd, j >= Hq + Hkv, block, ri.pos % PK_BLOCK);
}

}  // namespace

// Runs F<HP, BITS>::go for the layout of (hd, bits).
#define KVR_PACKED_DISPATCH(hd, bits, CALL)                      \
    do {                                                         \
        if (pk_width(hd) == 64) {                                \
            if ((bits) == 4) { CALL(64, 4); } else { CALL(64, 8); }   \
        } else {                                                 \
            if ((bits) == 4) { CALL(128, 4); } else { CALL(128, 8); } \
        }                                                        \
    } while (0)

hipError_t launch_packed_append(bool bf16, int bits, const PackedTable &t, int n_docs, int n_rows, const void *k,
                                const void *v, int64_t stride, int layer, int Hkv, int hd, hipStream_t s) {
    if (n_rows <= 0) return hipSuccess;
    if (n_docs < 1 || n_docs > PK_MAX_DOCS || hd > 128 || (bits != 4 && bits != 8)) return hipErrorInvalidValue;
    const dim3 grid(n_rows, (2 * Hkv + 3) / 4);
    pk_with_words(t, n_docs, [&](const auto &words) {
        constexpr int N = sizeof(words) / 4;
#define KVR_CALL(HP, BITS)                                                                                              \
    if (bf16)                                                                                                           \
        kvr_launch((packed_append_kernel<bf16_t, HP, BITS, N>), grid, dim3(256), 0, s, words, n_docs, (const bf16_t *)k, \
                   (const bf16_t *)v, stride, layer, Hkv, hd);                                                          \
    else                                                                                                                \
        kvr_launch((packed_append_kernel<float, HP, BITS, N>), grid, dim3(256), 0, s, words, n_docs, (const float *)k,  \
                   (const float *)v, stride, layer, Hkv, hd)
        KVR_PACKED_DISPATCH(hd, bits, KVR_CALL);
#undef KVR_CALL
    });
    return hipGetLastError();
}

hipError_t launch_packed_copy(bool bf16, int bits, bool unpack, const PackedTable &t, int n_docs, int n_units, int planes,
                              int Hkv, int hd, hipStream_t s) {
    if (n_units <= 0) return hipSuccess;
    if (n_docs < 1 || n_docs > PK_MAX_DOCS || hd > 128 || (bits != 4 && bits != 8)) return hipErrorInvalidValue;
    const int units = pk_width(hd) == 64 ? 2 : 1;
    for (int p0 = 0; p0 < planes; p0 += 32768) {
        const dim3 grid((n_units + units - 1) / units, std::min(planes - p0, 32768));
        pk_with_words(t, n_docs, [&](const auto &words) {
            constexpr int N = sizeof(words) / 4;
#define KVR_COPY(T, HP, BITS, UN)                                                                                              \
    if (hd == HP)                                                                                                              \
        kvr_launch((packed_copy_kernel<T, HP, BITS, UN, true, N>), grid, dim3(256), 0, s, words, n_docs, n_units, hd, Hkv, p0); \
    else                                                                                                                       \
        kvr_launch((packed_copy_kernel<T, HP, BITS, UN, false, N>), grid, dim3(256), 0, s, words, n_docs, n_units, hd, Hkv, p0)
#define KVR_CALL(HP, BITS)                                   \
    if (bf16 && unpack) {                                    \
        KVR_COPY(bf16_t, HP, BITS, true);                    \
    } else if (bf16) {                                       \
        KVR_COPY(bf16_t, HP, BITS, false);                   \
    } else if (unpack) {                                     \
        KVR_COPY(float, HP, BITS, true);                     \
    } else {                                                 \
        KVR_COPY(float, HP, BITS, false);                    \
    }
            KVR_PACKED_DISPATCH(hd, bits, KVR_CALL);
#undef KVR_CALL
#undef KVR_COPY
        });
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

hipError_t launch_rope_pack(bool bf16, int bits, const float *qkv, int nsplit, const void *bq, const void *bk,
                            const void *bv, const RowInfo *rows, const DocInfo *docs, int R, int layer, int Hq, int Hkv,
                            int hd, const float *rope_cos, const float *rope_sin, void *Q, void *Q_lo, hipStream_t s) {
    if (R <= 0) return hipSuccess;
    if (hd > 128 || (bits != 4 && bits != 8)) return hipErrorInvalidValue;
    const dim3 grid(R, (Hq + 2 * Hkv + 3) / 4);
#define KVR_CALL(HP, BITS)                                                                                              \
    if (bf16)                                                                                                           \
        kvr_launch((rope_pack_kernel<bf16_t, HP, BITS>), grid, dim3(256), 0, s, qkv, nsplit, R, (const bf16_t *)bq,     \
                   (const bf16_t *)bk, (const bf16_t *)bv, rows, docs, layer, Hq, Hkv, hd, rope_cos, rope_sin,          \
                   (bf16_t *)Q, (bf16_t *)Q_lo);                                                                        \
    else                                                                                                                \
        kvr_launch((rope_pack_kernel<float, HP, BITS>), grid, dim3(256), 0, s, qkv, nsplit, R, (const float *)bq,       \
                   (const float *)bk, (const float *)bv, rows, docs, layer, Hq, Hkv, hd, rope_cos, rope_sin,            \
                   (float *)Q, (float *)nullptr)
    KVR_PACKED_DISPATCH(hd, bits, KVR_CALL);
#undef KVR_CALL
    return hipGetLastError();
}

}  // namespace kvr
