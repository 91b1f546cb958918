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

__device__ __forceinline__ float wave_min(float v) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v = fminf(v, __shfl_xor(v, o, 64));
    return v;
}
__device__ __forceinline__ float wave_max(float v) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor(v, o, 64));
    return v;
}

// Scale and offset of a group of finite values within [lo, hi] (not `good`: one of
// them is not finite), and the reciprocal that its codes are made with.
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
template <int BITS>
__device__ __forceinline__ uint32_t code_of(float x, float off, float inv) {
    constexpr float top = (float)((1 << BITS) - 1);
    return (uint32_t)fminf(fmaxf(rintf((x - off) * inv), 0.f), top);
}

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
        float off, inv;
        const uint32_t word = group_word<BITS>(wave_min(real ? x[g] : INFINITY), wave_max(real ? x[g] : -INFINITY), good,
                                               &off, &inv);
        uint32_t c = real && good && inv != 0.f ? code_of<BITS>(x[g], off, inv) : 0;
        int bit;
        if (value) {
            const int at = pk_value_byte(HP, BITS, r, d, &bit);
            if (BITS == 4) c = (c | (__shfl_xor(c, 16, 64) << 4)) & 0xffu;
            if (BITS == 8 || !(lane & 16)) block[at] = (char)c;
        } else {
            // the lanes of a word put their codes together
            const int at = pk_key_byte(HP, BITS, r, d, &bit);
            c <<= 8 * (at & 3) + bit;
#pragma unroll
            for (int o = 1; o < 32 / BITS; o *= 2) c |= __shfl_xor(c, o, 64);
            if ((lane & (32 / BITS - 1)) == 0) *reinterpret_cast<uint32_t *>(block + (at & ~3)) = c;
        }
        if (lane == 0) *reinterpret_cast<uint32_t *>(block + pk_code_bytes(HP, BITS) + (r * GS + g) * 4) = word;
    }
}

// One wavefront per (row, plane): fresh rows of one layer.
template <typename T, int HP, int BITS>
__global__ __launch_bounds__(256) void packed_append_kernel(PackedTable t, int n_docs, const T *k, const T *v,
                                                            int64_t stride, int layer, int Hkv, int hd) {
    const int lane = threadIdx.x & 63, plane = blockIdx.y * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t *first = t.w;
    const int row = (int)first[PKE_ROW0] + blockIdx.x;
    const uint32_t *e = t.w + pk_find(t, n_docs, PKE_ROW0, row) * PK_ENTRY;
    if (plane >= 2 * Hkv) return;
    const bool value = plane >= Hkv;
    const T *src = (value ? v : k) + (size_t)row * stride + (plane - (value ? Hkv : 0)) * hd;
    const float x[2] = {lane < hd ? to_f32(src[lane]) : 0.f, 64 + lane < hd ? to_f32(src[64 + lane]) : 0.f};
    const int p = pk_position(t, e, row - (int)e[PKE_ROW0], nullptr);
    constexpr int BB = pk_block_bytes(HP, BITS);
    char *base = pk_pointer(e) + (((size_t)layer * 2 * Hkv + plane) * e[PKE_BLOCKS] + p / PK_BLOCK) * BB;
    write_row<HP, BITS>(x, hd, value, base, p % PK_BLOCK);
}

// One wavefront per (position, plane) of a cache.
template <typename T, int HP, int BITS, bool UNPACK>
__global__ __launch_bounds__(256) void packed_copy_kernel(PackedTable t, int n_docs, int planes, int hd, int Hkv) {
    constexpr int GS = HP / PK_GROUP, BB = pk_block_bytes(HP, BITS);
    const int lane = threadIdx.x & 63, plane = blockIdx.y * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int row = (int)t.w[PKE_ROW0] + blockIdx.x;
    const uint32_t *e = t.w + pk_find(t, n_docs, PKE_ROW0, row) * PK_ENTRY;
    if (plane >= planes) return;
    const int p = pk_position(t, e, row - (int)e[PKE_ROW0], nullptr);
    char *block = pk_pointer(e) + ((size_t)plane * e[PKE_BLOCKS] + p / PK_BLOCK) * BB;
    T *cache = (T *)pk_pointer(e + PKE_CACHE) + ((size_t)plane * e[PKE_NCAP] + p) * hd;
    const bool value = plane / Hkv & 1;
    const int r = p % PK_BLOCK;
    if constexpr (UNPACK) {
#pragma unroll
        for (int g = 0; g < GS; ++g) {
            const int d = g * PK_GROUP + lane;
            if (d >= hd) continue;
            int bit;
            const int at = value ? pk_value_byte(HP, BITS, r, d, &bit) : pk_key_byte(HP, BITS, r, d, &bit);
            const uint32_t c = ((uint32_t)(uint8_t)block[at] >> bit) & ((1u << BITS) - 1);
            const uint32_t w = *reinterpret_cast<const uint32_t *>(block + pk_code_bytes(HP, BITS) + (r * GS + g) * 4);
            // exact product: 8 significant bits each
            cache[d] = from_f32<T>(__uint_as_float(w & 0xffff0000u) + __uint_as_float(w << 16) * (float)c);
        }
    } else {
        const float x[2] = {lane < hd ? to_f32(cache[lane]) : 0.f, 64 + lane < hd ? to_f32(cache[64 + lane]) : 0.f};
        write_row<HP, BITS>(x, hd, value, block, r);
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
#define KVR_CALL(HP, BITS)                                                                                             \
    if (bf16)                                                                                                          \
        kvr_launch((packed_append_kernel<bf16_t, HP, BITS>), grid, dim3(256), 0, s, t, n_docs, (const bf16_t *)k,      \
                   (const bf16_t *)v, stride, layer, Hkv, hd);                                                         \
    else                                                                                                               \
        kvr_launch((packed_append_kernel<float, HP, BITS>), grid, dim3(256), 0, s, t, n_docs, (const float *)k,        \
                   (const float *)v, stride, layer, Hkv, hd)
    KVR_PACKED_DISPATCH(hd, bits, KVR_CALL);
#undef KVR_CALL
    return hipGetLastError();
}

hipError_t launch_packed_copy(bool bf16, int bits, bool unpack, const PackedTable &t, int n_docs, int n_rows, int planes,
                              int Hkv, int hd, hipStream_t s) {
    if (n_rows <= 0) return hipSuccess;
    if (n_docs < 1 || n_docs > PK_MAX_DOCS || hd > 128 || (bits != 4 && bits != 8)) return hipErrorInvalidValue;
    const dim3 grid(n_rows, (planes + 3) / 4);
#define KVR_CALL(HP, BITS)                                                                                           \
    if (bf16 && unpack)                                                                                              \
        kvr_launch((packed_copy_kernel<bf16_t, HP, BITS, true>), grid, dim3(256), 0, s, t, n_docs, planes, hd, Hkv); \
    else if (bf16)                                                                                                   \
        kvr_launch((packed_copy_kernel<bf16_t, HP, BITS, false>), grid, dim3(256), 0, s, t, n_docs, planes, hd, Hkv); \
    else if (unpack)                                                                                                 \
        kvr_launch((packed_copy_kernel<float, HP, BITS, true>), grid, dim3(256), 0, s, t, n_docs, planes, hd, Hkv);  \
    else                                                                                                             \
        kvr_launch((packed_copy_kernel<float, HP, BITS, false>), grid, dim3(256), 0, s, t, n_docs, planes, hd, Hkv)
    KVR_PACKED_DISPATCH(hd, bits, KVR_CALL);
#undef KVR_CALL
    return hipGetLastError();
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
