// Attention over packed caches: the 128-wide part, the combine of split key ranges
// and the launchers.
#include <algorithm>

#include "attention_packed.h"

namespace kvr {

namespace {

// Joins the partials of a column group's key ranges: a wavefront per column.
template <typename T, int HP>
__global__ __launch_bounds__(256) void attention_packed_combine_kernel(PackedTable t, PackedAttnArgs a, int cols, int o_vec) {
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), kvh = blockIdx.y;
    const int tiles = cols / 16, x = blockIdx.x / tiles;
    const uint32_t *e = t.w + pk_find(t, a.n_docs, PKE_CG0, x) * PK_ENTRY;
    const int ns = e[PKE_SPLITS], cg = x - (int)e[PKE_CG0], G = a.Hq / a.Hkv;
    if (ns <= 1) return;
    const int ncols = (int)e[PKE_ROWS] * G;
    for (int k = w; k < 16; k += 4) {
        const int cc = (blockIdx.x % tiles) * 16 + k, c = cg * cols + cc;
        if (c >= ncols) return;
        const size_t step = (size_t)a.Hkv * cols * (HP + 4);
        const float *p = a.part + (((size_t)((int)e[PKE_PART0] + cg * ns) * a.Hkv + kvh) * cols + cc) * (HP + 4);
        // the ranges' maxima and sums, one range a lane
        float mx = -INFINITY;
        for (int i = lane; i < ns; i += 64) mx = fmaxf(mx, p[i * step + HP]);
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) mx = fmaxf(mx, __shfl_xor(mx, o, 64));
        float l = 0.f;
        for (int i = lane; i < ns; i += 64) l += p[i * step + HP + 1] * pk_weight(p[i * step + HP], mx);
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) l += __shfl_xor(l, o, 64);
        const float inv = l == 0.f ? 0.f : 1.0f / l;
        // the outputs: half a wavefront (64 wide: a quarter) takes every other (fourth) range
        constexpr int L = HP / 4, PARTS = 64 / L;
        const int d = (lane % L) * 4, part = lane / L;
        f32x4 y = {0.f, 0.f, 0.f, 0.f};
        for (int i = part; i < ns; i += PARTS)
            y += *reinterpret_cast<const f32x4 *>(p + i * step + d) * pk_weight(p[i * step + HP], mx);
#pragma unroll
        for (int o = 32; o >= L; o >>= 1)
#pragma unroll
            for (int i = 0; i < 4; ++i) y[i] += __shfl_xor(y[i], o, 64);
        if (part == 0 && d < a.hd) {
            const int r = c / G, h = kvh * G + c - r * G;
            pk_store<T>(a, (int64_t)e[PKE_ROW0] + r, h * a.hd + d, min(4, a.hd - d), o_vec, y * inv);
        }
    }
}

}  // namespace

hipError_t launch_attention_packed64(bool bf16, int bits, PackedShape sh, const PackedTable &t, const PackedAttnArgs &a,
                                     hipStream_t s);

hipError_t launch_attention_packed(bool bf16, int bits, PackedShape sh, const PackedTable &t, const PackedAttnArgs &a,
                                   hipStream_t s) {
    if (a.n_items <= 0) return hipSuccess;
    if (a.hd > 128 || (bits != 4 && bits != 8) || a.n_docs > PK_MAX_DOCS || sh.nt != 1 ||
        (sh.cw != 1 && sh.cw != 2 && sh.cw != 4) || a.range % PK_BLOCK != 0)
        return hipErrorInvalidValue;
    return pk_width(a.hd) == 64 ? launch_attention_packed64(bf16, bits, sh, t, a, s)
                                : pk_launch_width<128>(bf16, bits, sh, t, a, s);
}

hipError_t launch_attention_packed_combine(bool bf16, PackedShape sh, const PackedTable &t, const PackedAttnArgs &a,
                                           hipStream_t s) {
    const int cols = pk_cols(sh);
    const dim3 grid(a.n_cg * (cols / 16), a.Hkv);
    const size_t es = bf16 ? 2 : 4;
    const int o_vec = a.hd % 4 == 0 && a.out_stride % 4 == 0 && ((uintptr_t)a.out & (4 * es - 1)) == 0 &&
                      ((uintptr_t)a.out_lo & (4 * es - 1)) == 0;
    if (pk_width(a.hd) == 64) {
        if (bf16) kvr_launch((attention_packed_combine_kernel<bf16_t, 64>), grid, dim3(256), 0, s, t, a, cols, o_vec);
        else kvr_launch((attention_packed_combine_kernel<float, 64>), grid, dim3(256), 0, s, t, a, cols, o_vec);
    } else {
        if (bf16) kvr_launch((attention_packed_combine_kernel<bf16_t, 128>), grid, dim3(256), 0, s, t, a, cols, o_vec);
        else kvr_launch((attention_packed_combine_kernel<float, 128>), grid, dim3(256), 0, s, t, a, cols, o_vec);
    }
    return hipGetLastError();
}

}  // namespace kvr
