// Attention over packed caches: the 128-wide part, the combine of split key ranges
// and the launchers.
#include <algorithm>

#include "attention_packed.h"

namespace kvr {

namespace {

// Joins the partials of a column's key ranges.  HP / 4 lanes read a partial; a column's
// WC wavefronts take WC * 256 / HP ranges at a time, UN of them in flight, each group
// keeps a running maximum, and the groups are joined through LDS.
template <typename T, int HP, int WC, int N>
__global__ __launch_bounds__(256) void attention_packed_combine_kernel(PackedAttnArgs a, PackedWords<N> t, int cols_log) {
    constexpr int L = HP / 4, GR = 64 / L, UN = 4;
    __shared__ float red[4][64][6];
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), kvh = blockIdx.y;
    const int x = blockIdx.x * (4 / WC) + w / WC;  // column of the launch
    const int cols = 1 << cols_log, cgx = min(x >> cols_log, a.n_cg - 1), cc = x & (cols - 1);
    const PackedEntry e = pk_entry(t, a.n_docs, PKE_CG0, cgx);
    const int G = a.G, c = (cgx - e.cg0) * cols + cc;
    const int ns = x >> cols_log < a.n_cg && c < e.rows * G ? e.splits : 1;
    // (the same for all wavefronts of a column; with WC > 1 of the block)
    float m = -INFINITY, l = 0.f;
    f32x4 y = {0.f, 0.f, 0.f, 0.f};
    if (ns > 1) {
        const size_t step = (size_t)a.Hkv * cols * (HP + 4);
        const float *p = a.part + (((size_t)(e.part0 + (cgx - e.cg0) * ns) * a.Hkv + kvh) * cols + cc) * (HP + 4);
        const int d = (lane % L) * 4, first = (w % WC) * GR + lane / L;
        for (int i0 = first; i0 < ns; i0 += UN * WC * GR) {
            f32x4 v[UN];
            float mi[UN], li[UN];
#pragma unroll
            for (int u = 0; u < UN; ++u) {
                const float *q = p + (size_t)min(i0 + u * WC * GR, ns - 1) * step;
                v[u] = *reinterpret_cast<const f32x4 *>(q + d);
                mi[u] = q[HP];
                li[u] = q[HP + 1];
            }
#pragma unroll
            for (int u = 0; u < UN; ++u) {
                if (i0 + u * WC * GR >= ns) continue;
                const float all = fmaxf(m, mi[u]), f0 = pk_weight(m, all), f1 = pk_weight(mi[u], all);
                m = all;
                l = l * f0 + li[u] * f1;
                y = y * f0 + v[u] * f1;
            }
        }
    }
    // the groups of lanes, then the wavefronts
#pragma unroll
    for (int o = L; o < 64; o *= 2) {
        const float m1 = __shfl_xor(m, o, 64), l1 = __shfl_xor(l, o, 64), all = fmaxf(m, m1);
        const float f0 = pk_weight(m, all), f1 = pk_weight(m1, all);
        m = all;
        l = l * f0 + l1 * f1;
#pragma unroll
        for (int i = 0; i < 4; ++i) y[i] = y[i] * f0 + __shfl_xor(y[i], o, 64) * f1;
    }
    if constexpr (WC > 1) {
        float *r = red[w][lane];
#pragma unroll
        for (int i = 0; i < 4; ++i) r[i] = y[i];
        r[4] = m;
        r[5] = l;
        __syncthreads();
        if (w > 0) return;
#pragma unroll
        for (int k = 1; k < WC; ++k) {
            const float *q = red[k][lane];
            const float all = fmaxf(m, q[4]), f0 = pk_weight(m, all), f1 = pk_weight(q[4], all);
            m = all;
            l = l * f0 + q[5] * f1;
#pragma unroll
            for (int i = 0; i < 4; ++i) y[i] = y[i] * f0 + q[i] * f1;
        }
    }
    const int d = (lane % L) * 4;
    if (ns <= 1 || lane >= L || d >= a.hd) return;
    const int r = c / G, h = kvh * G + c - r * G;
    pk_store<T>(a, (int64_t)e.row0 + r, h * a.hd + d, min(4, a.hd - d), a.o_vec, y * (l == 0.f ? 0.f : 1.0f / l));
}

}  // namespace

hipError_t launch_attention_packed64(bool bf16, int bits, PackedShape sh, const PackedTable &t, const PackedAttnArgs &a,
                                     hipStream_t s, int *resident);
hipError_t launch_attention_packed_rows(int bits, const PackedTable &t, const PackedAttnArgs &a, hipStream_t s, int *resident);

hipError_t launch_attention_packed(bool bf16, int bits, PackedShape sh, const PackedTable &t, const PackedAttnArgs &args,
                                   hipStream_t s, int *resident) {
    const PackedAttnArgs a = pk_complete(bf16, sh, args);
    if (!resident && a.n_items <= 0) return hipSuccess;
    if (a.hd > 128 || (bits != 4 && bits != 8) || (!resident && a.n_docs < 1) || a.n_docs > PK_MAX_DOCS || a.range % PK_BLOCK != 0)
        return hipErrorInvalidValue;
    if (sh.rows) return bf16 ? launch_attention_packed_rows(bits, t, a, s, resident) : hipErrorInvalidValue;
    // (a step is two blocks where a tile holds four copies)
    if (sh.cw < 1 || sh.waves % sh.cw != 0 || (sh.waves != 4 && sh.waves != 8) ||
        (sh.copies != 1 && sh.copies != 2 && sh.copies != 4) || (sh.copies > 1 && sh.cw > 1) ||
        a.range % (PK_BLOCK * (sh.copies == 4 ? 2 : 1)) != 0)
        return hipErrorInvalidValue;
    return pk_width(a.hd) == 64 ? launch_attention_packed64(bf16, bits, sh, t, a, s, resident)
                                : pk_launch_width<128>(bf16, bits, sh, t, a, s, resident);
}

hipError_t launch_attention_packed_combine(bool bf16, PackedShape sh, const PackedTable &t, const PackedAttnArgs &args,
                                           hipStream_t s) {
    const int cols = pk_cols(sh), cols_log = pk_log(cols);
    const PackedAttnArgs a = pk_complete(bf16, sh, args);
    const int wc = a.max_splits > 8 ? 4 : 1;
    const dim3 grid((unsigned)(((size_t)a.n_cg * cols * wc + 3) / 4), a.Hkv);
    pk_with_words(t, a.n_docs, [&](const auto &words) {
        constexpr int N = sizeof(words) / 4;
#define KVR_COMBINE(T, HP)                                                                                                      \
    do {                                                                                                                        \
        if (wc == 4) kvr_launch((attention_packed_combine_kernel<T, HP, 4, N>), grid, dim3(256), 0, s, a, words, cols_log); \
        else kvr_launch((attention_packed_combine_kernel<T, HP, 1, N>), grid, dim3(256), 0, s, a, words, cols_log);         \
    } while (0)
        if (pk_width(a.hd) == 64) {
            if (bf16) KVR_COMBINE(bf16_t, 64);
            else KVR_COMBINE(float, 64);
        } else {
            if (bf16) KVR_COMBINE(bf16_t, 128);
            else KVR_COMBINE(float, 128);
        }
#undef KVR_COMBINE
    });
    return hipGetLastError();
}

}  // namespace kvr
