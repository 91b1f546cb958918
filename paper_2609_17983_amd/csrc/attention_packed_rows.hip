// Attention of many rows over packed caches (bf16 models): a prompt, the rows of a
// repair.
//
// With hundreds of columns the work per column counts, and of attention_packed.h's
// kernel most of it is scales: two products and two sums per key and group of 64
// dimensions, in every column.  Here a block of eight wavefronts goes through the
// keys together: each 32-key block is read once, its values m + s c are put into LDS
// as compensated bf16 pairs (hi + lo, 16 significant bits, in the order of the matrix
// operands, so every access is one contiguous piece), and all wavefronts' columns
// use them.  A column then costs its exponentials and the matrix products: scores
// K_hi Q + K_lo Q (a compensated query: + K_hi Q_lo), outputs V_hi P_hi + V_hi P_lo +
// V_lo P_hi.
//
// The pairs are double buffered, one barrier per block of keys; the packed words of
// the block after the next are in flight meanwhile.  Matrix and vector instructions
// bound it together: over a prompt of 4000 tokens (32 heads of 8, 4 bits, 290 us) the
// matrix units are busy half of the time and the vector units 45 %.  Without the
// staging it would take 227 us, with one output product of three 240, without its LDS
// reads 258, without exponentials 263.  Operands read further ahead (313) and staging put
// between the matrix instructions (up to 312) were slower.  Zero times a value that is not
// finite is not zero, so such values are staged as zeros and flagged, and the rows
// that see their slot get NaN afterwards.
#include "attention_packed.h"

namespace kvr {

namespace {

// Eight values as a pair of operands.
__device__ __forceinline__ void pr_split(const float v[8], u32x4 *hi, u32x4 *lo) {
    bf16x8 p[2];
    pk_pieces<2>(v, p);
    *hi = __builtin_bit_cast(u32x4, p[0]);
    *lo = __builtin_bit_cast(u32x4, p[1]);
}

template <int HP, int BITS, int QP>
__global__ __launch_bounds__(64 * PR_WAVES) void attention_packed_rows_kernel(PackedAttnArgs a, PackedWords<PK_WORDS> t) {
    constexpr int KS = HP / 32, GS = HP / PK_GROUP, DT = HP / 16, BB = pk_block_bytes(HP, BITS), CB = pk_code_bytes(HP, BITS);
    constexpr int NT = PR_TILES, COLS = pk_cols(PACKED_ROWS);
    // operands of a key block: keys [16-key tile][step][lane], values [16-dimension tile][lane]
    constexpr int KU = 2 * KS, VU = DT;
    static_assert(KU == VU && KU + VU == (HP == 128 ? 2 : 1) * PR_WAVES, "operands of a block over the wavefronts");
    extern __shared__ u32x4 lds[];               // [buffer][hi, lo][operand][lane], flags [buffer][group], tops
    constexpr int BUF = 2 * (KU + VU) * 64;
    int *const flags = reinterpret_cast<int *>(lds + 2 * BUF);

    const int lane = threadIdx.x & 63, g4 = lane >> 4, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    // kv heads first: the longest items of all of them start before the shorter ones
    const int kvh = blockIdx.x;
    const PackedEntry e = pk_entry(t, a.n_docs, PKE_ITEM0, blockIdx.y);
    const int nsplit = e.splits, item = (int)blockIdx.y - e.item0;
    const int split = nsplit == 1 ? 0 : item % nsplit;
    const size_t plane = (size_t)e.blocks * BB;
    const char *kp = e.packed + ((size_t)a.layer * 2 * a.Hkv + kvh) * plane;
    const char *vp = kp + a.Hkv * plane;
    const int last = e.blocks - 1, keys = e.keys;
    const int b0 = split * (a.range / PK_BLOCK);

    // A thread's units of a block: wavefront w makes key operand w and value operand w
    // (128 wide), or one of them (64 wide).
    const bool has_key = HP == 128 || w < KU, has_value = HP == 128 || w >= KU;
    const int ku = w, vu = HP == 128 ? w : w - KU;  // operand index
    uint32_t kword[BITS / 4], vword[2];
    uint32_t kpar;
    u32x4 vpar[2][GS];  // GS words a position: elements 0 and 2 (one group: all) are the operand's group
    auto fetch = [&](int b) {
        const char *kblk = kp + (size_t)min(b, last) * BB, *vblk = vp + (size_t)min(b, last) * BB;
        if (has_key) {
            const int tile = ku / KS, st = ku % KS;
            const uint32_t *p = reinterpret_cast<const uint32_t *>(kblk) + (tile * 64 + lane) * KS * (BITS / 4) + st * (BITS / 4);
#pragma unroll
            for (int i = 0; i < BITS / 4; ++i) kword[i] = p[i];
            kpar = *reinterpret_cast<const uint32_t *>(kblk + CB + ((16 * tile + (lane & 15)) * GS + st / 2) * 4);
        }
        if (has_value) {
            // 4 bits: the words of dimensions 32 (vu / 2) .., of which this operand takes one half
            const uint32_t *p = reinterpret_cast<const uint32_t *>(vblk) + (lane * (BITS == 4 ? KS : DT) + (BITS == 4 ? vu >> 1 : vu)) * 2;
            vword[0] = p[0];
            vword[1] = p[1];
            const uint32_t *q = reinterpret_cast<const uint32_t *>(vblk + CB) + (GS > 1 ? vu / 4 : 0);
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int i = 0; i < GS; ++i) {
                    const uint32_t *r = q + (16 * h + 4 * g4) * GS + 4 * i;
                    if constexpr (GS == 1) {
                        vpar[h][i] = *reinterpret_cast<const u32x4 *>(r);
                    } else {
                        vpar[h][i][0] = r[0];
                        vpar[h][i][2] = r[2];
                    }
                }
        }
    };
    // The fetched block's operands into a buffer.
    auto stage = [&](int buf) {
        u32x4 *const base = lds + buf * BUF;
        if (has_key) {
            float v[8];
            const float s = __uint_as_float(kpar << 16), m = __uint_as_float(kpar & 0xffff0000u);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                // 4 bits: nibble (j%2) * 4 + j/2, in byte 2 (j%2) + j/4
                const uint32_t word = BITS == 4 ? kword[0] >> (4 * (j >> 1 & 1)) & 0x0f0f0f0fu : kword[BITS == 4 ? 0 : j >> 2];
                const int byte = BITS == 4 ? 2 * (j & 1) + (j >> 2) : j & 3;
                v[j] = fmaf(s, (float)(word >> (8 * byte) & 0xffu), m);
            }
            pr_split(v, base + ku * 64 + lane, base + (KU + VU + ku) * 64 + lane);
        }
        if (has_value) {
            float v[8];
            uint32_t t = 0;  // an offset of 2^125 or a scale of 2^119 or more (or NaN) carries into the sign bits
            const uint32_t c4[2] = {BITS == 4 ? vword[0] >> (4 * (vu & 1)) & 0x0f0f0f0fu : vword[0],
                                    BITS == 4 ? vword[1] >> (4 * (vu & 1)) & 0x0f0f0f0fu : vword[1]};
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const int h = j >> 2, i = j & 3;
                const uint32_t u = GS == 1 ? vpar[h][0][i] : vpar[h][i >> 1][2 * (i & 1)];
                v[j] = fmaf(__uint_as_float(u << 16), (float)(c4[h] >> (8 * i) & 0xffu), __uint_as_float(u & 0xffff0000u));
                t |= (u & 0x7f807f80u) + 0x02000500u;
            }
            if (__any((t & 0x80008000u) != 0)) {
                // values that are not finite (or are infinite as bf16), in this lane's slots
                uint32_t slots = 0;
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (!(fabsf(v[j]) < 3.38e38f)) {
                        v[j] = 0.f;
                        slots |= 1u << (16 * (j >> 2) + 4 * g4 + (j & 3));
                    }
                if (slots) atomicOr(&flags[buf * 2 + (GS > 1 ? vu / 4 : 0)], (int)slots);
            }
            pr_split(v, base + (KU + vu) * 64 + lane, base + (KU + VU + KU + vu) * 64 + lane);
        }
    };
    fetch(min(b0, last));

    const int G = a.G, ncols_doc = e.rows * G;
    // column groups from the last one down: later rows see more keys
    const int ncg = (ncols_doc + COLS - 1) / COLS;
    const int cg = ncg - 1 - (nsplit == 1 ? item : item / nsplit);
    const int row0 = e.row0;
    int row[NT], head[NT], limit[NT];
    bool valid[NT];
    bf16x8 qv[NT][QP][KS];
    int top = 0, least = 0x7fffffff;
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        const int c = cg * COLS + (w * NT + n) * 16 + (lane & 15);
        valid[n] = c < ncols_doc;
        row[n] = valid[n] ? c / G : 0;
        head[n] = kvh * G + (valid[n] ? c - row[n] * G : 0);
        limit[n] = valid[n] ? min(pk_position(t, e, row[n], a.rows) + 1, keys) : 0;
        float unused[GS];
        pk_query<bf16_t, HP, QP>(a, row0 + row[n], head[n], g4, a.q_vec, qv[n], unused);
        top = max(top, limit[n]);
        if (valid[n]) least = min(least, limit[n]);
    }
    pk_minmax16(&least, &top);
    // the block's last key: the largest of its wavefronts'
    int *const tops = flags + 4;
    if (lane == 0) tops[w] = top;
    if (threadIdx.x < 4) flags[threadIdx.x] = 0;
    __syncthreads();
    int all_top = 0;
#pragma unroll
    for (int k = 0; k < PR_WAVES; ++k) all_top = max(all_top, tops[k]);
    all_top = __builtin_amdgcn_readfirstlane(all_top);
    const int end = min(all_top, (split + 1) * a.range);
    const int b1 = (end + PK_BLOCK - 1) / PK_BLOCK;

    f32x4 o[NT][DT];
    float m[NT], l[NT];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
#pragma unroll
        for (int d = 0; d < DT; ++d) o[n][d] = f32x4{0.f, 0.f, 0.f, 0.f};
        m[n] = -INFINITY;
        l[n] = 0.f;
    }
    const float sc = a.scale;
    if (b0 < b1) {
        stage(0);
        if (b0 + 1 < b1) fetch(b0 + 1);
    }
    for (int b = b0; b < b1; ++b) {
        const int buf = (b - b0) & 1;
        __syncthreads();  // block b is staged; nobody reads the other buffer any more
        // half of the wavefronts (one of two on a SIMD) stage the next block before their
        // products, half after them: vector and matrix instructions then run side by side
        auto next = [&] {
            if (b + 1 < b1) {
                stage(buf ^ 1);
                if (b + 2 < b1) fetch(b + 2);
            }
        };
        if (w < PR_WAVES / 2) next();
        if (b * PK_BLOCK >= top) {  // none of this wavefront's columns sees it
            if (w >= PR_WAVES / 2) next();
            continue;
        }
        const u32x4 *const base = lds + buf * BUF;
        f32x4 s[NT][2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
#pragma unroll
            for (int n = 0; n < NT; ++n) s[n][h] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int st = 0; st < KS; ++st) {
                const bf16x8 kh = __builtin_bit_cast(bf16x8, base[(h * KS + st) * 64 + lane]);
                const bf16x8 kl = __builtin_bit_cast(bf16x8, base[(KU + VU + h * KS + st) * 64 + lane]);
#pragma unroll
                for (int n = 0; n < NT; ++n) {
#pragma unroll
                    for (int x = 0; x < QP; ++x) s[n][h] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kh, qv[n][x][st], s[n][h], 0, 0, 0);
                    s[n][h] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kl, qv[n][0][st], s[n][h], 0, 0, 0);
                }
            }
        }
        const bool full = (b + 1) * PK_BLOCK <= least;
        bf16x8 pb[NT][2];
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            if (!full) {
                const int key0 = b * PK_BLOCK + 4 * g4;
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int i = 0; i < 4; ++i) s[n][h][i] = key0 + 16 * h + i < limit[n] ? s[n][h][i] : -INFINITY;
            }
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
                for (int d = 0; d < DT; ++d) o[n][d] *= corr;
            }
            const float mu = m[n] == -INFINITY ? 0.f : m[n];
            float p[8];
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    p[4 * h + i] = __builtin_amdgcn_exp2f(fmaf(s[n][h][i], sc, -mu));
                    l[n] += p[4 * h + i];
                }
            pk_pieces<2>(p, pb[n]);
        }
#pragma unroll
        for (int d = 0; d < DT; ++d) {
            const bf16x8 vh = __builtin_bit_cast(bf16x8, base[(KU + d) * 64 + lane]);
            const bf16x8 vl = __builtin_bit_cast(bf16x8, base[(KU + VU + KU + d) * 64 + lane]);
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                o[n][d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vh, pb[n][0], o[n][d], 0, 0, 0);
                o[n][d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vh, pb[n][1], o[n][d], 0, 0, 0);
                o[n][d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vl, pb[n][0], o[n][d], 0, 0, 0);
            }
        }
        // values that are not finite: a buffer's flags are only ever added to; a row that
        // sees a slot of a later block has seen the same slot of the earlier ones too
#pragma unroll
        for (int g = 0; g < GS; ++g) {
            const uint32_t bad = flags[buf * 2 + g];
            if (bad) {
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    const int seen = min(limit[n] - b * PK_BLOCK, PK_BLOCK);
                    if (seen > 0 && (bad & (0xffffffffu >> (32 - seen)))) {
#pragma unroll
                        for (int q = 0; q < 4; ++q)
#pragma unroll
                            for (int i = 0; i < 4; ++i) o[n][4 * g + q][i] = NAN;
                    }
                }
            }
        }
        if (w >= PR_WAVES / 2) next();
    }
    // lane: column lane%16, dimensions 16 d + 4 g4 + i
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        const float sum = pk_sum4(l[n]);
        if (!valid[n]) continue;
        const float inv = sum == 0.f ? 0.f : 1.0f / sum;
        float *part = a.part + (((size_t)(e.part0 + cg * nsplit + split) * a.Hkv + kvh) * COLS +
                                (w * NT + n) * 16 + (lane & 15)) * (HP + 4);
#pragma unroll
        for (int d = 0; d < DT; ++d) {
            const int dim = 16 * d + 4 * g4;
            if (nsplit > 1) *reinterpret_cast<f32x4 *>(part + dim) = o[n][d];
            else if (dim < a.hd) pk_store<bf16_t>(a, row0 + row[n], head[n] * a.hd + dim, min(4, a.hd - dim), a.o_vec, o[n][d] * inv);
        }
        if (nsplit > 1 && g4 == 0) {
            part[HP] = m[n];
            part[HP + 1] = sum;
        }
    }
}

template <int HP, int BITS>
hipError_t pr_launch(const PackedTable &t, const PackedAttnArgs &a, hipStream_t s, int *resident) {
    const dim3 grid(a.Hkv, a.n_items), block(64 * PR_WAVES);
    const uint32_t bytes = 2 * 2 * (HP / 8) * 64 * 16 + (4 + PR_WAVES) * 4;
    static std::atomic<int> known[2][2];
    if (resident)
        return a.q_lo ? pk_resident(attention_packed_rows_kernel<HP, BITS, 2>, PR_WAVES, bytes, known[1], resident)
                      : pk_resident(attention_packed_rows_kernel<HP, BITS, 1>, PR_WAVES, bytes, known[0], resident);
    if (a.q_lo) kvr_launch((attention_packed_rows_kernel<HP, BITS, 2>), grid, block, bytes, s, a, t.words);
    else kvr_launch((attention_packed_rows_kernel<HP, BITS, 1>), grid, block, bytes, s, a, t.words);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_attention_packed_rows(int bits, const PackedTable &t, const PackedAttnArgs &a, hipStream_t s, int *resident) {
    if (pk_width(a.hd) == 64) return bits == 4 ? pr_launch<64, 4>(t, a, s, resident) : pr_launch<64, 8>(t, a, s, resident);
    return bits == 4 ? pr_launch<128, 4>(t, a, s, resident) : pr_launch<128, 8>(t, a, s, resident);
}

}  // namespace kvr
