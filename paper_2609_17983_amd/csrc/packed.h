// Packed caches: a cache's rows in codes of 4 or 8 bits (layout and rounding are
// stated in include/kvr.h).  Shared by the kernels that write, read and attend
// over them.
#pragma once

#include <algorithm>
#include <atomic>

#include "common.h"

namespace kvr {

constexpr int PK_BLOCK = 32;  // positions of a block
constexpr int PK_GROUP = 64;  // dimensions that share a scale and an offset
constexpr int PK_MAX_SLOTS = 1 << 30;  // of a cache: positions rounded up to a step's stay within 31 bits

// head_dim as the codes hold it
__host__ __device__ constexpr int pk_width(int hd) { return hd <= 64 ? 64 : 128; }
// bytes of a block's codes, and of the block (codes, then a 32-bit word of scale
// and offset per position and group)
__host__ __device__ constexpr int pk_code_bytes(int hp, int bits) { return PK_BLOCK * hp * bits / 8; }
__host__ __device__ constexpr int pk_block_bytes(int hp, int bits) {
    return pk_code_bytes(hp, bits) + PK_BLOCK * (hp / PK_GROUP) * 4;
}
__host__ __device__ constexpr int pk_blocks(int n_cap) { return (n_cap + PK_BLOCK - 1) / PK_BLOCK; }

// Byte of the code of (position r of the block, dimension d), and the bit it
// starts at.  Keys: 16-position tiles, in each [8-dimension group of a step of
// 32][position][step], eight dimensions side by side: what a lane of the score
// product's A operand reads.  Values: [group of four positions][dimension of
// 16][16 dimensions, in 4 bits paired][half of the block], four positions side by
// side: what a lane of the output product's A operand reads.
__host__ __device__ __forceinline__ int pk_key_byte(int hp, int bits, int r, int d, int *bit) {
    const int word = (((r >> 4) * 4 + ((d >> 3) & 3)) * 16 + (r & 15)) * (hp >> 5) + (d >> 5);
    const int j = d & 7;
    if (bits == 8) {
        *bit = 0;
        return word * 8 + j;
    }
    const int nib = (j & 1) * 4 + (j >> 1);  // even dimensions in the low half, odd ones in the high half
    *bit = 4 * (nib & 1);
    return word * 4 + (nib >> 1);
}
__host__ __device__ __forceinline__ int pk_value_byte(int hp, int bits, int r, int d, int *bit) {
    const int lane = ((r >> 2) & 3) * 16 + (d & 15);
    if (bits == 8) {
        *bit = 0;
        return ((lane * (hp >> 4) + (d >> 4)) * 2 + (r >> 4)) * 4 + (r & 3);
    }
    *bit = 4 * ((d >> 4) & 1);
    return ((lane * (hp >> 5) + (d >> 5)) * 2 + (r >> 4)) * 4 + (r & 3);
}

// The documents and positions of one launch, in the kernel's argument (HIP's
// limit is 4 KB), so that a call stages nothing in memory and a captured one
// keeps its own.  Entries of PK_ENTRY words stand at the front, positions at the
// back (from word `tail` on).  What fits PK_FEW_WORDS is passed in as many: 3.6 KB
// of arguments take the host 0.9 us longer a launch, and a call on an idle device
// ends 5 us later (one document of 509 positions: 28 us, 22).
constexpr int PK_WORDS = 896, PK_FEW_WORDS = 64, PK_ENTRY = 12;
constexpr int PK_MAX_DOCS = PK_WORDS / PK_ENTRY;
template <int N>
struct PackedWords {
    alignas(8) uint32_t w[N];
};
struct PackedTable {
    PackedWords<PK_WORDS> words;
    int tail = PK_WORDS;
};
// Words of an entry.  Rows r of an entry are rows ROW0 + r of the launch's row
// arrays; their positions are POS + r (POS >= 0 or -1) when REF is PK_RUN, those of
// the pass's row table when it is PK_ROWS, otherwise the words REF - r before the
// table's end.
enum {
    PKE_PACKED = 0,  // packed cache (two words)
    PKE_BLOCKS = 2,  // its blocks per plane
    PKE_ROW0 = 3,
    PKE_ROWS = 4,
    PKE_REF = 5,
    PKE_POS = 6,
    // attention: first work item and column group of the entry in the launch, key
    // ranges per column group, first partial slot, keys that a row sees at most
    PKE_ITEM0 = 7,
    PKE_CG0 = 8,
    PKE_SPLITS = 9,
    PKE_PART0 = 10,
    PKE_KEYS = 11,
    // copies: the units (blocks with listed positions) of the entry, by the first one's
    // index in the launch; POS and RUN are a run of positions, otherwise the words REF - 2 i
    // before the table's end are unit i's block and the mask of its positions; the cache
    // (two words) and its rows per plane
    PKC_UNIT0 = 3,
    PKC_CACHE = 7,
    PKC_NCAP = 9,
    PKC_RUN = 10,
};
constexpr uint32_t PK_RUN = 0xffffffffu, PK_ROWS = 0xfffffffeu;
// Blocks (attention), rows (append) and units (copies) of a launch at most: enough to
// fill a device many times, and far from the limits of a grid.
constexpr int PK_MAX_GRID = 1 << 15;

// Quantise the listed rows of k and v ([rows][stride] values, heads side by side)
// into one layer's planes of the entries' packed caches.
hipError_t launch_packed_append(bool bf16, int bits, const PackedTable &t, int n_docs, int n_rows, const void *k,
                                const void *v, int64_t stride, int layer, int Hkv, int hd, hipStream_t s);
// Quantise (unpack: read back) the listed positions of every plane.
hipError_t launch_packed_copy(bool bf16, int bits, bool unpack, const PackedTable &t, int n_docs, int n_units, int planes,
                              int Hkv, int hd, hipStream_t s);
// launch_rope_scatter for packed caches: the fresh keys (after the rotation) and
// values are quantised into their documents' caches; q is written row-major.
hipError_t launch_rope_pack(bool bf16, int bits, const float *qkv, int nsplit, const void *bq, const void *bk,
                            const void *bv, const RowInfo *rows, const DocInfo *docs, int R, int layer, int Hq, int Hkv,
                            int hd, const float *rope_cos, const float *rope_sin, void *Q, void *Q_lo, hipStream_t s);

// One attention launch and its combine (attention_packed.h).
struct PackedAttnArgs {
    const void *q, *q_lo;   // [rows][q_stride]; q_lo: low parts of a compensated pair, or null
    int64_t q_stride;
    void *out, *out_lo;     // [rows][out_stride], or operand order (o_perm)
    int64_t out_stride;
    int32_t o_perm;
    const RowInfo *rows;    // the pass's row table (PK_ROWS), or null
    float *part;
    int32_t layer, Hq, Hkv, hd;
    int32_t n_docs, n_items, n_cg;
    int32_t range;          // keys of a key range (a multiple of a step's)
    int32_t max_splits;     // largest number of key ranges of a document
    // set by the launchers (a block's start is latency: no divisions there that the host
    // can make): Hq / Hkv, log2(e) / sqrt(hd), base-2 logarithms of a block's wavefronts
    // and of its column tiles, and whether rows can be moved in vectors
    int32_t G;
    float scale;
    int32_t waves_log, cw_log;
    int32_t q_vec, o_vec;
};
// A block of `waves` wavefronts: cw of them hold a column tile each, with the columns
// (row, query head of the kv head's group) `copies` times in it; the waves / cw
// wavefronts of a tile take alternate key blocks.  rows: the kernel for many rows
// (attention_packed_rows.hip), whose wavefronts hold PR_TILES column tiles each and go
// through the keys together.
struct PackedShape { int cw, copies, waves; bool rows; };
constexpr int PR_WAVES = 8, PR_TILES = 2;
constexpr PackedShape PACKED_ROWS = {PR_WAVES, 1, PR_WAVES, true};
constexpr int pk_cols(PackedShape s) { return 16 / s.copies * s.cw * (s.rows ? PR_TILES : 1); }
constexpr int PK_WAVES_MAX = 8;
constexpr int pk_part_row(int hd) { return pk_width(hd) + 4; }
// resident given: nothing is launched, and it receives the number of blocks that a
// compute unit holds at a time (only hd and q_lo of `a` are looked at).
hipError_t launch_attention_packed(bool bf16, int bits, PackedShape sh, const PackedTable &t, const PackedAttnArgs &a,
                                   hipStream_t s, int *resident = nullptr);
// The number of blocks of `waves` wavefronts with `lds` bytes that a compute unit holds
// at a time, the same on every device.  `known`: the answers so far, by waves / 4 - 1.
template <typename K>
inline hipError_t pk_resident(K kernel, int waves, size_t lds, std::atomic<int> *known, int *resident) {
    int n = known[waves / 4 - 1].load(std::memory_order_relaxed);
    if (n == 0) {
        const hipError_t e = hipOccupancyMaxActiveBlocksPerMultiprocessor(&n, kernel, 64 * waves, lds);
        if (e != hipSuccess) return e;
        if (n < 1) n = 1;
        known[waves / 4 - 1].store(n, std::memory_order_relaxed);
    }
    *resident = n;
    return hipSuccess;
}
hipError_t launch_attention_packed_combine(bool bf16, PackedShape sh, const PackedTable &t, const PackedAttnArgs &a,
                                           hipStream_t s);

#ifdef __HIPCC__
// Entry of a launch that holds index `x`: the last one whose word `word` is not
// above it.  Every lane looks at one entry, so the search is one load deep.
template <int N>
__device__ __forceinline__ int pk_find(const PackedWords<N> &t, int n_docs, int word, int x) {
    if (n_docs == 1) return 0;
    const int lane = threadIdx.x & 63;
    constexpr int B = (N / PK_ENTRY + 63) / 64;
    int v[B], n = 0;
#pragma unroll
    for (int b = 0; b < B; ++b) v[b] = (int)t.w[min(b * 64 + lane, n_docs - 1) * PK_ENTRY + word];
#pragma unroll
    for (int b = 0; b < B; ++b) n += __popcll(__ballot(b * 64 + lane < n_docs && v[b] <= x));
    return __builtin_amdgcn_readfirstlane(n - 1);
}
// An attention entry, as its words stand in the table.
struct PackedEntry {
    const char *packed;
    int32_t blocks, row0, rows;
    uint32_t ref;
    int32_t pos, item0, cg0, splits, part0, keys;
};
static_assert(sizeof(PackedEntry) == PK_ENTRY * 4, "entry words");
// The entry that holds index x.  The first one is loaded with the arguments, so that
// the usual launch of one document has no second round trip.
template <int N>
__device__ __forceinline__ PackedEntry pk_entry(const PackedWords<N> &t, int n_docs, int word, int x) {
    PackedEntry e = *reinterpret_cast<const PackedEntry *>(t.w);
    if (n_docs > 1) e = *reinterpret_cast<const PackedEntry *>(t.w + pk_find(t, n_docs, word, x) * PK_ENTRY);
    return e;
}
template <int N>
__device__ __forceinline__ int pk_position(const PackedWords<N> &t, const PackedEntry &e, int r, const RowInfo *rows) {
    if (e.ref == PK_RUN) return e.pos + r;
    if (e.ref == PK_ROWS) return rows[e.row0 + r].pos;
    return (int)t.w[N - e.ref + r];
}
__device__ __forceinline__ char *pk_pointer(const uint32_t *e) {
    // (into device memory: its accesses need not be those of any address)
    return (char *)(__attribute__((address_space(1))) char *)(((uint64_t)e[1] << 32) | e[0]);
}
// Position of row r of entry e of an append.
template <int N>
__device__ __forceinline__ int pk_position(const PackedWords<N> &t, const uint32_t *e, int r) {
    return e[PKE_REF] == PK_RUN ? (int)e[PKE_POS] + r : (int)t.w[N - e[PKE_REF] + r];
}
// launch(words) with the words that a launch's table needs.
template <typename Launch>
inline void pk_with_words(const PackedTable &t, int n_docs, Launch launch) {
    const int front = n_docs * PK_ENTRY, back = PK_WORDS - t.tail;
    if (front + back > PK_FEW_WORDS) {
        launch(t.words);
        return;
    }
    PackedWords<PK_FEW_WORDS> few;
    std::copy(t.words.w, t.words.w + front, few.w);
    std::copy(t.words.w + t.tail, t.words.w + PK_WORDS, few.w + PK_FEW_WORDS - back);
    launch(few);
}
#endif

}  // namespace kvr
