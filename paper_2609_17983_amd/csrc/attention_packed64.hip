// The 64-wide part of the attention over packed caches.
#include "attention_packed.h"

namespace kvr {

hipError_t launch_attention_packed64(bool bf16, int bits, PackedShape sh, const PackedTable &t, const PackedAttnArgs &a,
                                     hipStream_t s, int *resident) {
    return pk_launch_width<64>(bf16, bits, sh, t, a, s, resident);
}

}  // namespace kvr
