// Both halves of attention behind shared prefixes in one launch, caches of 8-bit codes.
#include "vq_attention_halves.hpp"

namespace vq {
template int launch_attention_halves<true>(const KvParams &, const AttentionParams &, const Split &, const Split &, const Prefixes &, const HalvesGrid &, bool, hipStream_t);
}
