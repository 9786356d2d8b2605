// Both halves of attention behind shared prefixes in one launch, caches of 16-bit numbers.
#include "vq_attention_halves.hpp"

namespace vq {
template int launch_attention_halves<false>(const KvParams &, const AttentionParams &, const Split &, const Split &, const Prefixes &, const HalvesGrid &, bool, hipStream_t);
}
