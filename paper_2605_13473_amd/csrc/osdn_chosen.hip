// Attention over chosen pages of a cache, a list of them for each key head.  (Instances of their own: with this decided at run time, attention of one
// sequence over 1531 tokens of the cache took 10.4 us in place of 9.8.)
#include "osdn_decode_tiles.h"

namespace osdn {

template <int K> using RowsBf16 = RowTile<bf16, K, true>;
template <int K> using RowsF32 = RowTile<float, K, true>;
int launch_chosen_decode(const DecodeArgs &a, bool bf16_io, hipStream_t st) { return bf16_io ? decode_by_width<RowsBf16>(a, st) : decode_by_width<RowsF32>(a, st); }

}  // namespace osdn
