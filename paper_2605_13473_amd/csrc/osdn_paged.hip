// Attention over a paged cache whose rows are of the type of the queries (bf16, fp32).
#include "osdn_decode_tiles.h"

namespace osdn {

template <int K> using RowsBf16 = RowTile<bf16, K>;
template <int K> using RowsF32 = RowTile<float, K>;
int launch_paged_decode(const DecodeArgs &a, bool bf16_io, hipStream_t st) { return bf16_io ? decode_by_width<RowsBf16>(a, st) : decode_by_width<RowsF32>(a, st); }

}  // namespace osdn
