// Attention over chosen pages of a cache in 4 bits.  Bound by its loads where heads lie side by side: a row of 64 bytes is half of a line, whose other half another head wants only if it
// chose the page too (48 sequences, 32 pages of 64 tokens for each of 8 heads, 107 MB: 44 us; heads apart, where a load takes whole lines, 28).  What of it the halves cost and what the
// scales, 4 bytes of a line a row, was not measured apart.
#include "osdn_decode_tiles.h"
#include "osdn_plan.h"

namespace osdn {

template <int K> using Fp4Bf16 = Fp4Tile<bf16, K, true, true>;
template <int K> using Fp4F32 = Fp4Tile<float, K, true, true>;
template <int K> using Fp4Bf16Any = Fp4Tile<bf16, K, false, true>;
template <int K> using Fp4F32Any = Fp4Tile<float, K, false, true>;
template <typename T, int K> using Once = Fp4Tile<T, K, true, true, true>;
int launch_chosen_decode_mx(const DecodeArgs &a, bool bf16_io, hipStream_t st) {
    if (a.regular && decode_mx_once((long long)a.B * a.Hk * a.max_length, a.K, a.cache_k.token, true)) {
        if (a.K == 64) bf16_io ? decode_of<Once<bf16, 64>>(a, st) : decode_of<Once<float, 64>>(a, st);
        else bf16_io ? decode_of<Once<bf16, 128>>(a, st) : decode_of<Once<float, 128>>(a, st);
        return 0;
    }
    if (a.regular) return bf16_io ? decode_by_width<Fp4Bf16>(a, st) : decode_by_width<Fp4F32>(a, st);
    return bf16_io ? decode_by_width<Fp4Bf16Any>(a, st) : decode_by_width<Fp4F32Any>(a, st);
}

}  // namespace osdn
