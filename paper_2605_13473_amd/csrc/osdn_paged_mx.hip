// Attention over a paged cache in 4 bits.
#include "osdn_decode_tiles.h"
#include "osdn_plan.h"

namespace osdn {

template <int K> using Fp4Bf16 = Fp4Tile<bf16, K, true>;
template <int K> using Fp4F32 = Fp4Tile<float, K, true>;
template <int K> using Fp4Bf16Any = Fp4Tile<bf16, K, false>;
template <int K> using Fp4F32Any = Fp4Tile<float, K, false>;
template <typename T, int K> using Once = Fp4Tile<T, K, true, false, true>;
int launch_paged_decode_mx(const DecodeArgs &a, bool bf16_io, hipStream_t st) {
    const int span = a.window && a.window < a.max_length ? a.window : a.max_length;
    if (a.regular && decode_mx_once((long long)a.B * a.Hk * span, a.K, a.cache_k.token, false)) {
        if (a.K == 64) bf16_io ? decode_of<Once<bf16, 64>>(a, st) : decode_of<Once<float, 64>>(a, st);
        else bf16_io ? decode_of<Once<bf16, 128>>(a, st) : decode_of<Once<float, 128>>(a, st);
        return 0;
    }
    if (a.regular) return bf16_io ? decode_by_width<Fp4Bf16>(a, st) : decode_by_width<Fp4F32>(a, st);
    return bf16_io ? decode_by_width<Fp4Bf16Any>(a, st) : decode_by_width<Fp4F32Any>(a, st);
}

}  // namespace osdn
