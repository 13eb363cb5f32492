// One layout and type of the products of linear.hip: LINEAR_PART / 2 names the layout, LINEAR_PART % 2 the type.
#include "linear_tiles.h"

namespace linear {

constexpr int kLayout = LINEAR_PART / 2;
constexpr bool kBf = LINEAR_PART % 2;
using Type = std::conditional_t<kBf, BF16, F16>;

template <int I>
static const void* pick(int tile, bool parts) {
    if constexpr (I < kTiles) {
        if (tile != I) return pick<I + 1>(tile, parts);
        return parts ? (const void*)product_kernel<Type, TileOf<I>, kLayout != TOKENS, kLayout == ROWS_N, true>
                     : (const void*)product_kernel<Type, TileOf<I>, kLayout != TOKENS, kLayout == ROWS_N, false>;
    }
    return nullptr;
}

template <>
const void* product_of<kLayout, kBf>(int tile, bool parts) { return pick<0>(tile, parts); }

}  // namespace linear
