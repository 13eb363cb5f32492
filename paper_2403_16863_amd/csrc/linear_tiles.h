// The tiles that products of linear.hip choose from, and the kernels for them, compiled in parts (linear_kernels.hip).
#pragma once
#include "linear_kernel.h"

namespace linear {

enum Layout { ROWS = 0, ROWS_N = 1, TOKENS = 2 };  // A, B: k along rows of A alone, of both, of neither

template <int I>
struct TileOf;
//                                       BM   BN  BK WM WN WK NB OCC
template <> struct TileOf<0> : Tile<16, 32, 64, 1, 1, 8, 3, 1> {};
template <> struct TileOf<1> : Tile<16, 64, 64, 1, 1, 4, 3, 1> {};
template <> struct TileOf<2> : Tile<32, 64, 64, 1, 2, 2, 3, 2> {};
template <> struct TileOf<3> : Tile<64, 64, 64, 2, 2, 1, 3, 3> {};
template <> struct TileOf<4> : Tile<64, 64, 64, 2, 2, 2, 4, 1> {};
template <> struct TileOf<5> : Tile<96, 64, 64, 2, 2, 2, 3, 1> {};
template <> struct TileOf<6> : Tile<128, 64, 64, 2, 2, 1, 3, 2> {};
template <> struct TileOf<7> : Tile<128, 128, 64, 2, 4, 1, 4, 1> {};
template <> struct TileOf<8> : Tile<128, 128, 64, 2, 4, 1, 2, 2> {};
template <> struct TileOf<9> : Tile<192, 128, 64, 2, 4, 1, 3, 1> {};
template <> struct TileOf<10> : Tile<128, 256, 64, 2, 4, 1, 3, 1> {};
template <> struct TileOf<11> : Tile<192, 256, 64, 2, 4, 1, 2, 1> {};
template <> struct TileOf<12> : Tile<256, 256, 64, 2, 4, 1, 2, 1> {};
template <> struct TileOf<13> : Tile<32, 32, 64, 1, 1, 4, 2, 2> {};
template <> struct TileOf<14> : Tile<16, 16, 64, 1, 1, 8, 4, 1> {};
constexpr int kTiles = 15;

// Kernel of a tile; parts: a range of k into the workspace.
template <int LAYOUT, bool BF>
const void* product_of(int tile, bool parts);

}  // namespace linear
