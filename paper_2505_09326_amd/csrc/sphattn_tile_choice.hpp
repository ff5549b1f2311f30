// The tiles that the products of sphattn_tiles.hpp are launched with, and which of them a launch takes.
#pragma once
#include "sphattn_host.hpp"
#include "sphattn_tiles.hpp"

namespace {

using namespace sphattn;

using Big = Tile<256, 256, 2, 4, 4>;               // eight waves of 128 x 64: one workgroup per CU
using Mid = Tile<128, 128, 2, 2, 4>;               // four of 64 x 64: two per CU

long long up_to(long long x, long long m) { return (x + m - 1) / m * m; }

// The tile of fewest rounds of the CUs' time: a Mid tile takes 0.36 of a Big one's in a CU that runs two of them
bool big_tiles(long long p, long long q)
{
    const long long big = ((p + 255) / 256) * ((q + 255) / 256), mid = ((p + 127) / 128) * ((q + 127) / 128);
    const double big_time = (double)((big + kCus - 1) / kCus), mid_time = 0.72 * (double)((mid + 2 * kCus - 1) / (2 * kCus));
    return big_time <= mid_time;
}

// whether the products can read rows of D elements at p as they are
bool ready(const void* p, int D, Store S) { return S != Store::F32 && !off(p, 16) && D % 8 == 0; }

}  // namespace
