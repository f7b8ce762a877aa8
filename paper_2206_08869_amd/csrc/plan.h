// What the rules that cut products into tiles (loss_plan.h, orth_plan.h) and the products themselves (products.h) share.
#pragma once
#include <stddef.h>
#include <stdint.h>

namespace iodf {

constexpr int PK = 64;  // of a tile along k

inline long long up(long long n, long long d) { return (n + d - 1) / d * d; }

}  // namespace iodf
