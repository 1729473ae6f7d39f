// nfad_dropout_args.h -- what the dropout kernels are given; plain data, shared by the kernels and the extern "C" boundary.
#pragma once

#include <stddef.h>
#include <stdint.h>

namespace nfad {

template <class T> struct IsVoid { static constexpr bool value = false; };
template <> struct IsVoid<void> { static constexpr bool value = true; };

struct DropoutArgs {
    const void *x, *other;           // other: without an activation the residual [n], with one the bias [cols]; or null
    void *y, *slope;                 // slope: with an activation
    size_t n;
    uint32_t cols, row_packets;      // with a bias
    uint64_t seed, offset;
    const unsigned long long* step;  // on the device, added to offset; or null
    uint32_t dropped;                // see kept()
    float scale;
};

}  // namespace nfad
