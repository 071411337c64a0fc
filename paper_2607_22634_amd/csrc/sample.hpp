// How a call of presto_sample is cut, and what its workspace holds.
#pragma once

#include <stddef.h>
#include <stdint.h>

namespace presto {
namespace sample {

constexpr int kGridWords = 3848;  // bins of a slice, padded

// counts (16 bits: a slice has at most 2^15 tokens), weights (fp32; bf16 needs
// one) and two words
constexpr size_t slice_bytes(bool f32) { return (kGridWords * 2 + (f32 ? kGridWords * 8 : 8) + 8 + 15) / 16 * 16; }

}  // namespace sample
}  // namespace presto
