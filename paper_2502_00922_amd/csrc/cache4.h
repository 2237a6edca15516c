// The rows of a cache that is held in 4 bits: a token's columns of one key head,
// G groups of 32 neighbouring columns, value = base + scale * (code - 8).
//   16 * G bytes   codes: byte n * G + g has those of columns 32g + 2n (its low
//                  half) and 32g + 2n + 1
//   G pairs        (scale, base) of group g, bf16
//   zeros          up to a multiple of 16 bytes
// The groups' bytes alternate so that both products of the attention get their
// operands from whole loads: 4 * G neighbouring bytes have 8 columns of every
// group, and G neighbouring ones 2 columns of each.
#pragma once
#include "gpu_host.h"

namespace hl {

__host__ __device__ constexpr uint32_t row4_bytes(uint32_t groups) { return (20 * groups + 15) / 16 * 16; }

}  // namespace hl
