// What the host side of the operators of language models shares: limits, checks of arguments, the zeros that stand for a missing bias.
#pragma once
#include <cstdint>
#include <initializer_list>

#include "../../include/bolt.h"
#include "bolt_device.hpp"

namespace bolt {

// Eight zeros on the current device; null where their address cannot be had (csrc/moe_api.hip).
const half_t* no_bias();

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
inline int64_t round_up(int64_t v, int64_t to) { return (v + to - 1) / to * to; }
inline int64_t blocks_of(int64_t v, int64_t by) { return (v + by - 1) / by; }
// Whether an output starts where one of the others does.  (Further than that two strided views of one buffer may mesh without sharing an element.)
inline bool starts_at(const void* out, std::initializer_list<const void*> others) {
  for (const void* at : others)
    if (out && out == at) return true;
  return false;
}
inline bool known_act(int a) { return a >= BOLT_ACT_NONE && a <= BOLT_ACT_SILU; }
inline bolt_status status_of(hipError_t e) { return e == hipSuccess ? BOLT_OK : BOLT_ERR_LAUNCH; }
constexpr int kMaxLength = 1 << 21;  // of a row, as in the other operators
// Rows and slots: the kernels count them in 32 bits, as far as the end of the last workgroup's share and one stride past it.
constexpr int64_t kMaxRows = (1ll << 31) - (1 << 16);
// Threads of a launch: the runtime counts them in 32 bits.  No workgroup whose number grows with the rows has more than 512.
inline bool launches(int64_t blocks) { return blocks <= UINT32_MAX / 512; }

}  // namespace bolt
