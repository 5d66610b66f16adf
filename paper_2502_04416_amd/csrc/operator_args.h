// Checks of the arguments that the norm, dropout and adapter entry points share (host code).
#pragma once
#include <cmath>
#include <cstdint>
#include <initializer_list>

#include "../../include/cmoe.h"
#include "cmoe_internal.h"
#include "dropout_device.h"

namespace cmoe {

// A buffer of a call: its name in messages, address (null: not given) and bytes.  In place: an output may be the very buffer of an input
// where both say so, which they may if every element of the output is written by the thread that has read it, and by then nothing
// else reads it.  Not what several rows read (weights), nor statistics, gradients of weights or workspaces.
struct Operand {
  const char* name;
  const void* ptr;
  uint64_t bytes;
  size_t align;
  bool in_place = false;
};

inline bool overlap(const Operand& a, const Operand& b) {
  const uint64_t pa = (uint64_t)(uintptr_t)a.ptr, pb = (uint64_t)(uintptr_t)b.ptr;
  return a.ptr && b.ptr && pa < pb + b.bytes && pb < pa + a.bytes;
}

// 0, or the code of a failure that has been recorded.  No output may overlap another or, but in place, an input.
inline int check_operands(const char* what, std::initializer_list<Operand> inputs, std::initializer_list<Operand> outputs) {
  for (const auto* list : {&inputs, &outputs})
    for (const Operand& o : *list)
      if ((uint64_t)(uintptr_t)o.ptr % o.align != 0) return fail(CMOE_EINVAL, "%s: %s is not aligned to %d bytes", what, o.name, (int)o.align);
  for (const Operand& o : outputs) {
    for (const Operand& i : inputs)
      if (overlap(o, i) && !(o.in_place && i.in_place && o.ptr == i.ptr && o.bytes == i.bytes))
        return fail(CMOE_EINVAL, "%s: %s overlaps %s", what, o.name, i.name);
    for (const Operand& q : outputs)
      if (&q != &o && overlap(o, q)) return fail(CMOE_EINVAL, "%s: %s overlaps %s", what, o.name, q.name);
  }
  return CMOE_OK;
}

// p in [0, 1] rounded to 1 / 65536 (half to even).
inline int make_drop(const char* what, double p, uint64_t seed, uint64_t offset, Drop* out) {
  if (!(p >= 0.0 && p <= 1.0)) return fail(CMOE_EINVAL, "%s: the dropout rate is not in [0, 1]", what);
  const uint32_t limit = (uint32_t)std::nearbyint(p * 65536.0);
  out->k0 = (uint32_t)seed;
  out->k1 = (uint32_t)(seed >> 32);
  out->o0 = (uint32_t)offset;
  out->o1 = (uint32_t)(offset >> 32);
  out->limit = limit;
  out->scale = limit < 65536u ? (float)(65536.0 / (65536 - limit)) : 0.0f;
  return CMOE_OK;
}

}  // namespace cmoe
