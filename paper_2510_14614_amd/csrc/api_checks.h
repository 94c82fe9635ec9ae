// Host-side argument checks shared by the entry points of the C ABI.  Each
// returns NULL or the message of the first argument that does not hold.
#pragma once

#include <cmath>
#include <cstdint>
#include <initializer_list>
#include <string>

#include "../../include/fal.h"

namespace fal {

// Message of the calling thread's last failed call without a context.
std::string& noctx_error();

inline bool overlaps(const void* a, int64_t abytes, const void* b, int64_t bbytes) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
  return x < y + (uintptr_t)bbytes && y < x + (uintptr_t)abytes;
}

inline bool aligned(const void* p, uintptr_t bytes) { return reinterpret_cast<uintptr_t>(p) % bytes == 0; }

// An array; p NULL: one that the call was not given.
struct Extent {
  const void* p;
  int64_t bytes;
};
inline bool meets(const Extent& out, std::initializer_list<Extent> others) {
  for (const Extent& o : others)
    if (o.p && overlaps(out.p, out.bytes, o.p, o.bytes)) return true;
  return false;
}
inline bool all_aligned(std::initializer_list<Extent> arrays, uintptr_t bytes) {
  for (const Extent& e : arrays)
    if (!aligned(e.p, bytes)) return false;
  return true;
}
// Whether an output overlaps another one or one of `others`.
inline bool outputs_meet(std::initializer_list<Extent> out, std::initializer_list<Extent> others) {
  for (const Extent& o : out) {
    if (!o.p) continue;
    if (meets(o, others)) return true;
    for (const Extent& e : out)
      if (&e != &o && meets(o, {e})) return true;
  }
  return false;
}

// (the kernels multiply by log2(e) / t, which has to be finite and not zero)
inline const char* check_temperature(float t) {
  const float k = 1.4426950408889634f / t;
  return std::isfinite(t) && t > 0.f && std::isfinite(k) && k > 0.f ? nullptr : "temperature must be finite and > 0";
}

inline const char* check_policy(const fal_policy_t* hp) {
  if (!hp) return "NULL hyper-parameters";
  if (!std::isfinite(hp->clip_low) || !std::isfinite(hp->clip_high) || !std::isfinite(hp->kl_coef))
    return "non-finite hyper-parameter";
  if (hp->clip_low < 0.f || hp->clip_low > 1.f || hp->clip_high < 0.f)
    return "clip_low must lie in [0, 1], clip_high be >= 0";
  if (hp->kl_coef < 0.f) return "kl_coef must be >= 0";
  if (hp->sequence_mean != 0 && hp->sequence_mean != 1) return "sequence_mean must be 0 or 1";
  return nullptr;
}

inline const char* check_preference(const fal_preference_t* hp) {
  if (!hp) return "NULL hyper-parameters";
  if (!std::isfinite(hp->beta) || !std::isfinite(hp->label_smoothing)) return "non-finite hyper-parameter";
  if (!(hp->beta > 0.f)) return "beta must be > 0";
  if (hp->label_smoothing < 0.f || hp->label_smoothing > 0.5f) return "label_smoothing must lie in [0, 0.5]";
  if (hp->ipo != 0 && hp->ipo != 1) return "ipo must be 0 or 1";
  if (hp->length_mean != 0 && hp->length_mean != 1) return "length_mean must be 0 or 1";
  if (hp->ipo && hp->label_smoothing != 0.f) return "label_smoothing does not apply to the squared loss";
  return nullptr;
}

}  // namespace fal
