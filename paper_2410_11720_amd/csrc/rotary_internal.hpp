// Arguments of the rotary kernel, shared with its entry points.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "divide.hpp"

namespace abft {

// Heads [batch, tokens, heads, head_dim], strides in bytes.
struct HeadTensor {
  char* p = nullptr;
  int64_t b = 0, t = 0, h = 0;
};

struct RotaryArgs {
  HeadTensor in[3], out[3];       // queries, keys, values (the last are copied)
  int32_t heads[3] = {0, 0, 0};
  const double* freqs = nullptr;  // [half] radians a position
  const int32_t* start = nullptr; // [batch] or null
  int32_t n_tokens = 0;           // of all sequences
  Divisor tokens;                 // of one
  int32_t head_dim = 0, half = 0; // half: pairs
  int32_t interleaved = 0;
  float sign = 1.f, magnitude = 1.f;
  int32_t append = 0;             // keys and values go to their positions ...
  int32_t capacity = 0;           // ... below this one
  // work: items of a token are parts (16 dims) of heads, `turned` ones in front; a
  // group of lanes takes `per` of them, `waves` groups a token; as many items as it has
  // lanes are dq heads and dr parts
  int32_t turned = 0, items = 0, per = 0, dq = 0, dr = 0;
  Divisor parts, waves;
};

hipError_t launch_rotary(RotaryArgs a, int dtype, hipStream_t s);

}  // namespace abft
