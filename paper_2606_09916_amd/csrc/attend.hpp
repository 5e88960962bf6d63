// Arguments and launch plan of the attention over the 8-bit cache and of the chunk
// attention (k_attend.hip). Plain C++: no HIP in here.
#pragma once

#include <stdint.h>

#include <algorithm>

#include "decode_plan.hpp"
#include "ikv.h"

namespace ikv {

// How the rows that attention reads are held.
enum KvFormat { KV_BF16 = 0, KV_INT8 = 1, KV_E4M3 = 2 };

struct AttendArgs {
  int L, Hq, Hkv, D;
  int64_t num_slots;
  int format;              // KvFormat
  bool io_f32;             // q and out are float32 (else bf16)
  const void *k, *v;       // rows or codes
  const float *scales;     // [L][num_slots][Hkv][2] (8-bit formats)
  const ikv_session *sess; // device
  int B;
  bool decode;             // one token per session, whatever its span
  const void *q;
  const int32_t *live, *n_live;
  int sinks, window;       // window 0: none (and sinks 0)
  void *out;
  float *ws;
};

struct AttendPlan {
  int max_n;               // longest chunk of the batch
  bool too_large;          // does not fit a launch grid
  int64_t ws_floats;
};

inline int attend_tokens(const ikv_session &s, bool decode) { return decode ? 1 : std::max(0, s.qe - s.qs); }

inline AttendPlan attend_plan(const AttendArgs &a, const ikv_session *sess, int B, bool decode, int sinks, int window) {
  AttendPlan p{};
  for (int b = 0; b < B; ++b) p.max_n = std::max(p.max_n, attend_tokens(sess[b], decode));
  p.too_large = B > 65535 || int64_t(a.L) * a.Hq > 65535;
  p.ws_floats = 0;
  return p;
}

}  // namespace ikv
