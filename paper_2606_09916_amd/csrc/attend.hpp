// Arguments and launch plan of the attention over the 8-bit cache and of the chunk
// attention (k_attend*.hip). Plain C++: no HIP in here.
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

constexpr int FEW_ROWS = 16;        // query rows per KV head up to which one wave holds them all
constexpr int FEW_ROUND = 1024;     // workgroups of one resident round of k_attend_few
constexpr int TILE_KEYS = 64;       // entries per tile of k_attend_tile

struct AttendPlan {
  int max_n;               // longest chunk of the batch
  bool too_large;          // does not fit a launch grid
  bool few;                // every session's rows per KV head fit one 16-row block
  int heads;               // adjacent KV heads of a workgroup (few)
  int splits;              // of the entries of a session
  int blocks;              // row blocks per (session, layer, KV head): one (few)
  int rows;                // rows per block in the split state
  int64_t ws_floats;
};

inline int attend_tokens(const ikv_session &s, bool decode) { return decode ? 1 : std::max(0, s.qe - s.qs); }

// Entries that a session's list may hold, as far as the host knows.
inline int64_t attend_bound(const ikv_session &s, bool decode) {
  return decode ? decode_live_bound(s) : std::max<int64_t>(1, s.N);
}

inline AttendPlan attend_plan(const AttendArgs &a, const ikv_session *sess, int B, bool decode, int sinks, int window) {
  AttendPlan p{};
  const int G = a.Hq / a.Hkv;
  int64_t longest = 1;
  for (int b = 0; b < B; ++b) {
    const int n = attend_tokens(sess[b], decode);
    p.max_n = std::max(p.max_n, n);
    int64_t len = attend_bound(sess[b], decode);
    if (window) len = std::min<int64_t>(len, int64_t(sinks) + window + n);
    longest = std::max(longest, len);
  }
  p.few = int64_t(p.max_n) * G <= FEW_ROWS;
  p.splits = p.blocks = 1;
  if (p.few) {
    p.rows = p.max_n * G;
    p.heads = a.Hkv % 4 == 0 ? 4 : a.Hkv % 2 == 0 ? 2 : 1;
    const int64_t wgs = std::max<int64_t>(1, int64_t(a.L) * (a.Hkv / p.heads) * std::max(1, B));
    int64_t s = std::max<int64_t>(1, FEW_ROUND / wgs);
    s = std::min<int64_t>(s, (longest + 127) / 128);
    p.splits = int(std::min<int64_t>(s, DEC_MAX_SPLITS));
  } else if (p.max_n > 0) {
    const int64_t rows = int64_t(p.max_n) * G;
    p.rows = rows <= 128 ? 128 : 256;
    p.blocks = int(std::min<int64_t>((rows + p.rows - 1) / p.rows, INT32_MAX));
    const int64_t wgs = int64_t(a.L) * a.Hkv * B * p.blocks;
    int64_t s = std::max<int64_t>(1, 1024 / wgs);
    s = std::min<int64_t>(s, (longest + 511) / 512);
    p.splits = int(std::min<int64_t>(s, DEC_MAX_SPLITS));
  }
  const int64_t parts = int64_t(B) * a.L * a.Hkv * p.blocks * p.splits * p.rows;
  if (p.splits > 1) p.ws_floats = parts * (a.D + 2);
  p.too_large = B > 65535 || int64_t(a.L) * a.Hq > 65535 || int64_t(B) * a.L * a.Hkv * p.blocks > (1 << 24);
  return p;
}

}  // namespace ikv
