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
  int sinks, window;       // at most ATTEND_MOST; window 0: none (and sinks 0)
  void *out;
  float *ws;
};

constexpr int FEW_ROWS = 16;        // query rows per KV head up to which one wave holds them all (twice that
                                    // over the 8-bit cache with bf16 outputs)
constexpr int FEW_WAVES = 8;        // of a workgroup of k_attend_few, at most
constexpr int CUS = 256;            // a round: one workgroup on each
constexpr int ATTEND_MOST = 1 << 30;       // entries of a list, rows of a KV head, sinks and window
constexpr int TILE_KEYS = 64;       // entries per tile of k_attend_tile

struct AttendPlan {
  int max_n;               // longest chunk of the batch
  bool too_large;          // does not fit a launch grid
  bool few;                // every session's rows per KV head fit one 16-row block
  int heads, parts;        // few: adjacent KV heads of a workgroup, waves that share a head's entries
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

// How full n > 0 workgroups leave their rounds of one per CU, in percent.
inline int64_t attend_fill(int64_t n) { return 100 * n / ((n + CUS - 1) / CUS * CUS); }

// Workgroups of the few-rows kernel: `heads` adjacent KV heads (their rows lie side by side, so
// together the waves read long pieces) times `parts` waves that share a head's entries and join
// in LDS, and `splits` of a list over workgroups, joined by a second kernel. Four waves a
// workgroup; us per call of one-token decodes over int8 rows, 36 layers x 8 KV heads unless
// stated, (heads, parts, splits):
//  - the fewest splits that fill a round to 70%, 95% where a wave keeps 4096 entries: one
//    session of 8192: (4, 1, 3) 105, (4, 1, 7) 110, (4, 1, 14) 117; of 1000: (4, 1, 3) 21,
//    (4, 1, 7) 24; 48 layers x 92,300 entries: (4, 2, 8) 1483, (4, 2, 10) 1495, (8, 1, 10) 1516.
//  - lists of uneven bounds (the longest 1.15 times the mean or more): four rounds, so that the
//    last workgroups are short ones. Five sessions of 2000 to 8000: (4, 2, 3) 354, (4, 1, 3) 369.
//  - more than a round of long lists: eight waves. 48 x 4 heads, 16 sessions of 517 to 4100:
//    (4, 2, 1) 480, (4, 1, 1) 507; 16 sessions of 500: (4, 1, 1) 117, (4, 2, 1) 127.
//  - few heads take fewer adjacent ones and more parts, which cost no second kernel: one layer of
//    8192: (1, 4, 16) 14.0, (8, 1, 64) 19.6. Lists of up to 512 entries take no splits at all:
//    300: (2, 2, 1) 11.8, (4, 1, 3) 14.2.
// A split's state costs rows (D + 2) floats, written and read: lists are cut no finer than 16
// entries a row, nor for their unevenness finer than 128 (3 tokens of 5 heads in 4 sessions of
// 700 to 2500: one split 72, four 79, six 87).
inline void attend_few_shape(AttendPlan &p, int Hkv, int64_t groups, int64_t longest, bool uneven) {
  int widest = 4;
  while (Hkv % widest) widest /= 2;
  const int64_t heads_all = groups * Hkv;
  if (longest <= 512) {
    p.heads = widest;
    while (p.heads > 1 && heads_all / p.heads < CUS / 2) p.heads /= 2;
    p.parts = heads_all < CUS / 2 && longest > 256 && p.rows <= FEW_ROWS ? 8 : 4 / p.heads;
    p.splits = 1;
    return;
  }
  for (p.heads = widest;; p.heads /= 2) {
    p.parts = 4 / p.heads;
    const int64_t units = heads_all / p.heads, finest = std::max(64, 16 * p.rows),
                  most = std::min<int64_t>(DEC_MAX_SPLITS, longest / (finest * p.parts));
    p.splits = 0;
    for (int64_t s = 1; s <= most && !p.splits; ++s)
      if (attend_fill(units * s) >= (longest / (s * p.parts) >= 4096 ? 95 : 70) && 
          (!uneven || units * s >= 4 * CUS || longest / (s + 1) < 128 * p.rows))
        p.splits = int(s);
    if ((p.splits && p.splits <= 8) || p.heads == 1) {
      if (!p.splits) p.splits = int(std::max<int64_t>(1, most));
      if (units * p.splits > CUS && longest / p.splits >= 2048 && p.rows <= FEW_ROWS) p.parts *= 2;
      return;
    }
  }
}

// Splits of the tile kernel, whose state is up to 256 rows of a split and worth only idle CUs
// (us, Qwen3-8B's heads, n new tokens over 8701 int8 entries):
//  - less than a round of workgroups: as many splits as stay within one, of at least 256 entries.
//    One layer, n = 509: 1 split 275, 4 111, 8 120; n = 64: 1 275, 24 36, 48 49. (From 129 to 255
//    workgroups that is one; what more would give there has not been measured.)
//  - one block of rows per head (mostly reading, and the state is small): of at least 1024
//    entries, five rounds for 128 rows (36 layers, n = 20: 333 with one split, 275 with three, 265
//    with five, 270 with eight), or the fewest that fill their rounds to 80% for 256 (n = 64: 616
//    with one, 553 with two, 527 with three, 545 with five).
//  - else none: n = 128: 903 with one, 944 with two.
inline int attend_tile_splits(int64_t wgs, int rows, int blocks, int64_t longest) {
  if (wgs < CUS) return int(std::max<int64_t>(1, std::min<int64_t>({CUS / wgs, longest / 256, DEC_MAX_SPLITS})));
  if (blocks > 1) return 1;
  const int64_t most = std::max<int64_t>(1, std::min<int64_t>(5, longest / 1024));
  if (rows == 128) return int(std::min<int64_t>(most, (5 * CUS + wgs - 1) / wgs));
  int64_t s = 1;
  while (s < most && attend_fill(wgs * s) < 80) ++s;
  return int(s);
}

inline AttendPlan attend_plan(const AttendArgs &a, const ikv_session *sess, int B, bool decode, int sinks, int window) {
  AttendPlan p{};
  const int G = a.Hq / a.Hkv;
  int64_t longest = 1, sum = 0, most = 0;
  for (int b = 0; b < B; ++b) {
    const int n = attend_tokens(sess[b], decode);
    p.max_n = std::max(p.max_n, n);
    int64_t len = attend_bound(sess[b], decode);
    if (window) len = std::min<int64_t>(len, int64_t(sinks) + window + n);
    longest = std::max(longest, len);
    sum += len;
    most = std::max<int64_t>(most, sess[b].N);
  }
  p.splits = p.blocks = 1;
  // launch grids: 65535 in y and z; entries and rows stay below 2^30 (and the products here in 64 bits)
  p.too_large = B > 65535 || int64_t(a.L) * a.Hq > 65535 || most > ATTEND_MOST || int64_t(p.max_n) * G > ATTEND_MOST;
  if (p.too_large) return p;
  p.few = int64_t(p.max_n) * G <= (a.format != KV_BF16 && !a.io_f32 ? 2 * FEW_ROWS : FEW_ROWS);
  const int64_t groups = std::max<int64_t>(1, int64_t(a.L) * B);
  if (p.few) {
    p.rows = p.max_n * G;
    attend_few_shape(p, a.Hkv, groups, longest, B > 1 && 20 * longest * B >= 23 * sum);
  } else {
    const int64_t rows = int64_t(p.max_n) * G;
    p.rows = rows <= 128 ? 128 : 256;            // four waves or eight
    p.blocks = int(std::min<int64_t>((rows + p.rows - 1) / p.rows, INT32_MAX));
    p.splits = attend_tile_splits(groups * a.Hkv * p.blocks, p.rows, p.blocks, longest);
  }
  // the workspace is sized without the window
  if (window) p.splits = std::min(p.splits, attend_plan(a, sess, B, decode, 0, 0).splits);
  if (p.splits > 1) p.ws_floats = int64_t(B) * a.L * a.Hkv * p.blocks * p.splits * p.rows * (a.D + 2);
  // under 2^32 threads in x
  const int64_t wgs = (groups * a.Hkv + 7) / 8 * 8 * p.blocks * p.splits;
  p.too_large = !p.few && wgs >= (int64_t(1) << 32) / (2 * p.rows);
  return p;
}

}  // namespace ikv
