// The plan of an attention over shared prefixes, as it lies in the caller's buffer: who has which prefix, and how the work is
// dealt to workgroups.
#pragma once
#include "common.h"

namespace scout {

// One workgroup's share: tokens [tok0, tok1) of a prefix, for rows [row0, row0 + rows) of a KV head.  The rows of a KV head are
// those of the sequences that have the prefix, the heads of the group of each: row = member * G + head.
struct PrefixItem {
  int32_t prefix, head;
  int32_t member0;       // where the prefix's sequences start in PrefixPlan::member
  int32_t row0, rows;
  int32_t tok0, tok1;
  int32_t split;  // the partial that it leaves, of those of its rows
};

struct PrefixPlan {
  static constexpr int kStampWords = 12;
  int32_t* stamp;    // what the plan was made for
  int32_t* head;     // [0] items
  int32_t* splits;   // [B] partials of a sequence's rows; 0: no prefix
  int32_t* member;   // [B] sequences, prefix by prefix
  PrefixItem* item;  // [max_items]
  int max_items;

  static long long up(long long n) { return (n + 63) / 64 * 64; }
  static long long words(int B, int max_items) { return 128 + 2 * up(B) + 8ll * max_items; }

  static PrefixPlan at(void* buffer, int B, int max_items) {
    PrefixPlan P;
    int32_t* const w = static_cast<int32_t*>(buffer);
    P.stamp = w;
    P.head = w + 64;
    P.splits = w + 128;
    P.member = P.splits + up(B);
    P.item = reinterpret_cast<PrefixItem*>(P.member + up(B));
    P.max_items = max_items;
    return P;
  }
};

constexpr int kMaxPrefixes = 2048;
constexpr int kMaxPrefixSplits = 64;  // partials of a row that the workspace has room for

// How a launch deals its work: fixed on the host by sizes and types.
struct PrefixShape {
  int tile_rows;   // rows of a workgroup
  int granule;     // tokens that a workgroup takes at a time
  int slots;       // workgroups that run at a time
  int head_cost;   // what an item costs beyond its tokens, in tokens
};

}  // namespace scout
