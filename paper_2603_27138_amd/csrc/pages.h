// The state of a pool whose slots several sequences share, as it lies in the caller's buffer.
#pragma once
#include "common.h"

namespace scout {

__host__ __device__ __forceinline__ long long words_of(long long n_slots) { return (n_slots + 31) / 32; }

struct Pages {
  int32_t* refs;   // [n_slots] block-table entries that name the slot: the state that a caller may read
  uint32_t* used;  // [words] bit per slot: refs > 0
  // what one launch of a call leaves for the next one; nothing outlives the call
  int32_t* head;    // [16]
  int32_t* base;    // [kPairs] first rank of a pair or sequence
  int32_t* parent;  // [kPairs] of a fork, -1 where it is refused
  int32_t* order;   // [kPairs] forks, those of one parent side by side
  int32_t* list;    // [n_slots] slots taken, or the holes that a compaction fills
  int32_t* list2;   // [n_slots] slots that a compaction empties
  uint32_t* old;    // [words] used before a compaction
  int32_t* rank;    // [words] used slots in front of each word
  long long n_slots;

  static constexpr int kPairs = 65536;
  static long long up(long long n) { return (n + 63) / 64 * 64; }  // sections start at 256 bytes
  static long long words(long long n_slots) { return 3 * up(n_slots) + 3 * up(words_of(n_slots)) + 64 + 3 * kPairs; }

  static Pages at(void* buffer, long long n_slots) {
    Pages P;
    int32_t* w = static_cast<int32_t*>(buffer);
    auto next = [&](long long n) {
      int32_t* const here = w;
      w += up(n);
      return here;
    };
    P.refs = next(n_slots);
    P.used = reinterpret_cast<uint32_t*>(next(words_of(n_slots)));
    P.head = next(64);
    P.base = next(kPairs);
    P.parent = next(kPairs);
    P.order = next(kPairs);
    P.list = next(n_slots);
    P.list2 = next(n_slots);
    P.old = reinterpret_cast<uint32_t*>(next(words_of(n_slots)));
    P.rank = next(words_of(n_slots));
    P.n_slots = n_slots;
    return P;
  }
};

}  // namespace scout
