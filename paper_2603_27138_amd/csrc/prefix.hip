// Attention of a batch over prefixes that several of its sequences share, computed once for all of them.
//
// For every sequence b with a prefix, KV head g and query head h of its group:
//   x_t = scale q_bh . k_t,  m = max x_t,  l = sum exp(x_t - m),  o = sum exp(x_t - m) v_t / l
// over the prefix's tokens that have a slot.  Attended to sequence by sequence the prefix's tiles are read once per sequence; here
// the heads of all its sequences are rows of one product with every tile, which is read once per tile of rows: n sequences read
// 1/n of the bytes, and beyond some 130 rows a KV head (6 flop a row for 4 bytes, 1.2 PFLOP/s over 6.2 TB/s) it is the matrix instructions
// that bound it.
//
// prefix_plan_kernel deals the work once for a batch (the lengths of prefixes and who has them do not change with the layer);
// prefix_attn_kernel leaves a partial per row and split; prefix_combine_kernel folds them, with the sequence's own partial.
#include <type_traits>

#include "attn_unit.h"
#include "plan_scan.h"
#include "prefix.h"

namespace scout {

typedef __attribute__((ext_vector_type(8))) short s16x8;

// ---------------------------------------------------------------- the plan

struct PrefixStamp {
  int32_t w[PrefixPlan::kStampWords];
};

// Splits that a prefix of len tokens is cut into where a chunk has `chunk` tokens.
__device__ __forceinline__ int splits_of(int len, int chunk) { return (len + chunk - 1) / chunk; }
__device__ __forceinline__ int round_up(int x, int to) { return (x + to - 1) / to * to; }

// One workgroup, bound by latency: 4 us with the launch for one prefix, 5.4 for 16, 17 for 256, 83 for 2048 of 4096 sequences.
__global__ __launch_bounds__(kPlanThreads) void prefix_plan_kernel(PrefixPlan P, PrefixStamp stamp, PrefixShape shape, int B, int Hkv,
                                                                   int G, int n_prefix, int max_tokens,
                                                                   const int32_t* __restrict__ prefix_of,
                                                                   const int32_t* __restrict__ prefix_len) {
  // of each prefix: its sequences, how many of them have been put in the list, where its part of the list starts, its tokens, its
  // tiles of rows (of all KV heads), its first item
  __shared__ int count[kMaxPrefixes], placed[kMaxPrefixes], first[kMaxPrefixes], len[kMaxPrefixes], tiles[kMaxPrefixes], base[kMaxPrefixes];
  __shared__ int lds[kPlanWaves], items_lds[kWave], longest_lds, chunk_lds;
  const int t = threadIdx.x, lane = lane_id();
  for (int p = t; p < n_prefix; p += kPlanThreads) {
    const int n = prefix_len[p];
    len[p] = n < 0 ? 0 : n > max_tokens ? max_tokens : n;
    count[p] = placed[p] = 0;
  }
  if (t < kWave) items_lds[t] = 0;
  if (t == 0) longest_lds = 0;
  __syncthreads();
  for (int b = t; b < B; b += kPlanThreads) {
    const int p = prefix_of[b];
    if (p >= 0 && p < n_prefix) atomicAdd(&count[p], 1);
  }
  __syncthreads();
  // How long a chunk is: candidate c cuts the longest prefix c + 1 ways.  shape.slots workgroups run at a time, so a candidate costs as
  // many rounds as its items fill, each as long as a chunk and what an item costs beyond its tokens.
  static_assert(kMaxPrefixSplits == kWave, "a candidate, and a split, per lane");
  auto chunk_of = [&](int longest, int c) {
    const int n = round_up((longest + c) / (c + 1), shape.granule);
    return n > shape.granule ? n : shape.granule;
  };
  auto cheapest = [&](int items, int chunk) {  // by a wave, lane c with candidate c's items (below kMostItems * kMaxPrefixSplits) and chunk
    const long long rounds = (items + shape.slots - 1) / shape.slots;
    long long cost = items > P.max_items ? 1ll << 62 : rounds * (chunk + shape.head_cost);  // without splits the items always fit
    int best = lane;
#pragma unroll
    for (int s = 1; s < kWave; s <<= 1) {  // the lowest cost, of equal ones the fewest splits
      const long long other = __shfl_xor(cost, s);
      const int who = __shfl_xor(best, s);
      if (other < cost || (other == cost && who < best)) {
        cost = other;
        best = who;
      }
    }
    return __shfl(chunk, best);
  };
  auto tiles_for = [&](int members) { return (members * G + shape.tile_rows - 1) / shape.tile_rows * Hkv; };
  int chunk, n_items = 0;
  if (n_prefix <= kWave) {  // a wave has a prefix in each lane, and need not wait for the others (4 prefixes: 5 us with the launch, 6 below)
    if (t < kWave) {
      const int members = lane < n_prefix ? count[lane] : 0, my_tiles = tiles_for(members), my_len = members > 0 ? len[lane] : 0;
      int longest = my_len, items = 0;
#pragma unroll
      for (int s = 1; s < kWave; s <<= 1) longest = max(longest, __shfl_xor(longest, s));
      const int my_chunk = chunk_of(longest, lane);
      for (int p = 0; p < n_prefix; ++p)
        items += __builtin_amdgcn_readlane(my_tiles, p) * splits_of(__builtin_amdgcn_readlane(my_len, p), my_chunk);
      const int best = cheapest(items, my_chunk), my_items = my_tiles * splits_of(my_len, best);
      const int behind = wave_scan(members, lane), items_behind = wave_scan(my_items, lane);
      if (lane < n_prefix) {
        first[lane] = behind - members;
        tiles[lane] = my_tiles;
        len[lane] = my_len;
        base[lane] = items_behind - my_items;
      }
      if (lane == kWave - 1) {
        chunk_lds = best;
        items_lds[0] = items_behind;
      }
    }
    __syncthreads();
    chunk = chunk_lds;
    n_items = items_lds[0];
  } else {
    for (int p0 = 0, at = 0; p0 < n_prefix; p0 += kPlanThreads) {
      const int p = p0 + t, members = p < n_prefix ? count[p] : 0;
      int total;
      const int before = plan_scan(members, lds, &total);
      if (p < n_prefix) {
        first[p] = at + before;
        tiles[p] = tiles_for(members);
        if (members == 0) len[p] = 0;  // nobody has it
        atomicMax(&longest_lds, len[p]);
      }
      at += total;
    }
    __syncthreads();
    const int my_chunk = chunk_of(longest_lds, lane);
    int items = 0;  // of the wave's prefixes
    for (int p = t / kWave; p < n_prefix; p += kPlanWaves) items += tiles[p] * splits_of(len[p], my_chunk);
    if (items > 0) atomicAdd(&items_lds[lane], items);
    __syncthreads();
    if (t < kWave) {
      const int best = cheapest(items_lds[lane], my_chunk);
      if (t == 0) chunk_lds = best;
    }
    __syncthreads();
    chunk = chunk_lds;
    for (int p0 = 0; p0 < n_prefix; p0 += kPlanThreads) {
      const int p = p0 + t;
      int total;
      const int before = plan_scan(p < n_prefix ? tiles[p] * splits_of(len[p], chunk) : 0, lds, &total);
      if (p < n_prefix) base[p] = n_items + before;
      n_items += total;
    }
    __syncthreads();
  }
  if (t == 0) P.head[0] = n_items;
  if (t < PrefixPlan::kStampWords) P.stamp[t] = stamp.w[t];
  for (int b = t; b < B; b += kPlanThreads) {
    const int p = prefix_of[b];
    const bool has = p >= 0 && p < n_prefix;
    P.splits[b] = has ? splits_of(len[p], chunk) : 0;
    // in whichever order the additions come: a row's result does not depend on the rows beside it
    if (has) P.member[first[p] + atomicAdd(&placed[p], 1)] = b;
  }
  for (int i = t; i < n_items; i += kPlanThreads) {
    int p = 0, hi = n_prefix - 1;  // the last prefix whose items start at i or before: the one that i belongs to
    while (p < hi) {
      const int mid = (p + hi + 1) >> 1;
      if (base[mid] <= i) p = mid;
      else hi = mid - 1;
    }
    const int s = splits_of(len[p], chunk), units = Hkv * s, of = tiles[p] / Hkv;  // tiles of rows of a unit
    // A unit (split, KV head) has a workgroup per tile of rows, and all of them read the same tokens: their numbers are eight apart,
    // so that they run on the same XCD and find in its L2 what one of them has read.
    const int k = i - base[p], full = units / 8 * 8 * of;
    int unit, tile;
    if (k < full) {
      unit = k / (8 * of) * 8 + k % 8;
      tile = k / 8 % of;
    } else {
      unit = units / 8 * 8 + (k - full) % (units % 8);
      tile = (k - full) / (units % 8);
    }
    const int split = unit / Hkv, rows = count[p] * G - tile * shape.tile_rows;
    const int even = round_up((len[p] + s - 1) / s, shape.granule);  // at most the chunk: no split is empty
    PrefixItem it;
    it.prefix = p;
    it.head = unit % Hkv;
    it.member0 = first[p];
    it.row0 = tile * shape.tile_rows;
    it.rows = rows < shape.tile_rows ? rows : shape.tile_rows;
    it.tok0 = split * even;
    it.tok1 = it.tok0 + even < len[p] ? it.tok0 + even : len[p];
    it.split = split;
    P.item[i] = it;
  }
}

// ---------------------------------------------------------------- the attention

// What a launch works on.
struct PrefixWork {
  int B, Hq, Hkv, G, S, s_shift, tile_stride, prefix_blocks, n_prefix;
  uint32_t g_magic;  // ceil(2^32 / G); 0 for G = 1
  float scale2;      // softmax scale in base-2 units
  long long n_slots;
  const void *q, *k_pool, *v_pool;
  const int32_t* table;  // [n_prefix][Hkv][prefix_blocks]
  float *po, *pm, *pl;   // partials [B * Hq][kMaxPrefixSplits]: unnormalised sums, maximum in base-2 units, sum
};

__device__ __forceinline__ bool made_for(const PrefixPlan& P, const PrefixStamp& stamp) {
  bool same = true;
#pragma unroll
  for (int i = 0; i < PrefixPlan::kStampWords; ++i) same &= P.stamp[i] == stamp.w[i];
  return same;
}

// The query row, of all [B * Hq], that row r of an item is.
__device__ __forceinline__ int query_row(const PrefixPlan& P, const PrefixWork& W, const PrefixItem& it, int r) {
  const uint32_t rr = (uint32_t)(it.row0 + r);
  const uint32_t m = W.g_magic ? __umulhi(rr, W.g_magic) : rr;
  return P.member[it.member0 + (int)m] * W.Hq + it.head * W.G + (int)(rr - m * W.G);
}

// bf16 terms of a softmax weight in the second product, for bf16.  All but the last are cut (7 explicit bits, what is left is below 2^-7), the last
// one is rounded: two lose 2^-15 of a weight at the most, three 2^-22.  Three where the attention over a sequence's own tokens keeps its weights
// in binary32 too, two where that one rounds them to a single term: what a batch shares is never held in fewer bits than what it does
// not, whoever else is in the batch and whatever is written of the result.  The sum l always has the weights as they are.
template <int DH>
constexpr int kTerms = kWeights32<SCOUT_BF16, DH> ? 3 : 2;

// A weight without its upper term.  Nothing left times an infinite value would be NaN, so of a weight there is always 2^-126 left (the least
// that one has; the bounds above are those of weights from 2^-104 on).  Of no weight nothing is: 2^-126 of the largest value would be 4.
__device__ __forceinline__ float what_is_left(float w, uint32_t term) {
  return __builtin_amdgcn_fmed3f(w - __uint_as_float(term), 0x1p-126f, w);
}

constexpr int kNarrowWaves = 8;

// Up to 32 rows, and fp32.  The waves of a workgroup take units of 16 tokens in turn (wave v: v, v + 8, ...); K and V rows go from memory
// into MFMA operand registers, and NQ column tiles of 16 rows are multiplied with them there (layout: see attn_unit.h).  The waves fold through LDS.
// Bound by memory, and where there is little of it by a launch's way in and out: 4 sequences of 4 heads over 8192 shared tokens (8 KV heads,
// 33.5 MB at bf16, d = 128) 8 us, of which 2.3 are the launch and 4 the way to the first unit and from the last; 2 of them over 65536 tokens 42 us (6.4 TB/s).
// With the fold's launch: 16 rows 9 us and each byte at 6.1 TB/s, 32 rows 13 and 5.9, fp32 11 and 6.0 (16 rows), 15 and 5.5 (32).
template <int DT, int DH, int NQ>
__global__ __launch_bounds__(kNarrowWaves* kWave) void prefix_narrow_kernel(PrefixPlan P, PrefixStamp stamp, PrefixWork W) {
  using L = Tile<DT, DH>;
  constexpr int WAVES = kNarrowWaves, ROW = DH + 4, TERMS = kTerms<DH>;
  __shared__ float smem[WAVES * (16 * ROW + 32)];
  const PrefixItem it = P.item[blockIdx.x];  // in the trip that says whether it is one
  if (!made_for(P, stamp) || (int)blockIdx.x >= P.head[0]) return;
  const int lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), ln = lane & 15, kg = lane >> 4;
  const int ush = W.s_shift - 4;
  const int u0 = it.tok0 / kUnitTokens + wave, u1 = (it.tok1 + kUnitTokens - 1) / kUnitTokens;
  const int32_t* row = W.table + ((size_t)it.prefix * W.Hkv + it.head) * W.prefix_blocks;
  // lane j: the slot of this wave's unit number j, 64 units at a time
  auto fetch_slots = [&](int u) {
    const int mine = u + lane * WAVES;
    return mine < u1 ? row[mine >> ush] : -1;
  };
  int slots = fetch_slots(u0), slots_next = -1;
  QRegs<DT, DH> qreg[NQ];
#pragma unroll
  for (int t = 0; t < NQ; ++t) {
    const int r = t * 16 + ln;
    const bool real = r < it.rows;
    const char* at = static_cast<const char*>(W.q) + (size_t)query_row(P, W, it, real ? r : it.rows - 1) * L::ROWB + kg * 16;
#pragma unroll
    for (int s = 0; s < L::KL; ++s) {
      qreg[t][s] = *reinterpret_cast<const u32x4*>(at + s * 64);
      qreg[t][s] &= real ? 0xffffffffu : 0u;
    }
  }
  f32x4 acc[NQ][L::NR];
  float m[NQ], l[NQ];
#pragma unroll
  for (int t = 0; t < NQ; ++t) {
#pragma unroll
    for (int r = 0; r < L::NR; ++r) acc[t][r] = (f32x4){0.f, 0.f, 0.f, 0.f};
    m[t] = -INFINITY;
    l[t] = 0.0f;
  }
  auto entry = [&](int j, int u) {
    Entry e{0, 0};
    const long long slot = __builtin_amdgcn_readlane(slots, j);
    if (u < u1 && slot >= 0 && slot < W.n_slots) {
      const int left = it.tok1 - u * kUnitTokens;
      e.valid = left < kUnitTokens ? left : kUnitTokens;
      e.elem_off = (size_t)slot * W.tile_stride + (size_t)(u & ((1 << ush) - 1)) * kUnitTokens * DH;
    }
    return e;
  };
  UnitRegs<DT, DH> T;  // one unit in flight: two or three are no faster
  Entry e = entry(0, u0);
  issue_unit<DT, DH>(T, W.k_pool, W.v_pool, e, ln, kg);
  slots_next = fetch_slots(u0 + kWave * WAVES);
  int j = 1;
  for (int u = u0; u < u1; u += WAVES) {
    if (j == kWave) {
      slots = slots_next;
      slots_next = fetch_slots(u + WAVES + kWave * WAVES);
      j = 0;
    }
    const Entry next = entry(j++, u + WAVES);
    if (e.valid > 0) {  // wave-uniform
      if (e.valid < kUnitTokens) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (4 * kg + i >= e.valid) {
#pragma unroll
            for (int c = 0; c < L::VC; ++c) T.v[i][c] = (u32x4){0, 0, 0, 0};
          }
      }
#pragma unroll
      for (int t = 0; t < NQ; ++t) {
        f32x4 st = (f32x4){0.f, 0.f, 0.f, 0.f};
        if constexpr (DT == SCOUT_BF16) {
#pragma unroll
          for (int s = 0; s < L::KL; ++s)
            st = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(T.k[s]), as_bf16x8(qreg[t][s]), st, 0, 0, 0);
        } else {
          // chains of 8 channels, joined pairwise: the rounding of one chain over all of them is what the outputs' error would show
          f32x4 part[L::KL];
#pragma unroll
          for (int s = 0; s < L::KL; ++s) {
            f32x4 half[2];
#pragma unroll
            for (int c = 0; c < 4; ++c) {
              if (c % 2 == 0) half[c / 2] = (f32x4){0.f, 0.f, 0.f, 0.f};
              half[c / 2] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(T.k[s][c]), __uint_as_float(qreg[t][s][c]), half[c / 2], 0, 0, 0);
            }
            part[s] = half[0] + half[1];
          }
#pragma unroll
          for (int n = L::KL / 2; n > 0; n /= 2)
#pragma unroll
            for (int s = 0; s < n; ++s) part[s] += part[s + n];
          st = part[0];
        }
        // Scaled here, in front of the branch: a product's result is first read in the block that the product stands in.  Where the
        // first reader was the maximum behind the branch, the compiler (ROCm 7.2) put no wait states in front of it, and it read the
        // registers' old contents.
        float x[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = st[i] * W.scale2;
        if (e.valid < kUnitTokens) {
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if (4 * kg + i >= e.valid) x[i] = -INFINITY;
        }
        const float bm = max_xor32(max_xor16(fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3]))));
        const float m_new = fmaxf(m[t], bm);
        const float m_sub = m_new == -INFINITY ? 0.0f : m_new;
        float p[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) p[i] = fast_exp2(x[i] - m_sub);
        if (__ballot(m_new != m[t]) != 0) {
          const float alpha = exp2_diff(m[t], m_new);
          l[t] *= alpha;
#pragma unroll
          for (int r = 0; r < L::NR; ++r) acc[t][r] *= alpha;
          m[t] = m_new;
        }
        l[t] += (p[0] + p[1]) + (p[2] + p[3]);
        if constexpr (DT == SCOUT_BF16) {
          s16x4 term[TERMS];
#pragma unroll
          for (int n = 0; n < TERMS; ++n) {
            if (n + 1 < TERMS) {  // cut, not rounded: what is left is not negative
              uint32_t hi[4];
#pragma unroll
              for (int i = 0; i < 4; ++i) {
                hi[i] = __float_as_uint(p[i]) & 0xffff0000u;
                p[i] = what_is_left(p[i], hi[i]);
              }
              term[n] = __builtin_bit_cast(s16x4, (uint2){pack_halves(hi[0], hi[1], 1), pack_halves(hi[2], hi[3], 1)});
            } else {
              term[n] = __builtin_bit_cast(s16x4, (uint2){cvt_pk_bf16(p[0], p[1]), cvt_pk_bf16(p[2], p[3])});
            }
          }
#pragma unroll
          for (int r = 0; r < L::NR; ++r) {
            const uint32_t a01 = pack_halves(T.v[0][0][r >> 1], T.v[1][0][r >> 1], r & 1);
            const uint32_t a23 = pack_halves(T.v[2][0][r >> 1], T.v[3][0][r >> 1], r & 1);
            const s16x4 v = __builtin_bit_cast(s16x4, (uint2){a01, a23});
#pragma unroll
            for (int n = TERMS - 1; n >= 0; --n) acc[t][r] = __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(v, term[n], acc[t][r], 0, 0, 0);
          }
        } else {
#pragma unroll
          for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int r = 0; r < L::NR; ++r)
              acc[t][r] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(T.v[i][r / 4][r % 4]), p[i], acc[t][r], 0, 0, 0);
        }
      }
    }
    e = next;
    issue_unit<DT, DH>(T, W.k_pool, W.v_pool, e, ln, kg);
  }
  // the waves' partials of 16 rows at a time
  constexpr int AREA = 16 * ROW + 32, Q = DH / 2;
#pragma unroll
  for (int t = 0; t < NQ; ++t) {
    if (t * 16 >= it.rows) break;
    const float lsum = sum_xor32(sum_xor16(l[t]));
    float* wo = smem + wave * AREA;
    if (t > 0) __syncthreads();
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int r = 0; r < L::NR; r += 4)
        *reinterpret_cast<float4*>(wo + ln * ROW + L::channel(r, 4 * kg + i)) =
            make_float4(acc[t][r][i], acc[t][r + 1][i], acc[t][r + 2][i], acc[t][r + 3][i]);
    if (kg == 0) {
      wo[16 * ROW + ln] = m[t];
      wo[16 * ROW + 16 + ln] = lsum;
    }
    __syncthreads();
    for (int x = threadIdx.x; x < 16 * Q; x += WAVES * kWave) {
      const int h = x / Q, c = (x % Q) * 2;
      if (t * 16 + h >= it.rows) continue;
      float M = -INFINITY, sum = 0.0f;
#pragma unroll
      for (int w = 0; w < WAVES; ++w) M = fmaxf(M, smem[w * AREA + 16 * ROW + h]);
      f32x2 o = (f32x2){0.f, 0.f};
#pragma unroll
      for (int w = 0; w < WAVES; ++w) {
        const float* base = smem + w * AREA;
        const float f = exp2_diff(base[16 * ROW + h], M);
        const f32x2 y = *reinterpret_cast<const f32x2*>(base + h * ROW + c);
        o[0] += f * y[0];
        o[1] += f * y[1];
        sum += f * base[16 * ROW + 16 + h];
      }
      const size_t at = (size_t)query_row(P, W, it, t * 16 + h) * kMaxPrefixSplits + it.split;
      *reinterpret_cast<f32x2*>(W.po + at * DH + c) = o;
      if (c == 0) {
        W.pm[at] = M;
        W.pl[at] = sum;
      }
    }
  }
}

// ---- More rows than that, bf16: tiles of K and V through LDS.
//
// A group of WM waves has WM * 32 rows (each wave 32 of them) and goes through tiles of TOK tokens, each wave bringing TOK / WM of their rows
// from memory into LDS, where all of the group read them.  WN groups take tiles in turn and fold their sums at the end.  RING tiles
// lie in LDS: while one is multiplied the next ones are on their way, without passing through registers.
//   logits^T[token][row] = K . Q^T       32x32x16: K rows are the first operand (lane: token lane % 32, channels 8 * (lane / 32) + ..)
//   out^T[channel][row] += V^T . P^T     32x32x16: the logits leave the first product with row lane % 32 and tokens 8 * (i / 4) + 4 * (lane / 32) +
//                                        i % 4 in register i: eight registers are the second operand of a step of 16 tokens, if the
//                                        first one, V^T, has its tokens in that order; the transposing LDS read delivers them
// 16-byte chunk c of token row r lies at place c ^ swizzle(r) of its row, so that the lanes that LDS serves together hit different banks.
// Units of 16 tokens without a slot are left out: every tile but an item's last one is full.
//
// Tiles by their rows (8 waves always; d = 128, 8 KV heads, 32k tokens):
//   64   2 waves x 4 groups, 32 tokens   bound by memory: 227 MB of tiles in 46 us, 4.9 TB/s (read alone: 6.1); d = 64, 62 MB in 20 us
//   128  4 waves x 2 groups, 64 tokens   by memory, and the way in and out: 134 MB, 26 GFLOP in 37 to 42 us
//   256  8 waves x 1 group, 128 tokens   by the matrix instructions and LDS: 103 GFLOP in 98 to 121 us, 0.85 to 1.05 PFLOP/s (a matrix product
//                                        of 8192^3: 1.21)
// With the fold's launch: 64 rows 15 us and each byte at 5.8 TB/s, 128 rows 18 and 4.6, d = 64 and 64 rows 10 and 4.2 (two tiles of a group are 16 KB there,
// half of what is in flight at d = 128).
// With 256 rows attention and fold take 113 us, without the matrix instructions 60, without the LDS reads that feed them 87, without these and
// the exponentials 83: each wave reads all of a tile for its 32 rows.  64 rows a wave would read half; with the next tile's logits held as well, to have
// both products at hand, they spill (375 us).  Two waves of a SIMD in opposite phases, another order of weights and products, raised
// priorities: no faster.
typedef __attribute__((ext_vector_type(16))) float f32x16;
typedef __attribute__((ext_vector_type(4))) int i32x4;

template <int DH>
struct WideTile {
  static constexpr int ROWB = DH * 2, CH = ROWB / 16;  // bytes and 16-byte chunks of a token row
  static constexpr int KS = DH / 16, DT = DH / 32;     // steps of the first product, channel tiles of the second
  static __device__ __forceinline__ int k_swizzle(int r) { return DH == 128 ? r & 15 : (r >> 1) & 7; }
  static __device__ __forceinline__ int v_swizzle(int r) { return DH == 128 ? (r & 3) << 2 : (r & 2) << 1; }
};

// N pieces of 1 KiB, one after the other in memory from lane to lane in the order of at[], to LDS at `to`.  The compiler does not know of them:
// await() says when they have arrived.
template <int N>
__device__ __forceinline__ void load_to_lds(const void* base, int bytes, const int (&at)[N], uint32_t to) {
  const uint64_t b = reinterpret_cast<uint64_t>(base);
  const i32x4 rsrc = {(int)(uint32_t)b, (int)(uint32_t)(b >> 32) & 0xffff, bytes, 0x00020000};
  static_assert(N == 2 || N == 4, "pieces");
  // One wait state between the write of m0 and the load that uses it; five between a vector instruction that wrote a scalar operand, which the
  // compiler knows of and the loads here it does not, and the load that reads it.
  if constexpr (N == 2)
    asm volatile("s_mov_b32 m0, %1\n\ts_nop 3\n\tbuffer_load_dwordx4 %2, %0, 0 offen lds\n\t"
                 "buffer_load_dwordx4 %3, %0, 0 offen offset:1024 lds" ::"s"(rsrc), "s"(to), "v"(at[0]), "v"(at[1])
                 : "memory", "m0");
  else
    asm volatile("s_mov_b32 m0, %1\n\ts_nop 3\n\tbuffer_load_dwordx4 %2, %0, 0 offen lds\n\t"
                 "buffer_load_dwordx4 %3, %0, 0 offen offset:1024 lds\n\tbuffer_load_dwordx4 %4, %0, 0 offen offset:2048 lds\n\t"
                 "buffer_load_dwordx4 %5, %0, 0 offen offset:%6 lds" ::"s"(rsrc), "s"(to), "v"(at[0]), "v"(at[1]), "v"(at[2]), "v"(at[3]), "n"(3 * 1024)
                 : "memory", "m0");
}
// All but the last N of the wave's loads from memory have arrived, and what it has read of LDS.
template <int N>
__device__ __forceinline__ void await() {
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(N) : "memory");
}

// Between what lanes of a wave store in LDS and what other lanes of it read there, and the other way round: LDS serves a wave's accesses in order, the
// compiler has to keep that order (no instruction).
__device__ __forceinline__ void wave_exchange() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// A row's sums are kept relative to a number that follows its maximum only when that has moved by more than 2^kLag: weights are below 2^kLag then,
// which binary32 sums and bf16 terms hold as well as weights below one, and the sums need not be rescaled whenever one of a wave's
// rows meets a larger logit, which is in most tiles.
constexpr float kLag = 16.0f;

template <int DH, int WM, int WN, int TOK>
__global__ __launch_bounds__(WM* WN* kWave) void prefix_wide_kernel(PrefixPlan P, PrefixStamp stamp, PrefixWork W) {
  using L = WideTile<DH>;
  constexpr int NH = TOK / 32, UNITS = TOK / 16, STEP = UNITS * WN, TERMS = kTerms<DH>;
  constexpr int TILE = TOK * L::ROWB;                // bytes of K, and of V, of a tile
  constexpr int MINE = TILE / WM, NP = MINE / 1024;  // bytes and pieces of it that a wave brings
  constexpr int ROWS = TOK / WM;                     // token rows of it
  constexpr int RING = 2;                            // (d = 128, one term of a weight: three or four of 32 tokens for 128 rows 38 to 39 us against 36 to 39; of 64 for 256 rows 92 to 96 against 87)
  typedef std::conditional_t<(UNITS > 4), uint64_t, uint32_t> Counts;  // tokens that count of each unit of a tile, a byte for each
  static_assert(UNITS <= 8 && ROWS <= 16 && MINE % 1024 == 0, "a wave's rows are of one unit, in whole pieces");
  static_assert(STEP <= 32, "steps are cut from 64 units");
  static_assert((WN - 1) * WM * (L::DT * 16 + 2) * 256 <= WN * RING * 2 * TILE, "the groups' sums fit where the tiles were");
  __shared__ __attribute__((aligned(1024))) char lds[WN * RING * 2 * TILE];  // [group][place][K, V][tile]
  __shared__ int2 queue[WM * WN][kWave];
  const PrefixItem it = P.item[blockIdx.x];  // in the trip that says whether it is one
  if (!made_for(P, stamp) || (int)blockIdx.x >= P.head[0]) return;
  const int lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int wm = wave % WM, grp = wave / WM, l32 = lane & 31, half = lane >> 5;
  const int ush = W.s_shift - 4, u1 = (it.tok1 + kUnitTokens - 1) / kUnitTokens;
  const int32_t* row = W.table + ((size_t)it.prefix * W.Hkv + it.head) * W.prefix_blocks;

  // The item's units that have a slot, in order, up to 64 at a time: lane j has the j-th's slot, and its tokens that count (16, or fewer
  // in the prefix's last unit; 0: no unit) | unit of the block << 8.  Behind them the table's entries that are still to be looked through
  // (of units raw_unit on, a bit of `pending` for each that has a slot), and those that are on their way.
  int u_slot = 0, u_what = 0, u_n = 0, u_pos = 0;
  uint64_t u_full = 0;
  int raw = 0, raw_what = 0, ahead, ahead_unit;
  uint64_t pending = 0;
  auto fetch = [&](int unit) __attribute__((always_inline)) {
    ahead_unit = unit;
    const int mine = unit + lane;
    ahead = mine < u1 ? row[mine >> ush] : -1;
  };
  // A step's units at least, as long as there are any: what is left moves to the front, what comes next joins it.
  auto refill = [&]() __attribute__((always_inline)) {
    int2* const q = queue[wave];
    int n = u_n - u_pos;
    if (lane >= u_pos && lane < u_n) q[lane - u_pos] = make_int2(u_slot, u_what);
    while (n < kWave && (pending != 0 || ahead_unit < u1)) {
      if (pending == 0) {
        const int unit = ahead_unit + lane, left = it.tok1 - unit * kUnitTokens;
        raw = ahead;
        raw_what = (left < kUnitTokens ? left : kUnitTokens) | (unit & ((1 << ush) - 1)) << 8;
        pending = __ballot(unit < u1 && raw >= 0 && raw < W.n_slots);
        fetch(ahead_unit + kWave);
      }
      const int rank = mbcnt64(pending);
      const bool takes = (pending >> lane & 1) != 0 && rank < kWave - n;
      if (takes) q[n + rank] = make_int2(raw, raw_what);
      const uint64_t taken = __ballot(takes);
      pending &= ~taken;
      n += (int)__popcll(taken);
    }
    u_pos = 0;
    u_n = n;
    wave_exchange();
    const int2 mine = q[lane];
    wave_exchange();
    u_slot = mine.x;
    u_what = lane < n ? mine.y : 0;
    u_full = __ballot((u_what & 255) == kUnitTokens);
  };

  fetch(it.tok0 / kUnitTokens);
  // the wave's rows as second operands of the first product: channels 16 * s + 8 * half on of row l32
  bf16x8 q[L::KS];
  const bool real = wm * 32 + l32 < it.rows;
  const size_t out_row = query_row(P, W, it, real ? wm * 32 + l32 : it.rows - 1);
  {
    const char* at = static_cast<const char*>(W.q) + out_row * L::ROWB + half * 16;
#pragma unroll
    for (int s = 0; s < L::KS; ++s) {
      u32x4 y = *reinterpret_cast<const u32x4*>(at + s * 32);
      y &= real ? 0xffffffffu : 0u;
      q[s] = as_bf16x8(y);
    }
  }

  // Where a lane's 16 bytes of the wave's pieces lie in memory, from the first of its rows on: place lane % CH of row r holds chunk
  // place ^ swizzle(r); less the kibibytes that the loads add to both addresses.
  int k_from[NP], v_from[NP];
  const int row0 = wm * ROWS;
#pragma unroll
  for (int i = 0; i < NP; ++i) {
    const int in = lane / L::CH, r = row0 + i * (kWave / L::CH) + in, c = lane % L::CH;
    k_from[i] = in * L::ROWB + ((c ^ L::k_swizzle(r)) << 4);
    v_from[i] = in * L::ROWB + ((c ^ L::v_swizzle(r)) << 4);
  }
  typedef __attribute__((address_space(3))) char* lds_ptr;
  char* const mine = lds + grp * RING * 2 * TILE;
  const uint32_t lds_at = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(lds_ptr)mine + wm * MINE);
  // The wave's part of the group's tile at u_pos, to place `to`.
  auto request = [&](int to) __attribute__((always_inline)) {
    const int j = u_pos + grp * UNITS + row0 / 16;
    const int what = j < kWave ? __builtin_amdgcn_readlane(u_what, j & 63) : 0;
    const long long slot = __builtin_amdgcn_readlane(u_slot, j & 63);
    const int valid = (what & 255) - row0 % 16;
    const size_t off = valid > 0 ? ((size_t)slot * W.tile_stride + (size_t)((what >> 8) * kUnitTokens + row0 % 16) * DH) * 2 : 0;
    const int bytes = valid > 0 ? valid * L::ROWB : 0;
    load_to_lds<NP>(static_cast<const char*>(W.k_pool) + off, bytes, k_from, lds_at + to * 2 * TILE);
    load_to_lds<NP>(static_cast<const char*>(W.v_pool) + off, bytes, v_from, lds_at + to * 2 * TILE + TILE);
  };
  constexpr uint64_t STEP_BITS = (1ull << STEP) - 1;
  auto is_full = [&]() __attribute__((always_inline)) { return (u_full >> u_pos & STEP_BITS) == STEP_BITS; };

  f32x16 acc[L::DT];
#pragma unroll
  for (int d = 0; d < L::DT; ++d)
#pragma unroll
    for (int i = 0; i < 16; ++i) acc[d][i] = 0.0f;
  float m = -INFINITY, l = 0.0f;

  // What the wave reads of a tile: K chunk 2 * s + half of row l32, and the values of tokens 4 * half + lane % 16 / 4 on (16-byte chunk
  // 4 * d + ..., 8 bytes of it).
  const int k_at = l32 * L::ROWB, k_x = L::k_swizzle(l32);
  const int v_tok = 4 * half + (lane & 15) / 4, v_x = L::v_swizzle(v_tok);
  const int v_at = v_tok * L::ROWB + ((lane & 3) & 1) * 8, v_c = 2 * ((lane >> 4) & 1) + (lane & 3) / 2;

  f32x16 x[NH];
  auto logits = [&](const char* k) __attribute__((always_inline)) {
#pragma unroll
    for (int hf = 0; hf < NH; ++hf)
#pragma unroll
      for (int i = 0; i < 16; ++i) x[hf][i] = 0.0f;
#pragma unroll
    for (int hf = 0; hf < NH; ++hf)
#pragma unroll
      for (int s = 0; s < L::KS; ++s) {
        const bf16x8 a = as_bf16x8(*reinterpret_cast<const u32x4*>(k + k_at + hf * 32 * L::ROWB + ((2 * s + half) ^ k_x) * 16));
        x[hf] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, q[s], x[hf], 0, 0, 0);
      }
  };
  auto largest = [&]() __attribute__((always_inline)) {  // of the tile's logits, in base-2 units
    float b = x[0][0];
#pragma unroll
    for (int hf = 0; hf < NH; ++hf)
#pragma unroll
      for (int i = 0; i < 16; ++i) b = fmaxf(b, x[hf][i]);
    return max_xor32(b) * W.scale2;
  };
  auto follow = [&](float b) __attribute__((always_inline)) {  // the maximum, where it has moved far
    const float m_new = b > m + kLag ? b : m, alpha = exp2_diff(m, m_new);
    l *= alpha;
#pragma unroll
    for (int d = 0; d < L::DT; ++d) acc[d] *= alpha;
    m = m_new;
  };
  auto values = [&](const char* v) __attribute__((always_inline)) {  // the logits' weights, and the weighted values
    const float m_sub = m == -INFINITY ? 0.0f : m;
    float sum[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    s16x8 p[TERMS][UNITS];
#pragma unroll
    for (int s = 0; s < UNITS; ++s) {  // eight registers: a step of the second product
      float w[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        w[e] = fast_exp2(fmaf(x[s / 2][8 * (s % 2) + e], W.scale2, -m_sub));
        sum[e & 3] += w[e];
      }
#pragma unroll
      for (int n = 0; n < TERMS; ++n) {
        u32x4 packed;
#pragma unroll
        for (int e = 0; e < 8; e += 2) {
          if (n + 1 < TERMS) {  // cut, not rounded: what is left is not negative
            const uint32_t a = __float_as_uint(w[e]), b = __float_as_uint(w[e + 1]);
            packed[e / 2] = pack_halves(a, b, 1);
            w[e] = what_is_left(w[e], a & 0xffff0000u);
            w[e + 1] = what_is_left(w[e + 1], b & 0xffff0000u);
          } else {
            packed[e / 2] = cvt_pk_bf16(w[e], w[e + 1]);
          }
        }
        p[n][s] = __builtin_bit_cast(s16x8, packed);
      }
    }
    l += (sum[0] + sum[1]) + (sum[2] + sum[3]);
#pragma unroll
    for (int s = 0; s < UNITS; ++s)
#pragma unroll
      for (int d = 0; d < L::DT; ++d) {
        typedef __attribute__((address_space(3))) s16x4* tr_ptr;
        const char* at = v + v_at + s * 16 * L::ROWB + ((4 * d + v_c) ^ v_x) * 16;
        const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((tr_ptr)(at));
        const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((tr_ptr)(at + 8 * L::ROWB));
        const bf16x8 a = __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
#pragma unroll
        for (int n = TERMS - 1; n >= 0; --n)
          acc[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, __builtin_bit_cast(bf16x8, p[n][s]), acc[d], 0, 0, 0);
      }
  };

  // Steps that are on their way, the one at hand among them; whether the last of them is not full, and the counts of the group's tile there.
  int flying = 0, at = 0, next = 0;
  bool partial = false;
  Counts tokens = 0;
  auto ask = [&]() __attribute__((always_inline)) {
    if (u_n <= u_pos) return;
    if (!is_full()) {
      partial = true;
#pragma unroll
      for (int u = 0; u < UNITS; ++u) {
        const int j = u_pos + grp * UNITS + u;
        tokens |= (Counts)(j < kWave ? __builtin_amdgcn_readlane(u_what, j & 63) & 255 : 0) << (8 * u);
      }
    }
    request(next);
    next = next == RING - 1 ? 0 : next + 1;
    ++flying;
    u_pos += STEP;
    if (u_n - u_pos < STEP) refill();
  };
  // The wave's part of the step at hand has arrived, so has everybody's behind the barrier, and nobody reads the step before it any more.
  auto arrive = [&]() __attribute__((always_inline)) {
    if (flying == RING - 1) await<(RING - 2) * 2 * NP>();
    else await<0>();
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
  };
  refill();
#pragma unroll
  for (int n = 0; n < RING - 1; ++n) ask();
  // full tiles
  while (flying > (int)partial) {
    arrive();
    ask();
    logits(mine + at * 2 * TILE);
    const float b = largest();
    if (__ballot(b > m + kLag) != 0) follow(b);
    values(mine + at * 2 * TILE + TILE);
    at = at == RING - 1 ? 0 : at + 1;
    --flying;
  }
  if (partial) {
    arrive();
    if (tokens != 0) {
      char* const v = mine + at * 2 * TILE + TILE;
      logits(mine + at * 2 * TILE);
#pragma unroll
      for (int hf = 0; hf < NH; ++hf)
#pragma unroll
        for (int i = 0; i < 16; ++i)
          if (8 * (i / 4 % 2) + 4 * half + i % 4 >= (int)(tokens >> (8 * (2 * hf + i / 8)) & 255)) x[hf][i] = -INFINITY;
      // rows that do not count become zero, whatever lies there (every wave sees to that by itself: LDS serves a wave's accesses in order)
      for (int c = lane; c < TOK * L::CH; c += kWave) {
        const int r = c / L::CH;
        if (r % 16 >= (int)(tokens >> (8 * (r / 16)) & 255)) *reinterpret_cast<u32x4*>(v + c * 16) = (u32x4){0, 0, 0, 0};
      }
      wave_exchange();
      follow(largest());
      values(v);
    }
  }
  l = sum_xor32(l);

  // the groups' sums, lane by lane, where the tiles were
  if constexpr (WN > 1) {
    constexpr int AREA = (L::DT * 16 + 2) * kWave;  // floats of a wave
    float* const sums = reinterpret_cast<float*>(lds);
    __syncthreads();
    if (grp > 0) {
      float* const to = sums + ((grp - 1) * WM + wm) * AREA + lane;
#pragma unroll
      for (int d = 0; d < L::DT; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) to[(d * 16 + i) * kWave] = acc[d][i];
      to[L::DT * 16 * kWave] = m;
      to[(L::DT * 16 + 1) * kWave] = l;
    }
    __syncthreads();
    if (grp > 0) return;
    float M = m;
#pragma unroll
    for (int g = 1; g < WN; ++g) M = fmaxf(M, sums[((g - 1) * WM + wm) * AREA + lane + L::DT * 16 * kWave]);
    const float f0 = exp2_diff(m, M);
    m = M;
    l *= f0;
#pragma unroll
    for (int d = 0; d < L::DT; ++d) acc[d] *= f0;
#pragma unroll
    for (int g = 1; g < WN; ++g) {
      const float* from = sums + ((g - 1) * WM + wm) * AREA + lane;
      const float f = exp2_diff(from[L::DT * 16 * kWave], M);
      l += f * from[(L::DT * 16 + 1) * kWave];
#pragma unroll
      for (int d = 0; d < L::DT; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[d][i] += f * from[(d * 16 + i) * kWave];
    }
  }
  if (!real) return;
  const size_t to = out_row * kMaxPrefixSplits + it.split;
#pragma unroll
  for (int d = 0; d < L::DT; ++d)
#pragma unroll
    for (int i = 0; i < 16; i += 4)
      *reinterpret_cast<float4*>(W.po + to * DH + d * 32 + 8 * (i / 4) + 4 * half) =
          make_float4(acc[d][i], acc[d][i + 1], acc[d][i + 2], acc[d][i + 3]);
  if (half == 0) {
    W.pm[to] = m;
    W.pl[to] = l;
  }
}

// ---------------------------------------------------------------- the splits, and the sequence's own partial

struct PrefixOut {
  const float *o_b, *m_b, *l_b;  // the other partial, or all null
  float *o, *m, *l;              // the joined partial, or all null
  void* out;                     // the joined result, or null
  float* lse;                    // or null
};

// A wave per query row: lane s holds the maximum and the sum of split s.  Bound by a launch and two trips to memory, then by the sums: 3 to 4 us
// for 128 rows, 5.3 for 1024 rows of 32 splits (17 MB), 8.4 for 4096 of 16 (34 MB).
template <int DT, int DH>
__global__ __launch_bounds__(256) void prefix_combine_kernel(PrefixPlan P, PrefixStamp stamp, PrefixWork W, PrefixOut E) {
  constexpr int N = DH / kWave;  // channels per lane
  typedef typename Channels<N>::f chans;
  const int lane = lane_id(), row = blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  if (row >= W.B * W.Hq) return;
  const int c = lane * N;
  float mb = -INFINITY, lb = 0.0f;
  chans ob{};
  if (E.o_b != nullptr) {
    mb = E.m_b[row];
    lb = E.l_b[row];
    ob = *reinterpret_cast<const typename Channels<N>::f_any*>(E.o_b + (size_t)row * DH + c);
  }
  // In the first trip: how many splits there are, all that they say, and the sums of the first ones.
  const size_t at = (size_t)row * kMaxPrefixSplits;
  constexpr int TRIP = 16;  // splits requested at a time
  float ms = W.pm[at + lane], ls = W.pl[at + lane];
  const __amdgpu_buffer_rsrc_t sums = __builtin_amdgcn_make_buffer_rsrc(W.po + at * DH, 0, kMaxPrefixSplits * DH * 4, 0x00020000);
  chans x[TRIP];
  auto request = [&](int s0) __attribute__((always_inline)) {
#pragma unroll
    for (int u = 0; u < TRIP; ++u) {
      const int off = ((s0 + u) * DH + c) * 4;
      if constexpr (N == 2) x[u] = __builtin_bit_cast(chans, __builtin_amdgcn_raw_buffer_load_b64(sums, off, 0, 0));
      else x[u][0] = __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(sums, off, 0, 0));
    }
  };
  request(0);
  const int n = made_for(P, stamp) ? P.splits[row / W.Hq] : 0;
  ms = lane < n ? ms : -INFINITY;
  ls = lane < n ? ls : 0.0f;
  float M = ms;
#pragma unroll
  for (int s = 1; s < kWave; s <<= 1) M = fmaxf(M, __shfl_xor(M, s));
  const float f = exp2_diff(ms, M);
  ls *= f;
#pragma unroll
  for (int s = 1; s < kWave; s <<= 1) ls += __shfl_xor(ls, s);
  chans o{};
  for (int s0 = 0; s0 < n; s0 += TRIP) {
    if (s0 > 0) request(s0);
#pragma unroll
    for (int u = 0; u < TRIP; ++u) {
      const float w = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(f), s0 + u));
      if (w != 0.0f) o += w * x[u];  // a split without tokens has no weight, and what lies beyond the last one none either
    }
  }
  // The two partials as one.  A side without tokens (sum zero) has no weight, whatever its other numbers; a sum that is NaN
  // stays one.
  const float ma = M * kLn2;
  const float top = fmaxf(ls == 0.0f ? -INFINITY : ma, lb == 0.0f ? -INFINITY : mb);
  const float ea = ls == 0.0f ? 0.0f : expf(ma - top), wb = lb == 0.0f ? 0.0f : lb * expf(mb - top);
  const float sum = ls * ea + wb;
  chans r{};
#pragma unroll
  for (int i = 0; i < N; ++i) {
    float y = ea == 0.0f ? 0.0f : ea * o[i];  // o is not divided by its sum
    if (wb != 0.0f) y += wb * ob[i];
    r[i] = sum == 0.0f ? 0.0f : y / sum;
  }
  const size_t to = (size_t)row * DH + c;
  if (E.out != nullptr) {
    if constexpr (DT == SCOUT_BF16) {
      typename Channels<N>::h w;
#pragma unroll
      for (int i = 0; i < N; ++i) w[i] = (uint16_t)f32_to_bf16_bits(r[i]);
      *reinterpret_cast<typename Channels<N>::h_any*>(static_cast<uint16_t*>(E.out) + to) = w;
    } else {
      *reinterpret_cast<typename Channels<N>::f_any*>(static_cast<float*>(E.out) + to) = r;
    }
    if (E.lse != nullptr && lane == 0) E.lse[row] = sum == 0.0f ? -INFINITY : top + logf(sum);
  }
  if (E.o != nullptr) {
    *reinterpret_cast<typename Channels<N>::f_any*>(E.o + to) = r;
    if (lane == 0) {
      E.m[row] = top;
      E.l[row] = sum;
    }
  }
}

// ---------------------------------------------------------------- launches

// How the work of a batch is dealt: by the rows that a prefix has on average (the rows of a prefix with more are several tiles), the least tile that
// holds them.  Attention and fold, 8 KV heads of 128 channels, one prefix, us with the smaller | the larger tile:
//   16 | 32    24 rows: 32k tokens 36 | 35, 128k 108 | 102; fp32, 32 rows: 8k tokens 23 | 26, 64k 119 | 112
//   32 | 64    48 rows: 32k 39.9 | 39.2; 64 rows: 128k 114 | 105
//   64 | 128   96 rows: 32k 46.9 | 46.9; 128 rows: 128k 145 | 129
//   128 | 256  192 rows: 32k 63.7 | 65.4, 256 rows: 69.7 | 68.2, 128k 220 | 199
// Over a few thousand tokens smaller tiles are faster, having more workgroups (64 rows, 4096 tokens: 13.5 with 16, 17.4 with 64).
// granule: a step of every kernel is 128 tokens; 64, 128 and 256 differ by 1 %, and short prefixes have more splits with 64.
// head_cost: 48 sequences over five prefixes of 3000 to 24000 tokens 83 us with 0 and 128, 78 with 256, 512 and 1024; others within 2 %.
static PrefixShape prefix_shape(const Dims& D, int dtype, int n_prefix) {
  const long long rows = ((long long)D.B * D.G + n_prefix - 1) / (n_prefix > 0 ? n_prefix : 1);
  PrefixShape s;
  if (dtype == SCOUT_F32) s.tile_rows = rows <= 16 ? 16 : 32;
  else s.tile_rows = rows <= 16 ? 16 : rows <= 32 ? 32 : rows <= 64 ? 64 : rows <= 128 ? 128 : 256;
  s.granule = 64;
  s.slots = 256;
  s.head_cost = 256;
  return s;
}

// Items are workgroups of 512 threads, of which a launch has below 2^32.
constexpr long long kMostItems = 1ll << 23;

static int max_items(const Dims& D, const PrefixShape& s, int n_prefix) {
  const long long tiles = (long long)D.B * D.G / s.tile_rows + n_prefix;
  const long long n = tiles * D.Hkv + 2 * s.slots;
  return n >= kMostItems ? -1 : (int)n;
}

static PrefixStamp prefix_stamp(const Dims& D, int dtype, const PrefixShape& s, int n_prefix, int prefix_blocks, int items) {
  return PrefixStamp{{0x50726669, D.B, D.Hq, D.Hkv, D.d, D.S, dtype, n_prefix, prefix_blocks, s.tile_rows, s.granule, items}};
}

long long prefix_plan_words(const Dims& D, int dtype, int n_prefix) {
  const int items = max_items(D, prefix_shape(D, dtype, n_prefix), n_prefix);
  return items < 0 ? -1 : PrefixPlan::words(D.B, items);
}

int launch_prefix_plan(const Dims& D, int dtype, int n_prefix, int prefix_blocks, const int32_t* prefix_of, const int32_t* prefix_len,
                       void* plan, hipStream_t st) {
  const PrefixShape s = prefix_shape(D, dtype, n_prefix);
  const int items = max_items(D, s, n_prefix);
  hipLaunchKernelGGL(prefix_plan_kernel, dim3(1), dim3(kPlanThreads), 0, st, PrefixPlan::at(plan, D.B, items),
                     prefix_stamp(D, dtype, s, n_prefix, prefix_blocks, items), s, D.B, D.Hkv, D.G, n_prefix, prefix_blocks * D.S,
                     prefix_of, prefix_len);
  return hipGetLastError() == hipSuccess ? SCOUT_OK : SCOUT_EHIP;
}

template <int DT, int DH>
static void launch_all(const Dims& D, const PrefixShape& s, int items, const PrefixPlan& P, const PrefixStamp& stamp, const PrefixWork& W,
                       const PrefixOut& E, hipStream_t st) {
  const dim3 g(items);
  if (s.tile_rows == 16) {
    hipLaunchKernelGGL((prefix_narrow_kernel<DT, DH, 1>), g, dim3(512), 0, st, P, stamp, W);
  } else if (s.tile_rows == 32) {
    hipLaunchKernelGGL((prefix_narrow_kernel<DT, DH, 2>), g, dim3(512), 0, st, P, stamp, W);
  } else if constexpr (DT == SCOUT_BF16) {
    if (s.tile_rows == 64) hipLaunchKernelGGL((prefix_wide_kernel<DH, 2, 4, 32>), g, dim3(512), 0, st, P, stamp, W);
    else if (s.tile_rows == 128) hipLaunchKernelGGL((prefix_wide_kernel<DH, 4, 2, 64>), g, dim3(512), 0, st, P, stamp, W);
    else hipLaunchKernelGGL((prefix_wide_kernel<DH, 8, 1, 128>), g, dim3(512), 0, st, P, stamp, W);
  }
  hipLaunchKernelGGL((prefix_combine_kernel<DT, DH>), dim3((D.B * D.Hq + 3) / 4), dim3(256), 0, st, P, stamp, W, E);
}

int launch_prefix_attn(const Dims& D, int dtype, int n_prefix, int prefix_blocks, void* plan, const void* q, const void* k_pool,
                       const void* v_pool, long long n_slots, const int32_t* table, const float* o_b, const float* m_b, const float* l_b,
                       float* o, float* m, float* l, void* out, float* lse, float* po, float* pm, float* pl, hipStream_t st) {
  const PrefixShape s = prefix_shape(D, dtype, n_prefix);
  const int items = max_items(D, s, n_prefix);
  const PrefixPlan P = PrefixPlan::at(plan, D.B, items);
  const PrefixStamp stamp = prefix_stamp(D, dtype, s, n_prefix, prefix_blocks, items);
  const PrefixWork W{D.B, D.Hq, D.Hkv, D.G, D.S, D.s_shift, D.tile_stride, prefix_blocks, n_prefix,
                     D.G > 1 ? (uint32_t)(((1ull << 32) + D.G - 1) / D.G) : 0, D.sm_scale * kLog2e, n_slots, q, k_pool, v_pool, table, po,
                     pm, pl};
  const PrefixOut E{o_b, m_b, l_b, o, m, l, out, lse};
  if (D.B == 0) return SCOUT_OK;
  if (dtype == SCOUT_BF16) D.d == 128 ? launch_all<SCOUT_BF16, 128>(D, s, items, P, stamp, W, E, st) : launch_all<SCOUT_BF16, 64>(D, s, items, P, stamp, W, E, st);
  else D.d == 128 ? launch_all<SCOUT_F32, 128>(D, s, items, P, stamp, W, E, st) : launch_all<SCOUT_F32, 64>(D, s, items, P, stamp, W, E, st);
  return hipGetLastError() == hipSuccess ? SCOUT_OK : SCOUT_EHIP;
}

}  // namespace scout
