// What the attention kernels share: how a unit of 16 tokens lies in the lanes and how it is requested, and how partial results
// meet and leave.
#pragma once
#include "common.h"

namespace scout {

typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;

// bare v_exp_f32: results below 2^-126 flush to zero, which rescaling factors and rounded weights can afford
__device__ __forceinline__ float fast_exp2(float x) { return __builtin_amdgcn_exp2f(x); }

__device__ __forceinline__ float exp2_diff(float a, float b) {
  // 2^(a-b) with the convention 2^(-inf - anything) = 0
  return a == -INFINITY ? 0.0f : fast_exp2(a - b);
}

// ---------------------------------------------------------------- MFMA family

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(2))) uint32_t u32x2;

__device__ __forceinline__ bf16x8 as_bf16x8(u32x4 v) { return __builtin_bit_cast(bf16x8, v); }

// Pack the low (sel = 0) or high (sel = 1) bf16 of two dwords into one dword:
// result.lo = half(a), result.hi = half(b).  One v_perm_b32: its selector bytes
// 0-3 address the second source operand, 4-7 the first.
__device__ __forceinline__ uint32_t pack_halves(uint32_t a, uint32_t b, int sel) {
  return sel ? __builtin_amdgcn_perm(b, a, 0x07060302u) : __builtin_amdgcn_perm(b, a, 0x05040100u);
}

typedef __attribute__((ext_vector_type(2))) float f32x2;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;

// two binary32 -> one dword of two bf16 (round to nearest even), x in the low half
__device__ __forceinline__ uint32_t cvt_pk_bf16(float x, float y) {
  return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2){x, y}, bf16x2));
}

// N consecutive channels of a head.  The arrays may start anywhere that an element of theirs may.
template <int N>
struct Channels {
  typedef __attribute__((ext_vector_type(N))) float f;
  typedef f f_any __attribute__((aligned(4)));
  typedef __attribute__((ext_vector_type(N))) uint16_t h;
  typedef h h_any __attribute__((aligned(2)));
};
// Channels per thread in the epilogues of the attention: the weights of the two partials are made once for them.  Two: of four, the
// divisions are a chain that few threads run; of one, every thread makes weights of its own.
constexpr int CH = 2;
typedef Channels<CH>::f fch;

// The host's partial for a thread's channels (mode 2 only); loaded ahead of the point of use so
// that its latency hides behind the fold.
template <int N>
struct HostPart {
  typename Channels<N>::f o;
  float m, l;
};

template <int N>
__device__ __forceinline__ HostPart<N> load_host(const Dims& D, const Epilogue& E, int bh, int c) {
  HostPart<N> hp{};
  hp.m = -INFINITY;
  if (E.mode == 2 && E.host_o != nullptr) {
    hp.m = E.host_m[bh];
    hp.l = E.host_l[bh];
    hp.o = *reinterpret_cast<const typename Channels<N>::f_any*>(E.host_o + (size_t)bh * D.d + c);
  }
  return hp;
}

// Merge of the partial (oa, ma, la) of head bh, channels c on, with the other one: `at` is the place of the channels in `out`.
template <int N>
__device__ __forceinline__ void merge_channels(void* out, int dtype_out, float* lse, size_t at, int bh, int c,
                                               typename Channels<N>::f oa, float ma, float la, const HostPart<N>& other) {
  const float mb = other.m, lb = other.l;
  float ms = -INFINITY;
  if (la > 0.0f) ms = fmaxf(ms, ma);
  if (lb > 0.0f) ms = fmaxf(ms, mb);
  const float wa = la > 0.0f ? la * expf(ma - ms) : 0.0f;
  const float wb = lb > 0.0f ? lb * expf(mb - ms) : 0.0f;
  const float ls = wa + wb;
  typename Channels<N>::f r;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    float x = 0.0f;
    if (wa > 0.0f) x += wa * oa[i];
    if (wb > 0.0f) x += wb * other.o[i];
    r[i] = ls > 0.0f ? x / ls : 0.0f;
  }
  if (dtype_out == SCOUT_BF16) {
    typename Channels<N>::h w;
#pragma unroll
    for (int i = 0; i < N; ++i) w[i] = (uint16_t)f32_to_bf16_bits(r[i]);
    *reinterpret_cast<typename Channels<N>::h_any*>(static_cast<uint16_t*>(out) + at) = w;
  } else {
    *reinterpret_cast<typename Channels<N>::f_any*>(static_cast<float*>(out) + at) = r;
  }
  if (lse != nullptr && c == 0) lse[bh] = ls > 0.0f ? ms + logf(ls) : -INFINITY;
}

// acc: unnormalised weighted value sums of the channels, l: weight sum, M2: base-2 maximum
template <int N>
__device__ __forceinline__ void finish(const Dims& D, const Epilogue& E, int bh, int c, typename Channels<N>::f acc, float l, float M2,
                                       const HostPart<N>& hp) {
  const float m_nat = M2 * kLn2;  // -inf stays -inf
  typename Channels<N>::f r;
#pragma unroll
  for (int i = 0; i < N; ++i) r[i] = l > 0.0f ? acc[i] / l : 0.0f;
  const size_t at = (size_t)bh * D.d + c;
  if (E.mode == 1) {
    *reinterpret_cast<typename Channels<N>::f_any*>(E.o + at) = r;
    if (c == 0) {
      E.m[bh] = m_nat;
      E.l[bh] = l;
    }
    return;
  }
  merge_channels<N>(E.out, E.dtype_out, E.lse, at, bh, c, r, m_nat, l, hp);
}

// The work of a pair is cut into units of 16 tokens (a block of S tokens is S/16 units; a unit's K
// rows and V rows are contiguous, 4 KiB each at bf16, d = 128).  The pair's units are dealt to the waves that share
// the pair (all waves of all its workgroups) in contiguous ranges whose lengths differ by at most
// one, so no wave waits for a neighbour that got a whole block more.  For each unit:
//   logits^T[token][head] = K[token][:] . Q[head][:]            bf16: d/32 x mfma 16x16x32, fp32: d/4 x mfma 16x16x4
//   online softmax per head (heads live in lane % 16)
//   out^T[dim][head]    += V^T[dim][token] . P^T[token][head]   bf16: d/16 x mfma 16x16x16 per term of a weight (kWeights32),
//                                                               fp32: d/4 x mfma 16x16x4
// Operand layout of the 16x16 MFMAs: lane L supplies, for A, row L%16 and for B, column L%16, the
// contraction elements of group L/16 (8 of them for x32, 4 for x16, 1 for x4); the result has column L%16 and
// rows 4*(L/16)+i.  The contraction index may be labelled freely as long as A and B agree, which
// lets the logits leave the first product in exactly the registers the second one needs: lane L
// ends up with the logits of head L%16 for tokens 4*(L/16) + i (i = 0..3), so the value rows are
// loaded in that same token order.  Element e of a lane's value chunk c feeds product r = c * CPC + e, whose
// output row index R then means channel CPC * (R + 16 * c) + e.
//
// fp32 goes through the fp32 matrix instructions (products and sums in binary32, as on the vector ALU,
// and the softmax weights are not rounded): 2048 matrix cycles per unit of 16 KiB at d = 128 are 8 bytes
// per cycle and SIMD, 2.5 times what HBM delivers, so the pass stays bandwidth-bound.
//
// The waves of a workgroup fold their partials through LDS; with one split per pair the workgroup
// finishes the pair itself (Epilogue modes 1 and 2), so the whole attention is one launch and
// nothing goes through the workspace.

constexpr int kUnitTokens = 16;

typedef __attribute__((ext_vector_type(4))) short s16x4;

// How a unit of (element type DT, head dim DH) lies in the lanes.
template <int DT, int DH>
struct Tile {
  static constexpr int ES = DT == SCOUT_BF16 ? 2 : 4;  // bytes per element
  static constexpr int ROWB = DH * ES;                 // bytes per token row
  static constexpr int UNITB = kUnitTokens * ROWB;     // bytes of K, and of V, per unit
  static constexpr int KL = ROWB / 64;                 // 16-byte K loads per lane: chunk 4 * s + kg of row ln
  static constexpr int CB = ROWB / 16 < 16 ? ROWB / 16 : 16;  // bytes of a lane's value chunk
  static constexpr int VC = ROWB / 16 / CB;            // value chunks per lane and row: chunk ln + 16 * c
  static constexpr int CPC = CB / ES;                  // channels per value chunk
  static constexpr int NR = DH / 16;                   // products (accumulator tiles) of the second contraction
  // channel of accumulator tile r, row index R
  static __device__ __forceinline__ constexpr int channel(int r, int R) { return CPC * (R + 16 * (r / CPC)) + r % CPC; }
};

// Whether the softmax weights enter the second product in binary32: for fp32, and for bf16 with d = 64 (bf16 with d = 128
// rounds them to bf16).  With bf16 values a binary32 weight goes as the sum of three bf16 terms, 24 bits, each multiplied
// with the values on the bf16 matrix instructions.  8 sequences x 8 KV heads with 128 blocks of 16 tokens listed: the
// attention takes 8.7 us, 8.5 with weights of one term, 9.8 through the fp32 matrix instructions, 30 on the vector ALU.
// Error of the outputs against binary64 (2-norm, lists of 64 to 2048 tokens, logits of standard deviation 0.3, 1, 2), three
// terms and vector ALU: 1.07 and 1.34e-7, 1.42 and 1.60e-7, 2.05 and 2.12e-7; one term: 3e-4 to 1.5e-3.  A term may be zero or negative, which
// makes a NaN of an infinite value, so a wave whose sums hold a NaN starts over with the weights whole, through the fp32
// matrix instructions (EXACT): infinite values give what they give everywhere.
template <int DT, int DH>
constexpr bool kWeights32 = DT == SCOUT_F32 || DH == 64;

// The group's queries as operand registers: 16-byte chunk 4 * s + kg of head ln.
template <int DT, int DH>
using QRegs = u32x4[Tile<DT, DH>::KL];

// K and V rows of one unit in MFMA operand registers.
template <int DT, int DH>
struct UnitRegs {
  u32x4 k[Tile<DT, DH>::KL];     // contraction step s: row = token ln, 16-byte chunk 4*s + kg
  u32x4 v[4][Tile<DT, DH>::VC];  // row = token 4*kg + i, chunk ln + 16*c (8-byte chunks use half the register)
};

// One unit, checked: where it starts in the pools (element offset) and how many of its tokens
// count (0 = nothing to read).
struct Entry {
  size_t elem_off;
  int valid;
};

// sel / slot_list point at the pair's list (global memory or LDS); u is wave-uniform.
template <int DH>
__device__ __forceinline__ Entry read_entry(const int32_t* sel, const int32_t* slot_list, int u, int u_end,
                                            int ush, int S, int ctx, long long n_slots, int tile_stride) {
  Entry e{0, 0};
  if (u < u_end) {
    const int i = u >> ush, sub = u - (i << ush);  // ush = log2(units per block)
    const int j = __builtin_amdgcn_readfirstlane(sel[i]);
    const long long slot = __builtin_amdgcn_readfirstlane(slot_list[i]);
    int valid = ctx - j * S - sub * kUnitTokens;
    valid = valid > kUnitTokens ? kUnitTokens : valid;
    if (j >= 0 && valid > 0 && slot >= 0 && slot < n_slots) {
      e.elem_off = (size_t)slot * tile_stride + sub * kUnitTokens * DH;
      e.valid = valid;
    }
  }
  return e;
}

// Request a unit.  The loads go through a buffer descriptor that covers exactly the unit, or nothing
// when the entry is void: then every lane gets zeros without touching memory.  That keeps the issue
// path free of branches, so the compiler can count outstanding loads exactly and a wave can wait for
// one unit while the next ones are still in flight.
template <int DT, int DH>
__device__ __forceinline__ void issue_unit(UnitRegs<DT, DH>& T, const void* __restrict__ k_pool,
                                           const void* __restrict__ v_pool, const Entry& e, int ln, int kg) {
  using L = Tile<DT, DH>;
  const int bytes = e.valid > 0 ? L::UNITB : 0;
  char* kp = static_cast<char*>(const_cast<void*>(k_pool)) + e.elem_off * L::ES;
  char* vp = static_cast<char*>(const_cast<void*>(v_pool)) + e.elem_off * L::ES;
  // Both descriptors stand before the first request.  Left to itself the compiler made the second one between the K and
  // the V requests and spread these over the matrix instructions in front of them: a selection per query head of 512 pairs
  // (64 listed blocks each) took 35.1 us for the attention instead of 33.2, inside a step 37.9 instead of 37.0; 256 ragged pairs 27.6 and 27.2.
  // Other types and head dims gain nothing from it.
  constexpr bool TOGETHER = DT == SCOUT_BF16 && DH == 128;
  if constexpr (TOGETHER) asm volatile("" : "+s"(kp), "+s"(vp));
  const __amdgpu_buffer_rsrc_t kr = __builtin_amdgcn_make_buffer_rsrc(kp, 0, bytes, 0x00020000);
  const __amdgpu_buffer_rsrc_t vr = __builtin_amdgcn_make_buffer_rsrc(vp, 0, bytes, 0x00020000);
  const int koff = ln * L::ROWB + kg * 16;           // row ln, 16-byte chunk 4*s + kg
  const int voff = kg * 4 * L::ROWB + ln * L::CB;    // row 4*kg + i, chunk ln + 16*c
  if constexpr (TOGETHER) __builtin_amdgcn_sched_barrier(0x00A);  // only vector and matrix instructions may pass
#pragma unroll
  for (int s = 0; s < L::KL; ++s)
    T.k[s] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(kr, koff + s * 64, 0, 0));
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int c = 0; c < L::VC; ++c) {
      const int off = voff + i * L::ROWB + c * 16 * L::CB;
      if constexpr (L::CB == 16) {
        T.v[i][c] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(vr, off, 0, 0));
      } else {
        const u32x2 w = __builtin_bit_cast(u32x2, __builtin_amdgcn_raw_buffer_load_b64(vr, off, 0, 0));
        T.v[i][c][0] = w[0];
        T.v[i][c][1] = w[1];
      }
    }
}

}  // namespace scout
