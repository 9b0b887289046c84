// The pages of a cache that several sequences share: who holds a slot, taking the lowest free ones, forking a sequence,
// freeing one, compacting the pool.
//
// State (struct Pages, one buffer of the caller's): refs[slot], how many block-table entries name the slot, and used, a bit per
// slot that is set while refs > 0.  The bits are what free slots are looked for in: 100 000 slots are 12.5 KB, one trip of one
// workgroup, where the counts themselves are 400 KB.  A slot is taken lowest first and in the order of the takers (child, KV
// head, block), by ranks: the r-th taker gets the r-th clear bit.  So the same state gives the same slots, whatever order
// the workgroups run in; the atomics that count references up and down are integer additions, whose order changes nothing.
//
// A fork and a compaction plan in one launch (who is refused, which ranks, which slots) and move bytes in the next one (digest rows,
// table rows, tiles).
#include "pages.h"

#include "plan_scan.h"

namespace scout {

constexpr int kCopyThreads = 256;

// Bits of slots that exist, of word w.
__device__ __forceinline__ uint32_t exists(long long n_slots, long long w) {
  const long long left = n_slots - w * 32;
  return left >= 32 ? 0xffffffffu : left <= 0 ? 0u : (1u << left) - 1u;
}

// Words of `used` that slots are taken from, put in a row so that all waves hand them out: few takers find their slots in few
// words, many in all of them.
struct TakenWords {
  int n[2];  // by turns, so that one can be cleared while the other is read
  uint32_t bits[kPlanThreads];
  int word[kPlanThreads], rank[kPlanThreads];
};

// The `want` lowest free slots, ascending, to list (as many as there are; the number is returned to every thread).  They
// become used with one reference each.  The whole planning workgroup calls this.
__device__ int take_lowest(const Pages& P, long long want, int32_t* list, int* lds) {
  __shared__ TakenWords T;
  const long long nw = words_of(P.n_slots);
  const int lane = lane_id();
  long long got = 0;
  int turn = 0;
  if (threadIdx.x < 2) T.n[threadIdx.x] = 0;
  for (long long w0 = 0; w0 < nw && got < want; w0 += kPlanThreads, turn ^= 1) {
    const long long w = w0 + threadIdx.x;
    const uint32_t old = w < nw ? P.used[w] : ~0u, free_bits = ~old & exists(P.n_slots, w);
    int total;
    const long long at = got + plan_scan(__popc(free_bits), lds, &total);
    if (threadIdx.x == 0) T.n[turn ^ 1] = 0;
    uint32_t taken = at < want ? free_bits : 0u;
    for (long long more = taken ? at + __popc(taken) - want : 0; more > 0; --more) taken &= ~(0x80000000u >> __clz(taken));  // the highest ones stay
    const uint64_t takes = __ballot(taken != 0);
    if (takes != 0) {
      int first = 0;
      if (lane == 0) first = atomicAdd(&T.n[turn], (int)__popcll(takes));
      first = __builtin_amdgcn_readfirstlane(first);
      if (taken) {
        P.used[w] = old | taken;
        const int to = first + mbcnt64(takes);
        T.bits[to] = taken;
        T.word[to] = (int)w;
        T.rank[to] = (int)at;
      }
    }
    __syncthreads();
    // two words of a wave at a time, a lane per slot, so that neighbours are stored together
    const int n = T.n[turn];
#pragma unroll 2
    for (int k = threadIdx.x / 32; k < n; k += kPlanThreads / 32) {
      const uint32_t bits = T.bits[k], bit = 1u << (lane & 31);
      if (bits & bit) {
        const int slot = T.word[k] * 32 + (lane & 31);
        list[T.rank[k] + __popc(bits & (bit - 1))] = slot;
        P.refs[slot] = 1;
      }
    }
    got += total;
  }
  return (int)(got < want ? got : want);
}

__device__ __forceinline__ bool has_slot(int entry, long long n_slots) { return entry >= 0 && entry < n_slots; }

// ---------------------------------------------------------------- the state of a cache that is there already

__global__ __launch_bounds__(kCopyThreads) void pages_clear_kernel(Pages P) {
  const long long n = P.n_slots, step = (long long)gridDim.x * kCopyThreads;
  for (long long i = (long long)blockIdx.x * kCopyThreads + threadIdx.x; i < n; i += step) P.refs[i] = 0;
}

__global__ __launch_bounds__(kCopyThreads) void pages_count_kernel(Dims D, Pages P, const int32_t* __restrict__ ctx_len, int32_t* table) {
  const int pair = grid_pair(), nb = num_blocks(D, ctx_len[blockIdx.z]);
  int32_t* const row = table + (size_t)pair * D.max_blocks;
  for (int j = blockIdx.x * kCopyThreads + threadIdx.x; j < D.max_blocks; j += gridDim.x * kCopyThreads) {
    const int e = row[j];
    if (j >= nb) row[j] = -1;
    else if (has_slot(e, P.n_slots)) atomicAdd(P.refs + e, 1);
  }
}

__global__ __launch_bounds__(kCopyThreads) void pages_bits_kernel(Pages P) {
  const long long nw = words_of(P.n_slots), step = (long long)gridDim.x * kCopyThreads;
  for (long long w = (long long)blockIdx.x * kCopyThreads + threadIdx.x; w < nw; w += step) {
    uint32_t bits = 0;
    for (int i = 0; i < 32 && w * 32 + i < P.n_slots; ++i) bits |= (uint32_t)(P.refs[w * 32 + i] > 0) << i;
    P.used[w] = bits;
  }
}

// ---------------------------------------------------------------- slots for the blocks that the next token opens

// Two trips to memory, one after the other, and a launch: 2.3 us where no block is opened, 4 for 128 takers among 20 000 slots.
__global__ __launch_bounds__(kPlanThreads) void reserve_kernel(Dims D, Pages P, const int32_t* __restrict__ ctx_len, int32_t* new_slot,
                                                               int32_t* n_short) {
  __shared__ int lds[kPlanWaves];
  const int capacity = D.max_blocks * D.S;
  long long want = 0;
  // sequences that open a block; the rank of a sequence's first KV head stays in scratch
  for (int b0 = 0; b0 < D.B; b0 += kPlanThreads) {
    const int b = b0 + threadIdx.x;
    const int t = b < D.B ? ctx_len[b] : -1;
    const bool opens = t >= 0 && t < capacity && (t & (D.S - 1)) == 0;
    int total;
    const int before = plan_scan(opens ? D.Hkv : 0, lds, &total);
    if (b < D.B) P.base[b] = opens ? (int)want + before : -1;
    want += total;
  }
  __syncthreads();
  const int got = want > 0 ? take_lowest(P, want, P.list, lds) : 0;
  __syncthreads();
  const int pairs = D.B * D.Hkv;
  for (int p = threadIdx.x; p < pairs; p += kPlanThreads) {
    const int b = p / D.Hkv, rank = P.base[b];
    const int r = rank + p - b * D.Hkv;
    new_slot[p] = rank >= 0 && r < got ? P.list[r] : -1;
  }
  if (threadIdx.x == 0) *n_short = (int)want - got;
}

// ---------------------------------------------------------------- fork

// Whether entry j of a sequence with ctx tokens gets a slot of its own in the child: every block (deep), or the last one where
// tokens will still be added to it.  Full blocks never change, so they can be shared for good.
__device__ __forceinline__ bool is_copied(const Dims& D, bool deep, int ctx, int nb, int j) {
  return deep ? j < nb : j == nb - 1 && (ctx & (D.S - 1)) != 0 && ctx < D.max_blocks * D.S;
}

// Entries with a slot of every row that a deep fork copies: a workgroup per row.
__global__ __launch_bounds__(kCopyThreads) void fork_count_kernel(Dims D, Pages P, const int32_t* __restrict__ src,
                                                                  const int32_t* __restrict__ ctx_len, const int32_t* __restrict__ table) {
  __shared__ int lds[kCopyThreads / kWave];
  const int r = blockIdx.x, i = r / D.Hkv, s = src[i];
  int c = 0;
  if (s >= 0 && s < D.B) {
    const int nb = num_blocks(D, ctx_len[s]);
    const int32_t* row = table + ((size_t)s * D.Hkv + (r - i * D.Hkv)) * D.max_blocks;
#pragma unroll 4
    for (int j = threadIdx.x; j < nb; j += kCopyThreads) c += has_slot(row[j], P.n_slots);
  }
  c = wave_scan(c, lane_id());
  if (lane_id() == kWave - 1) lds[threadIdx.x / kWave] = c;
  __syncthreads();
  if (threadIdx.x == 0) {
    int all = 0;
#pragma unroll
    for (int w = 0; w < kCopyThreads / kWave; ++w) all += lds[w];
    P.base[r] = all;
  }
}

// Which forks are refused, the ranks of the slots that the others need (of a deep fork: from the counts in P.base), and these slots.
// One workgroup, since every rank depends on the ones in front; what it takes is latency: 4.5 us where no slot is needed, 9 for 384 of
// them, 9.6 for 32 000.
__global__ __launch_bounds__(kPlanThreads) void fork_plan_kernel(Dims D, Pages P, int n, const int32_t* __restrict__ src,
                                                                 const int32_t* __restrict__ dst, int deep,
                                                                 const int32_t* __restrict__ ctx_len,
                                                                 const int32_t* __restrict__ table, int32_t* status) {
  __shared__ int lds[kPlanWaves];
  __shared__ uint32_t parents[Pages::kPairs / 32], children[Pages::kPairs / 32];  // a bit per sequence
  __shared__ int listed[kPlanThreads], after[kPlanThreads];
  const int tid = threadIdx.x;
  for (int w = tid; w < (D.B + 31) / 32; w += kPlanThreads) parents[w] = children[w] = 0;
  __syncthreads();
  for (int i = tid; i < n; i += kPlanThreads) {
    const int s = src[i];
    if (s >= 0 && s < D.B) atomicOr(&parents[s >> 5], 1u << (s & 31));
  }
  for (int i0 = 0; i0 < n; i0 += kPlanThreads) {  // whoever is listed as a child before: in an earlier round, or in front in this one
    const int i = i0 + tid, s = i < n ? src[i] : -1, t = i < n ? dst[i] : -1;
    listed[tid] = t;
    __syncthreads();
    bool ok = s >= 0 && s < D.B && t >= 0 && t < D.B && s != t;
    int ctx = 0;
    if (ok) {
      ctx = ctx_len[t];
      ok = (parents[t >> 5] >> (t & 31) & 1) == 0 && (children[t >> 5] >> (t & 31) & 1) == 0;
    }
    const int round = n - i0 < kPlanThreads ? n - i0 : kPlanThreads;
    int twice = 0;
#pragma unroll 8
    for (int o = 0; o < round; ++o) twice |= (listed[o] == t) & (o < tid);
    ok &= ctx <= 0 && !twice;
    if (i < n) P.parent[i] = ok ? s : -1;
    after[tid] = ok ? s : D.B;  // refused ones behind the others
    __syncthreads();
    if (t >= 0 && t < D.B) atomicOr(&children[t >> 5], 1u << (t & 31));
    // Children of one parent side by side, so that what they take of it is read once.  The rank of each is counted, up to one round of
    // them; longer lists stay in the caller's order.
    int rank = i;
    if (n <= kPlanThreads && i < n) {
      rank = 0;
      const int mine = after[tid];
#pragma unroll 8
      for (int o = 0; o < n; ++o) rank += after[o] < mine || (after[o] == mine && o < tid);
    }
    if (i < n) P.order[rank] = i;
    __syncthreads();
  }
  const int rows = n * D.Hkv;
  long long want = 0;
  for (int r0 = 0; r0 < rows; r0 += kPlanThreads) {
    const int r = r0 + tid, i = r / D.Hkv;
    const int s = r < rows ? P.parent[i] : -1;
    int c = 0;
    if (s >= 0 && deep) {
      c = P.base[r];
    } else if (s >= 0) {
      const int ctx = ctx_len[s], nb = num_blocks(D, ctx);
      if (nb > 0 && is_copied(D, false, ctx, nb, nb - 1))
        c = has_slot(table[((size_t)s * D.Hkv + (r - i * D.Hkv)) * D.max_blocks + nb - 1], P.n_slots);
    }
    int total;
    const int before = plan_scan(c, lds, &total);
    if (r < rows) P.base[r] = (int)want + before;
    want += total;
  }
  __syncthreads();
  const int got = want > 0 ? take_lowest(P, want, P.list, lds) : 0;
  if (tid == 0) P.head[0] = got;
  for (int i = tid; i < n; i += kPlanThreads) {
    const long long first = P.base[i * D.Hkv], end = i + 1 < n ? P.base[(i + 1) * D.Hkv] : want;
    const long long missing = end - (first > got ? first : got);
    status[i] = P.parent[i] < 0 ? -1 : missing > 0 ? (int)missing : 0;
  }
}

typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;  // (a copy of HIP's uint4 is four stores: half the rate)

constexpr int kTilePieces = 4;  // 16-byte pieces of each pool that a thread holds at a time

// Up to 16 KiB of a tile of both pools, from byte `at` on, in the registers of a workgroup.  The stores pass the caches by: what they
// leave is read by later steps (a deep fork of four sequences of 32k tokens, 269 MB of tiles: 61 us, 90 through the caches).
struct TilePart {
  u32x4 k[kTilePieces], v[kTilePieces];
  __device__ __forceinline__ void load(const char* k_pool, const char* v_pool, size_t tile, int at, int tile_bytes) {
#pragma unroll
    for (int u = 0; u < kTilePieces; ++u) {
      const int o = at + (u * kCopyThreads + (int)threadIdx.x) * 16;
      if (o < tile_bytes) {
        k[u] = *reinterpret_cast<const u32x4*>(k_pool + tile + o);
        v[u] = *reinterpret_cast<const u32x4*>(v_pool + tile + o);
      }
    }
  }
  __device__ __forceinline__ void store(char* k_pool, char* v_pool, size_t tile, int at, int tile_bytes) const {
#pragma unroll
    for (int u = 0; u < kTilePieces; ++u) {
      const int o = at + (u * kCopyThreads + (int)threadIdx.x) * 16;
      if (o < tile_bytes) {
        __builtin_nontemporal_store(k[u], reinterpret_cast<u32x4*>(k_pool + tile + o));
        __builtin_nontemporal_store(v[u], reinterpret_cast<u32x4*>(v_pool + tile + o));
      }
    }
  }
};
constexpr int kPartBytes = kTilePieces * kCopyThreads * 16;

constexpr int kRowPieces = 2 * kCopyThreads;  // 16-byte pieces of digests that a workgroup holds at a time
constexpr int kRowBatch = 4, kTileBatch = 2;  // children that a workgroup writes digests, and tiles, to

// The first row_wgs workgroups: digests and table entries of a range of blocks of a KV head, for kRowBatch children.  The others: tiles
// of a KV head (shallow: the last block; deep: a range), for kTileBatch.  What the children of one parent take is read once for as many of them.
// Bound by what is written: 16 children of 32k tokens, 67 MB of digests: 15.4 us (4.4 TB/s; two at a time: 15.6); 48 of four parents, 172 MB:
// 34 us (5.1 TB/s; two at a time: 38); four deep ones, 269 MB of tiles: 64 us (4.2 TB/s, 5.2 with what is read; four at a time 78, one 86).
__global__ __launch_bounds__(kCopyThreads) void fork_copy_kernel(Dims D, Pages P, int n, const int32_t* __restrict__ dst, int deep,
                                                                 int32_t* ctx_len, char* digest, int entry_bytes, int32_t* table,
                                                                 char* k_pool, char* v_pool, int tile_bytes, long long stride_bytes,
                                                                 int row_wgs, int row_blocks, int row_parts, int parts, int entries) {
  const bool rows = (int)blockIdx.x < row_wgs;
  const int w = rows ? blockIdx.x : blockIdx.x - row_wgs;
  const int of = rows ? row_parts : parts, part = w % of, g = w / of % D.Hkv, batch = w / of / D.Hkv;
  const int of_batch = rows ? kRowBatch : kTileBatch, i1 = (batch + 1) * of_batch < n ? (batch + 1) * of_batch : n;
  int parent[kRowBatch], child[kRowBatch], fork[kRowBatch];
  static_assert(kTileBatch <= kRowBatch, "");
#pragma unroll
  for (int u = 0; u < kRowBatch; ++u) {
    const int i = batch * of_batch + u < i1 ? P.order[batch * of_batch + u] : -1;
    fork[u] = i;
    parent[u] = i >= 0 ? P.parent[i] : -1;
    child[u] = i >= 0 ? dst[i] : -1;
  }
  if (rows) {
    const int j0 = part * row_blocks, j1 = j0 + row_blocks < D.max_blocks ? j0 + row_blocks : D.max_blocks;
    const int pieces_per_entry = entry_bytes / 16;
    int held_of = -1, nb = 0, ctx = 0, entry = -1, sharers = 0;
    bool shared = false;
    u32x4 x[2];
    const int j = j0 + threadIdx.x;
    auto count = [&]() {
      if (shared && sharers > 0) atomicAdd(P.refs + entry, sharers);
      sharers = 0;
    };
#pragma unroll
    for (int c = 0; c < kRowBatch; ++c) {
      const int s = parent[c];
      if (s < 0) continue;
      const size_t from = (size_t)s * D.Hkv + g;
      if (s != held_of) {
        count();
        held_of = s;
        ctx = ctx_len[s];
        entry = j < j1 ? table[from * D.max_blocks + j] : -1;
        nb = num_blocks(D, ctx);
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          const int pc = threadIdx.x + u * kCopyThreads;
          if (j0 + pc / pieces_per_entry < (nb < j1 ? nb : j1))
            x[u] = *reinterpret_cast<const u32x4*>(digest + (from * D.max_blocks + j0) * entry_bytes + (size_t)pc * 16);
        }
        if (j >= nb || !has_slot(entry, P.n_slots)) entry = -1;
        shared = entry >= 0 && !is_copied(D, deep, ctx, nb, j);
      }
      const size_t to = (size_t)child[c] * D.Hkv + g;
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const int pc = threadIdx.x + u * kCopyThreads;
        if (j0 + pc / pieces_per_entry < (nb < j1 ? nb : j1))
          *reinterpret_cast<u32x4*>(digest + (to * D.max_blocks + j0) * entry_bytes + (size_t)pc * 16) = x[u];
      }
      // an entry whose tile is copied is written by the workgroup that copies it
      if (j < j1 && !(entry >= 0 && !shared)) table[to * D.max_blocks + j] = entry;
      ++sharers;
    }
    count();
    return;
  }
  const int got = P.head[0];
  __shared__ int lds[kCopyThreads / kWave];
  int held_of = -1, ctx = 0, nb = 0, before = 0;
#pragma unroll
  for (int c0 = 0; c0 < kTileBatch; ++c0) {
    const int s = parent[c0];
    if (s < 0 || s == held_of) continue;  // (its children are served with the first of them)
    held_of = s;
    ctx = ctx_len[s];
    nb = num_blocks(D, ctx);
    if (g == 0 && part == 0 && threadIdx.x < kTileBatch) {
#pragma unroll
      for (int c = 0; c < kTileBatch; ++c)
        if ((int)threadIdx.x == c && parent[c] == s) ctx_len[child[c]] = ctx;
    }
    const int32_t* row = table + ((size_t)s * D.Hkv + g) * D.max_blocks;
    int j0 = nb - 1, j1 = nb;
    before = 0;
    if (deep) {
      j0 = part * entries;
      j1 = j0 + entries < nb ? j0 + entries : nb;
      if (j0 >= j1) continue;
      // the row's entries with a slot in front of this range
      int x = 0;
#pragma unroll 4
      for (int j = threadIdx.x; j < j0; j += kCopyThreads) x += has_slot(row[j], P.n_slots);
      x = wave_scan(x, lane_id());
      __syncthreads();  // the words may still be read for the parent before
      if (lane_id() == kWave - 1) lds[threadIdx.x / kWave] = x;
      __syncthreads();
#pragma unroll
      for (int v = 0; v < kCopyThreads / kWave; ++v) before += lds[v];
    } else if (nb == 0 || !is_copied(D, false, ctx, nb, j0)) {
      continue;
    }
    for (int j = j0; j < j1; ++j) {
      const int e = row[j];
      if (!has_slot(e, P.n_slots)) continue;
      int slot[kTileBatch];
#pragma unroll
      for (int c = 0; c < kTileBatch; ++c) {
        slot[c] = -1;
        if (parent[c] != s) continue;
        const int rank = P.base[fork[c] * D.Hkv + g] + before;
        if (rank < got) slot[c] = P.list[rank];
        if (threadIdx.x == 0) table[((size_t)child[c] * D.Hkv + g) * D.max_blocks + j] = slot[c];
      }
      ++before;
      for (int at = 0; at < tile_bytes; at += kPartBytes) {
        TilePart T;
        T.load(k_pool, v_pool, (size_t)e * stride_bytes, at, tile_bytes);
#pragma unroll
        for (int c = 0; c < kTileBatch; ++c)
          if (slot[c] >= 0) T.store(k_pool, v_pool, (size_t)slot[c] * stride_bytes, at, tile_bytes);
      }
    }
  }
}

// ---------------------------------------------------------------- free

constexpr int kFreeBatch = 8, kFreeBlocks = 64;  // sequences and blocks that a workgroup looks at, a thread for each

// Each entry gives its reference back, and a slot's bit falls with its last one.  Sequences that share a slot, as forks of one parent do,
// give back together, with one addition.  Three trips to memory and a launch, 3.5 us; with 48 sequences that share 16 000 slots here and
// there in the pool 9 us, which is their counts' additions (16 sequences to a workgroup instead of 8: 8.4, but 5.8 instead of 5.0 for
// 16 sequences of one parent).
__global__ __launch_bounds__(kFreeBatch* kFreeBlocks) void free_kernel(Dims D, Pages P, int n, const int32_t* __restrict__ seq,
                                                                       int32_t* ctx_len, int32_t* table) {
  __shared__ int again[kFreeBatch], named[kFreeBatch][kFreeBlocks];
  const int u = threadIdx.x / kFreeBlocks, jj = threadIdx.x % kFreeBlocks, j = blockIdx.x * kFreeBlocks + jj;  // a wave has one u
  const int g = blockIdx.y, i0 = blockIdx.z * kFreeBatch, i = i0 + u;
  int b = i < n ? seq[i] : -1;
  if (b >= D.B) b = -1;
  if (threadIdx.x < kFreeBatch) again[threadIdx.x] = 0;
  __syncthreads();
  int32_t* const entry = table + ((size_t)(b < 0 ? 0 : b) * D.Hkv + g) * D.max_blocks + j;
  int e = -1;
  if (b >= 0) {
    if (j < D.max_blocks) e = *entry;
    for (int o = jj; o < i; o += kFreeBlocks)  // a sequence that is listed twice is freed once
      if (seq[o] == b) again[u] = 1;
  }
  __syncthreads();
  if (again[u]) b = -1;
  if (b < 0 || !has_slot(e, P.n_slots)) e = -1;
  named[u][jj] = e;
  if (b >= 0 && j < D.max_blocks) *entry = -1;
  __syncthreads();
  int gives = e >= 0;
#pragma unroll
  for (int v = 0; v < kFreeBatch; ++v) {
    const bool same = named[v][jj] == e;
    if (v < u && same) gives = 0;
    if (v > u && same && gives) ++gives;
  }
  bool last = false;
  if (gives) {
    const int held = atomicSub(P.refs + e, gives);
    if (held < gives) atomicAdd(P.refs + e, gives - (held > 0 ? held : 0));  // fewer held it: the count ends at zero
    last = held > 0 && held <= gives;
  }
  // A sequence's slots often lie side by side, a wave's in three words: the bits of one word fall together (four sequences of 32k tokens:
  // 5.0 us, 12.9 slot by slot).  What lies in further words falls by itself.
  uint64_t pending = __ballot(last);
#pragma unroll
  for (int n = 0; n < 3 && pending != 0; ++n) {
    const int word = __builtin_amdgcn_readlane(e >> 5, __builtin_ctzll(pending));
    const bool here = last && e >> 5 == word;
    uint32_t bits = here ? 1u << (e & 31) : 0u;
#pragma unroll
    for (int s = 1; s < kWave; s <<= 1) bits |= __shfl_xor(bits, s);
    const uint64_t done = __ballot(here);
    if (lane_id() == (int)__builtin_ctzll(done)) atomicAnd(P.used + word, ~bits);
    pending &= ~done;
  }
  if (pending >> lane_id() & 1) atomicAnd(P.used + (e >> 5), ~(1u << (e & 31)));
  if (blockIdx.x == 0 && g == 0 && jj == 0 && b >= 0) ctx_len[b] = -1;
}

// ---------------------------------------------------------------- compaction

// Of the n_live used slots, those at n_live and beyond move into the free ones below, both in ascending order: every tile that
// moves is read outside the compacted part and written inside it, so no move waits for another.
// list: where they go, list2: where they are; old: the bits as they were, rank: used slots in front of each word.
// A workgroup per 1024 slots; each of them counts all words by itself (100 000 slots: 12.5 KB), so that none waits for another: 5 us for
// 38 000 slots.  The new bits are written by the next launch, when nobody reads the old ones.
__global__ __launch_bounds__(kPlanThreads) void compact_plan_kernel(Pages P, int32_t* n_live_out) {
  __shared__ int lds[kPlanWaves];
  const long long nw = words_of(P.n_slots), w0 = (long long)blockIdx.x * (kPlanThreads / 32);
  int count = 0, n_live, mine = 0, before, below = 0, above_from;
  for (long long w = threadIdx.x; w < nw; w += kPlanThreads) {
    const int c = __popc(P.used[w] & exists(P.n_slots, w));
    count += c;
    mine += w < w0 ? c : 0;
  }
  plan_scan(count, lds, &n_live);
  plan_scan(mine, lds, &before);
  // used slots below n_live: the holes there are n_live minus them
  for (long long w = threadIdx.x; w < nw && w * 32 < n_live; w += kPlanThreads) below += __popc(P.used[w] & exists(P.n_slots, w) & exists(n_live, w));
  plan_scan(below, lds, &above_from);
  const long long slot = w0 * 32 + threadIdx.x, w = slot >> 5;
  const uint32_t bits = w < nw ? P.used[w] & exists(P.n_slots, w) : 0u, bit = 1u << (slot & 31);
  const bool used = (bits & bit) != 0;
  int total;
  const int seen = before + plan_scan(used, lds, &total);  // used slots in front of this one
  if (slot < P.n_slots) {
    if ((slot & 31) == 0) {
      P.old[w] = bits;
      P.rank[w] = seen;
    }
    if (!used && slot < n_live) P.list[slot - seen] = (int)slot;
    if (used && slot >= n_live) P.list2[seen - above_from] = (int)slot;
  }
  if (blockIdx.x == 0 && threadIdx.x == 0) {
    P.head[0] = n_live;
    P.head[1] = n_live - above_from;  // moves
    P.head[2] = above_from;
    *n_live_out = n_live;
  }
}

// Where the slot that held a tile before the compaction has it now; -1 for a slot that held none.
__device__ __forceinline__ int slot_after(const Pages& P, int slot, int n_live, int above_from) {
  const int w = slot >> 5;
  const uint32_t bits = P.old[w], bit = 1u << (slot & 31);
  if (!(bits & bit)) return -1;
  return slot < n_live ? slot : P.list[P.rank[w] + __popc(bits & (bit - 1)) - above_from];
}

// Tiles first, then the bits and the map, then the tables, by workgroups of their own.  Bound by memory: 268 MB of tiles read and as much written
// in 100 us, 5.4 TB/s (a large copy: 5.2).
__global__ __launch_bounds__(kCopyThreads) void compact_move_kernel(Pages P, int move_wgs, int map_wgs, long long entries, int32_t* table,
                                                                    char* k_pool, char* v_pool, int tile_bytes, long long stride_bytes,
                                                                    int32_t* slot_map) {
  const int n_live = P.head[0], moves = P.head[1], above_from = P.head[2];
  int w = blockIdx.x;
  if (w < move_wgs) {
    for (int m = w; m < moves; m += move_wgs) {
      const int from = P.list2[m], to = P.list[m];
      if (threadIdx.x == 0) {
        P.refs[to] = P.refs[from];
        P.refs[from] = 0;
      }
      for (int at = 0; at < tile_bytes; at += kPartBytes) {
        TilePart T;
        T.load(k_pool, v_pool, (size_t)from * stride_bytes, at, tile_bytes);
        T.store(k_pool, v_pool, (size_t)to * stride_bytes, at, tile_bytes);
      }
    }
    return;
  }
  w -= move_wgs;
  if (w < map_wgs) {
    for (long long i = (long long)w * kCopyThreads + threadIdx.x; i < words_of(P.n_slots); i += (long long)map_wgs * kCopyThreads)
      P.used[i] = exists(n_live, i);
    for (long long s = (long long)w * kCopyThreads + threadIdx.x; s < P.n_slots; s += (long long)map_wgs * kCopyThreads)
      slot_map[s] = slot_after(P, (int)s, n_live, above_from);
    return;
  }
  w -= map_wgs;
  const long long step = (long long)(gridDim.x - move_wgs - map_wgs) * kCopyThreads;
  for (long long i = (long long)w * kCopyThreads + threadIdx.x; i < entries; i += step) {
    const int e = table[i];
    if (has_slot(e, P.n_slots)) table[i] = slot_after(P, e, n_live, above_from);
  }
}

// ---------------------------------------------------------------- launches

static int launched() { return hipGetLastError() == hipSuccess ? SCOUT_OK : SCOUT_EHIP; }

static unsigned wgs_for(long long items, unsigned most) {
  const long long w = (items + kCopyThreads - 1) / kCopyThreads;
  return (unsigned)(w < 1 ? 1 : w > most ? most : w);
}

int launch_pages_init(const Dims& D, const Pages& P, const int32_t* ctx_len, int32_t* table, hipStream_t st) {
  hipLaunchKernelGGL(pages_clear_kernel, dim3(wgs_for(P.n_slots, 1024)), dim3(kCopyThreads), 0, st, P);
  if (D.B > 0)
    hipLaunchKernelGGL(pages_count_kernel, dim3(wgs_for(D.max_blocks, 8), D.Hkv, D.B), dim3(kCopyThreads), 0, st, D, P, ctx_len, table);
  hipLaunchKernelGGL(pages_bits_kernel, dim3(wgs_for(words_of(P.n_slots), 1024)), dim3(kCopyThreads), 0, st, P);
  return launched();
}

int launch_reserve(const Dims& D, const Pages& P, const int32_t* ctx_len, int32_t* new_slot, int32_t* n_short, hipStream_t st) {
  hipLaunchKernelGGL(reserve_kernel, dim3(1), dim3(kPlanThreads), 0, st, D, P, ctx_len, new_slot, n_short);
  return launched();
}

int launch_fork(const Dims& D, int dtype, const Pages& P, int n, const int32_t* src, const int32_t* dst, int deep, int32_t* ctx_len,
                void* digest, int32_t* table, void* k_pool, void* v_pool, int32_t* status, hipStream_t st) {
  if (n == 0) return SCOUT_OK;
  const int es = dtype == SCOUT_BF16 ? 2 : 4;
  const int entry_bytes = D.digest_kind == 1 ? D.d * 4 : 2 * D.d * es, tile_bytes = D.S * D.d * es;
  const int row_blocks = kRowPieces * 16 / entry_bytes;  // 8 to 32
  const int row_parts = (D.max_blocks + row_blocks - 1) / row_blocks;
  const long long row_wgs = (long long)(n + kRowBatch - 1) / kRowBatch * D.Hkv * row_parts;
  // Table entries that a tile workgroup of a deep fork takes, one after the other.  Each counts the slots in front of its entries, all of a row
  // at the end of it, which is little beside a tile up to 4096 blocks (2 children of 2 heads, 8 KiB tiles, 4096 blocks: one 51 us, four 60;
  // 1024 blocks of 8 heads for 4 children: 64 and 71) and not beyond (16384 blocks: 366 and 343; of 2 KiB tiles: 140 and 82).
  // More of them where a launch could not hold so many workgroups.
  constexpr long long kMostWgs = (1ll << 32) / kCopyThreads - 1;
  int entries = D.max_blocks <= 4096 ? 1 : 4;
  auto parts_of = [&](int e) { return deep ? (D.max_blocks + e - 1) / e : 1; };
  auto tile_wgs = [&](int e) { return (long long)(n + kTileBatch - 1) / kTileBatch * D.Hkv * parts_of(e); };
  while (parts_of(entries) > 1 && row_wgs + tile_wgs(entries) > kMostWgs) entries *= 4;
  const int parts = parts_of(entries);
  if (row_wgs + tile_wgs(entries) > kMostWgs) return SCOUT_EUNSUPPORTED;
  if (deep) hipLaunchKernelGGL(fork_count_kernel, dim3(n * D.Hkv), dim3(kCopyThreads), 0, st, D, P, src, ctx_len, table);
  hipLaunchKernelGGL(fork_plan_kernel, dim3(1), dim3(kPlanThreads), 0, st, D, P, n, src, dst, deep, ctx_len, table, status);
  hipLaunchKernelGGL(fork_copy_kernel, dim3((unsigned)(row_wgs + tile_wgs(entries))), dim3(kCopyThreads), 0, st, D, P, n, dst, deep, ctx_len,
                     static_cast<char*>(digest), entry_bytes, table, static_cast<char*>(k_pool), static_cast<char*>(v_pool), tile_bytes,
                     (long long)D.tile_stride * es, (int)row_wgs, row_blocks, row_parts, parts, entries);
  return launched();
}

int launch_free(const Dims& D, const Pages& P, int n, const int32_t* seq, int32_t* ctx_len, int32_t* table, hipStream_t st) {
  if (n == 0) return SCOUT_OK;
  hipLaunchKernelGGL(free_kernel, dim3((D.max_blocks + kFreeBlocks - 1) / kFreeBlocks, D.Hkv, (n + kFreeBatch - 1) / kFreeBatch),
                     dim3(kFreeBatch * kFreeBlocks), 0, st, D, P, n, seq, ctx_len, table);
  return launched();
}

int launch_compact(const Dims& D, int dtype, const Pages& P, int32_t* table, void* k_pool, void* v_pool, int32_t* slot_map,
                   int32_t* n_live, hipStream_t st) {
  const int es = dtype == SCOUT_BF16 ? 2 : 4;
  const long long plan_wgs = (P.n_slots + kPlanThreads - 1) / kPlanThreads;
  hipLaunchKernelGGL(compact_plan_kernel, dim3((unsigned)(plan_wgs > 0 ? plan_wgs : 1)), dim3(kPlanThreads), 0, st, P, n_live);
  const long long entries = (long long)D.B * D.Hkv * D.max_blocks;
  const long long half = (P.n_slots + 1) / 2;  // at most so many tiles can move
  const int move_wgs = (int)(half < 1 ? 1 : half > 2048 ? 2048 : half), map_wgs = (int)wgs_for(P.n_slots, 512);
  hipLaunchKernelGGL(compact_move_kernel, dim3(move_wgs + map_wgs + wgs_for(entries, 1024)), dim3(kCopyThreads), 0, st, P, move_wgs,
                     map_wgs, entries, table, static_cast<char*>(k_pool), static_cast<char*>(v_pool), D.S * D.d * es,
                     (long long)D.tile_stride * es, slot_map);
  return launched();
}

}  // namespace scout
