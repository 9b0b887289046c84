// The pages of a cache that several sequences share: who holds a slot, taking the lowest free ones, forking a sequence,
// freeing one, compacting the pool.
//
// State (struct Pages, one buffer of the caller's): refs[slot], how many block-table entries name the slot, and used, a bit per
// slot that is set while refs > 0.  The bits are what free slots are looked for in: 100 000 slots are 12.5 KB, one trip of one
// workgroup, where the counts themselves are 400 KB.  A slot is taken lowest first and in the order of the takers (child, KV
// head, block), by ranks: the r-th taker gets the r-th clear bit.  So the same state gives the same slots, whatever order
// the workgroups run in; the atomics that count references up and down are integer additions, whose order changes nothing.
//
// A fork and a compaction are two launches: one workgroup that plans (who is refused, which ranks, which slots), and a launch
// that moves bytes (digest rows, table rows, tiles).
#include "pages.h"

namespace scout {

constexpr int kPlanThreads = 1024;
constexpr int kPlanWaves = kPlanThreads / kWave;
constexpr int kCopyThreads = 256;

// Inclusive sum over the lanes of a wave.
__device__ __forceinline__ int wave_scan(int x, int lane) {
#pragma unroll
  for (int s = 1; s < kWave; s <<= 1) {
    const int y = __shfl_up(x, s);
    if (lane >= s) x += y;
  }
  return x;
}

// Exclusive sum over the threads of the planning workgroup, and the total; `lds`: kPlanWaves words.
__device__ __forceinline__ int plan_scan(int x, int* lds, int* total) {
  const int lane = lane_id(), wave = threadIdx.x / kWave;
  const int inc = wave_scan(x, lane);
  __syncthreads();  // the words may still be read from the call before
  if (lane == kWave - 1) lds[wave] = inc;
  __syncthreads();
  int before = 0, all = 0;
#pragma unroll
  for (int w = 0; w < kPlanWaves; ++w) {
    const int t = lds[w];
    before += w < wave ? t : 0;
    all += t;
  }
  *total = all;
  return before + inc - x;
}

// Bits of slots that exist, of word w.
__device__ __forceinline__ uint32_t exists(long long n_slots, long long w) {
  const long long left = n_slots - w * 32;
  return left >= 32 ? 0xffffffffu : left <= 0 ? 0u : (1u << left) - 1u;
}

// The `want` lowest free slots, ascending, to list (as many as there are; the number is returned to every thread).  They
// become used with one reference each.  The whole planning workgroup calls this.
__device__ int take_lowest(const Pages& P, long long want, int32_t* list, int* lds) {
  const long long nw = words_of(P.n_slots);
  long long got = 0;
  for (long long w0 = 0; w0 < nw && got < want; w0 += kPlanThreads) {
    const long long w = w0 + threadIdx.x;
    uint32_t free_bits = 0;
    if (w < nw) free_bits = ~P.used[w] & exists(P.n_slots, w);
    int total;
    long long at = got + plan_scan(__popc(free_bits), lds, &total);
    uint32_t taken = 0;
    while (free_bits != 0 && at < want) {
      const uint32_t bit = free_bits & -free_bits;
      const int slot = (int)(w * 32) + __ffs(bit) - 1;
      list[at++] = slot;
      P.refs[slot] = 1;
      taken |= bit;
      free_bits ^= bit;
    }
    if (taken) P.used[w] |= taken;
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

__global__ __launch_bounds__(kCopyThreads) void pages_count_kernel(Dims D, Pages P, const int32_t* __restrict__ ctx_len,
                                                                   const int32_t* __restrict__ table) {
  const int pair = grid_pair(), nb = num_blocks(D, ctx_len[blockIdx.z]);
  for (int j = blockIdx.x * kCopyThreads + threadIdx.x; j < nb; j += gridDim.x * kCopyThreads) {
    const int e = table[(size_t)pair * D.max_blocks + j];
    if (has_slot(e, P.n_slots)) atomicAdd(P.refs + e, 1);
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

// Which forks are refused, the ranks of the slots that the others need, and these slots.
__global__ __launch_bounds__(kPlanThreads) void fork_plan_kernel(Dims D, Pages P, int n, const int32_t* __restrict__ src,
                                                                 const int32_t* __restrict__ dst, int deep,
                                                                 const int32_t* __restrict__ ctx_len,
                                                                 const int32_t* __restrict__ table, int32_t* status) {
  __shared__ int lds[kPlanWaves];
  const int lane = lane_id(), wave = threadIdx.x / kWave;
  for (int i = threadIdx.x; i < n; i += kPlanThreads) {
    const int s = src[i], t = dst[i];
    bool ok = s >= 0 && s < D.B && t >= 0 && t < D.B && s != t;
    for (int o = 0; o < n; ++o) ok &= src[o] != t && (o >= i || dst[o] != t);
    if (ok) ok = ctx_len[t] <= 0;
    P.parent[i] = ok ? s : -1;
  }
  __syncthreads();
  const int rows = n * D.Hkv;
  if (deep) {  // a wave counts a row
    for (int r = wave; r < rows; r += kPlanWaves) {
      const int i = r / D.Hkv, s = P.parent[i];
      int c = 0;
      if (s >= 0) {
        const int nb = num_blocks(D, ctx_len[s]);
        const int32_t* row = table + ((size_t)s * D.Hkv + (r - i * D.Hkv)) * D.max_blocks;
        for (int j = lane; j < nb; j += kWave) c += has_slot(row[j], P.n_slots);
        c = wave_scan(c, lane);
      }
      if (lane == kWave - 1) P.base[r] = c;
    }
  } else {
    for (int r = threadIdx.x; r < rows; r += kPlanThreads) {
      const int i = r / D.Hkv, s = P.parent[i];
      int c = 0;
      if (s >= 0) {
        const int ctx = ctx_len[s], nb = num_blocks(D, ctx);
        if (nb > 0 && is_copied(D, false, ctx, nb, nb - 1))
          c = has_slot(table[((size_t)s * D.Hkv + (r - i * D.Hkv)) * D.max_blocks + nb - 1], P.n_slots);
      }
      P.base[r] = c;
    }
  }
  __syncthreads();
  long long want = 0;
  for (int r0 = 0; r0 < rows; r0 += kPlanThreads) {
    const int r = r0 + threadIdx.x;
    int total;
    const int before = plan_scan(r < rows ? P.base[r] : 0, lds, &total);
    if (r < rows) P.base[r] = (int)want + before;
    want += total;
  }
  __syncthreads();
  const int got = want > 0 ? take_lowest(P, want, P.list, lds) : 0;
  if (threadIdx.x == 0) P.head[0] = got;
  __syncthreads();
  for (int i = threadIdx.x; i < n; i += kPlanThreads) {
    const long long first = P.base[i * D.Hkv], end = i + 1 < n ? P.base[(i + 1) * D.Hkv] : want;
    const long long missing = end - (first > got ? first : got);
    status[i] = P.parent[i] < 0 ? -1 : missing > 0 ? (int)missing : 0;
  }
}

// Tile `from` to tile `to` in both pools, by `threads` threads of which this is `thread`: four reads of each pool in flight.
__device__ __forceinline__ void copy_tile(char* k_pool, char* v_pool, size_t from, size_t to, int tile_bytes, int thread, int threads) {
  for (int at = thread * 16; at < tile_bytes; at += threads * 64) {
    uint4 k[4], v[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int o = at + u * threads * 16;
      if (o < tile_bytes) {
        k[u] = *reinterpret_cast<const uint4*>(k_pool + from + o);
        v[u] = *reinterpret_cast<const uint4*>(v_pool + from + o);
      }
    }
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int o = at + u * threads * 16;
      if (o < tile_bytes) {
        *reinterpret_cast<uint4*>(k_pool + to + o) = k[u];
        *reinterpret_cast<uint4*>(v_pool + to + o) = v[u];
      }
    }
  }
}

constexpr int kRowPieces = 2 * kCopyThreads;  // 16-byte pieces of digests that a workgroup holds at a time
constexpr int kForkEntries = 8;               // table entries that a tile workgroup of a deep fork takes

// The first row_wgs workgroups: digests and table entries of a range of blocks of a KV head, read once and written to every child
// of that parent in the list's order.  The others: tiles, of one child's KV head (shallow: its last block; deep: a range).
__global__ __launch_bounds__(kCopyThreads) void fork_copy_kernel(Dims D, Pages P, int n, const int32_t* __restrict__ dst, int deep,
                                                                 int32_t* ctx_len, char* digest, int entry_bytes, int32_t* table,
                                                                 char* k_pool, char* v_pool, int tile_bytes, int stride_bytes,
                                                                 int row_wgs, int row_blocks, int tile_wgs_per_pair) {
  if ((int)blockIdx.x < row_wgs) {
    const int g = blockIdx.x % D.Hkv, j0 = blockIdx.x / D.Hkv * row_blocks;
    const int j1 = j0 + row_blocks < D.max_blocks ? j0 + row_blocks : D.max_blocks;
    const int pieces_per_entry = entry_bytes / 16;
    int held_of = -1, nb = 0, ctx = 0, entry = -1, sharers = 0;
    bool shared = false;
    uint4 x[2];
    const int j = j0 + threadIdx.x;
    auto count = [&]() {
      if (shared && sharers > 0) atomicAdd(P.refs + entry, sharers);
      sharers = 0;
    };
    for (int i = 0; i < n; ++i) {
      const int s = P.parent[i];
      if (s < 0) continue;
      const size_t from = (size_t)s * D.Hkv + g;
      if (s != held_of) {
        count();
        held_of = s;
        ctx = ctx_len[s];
        nb = num_blocks(D, ctx);
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          const int pc = threadIdx.x + u * kCopyThreads;
          if (j0 + pc / pieces_per_entry < (nb < j1 ? nb : j1))
            x[u] = *reinterpret_cast<const uint4*>(digest + (from * D.max_blocks + j0) * entry_bytes + (size_t)pc * 16);
        }
        entry = -1;
        if (j < j1 && j < nb) {
          const int e = table[from * D.max_blocks + j];
          if (has_slot(e, P.n_slots)) entry = e;
        }
        shared = entry >= 0 && !is_copied(D, deep, ctx, nb, j);
      }
      const size_t to = (size_t)dst[i] * D.Hkv + g;
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const int pc = threadIdx.x + u * kCopyThreads;
        if (j0 + pc / pieces_per_entry < (nb < j1 ? nb : j1))
          *reinterpret_cast<uint4*>(digest + (to * D.max_blocks + j0) * entry_bytes + (size_t)pc * 16) = x[u];
      }
      // an entry whose tile is copied is written by the workgroup that copies it
      if (j < j1 && !(entry >= 0 && !shared)) table[to * D.max_blocks + j] = entry;
      ++sharers;
    }
    count();
    return;
  }
  const int w = blockIdx.x - row_wgs;
  const int r = w / tile_wgs_per_pair, part = w - r * tile_wgs_per_pair;
  const int i = r / D.Hkv, g = r - i * D.Hkv;
  const int s = P.parent[i];
  if (s < 0) return;
  const int t = dst[i], ctx = ctx_len[s], nb = num_blocks(D, ctx), got = P.head[0];
  if (g == 0 && part == 0 && threadIdx.x == 0) ctx_len[t] = ctx;
  const int32_t* row = table + ((size_t)s * D.Hkv + g) * D.max_blocks;
  int32_t* child = table + ((size_t)t * D.Hkv + g) * D.max_blocks;
  int j0 = nb - 1, j1 = nb, rank = P.base[r];
  if (deep) {
    j0 = part * kForkEntries;
    j1 = j0 + kForkEntries < nb ? j0 + kForkEntries : nb;
    if (j0 >= j1) return;
    // the row's entries with a slot in front of this range
    __shared__ int lds[kCopyThreads / kWave];
    int c = 0;
    for (int j = threadIdx.x; j < j0; j += kCopyThreads) c += has_slot(row[j], P.n_slots);
    c = wave_scan(c, lane_id());
    if (lane_id() == kWave - 1) lds[threadIdx.x / kWave] = c;
    __syncthreads();
#pragma unroll
    for (int v = 0; v < kCopyThreads / kWave; ++v) rank += lds[v];
  } else if (nb == 0 || !is_copied(D, false, ctx, nb, j0)) {
    return;
  }
  for (int j = j0; j < j1; ++j) {
    const int e = row[j];
    if (!has_slot(e, P.n_slots)) continue;
    const int slot = rank < got ? P.list[rank] : -1;
    ++rank;
    if (threadIdx.x == 0) child[j] = slot;
    if (slot >= 0) copy_tile(k_pool, v_pool, (size_t)e * stride_bytes, (size_t)slot * stride_bytes, tile_bytes, threadIdx.x, kCopyThreads);
  }
}

// ---------------------------------------------------------------- free

// A workgroup per listed sequence: each of its entries gives its reference back, and the slot's bit falls with the last one.
__global__ __launch_bounds__(1024) void free_kernel(Dims D, Pages P, int n, const int32_t* __restrict__ seq, int32_t* ctx_len,
                                                    int32_t* table) {
  const int i = blockIdx.x, b = seq[i];
  if (b < 0 || b >= D.B) return;
  int before = 0;  // a sequence that is listed twice is freed once
  for (int o = threadIdx.x; o < i; o += blockDim.x) before |= seq[o] == b;
  const int nb = num_blocks(D, ctx_len[b]);
  if (__syncthreads_or(before)) return;
  if (threadIdx.x == 0) ctx_len[b] = -1;
  int32_t* rows = table + (size_t)b * D.Hkv * D.max_blocks;
  for (int g = 0; g < D.Hkv; ++g, rows += D.max_blocks)
    for (int j = threadIdx.x; j < D.max_blocks; j += blockDim.x) {
      if (j < nb) {
        const int e = rows[j];
        if (has_slot(e, P.n_slots)) {
          const int held = atomicSub(P.refs + e, 1);
          if (held == 1) atomicAnd(P.used + (e >> 5), ~(1u << (e & 31)));
          if (held <= 0) atomicAdd(P.refs + e, 1);  // nobody held it: the count stays
        }
      }
      rows[j] = -1;
    }
}

// ---------------------------------------------------------------- compaction

// Of the n_live used slots, those at n_live and beyond move into the free ones below, both in ascending order: every tile that
// moves is read outside the compacted part and written inside it, so no move waits for another.
// list: where they go, list2: where they are; old: the bits as they were, rank: used slots in front of each word.
__global__ __launch_bounds__(kPlanThreads) void compact_plan_kernel(Pages P, int32_t* n_live_out) {
  __shared__ int lds[kPlanWaves];
  const long long nw = words_of(P.n_slots);
  int count = 0, n_live;
  for (long long w = threadIdx.x; w < nw; w += kPlanThreads) count += __popc(P.used[w] & exists(P.n_slots, w));
  plan_scan(count, lds, &n_live);
  int seen = 0, above_from = 0;  // used slots before the chunk; used slots below n_live (once known)
  // used slots below n_live: the holes there are n_live minus them
  int below = 0;
  for (long long w = threadIdx.x; w < nw; w += kPlanThreads) {
    const uint32_t bits = P.used[w] & exists(P.n_slots, w), in = exists(n_live, w);
    below += __popc(bits & in);
  }
  plan_scan(below, lds, &above_from);
  for (long long w0 = 0; w0 < nw; w0 += kPlanThreads) {
    const long long w = w0 + threadIdx.x;
    uint32_t bits = 0, in = 0;
    if (w < nw) {
      bits = P.used[w] & exists(P.n_slots, w);
      in = exists(n_live, w);
    }
    int total;
    const int before = seen + plan_scan(__popc(bits), lds, &total);
    if (w < nw) {
      P.old[w] = bits;
      P.rank[w] = before;
      P.used[w] = in;
      // slots of this word below n_live in front of it: w * 32, of which `before` are used
      long long at = w * 32 - before;
      for (uint32_t hole = ~bits & in; hole != 0; hole &= hole - 1) P.list[at++] = (int)(w * 32) + __ffs(hole) - 1;
      long long m = (long long)before + __popc(bits & in) - above_from;
      for (uint32_t out = bits & ~in; out != 0; out &= out - 1) P.list2[m++] = (int)(w * 32) + __ffs(out) - 1;
    }
    seen += total;
  }
  if (threadIdx.x == 0) {
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

__global__ __launch_bounds__(kCopyThreads) void compact_move_kernel(Pages P, int move_wgs, int map_wgs, long long entries, int32_t* table,
                                                                    char* k_pool, char* v_pool, int tile_bytes, int stride_bytes,
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
      copy_tile(k_pool, v_pool, (size_t)from * stride_bytes, (size_t)to * stride_bytes, tile_bytes, threadIdx.x, kCopyThreads);
    }
    return;
  }
  w -= move_wgs;
  if (w < map_wgs) {
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

int launch_pages_init(const Dims& D, const Pages& P, const int32_t* ctx_len, const int32_t* table, hipStream_t st) {
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
  hipLaunchKernelGGL(fork_plan_kernel, dim3(1), dim3(kPlanThreads), 0, st, D, P, n, src, dst, deep, ctx_len, table, status);
  const int row_blocks = kRowPieces * 16 / entry_bytes;  // 8 to 32
  const int row_wgs = (D.max_blocks + row_blocks - 1) / row_blocks * D.Hkv;
  const int per_pair = deep ? (D.max_blocks + kForkEntries - 1) / kForkEntries : 1;
  const long long wgs = row_wgs + (long long)n * D.Hkv * per_pair;
  hipLaunchKernelGGL(fork_copy_kernel, dim3((unsigned)wgs), dim3(kCopyThreads), 0, st, D, P, n, dst, deep, ctx_len,
                     static_cast<char*>(digest), entry_bytes, table, static_cast<char*>(k_pool), static_cast<char*>(v_pool), tile_bytes,
                     D.tile_stride * es, row_wgs, row_blocks, per_pair);
  return launched();
}

int launch_free(const Dims& D, const Pages& P, int n, const int32_t* seq, int32_t* ctx_len, int32_t* table, hipStream_t st) {
  if (n == 0) return SCOUT_OK;
  hipLaunchKernelGGL(free_kernel, dim3(n), dim3(1024), 0, st, D, P, n, seq, ctx_len, table);
  return launched();
}

int launch_compact(const Dims& D, int dtype, const Pages& P, int32_t* table, void* k_pool, void* v_pool, int32_t* slot_map,
                   int32_t* n_live, hipStream_t st) {
  const int es = dtype == SCOUT_BF16 ? 2 : 4;
  hipLaunchKernelGGL(compact_plan_kernel, dim3(1), dim3(kPlanThreads), 0, st, P, n_live);
  const long long entries = (long long)D.B * D.Hkv * D.max_blocks;
  const long long half = (P.n_slots + 1) / 2;  // at most so many tiles can move
  const int move_wgs = (int)(half < 1 ? 1 : half > 2048 ? 2048 : half), map_wgs = (int)wgs_for(P.n_slots, 512);
  hipLaunchKernelGGL(compact_move_kernel, dim3(move_wgs + map_wgs + wgs_for(entries, 1024)), dim3(kCopyThreads), 0, st, P, move_wgs,
                     map_wgs, entries, table, static_cast<char*>(k_pool), static_cast<char*>(v_pool), D.S * D.d * es, D.tile_stride * es,
                     slot_map);
  return launched();
}

}  // namespace scout
