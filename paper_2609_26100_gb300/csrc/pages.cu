// Bookkeeping of a paged cache on the device: reserving, freeing, forking and compacting pages.
//
// The state is the caller's page table, pages held per sequence and reference counts.  A page is free
// where its count is 0 and the lowest free page is taken first, so results do not depend on the order in
// which threads run.  Choosing pages is one CTA's work: rounds of 16384 counts become a bitmap in
// shared memory (a ballot per 32), whose set bits are ranked by one scan of the words.  What needs no
// choice (rows, counts, page data) is spread over the GPU in a second launch.
//
// Bounds: the choosing launch is latency (one CTA, one read of the counts up to the last page taken): twelve sequences
// freed and forked again with a tail page in 8 layers each, 9 us in all.  The copies are HBM, each byte read and written
// once: 900 pages of 128 KB moved in each of 2 layers (472 MB) in 81 us, 5.8 TB/s.  A reorder of 64 beams over 32 layers: the choice 10 us
// (parents read, takers and free pages found), rows and copies of 60 tails a layer 20 us; of 8 beams over 8 layers 9 us in all.
#include "ops.cuh"

struct tss_pages {
  int n_seqs, max_pages, n_pages, dev, sms;
  int* status;  // device word: first failure
  int* go;      // device word: the last choosing launch found its pages (1) or left everything as it was (0)
  int* moves;   // device [1 + 2 * n_pages]: their number, then sources, then destinations (or chosen pages)
  int* map;     // device [n_pages]: new id of every page
  int* plan;    // device [4][64]: a reorder's parents, first copies, pages held before; [3][0] the most held
};

namespace tss {
namespace {

constexpr int kPlanThreads = 512;
constexpr int kMaxPoolPages = 1 << 20;
constexpr int kMaxCalls = 64;     // entries of one call
constexpr int kMaxPoolLayers = 128;

struct PoolTables {
  int *table, *held, *refs;
  int n_seqs, max_pages, n_pages;
  int* status;
};
struct SeqList {
  int n;
  int a[kMaxCalls], b[kMaxCalls], c[kMaxCalls], d[kMaxCalls];
};
struct Layers {
  int n;
  size_t page_bytes;
  uint8_t* base[kMaxPoolLayers];
};

// Exclusive prefix sum of v over the CTA; *total the sum.  scratch: kPlanThreads / 32 + 1 words.
__device__ int block_scan(int v, int* scratch, int* total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int x = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int y = __shfl_up_sync(0xffffffffu, x, o);
    if (lane >= o) x += y;
  }
  __syncthreads();
  if (lane == 31) scratch[warp] = x;
  __syncthreads();
  if (warp == 0) {
    int s = lane < kPlanThreads / 32 ? scratch[lane] : 0;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int y = __shfl_up_sync(0xffffffffu, s, o);
      if (lane >= o) s += y;
    }
    if (lane < kPlanThreads / 32) scratch[lane] = s;
  }
  __syncthreads();
  *total = scratch[kPlanThreads / 32 - 1];
  return x - v + (warp ? scratch[warp - 1] : 0);
}

// The `need` lowest free pages, ascending, to ids; returns how many there are (at most need).
constexpr int kRoundWords = kPlanThreads;  // bitmap words of a round: 16384 pages
__device__ int lowest_free(const int* refs, int n_pages, int need, int* ids, uint32_t* bits, int* scratch) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int found = 0;
  for (int p0 = 0; p0 < n_pages && found < need; p0 += kRoundWords * 32) {
    // warp w makes words w, w + 16, ...: coalesced loads, eight in flight
#pragma unroll
    for (int k0 = 0; k0 < 32; k0 += 8) {
      int v[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const int page = p0 + ((k0 + k) * (kPlanThreads / 32) + warp) * 32 + lane;
        v[k] = page < n_pages ? refs[page] : 1;
      }
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const uint32_t w = __ballot_sync(0xffffffffu, v[k] == 0);
        if (lane == 0) bits[(k0 + k) * (kPlanThreads / 32) + warp] = w;
      }
    }
    __syncthreads();
    uint32_t w = bits[threadIdx.x];
    int total, at = found + block_scan(__popc(w), scratch, &total);
    while (w && at < need) {
      ids[at++] = p0 + threadIdx.x * 32 + __ffs(w) - 1;
      w &= w - 1;
    }
    found += total;
    __syncthreads();
  }
  return min(found, need);
}

// reserve: sequence a[i] grows to b[i] pages
__global__ void __launch_bounds__(kPlanThreads) reserve_kernel(const __grid_constant__ SeqList list, PoolTables t, int* ids) {
  __shared__ uint32_t bits[kRoundWords];
  __shared__ int scratch[kPlanThreads / 32], off[kMaxCalls + 1], from[kMaxCalls];
  const int tid = threadIdx.x;
  griddep_wait();
  griddep_launch();
  if (tid < list.n) {
    const int have = t.held[list.a[tid]];
    from[tid] = have;
    off[tid + 1] = have >= 0 ? max(0, list.b[tid] - have) : -1;  // (a count below zero is no count)
  }
  __syncthreads();
  if (tid == 0) {
    off[0] = 0;
    bool bad = false;
    for (int i = 0; i < list.n; ++i) {
      bad |= off[i + 1] < 0;
      off[i + 1] = min(off[i] + max(off[i + 1], 0), t.n_pages + 1);
    }
    if (bad) {
      report(t.status, kStatusCheck);
      off[list.n] = -1;
    }
  }
  __syncthreads();
  const int need = off[list.n];
  if (need <= 0) return;
  if (need > t.n_pages || lowest_free(t.refs, t.n_pages, need, ids, bits, scratch) < need) {
    if (tid == 0) report(t.status, TSS_ERR_KV_CAPACITY);
    return;
  }
  __syncthreads();
  for (int x = tid; x < need; x += kPlanThreads) {
    int i = 0;
    while (off[i + 1] <= x) ++i;
    const int page = ids[x];
    t.table[static_cast<long long>(list.a[i]) * t.max_pages + from[i] + x - off[i]] = page;
    t.refs[page] = 1;
  }
  if (tid < list.n) t.held[list.a[tid]] = max(from[tid], list.b[tid]);
}

// free: a CTA for each sequence a[i], which keeps b[i] pages
__global__ void __launch_bounds__(256) free_kernel(const __grid_constant__ SeqList list, PoolTables t) {
  griddep_wait();
  griddep_launch();
  const int seq = list.a[blockIdx.x], keep = list.b[blockIdx.x], held = t.held[seq];
  __syncthreads();
  if (held < 0 || held > t.max_pages) {
    if (threadIdx.x == 0) report(t.status, kStatusCheck);
    return;
  }
  int* row = t.table + static_cast<long long>(seq) * t.max_pages;
  for (int i = keep + threadIdx.x; i < held; i += blockDim.x) {
    const int page = row[i];
    row[i] = -1;
    if (page < 0 || page >= t.n_pages || atomicSub(&t.refs[page], 1) <= 0) {
      if (page >= 0 && page < t.n_pages) atomicAdd(&t.refs[page], 1);
      report(t.status, kStatusCheck);
    }
  }
  if (threadIdx.x == 0 && held > keep) t.held[seq] = keep;
}

// fork, first part: pages for the copies of all entries (list: src, dst, shared, total), or nothing at all
__global__ void __launch_bounds__(kPlanThreads) fork_choose_kernel(const __grid_constant__ SeqList list, PoolTables t, int need,
                                                                   int* ids, int* go) {
  __shared__ uint32_t bits[kRoundWords];
  __shared__ int scratch[kPlanThreads / 32], bad;
  const int tid = threadIdx.x;
  griddep_wait();
  griddep_launch();
  if (tid == 0) bad = 0;
  __syncthreads();
  if (tid < list.n) {
    const int have = t.held[list.a[tid]];
    if (have < list.d[tid] || have > t.max_pages || t.held[list.b[tid]] != 0) bad = 1;
  }
  // every page that will be shared or copied has to be one of the pool that somebody holds
  for (int i = tid >> 5; i < list.n; i += kPlanThreads / 32) {
    if (t.held[list.a[i]] < list.d[i]) continue;
    const int* row = t.table + static_cast<long long>(list.a[i]) * t.max_pages;
    for (int x = tid & 31; x < list.d[i]; x += 32) {
      const int page = row[x];
      if (page < 0 || page >= t.n_pages || t.refs[page] < 1) bad = 1;
    }
  }
  __syncthreads();
  if (bad) {
    if (tid == 0) {
      report(t.status, kStatusCheck);
      *go = 0;
    }
    return;
  }
  const int got = need > 0 ? lowest_free(t.refs, t.n_pages, need, ids, bits, scratch) : 0;
  if (tid == 0) {
    if (got < need) report(t.status, TSS_ERR_KV_CAPACITY);
    *go = got >= need;
  }
}

// A 16 KiB piece (or the rest) of one page of one layer.
constexpr int kPiece = 16384, kCopyThreads = 256;
__device__ __forceinline__ void copy_piece(uint8_t* base, size_t page_bytes, int src, int dst, int piece) {
  const size_t from = static_cast<size_t>(piece) * kPiece;
  const int n = static_cast<int>(min(page_bytes - from, static_cast<size_t>(kPiece)) / 16);
  const uint4* s = reinterpret_cast<const uint4*>(base + static_cast<size_t>(src) * page_bytes + from);
  uint4* d = reinterpret_cast<uint4*>(base + static_cast<size_t>(dst) * page_bytes + from);
  uint4 v[kPiece / 16 / kCopyThreads];
#pragma unroll
  for (int k = 0; k < kPiece / 16 / kCopyThreads; ++k) {
    const int i = k * kCopyThreads + threadIdx.x;
    if (i < n) v[k] = __ldcs(s + i);
  }
#pragma unroll
  for (int k = 0; k < kPiece / 16 / kCopyThreads; ++k) {
    const int i = k * kCopyThreads + threadIdx.x;
    if (i < n) d[i] = v[k];
  }
}

// fork, second part: CTAs [0, n) write an entry's row and counts, the others copy pages
__global__ void __launch_bounds__(kCopyThreads) fork_kernel(const __grid_constant__ SeqList list, PoolTables t, const __grid_constant__ Layers ly,
                                                            const int* ids, const int* go) {
  griddep_wait();
  griddep_launch();
  if (*go == 0) return;
  const int cta = blockIdx.x;
  if (cta < list.n) {
    int first = 0;  // entry's first new page
    for (int i = 0; i < cta; ++i) first += list.d[i] - list.c[i];
    const int* from = t.table + static_cast<long long>(list.a[cta]) * t.max_pages;
    int* to = t.table + static_cast<long long>(list.b[cta]) * t.max_pages;
    for (int x = threadIdx.x; x < list.d[cta]; x += kCopyThreads) {
      if (x < list.c[cta]) {
        to[x] = from[x];
        atomicAdd(&t.refs[from[x]], 1);
      } else {
        const int page = ids[first + x - list.c[cta]];
        to[x] = page;
        t.refs[page] = 1;
      }
    }
    if (threadIdx.x == 0) t.held[list.b[cta]] = list.d[cta];
    return;
  }
  const int pieces = static_cast<int>((ly.page_bytes + kPiece - 1) / kPiece);
  // unit: (new page, layer, piece), pieces fastest
  int before = 0, entry = 0;
  int copies = 0;
  for (int i = 0; i < list.n; ++i) copies += list.d[i] - list.c[i];
  const long long units = static_cast<long long>(copies) * ly.n * pieces;
  for (long long u = cta - list.n; u < units; u += gridDim.x - list.n) {
    const int c = static_cast<int>(u / (static_cast<long long>(ly.n) * pieces));
    const int rest = static_cast<int>(u - static_cast<long long>(c) * ly.n * pieces);
    while (c >= before + list.d[entry] - list.c[entry]) {
      before += list.d[entry] - list.c[entry];
      ++entry;
    }
    const int src = t.table[static_cast<long long>(list.a[entry]) * t.max_pages + list.c[entry] + c - before];
    copy_piece(ly.base[rest / pieces], ly.page_bytes, src, ids[c], rest % pieces);
  }
}

// reorder.  Entry i takes the first d[p] pages of entry p = parent[i] (a: sequences; c: pages of p that its takers share).
// The others are the taker's that goes on in p's own place, or else its first, the keeper; the rest get copies.
//
// First part: what each entry takes, the copies (sources to src, pages that were free before the call to ids), or nothing.
__global__ void __launch_bounds__(kPlanThreads) reorder_choose_kernel(const __grid_constant__ SeqList list, PoolTables t, const int* parents,
                                                                      int* plan, int* src, int* ids, int* n_copies, int* go) {
  __shared__ uint32_t bits[kRoundWords];
  __shared__ int scratch[kPlanThreads / 32], parent[kMaxCalls], keeper[kMaxCalls], off[kMaxCalls + 1], bad, most;  // keeper: -1 for p itself
  const int tid = threadIdx.x;
  griddep_wait();
  griddep_launch();
  if (tid == 0) bad = most = 0;
  if (tid < kMaxCalls) keeper[tid] = kMaxCalls;
  if (tid < list.n) parent[tid] = parents[tid];
  __syncthreads();
  int held = 0;
  if (tid < list.n) {
    held = t.held[list.a[tid]];
    const int p = parent[tid];
    if (held < 0 || held > t.max_pages || p < -1 || p >= list.n) bad = 1;
    if (p >= 0 && p < list.n) {
      atomicMin(&keeper[p], p == tid ? -1 : tid);
      if (t.held[list.a[p]] < list.d[p]) bad = 1;
    }
    atomicMax(&most, held);
  }
  __syncthreads();
  if (!bad && tid < list.n) {
    const int p = parent[tid];
    off[tid + 1] = p < 0 || keeper[p] == (p == tid ? -1 : tid) ? 0 : list.d[p] - list.c[p];
  }
  __syncthreads();
  if (!bad && tid < 32) {  // sums of the entries before, two a lane, up to one more than there are pages
    static_assert(kMaxCalls == 64, "two entries a lane");
    const int cap = t.n_pages + 1, a = 2 * tid < list.n ? min(off[2 * tid + 1], cap) : 0, b = 2 * tid + 1 < list.n ? min(off[2 * tid + 2], cap) : 0;
    int all = min(a + b, cap);
#pragma unroll
    for (int o = 1; o < 32; o *= 2) {
      const int y = __shfl_up_sync(0xffffffffu, all, o);
      if (tid >= o) all = min(all + y, cap);
    }
    int before = __shfl_up_sync(0xffffffffu, all, 1);
    if (tid == 0) before = off[0] = 0;
    off[2 * tid + 1] = min(before + a, cap);
    off[2 * tid + 2] = all;
  }
  __syncthreads();
  const int need = bad ? 0 : off[list.n];
  if (!bad && need <= t.n_pages)  // every page that will be copied has to be one of the pool that somebody holds
    for (int i = tid >> 5; i < list.n; i += kPlanThreads / 32) {
      const int p = parent[i];
      for (int x = tid & 31; x < off[i + 1] - off[i]; x += 32) {
        const int page = t.table[static_cast<long long>(list.a[p]) * t.max_pages + list.c[p] + x];
        if (page < 0 || page >= t.n_pages || t.refs[page] < 1)
          bad = 1;
        else
          src[off[i] + x] = page;
      }
    }
  __syncthreads();
  if (bad) {
    if (tid == 0) {
      report(t.status, kStatusCheck);
      *go = 0;
    }
    return;
  }
  const bool room = need <= t.n_pages && (need == 0 || lowest_free(t.refs, t.n_pages, need, ids, bits, scratch) == need);
  if (tid < list.n) {
    const int p = parent[tid];
    plan[tid] = p;
    plan[kMaxCalls + tid] = off[tid + 1] > off[tid] ? off[tid] : -1;
    plan[2 * kMaxCalls + tid] = held;
  }
  if (tid == 0) {
    if (!room) report(t.status, TSS_ERR_KV_CAPACITY);
    plan[3 * kMaxCalls] = most;
    *n_copies = need;
    *go = room;
  }
}

// Second part: CTAs [0, col_ctas) change 64 columns each of the entries' rows, and the counts of what changes (a column depends
// on no other, so that rows may change places in place); the others copy pages.
constexpr int kReorderCols = 64;
__global__ void __launch_bounds__(kCopyThreads) reorder_kernel(const __grid_constant__ SeqList list, PoolTables t, const __grid_constant__ Layers ly,
                                                               const int* plan, const int* src, const int* ids, const int* n_copies,
                                                               const int* go, int col_ctas) {
  __shared__ int old[kMaxCalls][kReorderCols];
  griddep_wait();
  griddep_launch();
  if (*go == 0) return;
  const int cta = blockIdx.x, tid = threadIdx.x;
  if (cta >= col_ctas) {
    const int pieces = static_cast<int>((ly.page_bytes + kPiece - 1) / kPiece);
    const long long units = static_cast<long long>(*n_copies) * ly.n * pieces;
    for (long long u = cta - col_ctas; u < units; u += gridDim.x - col_ctas) {
      const int c = static_cast<int>(u / (static_cast<long long>(ly.n) * pieces));
      const int rest = static_cast<int>(u - static_cast<long long>(c) * ly.n * pieces);
      copy_piece(ly.base[rest / pieces], ly.page_bytes, src[c], ids[c], rest % pieces);
    }
    return;
  }
  if (cta == 0 && tid < list.n) t.held[list.a[tid]] = plan[tid] < 0 ? 0 : list.d[plan[tid]];
  constexpr int kStep = kCopyThreads / kReorderCols;
  const int c = tid % kReorderCols, first = tid / kReorderCols;
  const auto valid = [&](int page) { return page >= 0 && page < t.n_pages; };
  for (long long x0 = static_cast<long long>(cta) * kReorderCols; x0 < plan[3 * kMaxCalls]; x0 += static_cast<long long>(col_ctas) * kReorderCols) {
    const int x = static_cast<int>(x0) + c;
    for (int i = first; i < list.n; i += kStep)
      old[i][c] = x < plan[2 * kMaxCalls + i] ? t.table[static_cast<long long>(list.a[i]) * t.max_pages + x] : -1;
    __syncthreads();
    for (int i = first; i < list.n; i += kStep) {
      const int p = plan[i], copy = plan[kMaxCalls + i], was = old[i][c];
      int now = -1;
      if (p >= 0 && x < list.d[p]) {
        now = copy >= 0 && x >= list.c[p] ? ids[copy + x - list.c[p]] : old[p][c];
        if (!valid(now)) report(t.status, kStatusCheck);
      }
      if (x >= plan[2 * kMaxCalls + i] && now < 0) continue;
      if (now == was && valid(was)) continue;
      if (x < plan[2 * kMaxCalls + i] && (!valid(was) || atomicSub(&t.refs[was], 1) <= 0)) {
        if (valid(was)) atomicAdd(&t.refs[was], 1);
        report(t.status, kStatusCheck);
      }
      if (valid(now)) atomicAdd(&t.refs[now], 1);
      t.table[static_cast<long long>(list.a[i]) * t.max_pages + x] = now;
    }
    __syncthreads();
  }
}

// compact, first part: moves[0] = number of moves, then their sources and destinations; the map of ids; the
// new counts
__global__ void __launch_bounds__(kPlanThreads) compact_plan_kernel(PoolTables t, int* refs_out, int* moves, int* map) {
  extern __shared__ uint32_t live[];  // a bit for every page
  __shared__ int scratch[kPlanThreads / 32];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, words = (t.n_pages + 31) / 32;
  griddep_wait();
  griddep_launch();
  int mine = 0;
  for (int w0 = warp; w0 < words; w0 += 8 * (kPlanThreads / 32)) {
    int v[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const int page = (w0 + k * (kPlanThreads / 32)) * 32 + lane;
      v[k] = page < t.n_pages ? t.refs[page] : 0;
    }
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const int w = w0 + k * (kPlanThreads / 32);
      const uint32_t b = __ballot_sync(0xffffffffu, v[k] > 0);
      if (w < words && lane == 0) {
        live[w] = b;
        mine += __popc(b);
      }
    }
  }
  int L;
  block_scan(mine, scratch, &L);
  // thread t ranks a run of words: free pages below L, pages in use from L on
  const int per = (words + kPlanThreads - 1) / kPlanThreads, w0 = min(tid * per, words), w1 = min(w0 + per, words);
  int nfree = 0, nhigh = 0;
  const auto below = [&](int w) {  // bits of word w that are pages below L
    const int k = L - w * 32;
    return k >= 32 ? 0xffffffffu : k <= 0 ? 0u : (1u << k) - 1u;
  };
  for (int w = w0; w < w1; ++w) {
    nfree += __popc(~live[w] & below(w));
    nhigh += __popc(live[w] & ~below(w));
  }
  int n_moves, total;
  int at_high = block_scan(nhigh, scratch, &n_moves);
  __syncthreads();
  int at_free = block_scan(nfree, scratch, &total);
  int *src = moves + 1, *dst = moves + 1 + t.n_pages;
  for (int w = w0; w < w1; ++w) {
    for (uint32_t x = ~live[w] & below(w); x; x &= x - 1) dst[at_free++] = w * 32 + __ffs(x) - 1;
    for (uint32_t x = live[w] & ~below(w); x; x &= x - 1) src[at_high++] = w * 32 + __ffs(x) - 1;
  }
  if (tid == 0) moves[0] = n_moves;
  __syncthreads();
  // (a free page below L is some move's destination: its count is written there alone)
  for (int i = tid; i < n_moves; i += kPlanThreads) {
    const int s = src[i], d = dst[i], r = t.refs[s];
    map[s] = d;
    refs_out[d] = r;
    refs_out[s] = 0;
  }
  for (int page = tid; page < t.n_pages; page += kPlanThreads) {
    const bool on = live[page >> 5] >> (page & 31) & 1u;
    if (page < L && on) refs_out[page] = t.refs[page];
    if (page >= L && !on) refs_out[page] = 0;
    if (page < L || !on) map[page] = page;
  }
}

// compact, second part: CTAs [0, row_ctas) rewrite the table, the others copy pages
__global__ void __launch_bounds__(kCopyThreads) compact_kernel(PoolTables t, const __grid_constant__ Layers ly, int* table_out, const int* moves,
                                                               const int* map, int row_ctas) {
  griddep_wait();
  griddep_launch();
  const int n_moves = moves[0];
  if (static_cast<int>(blockIdx.x) < row_ctas) {
    const long long n = static_cast<long long>(t.n_seqs) * t.max_pages;
    for (long long i = blockIdx.x * static_cast<long long>(kCopyThreads) + threadIdx.x; i < n; i += static_cast<long long>(row_ctas) * kCopyThreads) {
      const int page = t.table[i];
      table_out[i] = page >= 0 && page < t.n_pages ? map[page] : page;
    }
    return;
  }
  const int pieces = static_cast<int>((ly.page_bytes + kPiece - 1) / kPiece);
  const int *src = moves + 1, *dst = moves + 1 + t.n_pages;
  const long long units = static_cast<long long>(n_moves) * ly.n * pieces;
  for (long long u = blockIdx.x - row_ctas; u < units; u += gridDim.x - row_ctas) {
    const int m = static_cast<int>(u / (static_cast<long long>(ly.n) * pieces));
    const int rest = static_cast<int>(u - static_cast<long long>(m) * ly.n * pieces);
    copy_piece(ly.base[rest / pieces], ly.page_bytes, src[m], dst[m], rest % pieces);
  }
}

__global__ void __launch_bounds__(kCopyThreads) copy_kernel(PoolTables t, const __grid_constant__ Layers ly, const int* src, const int* dst, int n) {
  griddep_wait();
  griddep_launch();
  const int pieces = static_cast<int>((ly.page_bytes + kPiece - 1) / kPiece);
  const long long units = static_cast<long long>(n) * ly.n * pieces;
  for (long long u = blockIdx.x; u < units; u += gridDim.x) {
    const int m = static_cast<int>(u / (static_cast<long long>(ly.n) * pieces));
    const int rest = static_cast<int>(u - static_cast<long long>(m) * ly.n * pieces);
    const int s = src[m], d = dst[m];
    if (s < 0 || s >= t.n_pages || d < 0 || d >= t.n_pages) {
      if (threadIdx.x == 0) report(t.status, kStatusCheck);
      continue;
    }
    copy_piece(ly.base[rest / pieces], ly.page_bytes, s, d, rest % pieces);
  }
}

tss_status take_layers(void* const* layer, int n_layers, size_t page_bytes, Layers* out) {
  if (!layer || n_layers < 1 || n_layers > kMaxPoolLayers) return refuse(TSS_ERR_INVALID_ARG, "n_layers must be in [1, 128]");
  if (page_bytes == 0 || page_bytes % 16 || page_bytes > (size_t(1) << 30))
    return refuse(TSS_ERR_INVALID_ARG, "page_bytes must be a multiple of 16, at most 2^30");
  out->n = n_layers;
  out->page_bytes = page_bytes;
  for (int i = 0; i < n_layers; ++i) {
    if (!layer[i] || !aligned16(layer[i])) return refuse(TSS_ERR_INVALID_ARG, "every layer's pages must be 16-byte aligned device memory");
    out->base[i] = static_cast<uint8_t*>(layer[i]);
  }
  return TSS_OK;
}
tss_status take_tables(const tss_pages* h, const tss_page_tables* t, PoolTables* out) {
  if (!h || !t || !t->table || !t->held || !t->refs) return refuse(TSS_ERR_INVALID_ARG, "NULL argument");
  const tss_status on = still_on(h->dev);
  if (on != TSS_OK) return on;
  *out = PoolTables{t->table, t->held, t->refs, h->n_seqs, h->max_pages, h->n_pages, h->status};
  return TSS_OK;
}
bool distinct(const int32_t* a, int n) {
  for (int i = 0; i < n; ++i)
    for (int j = 0; j < i; ++j)
      if (a[i] == a[j]) return false;
  return true;
}
tss_status take_seqs(const tss_pages* h, int n, const int32_t* seq, const char* what) {
  if (n < 0 || n > kMaxCalls) return refuse(TSS_ERR_INVALID_ARG, "n must be in [0, 64]");
  if (n > 0 && !seq) return refuse(TSS_ERR_INVALID_ARG, "NULL argument");
  for (int i = 0; i < n; ++i)
    if (seq[i] < 0 || seq[i] >= h->n_seqs) return refuse(TSS_ERR_INVALID_ARG, what);
  return TSS_OK;
}
unsigned copy_grid(long long pages, const Layers& ly, int sms) {
  const long long units = pages * ly.n * static_cast<long long>((ly.page_bytes + kPiece - 1) / kPiece);
  const long long most = static_cast<long long>(sms) * 6;
  return static_cast<unsigned>(units < most ? units : most);
}
tss_status launched(cudaError_t e) {
  return e == cudaSuccess ? TSS_OK : refuse_cuda(e, "launch");
}

}  // namespace
}  // namespace tss

using namespace tss;

extern "C" tss_status tss_pages_create(int n_seqs, int max_pages, int n_pages, tss_pages** out) {
  if (!out) return refuse(TSS_ERR_INVALID_ARG, "out is NULL");
  *out = nullptr;
  if (n_seqs < 1 || max_pages < 1 || static_cast<long long>(n_seqs) * max_pages > 0x7fffffffLL)
    return refuse(TSS_ERR_INVALID_ARG, "n_seqs and max_pages must be >= 1 and their product below 2^31");
  if (n_pages < 1 || n_pages > kMaxPoolPages) return refuse(TSS_ERR_INVALID_ARG, "n_pages must be in [1, 2^20]");
  int dev = 0, sms = 0;
  const tss_status st = this_device(&dev, &sms);
  if (st != TSS_OK) return st;
  tss_pages* h = new (std::nothrow) tss_pages{};
  if (!h) return refuse(TSS_ERR_OUT_OF_MEMORY, "no host memory");
  h->n_seqs = n_seqs;
  h->max_pages = max_pages;
  h->n_pages = n_pages;
  h->dev = dev;
  h->sms = sms;
  cudaError_t e = cudaMalloc(&h->status, 256);
  if (e == cudaSuccess) e = zero_now(h->status, 256);
  if (e == cudaSuccess) e = cudaMalloc(&h->moves, sizeof(int) * (1 + 2 * static_cast<size_t>(n_pages)));
  if (e == cudaSuccess) e = cudaMalloc(&h->map, sizeof(int) * static_cast<size_t>(n_pages));
  if (e == cudaSuccess) e = cudaMalloc(&h->plan, sizeof(int) * 4 * kMaxCalls);
  if (e == cudaSuccess) e = cudaFuncSetAttribute(compact_plan_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kMaxPoolPages / 8);
  if (e != cudaSuccess) {
    tss_pages_destroy(h);
    const tss_status r = refuse_cuda(e, "workspace");
    return e == cudaErrorMemoryAllocation ? TSS_ERR_OUT_OF_MEMORY : r;
  }
  h->go = h->status + 16;
  *out = h;
  return TSS_OK;
}

extern "C" void tss_pages_destroy(tss_pages* h) {
  if (!h) return;
  cudaFree(h->status);
  cudaFree(h->moves);
  cudaFree(h->map);
  cudaFree(h->plan);
  delete h;
}

extern "C" tss_status tss_pages_sync_status(tss_pages* h, void* stream) {
  if (!h) return refuse(TSS_ERR_INVALID_ARG, "NULL argument");
  const tss_status on = still_on(h->dev);
  if (on != TSS_OK) return on;
  int v = 0;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  cudaError_t e = cudaMemcpyAsync(&v, h->status, sizeof(int), cudaMemcpyDeviceToHost, s);
  if (e == cudaSuccess) e = cudaMemsetAsync(h->status, 0, sizeof(int), s);
  if (e == cudaSuccess) e = cudaStreamSynchronize(s);
  if (e != cudaSuccess) return refuse_cuda(e, "status read");
  if (v != TSS_OK) return refuse(v, "device status of the page calls");
  return TSS_OK;
}

extern "C" tss_status tss_pages_reserve(tss_pages* h, const tss_page_tables* t, int n, const int32_t* seq, const int32_t* want, void* stream) {
  PoolTables pt;
  tss_status st = take_tables(h, t, &pt);
  if (st == TSS_OK) st = take_seqs(h, n, seq, "seq must be in [0, n_seqs)");
  if (st != TSS_OK) return st;
  if (n == 0) return TSS_OK;
  if (!want) return refuse(TSS_ERR_INVALID_ARG, "NULL argument");
  if (!distinct(seq, n)) return refuse(TSS_ERR_INVALID_ARG, "a sequence appears twice");
  SeqList list{};
  list.n = n;
  for (int i = 0; i < n; ++i) {
    if (want[i] < 0) return refuse(TSS_ERR_INVALID_ARG, "want must be >= 0");
    if (want[i] > h->max_pages) return refuse(TSS_ERR_KV_CAPACITY, "want exceeds max_pages");
    list.a[i] = seq[i];
    list.b[i] = want[i];
  }
  return launched(launch_k(reserve_kernel, dim3(1), dim3(kPlanThreads), 0, static_cast<cudaStream_t>(stream), true, list, pt, h->moves + 1));
}

extern "C" tss_status tss_pages_free(tss_pages* h, const tss_page_tables* t, int n, const int32_t* seq, const int32_t* keep, void* stream) {
  PoolTables pt;
  tss_status st = take_tables(h, t, &pt);
  if (st == TSS_OK) st = take_seqs(h, n, seq, "seq must be in [0, n_seqs)");
  if (st != TSS_OK) return st;
  if (n == 0) return TSS_OK;
  if (!distinct(seq, n)) return refuse(TSS_ERR_INVALID_ARG, "a sequence appears twice");
  SeqList list{};
  list.n = n;
  for (int i = 0; i < n; ++i) {
    if (keep && keep[i] < 0) return refuse(TSS_ERR_INVALID_ARG, "keep must be >= 0");
    list.a[i] = seq[i];
    // (no sequence holds more: the kernel counts up from here, which would wrap near the largest int)
    list.b[i] = !keep ? 0 : keep[i] < h->max_pages ? keep[i] : h->max_pages;
  }
  return launched(launch_k(free_kernel, dim3(n), dim3(256), 0, static_cast<cudaStream_t>(stream), true, list, pt));
}

extern "C" tss_status tss_pages_fork(tss_pages* h, const tss_page_tables* t, void* const* layer, int n_layers, size_t page_bytes, int n,
                                     const int32_t* src, const int32_t* dst, const int32_t* shared, const int32_t* total, void* stream) {
  PoolTables pt;
  Layers ly{};
  tss_status st = take_tables(h, t, &pt);
  if (st == TSS_OK) st = take_seqs(h, n, src, "src must be in [0, n_seqs)");
  if (st == TSS_OK) st = take_seqs(h, n, dst, "dst must be in [0, n_seqs)");
  if (st == TSS_OK) st = take_layers(layer, n_layers, page_bytes, &ly);
  if (st != TSS_OK) return st;
  if (n == 0) return TSS_OK;
  if (!shared || !total) return refuse(TSS_ERR_INVALID_ARG, "NULL argument");
  if (!distinct(dst, n)) return refuse(TSS_ERR_INVALID_ARG, "a dst appears twice");
  SeqList list{};
  list.n = n;
  long long need = 0;
  for (int i = 0; i < n; ++i) {
    for (int j = 0; j < n; ++j)
      if (dst[i] == src[j]) return refuse(TSS_ERR_INVALID_ARG, "a dst is a src");
    if (shared[i] < 0 || total[i] < shared[i]) return refuse(TSS_ERR_INVALID_ARG, "0 <= shared <= total is wanted");
    if (total[i] > h->max_pages) return refuse(TSS_ERR_KV_CAPACITY, "total exceeds max_pages");
    list.a[i] = src[i];
    list.b[i] = dst[i];
    list.c[i] = shared[i];
    list.d[i] = total[i];
    need += total[i] - shared[i];
  }
  if (need > h->n_pages) return refuse(TSS_ERR_KV_CAPACITY, "more copies than the pool has pages");
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  int* ids = h->moves + 1;
  st = launched(launch_k(fork_choose_kernel, dim3(1), dim3(kPlanThreads), 0, s, true, list, pt, static_cast<int>(need), ids, h->go));
  if (st != TSS_OK) return st;
  return launched(launch_k(fork_kernel, dim3(n + copy_grid(need, ly, h->sms)), dim3(kCopyThreads), 0, s, true, list, pt, ly, ids, h->go));
}

extern "C" tss_status tss_pages_reorder(tss_pages* h, const tss_page_tables* t, void* const* layer, int n_layers, size_t page_bytes, int n,
                                        const int32_t* seq, const int32_t* parent, const int32_t* shared, const int32_t* total, void* stream) {
  PoolTables pt;
  Layers ly{};
  tss_status st = take_tables(h, t, &pt);
  if (st == TSS_OK) st = take_seqs(h, n, seq, "seq must be in [0, n_seqs)");
  if (st == TSS_OK) st = take_layers(layer, n_layers, page_bytes, &ly);
  if (st != TSS_OK) return st;
  if (n == 0) return TSS_OK;
  if (!parent || !shared || !total) return refuse(TSS_ERR_INVALID_ARG, "NULL argument");
  if (reinterpret_cast<uintptr_t>(parent) & 3u) return refuse(TSS_ERR_INVALID_ARG, "parent is not aligned to its elements");
  if (!distinct(seq, n)) return refuse(TSS_ERR_INVALID_ARG, "a sequence appears twice");
  SeqList list{};
  list.n = n;
  int tail = 0;
  for (int i = 0; i < n; ++i) {
    if (shared[i] < 0 || total[i] < shared[i]) return refuse(TSS_ERR_INVALID_ARG, "0 <= shared <= total is wanted");
    if (total[i] > h->max_pages) return refuse(TSS_ERR_KV_CAPACITY, "total exceeds max_pages");
    list.a[i] = seq[i];
    list.c[i] = shared[i];
    list.d[i] = total[i];
    tail = tail > total[i] - shared[i] ? tail : total[i] - shared[i];
  }
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  int *src = h->moves + 1, *ids = h->moves + 1 + h->n_pages;
  st = launched(launch_k(reorder_choose_kernel, dim3(1), dim3(kPlanThreads), 0, s, true, list, pt, parent, h->plan, src, ids, h->moves, h->go));
  if (st != TSS_OK) return st;
  const int cols = (h->max_pages + kReorderCols - 1) / kReorderCols, col_ctas = cols < h->sms ? cols : h->sms;
  return launched(launch_k(reorder_kernel, dim3(col_ctas + copy_grid(static_cast<long long>(n - 1) * tail, ly, h->sms)), dim3(kCopyThreads), 0, s,
                           true, list, pt, ly, h->plan, src, ids, h->moves, h->go, col_ctas));
}

extern "C" tss_status tss_pages_compact(tss_pages* h, const tss_page_tables* t, int32_t* table_out, int32_t* refs_out, void* const* layer,
                                        int n_layers, size_t page_bytes, void* stream) {
  PoolTables pt;
  Layers ly{};
  tss_status st = take_tables(h, t, &pt);
  if (st == TSS_OK) st = take_layers(layer, n_layers, page_bytes, &ly);
  if (st != TSS_OK) return st;
  if (!table_out || !refs_out) return refuse(TSS_ERR_INVALID_ARG, "NULL argument");
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  const size_t smem = static_cast<size_t>((h->n_pages + 31) / 32) * 4;
  st = launched(launch_k(compact_plan_kernel, dim3(1), dim3(kPlanThreads), smem, s, true, pt, refs_out, h->moves, h->map));
  if (st != TSS_OK) return st;
  const long long entries = static_cast<long long>(h->n_seqs) * h->max_pages;
  const int row_ctas = static_cast<int>(entries < 64LL * kCopyThreads * 4 ? (entries + kCopyThreads * 4 - 1) / (kCopyThreads * 4) : 64);
  return launched(launch_k(compact_kernel, dim3(row_ctas + copy_grid(h->n_pages, ly, h->sms)), dim3(kCopyThreads), 0, s, true, pt, ly, table_out,
                           h->moves, h->map, row_ctas));
}

extern "C" tss_status tss_pages_copy(tss_pages* h, void* const* layer, int n_layers, size_t page_bytes, int n, const int32_t* src,
                                     const int32_t* dst, void* stream) {
  Layers ly{};
  if (!h) return refuse(TSS_ERR_INVALID_ARG, "NULL argument");
  tss_status st = still_on(h->dev);
  if (st == TSS_OK) st = take_layers(layer, n_layers, page_bytes, &ly);
  if (st != TSS_OK) return st;
  if (n < 0) return refuse(TSS_ERR_INVALID_ARG, "n must be >= 0");
  if (n == 0) return TSS_OK;
  if (!src || !dst) return refuse(TSS_ERR_INVALID_ARG, "NULL argument");
  PoolTables pt{nullptr, nullptr, nullptr, h->n_seqs, h->max_pages, h->n_pages, h->status};
  return launched(launch_k(copy_kernel, dim3(copy_grid(n, ly, h->sms)), dim3(kCopyThreads), 0, static_cast<cudaStream_t>(stream), true, pt, ly, src,
                           dst, n));
}
