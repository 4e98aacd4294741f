// Paged cache of ciphertext rows (gfx950): the bookkeeping and the row moves of
// append, fork, free, compact and gather.  Layouts and meanings:
// include/ckks_linear.h (ckks_cache).
//
// The bookkeeping (lengths, tables, holders of a page) lives on the device, so a
// step is a chain of launches with no copy to the host between them and can be
// captured.  Every result is a function of the inputs alone: pages are handed
// out in ascending order to the requests in order, and the only atomics are
// integer sums and maxima.  Page numbers read from a table are checked against
// the pool before use, so a table that the caller corrupted reads as absent rows.
#include "ckks_internal.hpp"

namespace ckks {
namespace {

typedef unsigned int v4u __attribute__((ext_vector_type(4)));

constexpr int kPlanThreads = 1024;          // the one workgroup of a plan
constexpr int kPlanWaves = kPlanThreads / 64;
constexpr int kWaveThreads = 256;           // kernels with one wave a request
constexpr int kMoveThreads = 256;
constexpr int kMoveVecs = 4;                // 16-byte pieces a thread has in flight
constexpr uint32_t kPieceWords = kMoveThreads * kMoveVecs * 4;  // 16 KiB

struct Move {
  const uint32_t* src;
  uint32_t* dst;
};

// Workspace of an append or a compaction.
struct Plan {
  uint32_t* moves_n;  // [1] number of moves
  Move* moves;
  int32_t* fresh;     // append: pages handed out, ascending; compact: holes
  int32_t* movers;    // compact: pages that move
  int32_t* to;        // compact: [pages] new page, -1 where it stays
  int32_t* sharers;   // append: [pages] requests that would write a shared last page
  int32_t* last;      // append: [pages] the highest of them
  int32_t* base;      // append: [count] first index into `fresh`, -1 for a refused request
  int32_t* copies;    // append: [count] first copy move
};

size_t take(size_t& at, size_t bytes) {
  const size_t o = at;
  at = (at + bytes + 255) & ~size_t(255);
  return o;
}

size_t append_moves(const Cache& c, uint32_t count, uint32_t rows) {
  return static_cast<size_t>(rows) + static_cast<size_t>(count) * (c.page_rows - 1);
}

size_t append_layout(const Cache& c, uint32_t count, uint32_t rows, uint8_t* base, Plan* p) {
  size_t at = 0;
  const size_t o_n = take(at, 4), o_m = take(at, append_moves(c, count, rows) * sizeof(Move));
  const size_t o_f = take(at, size_t(c.pages) * 4), o_s = take(at, size_t(c.pages) * 4);
  const size_t o_l = take(at, size_t(c.pages) * 4), o_b = take(at, size_t(count) * 4), o_c = take(at, size_t(count) * 4);
  if (p) {
    *p = Plan{};
    p->moves_n = reinterpret_cast<uint32_t*>(base + o_n);
    p->moves = reinterpret_cast<Move*>(base + o_m);
    p->fresh = reinterpret_cast<int32_t*>(base + o_f);
    p->sharers = reinterpret_cast<int32_t*>(base + o_s);
    p->last = reinterpret_cast<int32_t*>(base + o_l);
    p->base = reinterpret_cast<int32_t*>(base + o_b);
    p->copies = reinterpret_cast<int32_t*>(base + o_c);
  }
  return at;
}

size_t compact_layout(const Cache& c, uint8_t* base, Plan* p) {
  size_t at = 0;
  const size_t half = (c.pages + 1) / 2;  // at most half of the pages move
  const size_t o_n = take(at, 4), o_m = take(at, half * sizeof(Move)), o_f = take(at, half * 4);
  const size_t o_v = take(at, half * 4), o_t = take(at, size_t(c.pages) * 4);
  if (p) {
    *p = Plan{};
    p->moves_n = reinterpret_cast<uint32_t*>(base + o_n);
    p->moves = reinterpret_cast<Move*>(base + o_m);
    p->fresh = reinterpret_cast<int32_t*>(base + o_f);
    p->movers = reinterpret_cast<int32_t*>(base + o_v);
    p->to = reinterpret_cast<int32_t*>(base + o_t);
  }
  return at;
}

// Pages that `rows` rows take.
__device__ __forceinline__ int32_t pages_of(int32_t rows, int32_t page_rows) {
  return static_cast<int32_t>((static_cast<uint32_t>(rows) + page_rows - 1) / page_rows);
}

// A length as the table can hold it (the caller's memory may hold anything).
__device__ __forceinline__ int32_t held_rows(const Cache& c, int32_t s) {
  const int64_t most = static_cast<int64_t>(c.max_pages) * c.page_rows;
  const int32_t n = c.lens[s];
  return n < 0 ? 0 : n < most ? n : static_cast<int32_t>(most);
}

__device__ __forceinline__ int32_t fresh_load(const int32_t* p) {
  return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

// Exclusive prefix sum of v over the workgroup's threads; *total the whole sum.
__device__ __forceinline__ uint32_t scan(uint32_t v, uint32_t* lds, uint32_t* total) {
  const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  uint32_t x = v;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const uint32_t y = __shfl_up(x, d);
    if (lane >= static_cast<uint32_t>(d)) x += y;
  }
  __syncthreads();  // earlier readers of lds are done
  if (lane == 63) lds[wave] = x;
  __syncthreads();
  uint32_t before = 0, sum = 0;
#pragma unroll
  for (int w = 0; w < kPlanWaves; ++w) {
    const uint32_t y = lds[w];
    before += static_cast<uint32_t>(w) < wave ? y : 0;
    sum += y;
  }
  *total = sum;
  return before + x - v;
}

__device__ __forceinline__ bool valid_page(const Cache& c, int32_t page) {
  return static_cast<uint32_t>(page) < c.pages;
}

__global__ __launch_bounds__(kWaveThreads) void cache_init_kernel(Cache c) {
  const size_t at = static_cast<size_t>(blockIdx.x) * kWaveThreads + threadIdx.x;
  const size_t step = static_cast<size_t>(gridDim.x) * kWaveThreads;
  for (size_t i = at; i < c.pages; i += step) c.refs[i] = 0;
  for (size_t i = at; i < c.seqs; i += step) c.lens[i] = 0;
  const size_t entries = static_cast<size_t>(c.seqs) * c.max_pages;
  for (size_t i = at; i < entries; i += step) c.table[i] = -1;
}

// One wave a request.  A sequence named twice is refused both times: the wave
// looks the whole list over, 64 requests at a time.
__global__ __launch_bounds__(kWaveThreads) void cache_free_kernel(Cache c, const int32_t* __restrict__ seq,
                                                                  const int32_t* __restrict__ keep, uint32_t count,
                                                                  int32_t* __restrict__ status) {
  const uint32_t i = (blockIdx.x * kWaveThreads + threadIdx.x) >> 6, lane = threadIdx.x & 63;
  if (i >= count) return;
  const int32_t s = seq[i];
  bool bad = static_cast<uint32_t>(s) >= c.seqs;
  for (uint32_t j = lane; j < count; j += 64) bad |= j != i && seq[j] == s;
  if (__any(bad)) {
    if (status && lane == 0) status[i] = kCacheBadRequest;
    return;
  }
  const int32_t rows = held_rows(c, s);
  int32_t kept = keep ? keep[i] : 0;
  kept = kept < 0 ? 0 : kept;
  if (kept < rows) {
    int32_t* t = c.table + static_cast<size_t>(s) * c.max_pages;
    const int32_t end = pages_of(rows, c.page_rows);
    for (int32_t at = pages_of(kept, c.page_rows) + lane; at < end; at += 64) {
      const int32_t page = t[at];
      if (valid_page(c, page)) atomicSub(&c.refs[page], 1);
      t[at] = -1;
    }
    if (lane == 0) c.lens[s] = kept;
  }
  if (status && lane == 0) status[i] = kCacheOk;
}

// One wave a request: the target's pages lose a holder, the source's gain one.
// Refused: numbers out of range, a target that another request names, or whose
// source is another's target.
__global__ __launch_bounds__(kWaveThreads) void cache_fork_kernel(Cache c, const int32_t* __restrict__ src,
                                                                  const int32_t* __restrict__ dst, uint32_t count,
                                                                  int32_t* __restrict__ status) {
  const uint32_t i = (blockIdx.x * kWaveThreads + threadIdx.x) >> 6, lane = threadIdx.x & 63;
  if (i >= count) return;
  const int32_t s = src[i], d = dst[i];
  bool bad = static_cast<uint32_t>(s) >= c.seqs || static_cast<uint32_t>(d) >= c.seqs || s == d;
  for (uint32_t j = lane; j < count; j += 64) {
    const int32_t sj = src[j], dj = dst[j];
    bad |= (j != i && dj == d) || sj == d || dj == s;
  }
  if (__any(bad)) {
    if (status && lane == 0) status[i] = kCacheBadRequest;
    return;
  }
  const int32_t rows = held_rows(c, s), old = held_rows(c, d);
  const int32_t end = pages_of(rows, c.page_rows), old_end = pages_of(old, c.page_rows);
  const int32_t* ts = c.table + static_cast<size_t>(s) * c.max_pages;
  int32_t* td = c.table + static_cast<size_t>(d) * c.max_pages;
  for (int32_t at = lane; at < static_cast<int32_t>(c.max_pages); at += 64) {
    const int32_t was = at < old_end ? td[at] : -1;
    if (valid_page(c, was)) atomicSub(&c.refs[was], 1);
    const int32_t page = at < end ? ts[at] : -1;
    if (valid_page(c, page)) atomicAdd(&c.refs[page], 1);
    td[at] = page;
  }
  if (lane == 0) {
    c.lens[d] = rows;
    if (status) status[i] = kCacheOk;
  }
}

// Rows that request i appends, as row0 says (one row each without it); -1 if row0
// is not ascending within the rows that there are.
__device__ __forceinline__ int32_t asked_rows(const int32_t* row0, uint32_t i, uint32_t rows) {
  if (!row0) return i < rows ? 1 : -1;
  const int32_t a = row0[i], b = row0[i + 1];
  return a >= 0 && b >= a && static_cast<uint32_t>(b) <= rows ? b - a : -1;
}

// What an append does, worked out by one workgroup: pages for every request,
// the tables, lengths and holders, and the list of row moves.
__global__ __launch_bounds__(kPlanThreads) void cache_append_plan_kernel(
    Cache c, const int32_t* __restrict__ seq, const int32_t* __restrict__ row0, uint32_t count,
    const uint32_t* __restrict__ rows_in, uint32_t rows, int32_t* __restrict__ status, Plan p) {
  __shared__ uint32_t seen[kCacheMaxSeqs / 32], twice[kCacheMaxSeqs / 32];
  __shared__ uint32_t lds[kPlanWaves];
  const uint32_t tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int32_t P = c.page_rows;
  for (uint32_t w = tid; w < (c.seqs + 31) / 32; w += kPlanThreads) seen[w] = twice[w] = 0;
  bool astray = false;  // row0 that runs backwards would give one row to two requests: nobody is served
  for (uint32_t i = tid; i < count; i += kPlanThreads) astray |= asked_rows(row0, i, rows) < 0;
  astray = __syncthreads_or(astray && row0);
  for (uint32_t i = tid; i < count; i += kPlanThreads) {
    const uint32_t s = seq[i];
    if (s >= c.seqs) continue;
    const uint32_t bit = 1u << (s & 31);
    if (atomicOr(&seen[s >> 5], bit) & bit) atomicOr(&twice[s >> 5], bit);
  }
  __syncthreads();
  // 0 for a request that is served, else why not
  auto refused = [&](uint32_t i, int32_t* s, int32_t* have, int32_t* want) {
    *s = seq[i];
    *want = asked_rows(row0, i, rows);
    if (astray || static_cast<uint32_t>(*s) >= c.seqs || *want < 0 || (twice[*s >> 5] >> (*s & 31) & 1)) return kCacheBadRequest;
    *have = held_rows(c, *s);
    const int64_t most = static_cast<int64_t>(c.max_pages) * P;
    return static_cast<int64_t>(*have) + *want > most || static_cast<int64_t>(*have) + *want > 0x7fffffff ? kCacheTableFull
                                                                                                          : kCacheOk;
  };
  // the page that the request's first row falls into, if it is partly filled and held by others too
  auto shared_last = [&](int32_t s, int32_t have, int32_t want) {
    if (want == 0 || have % P == 0) return -1;
    const int32_t page = c.table[static_cast<size_t>(s) * c.max_pages + have / P];
    return valid_page(c, page) && fresh_load(&c.refs[page]) > 1 ? page : -1;
  };
  int32_t s, have, want;
  for (uint32_t i = tid; i < count; i += kPlanThreads) {
    if (refused(i, &s, &have, &want) != kCacheOk) continue;
    const int32_t page = shared_last(s, have, want);
    if (page >= 0) p.sharers[page] = 0, p.last[page] = -1;
  }
  __threadfence();  // the stores are in memory before the atomics on the same words
  __syncthreads();
  for (uint32_t i = tid; i < count; i += kPlanThreads) {
    if (refused(i, &s, &have, &want) != kCacheOk) continue;
    const int32_t page = shared_last(s, have, want);
    if (page >= 0) {
      atomicAdd(&p.sharers[page], 1);
      atomicMax(&p.last[page], static_cast<int32_t>(i));
    }
  }
  __syncthreads();
  // Where every holder of a page is in the call, the last of them keeps it.
  auto copies_page = [&](uint32_t i, int32_t page) {
    return page >= 0 && !(fresh_load(&p.sharers[page]) == fresh_load(&c.refs[page]) &&
                          fresh_load(&p.last[page]) == static_cast<int32_t>(i));
  };
  uint32_t pages_total = 0, copies_total = 0;
  for (uint32_t i0 = 0; i0 < count; i0 += kPlanThreads) {
    const uint32_t i = i0 + tid;
    uint32_t need = 0, copies = 0;
    bool serve = false;
    if (i < count) {
      const int32_t why = refused(i, &s, &have, &want);
      serve = why == kCacheOk;
      if (serve) {
        const bool copy = copies_page(i, shared_last(s, have, want));
        need = pages_of(have + want, P) - pages_of(have, P) + copy;
        copies = copy ? have % P : 0;
      } else if (status) {
        status[i] = why;
      }
    }
    uint32_t sum;
    const uint32_t a = scan(need, lds, &sum);
    uint32_t csum;
    const uint32_t b = scan(copies, lds, &csum);
    if (i < count) {
      p.base[i] = serve ? static_cast<int32_t>(pages_total + a) : -1;
      p.copies[i] = static_cast<int32_t>(copies_total + b);
    }
    pages_total += sum;
    copies_total += csum;
  }
  // the lowest free pages, in order
  uint32_t found = 0;
  for (uint32_t g0 = 0; g0 < c.pages && found < pages_total; g0 += kPlanThreads) {
    const uint32_t page = g0 + tid;
    const bool vacant = page < c.pages && fresh_load(&c.refs[page]) == 0;
    uint32_t sum;
    const uint32_t at = found + scan(vacant, lds, &sum);
    if (vacant) p.fresh[at] = static_cast<int32_t>(page);
    found += sum;
  }
  __syncthreads();
  if (found < pages_total) {  // not enough: nobody is served
    for (uint32_t i = tid; i < count; i += kPlanThreads)
      if (status && p.base[i] >= 0) status[i] = kCacheNoPages;
    if (tid == 0) *p.moves_n = 0;
    return;
  }
  // rows that no served request has stay where they are
  for (uint32_t r = tid; r < rows; r += kPlanThreads) p.moves[r].dst = nullptr;
  __syncthreads();
  for (uint32_t i = wave; i < count; i += kPlanWaves) {
    const int32_t base = p.base[i];
    if (base < 0) continue;
    refused(i, &s, &have, &want);
    int32_t* t = c.table + static_cast<size_t>(s) * c.max_pages;
    const int32_t first = have / P, part = have % P;
    const int32_t was = part && want ? t[first] : -1;
    const bool shared = valid_page(c, was) && fresh_load(&c.refs[was]) > 1;
    const bool copy = shared && copies_page(i, was);
    const int32_t start = copy ? first : pages_of(have, P);  // first position that gets a page
    const int32_t end = pages_of(have + want, P);
    const uint32_t r0 = row0 ? row0[i] : i;
    for (int32_t at = start + lane; at < end; at += 64) {
      const int32_t page = p.fresh[base + at - start];
      t[at] = page;
      c.refs[page] = 1;
    }
    for (int32_t r = lane; r < want; r += 64) {
      const int32_t at = (have + r) / P;
      const int32_t page = at < start ? was : p.fresh[base + at - start];
      if (!valid_page(c, page)) continue;  // the caller's table had no page there
      p.moves[r0 + r] = {rows_in + static_cast<size_t>(r0 + r) * c.row_words,
                         c.pool + (static_cast<size_t>(page) * P + (have + r) % P) * c.row_words};
    }
    if (copy)
      for (int32_t r = lane; r < part; r += 64)
        p.moves[rows + p.copies[i] + r] = {c.pool + (static_cast<size_t>(was) * P + r) * c.row_words,
                                           c.pool + (static_cast<size_t>(p.fresh[base]) * P + r) * c.row_words};
    if (lane == 0) {
      c.lens[s] = have + want;
      if (status) status[i] = kCacheOk;
    }
  }
  __syncthreads();
  // a copied page loses the holder; after every request has looked at its holders
  for (uint32_t i = tid; i < count; i += kPlanThreads) {
    if (p.base[i] < 0) continue;
    const int32_t next = i + 1 < count ? p.copies[i + 1] : static_cast<int32_t>(copies_total);
    if (next == p.copies[i]) continue;
    const Move m = p.moves[rows + p.copies[i]];
    atomicSub(&c.refs[(m.src - c.pool) / (c.row_words * P)], 1);
  }
  if (tid == 0) *p.moves_n = rows + copies_total;
}

// Live pages past the compacted end move into the holes below it, both in
// ascending order.
__global__ __launch_bounds__(kPlanThreads) void cache_compact_plan_kernel(Cache c, int32_t* __restrict__ live_out,
                                                                          Plan p) {
  __shared__ uint32_t lds[kPlanWaves];
  const uint32_t tid = threadIdx.x;
  uint32_t mine = 0, live;
  for (uint32_t g = tid; g < c.pages; g += kPlanThreads) mine += c.refs[g] > 0;
  scan(mine, lds, &live);
  uint32_t holes = 0, movers = 0;
  for (uint32_t g0 = 0; g0 < c.pages; g0 += kPlanThreads) {
    const uint32_t g = g0 + tid;
    const bool held = g < c.pages && c.refs[g] > 0;
    const bool hole = g < live && !held, mover = g >= live && held;
    uint32_t hs, ms;
    const uint32_t h = holes + scan(hole, lds, &hs), m = movers + scan(mover, lds, &ms);
    if (hole) p.fresh[h] = static_cast<int32_t>(g);
    if (mover) p.movers[m] = static_cast<int32_t>(g);
    if (g < c.pages) p.to[g] = -1;
    holes += hs;
    movers += ms;
  }
  __threadfence();
  __syncthreads();
  const size_t page_words = c.row_words * c.page_rows;
  for (uint32_t k = tid; k < movers; k += kPlanThreads) {
    const int32_t from = p.movers[k], to = p.fresh[k];
    p.moves[k] = {c.pool + from * page_words, c.pool + to * page_words};
    p.to[from] = to;
    c.refs[to] = c.refs[from];
    c.refs[from] = 0;
  }
  if (tid == 0) {
    *p.moves_n = movers;
    if (live_out) *live_out = static_cast<int32_t>(live);
  }
}

// One workgroup copies one piece of up to 16 KiB.
__device__ __forceinline__ void copy_piece(const uint32_t* src, uint32_t* dst, size_t words) {
  const v4u* s = reinterpret_cast<const v4u*>(src);
  v4u* d = reinterpret_cast<v4u*>(dst);
  const uint32_t vecs = words < kPieceWords ? words / 4 : kPieceWords / 4;
  v4u x[kMoveVecs];
#pragma unroll
  for (int e = 0; e < kMoveVecs; ++e)
    if (e * kMoveThreads + threadIdx.x < vecs) x[e] = __builtin_nontemporal_load(&s[e * kMoveThreads + threadIdx.x]);
#pragma unroll
  for (int e = 0; e < kMoveVecs; ++e)
    if (e * kMoveThreads + threadIdx.x < vecs) __builtin_nontemporal_store(x[e], &d[e * kMoveThreads + threadIdx.x]);
}

// Carries out the moves (each `words` long), and sends table entries through
// `to` where a compaction gives it.
__global__ __launch_bounds__(kMoveThreads) void cache_move_kernel(Cache c, Plan p, size_t words) {
  const size_t pieces = (words + kPieceWords - 1) / kPieceWords, items = pieces * *p.moves_n;
  for (size_t k = blockIdx.x; k < items; k += gridDim.x) {
    const size_t m = k / pieces, at = (k - m * pieces) * kPieceWords;
    const Move mv = p.moves[m];
    if (mv.dst) copy_piece(mv.src + at, mv.dst + at, words - at);
  }
  if (p.to) {
    const size_t entries = static_cast<size_t>(c.seqs) * c.max_pages;
    for (size_t e = static_cast<size_t>(blockIdx.x) * kMoveThreads + threadIdx.x; e < entries;
         e += static_cast<size_t>(gridDim.x) * kMoveThreads) {
      const int32_t page = c.table[e];
      if (valid_page(c, page) && p.to[page] >= 0) c.table[e] = p.to[page];
    }
  }
}

__global__ __launch_bounds__(kMoveThreads) void cache_gather_kernel(Cache c, const int32_t* __restrict__ seq,
                                                                    const int32_t* __restrict__ pos, uint32_t pieces,
                                                                    uint32_t* __restrict__ out) {
  const uint32_t r = blockIdx.x / pieces;
  const size_t at = static_cast<size_t>(blockIdx.x - r * pieces) * kPieceWords;
  const uint32_t* src = cache_row(c, seq[r], pos[r]);
  uint32_t* dst = out + r * c.row_words + at;
  const size_t words = c.row_words - at;
  if (src) {
    copy_piece(src + at, dst, words);
    return;
  }
  const uint32_t vecs = words < kPieceWords ? words / 4 : kPieceWords / 4;
  for (uint32_t v = threadIdx.x; v < vecs; v += kMoveThreads) reinterpret_cast<v4u*>(dst)[v] = v4u{0, 0, 0, 0};
}

}  // namespace

size_t cache_workspace_bytes(const Cache& c, bool append, uint32_t count, uint32_t rows) {
  return append ? append_layout(c, count, rows, nullptr, nullptr) : compact_layout(c, nullptr, nullptr);
}

hipError_t launch_cache_init(const Cache& c, hipStream_t s) {
  cache_init_kernel<<<256, kWaveThreads, 0, s>>>(c);
  return hipGetLastError();
}

hipError_t launch_cache_free(const Cache& c, const int32_t* seq, const int32_t* keep, uint32_t count, int32_t* status,
                             hipStream_t s) {
  cache_free_kernel<<<(count + 3) / 4, kWaveThreads, 0, s>>>(c, seq, keep, count, status);
  return hipGetLastError();
}

hipError_t launch_cache_fork(const Cache& c, const int32_t* src, const int32_t* dst, uint32_t count, int32_t* status,
                             hipStream_t s) {
  cache_fork_kernel<<<(count + 3) / 4, kWaveThreads, 0, s>>>(c, src, dst, count, status);
  return hipGetLastError();
}

// Workgroups of the move kernel: as many as there can be pieces, at most eight
// a CU, which walk the pieces.
static uint32_t move_blocks(size_t moves, size_t words, uint32_t num_cus) {
  const size_t items = moves * ((words + kPieceWords - 1) / kPieceWords), most = size_t(8) * num_cus;
  return static_cast<uint32_t>(items < 1 ? 1 : items < most ? items : most);
}

hipError_t launch_cache_append(const Cache& c, const int32_t* seq, const int32_t* row0, uint32_t count,
                               const uint32_t* rows_in, uint32_t rows, int32_t* status, void* workspace,
                               uint32_t num_cus, hipStream_t s) {
  Plan p;
  append_layout(c, count, rows, static_cast<uint8_t*>(workspace), &p);
  cache_append_plan_kernel<<<1, kPlanThreads, 0, s>>>(c, seq, row0, count, rows_in, rows, status, p);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  cache_move_kernel<<<move_blocks(append_moves(c, count, rows), c.row_words, num_cus), kMoveThreads, 0, s>>>(
      c, p, c.row_words);
  return hipGetLastError();
}

hipError_t launch_cache_compact(const Cache& c, int32_t* live, void* workspace, uint32_t num_cus, hipStream_t s) {
  Plan p;
  compact_layout(c, static_cast<uint8_t*>(workspace), &p);
  cache_compact_plan_kernel<<<1, kPlanThreads, 0, s>>>(c, live, p);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const size_t page_words = c.row_words * c.page_rows;
  cache_move_kernel<<<move_blocks((c.pages + 1) / 2, page_words, num_cus), kMoveThreads, 0, s>>>(c, p, page_words);
  return hipGetLastError();
}

hipError_t launch_cache_gather(const Cache& c, const int32_t* seq, const int32_t* pos, uint32_t count, uint32_t* out,
                               hipStream_t s) {
  const uint32_t pieces = static_cast<uint32_t>((c.row_words + kPieceWords - 1) / kPieceWords);
  cache_gather_kernel<<<count * pieces, kMoveThreads, 0, s>>>(c, seq, pos, pieces, out);
  return hipGetLastError();
}

}  // namespace ckks
