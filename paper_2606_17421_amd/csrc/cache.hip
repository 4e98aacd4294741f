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
  uint32_t* dst;  // null: nothing to do
};

// One request of an append.
struct Request {
  int32_t why;      // kCacheOk: served
  int32_t seq;
  int32_t want;     // rows to append; -1 for a row0 that runs backwards
  int32_t first;    // first input row
  uint32_t at;      // whole pages before the call
  uint32_t part;    // rows on the page after them
  int32_t last;     // that page; -1 where there is none or the call does not write it
  int32_t holders;  // of `last`
  int32_t copy;     // 1: `last` is held by others too and copied before it is written
  uint32_t need;    // pages from the free ones, the copy's among them
};
__device__ __forceinline__ Request no_request() { return {kCacheBadRequest, 0, 0, 0, 0, 0, -1, 0, 0, 0}; }
// Of the requests that write one shared page the highest rank has the most rows on it, and is the
// last of those.
__device__ __forceinline__ unsigned long long rank(uint32_t part, uint32_t i) {
  return static_cast<unsigned long long>(part) << 32 | i;
}
// The first position of the sequence's table that gets a page.
__device__ __forceinline__ uint32_t first_new(const Request& r) { return r.at + (r.part != 0 && !r.copy); }

// Workspace of an append or a compaction.
struct Plan {
  uint32_t* moves_n;  // [1] number of moves
  Move* moves;
  int32_t* fresh;     // append: pages handed out, ascending; compact: holes
  int32_t* movers;    // compact: pages that move
  int32_t* to;        // compact: [pages] new page, -1 where it stays
  int32_t* sharers;   // append: [pages] requests that would write a shared last page
  unsigned long long* keeper;  // append: [pages] the highest rank (rank()) among them
  Request* requests;  // append: [count]
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
  const size_t o_k = take(at, size_t(c.pages) * 8), o_r = take(at, size_t(count) * sizeof(Request));
  if (p) {
    *p = Plan{};
    p->moves_n = reinterpret_cast<uint32_t*>(base + o_n);
    p->moves = reinterpret_cast<Move*>(base + o_m);
    p->fresh = reinterpret_cast<int32_t*>(base + o_f);
    p->sharers = reinterpret_cast<int32_t*>(base + o_s);
    p->keeper = reinterpret_cast<unsigned long long*>(base + o_k);
    p->requests = reinterpret_cast<Request*>(base + o_r);
  }
  return at;
}

size_t compact_layout(const Cache& c, uint8_t* base, Plan* p) {
  size_t at = 0;
  const size_t half = (size_t(c.pages) + 1) / 2;  // at most half of the pages move
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

template <class T>
__device__ __forceinline__ T fresh_load(const T* p) {
  return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

// Exclusive prefix sums of a pair of counts over the workgroup's threads; *total the whole sums.
__device__ __forceinline__ uint2 scan(uint2 v, uint2* lds, uint2* total) {
  const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  uint2 x = v;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const uint32_t a = __shfl_up(x.x, d), b = __shfl_up(x.y, d);
    if (lane >= static_cast<uint32_t>(d)) x.x += a, x.y += b;
  }
  __syncthreads();  // earlier readers of lds are done
  if (lane == 63) lds[wave] = x;
  __syncthreads();
  uint2 before = make_uint2(0, 0), sum = make_uint2(0, 0);
#pragma unroll
  for (int w = 0; w < kPlanWaves; ++w) {
    const uint2 y = lds[w];
    if (static_cast<uint32_t>(w) < wave) before.x += y.x, before.y += y.y;
    sum.x += y.x;
    sum.y += y.y;
  }
  *total = sum;
  return make_uint2(before.x + x.x - v.x, before.y + x.y - v.y);
}

// The last of the n ascending starts that is at most k (starts[0] <= k).
__device__ __forceinline__ uint32_t owner(const uint32_t* starts, uint32_t n, uint32_t k) {
  uint32_t lo = 0, hi = n;
  while (hi - lo > 1) {
    const uint32_t mid = (lo + hi) / 2;
    if (starts[mid] <= k) lo = mid;
    else hi = mid;
  }
  return lo;
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
// looks the whole list over, 64 requests at a time (5 us up to 1024 requests, 25 us for 8192, 1.4 ms for
// 65,536; a fork of 4096 11 us, of 32,768 350 us).
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
// the tables, lengths and holders, and the list of row moves (first the input rows', then
// the copied rows').  Each request is looked up once (its sequence, length, table entry
// and page's holders are four loads that wait for each other); pages, rows and copies are then
// dealt out to all threads, each finding its request by bisection of the requests' starts in
// LDS.  kFew: at most one request a thread, kept in registers and LDS (with both forms in one
// kernel its code alone, 14 KB, took microseconds to fetch); otherwise requests wait in memory
// and shared pages are counted by atomics.  1 row for each of 64 forks, 1024 pages: 20 us with a wave
// a request, 9 us so.
template <bool kFew>
__global__ __launch_bounds__(kPlanThreads) void cache_append_plan_kernel(
    Cache c, const int32_t* __restrict__ seq, const int32_t* __restrict__ row0, uint32_t count,
    const uint32_t* __restrict__ rows_in, uint32_t rows, int32_t* __restrict__ status, Plan p) {
  __shared__ uint32_t seen[kCacheMaxSeqs / 32], twice[kCacheMaxSeqs / 32];
  __shared__ uint2 lds[kPlanWaves];
  __shared__ Request reqs[kPlanThreads];
  __shared__ uint32_t page0[kPlanThreads], copy0[kPlanThreads];
  __shared__ __align__(16) int32_t pages[kPlanThreads];  // shared pages of the requests, then the first free pages
  __shared__ __align__(16) uint32_t parts[kPlanThreads];  // rows on the shared pages
  const uint32_t tid = threadIdx.x, P = c.page_rows;
  const uint32_t blocks = kFew ? 1 : (count + kPlanThreads - 1) / kPlanThreads;  // of requests
  const int32_t holders0 = tid < c.pages ? c.refs[tid] : 1;  // of the first pages, looked at further down
  // What memory says of a request (loads that wait for each other: before any barrier), and
  // what the call makes of it.
  auto look_up = [&](uint32_t i) {
    Request r = no_request();
    r.seq = seq[i];
    r.want = asked_rows(row0, i, rows);
    r.first = row0 ? row0[i] : static_cast<int32_t>(i);
    if (static_cast<uint32_t>(r.seq) < c.seqs) {
      const uint32_t have = held_rows(c, r.seq);
      r.at = have / P;
      r.part = have - r.at * P;
      if (r.want > 0 && r.part != 0) {
        r.last = c.table[static_cast<size_t>(r.seq) * c.max_pages + r.at];
        if (valid_page(c, r.last)) r.holders = c.refs[r.last];
        else r.last = -1;
      }
    }
    return r;
  };
  Request mine = tid < count ? look_up(tid) : no_request();
  for (uint32_t w = tid; w < (c.seqs + 31) / 32; w += kPlanThreads) seen[w] = twice[w] = 0;
  bool astray = mine.want < 0;  // row0 that runs backwards would give one row to two requests: nobody is served
  if constexpr (!kFew)
    for (uint32_t i = tid + kPlanThreads; i < count; i += kPlanThreads) astray |= asked_rows(row0, i, rows) < 0;
  astray = __syncthreads_or(astray && row0);
  for (uint32_t b = 0; b < blocks; ++b) {
    const uint32_t i = b * kPlanThreads + tid;
    const uint32_t s = i >= count ? c.seqs : b == 0 ? mine.seq : seq[i];
    if (s >= c.seqs) continue;
    const uint32_t bit = 1u << (s & 31);
    if (atomicOr(&seen[s >> 5], bit) & bit) atomicOr(&twice[s >> 5], bit);
  }
  __syncthreads();
  auto judge = [&](Request& r) {
    if (astray || static_cast<uint32_t>(r.seq) >= c.seqs || r.want < 0 || (twice[r.seq >> 5] >> (r.seq & 31) & 1))
      r.why = kCacheBadRequest;
    else if (static_cast<uint64_t>(r.at) * P + r.part + r.want > static_cast<uint64_t>(c.max_pages) * P)
      r.why = kCacheTableFull;
    else
      r.why = kCacheOk;
  };
  auto sharing = [](const Request& r) { return r.why == kCacheOk && r.holders > 1; };
  // Where every holder of a shared page is in the call, the one of the highest rank keeps it; the
  // others copy it.  None of them copies a row that the keeper writes: it has as many rows or more
  // on the page, and writes past them (the moves run in no order).  Then the pages that the request takes.
  auto settle = [&](Request& r, uint32_t i, int32_t sharers, unsigned long long keeper) {
    if (r.why != kCacheOk) return;
    r.copy = r.holders > 1 && !(sharers == r.holders && keeper == rank(r.part, i));
    r.need = r.at + (r.part + r.want + P - 1) / P - first_new(r);
  };
  auto needs = [](const Request& r) { return make_uint2(r.need, r.copy ? r.part : 0); };  // pages, rows to copy
  uint2 total = make_uint2(0, 0), mine0 = make_uint2(0, 0);
  if (tid < count) judge(mine);
  if constexpr (kFew) {
    pages[tid] = sharing(mine) ? mine.last : -1;
    parts[tid] = mine.part;
    __syncthreads();
    int32_t sharers = 0;
    uint32_t most = 0, keeper = 0;
    if (sharing(mine)) {
      auto meet = [&](int32_t page, uint32_t part, uint32_t j) {
        const bool same = page == mine.last, ahead = same && part >= most;
        sharers += same;
        most = ahead ? part : most;
        keeper = ahead ? j : keeper;
      };
      for (uint32_t j = 0; j < count; j += 4) {  // `pages` is padded with -1
        const int4 v = *reinterpret_cast<const int4*>(&pages[j]);
        const uint4 n = *reinterpret_cast<const uint4*>(&parts[j]);
        meet(v.x, n.x, j);
        meet(v.y, n.y, j + 1);
        meet(v.z, n.z, j + 2);
        meet(v.w, n.w, j + 3);
      }
    }
    settle(mine, tid, sharers, rank(most, keeper));
    mine0 = scan(needs(mine), lds, &total);
    reqs[tid] = mine;
    if (status && tid < count && mine.why != kCacheOk) status[tid] = mine.why;
  } else {
    for (uint32_t i = tid; i < count; i += kPlanThreads) {
      Request r = look_up(i);
      judge(r);
      p.requests[i] = r;
      if (sharing(r)) p.sharers[r.last] = 0, p.keeper[r.last] = 0;
    }
    __threadfence();  // the stores are in memory before the atomics on the same words
    __syncthreads();
    for (uint32_t i = tid; i < count; i += kPlanThreads) {
      const Request r = p.requests[i];
      if (!sharing(r)) continue;
      atomicAdd(&p.sharers[r.last], 1);
      atomicMax(&p.keeper[r.last], rank(r.part, i));
    }
    __syncthreads();
    for (uint32_t b = 0; b < blocks; ++b) {
      const uint32_t i = b * kPlanThreads + tid;
      Request r = no_request();
      if (i < count) {
        r = p.requests[i];
        settle(r, i, sharing(r) ? fresh_load(&p.sharers[r.last]) : 0, sharing(r) ? fresh_load(&p.keeper[r.last]) : 0);
        p.requests[i] = r;
        if (status && r.why != kCacheOk) status[i] = r.why;
      }
      uint2 sum;
      scan(needs(r), lds, &sum);
      total.x += sum.x;
      total.y += sum.y;
    }
  }
  // the lowest free pages, in order
  uint32_t found = 0;
  for (uint32_t g0 = 0; g0 < c.pages && found < total.x; g0 += kPlanThreads) {
    const uint32_t page = g0 + tid;
    const bool vacant = page < c.pages && (g0 == 0 ? holders0 : c.refs[page]) == 0;
    uint2 sum;
    const uint32_t at = found + scan(make_uint2(vacant, 0), lds, &sum).x;
    if (vacant) {
      p.fresh[at] = static_cast<int32_t>(page);
      if (at < kPlanThreads) pages[at] = static_cast<int32_t>(page);
    }
    found += sum.x;
  }
  __syncthreads();
  const bool short_of = found < total.x;  // not enough: nobody is served
  if (tid == 0) *p.moves_n = short_of ? 0 : rows + total.y;
  if (short_of) {
    for (uint32_t i = tid; i < count; i += kPlanThreads)
      if (status && (kFew ? mine.why : p.requests[i].why) == kCacheOk) status[i] = kCacheNoPages;
    return;
  }
  // input rows that no request names stay where they are
  const uint32_t named0 = row0 && !astray ? row0[0] : 0;
  const uint32_t named1 = astray ? 0 : row0 ? row0[count] : min(count, rows);
  for (uint32_t r = tid; r < rows; r += kPlanThreads)
    if (r < named0 || r >= named1) p.moves[r].dst = nullptr;
  if (astray) return;
  auto fresh = [&](uint32_t k) { return k < kPlanThreads ? pages[k] : p.fresh[k]; };
  uint2 done = make_uint2(0, 0);
  for (uint32_t b = 0; b < blocks; ++b) {
    const uint32_t i0 = b * kPlanThreads, n = min(count - i0, static_cast<uint32_t>(kPlanThreads));
    uint2 at = mine0, sum = total;
    if constexpr (!kFew) {
      __syncthreads();  // the block before is read out
      mine = tid < n ? p.requests[i0 + tid] : no_request();
      reqs[tid] = mine;
      at = scan(needs(mine), lds, &sum);
    }
    page0[tid] = at.x;
    copy0[tid] = at.y;
    if (tid < n && mine.why == kCacheOk) {
      c.lens[mine.seq] = static_cast<int32_t>(mine.at * P + mine.part + mine.want);
      if (status) status[i0 + tid] = kCacheOk;
      if (mine.copy) atomicSub(&c.refs[mine.last], 1);
    }
    __syncthreads();
    for (uint32_t k = tid; k < sum.x; k += kPlanThreads) {  // pages
      const uint32_t j = owner(page0, n, k);
      const int32_t page = fresh(done.x + k);
      c.table[static_cast<size_t>(reqs[j].seq) * c.max_pages + first_new(reqs[j]) + (k - page0[j])] = page;
      c.refs[page] = 1;
    }
    const uint32_t end = row0 ? row0[i0 + n] : min(i0 + n, rows);
    for (uint32_t k = (row0 ? reqs[0].first : i0) + tid; k < end; k += kPlanThreads) {  // input rows
      uint32_t j = k - i0;
      if (row0) {  // the last request that starts at or before row k (empty ones before it start there too)
        uint32_t lo = 0, hi = n;
        while (hi - lo > 1) {
          const uint32_t mid = (lo + hi) / 2;
          if (static_cast<uint32_t>(reqs[mid].first) <= k) lo = mid;
          else hi = mid;
        }
        j = lo;
      }
      const Request r = reqs[j];
      uint32_t* dst = nullptr;
      if (r.why == kCacheOk) {
        const uint32_t off = r.part + (k - r.first), ahead = off / P;
        const int32_t page = r.at + ahead < first_new(r) ? r.last : fresh(done.x + page0[j] + r.at + ahead - first_new(r));
        if (valid_page(c, page)) dst = c.pool + (static_cast<size_t>(page) * P + (off - ahead * P)) * c.row_words;  // else the caller's table had no page there
      }
      p.moves[k] = {rows_in + static_cast<size_t>(k) * c.row_words, dst};
    }
    for (uint32_t k = tid; k < sum.y; k += kPlanThreads) {  // copied rows
      const uint32_t j = owner(copy0, n, k), slot = k - copy0[j];
      p.moves[rows + done.y + k] = {c.pool + (static_cast<size_t>(reqs[j].last) * P + slot) * c.row_words,
                                    c.pool + (static_cast<size_t>(fresh(done.x + page0[j])) * P + slot) * c.row_words};
    }
    done.x += sum.x;
    done.y += sum.y;
  }
}

// Live pages past the compacted end move into the holes below it, both in
// ascending order.  A thread looks at four adjacent pages; a pool of up to 4096 pages is read
// once, and its holes and movers meet in LDS (40 pages 4.2 us, 1024 pages 5.3 us).
__global__ __launch_bounds__(kPlanThreads) void cache_compact_plan_kernel(Cache c, int32_t* __restrict__ live_out,
                                                                          Plan p) {
  constexpr uint32_t kEach = 4, kBlock = kPlanThreads * kEach;
  __shared__ uint2 lds[kPlanWaves];
  __shared__ int32_t holes[kBlock / 2], movers[kBlock / 2], holders[kBlock / 2];
  const uint32_t tid = threadIdx.x;
  const bool small = c.pages <= kBlock;
  int32_t refs[kEach];
  auto look = [&](uint32_t g0) {
    uint32_t n = 0;
#pragma unroll
    for (uint32_t e = 0; e < kEach; ++e) {
      const uint32_t g = g0 + tid * kEach + e;
      refs[e] = g < c.pages ? c.refs[g] : 0;
      n += refs[e] > 0;
    }
    return n;
  };
  uint32_t mine = 0;
  for (uint32_t g0 = 0; g0 < c.pages; g0 += kBlock) mine += look(g0);
  uint2 total;
  scan(make_uint2(mine, 0), lds, &total);
  const uint32_t live = total.x;
  uint2 done = make_uint2(0, 0);  // holes, movers
  for (uint32_t g0 = 0; g0 < c.pages; g0 += kBlock) {
    if (!small) look(g0);
    uint2 n = make_uint2(0, 0);
#pragma unroll
    for (uint32_t e = 0; e < kEach; ++e) {
      const uint32_t g = g0 + tid * kEach + e;
      n.x += g < live && refs[e] <= 0;
      n.y += g >= live && refs[e] > 0;
    }
    uint2 sum, at = scan(n, lds, &sum);
    at.x += done.x;
    at.y += done.y;
#pragma unroll
    for (uint32_t e = 0; e < kEach; ++e) {
      const uint32_t g = g0 + tid * kEach + e;
      if (g < live && refs[e] <= 0) (small ? holes : p.fresh)[at.x++] = static_cast<int32_t>(g);
      if (g >= live && refs[e] > 0) {
        if (small) holders[at.y] = refs[e];
        (small ? movers : p.movers)[at.y++] = static_cast<int32_t>(g);
      } else if (g < c.pages) {
        p.to[g] = -1;
      }
    }
    done.x += sum.x;
    done.y += sum.y;
  }
  __syncthreads();
  const size_t page_words = c.row_words * c.page_rows;
  for (uint32_t k = tid; k < done.y; k += kPlanThreads) {
    const int32_t from = small ? movers[k] : p.movers[k], to = small ? holes[k] : p.fresh[k];
    const int32_t n = small ? holders[k] : c.refs[from];
    p.moves[k] = {c.pool + from * page_words, c.pool + to * page_words};
    p.to[from] = to;
    c.refs[to] = n;
    c.refs[from] = 0;
  }
  if (tid == 0) {
    *p.moves_n = done.y;
    if (live_out) *live_out = static_cast<int32_t>(live);
  }
}

// One workgroup copies one piece of up to 16 KiB: each byte crosses memory once and is not kept in the
// caches (a gather of 1.3 GB: 6.3 TB/s read and written).
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

// Workgroups of the move kernel: one a piece that there can be, up to 2^20 (then they walk
// the pieces).  1 GiB of moved pages: 6.2 TB/s read and written (a library copy of 4 GiB: 4.7); resident
// workgroups that walk from the start, eight a CU, 5.0.  The host does not know how many rows are copied, so a call that
// copies none pays for workgroups that find nothing, 20 us for 127,000 of them: one row of 1 MiB for each of 64 sequences takes
// 27 us with pages of up to 8 rows (4,096 pieces, up to 32,768 workgroups), 47 us with pages of 32 (131,072);
// a compaction of 1024 pages of 4 MiB that moves none 32 us, ten 39 us.
static uint32_t move_blocks(size_t moves, size_t words) {
  const size_t items = moves * ((words + kPieceWords - 1) / kPieceWords), most = size_t(1) << 20;
  return static_cast<uint32_t>(items < 1 ? 1 : items < most ? items : most);
}

hipError_t launch_cache_append(const Cache& c, const int32_t* seq, const int32_t* row0, uint32_t count,
                               const uint32_t* rows_in, uint32_t rows, int32_t* status, void* workspace,
                               hipStream_t s) {
  Plan p;
  append_layout(c, count, rows, static_cast<uint8_t*>(workspace), &p);
  const auto plan = count <= kPlanThreads ? cache_append_plan_kernel<true> : cache_append_plan_kernel<false>;
  plan<<<1, kPlanThreads, 0, s>>>(c, seq, row0, count, rows_in, rows, status, p);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  cache_move_kernel<<<move_blocks(append_moves(c, count, rows), c.row_words), kMoveThreads, 0, s>>>(
      c, p, c.row_words);
  return hipGetLastError();
}

hipError_t launch_cache_compact(const Cache& c, int32_t* live, void* workspace, hipStream_t s) {
  Plan p;
  compact_layout(c, static_cast<uint8_t*>(workspace), &p);
  cache_compact_plan_kernel<<<1, kPlanThreads, 0, s>>>(c, live, p);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const size_t page_words = c.row_words * c.page_rows;
  cache_move_kernel<<<move_blocks((c.pages + 1) / 2, page_words), kMoveThreads, 0, s>>>(c, p, page_words);
  return hipGetLastError();
}

hipError_t launch_cache_gather(const Cache& c, const int32_t* seq, const int32_t* pos, uint32_t count, uint32_t* out,
                               hipStream_t s) {
  const uint32_t pieces = static_cast<uint32_t>((c.row_words + kPieceWords - 1) / kPieceWords);
  const uint32_t most = pieces < kMostGroups ? kMostGroups / pieces : 1;  // rows of a launch
  for (uint32_t r = 0; r < count;) {
    const uint32_t now = count - r < most ? count - r : most;
    cache_gather_kernel<<<now * pieces, kMoveThreads, 0, s>>>(c, seq + r, pos + r, pieces, out + r * c.row_words);
    if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    r += now;
  }
  return hipSuccess;
}

}  // namespace ckks
