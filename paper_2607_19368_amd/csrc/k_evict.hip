// Eviction from a paged cache by accumulated attention weight.  Of each sequence and head that has more rows than
// `budget`, the first and last few stay, and of the others those with the largest weights; what stays moves together in
// its order, to the first `budget` rows of the sequence's pages, with its weights.
//
// k_evict_pick: weights as unsigned numbers of the same order; the smallest that stays by counts of their upper twelve bits, then,
// of those that share them (few, as a rule: gathered into a list), of the next and the last ten; then the rows that stay, in
// their order: of equal weights the first rows.  A block a sequence and head, which reads its weights once: 32 a thread stay
// in LDS, and only those behind are read in every pass.  A wave holds a run of the rows, so that the list of what stays needs
// the counts of the waves in front and no more barriers.  Bound by latency where rows are few (8 sequences of 97 rows, 4 heads:
// 8 us) and by its one compute unit where they are many: 16384 rows 22 us, of which the counts, one LDS atomic a row, and the
// list take most.
//
// k_evict_count, k_evict_gather, k_evict_list: the same for few long sequences, several blocks each: counts of a run; from all
// counts the bin, and a run's rows in it and above; from all runs' rows in the bin the smallest that stays, then a run's
// rows behind those of the runs in front.  Integers throughout, so that the order in which blocks run does not show.  48
// sequences and heads of up to 49157 rows: 8 + 10 + 18 us, where one block each takes 71.
//
// k_evict_move: rows are moved in place, in chunks of 256, a block a chunk.  Row i of the result comes from row
// kept[i] >= i, so the rows that a chunk overwrites are read by it and by chunks in front of it, no others: a block loads its
// chunk whole, says so, waits until those in front of it that read what it overwrites have said so, and stores.  Chunks are
// numbered as their blocks start, and none waits before it has said that its rows are loaded, so what is waited for is always
// running or done.  Keys and values, and parts of 128 bytes of a row, move independently: 300 MB read and written in 82 us, 3.7
// TB/s of the 4.7 of a plain copy; a row is 128 bytes in 8 bits, and what stays lies scattered.  In 8 bits
// a block of the cache gets the smallest power of two for the rows that it now holds, and their codes follow (exact but
// for codes that become subnormal).
#include "attend_plan.h"
#include "cache8.h"

#include <algorithm>
#include <type_traits>

namespace slh {

struct EvictArgs {
  void* cache[2];          // [n_pages][H][page] rows of `row_bytes`
  uint8_t* two[2];         // 8 bits: [n_pages][H][page / block]
  int row_bytes;
  int n_pages, H, lg_page, lg_block;
  const int* pages;        // [B][ld_pages]
  int64_t ld_pages;
  int max_rows;
  const int* lens;
  int* lens_out;
  const float* w;          // [B][H][max_rows]
  float* w_out;
  int* kept;               // [B][H][budget]
  int* count;              // [B][H] rows before
  int* started;            // [streams] chunks whose blocks have started
  int* loaded;             // [streams][chunks] whether a chunk has been loaded
  int B, budget, first, last;
  int parts, chunks;       // of 128 bytes of a row; of EM_ROWS rows of the result
  // where several blocks pick of one sequence and head:
  int runs;                // blocks of a pair
  uint32_t* key;           // [B][H][max_rows] weights as numbers
  uint32_t* same;          // [B][H][max_rows] by run: those that share the upper bits of the smallest that stays
  int* hist;               // [B][H][runs][EV_BINS]
  int* found;              // [B][H][runs][2] of a run: rows that stay for sure by the upper bits, entries of `same`
};

// Order of weights as unsigned numbers: NaN the largest, zeros equal.
__device__ __forceinline__ uint32_t ev_key(float w) {
  if (w != w) return 0xffffffffu;
  const uint32_t u = __float_as_uint(w + 0.f);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}
// and back
__device__ __forceinline__ float ev_weight(uint32_t k) { return __uint_as_float(k & 0x80000000u ? k ^ 0x80000000u : ~k); }

// lanes below this one of a mask
__device__ __forceinline__ int ev_below(unsigned long long m) {
  return __builtin_amdgcn_mbcnt_hi((uint32_t)(m >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)m, 0));
}

constexpr int EV_THREADS = 1024, EV_WAVES = EV_THREADS / 64;
constexpr int EV_BINS = 4096, EV_LIST = 1024;
constexpr int EV_LEAST = 2, EV_RUNS = 8, EV_HELD = 16;     // rows of a thread where several blocks pick; blocks of a pair at most

constexpr int EM_THREADS = 512, EM_PASS = EM_THREADS / 8, EM_N = 4, EM_ROWS = EM_PASS * EM_N;   // 8 lanes a row
static_assert(EM_ROWS >= C8_BLOCK_MOST, "a chunk holds whole blocks");

// Of a wave's 64 rows those stay that are `in`, and of the equal ones the first: `need` in all, `equal` before; f(at) for each,
// at: four bytes times its place behind `done` (fewer than 2^31; 32 bits beside a base that the wave shares).
template <class F>
__device__ __forceinline__ void ev_keep(bool in, bool eq, int need, int& done, int& equal, F&& f) {
  const unsigned long long sure = __ballot(in), same = __ballot(eq);
  if (__builtin_expect(same != 0, 0)) {
    const int before = equal + ev_below(same);
    if (in || (eq && before < need)) f(4u * (uint32_t)(done + ev_below(sure) + min(before, need)));
    equal += __popcll(same);
  } else if (in) {
    f(4u * (uint32_t)(done + min(equal, need) + ev_below(sure)));
  }
  done += __popcll(sure);
}

// What k_evict_move starts from: rows before; of the chunks to be moved how many have started, and which are loaded.
__device__ __forceinline__ void ev_start(const EvictArgs& a, int64_t at, int n, int i0, int step) {
  if (i0 == 0) a.count[at] = n;
  const int streams = 2 * a.parts;
  for (int i = i0; i < streams; i += step) a.started[at * streams + i] = 0;
  for (int i = i0; i < streams * a.chunks; i += step) a.loaded[at * streams * a.chunks + i] = 0;
}

// The bin at which the counts from the top reach `need`, which becomes how many of that bin stay; a thread four bins.
__device__ __forceinline__ uint32_t ev_find(const int* hist, int* scan, int* found, int& need) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  __syncthreads();
  int c[4], total = 0;
#pragma unroll
  for (int e = 0; e < 4; ++e) c[e] = hist[EV_BINS - 1 - (4 * tid + e)], total += c[e];
  const int upto = c8_wave_scan(total);
  if (lane == 63) scan[wave] = upto;
  __syncthreads();
  int above = upto - total;
#pragma unroll
  for (int v = 0; v < EV_WAVES; ++v)
    if (v < wave) above += scan[v];
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    if (above < need && need <= above + c[e]) found[0] = EV_BINS - 1 - (4 * tid + e), found[1] = need - above;
    above += c[e];
  }
  __syncthreads();
  need = found[1];
  return (uint32_t)found[0];
}

// LDS: weights of a thread that stay in LDS.
template <int LDS>
__global__ __launch_bounds__(EV_THREADS) void k_evict_pick(EvictArgs a) {
  __shared__ uint32_t s_key[LDS * EV_THREADS];
  __shared__ int s_hist[EV_BINS];
  __shared__ int s_same[EV_WAVES], s_sure[EV_WAVES];
  __shared__ int s_found[2], s_listed;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int64_t at = blockIdx.x;
  const int b = (int)(at / a.H);
  const int n = min(max(a.lens[b], 0), a.max_rows);
  const float* const w = a.w + at * a.max_rows;
  float* const w_out = a.w_out + at * a.max_rows;
  int* const kept = a.kept + at * a.budget;
  ev_start(a, at, n, tid, EV_THREADS);
  if (n <= a.budget) {
    for (int i = tid; i < a.budget; i += EV_THREADS) kept[i] = i < n ? i : -1;
    for (int i = tid; i < a.max_rows; i += EV_THREADS) w_out[i] = i < n ? w[i] : 0.f;
    return;
  }
  // rows of this wave, 64 at a time
  const int steps = (n + EV_THREADS - 1) / EV_THREADS, in_lds = min(steps, LDS), row0 = wave * steps * 64 + lane;
  // past the end the last again: a load under a branch would be waited for in it
  auto key_of = [&](int i) {
    const float x = w[min(row0 + 64 * i, n - 1)];
    return row0 + 64 * i < n ? ev_key(x) : 0u;
  };
  // candidates: rows [lo, lo + m), of which `need` stay
  const int lo = a.first, m = n - a.last - lo;
  int need = a.budget - a.first - a.last;
  auto is_candidate = [&](int j) { return (unsigned)(j - lo) < (unsigned)m; };
  // f(whole, row, weight) for this wave's rows; whole: all 64 are candidates
  auto one = [&](auto&& f, int i, uint32_t k) __attribute__((always_inline)) {
    const int first = wave * steps * 64 + 64 * i;
    if (first >= lo && first + 63 < lo + m)
      f(std::true_type{}, row0 + 64 * i, k);
    else
      f(std::false_type{}, row0 + 64 * i, k);
  };
  auto each = [&](auto&& f) __attribute__((always_inline)) {
#pragma unroll 4
    for (int i = 0; i < in_lds; ++i) one(f, i, s_key[i * EV_THREADS + tid]);
    for (int i0 = LDS; i0 < steps; i0 += 8) {
      uint32_t k[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) k[e] = key_of(min(i0 + e, steps - 1));
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (i0 + e < steps) one(f, i0 + e, k[e]);
    }
  };
  auto clear = [&] {
    for (int i = tid; i < EV_BINS; i += EV_THREADS) s_hist[i] = 0;
    __syncthreads();
  };
  auto find = [&] { return ev_find(s_hist, s_same, s_found, need); };
  // rows that stay for sure, and those with the smallest weight that stays, of which the first `need` do
  uint32_t least = 0xffffffffu;                    // none: behind all of them
  auto is_sure = [&](auto whole, int j, uint32_t k) __attribute__((always_inline)) {
    return decltype(whole)::value || is_candidate(j) ? k > least : j < n;
  };
  auto is_same = [&](auto whole, int j, uint32_t k) __attribute__((always_inline)) {
    return (decltype(whole)::value || is_candidate(j)) && k == least;
  };
  clear();
  auto take = [&](int i, uint32_t k) __attribute__((always_inline)) {
    if (i < LDS) s_key[i * EV_THREADS + tid] = k;
    one([&](auto whole, int j, uint32_t) {
      if (decltype(whole)::value || is_candidate(j)) atomicAdd(&s_hist[k >> 20], 1);
    }, i, k);
  };
  for (int i0 = 0; i0 < steps; i0 += 8) {
    uint32_t k[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) k[e] = key_of(min(i0 + e, steps - 1));
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (i0 + e < steps) take(i0 + e, k[e]);
  }
  int n_same = 0, n_sure = 0;                      // of this wave
  bool short_list = false;
  if (need > 0) {
    const uint32_t top = find();
    // those that share the upper bits: into a list in the place of the counts' upper half, key and wave, or, where they are
    // too many, all rows are gone through again
    if (tid == 0) s_listed = 0;
    __syncthreads();
    uint32_t* const listed = (uint32_t*)s_hist + EV_BINS - 2 * EV_LIST;
    each([&](auto whole, int j, uint32_t k) {
      const bool candidate = decltype(whole)::value || is_candidate(j), in = candidate && k >> 20 == top;
      n_sure += __popcll(__ballot(candidate ? k >> 20 > top : j < n));
      const unsigned long long who = __ballot(in);
      if (!who) return;
      int to = 0;
      if (lane == 0) to = atomicAdd(&s_listed, __popcll(who));
      to = __builtin_amdgcn_readfirstlane(to) + ev_below(who);
      if (in && to < EV_LIST) listed[to] = k, listed[EV_LIST + to] = wave;
    });
    if (lane == 0) s_sure[wave] = n_sure;
    __syncthreads();
    const int many = s_listed;
    short_list = many <= EV_LIST;
    uint32_t mine[EV_LIST / EV_THREADS], of[EV_LIST / EV_THREADS];
#pragma unroll
    for (int e = 0; e < EV_LIST / EV_THREADS; ++e) {
      const bool there = short_list && tid + e * EV_THREADS < many;
      mine[e] = there ? listed[tid + e * EV_THREADS] : 0;
      of[e] = there ? listed[EV_LIST + tid + e * EV_THREADS] : 0;
    }
    __syncthreads();
    uint32_t prefix = top << 20;
#pragma unroll 1
    for (int shift = 10; shift >= 0; shift -= 10) {
      const uint32_t above = ~0u << (shift + 10);
      clear();
      if (short_list) {
#pragma unroll
        for (int e = 0; e < EV_LIST / EV_THREADS; ++e)
          if (tid + e * EV_THREADS < many && (mine[e] & above) == prefix) atomicAdd(&s_hist[mine[e] >> shift & 1023], 1);
      } else {
        each([&](auto, int j, uint32_t k) {
          if (is_candidate(j) && (k & above) == prefix) atomicAdd(&s_hist[k >> shift & 1023], 1);
        });
      }
      prefix |= find() << shift;
    }
    least = prefix;
    __syncthreads();
    if (short_list) {                              // of the list, by the waves whose rows they are
      if (tid < EV_WAVES) s_same[tid] = 0;
      __syncthreads();
#pragma unroll
      for (int e = 0; e < EV_LIST / EV_THREADS; ++e)
        if (tid + e * EV_THREADS < many && mine[e] >= least) atomicAdd(mine[e] > least ? &s_sure[of[e]] : &s_same[of[e]], 1);
    }
  }
  if (!short_list) {
    n_sure = 0;
    each([&](auto whole, int j, uint32_t k) {
      n_same += __popcll(__ballot(is_same(whole, j, k))), n_sure += __popcll(__ballot(is_sure(whole, j, k)));
    });
    __syncthreads();
    if (lane == 0) s_same[wave] = n_same, s_sure[wave] = n_sure;
  }
  __syncthreads();
  int equal = 0, done = 0;
#pragma unroll
  for (int v = 0; v < EV_WAVES; ++v)
    if (v < wave) equal += s_same[v], done += s_sure[v];
  // weights_out may be the weights: where not all are held, rows are listed first then, and their weights moved a chunk at a
  // time, a chunk's loads before its stores
  const bool all_held = steps <= LDS || a.w != a.w_out;
  each([&](auto whole, int j, uint32_t k) {
    const bool in = is_sure(whole, j, k), eq = is_same(whole, j, k);
    ev_keep(in, eq, need, done, equal, [&](uint32_t at) {
      *(int*)((char*)kept + at) = j;
      if (all_held) *(float*)((char*)w_out + at) = ev_weight(k);
    });
  });
  if (!all_held) {
    __threadfence_block();
    __syncthreads();
    constexpr int N = 4;
    for (int i0 = 0; i0 < a.budget; i0 += N * EV_THREADS) {
      float x[N];
#pragma unroll
      for (int e = 0; e < N; ++e) x[e] = i0 + e * EV_THREADS + tid < a.budget ? w[kept[i0 + e * EV_THREADS + tid]] : 0.f;
#pragma unroll
      for (int e = 0; e < N; ++e) asm volatile("" : "+v"(x[e]));
      __syncthreads();
#pragma unroll
      for (int e = 0; e < N; ++e)
        if (i0 + e * EV_THREADS + tid < a.budget) w_out[i0 + e * EV_THREADS + tid] = x[e];
    }
  }
  __syncthreads();
  for (int i = a.budget + tid; i < a.max_rows; i += EV_THREADS) w_out[i] = 0.f;
}

// ---- several blocks a sequence and head: a run of the rows each ----
struct EvRun {
  int64_t at;              // pair
  int n, run, steps;       // rows of the pair; this block's run, 64 rows a wave and step
  int begin;               // its first row
};
__device__ __forceinline__ EvRun ev_run(const EvictArgs& a) {
  EvRun r;
  r.at = blockIdx.x / a.runs, r.run = (int)(blockIdx.x - r.at * a.runs);
  r.n = min(max(a.lens[r.at / a.H], 0), a.max_rows);
  r.steps = max(EV_LEAST, (int)(((int64_t)r.n + a.runs * EV_THREADS - 1) / (a.runs * EV_THREADS)));
  r.begin = (int)min((int64_t)r.n, (int64_t)r.run * r.steps * EV_THREADS);
  return r;
}
__device__ __forceinline__ int ev_run_begin(const EvRun& r, int run) { return (int)min((int64_t)r.n, (int64_t)run * r.steps * EV_THREADS); }

// The rows of a run, whose waves hold runs in turn.  The first EV_HELD of a thread are loaded together, before anything else
// (in order behind stores they would be waited for with these), and stay in registers; those behind (only where a run has
// more than 16384 rows) are loaded eight at a time in each pass.
struct EvRows {
  const uint32_t* from;
  int first, row0;         // of the wave, of the thread
  uint32_t held[EV_HELD];
  __device__ __forceinline__ EvRows(const EvRun& r, const uint32_t* x) : from(x) {
    first = r.begin + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) * r.steps * 64, row0 = first + (threadIdx.x & 63);
#pragma unroll
    for (int e = 0; e < EV_HELD; ++e) held[e] = at(r, e);
  }
  __device__ __forceinline__ uint32_t at(const EvRun& r, int i) const {   // past the end the last row
    return from[min((int64_t)row0 + 64 * (int64_t)min(i, r.steps - 1), (int64_t)r.n - 1)];
  }
  // f(whole, row, value); whole: all 64 of the wave's step are candidates, rows [lo, lo + m)
  template <class F>
  __device__ __forceinline__ void each(const EvRun& r, int lo, int m, F&& f) const {
    auto one = [&](int i, uint32_t k) __attribute__((always_inline)) {
      if (first + 64 * i >= lo && first + 64 * i + 63 < lo + m)
        f(std::true_type{}, row0 + 64 * i, k);
      else
        f(std::false_type{}, row0 + 64 * i, k);
    };
#pragma unroll
    for (int e = 0; e < EV_HELD; ++e)
      if (e < r.steps && first + 64 * e < r.n) one(e, held[e]);
    for (int i0 = EV_HELD; i0 < r.steps && first + 64 * i0 < r.n; i0 += 8) {
      uint32_t k[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) k[e] = at(r, i0 + e);
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (i0 + e < r.steps) one(i0 + e, k[e]);
    }
  }
};

// counts of the upper twelve bits, and the weights as numbers: weights_out may be the weights
__global__ __launch_bounds__(EV_THREADS) void k_evict_count(EvictArgs a) {
  __shared__ int s_hist[EV_BINS];
  const int tid = threadIdx.x;
  const EvRun r = ev_run(a);
  ev_start(a, r.at, r.n, r.run * EV_THREADS + tid, a.runs * EV_THREADS);
  if (r.begin >= r.n) return;
  const EvRows rows(r, (const uint32_t*)(a.w + r.at * a.max_rows));
  for (int i = tid; i < EV_BINS; i += EV_THREADS) s_hist[i] = 0;
  __syncthreads();
  const int lo = a.first, m = r.n - a.last - lo;
  uint32_t* const key = a.key + r.at * a.max_rows;
  rows.each(r, lo, m, [&](auto whole, int j, uint32_t x) {
    const uint32_t k = ev_key(__uint_as_float(x));
    if (decltype(whole)::value || j < r.n) key[j] = k;
    if (decltype(whole)::value || (unsigned)(j - lo) < (unsigned)m) atomicAdd(&s_hist[k >> 20], 1);
  });
  __syncthreads();
  int4* const to = (int4*)(a.hist + (r.at * a.runs + r.run) * EV_BINS);
  for (int i = tid; i < EV_BINS / 4; i += EV_THREADS) to[i] = ((const int4*)s_hist)[i];
}

// The bin in which the smallest that stays lies, and `need` as by ev_find.
__device__ __forceinline__ uint32_t ev_top(const EvictArgs& a, const EvRun& r, int* hist, int* scan, int* found, int& need) {
  static_assert(EV_BINS == 4 * EV_THREADS, "four bins a thread");
  int4 sum = make_int4(0, 0, 0, 0);
  const int4* const from = (const int4*)(a.hist + r.at * a.runs * EV_BINS) + threadIdx.x;
  const int runs = (int)(((int64_t)r.n + r.steps * EV_THREADS - 1) / (r.steps * EV_THREADS));
#pragma unroll 4
  for (int v = 0; v < runs; ++v) {
    const int4 x = from[v * EV_THREADS];
    sum.x += x.x, sum.y += x.y, sum.z += x.z, sum.w += x.w;
  }
  ((int4*)hist)[threadIdx.x] = sum;
  return ev_find(hist, scan, found, need);
}

// a run's candidates in that bin, in any order, and its rows that stay for sure
__global__ __launch_bounds__(EV_THREADS) void k_evict_gather(EvictArgs a) {
  __shared__ int s_hist[EV_BINS];
  __shared__ int s_scan[EV_WAVES], s_found[2], s_listed, s_sure;
  const int tid = threadIdx.x, lane = tid & 63;
  const EvRun r = ev_run(a);
  int need = a.budget - a.first - a.last;
  if (r.begin >= r.n || r.n <= a.budget || need == 0) return;
  const EvRows rows(r, a.key + r.at * a.max_rows);
  if (tid == 0) s_listed = 0, s_sure = 0;
  const uint32_t top = ev_top(a, r, s_hist, s_scan, s_found, need);
  const int lo = a.first, m = r.n - a.last - lo;
  uint32_t* const same = a.same + r.at * a.max_rows + r.begin;
  int n_sure = 0;
  rows.each(r, lo, m, [&](auto whole, int j, uint32_t k) {
    const bool candidate = decltype(whole)::value || (unsigned)(j - lo) < (unsigned)m, in = candidate && k >> 20 == top;
    n_sure += __popcll(__ballot(candidate ? k >> 20 > top : j < r.n));
    const unsigned long long who = __ballot(in);
    if (!who) return;
    int to = 0;
    if (lane == 0) to = atomicAdd(&s_listed, __popcll(who));
    to = __builtin_amdgcn_readfirstlane(to) + ev_below(who);
    if (in) same[to] = k;
  });
  if (lane == 0 && n_sure) atomicAdd(&s_sure, n_sure);
  __syncthreads();
  if (tid < 2) a.found[(r.at * a.runs + r.run) * 2 + tid] = tid ? s_listed : s_sure;
}

// the smallest that stays, from all runs' lists; a run's rows that stay, behind those of the runs in front of it
__global__ __launch_bounds__(EV_THREADS) void k_evict_list(EvictArgs a) {
  __shared__ int s_hist[EV_BINS];
  __shared__ int s_scan[EV_WAVES], s_found[2], s_front[2], s_same[EV_WAVES], s_sure[EV_WAVES];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const EvRun r = ev_run(a);
  const float* const w = a.w + r.at * a.max_rows;
  float* const w_out = a.w_out + r.at * a.max_rows;
  int* const kept = a.kept + r.at * a.budget;
  const int i0 = r.run * EV_THREADS + tid, step = a.runs * EV_THREADS;
  if (r.n <= a.budget) {
    for (int i = i0; i < a.budget; i += step) kept[i] = i < r.n ? i : -1;
    for (int i = i0; i < a.max_rows; i += step) w_out[i] = i < r.n ? w[i] : 0.f;
    return;
  }
  auto clear = [&] {
    for (int i = a.budget + i0; i < a.max_rows; i += step) w_out[i] = 0.f;
  };
  if (r.begin >= r.n) return clear();
  const int lo = a.first, m = r.n - a.last - lo;
  const EvRows rows(r, a.key + r.at * a.max_rows);
  int need = a.budget - a.first - a.last;
  uint32_t least = 0xffffffffu;                    // none: behind all of them
  int done = 0, equal = 0;                         // rows in front of the run that stay for sure, and that are equal to the least
  if (need > 0) {
    const uint32_t top = ev_top(a, r, s_hist, s_scan, s_found, need);
    const int runs = (int)(((int64_t)r.n + r.steps * EV_THREADS - 1) / (r.steps * EV_THREADS));
    const int* const found = a.found + r.at * a.runs * 2;
    // f(value) for what the runs' lists hold: the first of a thread of each are loaded together, and stay in registers
    int many[EV_RUNS];
    uint32_t held[EV_RUNS];
#pragma unroll
    for (int v = 0; v < EV_RUNS; ++v) many[v] = found[2 * min(v, runs - 1) + 1];
#pragma unroll
    for (int v = 0; v < EV_RUNS; ++v)
      held[v] = a.same[r.at * a.max_rows + ev_run_begin(r, min(v, runs - 1)) + min(tid, max(many[v] - 1, 0))];
    auto lists = [&](int upto, auto&& f) {
#pragma unroll
      for (int v = 0; v < EV_RUNS; ++v) {
        if (v >= upto) break;
        if (tid < many[v]) f(held[v]);
        const uint32_t* const list = a.same + r.at * a.max_rows + ev_run_begin(r, v);
        for (int i = tid + EV_THREADS; i < many[v]; i += EV_THREADS) f(list[i]);
      }
    };
    uint32_t prefix = top << 20;
#pragma unroll 1
    for (int shift = 10; shift >= 0; shift -= 10) {
      const uint32_t above = ~0u << (shift + 10);
      for (int i = tid; i < EV_BINS; i += EV_THREADS) s_hist[i] = 0;
      __syncthreads();
      lists(runs, [&](uint32_t k) {
        if ((k & above) == prefix) atomicAdd(&s_hist[k >> shift & 1023], 1);
      });
      prefix |= ev_find(s_hist, s_scan, s_found, need) << shift;
    }
    least = prefix;
    if (tid < 2) s_front[tid] = 0;
    __syncthreads();
    int more = 0, same = 0;                        // lane 0's are the wave's: it has an entry where any lane has
    lists(r.run, [&](uint32_t k) { more += __popcll(__ballot(k > least)), same += __popcll(__ballot(k == least)); });
    if (lane == 0 && more) atomicAdd(&s_front[0], more);
    if (lane == 0 && same) atomicAdd(&s_front[1], same);
    __syncthreads();
    done = s_front[0], equal = s_front[1];
    for (int v = 0; v < r.run; ++v) done += found[2 * v];
  } else {
    done = min(r.begin, a.first) + max(0, r.begin - (r.n - a.last));
  }
  auto is_candidate = [&](int j) { return (unsigned)(j - lo) < (unsigned)m; };
  auto is_sure = [&](auto whole, int j, uint32_t k) __attribute__((always_inline)) {
    return decltype(whole)::value || is_candidate(j) ? k > least : j < r.n;
  };
  auto is_same = [&](auto whole, int j, uint32_t k) __attribute__((always_inline)) {
    return (decltype(whole)::value || is_candidate(j)) && k == least;
  };
  int n_same = 0, n_sure = 0;
  rows.each(r, lo, m, [&](auto whole, int j, uint32_t k) {
    n_same += __popcll(__ballot(is_same(whole, j, k))), n_sure += __popcll(__ballot(is_sure(whole, j, k)));
  });
  if (lane == 0) s_same[wave] = n_same, s_sure[wave] = n_sure;
  __syncthreads();
#pragma unroll
  for (int v = 0; v < EV_WAVES; ++v)
    if (v < wave) equal += s_same[v], done += s_sure[v];
  rows.each(r, lo, m, [&](auto whole, int j, uint32_t k) {
    const bool in = is_sure(whole, j, k), eq = is_same(whole, j, k);
    ev_keep(in, eq, need, done, equal, [&](uint32_t at) {
      *(int*)((char*)kept + at) = j;
      *(float*)((char*)w_out + at) = ev_weight(k);
    });
  });
  clear();
}

// Blocks that pick of a sequence and head: as many as find a compute unit each, where a table holds so many rows that three
// launches and what passes between them cost less than one block's time.  One block and several, whole calls (budget 512, 8 to 64
// sequences and heads): 8192 rows 30-32 and 37-44 us, 16384 rows 40-41 and 41-47, 49152 rows 74-77 and 47-59, 131072 rows 230-243
// and 61-88; 128 sequences and heads, two blocks each: 49152 rows 81 and 72; 256: 91 and 111.
inline int ev_runs(int64_t pairs, int64_t max_rows) {
  if (max_rows <= 16 * EV_THREADS || pairs < 1) return 1;
  return (int)std::max<int64_t>(1, std::min<int64_t>(EV_RUNS, attend_cus() / pairs));
}

inline int ev_row_bytes(int d, int dtype) { return d * (dtype == SLH_E4M3 ? 1 : dtype == SLH_F32 ? 4 : 2); }
inline int ev_parts(int d, int dtype) { return (ev_row_bytes(d, dtype) + 127) / 128; }

// Address of a row of the cache, in rows; pages that lie outside are not reached: -1.
__device__ __forceinline__ int64_t ev_line(const EvictArgs& a, const int* list, int h, int row) {
  const int page = list[row >> a.lg_page];
  if ((unsigned)page >= (unsigned)a.n_pages) return -1;
  return (((int64_t)page * a.H + h) << a.lg_page) + (row & ((1 << a.lg_page) - 1));
}

typedef unsigned short ev_u16x2 __attribute__((ext_vector_type(2)));

template <bool E8>
__global__ __launch_bounds__(EM_THREADS) void k_evict_move(EvictArgs a) {
  __shared__ uint32_t s_top[EM_N][EM_THREADS / 64];
  __shared__ int s_chunk;
  const int tid = threadIdx.x, r = tid >> 3;
  // streams of chunks: (sequence, head, keys or values, part of a row); the first chunks of all come first
  const int streams = a.B * a.H * 2 * a.parts, stream = blockIdx.x % streams;
  const int part = stream % a.parts, kv = stream / a.parts & 1;
  const int64_t at = stream / (2 * a.parts);
  const int b = (int)(at / a.H), h = (int)(at - (int64_t)b * a.H);
  const int n = a.count[at];
  if (stream % (2 * a.parts * a.H) == 0 && (int)blockIdx.x < streams && tid == 0) a.lens_out[b] = min(n, a.budget);
  if (n <= a.budget) return;
  int chunk = 0;
  if (a.chunks > 1) {
    if (tid == 0) s_chunk = __hip_atomic_fetch_add(a.started + stream, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    __syncthreads();
    chunk = __builtin_amdgcn_readfirstlane(s_chunk);
  }
  const int* const list = a.pages + b * a.ld_pages;
  const int* const kept = a.kept + at * a.budget;
  uint8_t* const cache = (uint8_t*)a.cache[kv];
  const int col = 128 * part + 16 * (tid & 7), i0 = chunk * EM_ROWS;
  const bool in_row = col < a.row_bytes;
  uint4 v[EM_N];
  int byte[EM_N];
  int64_t to[EM_N];
  int source[EM_N];
#pragma unroll
  for (int p = 0; p < EM_N; ++p) source[p] = i0 + p * EM_PASS + r < a.budget ? kept[i0 + p * EM_PASS + r] : -1;
#pragma unroll
  for (int p = 0; p < EM_N; ++p) {
    v[p] = make_uint4(0, 0, 0, 0), byte[p] = C8_LEAST, to[p] = -1;
    if (source[p] < 0) continue;
    const int64_t from = ev_line(a, list, h, source[p]);
    to[p] = ev_line(a, list, h, i0 + p * EM_PASS + r);
    if (from >= 0 && in_row) v[p] = *(const uint4*)(cache + from * a.row_bytes + col);
    if (E8 && from >= 0) byte[p] = a.two[kv][from >> a.lg_block];
  }
  if constexpr (E8) {
#pragma unroll
    for (int p = 0; p < EM_N; ++p) {
      const uint32_t c[4] = {v[p].x, v[p].y, v[p].z, v[p].w};
      ev_u16x2 pair = {0, 0};
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        pair = __builtin_elementwise_max(pair, __builtin_bit_cast(ev_u16x2, c[e] & 0x007f007fu));
        pair = __builtin_elementwise_max(pair, __builtin_bit_cast(ev_u16x2, c[e] >> 8 & 0x007f007fu));
      }
      uint32_t most = max((uint32_t)pair[0], (uint32_t)pair[1]);
      if (most == 0x7fu) {                         // NaN codes are left out
        most = 0;
        for (int e = 0; e < 4; ++e)
          for (int s = 0; s < 32; s += 8) most = max(most, (c[e] >> s & 0x7fu) == 0x7fu ? 0u : c[e] >> s & 0x7fu);
      }
      // Maxima of eight rows each, of code 2^byte by its bits with 2^127 more than a value's, which pass neither end of 32 bits
      // (exponents up to 135 + 254) as values would that of fp32.
      const uint32_t top = c8_wave_max(most ? __float_as_uint(__builtin_amdgcn_cvt_pk_f32_fp8(most, false)[0]) + ((uint32_t)byte[p] << 23) : 0u);
      if ((tid & 63) == 0) s_top[p][tid >> 6] = top;
    }
  }
  // every load of this wave has landed, and, behind the barrier, of the block
#pragma unroll
  for (int p = 0; p < EM_N; ++p) asm volatile("" : "+v"(v[p].x), "+v"(v[p].y), "+v"(v[p].z), "+v"(v[p].w), "+v"(byte[p]));
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
  if (a.chunks > 1) {
    int* const loaded = a.loaded + (int64_t)stream * a.chunks;
    if (tid == 0) __hip_atomic_store(loaded + chunk, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    if (tid < 64) {
      for (int c0 = chunk - 1;; c0 -= 64) {
        // chunk c reads rows up to kept[its last row]: those that reach this chunk's are waited for
        const int c = c0 - tid;
        const bool reads = c >= 0 && kept[(c + 1) * EM_ROWS - 1] >= i0;
        while (__ballot(reads && __hip_atomic_load(loaded + c, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == 0))
          __builtin_amdgcn_s_sleep(2);
        if (~__ballot(reads)) break;
      }
    }
    __syncthreads();
  }
  if constexpr (E8) {
    const uint32_t* const all = &s_top[0][0];
    const int lg = a.lg_block - 3;               // eights of rows of a block
#pragma unroll
    for (int p = 0; p < EM_N; ++p) {
      const int g8 = (p * EM_PASS + r) >> 3;
      uint32_t most = 0;
      for (int e = (g8 >> lg) << lg; e < ((g8 >> lg) + 1) << lg; ++e) most = max(most, all[e]);
      if (to[p] < 0) continue;
      const int now = min(max(c8_byte(most) - 127, C8_LEAST), 254);
      const float by = c8_two(127 + min(max(byte[p] - now, -126), 127));
      uint4 y = v[p];
      if (byte[p] != now) y = make_uint4(c8_rescaled(y.x, by), c8_rescaled(y.y, by), c8_rescaled(y.z, by), c8_rescaled(y.w, by));
      if (in_row) *(uint4*)(cache + to[p] * a.row_bytes + col) = y;
      if (((p * EM_PASS + r) & ((1 << a.lg_block) - 1)) == 0 && (tid & 7) == 0) a.two[kv][to[p] >> a.lg_block] = (uint8_t)now;
    }
  } else {
#pragma unroll
    for (int p = 0; p < EM_N; ++p)
      if (to[p] >= 0 && in_row) *(uint4*)(cache + to[p] * a.row_bytes + col) = v[p];
  }
}

}  // namespace slh

extern "C" {

int64_t slh_kv_evict_workspace(int32_t B, int32_t H, int32_t d, int32_t dtype, int32_t budget, int64_t max_len) {
  using namespace slh;
  if (B < 0 || B > (1 << 20) || H < 1 || H > 65535 || d < 1 || d > 256 || budget < 1) return SLH_EINVAL;
  if (max_len < 0 || max_len > INT32_MAX / 4) return SLH_EINVAL;
  if (dtype != SLH_BF16 && dtype != SLH_F16 && dtype != SLH_F32 && dtype != SLH_E4M3) return SLH_EINVAL;
  const int64_t chunks = ((int64_t)budget + EM_ROWS - 1) / EM_ROWS, streams = 2 * (int64_t)B * H * ev_parts(d, dtype);
  if (streams * chunks > (1 << 22)) return SLH_EINVAL;
  const int64_t pairs = (int64_t)B * H, runs = ev_runs(pairs, max_len);
  return 4 * (pairs + streams * (1 + chunks)) + (runs > 1 ? 4 * pairs * (runs * (EV_BINS + 2) + 2 * max_len) : 0);
}

int slh_kv_evict(void* k_cache, void* v_cache, void* k_scale, void* v_scale, int32_t dtype, int64_t n_pages, int32_t page_size,
                 int32_t block, int32_t B, int32_t H, int32_t d, const int32_t* page_table, int64_t ld_pages, int32_t max_pages,
                 const int32_t* lens, int32_t* lens_out, const float* weights, float* weights_out, int32_t budget,
                 int32_t first, int32_t last, int32_t* kept, void* workspace, int64_t workspace_bytes, void* stream) {
  using namespace slh;
  const bool e8 = dtype == SLH_E4M3;
  if (max_pages < 0 || page_size < 1) return SLH_EINVAL;
  const int64_t need = slh_kv_evict_workspace(B, H, d, dtype, budget, (int64_t)max_pages * page_size);
  if (need < 0 || e8 != (k_scale != nullptr) || e8 != (v_scale != nullptr)) return SLH_EINVAL;
  if (e8 ? d != 64 && d != 80 && d != 96 && d != 128 : d % 8 != 0) return SLH_EINVAL;
  if (page_size > 65536 || (page_size & (page_size - 1))) return SLH_EINVAL;
  if (n_pages < 1 || n_pages > INT32_MAX || n_pages * H > INT32_MAX / page_size) return SLH_EINVAL;
  if (e8 && !c8_sizes_ok(n_pages, page_size, H, block)) return SLH_EINVAL;
  if (ld_pages < max_pages) return SLH_EINVAL;
  if (first < 0 || last < 0 || (int64_t)first + last > budget) return SLH_EINVAL;
  if (B == 0) return SLH_OK;
  if (((uintptr_t)k_cache | (uintptr_t)v_cache) % 16 != 0 || !k_cache || !v_cache || !lens || !lens_out || !kept ||
      (max_pages > 0 && (!page_table || !weights || !weights_out)))
    return SLH_EINVAL;
  if (!workspace || ((uintptr_t)workspace) % 16 != 0 || workspace_bytes < need) return SLH_EINVAL;
  EvictArgs a = {};
  a.cache[0] = k_cache, a.cache[1] = v_cache;
  a.two[0] = (uint8_t*)k_scale, a.two[1] = (uint8_t*)v_scale;
  a.row_bytes = ev_row_bytes(d, dtype), a.parts = ev_parts(d, dtype);
  a.n_pages = (int)n_pages, a.H = H, a.lg_page = __builtin_ctz((unsigned)page_size);
  a.lg_block = e8 ? __builtin_ctz((unsigned)block) : 0;
  a.pages = page_table, a.ld_pages = ld_pages, a.max_rows = max_pages * page_size;
  a.lens = lens, a.lens_out = lens_out, a.w = weights, a.w_out = weights_out, a.kept = kept;
  const int64_t n_pairs = (int64_t)B * H;
  a.runs = ev_runs(n_pairs, a.max_rows);
  a.hist = (int*)workspace;
  a.key = (uint32_t*)(a.hist + (a.runs > 1 ? n_pairs * a.runs * EV_BINS : 0));
  a.same = a.key + (a.runs > 1 ? n_pairs * a.max_rows : 0);
  a.found = (int*)(a.same + (a.runs > 1 ? n_pairs * a.max_rows : 0));
  a.count = a.found + (a.runs > 1 ? n_pairs * a.runs * 2 : 0), a.started = a.count + (int64_t)B * H, a.loaded = a.started + 2 * (int64_t)B * H * a.parts;
  a.B = B, a.budget = budget, a.first = first, a.last = last;
  // a sequence is cut to `budget` only if the table holds more
  a.chunks = (int)(((int64_t)std::min(budget, a.max_rows) + EM_ROWS - 1) / EM_ROWS);
  const dim3 pairs((unsigned)(B * H)), blocks((unsigned)(B * H * 2 * a.parts * std::max(1, a.chunks)));
  hipStream_t s = (hipStream_t)stream;
  (void)hipGetLastError();
  if (a.runs > 1) {
    const dim3 all((unsigned)(B * H * a.runs));
    hipLaunchKernelGGL(k_evict_count, all, dim3(EV_THREADS), 0, s, a);
    hipLaunchKernelGGL(k_evict_gather, all, dim3(EV_THREADS), 0, s, a);
    hipLaunchKernelGGL(k_evict_list, all, dim3(EV_THREADS), 0, s, a);
  } else if (a.max_rows <= 8 * EV_THREADS) {
    // 4 KB of LDS for 1024 rows; the smaller kernel leaves room for a second block on a compute unit
    hipLaunchKernelGGL(k_evict_pick<8>, pairs, dim3(EV_THREADS), 0, s, a);
  } else {
    hipLaunchKernelGGL(k_evict_pick<32>, pairs, dim3(EV_THREADS), 0, s, a);
  }
  if (hipGetLastError() != hipSuccess) return SLH_EHIP;
  if (e8)
    hipLaunchKernelGGL(k_evict_move<true>, blocks, dim3(EM_THREADS), 0, s, a);
  else
    hipLaunchKernelGGL(k_evict_move<false>, blocks, dim3(EM_THREADS), 0, s, a);
  return hipGetLastError() == hipSuccess ? SLH_OK : SLH_EHIP;
}

}  // extern "C"
