// Eviction from a paged cache by accumulated attention weight.  Of each sequence and head that has more rows than
// `budget`, the first and last few stay, and of the others those with the largest weights; what stays moves together in
// its order, to the first `budget` rows of the sequence's pages, with its weights.
//
// k_evict_pick: weights as unsigned numbers of the same order; the smallest that stays by counts of their upper twelve bits, then,
// of those that share them (few, as a rule: gathered into a list), of the next and the last ten; then the rows that stay, in
// their order: of equal weights the first rows.  A block a sequence and head, which reads its weights once: 32 a thread stay
// in LDS, and only those behind are read in every pass.  A wave holds a run of the rows, so that the list of what stays needs
// the counts of the waves in front and no more barriers.
//
// k_evict_move: rows are moved in place, in chunks of 256, a block a chunk.  Row i of the result comes from row
// kept[i] >= i, so the rows that a chunk overwrites are read by it and by chunks in front of it, no others: a block loads its
// chunk whole, says so, waits until those in front of it that read what it overwrites have said so, and stores.  Chunks are
// numbered as their blocks start, and none waits before it has said that its rows are loaded, so what is waited for is always
// running or done.  Keys and values, and parts of 128 bytes of a row, move independently.  In 8 bits
// a block of the cache gets the smallest power of two for the rows that it now holds, and their codes follow (exact but
// for codes that become subnormal).
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

constexpr int EM_THREADS = 512, EM_PASS = EM_THREADS / 8, EM_N = 4, EM_ROWS = EM_PASS * EM_N;   // 8 lanes a row
static_assert(EM_ROWS >= C8_BLOCK_MOST, "a chunk holds whole blocks");

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
  if (tid == 0) a.count[at] = n;
  // of the chunks to be moved: how many have started, and which are loaded
  const int streams = 2 * a.parts;
  for (int i = tid; i < streams; i += EV_THREADS) a.started[at * streams + i] = 0;
  for (int i = tid; i < streams * a.chunks; i += EV_THREADS) a.loaded[at * streams * a.chunks + i] = 0;
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
  // the bin at which the counts from the top reach `need`, and how many of it do; a thread four bins
  auto find = [&] {
    __syncthreads();
    int c[4], total = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) c[e] = s_hist[EV_BINS - 1 - (4 * tid + e)], total += c[e];
    const int upto = c8_wave_scan(total);
    if (lane == 63) s_same[wave] = upto;
    __syncthreads();
    int above = upto - total;
#pragma unroll
    for (int v = 0; v < EV_WAVES; ++v)
      if (v < wave) above += s_same[v];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if (above < need && need <= above + c[e]) s_found[0] = EV_BINS - 1 - (4 * tid + e), s_found[1] = need - above;
      above += c[e];
    }
    __syncthreads();
    need = s_found[1];
    return (uint32_t)s_found[0];
  };
  // rows that stay for sure, and those with the smallest weight that stays, of which the first `need` do
  uint32_t least = 0xffffffffu;                    // none: behind all of them
  auto kind = [&](auto whole, int j, uint32_t k, unsigned long long& same, unsigned long long& sure) __attribute__((always_inline)) {
    const bool candidate = decltype(whole)::value || is_candidate(j);
    same = __ballot(candidate && k == least);
    sure = __ballot(candidate ? k > least : j < n);
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
      unsigned long long same, sure;
      kind(whole, j, k, same, sure);
      n_same += __popcll(same), n_sure += __popcll(sure);
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
    unsigned long long same, sure;
    kind(whole, j, k, same, sure);
    const int eq = equal + ev_below(same), to = done + ev_below(sure) + min(eq, need);
    const bool stays = (sure >> lane & 1) || ((same >> lane & 1) && eq < need);
    equal += __popcll(same), done += __popcll(sure);
    if (stays) {
      kept[to] = j;
      if (all_held) w_out[to] = ev_weight(k);
    }
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
      // maxima of eight rows each
      const uint32_t top = c8_wave_max(__float_as_uint(__builtin_amdgcn_cvt_pk_f32_fp8(most, false)[0] * c8_two(byte[p])));
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
      const int now = min(max(c8_byte(most), C8_LEAST), 254);
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

int64_t slh_kv_evict_workspace(int32_t B, int32_t H, int32_t d, int32_t dtype, int32_t budget) {
  using namespace slh;
  if (B < 0 || B > (1 << 20) || H < 1 || H > 65535 || d < 1 || d > 256 || budget < 1) return SLH_EINVAL;
  if (dtype != SLH_BF16 && dtype != SLH_F16 && dtype != SLH_F32 && dtype != SLH_E4M3) return SLH_EINVAL;
  const int64_t chunks = ((int64_t)budget + EM_ROWS - 1) / EM_ROWS, streams = 2 * (int64_t)B * H * ev_parts(d, dtype);
  return streams * chunks > (1 << 22) ? SLH_EINVAL : 4 * ((int64_t)B * H + streams * (1 + chunks));
}

int slh_kv_evict(void* k_cache, void* v_cache, void* k_scale, void* v_scale, int32_t dtype, int64_t n_pages, int32_t page_size,
                 int32_t block, int32_t B, int32_t H, int32_t d, const int32_t* page_table, int64_t ld_pages, int32_t max_pages,
                 const int32_t* lens, int32_t* lens_out, const float* weights, float* weights_out, int32_t budget,
                 int32_t first, int32_t last, int32_t* kept, void* workspace, int64_t workspace_bytes, void* stream) {
  using namespace slh;
  const bool e8 = dtype == SLH_E4M3;
  const int64_t need = slh_kv_evict_workspace(B, H, d, dtype, budget);
  if (need < 0 || e8 != (k_scale != nullptr) || e8 != (v_scale != nullptr)) return SLH_EINVAL;
  if (e8 ? d != 64 && d != 80 && d != 96 && d != 128 : d % 8 != 0) return SLH_EINVAL;
  if (page_size < 1 || page_size > 65536 || (page_size & (page_size - 1))) return SLH_EINVAL;
  if (n_pages < 1 || n_pages > INT32_MAX || n_pages * H > INT32_MAX / page_size) return SLH_EINVAL;
  if (e8 && !c8_sizes_ok(n_pages, page_size, H, block)) return SLH_EINVAL;
  if (max_pages < 0 || ld_pages < max_pages || (int64_t)max_pages * page_size > INT32_MAX / 4) return SLH_EINVAL;
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
  a.count = (int*)workspace, a.started = a.count + (int64_t)B * H, a.loaded = a.started + 2 * (int64_t)B * H * a.parts;
  a.B = B, a.budget = budget, a.first = first, a.last = last;
  // a sequence is cut to `budget` only if the table holds more
  a.chunks = (int)(((int64_t)std::min(budget, a.max_rows) + EM_ROWS - 1) / EM_ROWS);
  const dim3 pairs((unsigned)(B * H)), blocks((unsigned)(B * H * 2 * a.parts * std::max(1, a.chunks)));
  hipStream_t s = (hipStream_t)stream;
  (void)hipGetLastError();
  // 4 KB of LDS for 1024 rows; the smaller kernel leaves room for a second block on a compute unit
  if (a.max_rows <= 8 * EV_THREADS)
    hipLaunchKernelGGL(k_evict_pick<8>, pairs, dim3(EV_THREADS), 0, s, a);
  else
    hipLaunchKernelGGL(k_evict_pick<32>, pairs, dim3(EV_THREADS), 0, s, a);
  if (hipGetLastError() != hipSuccess) return SLH_EHIP;
  if (e8)
    hipLaunchKernelGGL(k_evict_move<true>, blocks, dim3(EM_THREADS), 0, s, a);
  else
    hipLaunchKernelGGL(k_evict_move<false>, blocks, dim3(EM_THREADS), 0, s, a);
  return hipGetLastError() == hipSuccess ? SLH_OK : SLH_EHIP;
}

}  // extern "C"
