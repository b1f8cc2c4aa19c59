// Eviction from a paged cache by accumulated attention weight.  Of each sequence and head that has more rows than
// `budget`, the first and last few stay, and of the others those with the largest weights; what stays moves together in
// its order, to the first `budget` rows of the sequence's pages, with its weights.
//
// k_evict_pick: the smallest weight that stays by four counts of eight bits each, from the top (weights as unsigned
// numbers of the same order), then one pass in the order of the rows that lists what stays: of equal weights
// the first rows.  A block a sequence and head.
//
// k_evict_move: rows are moved in place.  Row i of the result comes from row kept[i] >= i, so that a block which
// takes the rows of a sequence and head in order, a chunk at a time, never overwrites what a later chunk reads: it loads a
// chunk whole, waits for all its loads, and stores.  Blocks share nothing: keys and values, and parts of 128 bytes of
// a row, move independently.  In 8 bits a block of the cache gets the smallest power of two for the rows that it now
// holds, and their codes follow (exact but for codes that become subnormal).
#include "cache8.h"

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
  int B, budget, first, last;
};

// Order of weights as unsigned numbers: NaN the largest, zeros equal.
__device__ __forceinline__ uint32_t ev_key(float w) {
  if (w != w) return 0xffffffffu;
  const uint32_t u = __float_as_uint(w + 0.f);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}

constexpr int EV_THREADS = 1024;

__global__ __launch_bounds__(EV_THREADS) void k_evict_pick(EvictArgs a) {
  __shared__ int s_hist[256];
  __shared__ int s_wave[EV_THREADS / 64];
  __shared__ uint32_t s_found[2];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int64_t at = blockIdx.x;
  const int b = (int)(at / a.H);
  const int n = min(max(a.lens[b], 0), a.max_rows);
  const float* const w = a.w + at * a.max_rows;
  float* const w_out = a.w_out + at * a.max_rows;
  int* const kept = a.kept + at * a.budget;
  if (tid == 0) a.count[at] = n;
  if (n <= a.budget) {
    for (int i = tid; i < a.budget; i += EV_THREADS) kept[i] = i < n ? i : -1;
    for (int i = tid; i < a.max_rows; i += EV_THREADS) w_out[i] = i < n ? w[i] : 0.f;
    return;
  }
  // candidates: rows [lo, hi), of which `need` stay
  const int lo = a.first, hi = n - a.last;
  int need = a.budget - a.first - a.last;
  uint32_t prefix = 0;
  for (int shift = 24; shift >= 0; shift -= 8) {
    if (tid < 256) s_hist[tid] = 0;
    __syncthreads();
    for (int j = lo + tid; j < hi; j += EV_THREADS) {
      const uint32_t k = ev_key(w[j]);
      if (shift == 24 || (k >> (shift + 8)) == (prefix >> (shift + 8))) atomicAdd(&s_hist[(k >> shift) & 255], 1);
    }
    __syncthreads();
    // the byte at which the counts from the top reach `need`
    if (wave == 0) {
      int c[4], total = 0;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        c[e] = s_hist[255 - (4 * lane + e)];
        total += c[e];
      }
      int above = c8_wave_scan(total) - total;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        if (above < need && need <= above + c[e]) s_found[0] = 255 - (4 * lane + e), s_found[1] = need - above;
        above += c[e];
      }
      if (need == 0 && lane == 0) s_found[0] = 255, s_found[1] = 0;
    }
    __syncthreads();
    prefix |= s_found[0] << shift;
    need = (int)s_found[1];
  }
  // rows above the smallest weight that stays, and the first `need` of those equal to it
  int done = 0, equal = 0;
  for (int j0 = 0; j0 < n; j0 += EV_THREADS) {
    const int j = j0 + tid;
    const float x = j < n ? w[j] : 0.f;
    const uint32_t k = ev_key(x);
    const bool candidate = j >= lo && j < hi;
    const bool same = candidate && k == prefix, sure = j < n && (!candidate || k > prefix);
    const unsigned long long m_same = __ballot(same), m_sure = __ballot(sure);
    if (lane == 0) s_wave[wave] = __popcll(m_same) << 16 | __popcll(m_sure);
    __syncthreads();
    int before = 0, total = 0;
#pragma unroll
    for (int v = 0; v < EV_THREADS / 64; ++v) {
      const int c = s_wave[v];
      if (v < wave) before += c;
      total += c;
    }
    const unsigned long long below = (1ull << lane) - 1;
    const int eq = equal + (before >> 16) + __popcll(m_same & below);
    // equal rows in front that stay: the first `need`
    const int to = done + (before & 0xffff) + __popcll(m_sure & below) + min(eq, need) - min(equal, need);
    if (sure || (same && eq < need)) {
      kept[to] = j;
      w_out[to] = x;
    }
    done += (total & 0xffff) + min(equal + (total >> 16), need) - min(equal, need);
    equal += total >> 16;
    __syncthreads();
  }
  for (int i = a.budget + tid; i < a.max_rows; i += EV_THREADS) w_out[i] = 0.f;
}

constexpr int EM_THREADS = 512, EM_PASS = EM_THREADS / 8, EM_N = 4, EM_ROWS = EM_PASS * EM_N;   // 8 lanes a row
static_assert(EM_ROWS >= C8_BLOCK_MOST, "a chunk holds whole blocks");

// Address of a row of the cache, in rows; pages that lie outside are not reached: -1.
__device__ __forceinline__ int64_t ev_line(const EvictArgs& a, const int* list, int h, int row) {
  const int page = list[row >> a.lg_page];
  if ((unsigned)page >= (unsigned)a.n_pages) return -1;
  return (((int64_t)page * a.H + h) << a.lg_page) + (row & ((1 << a.lg_page) - 1));
}

template <bool E8>
__global__ __launch_bounds__(EM_THREADS) void k_evict_move(EvictArgs a, int parts) {
  __shared__ uint32_t s_top[2][EM_N][EM_THREADS / 64];
  const int tid = threadIdx.x, r = tid >> 3;
  int x = blockIdx.x;
  const int part = x % parts;
  x /= parts;
  const int kv = x & 1;
  x >>= 1;
  const int64_t at = x;
  const int b = (int)(at / a.H), h = (int)(at - (int64_t)b * a.H);
  const int n = a.count[at];
  if (part == 0 && kv == 0 && h == 0 && tid == 0) a.lens_out[b] = min(n, a.budget);
  if (n <= a.budget) return;
  const int* const list = a.pages + b * a.ld_pages;
  const int* const kept = a.kept + at * a.budget;
  uint8_t* const cache = (uint8_t*)a.cache[kv];
  const int col = 128 * part + 16 * (tid & 7);
  const bool in_row = col < a.row_bytes;
  for (int i0 = 0; i0 < a.budget; i0 += EM_ROWS) {
    uint4 v[EM_N];
    int byte[EM_N];
    int64_t to[EM_N];
    uint32_t top[EM_N];
#pragma unroll
    for (int p = 0; p < EM_N; ++p) {
      const int i = i0 + p * EM_PASS + r;
      v[p] = make_uint4(0, 0, 0, 0), byte[p] = C8_LEAST, to[p] = -1, top[p] = 0;
      if (i >= a.budget) continue;
      const int j = kept[i];
      const int64_t from = ev_line(a, list, h, j);
      to[p] = ev_line(a, list, h, i);
      if (from >= 0 && in_row) v[p] = *(const uint4*)(cache + from * a.row_bytes + col);
      if (E8 && from >= 0) byte[p] = a.two[kv][from >> a.lg_block];
    }
    if constexpr (E8) {
#pragma unroll
      for (int p = 0; p < EM_N; ++p) {
        const uint32_t c[4] = {v[p].x, v[p].y, v[p].z, v[p].w};
        uint32_t most = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e)
#pragma unroll
          for (int s = 0; s < 32; s += 8) {
            const uint32_t code = (c[e] >> s) & 0x7fu;
            if (code != 0x7fu) most = max(most, code);
          }
        top[p] = c8_wave_max(__float_as_uint(__builtin_amdgcn_cvt_pk_f32_fp8(most, false)[0] * c8_two(byte[p])));
      }
    }
    // every load of the chunk has landed before the first of its rows is written
#pragma unroll
    for (int p = 0; p < EM_N; ++p) asm volatile("" : "+v"(v[p].x), "+v"(v[p].y), "+v"(v[p].z), "+v"(v[p].w), "+v"(byte[p]));
    if constexpr (E8) {
      // maxima of eight rows each, two buffers so that one barrier a chunk does
      uint32_t(&tops)[EM_N][EM_THREADS / 64] = s_top[(i0 / EM_ROWS) & 1];
      if ((tid & 63) == 0)
#pragma unroll
        for (int p = 0; p < EM_N; ++p) tops[p][tid >> 6] = top[p];
      __syncthreads();
      const uint32_t* const all = &tops[0][0];
      const int lg = a.lg_block - 3;               // eights of rows of a block
#pragma unroll
      for (int p = 0; p < EM_N; ++p) {
        const int g8 = (p * EM_PASS + r) >> 3;
        uint32_t most = 0;
        for (int e = (g8 >> lg) << lg; e < ((g8 >> lg) + 1) << lg; ++e) most = max(most, all[e]);
        if (to[p] < 0) continue;
        const int now = min(max(c8_byte(most), C8_LEAST), 254);
        const float by = c8_two(127 + min(max(byte[p] - now, -126), 127));
        const uint4 y = make_uint4(c8_rescaled(v[p].x, by), c8_rescaled(v[p].y, by), c8_rescaled(v[p].z, by), c8_rescaled(v[p].w, by));
        if (in_row) *(uint4*)(cache + to[p] * a.row_bytes + col) = y;
        if (((i0 + p * EM_PASS + r) & ((1 << a.lg_block) - 1)) == 0 && (tid & 7) == 0) a.two[kv][to[p] >> a.lg_block] = (uint8_t)now;
      }
    } else {
      __syncthreads();
#pragma unroll
      for (int p = 0; p < EM_N; ++p)
        if (to[p] >= 0 && in_row) *(uint4*)(cache + to[p] * a.row_bytes + col) = v[p];
    }
  }
}

}  // namespace slh

extern "C" {

int64_t slh_kv_evict_workspace(int32_t B, int32_t H) {
  if (B < 0 || B > (1 << 20) || H < 1 || H > 65535 || (int64_t)B * H > (1 << 23)) return SLH_EINVAL;
  return 4 * (int64_t)B * H;
}

int slh_kv_evict(void* k_cache, void* v_cache, void* k_scale, void* v_scale, int32_t dtype, int64_t n_pages, int32_t page_size,
                 int32_t block, int32_t B, int32_t H, int32_t d, const int32_t* page_table, int64_t ld_pages, int32_t max_pages,
                 const int32_t* lens, int32_t* lens_out, const float* weights, float* weights_out, int32_t budget,
                 int32_t first, int32_t last, int32_t* kept, void* workspace, int64_t workspace_bytes, void* stream) {
  using namespace slh;
  const bool e8 = k_scale || v_scale;
  if (!e8 && dtype != SLH_BF16 && dtype != SLH_F16 && dtype != SLH_F32) return SLH_EINVAL;
  const int64_t need = slh_kv_evict_workspace(B, H);
  if (need < 0) return SLH_EINVAL;
  if (e8 ? d != 64 && d != 80 && d != 96 && d != 128 : d < 8 || d > 256 || d % 8 != 0) return SLH_EINVAL;
  if (page_size < 1 || page_size > 65536 || (page_size & (page_size - 1))) return SLH_EINVAL;
  if (n_pages < 1 || n_pages > INT32_MAX || n_pages * H > INT32_MAX / page_size) return SLH_EINVAL;
  if (e8 && (!k_scale || !v_scale || !c8_sizes_ok(n_pages, page_size, H, block))) return SLH_EINVAL;
  if (max_pages < 0 || ld_pages < max_pages || (int64_t)max_pages * page_size > INT32_MAX / 4) return SLH_EINVAL;
  if (budget < 1 || first < 0 || last < 0 || (int64_t)first + last > budget) return SLH_EINVAL;
  if (B == 0) return SLH_OK;
  if (((uintptr_t)k_cache | (uintptr_t)v_cache) % 16 != 0 || !k_cache || !v_cache || !lens || !lens_out || !kept ||
      (max_pages > 0 && (!page_table || !weights || !weights_out)))
    return SLH_EINVAL;
  if (!workspace || ((uintptr_t)workspace) % 16 != 0 || workspace_bytes < need) return SLH_EINVAL;
  EvictArgs a = {};
  a.cache[0] = k_cache, a.cache[1] = v_cache;
  a.two[0] = (uint8_t*)k_scale, a.two[1] = (uint8_t*)v_scale;
  a.row_bytes = d * (e8 ? 1 : dtype == SLH_F32 ? 4 : 2);
  a.n_pages = (int)n_pages, a.H = H, a.lg_page = __builtin_ctz((unsigned)page_size);
  a.lg_block = e8 ? __builtin_ctz((unsigned)block) : 0;
  a.pages = page_table, a.ld_pages = ld_pages, a.max_rows = max_pages * page_size;
  a.lens = lens, a.lens_out = lens_out, a.w = weights, a.w_out = weights_out, a.kept = kept, a.count = (int*)workspace;
  a.B = B, a.budget = budget, a.first = first, a.last = last;
  const int parts = e8 ? 1 : (a.row_bytes + 127) / 128;
  hipStream_t s = (hipStream_t)stream;
  (void)hipGetLastError();
  hipLaunchKernelGGL(k_evict_pick, dim3((unsigned)(B * H)), dim3(EV_THREADS), 0, s, a);
  if (hipGetLastError() != hipSuccess) return SLH_EHIP;
  const dim3 grid((unsigned)(B * H * 2 * parts));
  if (e8)
    hipLaunchKernelGGL((k_evict_move<true>), grid, dim3(EM_THREADS), 0, s, a, parts);
  else
    hipLaunchKernelGGL((k_evict_move<false>), grid, dim3(EM_THREADS), 0, s, a, parts);
  return hipGetLastError() == hipSuccess ? SLH_OK : SLH_EHIP;
}

}  // extern "C"
