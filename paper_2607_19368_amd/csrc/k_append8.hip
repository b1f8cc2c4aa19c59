// New keys (normed, rotated) and values into a paged cache held in 8 bits (cache8.h).
//
// Of a block of rows of a page and head, with new rows x:
//   2^k the smallest power with max |x| <= 448 2^k, and at least the block's own where earlier rows of the
//   sequence are in it; codes e4m3(x 2^-k), to nearest even; the earlier rows' codes times 2^(old - k)
// Infinities and NaN are left out of the maximum and become NaN (e4m3 has no infinities).  The largest power (of
// which 240-folds are used at most, a sixteenth below what the type holds) keeps every value in the type's range.
//
// A unit of work is the block of one key or value head: a wave for each 16 of its rows, the rows in registers from the
// load to the codes, so that each is read once.  The new rows of a sequence are contiguous, so
// no two units share a block and there are no atomics.  Arithmetic in fp32; x 2^-k is exact, so that the codes are rounded
// once.
//
// Bound by the latency from cu and lens through the page table to the rows where tokens are few (61 sequences, one token
// each: 6 us), else by memory: 16384 tokens of 8 heads of 128 (fp16 read, codes written, 109 MB) 31 us, 3.5 TB/s (fp32, 176 MB: 42, 4.2); a
// unit's loads all go out before the first is looked at, which is 4 us of that.
#include "cache8.h"
#include "rope_rows.h"

namespace slh {

struct Append8Args {
  const void* x[2];          // keys and values: element (t, h, e) at t st + h sh + e
  int64_t st[2], sh[2];
  const void* w;             // [d] norm weights of the keys, NULL: no norm
  RopeForm form;
  const int* pos;            // [T]
  uint8_t* cache[2];         // [pages][H][page][d]
  uint8_t* two[2];           // [pages][H][page / block]
  int n_pages, H, lg_page, lg_block;
  const int* pages;          // [B][ld_pages]
  int64_t ld_pages;
  int max_pages;
  const int *lens, *cu;      // [B], [B + 1] (NULL: n_each tokens a sequence)
  int B, n_each;
  int64_t T, unit0, units;   // units [unit0, units) are this launch's
};

template <int DT, int LPR, int WPU>
__global__ __launch_bounds__(WPU < 4 ? 256 : 64 * WPU) void k_append8(Append8Args a) {
  typedef typename RpType<DT>::elem elem;
  constexpr int WAVES = WPU < 4 ? 4 : WPU, UNITS = WAVES / WPU;
  constexpr int RPI = 64 / LPR, IT = 16 / RPI;                  // rows of a wave at a time
  constexpr int MOST = DT == SLH_F16 ? C8_MOST_F16 : C8_MOST;
  __shared__ uint32_t s_top[WAVES];
  __shared__ int s_old[UNITS];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int strip = wave % WPU, mine = wave / WPU;
  const int64_t unit = a.unit0 + (int64_t)blockIdx.x * UNITS + mine;
  const int kv = (int)(unit & 1);
  const int64_t x = unit >> 1;
  int at = (int)(x / a.H);
  const int h = (int)(x - (int64_t)at * a.H);

  // the sequence and block of task `at`: blocks that a sequence's new rows touch, counted by 64 lanes at a time
  const int most = a.max_pages << a.lg_page;
  bool real = false;
  int b = 0, begin = 0, end = 0, row0 = 0, tok_end = 0;
  if (unit < a.units) {
    for (int b0 = 0; b0 < a.B; b0 += 64) {
      // lanes past the last sequence read its entries and have no blocks; loads under a branch would wait in it, one by one
      const int s = min(b0 + lane, a.B - 1);
      const int* const cu = a.cu ? a.cu + s : a.lens;
      const int c0 = cu[0], c1 = cu[a.cu ? 1 : 0], len = a.lens[s];
      const int64_t q0 = a.cu ? (int64_t)c0 : (int64_t)s * a.n_each, q1 = a.cu ? (int64_t)c1 : q0 + a.n_each;
      const int t1 = (int)max((int64_t)0, min(q1, a.T)), n = max(0, t1 - (int)max((int64_t)0, min(q0, a.T)));
      const int hi = b0 + lane < a.B ? min(max(len, 0), most) : 0, lo = max(0, hi - n);
      const int count = hi > lo ? ((hi - 1) >> a.lg_block) - (lo >> a.lg_block) + 1 : 0;
      const int upto = c8_wave_scan(count);
      const unsigned long long hit = __ballot(upto > at);
      if (hit) {
        const int l = __builtin_ctzll(hit);
        b = b0 + l;
        begin = __builtin_amdgcn_readlane(lo, l);
        end = __builtin_amdgcn_readlane(hi, l);
        tok_end = __builtin_amdgcn_readlane(t1, l);
        row0 = ((begin >> a.lg_block) + at - __builtin_amdgcn_readlane(upto - count, l)) << a.lg_block;
        real = true;
        break;
      }
      at -= __builtin_amdgcn_readlane(upto, 63);
    }
  }
  // earlier rows of the sequence in the block; the rows themselves are on their way before the page is known
  const int before = real ? max(0, begin - row0) : 0;
  const int page = real ? a.pages[b * a.ld_pages + (row0 >> a.lg_page)] : -1;

  // Every load of the rows goes out before any is looked at: where a lane has nothing to load, it loads the first token's
  // or the first chunk.
  const int p = lane % LPR;
  const RopeLane l = rp_lane(p, kv ? 0 : a.form.rot, a.form.d);
  const int c0 = l.has0 ? 8 * l.c0 : 0, c1 = l.has1 ? 8 * l.c1 : 0;
  RpRaw<DT> raw[IT][2], raw_w[2];
  int at_pos[IT];
  bool is_new[IT];
  const bool turn = !kv && a.form.table, norm = !kv && a.w;
#pragma unroll
  for (int i = 0; i < IT; ++i) {
    const int r = 16 * strip + i * RPI + lane / LPR;
    is_new[i] = real && r >= before && row0 + r < end;
    const int64_t t = is_new[i] ? (int64_t)tok_end - end + row0 + r : 0;
    const elem* src = (const elem*)a.x[kv] + t * a.st[kv] + h * a.sh[kv];
    raw[i][0].load(src + c0), raw[i][1].load(src + c1);
    at_pos[i] = turn ? a.pos[t] : 0;
  }
  if (norm) raw_w[0].load((const elem*)a.w + c0), raw_w[1].load((const elem*)a.w + c1);
  RopeTurn turns[IT];
  if (turn) {
    const RopeLane first = rp_lane(0, a.form.rot, a.form.d);
#pragma unroll
    for (int i = 0; i < IT; ++i) turns[i] = rp_turn_of(a.form, l.pair ? l : first, l.pair ? p : 0, at_pos[i]);
  }
  float x0[IT][8], x1[IT][8];
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < IT; ++i) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      x0[i][e] = is_new[i] && l.has0 ? raw[i][0].get(e) : 0.f;
      x1[i][e] = is_new[i] && l.has1 ? raw[i][1].get(e) : 0.f;
    }
    if (norm) {
      const float inv = rp_inverse<LPR>(a.form, x0[i], x1[i]);
#pragma unroll
      for (int e = 0; e < 8; ++e) x0[i][e] = x0[i][e] * inv * raw_w[0].get(e), x1[i][e] = x1[i][e] * inv * raw_w[1].get(e);
    }
    if (turn && l.pair) rp_turn(a.form, turns[i], x0[i], x1[i]);
    if (is_new[i]) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const uint32_t m0 = __float_as_uint(x0[i][e]) & 0x7fffffffu, m1 = __float_as_uint(x1[i][e]) & 0x7fffffffu;
        if (l.has0 && m0 < 0x7f800000u) top = max(top, m0);
        if (l.has1 && m1 < 0x7f800000u) top = max(top, m1);
      }
    }
  }
  top = c8_wave_max(top);
  real = (unsigned)page < (unsigned)a.n_pages;
  // of the block's first row, in rows of the cache
  const int64_t line = real ? (((int64_t)page * a.H + h) << a.lg_page) + (row0 & ((1 << a.lg_page) - 1)) : 0;
  uint8_t* const cache = a.cache[kv] + line * a.form.d;
  uint8_t* const two = a.two[kv] + (line >> a.lg_block);
  int old;
  if constexpr (WPU > 1) {
    if (lane == 0) s_top[wave] = top;
    // one wave reads the power that it will write
    if (strip == 0 && lane == 0) s_old[mine] = real && before ? *two : 0;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < WPU; ++w) top = max(top, s_top[mine * WPU + w]);
    old = s_old[mine];
  } else {
    old = real && before ? *two : 0;
  }
  if (!real) return;
  old = min(old, 254);
  const int byte = max(min(max(c8_byte(top), C8_LEAST), MOST), old);
  const float limit = byte == MOST ? C8_TOP_LAST : C8_TOP;
  const float down = byte == 254 ? 0x1p-127f : c8_two(254 - byte);
#pragma unroll
  for (int i = 0; i < IT; ++i) {
    const int r = 16 * strip + i * RPI + lane / LPR;
    uint8_t* const dst = cache + (int64_t)r * a.form.d;
    if (r < before) {
      if (byte == old) continue;
      const float by = byte - old < 127 ? c8_two(127 - (byte - old)) : 0.f;
#pragma unroll
      for (int c = 0; c < 2; ++c)
        if (c ? l.has1 : l.has0) {
          uint2* const at8 = (uint2*)(dst + 8 * (c ? l.c1 : l.c0));
          uint2 v = *at8;
          v.x = c8_rescaled(v.x, by), v.y = c8_rescaled(v.y, by);
          *at8 = v;
        }
    } else if (row0 + r < end) {
#pragma unroll
      for (int c = 0; c < 2; ++c)
        if (c ? l.has1 : l.has0) {
          float y[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const float f = c ? x1[i][e] : x0[i][e];
            const bool finite = (__float_as_uint(f) & 0x7fffffffu) < 0x7f800000u;
            y[e] = finite ? fminf(fmaxf(f * down, -limit), limit) : __builtin_nanf("");
          }
          *(uint2*)(dst + 8 * (c ? l.c1 : l.c0)) = make_uint2(c8_codes(y[0], y[1], y[2], y[3]), c8_codes(y[4], y[5], y[6], y[7]));
        }
    }
  }
  if (strip == 0 && lane == 0 && byte != old) *two = (uint8_t)byte;
}

template <int DT, int LPR>
static hipError_t append8_launch(Append8Args a, hipStream_t s) {
  // a launch has fewer than 2^32 threads
  constexpr int64_t MOST = (int64_t)1 << 21;
  auto go = [&](auto kernel, int per_block, int waves) {
    for (a.unit0 = 0; a.unit0 < a.units; a.unit0 += MOST * per_block) {
      const int64_t n = a.units - a.unit0 < MOST * per_block ? a.units - a.unit0 : MOST * per_block;
      hipLaunchKernelGGL(kernel, dim3((unsigned)((n + per_block - 1) / per_block)), dim3(64 * waves), 0, s, a);
    }
  };
  switch (a.lg_block) {
    case 4: go(k_append8<DT, LPR, 1>, 4, 4); break;
    case 5: go(k_append8<DT, LPR, 2>, 2, 4); break;
    case 6: go(k_append8<DT, LPR, 4>, 1, 4); break;
    case 7: go(k_append8<DT, LPR, 8>, 1, 8); break;
    default: go(k_append8<DT, LPR, 16>, 1, 16); break;
  }
  return hipGetLastError();
}

template <int DT>
static hipError_t append8_run(const Append8Args& a, hipStream_t s) {
  return a.form.d == 64 ? append8_launch<DT, 4>(a, s) : append8_launch<DT, 8>(a, s);
}

}  // namespace slh

extern "C" int slh_kv_append_e4m3(const void* k, int64_t k_st, int64_t k_sh, const void* v, int64_t v_st, int64_t v_sh,
                                  int32_t dtype, int64_t T, int32_t B, int32_t H, int32_t d, const void* k_weight, double eps,
                                  const float* table, int64_t n_pos, int32_t rot_dim, const int32_t* pos,
                                  int32_t interleaved, void* k_cache, void* v_cache, void* k_scale, void* v_scale,
                                  int64_t n_pages, int32_t page_size, int32_t block, const int32_t* page_table,
                                  int64_t ld_pages, int32_t max_pages, const int32_t* lens, const int32_t* cu,
                                  void* stream) {
  using namespace slh;
  if (d != 64 && d != 80 && d != 96 && d != 128) return SLH_EINVAL;
  if (!c8_sizes_ok(n_pages, page_size, H, block) || B < 0 || B > (1 << 20)) return SLH_EINVAL;
  if (!rope_common_ok(dtype, T, 2 * (int64_t)H, d, k_weight, nullptr, eps, table, n_pos, rot_dim, pos)) return SLH_EINVAL;
  if (max_pages < 0 || ld_pages < max_pages || (int64_t)max_pages * page_size > INT32_MAX / 4) return SLH_EINVAL;
  if (!cu && (B ? T % B != 0 : T != 0)) return SLH_EINVAL;
  if (T == 0 || B == 0 || max_pages == 0) return SLH_OK;
  if (!rope_rows_ok(k, k_st, k_sh) || !rope_rows_ok(v, v_st, v_sh) || !rope_rows_ok(k_cache, 0, 0) ||
      !rope_rows_ok(v_cache, 0, 0) || !k_scale || !v_scale || !page_table || !lens)
    return SLH_EINVAL;
  Append8Args a = {};
  a.x[0] = k, a.st[0] = k_st, a.sh[0] = k_sh;
  a.x[1] = v, a.st[1] = v_st, a.sh[1] = v_sh;
  a.w = k_weight;
  a.form = RopeForm{d, rot_dim, interleaved != 0, (float)eps, table, n_pos};
  a.pos = pos;
  a.cache[0] = (uint8_t*)k_cache, a.cache[1] = (uint8_t*)v_cache;
  a.two[0] = (uint8_t*)k_scale, a.two[1] = (uint8_t*)v_scale;
  a.n_pages = (int)n_pages, a.H = H, a.lg_page = __builtin_ctz((unsigned)page_size), a.lg_block = __builtin_ctz((unsigned)block);
  a.pages = page_table, a.ld_pages = ld_pages, a.max_pages = max_pages;
  a.lens = lens, a.cu = cu, a.B = B, a.n_each = cu ? 0 : (int)(T / B), a.T = T;
  // blocks touched: at most one for each new row, and two more than what the rows fill for each sequence
  const int64_t tasks = T / block + 2 * (T < B ? T : (int64_t)B);
  a.units = 2 * (int64_t)H * (tasks < T ? tasks : T);
  (void)hipGetLastError();
  hipStream_t s = (hipStream_t)stream;
  const hipError_t e = dtype == SLH_BF16  ? append8_run<SLH_BF16>(a, s)
                       : dtype == SLH_F16 ? append8_run<SLH_F16>(a, s)
                                          : append8_run<SLH_F32>(a, s);
  return e == hipSuccess ? SLH_OK : SLH_EHIP;
}
