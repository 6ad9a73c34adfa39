// Page selection: for every new token and KV head, the pages whose keys could score highest.
//
//   bound(page) = max over the group's query heads of sum_c max(q_c lo_c, q_c hi_c) = max sum_c (q+_c hi_c + q-_c lo_c),
// lo, hi the element-wise minimum and maximum of the page's keys, q+ and q- the query's positive and negative part: no key
// of the page scores more.  The first n_sink and the last n_tail pages that the token sees are always taken, of those
// between the topk with the largest bounds, equal ones towards the lower page.
//
// The selection is exact.  All bounds are computed on the tensor cores in 32 bits, together with the sum of their terms'
// magnitudes, which bounds their error; with the k-th largest of them, t, and an error of e, pages above t + 2e are in and
// those below t - 2e out whatever the errors are.  Only the pages between are evaluated in 64 bits, where a sum of
// products of 16-bit floats does not round unless their exponents span more than about 25 binades, so that the order does
// not depend on how it is split.  Where a bound is infinite (an fp16 key that overflowed), or the sums are too large for
// 32 bits, the magnitudes are not finite or very large, and all pages are evaluated in 64 bits: there a term whose query
// element is 0 counts 0, and a query head whose sum is no number has no say.  (In 32 bits alone, neighbours among thousands of pages swap; 64 bits for all pages took
// 132 us where this takes 30: 236 tokens over 27K of 32 / 8 heads of 64.)
#include <climits>

#include "paged.cuh"

namespace tkphi {

constexpr int kScoreThreads = 256;
constexpr int kScorePages = 128;           // pages of a scoring CTA's round: 8 warps x 2 steps x 8 pages
// Error of a 32-bit bound over the sum of its terms' magnitudes: 2 D / 16 matrix instructions of 17 addends (16 products
// and the running sum), each cut to 24 bits below the largest and rounded once: 16 * 18 * 2^-24 < 2^-15.8 at D = 128.
constexpr float kBoundError = 1.f / 32768.f;

// Token's position and the candidate pages [first, first + n).
struct Candidates {
  int pos, seen, first, n;
};
__device__ __forceinline__ Candidates candidates_of(const PagedProblem& p, int b, int tok) {
  Candidates c;
  c.pos = paged_kv_len(p, b) - paged_q_len(p, b) + (tok - (int)__ldg(p.cu_q + b));
  if (c.pos < 0) c.pos = 0;
  c.seen = (c.pos >> p.page_shift) + 1;
  c.first = p.n_sink < c.seen ? p.n_sink : c.seen;
  const int n = c.seen - p.n_tail - c.first;
  c.n = n > 0 ? n : 0;
  return c;
}

// The larger one; NaN if either is (as the positive NaN).
__device__ __forceinline__ float max_nan(float a, float b) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}

// Bounds of all candidate pages.  A tile of the matrix instruction is 16 query rows x 8 pages; a lane reads 16 bytes of
// its page at a time and uses them as they lie: which of the 16 terms of a step an element is does not matter as long as
// the query's fragment holds its partner there.  Bound: DRAM, the bounds are read once per tile of rows.
template <typename T, int D>
__global__ void __launch_bounds__(kScoreThreads, 2) paged_score_kernel(const __grid_constant__ PagedProblem p) {
  constexpr int CH = D / 32;                 // 16-byte pieces of a lane per bound
  __shared__ int s_find[2];
  __shared__ int s_mag[16], s_min[16], s_max[16];      // per token: largest magnitude; smallest and largest ordered score
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int gp = padded_group(p.group), tpt = kRowTile / gp;         // tokens of a tile
  pdl_wait();
  pdl_launch_next();
  const int h = blockIdx.x % p.hkv, tile = blockIdx.x / p.hkv;
  if (warp == 0) {                           // which sequence, which of its tiles
    int base = 0;
    if (lane == 0) s_find[0] = -1;
    for (int s = 0; s < p.batch; s += 32) {
      const int m = s + lane < p.batch ? paged_q_len(p, s + lane) : 0;
      const int n = m > 0 ? (m + tpt - 1) / tpt : 0, incl = warp_inclusive_scan(n) + base;
      if (incl > tile && incl - n <= tile) { s_find[0] = s + lane; s_find[1] = tile - (incl - n); }
      base = __shfl_sync(0xffffffffu, incl, 31);
      if (base > tile) break;
    }
  } else if (warp == 1 && lane < 16) {
    s_mag[lane] = 0;
    s_min[lane] = INT_MAX;
    s_max[lane] = INT_MIN;
  }
  __syncthreads();
  const int b = s_find[0];
  if (b < 0) return;
  const int tok0 = (int)__ldg(p.cu_q + b) + s_find[1] * tpt, tok_end = (int)__ldg(p.cu_q + b + 1);
  const int n_tok = tok_end - tok0 < tpt ? tok_end - tok0 : tpt;
  // tokens later in the tile see at least as many pages
  const Candidates last = candidates_of(p, b, tok0 + n_tok - 1);
  int j0 = blockIdx.y * kScorePages;
  if (last.n <= p.topk || j0 >= last.n) return;          // all are taken, or none is left for this CTA
  const int n_all = last.n, stride = gridDim.y * kScorePages;
  const int* table = p.table + (size_t)b * p.max_pages + last.first;
  int ids[2];                                // of this round's pages; the next round's are fetched a round ahead
  auto load_ids = [&](int j) {
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      const int x = j + warp * 16 + s * 8 + (lane >> 2);
      ids[s] = x < n_all ? __ldg(table + x) : 0;
    }
  };
  load_ids(j0);

  // ---- query rows as A operands: q+ against hi, q- against lo
  const int r = lane >> 2, kq = lane & 3;
  uint32_t ap[CH][2][4], an[CH][2][4];
#pragma unroll
  for (int half = 0; half < 2; ++half) {
    const int row = r + half * 8, t = row / gp, g = row % gp;
    const bool live = t < n_tok && g < p.group;
    const uint4* q = reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(p.q) + ((size_t)(tok0 + (live ? t : 0)) * p.hq + h * p.group + (live ? g : 0)) * D);
#pragma unroll
    for (int i = 0; i < CH; ++i) {
      const uint4 v = live ? __ldg(q + kq + 4 * i) : make_uint4(0, 0, 0, 0);
      const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        // fragment e & 1 of the step e >> 1: registers half (dims 2k, 2k+1) and 2 + half (the upper eight)
        const uint32_t neg = T::min2(w[e], 0u), pos = T::max2(w[e], 0u);
        ap[i][e >> 1][(e & 1) * 2 + half] = pos;
        an[i][e >> 1][(e & 1) * 2 + half] = neg;
      }
    }
  }
  const uint4* bounds = static_cast<const uint4*>(p.bounds) + (size_t)h * (2 * D / 8) + kq;
  const size_t page_step = (size_t)p.hkv * (2 * D / 8);
  // this thread's rows (two tokens at most) and their candidates; the writers are the first lanes of a group's rows
  const int tA = r / gp, tB = (r + 8) / gp;
  const bool writes = r % gp == 0;
  int nA = 0, nB = 0;
  if (tA < n_tok) nA = candidates_of(p, b, tok0 + tA).n;
  if (tB < n_tok && gp < 16) nB = candidates_of(p, b, tok0 + tB).n;
  if (nA <= p.topk) nA = 0;
  if (nB <= p.topk) nB = 0;
  float* keysA = p.page_scores + ((size_t)(tok0 + tA) * p.hkv + h) * p.key_stride;
  float* keysB = p.page_scores + ((size_t)(tok0 + tB) * p.hkv + h) * p.key_stride;
  float magA = 0.f, magB = 0.f, minA = INFINITY, minB = INFINITY, maxA = -INFINITY, maxB = -INFINITY;
  for (; j0 < n_all; j0 += stride) {
    uint4 lo[2][CH], hi[2][CH];
    bool ok[2];
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      const int phys = ids[s];
      ok[s] = phys >= 0 && phys < p.n_pages;
      if (!ok[s] && kq == 0) atomicExch(p.status, kStatusBadPage);
      const uint4* src = bounds + (ok[s] ? phys : 0) * page_step;
#pragma unroll
      for (int i = 0; i < CH; ++i) { lo[s][i] = __ldg(src + 4 * i); hi[s][i] = __ldg(src + D / 8 + 4 * i); }
    }
    load_ids(j0 + stride);
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      float v[4] = {0.f, 0.f, 0.f, 0.f}, m[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int i = 0; i < CH; ++i) {
        const uint32_t* wl = reinterpret_cast<const uint32_t*>(&lo[s][i]);
        const uint32_t* wh = reinterpret_cast<const uint32_t*>(&hi[s][i]);
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          T::mma(v, ap[i][u], wh[2 * u], wh[2 * u + 1]);
          T::mma(v, an[i][u], wl[2 * u], wl[2 * u + 1]);
          // magnitudes: q+ |hi| and q- (-|lo|)
          T::mma(m, ap[i][u], wh[2 * u] & 0x7fff7fffu, wh[2 * u + 1] & 0x7fff7fffu);
          T::mma(m, an[i][u], wl[2 * u] | 0x80008000u, wl[2 * u + 1] | 0x80008000u);
        }
      }
      // rows of padding repeat nothing of a real row: they must not win
      if (r % gp >= p.group) { v[0] = v[1] = -INFINITY; if (gp < 16) v[2] = v[3] = -INFINITY; }
      if (gp == 16 && 8 + r >= p.group) v[2] = v[3] = -INFINITY;
      for (int o = 4; o < 4 * (gp < 8 ? gp : 8); o <<= 1) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          v[e] = fmaxf(v[e], __shfl_xor_sync(0xffffffffu, v[e], o));
          m[e] = max_nan(m[e], __shfl_xor_sync(0xffffffffu, m[e], o));
        }
      }
      if (gp == 16) {
#pragma unroll
        for (int e = 0; e < 2; ++e) { v[e] = fmaxf(v[e], v[2 + e]); m[e] = max_nan(m[e], m[2 + e]); }
      }
      // a page with a bad id comes last (its lanes hold page r, its results are in lanes of every row)
      const unsigned bad = __ballot_sync(0xffffffffu, !ok[s]);
      const int j = j0 + warp * 16 + s * 8 + 2 * kq;
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        if (bad >> (4 * (2 * kq + e)) & 1u) v[e] = v[2 + e] = -INFINITY;
        if (writes && j + e < nA) {
          keysA[j + e] = v[e];
          magA = max_nan(magA, m[e]); minA = fminf(minA, v[e]); maxA = fmaxf(maxA, v[e]);
        }
        if (writes && j + e < nB) {
          keysB[j + e] = v[2 + e];
          magB = max_nan(magB, m[2 + e]); minB = fminf(minB, v[2 + e]); maxB = fmaxf(maxB, v[2 + e]);
        }
      }
    }
  }
  // each token's largest magnitude and range of scores here (non-negative floats order like their bits, NaN last)
  auto note = [&](int t, float mag, float lo, float hi) {
    atomicMax(&s_mag[t], __float_as_int(mag));
    atomicMin(&s_min[t], (int)(ordered_key(lo + 0.f) ^ 0x80000000u));
    atomicMax(&s_max[t], (int)(ordered_key(hi + 0.f) ^ 0x80000000u));
  };
  if (writes && nA > 0) note(tA, magA, minA, maxA);
  if (writes && nB > 0) note(tB, magB, minB, maxB);
  __syncthreads();
  if (tid < n_tok)
    p.page_mags[((size_t)(tok0 + tid) * p.hkv + h) * gridDim.y + blockIdx.y] =
        make_uint4((unsigned)s_mag[tid], (unsigned)s_min[tid] ^ 0x80000000u, (unsigned)s_max[tid] ^ 0x80000000u, 0u);
}

template <typename K>
__device__ __forceinline__ K shr_key(K x, int s) { return s >= (int)sizeof(K) * 8 ? (K)0 : x >> s; }
__device__ __forceinline__ float ordered_value(uint32_t k) { return __uint_as_float((k >> 31) ? (k & 0x7fffffffu) : ~k); }

constexpr int kPageBins = 2048;
constexpr int kBorder = 512;               // pages between in and out that are ranked directly

// Threshold of the `need` largest of `count` keys: keys above `prefix` (both shifted right by `top`) are taken, of the
// `count` equal to it `need`.
template <typename K>
struct Threshold { K prefix; int top, need, count; };
constexpr int kAllBits = 64;               // passes of any search that is to know every bit

// Whole CTA; the keys that matter are in [mn, mx], smaller ones are passed over.  each(fn) calls fn(key) for this thread's
// keys.  Stops after `passes`, when at most `enough` keys equal the prefix, exactly as many as are needed, or when all bits
// of the keys are known (kAllBits passes at most).  s_hist:
// kPageBins zeros on entry and on return.
template <typename K, int NT, typename Each>
__device__ __forceinline__ Threshold<K> find_threshold(Each each, K mn, K mx, int need, int count, int enough, int passes,
                                                       int* s_hist, int* s_sum, int* s_out) {
  constexpr int BITS = (int)sizeof(K) * 8, W = NT >= 1024 ? 11 : NT >= 512 ? 10 : 9;     // two bins per thread
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  // The keys share all bits above `top`; of those that share `prefix` above it, `need` are still to be taken.  A pass
  // counts them by their next W bits.
  Threshold<K> t;
  const K diff = mn ^ mx;
  t.top = diff == 0 ? 0 : BITS - (sizeof(K) == 8 ? __clzll((long long)diff) : __clz((int)diff));
  t.prefix = shr_key(mx, t.top);
  t.need = need;
  t.count = count;
  for (; passes > 0 && t.top > 0 && t.count > t.need && t.count > enough; --passes) {
    const int width = t.top < W ? t.top : W, shift = t.top - width, bins = 1 << width;
    each([&](K k) {
      if (k >= mn && shr_key(k, t.top) == t.prefix) atomicAdd(&s_hist[(int)(k >> shift) & (bins - 1)], 1);
    });
    __syncthreads();
    // from the largest bin down: thread t owns a run of bins, thread 0 the largest
    const int run = (bins + NT - 1) / NT;
    int mine = 0;
    for (int i = 0; i < run; ++i) {
      const int bin = bins - 1 - (tid * run + i);
      if (bin >= 0) mine += s_hist[bin];
    }
    const int incl = warp_inclusive_scan(mine);
    if (lane == 31) s_sum[warp] = incl;
    __syncthreads();
    int before = incl - mine + __reduce_add_sync(0xffffffffu, lane < warp ? s_sum[lane] : 0);
    if (before < t.need && before + mine >= t.need) {
      for (int i = 0; i < run; ++i) {
        const int bin = bins - 1 - (tid * run + i), n = s_hist[bin];
        if (before + n >= t.need) { s_out[0] = bin; s_out[1] = t.need - before; s_out[2] = n; break; }
        before += n;
      }
    }
    __syncthreads();
    for (int i = tid; i < bins; i += NT) s_hist[i] = 0;
    t.prefix = (t.prefix << width) | (K)s_out[0];
    t.need = s_out[1];
    t.count = s_out[2];
    t.top = shift;
    __syncthreads();
  }
  return t;
}

template <typename T>
__device__ __forceinline__ double to_double(uint32_t w, bool upper) { return (double)(upper ? T::hi(w) : T::lo(w)); }

// Exact bound of one page as an ordered key (whole warp; q: the unit's first query head).
template <typename T, int D>
__device__ __forceinline__ unsigned long long exact_bound(const PagedProblem& p, const uint32_t* q, int phys, int h) {
  constexpr int WPL = D / 64;                // 32-bit words of a lane
  const int lane = threadIdx.x & 31;
  if (phys < 0 || phys >= p.n_pages) return 0ull;
  const uint32_t* lo = static_cast<const uint32_t*>(p.bounds) + ((size_t)phys * p.hkv + h) * D + lane;
  uint32_t wl[WPL], wh[WPL];
#pragma unroll
  for (int i = 0; i < WPL; ++i) { wl[i] = __ldg(lo + 32 * i); wh[i] = __ldg(lo + D / 2 + 32 * i); }
  double best = -INFINITY;
  for (int g0 = 0; g0 < p.group; g0 += 4) {              // four heads at a time: their loads and sums overlap
    uint32_t w[4][WPL];
    double acc[4];
#pragma unroll
    for (int g = 0; g < 4; ++g)
#pragma unroll
      for (int i = 0; i < WPL; ++i) w[g][i] = __ldg(q + (g0 + g < p.group ? g0 + g : g0) * (D / 2) + lane + 32 * i);
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      acc[g] = 0.;
#pragma unroll
      for (int i = 0; i < WPL; ++i)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const double x = to_double<T>(w[g][i], e);
          if (x != 0.) acc[g] = fma(x, to_double<T>(x < 0. ? wl[i] : wh[i], e), acc[g]);      // 0 * inf would be NaN
        }
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1)
#pragma unroll
      for (int g = 0; g < 4; ++g) acc[g] += __shfl_xor_sync(0xffffffffu, acc[g], o);
    best = fmax(best, fmax(fmax(acc[0], acc[1]), fmax(acc[2], acc[3])));
  }
  const unsigned long long x = (unsigned long long)__double_as_longlong(best + 0.0);     // -0 counts as 0
  return (x >> 63) ? ~x : (x | (1ull << 63));
}

// Scores that a selecting CTA keeps in shared memory at most.  What a launch gets goes by its longest sequence; every CTA of
// it goes by what the launch got (its own token may see fewer pages: a shorter sequence, a replay with other lengths).
constexpr int kHeldScores = 40960;
static int held_scores(int n) { return n < 1 ? 4 : n < kHeldScores ? (n + 3) & ~3 : kHeldScores; }

// Exact topk of the unit's pages, one CTA per unit, scores in shared memory (in global memory where there are more).
// Loops are left rolled: the kernel is short enough for instruction fetches to count.
template <typename T, int D, int NT>
__global__ void __launch_bounds__(NT, NT == 256 ? 4 : 1) paged_select_kernel(const __grid_constant__ PagedProblem p) {
  constexpr int NW = NT / 32;
  extern __shared__ __align__(16) uint32_t s_held[];
  __shared__ uint32_t s_bits[kMaxSelectPages / 32];      // the taken pages
  __shared__ int s_hist[kPageBins];
  __shared__ int s_sum[NW], s_out[3];
  __shared__ unsigned long long s_key[kBorder];
  __shared__ int s_page[kBorder], s_phys[kBorder];
  __shared__ int s_border, s_sure;
  __shared__ uint32_t s_mag, s_min, s_max;
  __shared__ unsigned long long s_min64, s_max64;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int unit = blockIdx.x, tok = unit / p.hkv, h = unit % p.hkv;
  // Behind the scoring grid this one starts when all of that has begun, which had waited for everything before it: the
  // call's inputs may be read before the wait, here and in the grid that follows.  As the call's first grid it waits.
  if (!p.scored) pdl_wait();
  pdl_launch_next();
  for (int i = tid; i < kPageBins; i += NT) s_hist[i] = 0;
  if (tid == 0) { s_border = 0; s_sure = 0; s_mag = 0; s_min = ~0u; s_max = 0; s_min64 = ~0ull; s_max64 = 0ull; }
  const int b = paged_seq_of(p, tok);
  const Candidates c = candidates_of(p, b, tok);
  const int* table = p.table + (size_t)b * p.max_pages;
  const int taken = c.n < p.topk ? c.n : p.topk;        // of the candidates
  const int last0 = c.first + c.n;                      // first page of the tail
  const int n_list = c.first + taken + (c.seen - last0);
  const bool search = c.n > p.topk && p.topk > 0;
  int* list = p.page_list + (size_t)unit * p.n_keep;
  int* out = p.page_out ? p.page_out + (size_t)unit * p.n_keep : nullptr;
  __syncthreads();
  pdl_wait();
  const float* scores = p.page_scores + (size_t)unit * p.key_stride;       // (16-byte aligned: the stride is a multiple of 4)
  const bool in_smem = c.n <= p.held;
  uint32_t top_key = 0;                                 // the largest of this thread's keys
  // four scores as keys; those behind the last page as 0, which no score gives
  auto four = [&](const float4& v, int i) {
    return make_uint4(ordered_key(v.x + 0.f), i + 1 < c.n ? ordered_key(v.y + 0.f) : 0u, i + 2 < c.n ? ordered_key(v.z + 0.f) : 0u,
                      i + 3 < c.n ? ordered_key(v.w + 0.f) : 0u);
  };
  if (search) {
    // what the scoring CTAs of this unit that had pages saw: largest magnitude, range of the scores
    const int parts = (c.n + kScorePages - 1) / kScorePages < p.mag_parts ? (c.n + kScorePages - 1) / kScorePages : p.mag_parts;
    uint4 seen = make_uint4(0, ~0u, 0, 0);
    for (int i = tid; i < parts; i += NT) {
      const uint4 x = __ldcg(p.page_mags + (size_t)unit * p.mag_parts + i);
      seen.x = max(seen.x, x.x); seen.y = min(seen.y, x.y); seen.z = max(seen.z, x.z);
    }
#pragma unroll 4
    for (int i = tid * 4; i < c.n; i += NT * 4) {
      const float4 v = __ldcg(reinterpret_cast<const float4*>(scores + i));
      const uint4 k = four(v, i);
      top_key = max(top_key, max(max(k.x, k.y), max(k.z, k.w)));
      if (in_smem) *reinterpret_cast<uint4*>(s_held + i) = k;
    }
    if (warp * 32 < parts) {
      seen.x = __reduce_max_sync(0xffffffffu, seen.x);
      seen.y = __reduce_min_sync(0xffffffffu, seen.y);
      seen.z = __reduce_max_sync(0xffffffffu, seen.z);
      if (lane == 0) { atomicMax(&s_mag, seen.x); atomicMin(&s_min, seen.y); atomicMax(&s_max, seen.z); }
    }
  }
  // the pages that are always taken, and the padding
  for (int i = tid; i < p.n_keep; i += NT) {
    const int page = i < c.first ? i : i < c.first + taken ? (search ? -2 : i) : i < n_list ? last0 + (i - c.first - taken) : -1;
    if (page != -2) {
      list[i] = page < 0 ? -1 : __ldg(table + page);
      if (out) out[i] = page;
    }
  }
  if (!search) return;
  __syncthreads();
  auto keys_of = [&](int i) {
    return in_smem ? *reinterpret_cast<const uint4*>(s_held + i) : four(__ldcg(reinterpret_cast<const float4*>(scores + i)), i);
  };
  const float mag = __uint_as_float(s_mag);
  const bool wide = !(mag < 1e37f);                     // no numbers, or sums that 32 bits may not hold
  if (!wide) {
    // ---- A key that topk of the threads' largest keys reach is a lower end of the search: nearly all keys are below it,
    // and are neither counted nor spread the bins.
    uint32_t floor_key = s_min;
    if (p.topk <= NT / 2 && c.n > 8 * NT) {
      const Threshold<uint32_t> t = find_threshold<uint32_t, NT>([&](auto&& fn) { fn(top_key); }, s_min, s_max, p.topk, NT, 0, 1,
                                                                 s_hist, s_sum, s_out);
      const uint32_t k = t.top >= 32 ? 0u : t.prefix << t.top;
      floor_key = k > s_min ? k : s_min;
    }
    // ---- the threshold up to a few keys: those are ranked in 64 bits, like the ones too close to it to tell
    const Threshold<uint32_t> t = find_threshold<uint32_t, NT>(
        [&](auto&& fn) {
  #pragma unroll 2
          for (int i = tid * 4; i < c.n; i += NT * 4) {
            const uint4 k = keys_of(i);
            if (max(max(k.x, k.y), max(k.z, k.w)) >= floor_key) { fn(k.x); fn(k.y); fn(k.z); fn(k.w); }
          }
        },
        floor_key, s_max, p.topk, c.n, NW, kAllBits, s_hist, s_sum, s_out);
    // (the k-th largest score lies in [prefix, prefix + 1) << top: both ends widen the range)
    const uint32_t k0 = t.top >= 32 ? 0u : t.prefix << t.top, k1 = t.top >= 32 ? ~0u : k0 | ((1u << t.top) - 1u);
    const float e2 = 2.f * kBoundError * 1.01f * mag + 1e-30f;
    float low = ordered_value(k0 > floor_key ? k0 : floor_key) - e2, high = ordered_value(k1 < s_max ? k1 : s_max) + e2;
    if (!(low >= -INFINITY)) low = -INFINITY;             // (ends of the range that are no numbers)
    if (!(high <= INFINITY)) high = INFINITY;
    const uint32_t kl = ordered_key(low), kh = ordered_key(high);
    // ---- in, out, or between: eight lanes of four pages make a word of the bit map
    int above = 0;
    for (int i0 = warp * 128; i0 < c.n; i0 += NT * 4) {
      const int i = i0 + lane * 4;
      const uint4 k = i < c.n ? keys_of(i) : make_uint4(0, 0, 0, 0);
      const unsigned in = (k.x > kh ? 1u : 0u) | (k.y > kh ? 2u : 0u) | (k.z > kh ? 4u : 0u) | (k.w > kh ? 8u : 0u);
      const unsigned word = __reduce_or_sync(0xffu << (lane & 24), in << (4 * (lane & 7)));
      if ((lane & 7) == 0 && i < c.n) s_bits[i >> 5] = word;
      above += __popc(in);
      if (max(max(k.x, k.y), max(k.z, k.w)) >= kl) {
        const uint32_t kk[4] = {k.x, k.y, k.z, k.w};
  #pragma unroll
        for (int e = 0; e < 4; ++e)
          if (kk[e] <= kh && kk[e] >= kl) {
            const int at = atomicAdd(&s_border, 1);
            if (at < kBorder) { s_page[at] = i + e; s_phys[at] = __ldg(table + c.first + i + e); }
          }
      }
      __syncwarp();
    }
    above = __reduce_add_sync(0xffffffffu, above);
    if (lane == 0 && above) atomicAdd(&s_sure, above);
    __syncthreads();
  }
  const int border = s_border, need = p.topk - s_sure;
  const uint32_t* q = static_cast<const uint32_t*>(p.q) + ((size_t)tok * p.hq + h * p.group) * (D / 2);
  // many equal bounds, or nothing known from 32 bits: the whole list in 64 bits
  if (wide || border > kBorder) {
    unsigned long long* exact = p.page_keys + (size_t)unit * p.key_stride;
    for (int j = warp; j < c.n; j += NW) {
      const unsigned long long k = exact_bound<T, D>(p, q, __ldg(table + c.first + j), h);
      if (lane == 0) {
        exact[j] = k;
        atomicMin(&s_min64, k);
        atomicMax(&s_max64, k);
      }
    }
    __syncthreads();
    const Threshold<unsigned long long> t64 = find_threshold<unsigned long long, NT>(
        [&](auto&& fn) { for (int j = tid; j < c.n; j += NT) fn(__ldcg(exact + j)); }, s_min64, s_max64, p.topk, c.n, 0, kAllBits,
        s_hist, s_sum, s_out);
    // keys above the prefix, and the first t64.need of those equal to it: counted over the words by one warp
    for (int j0 = warp * 32; j0 < c.n; j0 += NT) {
      const unsigned long long x = j0 + lane < c.n ? shr_key(__ldcg(exact + j0 + lane), t64.top) : 0ull;
      const unsigned in = __ballot_sync(0xffffffffu, j0 + lane < c.n && x > t64.prefix);
      if (lane == 0) s_bits[j0 >> 5] = in;
    }
    __syncthreads();
    if (warp == 0) {
      int left = t64.need;
      for (int j0 = 0; j0 < c.n && left > 0; j0 += 32) {
        const unsigned eq = __ballot_sync(0xffffffffu, j0 + lane < c.n && shr_key(__ldcg(exact + (j0 + lane < c.n ? j0 + lane : 0)), t64.top) == t64.prefix);
        const bool mine = (eq >> lane & 1u) && __popc(eq & ((1u << lane) - 1)) < left;
        const unsigned in = __ballot_sync(0xffffffffu, mine);
        if (lane == 0) s_bits[j0 >> 5] |= in;
        left -= __popc(in);
      }
    }
  } else if (border == need) {
    for (int i = tid; i < border; i += NT) atomicOr(&s_bits[s_page[i] >> 5], 1u << (s_page[i] & 31));
  } else {
    for (int i = warp; i < border; i += NW) {
      const unsigned long long k = exact_bound<T, D>(p, q, s_phys[i], h);
      if (lane == 0) s_key[i] = k;
    }
    __syncthreads();
    for (int i = tid; i < border; i += NT) {
      const unsigned long long k = s_key[i];
      const int j = s_page[i];
      int better = 0;
      for (int x = 0; x < border; ++x) better += s_key[x] > k || (s_key[x] == k && s_page[x] < j);
      if (better < need) atomicOr(&s_bits[j >> 5], 1u << (j & 31));
    }
  }
  __syncthreads();
  // ---- the taken pages in order: a thread's run of words
  const int words = (c.n + 31) >> 5, per = (words + NT - 1) / NT;
  int mine = 0;
  for (int i = tid * per; i < words && i < (tid + 1) * per; ++i) mine += __popc(s_bits[i]);
  const int incl = warp_inclusive_scan(mine);
  if (lane == 31) s_sum[warp] = incl;
  __syncthreads();
  int at = incl - mine + __reduce_add_sync(0xffffffffu, lane < warp ? s_sum[lane] : 0);
  // first into shared memory (the histogram's), then one table entry per thread: otherwise each page waits for its own
  const bool staged = taken <= kPageBins;
  auto put = [&](int x, int page) {
    list[c.first + x] = __ldg(table + page);
    if (out) out[c.first + x] = page;
  };
  for (int i = tid * per; i < words && i < (tid + 1) * per; ++i)
    for (uint32_t w = s_bits[i]; w; w &= w - 1, ++at) {
      const int page = c.first + i * 32 + __ffs(w) - 1;
      if (at >= taken) break;                           // (never, unless scores are not numbers)
      if (staged) s_hist[at] = page;
      else put(at, page);
    }
  if (!staged) return;
  __syncthreads();
  for (int x = tid; x < taken; x += NT) put(x, s_hist[x]);
}

template <typename T, int D, int NT>
static cudaError_t select_nt(PagedProblem p, int n, cudaStream_t st) {
  static PerDeviceFlag configured;
  const cudaError_t e = set_max_dynamic_smem(configured, reinterpret_cast<const void*>(paged_select_kernel<T, D, NT>), kHeldScores * 4);
  if (e != cudaSuccess) return e;
  p.held = held_scores(n);
  return launch_pdl(paged_select_kernel<T, D, NT>, dim3(p.total_q * p.hkv), dim3(NT), (size_t)p.held * 4, st, p);
}

template <typename T, int D>
static cudaError_t select_t(PagedProblem p, int n, int row_tiles, cudaStream_t st) {
  p.scored = n > p.topk && p.topk > 0;
  if (p.scored) {
    const cudaError_t e = launch_pdl(paged_score_kernel<T, D>, dim3(row_tiles * p.hkv, p.mag_parts), dim3(kScoreThreads), 0, st, p);
    if (e != cudaSuccess) return e;
  }
  if (n <= 1024) return select_nt<T, D, 256>(p, n, st);
  if (n <= 4096) return select_nt<T, D, 512>(p, n, st);
  return select_nt<T, D, 1024>(p, n, st);
}

int paged_score_parts(int row_tiles, int hkv, int n) {
  // A row tile's pages over enough CTAs for two per multiprocessor, and no more: each builds its fragments anew.  (Four per
  // multiprocessor, one token of 16 to 96 sequences of 16K or 4K-30K each: a call is up to 2.5% shorter at head_dim 128 and up
  // to 7% longer at 64, at either where the row tiles alone are three per multiprocessor.)
  const int have = row_tiles * hkv, ctas = 2 * sm_count_current_device();
  const int want = (ctas + have - 1) / (have > 0 ? have : 1);
  const int most = (n + kScorePages - 1) / kScorePages;
  return want < most ? want : most > 0 ? most : 1;
}

cudaError_t launch_paged_select(const PagedProblem& p, int d, bool bf16, int max_pages_seq, int row_tiles, cudaStream_t st) {
  const int n = max_pages_seq - p.n_sink - p.n_tail;      // most candidates of a token
  if (d == 64) return bf16 ? select_t<Bf16, 64>(p, n, row_tiles, st) : select_t<Fp16, 64>(p, n, row_tiles, st);
  return bf16 ? select_t<Bf16, 128>(p, n, row_tiles, st) : select_t<Fp16, 128>(p, n, row_tiles, st);
}

}  // namespace tkphi
