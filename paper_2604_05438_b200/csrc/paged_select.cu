// Page selection: for every new token and KV head, the pages whose keys could score highest.
//
//   bound(page) = max over the group's query heads of sum_c max(q_c lo_c, q_c hi_c),
// lo, hi the element-wise minimum and maximum of the page's keys: no key of the page scores more.  The first n_sink
// and the last n_tail pages that the token sees are always taken, of those between the topk with the largest bounds,
// equal ones towards the lower page.
//
// The selection is exact: a product of two 16-bit floats has 22 bits at most, and 128 of them add up in 64 bits without
// rounding unless their exponents span more than about 25 binades, so the order does not depend on how the sum is
// split.  (In 32 bits, neighbours among thousands of pages swap.)  The 64-bit conversion is an integer shift: the
// exponent field of a 16-bit float placed at the bottom of a double's is the same number times 2^-896 (bf16) or
// 2^-1008 (fp16), subnormals and zero included, and the query carries the inverse factor.
#include "paged.cuh"

namespace tkphi {

constexpr int kScoreThreads = 256;
constexpr int kScoreSteps = 4;             // page steps of a warp, all loads in flight at once

template <typename T>
__device__ __forceinline__ int dbl_hi_word(uint32_t w, bool upper) {       // scaled double of one half of w (low word 0)
  const int x = (int)(upper ? w : w << 16);
  return T::kBf16 ? ((x >> 3) & (int)0x8fffe000) : ((x >> 6) & (int)0x81fffc00);
}

// Token's position and the candidate pages [first, first + n).
struct Candidates {
  int b, pos, seen, first, n;
};
__device__ __forceinline__ Candidates candidates_of(const PagedProblem& p, int tok) {
  Candidates c;
  c.b = paged_seq_of(p, tok);
  c.pos = paged_kv_len(p, c.b) - paged_q_len(p, c.b) + (tok - (int)__ldg(p.cu_q + c.b));
  if (c.pos < 0) c.pos = 0;
  c.seen = (c.pos >> p.page_shift) + 1;
  c.first = p.n_sink < c.seen ? p.n_sink : c.seen;
  const int n = c.seen - p.n_tail - c.first;
  c.n = n > 0 ? n : 0;
  return c;
}

// Lanes of a page: 8 dims (16 bytes of each bound) per lane.  Pages of a CTA.
template <int D>
struct ScoreCfg {
  static constexpr int LPP = D / 8;
  static constexpr int PPS = 32 / LPP;                       // pages of a warp's step
  static constexpr int PAGES = kScoreThreads / 32 * kScoreSteps * PPS;
};

// Bound: DRAM for single tokens, the 64-bit FMA rate (64 per clock and SM) for several query heads or tokens.  The
// bounds of a page are converted once and serve all query heads of the group; per element and head a select by the
// query's sign and one FMA remain.
template <typename T, int D>
__global__ void __launch_bounds__(kScoreThreads, 2) paged_score_kernel(const __grid_constant__ PagedProblem p) {
  using C = ScoreCfg<D>;
  __shared__ double2 s_q[kMaxGroup * D / 2];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  pdl_wait();
  pdl_launch_next();
  const int unit = blockIdx.x, tok = unit / p.hkv, h = unit % p.hkv;
  const Candidates c = candidates_of(p, tok);
  if (c.n <= p.topk || (int)blockIdx.y * C::PAGES >= c.n) return;      // all are taken, or none is left for this CTA
  const int sub = lane % C::LPP, stride = gridDim.y * C::PAGES;
  const int* table = p.table + (size_t)c.b * p.max_pages + c.first;
  const uint4* bounds = static_cast<const uint4*>(p.bounds) + (size_t)h * (2 * D / 8) + sub;
  const size_t page_step = (size_t)p.hkv * (2 * D / 8);
  int j0 = blockIdx.y * C::PAGES + warp * kScoreSteps * C::PPS + lane / C::LPP;        // this lane's page of step 0
  // a round's bounds are loaded while the round before is computed, its page ids one round earlier still
  int ids[kScoreSteps];
  uint4 rl[kScoreSteps], rh[kScoreSteps];
  unsigned fine = 0;                                       // steps of the loaded round with a valid page id
  auto load_ids = [&](int j) {
#pragma unroll
    for (int s = 0; s < kScoreSteps; ++s) ids[s] = j + s * C::PPS < c.n ? __ldg(table + j + s * C::PPS) : 0;
  };
  auto load_bounds = [&]() {
    fine = 0;
#pragma unroll
    for (int s = 0; s < kScoreSteps; ++s) {
      const bool ok = ids[s] >= 0 && ids[s] < p.n_pages;
      if (!ok && sub == 0) atomicExch(p.status, kStatusBadPage);
      fine |= (ok ? 1u : 0u) << s;
      const uint4* src = bounds + (ok ? ids[s] : 0) * page_step;
      rl[s] = __ldg(src);
      rh[s] = __ldg(src + D / 8);
    }
  };
  load_ids(j0);
  const double up = T::kBf16 ? __hiloint2double((1023 + 896) << 20, 0) : __hiloint2double((1023 + 1008) << 20, 0);
  const uint32_t* q = static_cast<const uint32_t*>(p.q) + ((size_t)tok * p.hq + h * p.group) * (D / 2);
  for (int i = tid; i < p.group * D / 2; i += kScoreThreads) {
    const uint32_t w = __ldg(q + i);
    // pair i of a head is read by lane (i / 4) of the page in its step i % 4: lanes beside each other, no bank twice
    const int g = i / (D / 2), x = i % (D / 2);
    s_q[(g * 4 + x % 4) * C::LPP + x / 4] = make_double2((double)T::lo(w) * up, (double)T::hi(w) * up);
  }
  load_bounds();
  load_ids(j0 + stride);
  __syncthreads();
  for (int r0 = blockIdx.y * C::PAGES; r0 < c.n; r0 += stride, j0 += stride) {
    // high words of the scaled doubles (their low words are 0)
    int lo[kScoreSteps][8], hi[kScoreSteps][8];
#pragma unroll
    for (int s = 0; s < kScoreSteps; ++s)
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        lo[s][e] = dbl_hi_word<T>(reinterpret_cast<const uint32_t*>(&rl[s])[e >> 1], e & 1);
        hi[s][e] = dbl_hi_word<T>(reinterpret_cast<const uint32_t*>(&rh[s])[e >> 1], e & 1);
        asm("" : "+r"(lo[s][e]), "+r"(hi[s][e]));          // kept, not converted again for every head
      }
    const unsigned fine_now = fine;
    if (r0 + stride < c.n) {
      load_bounds();
      load_ids(j0 + 2 * stride);
    }
    double best = -INFINITY;                   // of the page step that this lane ends up with
    for (int g = 0; g < p.group; ++g) {
      double acc[kScoreSteps] = {0., 0., 0., 0.};
      const double2* qs = s_q + g * 4 * C::LPP + sub;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const double2 qq = qs[e * C::LPP];
        const bool n0 = __double2hiint(qq.x) < 0, n1 = __double2hiint(qq.y) < 0;
#pragma unroll
        for (int s = 0; s < kScoreSteps; ++s) {
          acc[s] = fma(qq.x, __hiloint2double(n0 ? lo[s][2 * e] : hi[s][2 * e], 0), acc[s]);
          acc[s] = fma(qq.y, __hiloint2double(n1 ? lo[s][2 * e + 1] : hi[s][2 * e + 1], 0), acc[s]);
        }
      }
      // four sums over the page's lanes: two are handed over, then one, so that a lane ends up with one of them
      const bool b0 = lane & 1, b1 = lane & 2;
      double u = b0 ? acc[2] : acc[0], v = b0 ? acc[3] : acc[1];
      u += __shfl_xor_sync(0xffffffffu, b0 ? acc[0] : acc[2], 1);
      v += __shfl_xor_sync(0xffffffffu, b0 ? acc[1] : acc[3], 1);
      double w = b1 ? v : u;
      w += __shfl_xor_sync(0xffffffffu, b1 ? u : v, 2);
#pragma unroll
      for (int o = 4; o < C::LPP; o <<= 1) w += __shfl_xor_sync(0xffffffffu, w, o);
      best = fmax(best, w);
    }
    if (sub < 4) {
      const int s = (lane & 1) * 2 + ((lane >> 1) & 1), j = j0 + s * C::PPS;
      if (j < c.n) {
        // larger bound <=> larger key; -0 counts as 0
        const unsigned long long x = (unsigned long long)__double_as_longlong(best + 0.0);
        p.page_keys[(size_t)unit * p.key_stride + j] = !(fine_now >> s & 1u) ? 0ull : (x >> 63) ? ~x : (x | (1ull << 63));
      }
    }
  }
}

__device__ __forceinline__ unsigned long long shr64(unsigned long long x, int s) { return s >= 64 ? 0ull : x >> s; }

constexpr int kPageBins = 2048;

// Exact topk of the unit's keys, one CTA per unit.  Thread t holds keys t, t + NT, ..: KPT of them in registers, any
// further ones are read again in each pass.
template <int NT, int KPT>
__global__ void __launch_bounds__(NT) paged_select_kernel(const __grid_constant__ PagedProblem p) {
  constexpr int NW = NT / 32;
  __shared__ int s_hist[kPageBins];
  __shared__ unsigned long long s_min[NW], s_max[NW];
  __shared__ int s_sum[NW], s_cnt[KPT * NW];
  __shared__ int s_bin, s_need, s_count;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int unit = blockIdx.x, tok = unit / p.hkv;
  pdl_launch_next();
  for (int i = tid; i < kPageBins; i += NT) s_hist[i] = 0;
  // (the call's inputs may be read before the wait: this grid starts when the scoring grid has begun, which had waited
  // for everything before it)
  const Candidates c = candidates_of(p, tok);
  pdl_wait();
  int* list = p.page_list + (size_t)unit * p.n_keep;
  int* out = p.page_out ? p.page_out + (size_t)unit * p.n_keep : nullptr;
  const int* table = p.table + (size_t)c.b * p.max_pages;
  const int taken = c.n < p.topk ? c.n : p.topk;        // of the candidates
  const int last0 = c.first + c.n;                      // first page of the tail
  const int n_list = c.first + taken + (c.seen - last0);
  const bool search = c.n > p.topk && p.topk > 0;
  const unsigned long long* keys = p.page_keys + (size_t)unit * p.key_stride;
  unsigned long long held[KPT];
  if (search) {
#pragma unroll
    for (int i = 0; i < KPT; ++i) held[i] = i * NT + tid < c.n ? __ldcg(keys + i * NT + tid) : 0ull;
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
  auto each = [&](auto&& fn) {
#pragma unroll
    for (int i = 0; i < KPT; ++i)
      if (i * NT + tid < c.n) fn(held[i]);
    for (int i = KPT * NT + tid; i < c.n; i += NT) fn(__ldcg(keys + i));
  };
  unsigned long long mn = ~0ull, mx = 0ull;
  each([&](unsigned long long k) { mn = k < mn ? k : mn; mx = k > mx ? k : mx; });
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    const unsigned long long a = __shfl_xor_sync(0xffffffffu, mn, o), b = __shfl_xor_sync(0xffffffffu, mx, o);
    mn = a < mn ? a : mn;
    mx = b > mx ? b : mx;
  }
  if (lane == 0) { s_min[warp] = mn; s_max[warp] = mx; }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < NW; ++i) { mn = s_min[i] < mn ? s_min[i] : mn; mx = s_max[i] > mx ? s_max[i] : mx; }
  // The keys share all bits above `top`; of those that share `prefix` above it, `need` are still to be taken.  A pass
  // counts them by their next 11 bits.
  int top = mn == mx ? 0 : 64 - __clzll((long long)(mn ^ mx));
  unsigned long long prefix = shr64(mx, top);
  int need = p.topk, count = c.n;
  bool clean = true;
  while (top > 0 && count > need) {
    const int width = top < 11 ? top : 11, shift = top - width, bins = 1 << width;
    if (!clean) {
      for (int i = tid; i < bins; i += NT) s_hist[i] = 0;
      __syncthreads();
    }
    clean = false;
    each([&](unsigned long long k) {
      if (shr64(k, top) == prefix) atomicAdd(&s_hist[(int)(k >> shift) & (bins - 1)], 1);
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
    int before = incl - mine;
    if (NW <= 8) {
#pragma unroll
      for (int i = 0; i < NW; ++i) before += i < warp ? s_sum[i] : 0;
    } else {
      before += __reduce_add_sync(0xffffffffu, lane < warp ? s_sum[lane] : 0);
    }
    if (before < need && before + mine >= need) {
      for (int i = 0; i < run; ++i) {
        const int bin = bins - 1 - (tid * run + i), n = s_hist[bin];
        if (before + n >= need) { s_bin = bin; s_need = need - before; s_count = n; break; }
        before += n;
      }
    }
    __syncthreads();
    need = s_need;
    count = s_count;
    prefix = (prefix << width) | (unsigned long long)s_bin;
    top = shift;
  }
  // Keys above the prefix are taken, of those equal to it the first `need` in page order.  32 consecutive pages are one
  // ballot of a warp; (taken, equal) counts of the ballots, 16 bits each, are scanned in page order.  KPT * NT pages at
  // a time (at most 16384, so that no count overflows).
  static_assert(KPT * NW <= NT && KPT * NT <= 16384, "one count per thread");
  int sure0 = 0, tie0 = 0;                              // of the pages before
  for (int base = 0; base < c.n; base += KPT * NT) {
    unsigned ms[KPT], mt[KPT];
#pragma unroll
    for (int i = 0; i < KPT; ++i) {
      const int j = base + i * NT + tid;
      const unsigned long long x = shr64(base == 0 ? held[i] : j < c.n ? __ldcg(keys + j) : 0ull, top);
      ms[i] = __ballot_sync(0xffffffffu, j < c.n && x > prefix);
      mt[i] = __ballot_sync(0xffffffffu, j < c.n && x == prefix);
      if (lane == 0) s_cnt[i * NW + warp] = __popc(ms[i]) | (__popc(mt[i]) << 16);
    }
    __syncthreads();
    const int mine = tid < KPT * NW ? s_cnt[tid] : 0, incl = warp_inclusive_scan(mine);
    if (lane == 31) s_sum[warp] = incl;
    __syncthreads();
    const int sums = lane < NW ? s_sum[lane] : 0;
    const int before = __reduce_add_sync(0xffffffffu, lane < warp ? sums : 0), all = __reduce_add_sync(0xffffffffu, sums);
    if (tid < KPT * NW) s_cnt[tid] = before + incl - mine;
    __syncthreads();
    const unsigned below = (1u << lane) - 1;
#pragma unroll
    for (int i = 0; i < KPT; ++i) {
      const int at0 = s_cnt[i * NW + warp];
      const int nsure = sure0 + (at0 & 0xffff) + __popc(ms[i] & below), ntie = tie0 + (at0 >> 16) + __popc(mt[i] & below);
      if ((ms[i] >> lane & 1u) || ((mt[i] >> lane & 1u) && ntie < need)) {
        const int at = c.first + nsure + (ntie < need ? ntie : need), page = c.first + base + i * NT + tid;
        list[at] = __ldg(table + page);
        if (out) out[at] = page;
      }
    }
    sure0 += all & 0xffff;
    tie0 += all >> 16;
    __syncthreads();
  }
}

cudaError_t launch_paged_select(const PagedProblem& p, int d, bool bf16, int max_pages_seq, cudaStream_t st) {
  const int units = p.total_q * p.hkv;
  const int n = max_pages_seq - p.n_sink - p.n_tail;      // most candidates of a token
  if (n > p.topk && p.topk > 0) {
    const int pages = d == 64 ? ScoreCfg<64>::PAGES : ScoreCfg<128>::PAGES;
    // a unit's pages over enough CTAs for two per multiprocessor twice over, and no more: each converts the queries anew
    const int want = (4 * sm_count_current_device() + units - 1) / units, most = (n + pages - 1) / pages;
    const dim3 grid(units, want < most ? want : most), block(kScoreThreads);
    cudaError_t e;
    if (d == 64) e = bf16 ? launch_pdl(paged_score_kernel<Bf16, 64>, grid, block, 0, st, p) : launch_pdl(paged_score_kernel<Fp16, 64>, grid, block, 0, st, p);
    else e = bf16 ? launch_pdl(paged_score_kernel<Bf16, 128>, grid, block, 0, st, p) : launch_pdl(paged_score_kernel<Fp16, 128>, grid, block, 0, st, p);
    if (e != cudaSuccess) return e;
  }
  if (n <= 1024) return launch_pdl(paged_select_kernel<256, 4>, dim3(units), dim3(256), 0, st, p);
  if (n <= 4096) return launch_pdl(paged_select_kernel<512, 8>, dim3(units), dim3(512), 0, st, p);
  return launch_pdl(paged_select_kernel<1024, 16>, dim3(units), dim3(1024), 0, st, p);
}

}  // namespace tkphi
