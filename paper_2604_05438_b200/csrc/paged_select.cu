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
constexpr int kScorePages = 128;           // pages of a scoring CTA: 8 warps x 4 steps x 4 pages (8 lanes each)

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

template <typename T, int D>
__global__ void __launch_bounds__(kScoreThreads) paged_score_kernel(const __grid_constant__ PagedProblem p) {
  constexpr int PIECES = D / 64;           // 16-byte pieces of a lane: piece sub + 8 i
  __shared__ double s_q[kMaxGroup][D];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int unit = blockIdx.x, tok = unit / p.hkv, h = unit % p.hkv;
  pdl_launch_next();
  const Candidates c = candidates_of(p, tok);
  const int p0 = blockIdx.y * kScorePages;
  if (c.n <= p.topk || p0 >= c.n) return;              // all are taken, or none is left for this CTA
  const double up = T::kBf16 ? __hiloint2double((1023 + 896) << 20, 0) : __hiloint2double((1023 + 1008) << 20, 0);
  const uint32_t* q = static_cast<const uint32_t*>(p.q) + ((size_t)tok * p.hq + h * p.group) * (D / 2);
  for (int i = tid; i < p.group * D / 2; i += kScoreThreads) {
    const uint32_t w = __ldg(q + i);
    s_q[0][2 * i] = (double)T::lo(w) * up;
    s_q[0][2 * i + 1] = (double)T::hi(w) * up;
  }
  __syncthreads();
  const int sub = lane & 7;
  const uint4* bounds = static_cast<const uint4*>(p.bounds);
  unsigned long long* keys = p.page_keys + (size_t)unit * p.key_stride;
  uint4 lo[4][PIECES], hi[4][PIECES];
  bool ok[4];
#pragma unroll
  for (int s = 0; s < 4; ++s) {
    const int j = p0 + warp * 16 + s * 4 + (lane >> 3);
    ok[s] = false;
    if (j < c.n) {
      const int phys = __ldg(p.table + (size_t)c.b * p.max_pages + c.first + j);
      ok[s] = phys >= 0 && phys < p.n_pages;
      if (!ok[s]) atomicExch(p.status, kStatusBadPage);
      const uint4* src = bounds + ((size_t)(ok[s] ? phys : 0) * p.hkv + h) * (2 * D / 8) + sub;
#pragma unroll
      for (int i = 0; i < PIECES; ++i) { lo[s][i] = __ldg(src + 8 * i); hi[s][i] = __ldg(src + D / 8 + 8 * i); }
    } else {
#pragma unroll
      for (int i = 0; i < PIECES; ++i) lo[s][i] = hi[s][i] = make_uint4(0, 0, 0, 0);
    }
  }
  double best[4];
#pragma unroll
  for (int s = 0; s < 4; ++s) best[s] = -INFINITY;
  for (int g = 0; g < p.group; ++g) {
    double acc[4] = {0., 0., 0., 0.};
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
      const double2* qs = reinterpret_cast<const double2*>(&s_q[g][(sub + 8 * i) * 8]);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const double2 qq = qs[e];
        const bool n0 = __double2hiint(qq.x) < 0, n1 = __double2hiint(qq.y) < 0;
#pragma unroll
        for (int s = 0; s < 4; ++s) {
          const uint32_t wl = reinterpret_cast<const uint32_t*>(&lo[s][i])[e], wh = reinterpret_cast<const uint32_t*>(&hi[s][i])[e];
          acc[s] = fma(qq.x, __hiloint2double(dbl_hi_word<T>(n0 ? wl : wh, false), 0), acc[s]);
          acc[s] = fma(qq.y, __hiloint2double(dbl_hi_word<T>(n1 ? wl : wh, true), 0), acc[s]);
        }
      }
    }
#pragma unroll
    for (int s = 0; s < 4; ++s) {
#pragma unroll
      for (int o = 1; o < 8; o <<= 1) acc[s] += __shfl_xor_sync(0xffffffffu, acc[s], o);
      best[s] = fmax(best[s], acc[s]);
    }
  }
  if (sub == 0) {
#pragma unroll
    for (int s = 0; s < 4; ++s) {
      const int j = p0 + warp * 16 + s * 4 + (lane >> 3);
      if (j < c.n) {
        // larger bound <=> larger key; -0 counts as 0
        const unsigned long long u = (unsigned long long)__double_as_longlong(best[s] + 0.0);
        keys[j] = !ok[s] ? 0ull : (u >> 63) ? ~u : (u | (1ull << 63));
      }
    }
  }
}

__device__ __forceinline__ unsigned long long shr64(unsigned long long x, int s) { return s >= 64 ? 0ull : x >> s; }

constexpr int kPageBins = 2048;
constexpr int kHeldKeys = 8;               // keys a thread keeps in registers; with more it reads them again

// Exact topk of n keys, one CTA per unit; thread t owns a contiguous run of keys, so that thread order is page order.
template <int NT>
__global__ void __launch_bounds__(NT) paged_select_kernel(const __grid_constant__ PagedProblem p) {
  __shared__ int s_hist[kPageBins];
  __shared__ unsigned long long s_min[NT / 32], s_max[NT / 32];
  __shared__ int s_sum[NT / 32], s_sum2[NT / 32];
  __shared__ int s_bin, s_need, s_count;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int unit = blockIdx.x, tok = unit / p.hkv;
  pdl_launch_next();
  const Candidates c = candidates_of(p, tok);
  int* list = p.page_list + (size_t)unit * p.n_keep;
  int* out = p.page_out ? p.page_out + (size_t)unit * p.n_keep : nullptr;
  const int* table = p.table + (size_t)c.b * p.max_pages;
  const int taken = c.n < p.topk ? c.n : p.topk;        // of the candidates
  const int last0 = c.first + c.n;                      // first page of the tail
  const int n_list = c.first + taken + (c.seen - last0);
  pdl_wait();
  // the pages that are always taken, and the padding
  for (int i = tid; i < p.n_keep; i += NT) {
    const int page = i < c.first ? i : i < c.first + taken ? -2 : i < n_list ? last0 + (i - c.first - taken) : -1;
    if (page != -2) {
      list[i] = page < 0 ? -1 : __ldg(table + page);
      if (out) out[i] = page;
    }
  }
  if (c.n <= p.topk) {
    for (int i = tid; i < c.n; i += NT) {
      list[c.first + i] = __ldg(table + c.first + i);
      if (out) out[c.first + i] = c.first + i;
    }
    return;
  }
  if (p.topk == 0) return;
  const unsigned long long* keys = p.page_keys + (size_t)unit * p.key_stride;
  const int per = (c.n + NT - 1) / NT, i0 = tid * per < c.n ? tid * per : c.n, i1 = i0 + per < c.n ? i0 + per : c.n;
  unsigned long long held[kHeldKeys];
#pragma unroll
  for (int i = 0; i < kHeldKeys; ++i) held[i] = i0 + i < i1 ? __ldcg(keys + i0 + i) : 0ull;
  auto each = [&](auto&& fn) {
#pragma unroll
    for (int i = 0; i < kHeldKeys; ++i)
      if (i0 + i < i1) fn(i0 + i, held[i]);
    for (int i = i0 + kHeldKeys; i < i1; ++i) fn(i, __ldcg(keys + i));
  };
  unsigned long long mn = ~0ull, mx = 0ull;
  each([&](int, unsigned long long k) { mn = k < mn ? k : mn; mx = k > mx ? k : mx; });
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    const unsigned long long a = __shfl_xor_sync(0xffffffffu, mn, o), b = __shfl_xor_sync(0xffffffffu, mx, o);
    mn = a < mn ? a : mn;
    mx = b > mx ? b : mx;
  }
  if (lane == 0) { s_min[warp] = mn; s_max[warp] = mx; }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < NT / 32; ++i) { mn = s_min[i] < mn ? s_min[i] : mn; mx = s_max[i] > mx ? s_max[i] : mx; }
  // the keys share all bits above `top`; of those that share `prefix` above it, `need` are still to be taken
  int top = mn == mx ? 0 : 64 - __clzll((long long)(mn ^ mx));
  unsigned long long prefix = shr64(mx, top);
  int need = p.topk, count = c.n;
  while (top > 0 && count > need) {
    const int width = top < 11 ? top : 11, shift = top - width, bins = 1 << width;
    for (int i = tid; i < bins; i += NT) s_hist[i] = 0;
    __syncthreads();
    each([&](int, unsigned long long k) {
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
    for (int i = 0; i < warp; ++i) before += s_sum[i];
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
    __syncthreads();
  }
  // larger than the prefix: taken; equal: the first `need` in page order
  int sure = 0, tie = 0;
  each([&](int, unsigned long long k) {
    const unsigned long long x = shr64(k, top);
    sure += x > prefix;
    tie += x == prefix;
  });
  const int isure = warp_inclusive_scan(sure), itie = warp_inclusive_scan(tie);
  if (lane == 31) { s_sum[warp] = isure; s_sum2[warp] = itie; }
  __syncthreads();
  int nsure = isure - sure, ntie = itie - tie;
  for (int i = 0; i < warp; ++i) { nsure += s_sum[i]; ntie += s_sum2[i]; }
  each([&](int j, unsigned long long k) {
    const unsigned long long x = shr64(k, top);
    const bool take = x > prefix || (x == prefix && ntie < need);
    if (take) {
      const int at = c.first + nsure + (ntie < need ? ntie : need);
      list[at] = __ldg(table + c.first + j);
      if (out) out[at] = c.first + j;
    }
    nsure += x > prefix;
    ntie += x == prefix;
  });
}

cudaError_t launch_paged_select(const PagedProblem& p, int d, bool bf16, int max_pages_seq, cudaStream_t st) {
  const int units = p.total_q * p.hkv;
  const int n = max_pages_seq - p.n_sink - p.n_tail;      // most candidates of a token
  if (n > p.topk && p.topk > 0) {
    const dim3 grid(units, (n + kScorePages - 1) / kScorePages);
    if (d == 64) {
      if (bf16) paged_score_kernel<Bf16, 64><<<grid, kScoreThreads, 0, st>>>(p);
      else paged_score_kernel<Fp16, 64><<<grid, kScoreThreads, 0, st>>>(p);
    } else {
      if (bf16) paged_score_kernel<Bf16, 128><<<grid, kScoreThreads, 0, st>>>(p);
      else paged_score_kernel<Fp16, 128><<<grid, kScoreThreads, 0, st>>>(p);
    }
    const cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) return e;
    if (n <= 256 * kHeldKeys) return launch_pdl(paged_select_kernel<256>, dim3(units), dim3(256), 0, st, p);
    return launch_pdl(paged_select_kernel<1024>, dim3(units), dim3(1024), 0, st, p);
  }
  paged_select_kernel<256><<<units, 256, 0, st>>>(p);
  return cudaGetLastError();
}

}  // namespace tkphi
