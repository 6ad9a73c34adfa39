// New tokens into a paged key/value cache, rotated by their positions on the way.
//
// For token i of sequence b (cache position t = kv_len - q_len + i, angle position x = positions[i] or t):
//   pair (a, c) of a key or query head -> (a cos w - c sin w, c cos w + a sin w),  w = x * inv_freq[pair],
// in 32 bits, rounded once to the element type; values are copied.  The rows go to slot t % page_size of page
// table[b][t / page_size].  With key bounds, every touched page's element-wise minimum and maximum over the rows
// below the sequence's new length is recomputed from the rows themselves (those of earlier calls are read back),
// so that the bounds never depend on what they were.
//
// Bound: memory.  A CTA takes one touched page of one KV head: 8 lanes per row at head_dim 128 (4 at 64), a lane
// owning the two 16-byte pieces whose elements are each other's partners, so that a pair never leaves a thread, and
// the sines of a lane's eight pairs serve the key row and all query rows of the group.  The angle is formed in 64
// bits as turns, x * inv_freq / 2 pi less its nearest integer, because 32 bits lose it at far positions (1e6 * 1.0
// has 0.06 rad of rounding); sincospi of the fraction is then exact to its own error.
#include "paged.cuh"

namespace tkphi {

constexpr int kAppendThreads = 256;

template <typename T>
__device__ __forceinline__ void rotate_pieces(uint4& x, uint4& y, const float (&cs)[8], const float (&sn)[8], bool pairs) {
  uint32_t* a = reinterpret_cast<uint32_t*>(&x);
  uint32_t* b = reinterpret_cast<uint32_t*>(&y);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if (pairs) {
      // partners are neighbours: pair i of the first piece, pair 4 + i of the second
      const float a0 = T::lo(a[i]), a1 = T::hi(a[i]), b0 = T::lo(b[i]), b1 = T::hi(b[i]);
      a[i] = T::pack(a0 * cs[i] - a1 * sn[i], a1 * cs[i] + a0 * sn[i]);
      b[i] = T::pack(b0 * cs[4 + i] - b1 * sn[4 + i], b1 * cs[4 + i] + b0 * sn[4 + i]);
    } else {
      const float a0 = T::lo(a[i]), a1 = T::hi(a[i]), b0 = T::lo(b[i]), b1 = T::hi(b[i]);
      const float c0 = cs[2 * i], s0 = sn[2 * i], c1 = cs[2 * i + 1], s1 = sn[2 * i + 1];
      a[i] = T::pack(a0 * c0 - b0 * s0, a1 * c1 - b1 * s1);
      b[i] = T::pack(b0 * c0 + a0 * s0, b1 * c1 + a1 * s1);
    }
  }
}

template <typename T, int D>
__global__ void __launch_bounds__(kAppendThreads) paged_append_kernel(const AppendProblem p) {
  constexpr int LPR = D / 16;                  // lanes of a row
  constexpr int RPI = kAppendThreads / LPR;    // rows of one pass of the CTA
  __shared__ int s_find[2];                    // sequence, page of the sequence's item list
  __shared__ uint4 s_red[2][kAppendThreads / 32][2 * LPR];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int item = blockIdx.x, h = blockIdx.y;

  // ---- which page: sequence b holds (q_len + ps - 2) / ps + 1 items, enough for every start inside a page
  const int ps = 1 << p.page_shift;
  if (warp == 0) {
    int base = 0;
    for (int s = 0; s < p.batch; s += 32) {
      int n = 0;
      if (s + lane < p.batch) {
        const long long m = __ldg(p.cu_q + s + lane + 1) - __ldg(p.cu_q + s + lane);
        n = m > 0 ? (int)((m + ps - 2) >> p.page_shift) + 1 : 0;
      }
      const int incl = warp_inclusive_scan(n) + base;
      const unsigned hit = __ballot_sync(0xffffffffu, incl > item);
      if (hit) {
        const int l = __ffs(hit) - 1;
        const int first = __shfl_sync(0xffffffffu, incl - n, l);
        if (lane == 0) { s_find[0] = s + l; s_find[1] = item - first; }
        break;
      }
      base = __shfl_sync(0xffffffffu, incl, 31);
      if (s + 32 >= p.batch && lane == 0) s_find[0] = -1;
    }
  }
  __syncthreads();
  const int b = s_find[0];
  if (b < 0) return;
  const long long tok0 = __ldg(p.cu_q + b), n_new = __ldg(p.cu_q + b + 1) - tok0;
  long long len = __ldg(p.kv_lens + b);
  if (len > p.max_kv) len = p.max_kv;
  const long long begin = len - n_new;                    // cache position of the first new token
  if (begin < 0) return;
  const long long page = (begin >> p.page_shift) + s_find[1];
  const long long page_t0 = page << p.page_shift;
  if (page_t0 >= len) return;
  const int lo = begin > page_t0 ? (int)(begin - page_t0) : 0;             // new rows of the page: slots lo .. hi-1
  const int hi = len - page_t0 < ps ? (int)(len - page_t0) : ps;
  const int phys = __ldg(p.table + (size_t)b * p.max_pages + page);
  const bool ok = phys >= 0 && phys < p.n_pages;
  if (!ok && tid == 0) atomicExch(p.status, kStatusBadPage);
  // a bad page takes no rows, but the queries of its tokens are still rotated

  const int l = lane % LPR, r0 = tid / LPR;
  // the lane's two pieces: partners of each other in the rotated part, otherwise neighbours
  int c0, c1, f0 = 0;
  const int turned = p.rot / 16;                          // lanes whose pieces are rotated
  const bool rotate = l < turned;
  if (rotate && !p.pairs) { c0 = l; c1 = l + turned; } else { c0 = 2 * l; c1 = 2 * l + 1; }
  f0 = 8 * l;
  double turn[8];
  if (rotate) {
#pragma unroll
    for (int i = 0; i < 8; ++i) turn[i] = (double)__ldg(p.inv_freq + f0 + i) * 0.15915494309189533577;
  }
  const size_t es = 2;
  char* kp = static_cast<char*>(p.k) + ((size_t)(ok ? phys : 0) * p.stride_page + (size_t)h * p.stride_head) * es;
  char* vp = static_cast<char*>(p.v) + ((size_t)(ok ? phys : 0) * p.stride_page + (size_t)h * p.stride_head) * es;
  uint4 mn0, mn1, mx0, mx1;
  bool any = false;
  for (int row = (p.bounds ? 0 : lo) + r0; row < hi; row += RPI) {
    uint4 a, c;
    if (row >= lo) {
      const long long t = page_t0 + row, tok = tok0 + (t - begin);
      const char* ks = static_cast<const char*>(p.k_new) + ((size_t)tok * p.k_new_token + (size_t)h * p.k_new_head) * es;
      const char* vs = static_cast<const char*>(p.v_new) + ((size_t)tok * p.v_new_token + (size_t)h * p.v_new_head) * es;
      a = __ldg(reinterpret_cast<const uint4*>(ks) + c0);
      c = __ldg(reinterpret_cast<const uint4*>(ks) + c1);
      const uint4 v0 = __ldg(reinterpret_cast<const uint4*>(vs) + 2 * l);
      const uint4 v1 = __ldg(reinterpret_cast<const uint4*>(vs) + 2 * l + 1);
      float cs[8], sn[8];
      if (rotate) {
        const double x = (double)(p.positions ? __ldg(p.positions + tok) : t);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const double w = x * turn[i];
          sincospif(2.f * (float)(w - rint(w)), &sn[i], &cs[i]);
        }
        rotate_pieces<T>(a, c, cs, sn, p.pairs);
      }
      if (ok) {
        char* kd = kp + (size_t)row * p.stride_token * es;
        char* vd = vp + (size_t)row * p.stride_token * es;
        reinterpret_cast<uint4*>(kd)[c0] = a;
        reinterpret_cast<uint4*>(kd)[c1] = c;
        reinterpret_cast<uint4*>(vd)[2 * l] = v0;
        reinterpret_cast<uint4*>(vd)[2 * l + 1] = v1;
      }
      if (p.q) {
        const char* qs = static_cast<const char*>(p.q) + ((size_t)tok * p.q_token + (size_t)h * p.group * p.q_head) * es;
        char* qd = static_cast<char*>(p.q_out) + ((size_t)tok * p.q_out_token + (size_t)h * p.group * p.q_out_head) * es;
        // (plain loads: q_out may be q itself)
        for (int g = 0; g < p.group; ++g) {
          const uint4* s = reinterpret_cast<const uint4*>(qs + (size_t)g * p.q_head * es);
          uint4 x = s[c0], y = s[c1];
          if (rotate) rotate_pieces<T>(x, y, cs, sn, p.pairs);
          uint4* o = reinterpret_cast<uint4*>(qd + (size_t)g * p.q_out_head * es);
          o[c0] = x;
          o[c1] = y;
        }
      }
    } else {
      if (!ok) continue;
      const uint4* kd = reinterpret_cast<const uint4*>(kp + (size_t)row * p.stride_token * es);
      a = kd[c0];
      c = kd[c1];
    }
    if (p.bounds) {
      if (!any) { mn0 = mx0 = a; mn1 = mx1 = c; any = true; }
      else {
        uint32_t *n0 = reinterpret_cast<uint32_t*>(&mn0), *n1 = reinterpret_cast<uint32_t*>(&mn1);
        uint32_t *x0 = reinterpret_cast<uint32_t*>(&mx0), *x1 = reinterpret_cast<uint32_t*>(&mx1);
        const uint32_t *pa = reinterpret_cast<const uint32_t*>(&a), *pc = reinterpret_cast<const uint32_t*>(&c);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          n0[i] = T::min2(n0[i], pa[i]); x0[i] = T::max2(x0[i], pa[i]);
          n1[i] = T::min2(n1[i], pc[i]); x1[i] = T::max2(x1[i], pc[i]);
        }
      }
    }
  }
  if (!p.bounds || !ok) return;
  // ---- the page's bounds: over the lanes of a warp with the same pieces, then over the warps; a thread without a
  // row takes its partner's
  unsigned have = __ballot_sync(0xffffffffu, any);
  uint32_t* w[4] = {reinterpret_cast<uint32_t*>(&mn0), reinterpret_cast<uint32_t*>(&mn1), reinterpret_cast<uint32_t*>(&mx0),
                    reinterpret_cast<uint32_t*>(&mx1)};
  for (int o = LPR; o < 32; o <<= 1) {
    const bool theirs = (have >> (lane ^ o)) & 1u;
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t x = __shfl_xor_sync(0xffffffffu, w[j][i], o);
        if (theirs) w[j][i] = !any ? x : j < 2 ? T::min2(w[j][i], x) : T::max2(w[j][i], x);
      }
    any = any || theirs;
    have = __ballot_sync(0xffffffffu, any);
  }
  // rows are dealt to the warps in order: if a warp holds none, neither do the later ones
  if (lane < LPR && any) {
    s_red[0][warp][c0] = mn0; s_red[0][warp][c1] = mn1;
    s_red[1][warp][c0] = mx0; s_red[1][warp][c1] = mx1;
  }
  __syncthreads();
  constexpr int RPW = 32 / LPR;
  const int warps = (hi + RPW - 1) / RPW < kAppendThreads / 32 ? (hi + RPW - 1) / RPW : kAppendThreads / 32;
  if (tid < 4 * LPR) {
    const int side = tid / (2 * LPR), c = tid % (2 * LPR);
    uint4 r = s_red[side][0][c];
    uint32_t* rr = reinterpret_cast<uint32_t*>(&r);
    for (int i = 1; i < warps; ++i) {
      const uint4 x = s_red[side][i][c];
      const uint32_t* xx = reinterpret_cast<const uint32_t*>(&x);
#pragma unroll
      for (int e = 0; e < 4; ++e) rr[e] = side == 0 ? T::min2(rr[e], xx[e]) : T::max2(rr[e], xx[e]);
    }
    uint4* out = reinterpret_cast<uint4*>(static_cast<char*>(p.bounds) + (((size_t)phys * p.hkv + h) * 2 + side) * D * es);
    out[c] = r;
  }
}

cudaError_t launch_paged_append(const AppendProblem& p, bool bf16, cudaStream_t st) {
  const dim3 grid(p.items, p.hkv);
  if (p.d == 64) {
    if (bf16) paged_append_kernel<Bf16, 64><<<grid, kAppendThreads, 0, st>>>(p);
    else paged_append_kernel<Fp16, 64><<<grid, kAppendThreads, 0, st>>>(p);
  } else {
    if (bf16) paged_append_kernel<Bf16, 128><<<grid, kAppendThreads, 0, st>>>(p);
    else paged_append_kernel<Fp16, 128><<<grid, kAppendThreads, 0, st>>>(p);
  }
  return cudaGetLastError();
}

}  // namespace tkphi
