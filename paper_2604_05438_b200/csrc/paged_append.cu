// New tokens into a paged key/value cache, rotated by their positions on the way.
//
// For token i of sequence b (cache position t = kv_len - q_len + i, angle position x = positions[i] or t):
//   pair (a, c) of a key or query head -> (a cos w - c sin w, c cos w + a sin w),  w = x * inv_freq[pair],
// in 32 bits, rounded once to the element type; values are copied.  The rows go to slot t % page_size of page
// table[b][t / page_size].  With key bounds, every touched page's element-wise minimum and maximum over the rows
// below the sequence's new length is recomputed from the rows themselves (those of earlier calls are read back),
// so that the bounds never depend on what they were.
//
// Bound: memory.  A CTA takes 64 positions of one KV head: 8 lanes per row at head_dim 128 (4 at 64), a lane
// owning the two 16-byte pieces whose elements are each other's partners, so that a pair never leaves a thread, and
// the sines of a lane's eight pairs serve the key row and all query rows of the group.  The angle is formed in 64
// bits as turns, x * inv_freq / 2 pi less its nearest integer, because 32 bits lose it at far positions (1e6 * 1.0
// has 0.06 rad of rounding); sincospi of the fraction is then exact to its own error.
#include "paged.cuh"

namespace tkphi {


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

// An item is one KV head of 64 aligned cache positions (128 where the page is that long): whole pages, so that their
// bounds need no other CTA.
template <typename T, int D, int NT>
__global__ void __launch_bounds__(NT, NT == 128 ? 5 : 2) paged_append_kernel(const __grid_constant__ AppendProblem p) {
  constexpr int LPR = D / 16;                  // lanes of a row
  constexpr int RPW = 32 / LPR;                // rows of a warp
  constexpr int RPP = NT / LPR;    // rows of one pass of the CTA
  constexpr size_t es = 2;
  __shared__ long long s_find[4];              // sequence, its first token row, cache length, first new position
  __shared__ int s_item;
  __shared__ uint4 s_red[128 / RPW][2][2 * LPR];     // a warp's rows: their minimum and maximum
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int h = blockIdx.y, span_shift = p.page_shift > 6 ? p.page_shift : 6;
  pdl_wait();
  pdl_launch_next();

  // ---- which positions: a sequence holds (q_len + span - 2) / span + 1 items, enough for every start inside one
  if (warp == 0) {
    const int item = blockIdx.x, span = 1 << span_shift;
    int base = 0;
    if (lane == 0) s_find[0] = -1;
    for (int s = 0; s < p.batch; s += 32) {
      int n = 0;
      long long t0 = 0, m = 0, len = 0;
      if (s + lane < p.batch) {
        t0 = __ldg(p.cu_q + s + lane);
        m = __ldg(p.cu_q + s + lane + 1) - t0;
        len = __ldg(p.kv_lens + s + lane);
        n = m > 0 ? (int)((m + span - 2) >> span_shift) + 1 : 0;
      }
      const int incl = warp_inclusive_scan(n) + base;
      if (incl > item && incl - n <= item) {           // one lane
        s_find[0] = s + lane; s_find[1] = t0;
        s_find[2] = len < p.max_kv ? len : p.max_kv;
        s_find[3] = s_find[2] - m;
        s_item = item - (incl - n);
      }
      base = __shfl_sync(0xffffffffu, incl, 31);
      if (base > item) break;
    }
  }
  __syncthreads();
  const int b = (int)s_find[0];
  const long long tok0 = s_find[1], len = s_find[2], begin = s_find[3];
  if (b < 0 || begin < 0) return;
  const long long t0 = ((begin >> span_shift) + s_item) << span_shift;       // first position of the item
  if (t0 >= len) return;
  const int lo = begin > t0 ? (int)(begin - t0) : 0;                         // new rows: lo .. hi-1 of the item
  const int hi = len - t0 < (1ll << span_shift) ? (int)(len - t0) : 1 << span_shift;
  const int ps = 1 << p.page_shift, first = p.bounds ? lo & ~(ps - 1) : lo;  // with bounds: every row of the touched pages
  const int* table = p.table + (size_t)b * p.max_pages + (t0 >> p.page_shift);

  const int l = lane % LPR;
  // the lane's two pieces: partners of each other in the rotated part, otherwise neighbours
  int c0 = 2 * l, c1 = 2 * l + 1;
  const int turned = p.rot / 16;                          // lanes whose pieces are rotated
  const bool rotate = l < turned;
  if (rotate && !p.pairs) { c0 = l; c1 = l + turned; }
  double turn[8];
  if (rotate) {
#pragma unroll
    for (int i = 0; i < 8; ++i) turn[i] = (double)__ldg(p.inv_freq + 8 * l + i) * 0.15915494309189533577;
  }
  for (int r0 = 0; r0 < hi; r0 += RPP) {
    const int row = r0 + tid / LPR;
    const bool in = row >= first && row < hi;
    uint4 a = make_uint4(0, 0, 0, 0), c = a;
    if (in) {
      // a page id outside the cache: its rows are dropped, the queries of its tokens are rotated all the same
      const int phys = __ldg(table + (row >> p.page_shift));
      const bool ok = phys >= 0 && phys < p.n_pages;
      if (!ok && l == 0) atomicExch(p.status, kStatusBadPage);
      const size_t at = ((size_t)(ok ? phys : 0) * p.stride_page + (size_t)h * p.stride_head + (size_t)(row & (ps - 1)) * p.stride_token) * es;
      uint4* kd = reinterpret_cast<uint4*>(static_cast<char*>(p.k) + at);
      if (row >= lo) {
        const long long t = t0 + row, tok = tok0 + (t - begin);
        const uint4* ks = reinterpret_cast<const uint4*>(static_cast<const char*>(p.k_new) + ((size_t)tok * p.k_new_token + (size_t)h * p.k_new_head) * es);
        const uint4* vs = reinterpret_cast<const uint4*>(static_cast<const char*>(p.v_new) + ((size_t)tok * p.v_new_token + (size_t)h * p.v_new_head) * es);
        a = __ldg(ks + c0);
        c = __ldg(ks + c1);
        const uint4 v0 = __ldg(vs + 2 * l), v1 = __ldg(vs + 2 * l + 1);
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
          uint4* vd = reinterpret_cast<uint4*>(static_cast<char*>(p.v) + at);
          kd[c0] = a;
          kd[c1] = c;
          vd[2 * l] = v0;
          vd[2 * l + 1] = v1;
        }
        if (p.q) {
          const char* qs = static_cast<const char*>(p.q) + ((size_t)tok * p.q_token + (size_t)h * p.group * p.q_head) * es;
          char* qd = static_cast<char*>(p.q_out) + ((size_t)tok * p.q_out_token + (size_t)h * p.group * p.q_out_head) * es;
          // four heads at a time, all loads before the stores (plain loads: q_out may be q itself)
          for (int g = 0; g < p.group; g += 4) {
            uint4 x[4], y[4];
#pragma unroll
            for (int i = 0; i < 4; ++i)
              if (g + i < p.group) {
                const uint4* s = reinterpret_cast<const uint4*>(qs + (size_t)(g + i) * p.q_head * es);
                x[i] = s[c0];
                y[i] = s[c1];
              }
#pragma unroll
            for (int i = 0; i < 4; ++i)
              if (g + i < p.group) {
                if (rotate) rotate_pieces<T>(x[i], y[i], cs, sn, p.pairs);
                uint4* o = reinterpret_cast<uint4*>(qd + (size_t)(g + i) * p.q_out_head * es);
                o[c0] = x[i];
                o[c1] = y[i];
              }
          }
        }
      } else {
        a = kd[c0];
        c = kd[c1];
      }
    }
    if (p.bounds) {
      // over the warp's rows (all of one page); lanes without a row take their partner's
      uint4 n0 = a, n1 = c, x0 = a, x1 = c;
      uint32_t* w[4] = {reinterpret_cast<uint32_t*>(&n0), reinterpret_cast<uint32_t*>(&n1), reinterpret_cast<uint32_t*>(&x0),
                        reinterpret_cast<uint32_t*>(&x1)};
      bool any = in;
#pragma unroll
      for (int o = LPR; o < 32; o <<= 1) {
        const bool theirs = __shfl_xor_sync(0xffffffffu, (int)any, o) != 0;
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const uint32_t x = __shfl_xor_sync(0xffffffffu, w[j][i], o);
            if (theirs) w[j][i] = !any ? x : j < 2 ? T::min2(w[j][i], x) : T::max2(w[j][i], x);
          }
        any = any || theirs;
      }
      if (lane < LPR) {
        const int grp = (r0 + warp * RPW) / RPW;
        s_red[grp][0][c0] = n0; s_red[grp][0][c1] = n1;
        s_red[grp][1][c0] = x0; s_red[grp][1][c1] = x1;
      }
    }
  }
  if (!p.bounds) return;
  __syncthreads();
  // ---- the touched pages' bounds: over their groups of rows (those that hold a row)
  for (int i = tid; i < 4 * LPR * ((hi - first + ps - 1) >> p.page_shift); i += NT) {
    const int c = i % (2 * LPR), side = i / (2 * LPR) % 2, page = (first >> p.page_shift) + i / (4 * LPR);
    const int g0 = (page << p.page_shift) / RPW, rows_end = ((page + 1) << p.page_shift) < hi ? (page + 1) << p.page_shift : hi;
    const int g1 = (rows_end + RPW - 1) / RPW;
    uint4 r = s_red[g0][side][c];
    uint32_t* rr = reinterpret_cast<uint32_t*>(&r);
    for (int g = g0 + 1; g < g1; ++g) {
      const uint4 x = s_red[g][side][c];
      const uint32_t* xx = reinterpret_cast<const uint32_t*>(&x);
#pragma unroll
      for (int e = 0; e < 4; ++e) rr[e] = side == 0 ? T::min2(rr[e], xx[e]) : T::max2(rr[e], xx[e]);
    }
    const int phys = __ldg(table + page);
    if (phys >= 0 && phys < p.n_pages)
      reinterpret_cast<uint4*>(static_cast<char*>(p.bounds) + (((size_t)phys * p.hkv + h) * 2 + side) * D * es)[c] = r;
  }
}

// 256 threads per CTA where items hold few new rows (decoding: the rows of earlier calls, read for the bounds, are then a
// single pass and the time is latency), 128 and five CTAs per multiprocessor otherwise.  One token of one sequence, 32 / 8
// heads of 64: 4.1 us a call against 5.2 with 128 threads; 15.8K tokens, 24 / 8 heads of 128: 68 us (4.8 TB/s) against 74.
template <typename T, int D>
static cudaError_t launch_append_t(const AppendProblem& p, cudaStream_t st) {
  const dim3 grid(p.items, p.hkv);
  return p.total_q <= 16ll * p.items ? launch_pdl(paged_append_kernel<T, D, 256>, grid, dim3(256), 0, st, p)
                                     : launch_pdl(paged_append_kernel<T, D, 128>, grid, dim3(128), 0, st, p);
}

cudaError_t launch_paged_append(const AppendProblem& p, bool bf16, cudaStream_t st) {
  if (p.d == 64) return bf16 ? launch_append_t<Bf16, 64>(p, st) : launch_append_t<Fp16, 64>(p, st);
  return bf16 ? launch_append_t<Bf16, 128>(p, st) : launch_append_t<Fp16, 128>(p, st);
}

}  // namespace tkphi
