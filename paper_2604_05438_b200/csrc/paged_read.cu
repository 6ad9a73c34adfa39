// Rows of an 8-bit paged cache back as 16-bit rows: out[cu_rows[b] + i] = codes * 2^(e - 127) of position first[b] + i of
// sequence b, for keys and values, rounded once to the element type (exact in bf16).
//
// Bound: memory, 2 (d + 1) bytes in and 4 d out per row and head.  A thread has 16 codes of a row and writes 32 bytes;
// a CTA takes 64 output rows of one KV head, two rows per thread with all loads before the stores.
#include "held8.cuh"

namespace tkphi {

constexpr int kReadRows = 64;
constexpr int kReadThreads = 256;

template <typename T, int D>
__global__ void __launch_bounds__(kReadThreads) paged_read_kernel(const __grid_constant__ ReadProblem p) {
  constexpr int LPR = D / 16, RPP = kReadThreads / LPR, PASSES = kReadRows / RPP > 0 ? kReadRows / RPP : 1;
  __shared__ int s_seq;
  const int tid = threadIdx.x, lane = tid & 31, h = blockIdx.y;
  const long long row0 = (long long)blockIdx.x * kReadRows;
  pdl_wait();
  pdl_launch_next();
  if (tid < 32) {
    // the sequence of the first row
    int b = 0;
    for (int s = 0; s < p.batch; s += 32) {
      const bool before = s + lane < p.batch && __ldg(p.cu_rows + s + lane + 1) <= row0;
      const unsigned m = __ballot_sync(0xffffffffu, before);
      b += __popc(m);
      if (m != 0xffffffffu) break;
    }
    if (lane == 0) s_seq = b;
  }
  __syncthreads();
  int b = s_seq;
  const int l = tid % LPR, ps = 1 << p.page_shift;
  uint4 kw[PASSES], vw[PASSES];
  uint32_t ke[PASSES], ve[PASSES];
  bool ok[PASSES];
#pragma unroll
  for (int i = 0; i < PASSES; ++i) {
    const long long row = row0 + i * RPP + tid / LPR;
    ok[i] = false;
    if (row >= p.total_rows || (RPP > kReadRows && tid / LPR >= kReadRows)) continue;
    while (b < p.batch && __ldg(p.cu_rows + b + 1) <= row) ++b;
    if (b >= p.batch) continue;
    const long long pos = row - __ldg(p.cu_rows + b) + (p.first ? __ldg(p.first + b) : 0ll);
    const long long have = __ldg(p.kv_lens + b);
    if (pos < 0 || pos >= have || pos >= p.max_kv) continue;       // (a replay with shorter device lengths: not written)
    const int page = __ldg(p.table + (size_t)b * p.max_pages + (pos >> p.page_shift));
    if (page < 0 || page >= p.n_pages) {
      if (l == 0) atomicExch(p.status, kStatusBadPage);
      continue;
    }
    ok[i] = true;
    const int slot = (int)(pos & (ps - 1));
    const size_t at = (size_t)page * p.stride_page + (size_t)h * p.stride_head + (size_t)slot * p.stride_token;
    const size_t scale_at = ((size_t)page * p.hkv + h) * ps + slot;
    if (p.k_out) { kw[i] = __ldg(reinterpret_cast<const uint4*>(p.k + at) + l); ke[i] = __ldg(p.held.k_scales + scale_at); }
    if (p.v_out) { vw[i] = __ldg(reinterpret_cast<const uint4*>(p.v + at) + l); ve[i] = __ldg(p.held.v_scales + scale_at); }
  }
#pragma unroll
  for (int i = 0; i < PASSES; ++i) {
    if (!ok[i]) continue;
    const size_t row = (size_t)(row0 + i * RPP + tid / LPR);
    auto put = [&](void* out, long long row_stride, long long head_stride, const uint4& w, uint32_t e) {
      const float s = held_scale(e);
      const uint2 a = held_values<T>(w.x, s), c = held_values<T>(w.y, s), d = held_values<T>(w.z, s), f = held_values<T>(w.w, s);
      uint4* o = reinterpret_cast<uint4*>(static_cast<uint16_t*>(out) + row * row_stride + (size_t)h * head_stride + l * 16);
      o[0] = make_uint4(a.x, a.y, c.x, c.y);
      o[1] = make_uint4(d.x, d.y, f.x, f.y);
    };
    if (p.k_out) put(p.k_out, p.k_row, p.k_head, kw[i], ke[i]);
    if (p.v_out) put(p.v_out, p.v_row, p.v_head, vw[i], ve[i]);
  }
}

cudaError_t launch_paged_read(const ReadProblem& p, bool bf16, cudaStream_t st) {
  const dim3 grid((unsigned)((p.total_rows + kReadRows - 1) / kReadRows), p.hkv), block(kReadThreads);
  if (p.d == 64)
    return bf16 ? launch_pdl(paged_read_kernel<Bf16, 64>, grid, block, 0, st, p) : launch_pdl(paged_read_kernel<Fp16, 64>, grid, block, 0, st, p);
  return bf16 ? launch_pdl(paged_read_kernel<Bf16, 128>, grid, block, 0, st, p) : launch_pdl(paged_read_kernel<Fp16, 128>, grid, block, 0, st, p);
}

// ---------------------------------------------------------------- for attention of many rows
// The caches of the sequences with many rows as 16-bit pages of 128 rows in the workspace, [page][head][slot][dim], one
// sequence's pages behind another's, and a page table of them; codes times powers of two, so nothing is lost.  A CTA takes
// a page of one KV head.  Rows at or behind a sequence's length and on bad pages become 0.
template <typename T, int D>
__global__ void __launch_bounds__(kReadThreads) paged_expand_kernel(const __grid_constant__ PagedProblem p, const __grid_constant__ ExpandProblem x) {
  constexpr int LPR = D / 16, RPP = kReadThreads / LPR, PASSES = kExpandRows / RPP;
  __shared__ int s_seq, s_page;
  const int tid = threadIdx.x, lane = tid & 31, h = blockIdx.y;
  pdl_wait();
  pdl_launch_next();
  if (tid < 32) {
    int base = 0;
    if (lane == 0) s_seq = -1;
    for (int s = 0; s < p.batch; s += 32) {
      int n = 0;
      if (s + lane < p.batch && (long long)paged_q_len(p, s + lane) * p.group > p.rows_limit) n = (paged_kv_len(p, s + lane) + kExpandRows - 1) / kExpandRows;
      const int incl = warp_inclusive_scan(n) + base;
      if (incl > (int)blockIdx.x && incl - n <= (int)blockIdx.x) {           // one lane
        s_seq = s + lane;
        s_page = blockIdx.x - (incl - n);
      }
      base = __shfl_sync(0xffffffffu, incl, 31);
      if (base > (int)blockIdx.x) break;
    }
  }
  __syncthreads();
  const int b = s_seq;
  if (b < 0) return;                           // (a replay with shorter lengths)
  const int l = tid % LPR, ps = 1 << p.page_shift, len = paged_kv_len(p, b);
  if (h == 0 && tid == 0) x.table[(size_t)b * x.max_pages + s_page] = blockIdx.x;
  uint4 kw[PASSES], vw[PASSES];
  uint32_t ke[PASSES], ve[PASSES];
#pragma unroll
  for (int i = 0; i < PASSES; ++i) {
    kw[i] = vw[i] = make_uint4(0, 0, 0, 0);
    ke[i] = ve[i] = 0;
    const int pos = s_page * kExpandRows + i * RPP + tid / LPR;
    if (pos >= len) continue;
    const int page = __ldg(p.table + (size_t)b * p.max_pages + (pos >> p.page_shift));
    if (page < 0 || page >= p.n_pages) {
      if (l == 0) atomicExch(p.status, kStatusBadPage);
      continue;
    }
    const int slot = pos & (ps - 1);
    const size_t at = (size_t)page * x.stride_page + (size_t)h * x.stride_head + (size_t)slot * x.stride_token;
    const size_t scale_at = ((size_t)page * p.hkv + h) * ps + slot;
    kw[i] = __ldg(reinterpret_cast<const uint4*>(x.k + at) + l);
    vw[i] = __ldg(reinterpret_cast<const uint4*>(x.v + at) + l);
    ke[i] = __ldg(x.held.k_scales + scale_at);
    ve[i] = __ldg(x.held.v_scales + scale_at);
  }
  const size_t out = ((size_t)blockIdx.x * p.hkv + h) * kExpandRows;
#pragma unroll
  for (int i = 0; i < PASSES; ++i) {
    auto put = [&](void* to, const uint4& w, uint32_t e) {
      const float s = held_scale(e);
      const uint2 a = held_values<T>(w.x, s), c = held_values<T>(w.y, s), d = held_values<T>(w.z, s), f = held_values<T>(w.w, s);
      uint4* o = reinterpret_cast<uint4*>(static_cast<uint16_t*>(to) + (out + i * RPP + tid / LPR) * D + l * 16);
      o[0] = make_uint4(a.x, a.y, c.x, c.y);
      o[1] = make_uint4(d.x, d.y, f.x, f.y);
    };
    put(x.k_out, kw[i], ke[i]);
    put(x.v_out, vw[i], ve[i]);
  }
}

cudaError_t launch_paged_expand(const PagedProblem& p, const ExpandProblem& x, int d, bool bf16, int pages, cudaStream_t st) {
  const dim3 grid(pages, p.hkv), block(kReadThreads);
  if (d == 64)
    return bf16 ? launch_pdl(paged_expand_kernel<Bf16, 64>, grid, block, 0, st, p, x) : launch_pdl(paged_expand_kernel<Fp16, 64>, grid, block, 0, st, p, x);
  return bf16 ? launch_pdl(paged_expand_kernel<Bf16, 128>, grid, block, 0, st, p, x) : launch_pdl(paged_expand_kernel<Fp16, 128>, grid, block, 0, st, p, x);
}

}  // namespace tkphi
