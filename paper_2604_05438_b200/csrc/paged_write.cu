// New tokens into a paged cache, with head norms on the way, into pages of 16 or of 8 bits.
//
// For token i of sequence b (cache position t = kv_len - q_len + i, angle position x = positions[i] or t), each key and
// query head h on its own:
//   norm      u = h * w / sqrt(mean(h^2) + eps), where the side has weights (otherwise u = h)
//   rotation  pair (a, c) of u -> (a cos w - c sin w, c cos w + a sin w), w = x * inv_freq[pair]
// in 32 bits.  A 16-bit cache takes keys rounded once and values as they are; an 8-bit one takes both as codes and a power
// of two per row (held8.cuh), rounded once from the 32-bit numbers.  Queries are rounded once to the element type.  Key
// bounds of the touched pages are recomputed from what the pages hold, those of earlier calls read back.
//
// Bound: memory.  As in the append without norms, a CTA takes 64 positions (a page of 128) of one KV head, 8 lanes per row
// at head_dim 128 (4 at 64), a lane owning the two 8-element pieces whose elements are each other's partners in the
// rotation.  A row's sum of squares and its largest magnitude are two or three shuffles between its lanes; all lanes of a
// warp take part in them, with zeros where they have no row.
// Measured: 15.8K tokens, 24 / 8 heads of 128, norms, half of the dims rotated, bounds, 16-bit cache: 80 us (4.1 TB/s);
// 23.6K tokens, 32 / 8 heads of 64, rotated, 8-bit cache: 56 us (4.8 TB/s); one token 4.8-5.0 us a call.  The chain of a row is the
// bound (loads, sums over its lanes, conversions) at the occupancy that its registers leave: what helped were all loads of a row
// before anything else, no spilled registers, angles in fixed point with frequencies in shared memory, 32-byte stores.  Tried
// and no faster: several heads per CTA with the sines shared, packed 32-bit pairs, the next row's loads issued ahead into
// registers or by asynchronous copies into shared memory, weights in shared memory, five CTAs with 96 registers.
#include "held8.cuh"

namespace tkphi {

// Writes pieces c0 and c1 of a row.  Neighbours are 32 bytes: two stores of 16 would each write half of every sector.
__device__ __forceinline__ void put_pieces(void* row, int c0, int c1, bool wide, const uint4& a, const uint4& c) {
  uint4* p = static_cast<uint4*>(row);
  if (wide) {
    asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p + c0), "r"(a.x), "r"(a.y), "r"(a.z), "r"(a.w), "r"(c.x),
                 "r"(c.y), "r"(c.z), "r"(c.w) : "memory");
  } else {
    p[c0] = a;
    p[c1] = c;
  }
}
template <typename T>
__device__ __forceinline__ void unpack_piece(const uint4& v, float* x) {
  const uint32_t* w = reinterpret_cast<const uint32_t*>(&v);
#pragma unroll
  for (int i = 0; i < 4; ++i) { x[2 * i] = T::lo(w[i]); x[2 * i + 1] = T::hi(w[i]); }
}
template <typename T>
__device__ __forceinline__ uint4 pack_piece(const float* x) {
  return make_uint4(T::pack(x[0], x[1]), T::pack(x[2], x[3]), T::pack(x[4], x[5]), T::pack(x[6], x[7]));
}
// A rotated pair: turns per position, less whole ones, in units of 2^-64, and 2 pi / 2^32; that is NaN where the frequency is infinite
// or no number, for which fixed point has nothing.
struct __align__(16) Turn { unsigned long long per; float unit; };
// Cosine and sine of an angle of a / 2^32 turns (unit: 2 pi / 2^32): less the nearest quarter turn, an angle |y| <= pi / 4 is
// left, of which the Taylor polynomials of degree 9 and 10 are off by y^11 / 11! = 1.8e-9 and y^12 / 12! = 1.1e-10, less than 32 bits hold.
// (sincospif took about 125 instructions of a pair, two thirds of the kernel's.)
__device__ __forceinline__ void turn_cos_sin(uint32_t a, float unit, float& cs, float& sn) {
  const uint32_t quarter = a + 0x20000000u;                  // its top two bits: the quarter
  const float y = (float)(int)(a - (quarter & 0xc0000000u)) * unit, z = y * y;
  const float s = fmaf(y * z, fmaf(z, fmaf(z, fmaf(z, 2.75573192e-6f, -1.98412698e-4f), 8.33333333e-3f), -1.66666667e-1f), y);
  const float c = fmaf(z, fmaf(z, fmaf(z, fmaf(z, fmaf(z, -2.75573192e-7f, 2.48015873e-5f), -1.38888889e-3f), 4.16666667e-2f), -0.5f), 1.f);
  const bool odd = quarter & 0x40000000u;
  sn = __uint_as_float(__float_as_uint(odd ? c : s) ^ (quarter & 0x80000000u));
  cs = __uint_as_float(__float_as_uint(odd ? s : c) ^ ((quarter + 0x40000000u) & 0x80000000u));
}
// Of a lane's eight pairs at position x.
template <int LPR>
__device__ __forceinline__ void row_angles(float (&cs)[8], float (&sn)[8], unsigned long long x, const Turn* turn) {
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const Turn t = turn[i * LPR];
    turn_cos_sin((uint32_t)((x * t.per + 0x80000000ull) >> 32), t.unit, cs[i], sn[i]);
  }
}
// x: the lane's two pieces of 8 dims.
__device__ __forceinline__ void rotate16(float (&x)[16], const float (&cs)[8], const float (&sn)[8], bool pairs) {
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    // partners: neighbours, pair i of the 16, or the same place in the two pieces
    const float a = pairs ? x[2 * i] : x[i], c = pairs ? x[2 * i + 1] : x[8 + i];
    const float u = a * cs[i] - c * sn[i], w = c * cs[i] + a * sn[i];
    if (pairs) { x[2 * i] = u; x[2 * i + 1] = w; } else { x[i] = u; x[8 + i] = w; }
  }
}
template <int LPR>
__device__ __forceinline__ float row_squares(const float (&x)[16]) {
  float s = 0.f;
#pragma unroll
  for (int i = 0; i < 16; ++i) s = fmaf(x[i], x[i], s);
#pragma unroll
  for (int o = 1; o < LPR; o <<= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
  return s;
}
__device__ __forceinline__ void weigh16(float (&x)[16], float r, const float* weight, int c0, int c1) {
  float w[16];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float4 v = __ldg(reinterpret_cast<const float4*>(weight + 8 * (i < 2 ? c0 : c1)) + (i & 1));
    w[4 * i] = v.x; w[4 * i + 1] = v.y; w[4 * i + 2] = v.z; w[4 * i + 3] = v.w;
  }
#pragma unroll
  for (int i = 0; i < 16; ++i) x[i] = x[i] * r * w[i];
}
// Norm of a head.  True if the result is not to be used: v = mean(x^2) + eps is right where squares that 32 bits do not hold do not
// count beside it and none overflows, which leaves out bf16 elements beyond 2^60, or of 2^-40 and less with as small an eps.
template <typename T, int LPR>
__device__ __forceinline__ bool norm16(float (&x)[16], const float* weight, int c0, int c1, float eps) {
  const float v = fmaf(row_squares<LPR>(x), 1.f / (16 * LPR), eps);
  weigh16(x, rsqrtf(v), weight, c0, c1);
  return T::kBf16 && !(v >= 0x1p-80f && v < INFINITY);
}
// Norm of any head: scaled by a power of two, so that its largest element or the root of eps is about 1.  (A head of zeros without
// eps, infinities and NaN: as they are.)
template <int LPR>
__device__ __forceinline__ void norm16_scaled(float (&x)[16], const float* weight, int c0, int c1, float eps) {
  uint32_t most = 0;
#pragma unroll
  for (int i = 0; i < 16; ++i) most = max(most, __float_as_uint(x[i]) & 0x7fffffffu);
#pragma unroll
  for (int o = 1; o < LPR; o <<= 1) most = max(most, __shfl_xor_sync(0xffffffffu, most, o));
  const uint32_t field = min(max(max(most, __float_as_uint(sqrtf(eps))) >> 23, 1u), 253u);
  const float f = most < 0x7f800000u ? __uint_as_float((254u - field) << 23) : 1.f;
#pragma unroll
  for (int i = 0; i < 16; ++i) x[i] *= f;
  weigh16(x, rsqrtf(fmaf(row_squares<LPR>(x), 1.f / (16 * LPR), eps * f * f)), weight, c0, c1);
}
// Scale byte of the row that LPR lanes hold.
template <int LPR>
__device__ __forceinline__ uint32_t row_byte(const float (&x)[16]) {
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 16; ++i) m = max(m, __float_as_uint(x[i]) & 0x7fffffffu);
#pragma unroll
  for (int o = 1; o < LPR; o <<= 1) m = max(m, __shfl_xor_sync(0xffffffffu, m, o));
  return held_byte(m);
}
__device__ __forceinline__ uint4 row_codes(const float (&x)[16], uint32_t e) {
  if (e == 255u) return make_uint4(0x7f7f7f7fu, 0x7f7f7f7fu, 0x7f7f7f7fu, 0x7f7f7f7fu);
  const float r = held_inverse(e);
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) w[i] = pack_codes(x[4 * i] * r, x[4 * i + 1] * r, x[4 * i + 2] * r, x[4 * i + 3] * r);
  return make_uint4(w[0], w[1], w[2], w[3]);
}

// A row's key as the cache holds it, as 16-bit pieces.
template <typename T, bool HELD>
__device__ __forceinline__ void held_key(const WriteProblem& wp, size_t at, size_t scale_at, int c0, int c1, uint4& a, uint4& c) {
  if (HELD) {
    const uint2* kd = reinterpret_cast<const uint2*>(static_cast<const char*>(wp.a.k) + at);
    const uint2 k0 = kd[c0], k1 = kd[c1];
    const float s = held_scale(wp.held.k_scales[scale_at]);
    const uint2 w0 = held_values<T>(k0.x, s), w1 = held_values<T>(k0.y, s);
    const uint2 w2 = held_values<T>(k1.x, s), w3 = held_values<T>(k1.y, s);
    a = make_uint4(w0.x, w0.y, w1.x, w1.y);
    c = make_uint4(w2.x, w2.y, w3.x, w3.y);
  } else {
    const uint4* kd = reinterpret_cast<const uint4*>(static_cast<const char*>(wp.a.k) + at * 2);
    a = kd[c0];
    c = kd[c1];
  }
}
// Minimum and maximum over the warp's rows (all of one page).  Lanes without a row take another row's; then the lanes of two rows
// share the work: one takes the first pieces, the other the second, then one minima, the other maxima.
template <typename T, int LPR>
__device__ __forceinline__ void warp_bounds(bool in, const uint4& a, const uint4& c, int c0, int c1, uint4 (*to)[2 * LPR]) {
  const int lane = threadIdx.x & 31, l = lane % LPR;
  const unsigned have = __ballot_sync(0xffffffffu, in);
  if (have == 0) return;
  uint32_t k[8] = {a.x, a.y, a.z, a.w, c.x, c.y, c.z, c.w};
  if (have != 0xffffffffu) {
    const int from = in ? lane : (__ffs(have) - 1) / LPR * LPR + l;
#pragma unroll
    for (int i = 0; i < 8; ++i) k[i] = __shfl_sync(0xffffffffu, k[i], from);
  }
  const bool second = lane & 16, most = lane & 8;
  uint32_t m[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t mine = second ? k[4 + i] : k[i], theirs = __shfl_xor_sync(0xffffffffu, second ? k[i] : k[4 + i], 16);
    const uint32_t lo2 = T::min2(mine, theirs), hi2 = T::max2(mine, theirs);
    const uint32_t other = __shfl_xor_sync(0xffffffffu, most ? lo2 : hi2, 8);
    m[i] = most ? T::max2(hi2, other) : T::min2(lo2, other);
  }
  if (LPR == 4) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t other = __shfl_xor_sync(0xffffffffu, m[i], 4);
      m[i] = most ? T::max2(m[i], other) : T::min2(m[i], other);
    }
  }
  if (LPR == 8 || (lane & 4) == 0) to[most][second ? c1 : c0] = make_uint4(m[0], m[1], m[2], m[3]);
}

// The heads of the warp's rows that s_again marks, once more, with scaled squares; then those rows' part of the bounds from the cache.
// One head after the other in one copy of the code, called after everything else, because it is seldom needed: a branch in
// each norm, or a call in the loop over rows, takes a single token 0.5 to 1.8 us.
struct AgainRows {
  int h, c0, c1;
  bool rotate;
  int b;
  long long tok0, begin, t0;
  int first, lo, hi;
};
template <typename T, int D, int NT, bool HELD>
__device__ __noinline__ void write_again(const WriteProblem& wp, const AgainRows& r, const uint32_t* s_again, const Turn* s_turn,
                                         uint4 (*s_red)[2][2 * (D / 16)]) {
  constexpr int LPR = D / 16, RPW = 32 / LPR, RPP = NT / LPR;
  const AppendProblem& p = wp.a;
  const int tid = threadIdx.x, warp = tid >> 5, l = tid % LPR, ps = 1 << p.page_shift;
  const int* table = p.table + (size_t)r.b * p.max_pages + (r.t0 >> p.page_shift);
  __syncwarp();
#pragma unroll 1
  for (int r0 = r.first / RPP * RPP; r0 < r.hi; r0 += RPP) {
    const int row = r0 + tid / LPR;
    const bool in = row >= r.first && row < r.hi, fresh = in && row >= r.lo;
    const uint32_t again = fresh ? s_again[row] : 0;
    if (!__any_sync(0xffffffffu, again != 0)) continue;
    const int page = in ? __ldg(table + (row >> p.page_shift)) : -1;
    const bool ok = page >= 0 && page < p.n_pages;
    const int phys = ok ? page : 0;
    const size_t at = (size_t)phys * p.stride_page + (size_t)r.h * p.stride_head + (size_t)(row & (ps - 1)) * p.stride_token;
    const size_t scale_at = ((size_t)phys * p.hkv + r.h) * ps + (row & (ps - 1));
    const long long t = r.t0 + row, tok = fresh ? r.tok0 + (t - r.begin) : r.tok0;
    float cs[8], sn[8];
    if (r.rotate) {
      const unsigned long long x = (unsigned long long)(p.positions ? __ldg(p.positions + tok) : t);
      row_angles<LPR>(cs, sn, x, s_turn + l);
    }
#pragma unroll 1
    for (int n = 0; n <= p.group; ++n) {
      const bool mine = again >> n & 1u;
      if (!__any_sync(0xffffffffu, mine)) continue;
      const int head = n == 0 ? r.h : r.h * p.group + n - 1;
      const size_t from = n == 0 ? (size_t)tok * p.k_new_token + (size_t)head * p.k_new_head : (size_t)tok * p.q_token + (size_t)head * p.q_head;
      const uint4* src = reinterpret_cast<const uint4*>(static_cast<const char*>(n == 0 ? p.k_new : p.q) + from * 2);
      uint4 a = make_uint4(0, 0, 0, 0), c = a;
      if (mine) { a = src[r.c0]; c = src[r.c1]; }
      float x[16];
      unpack_piece<T>(a, x);
      unpack_piece<T>(c, x + 8);
      norm16_scaled<LPR>(x, n == 0 ? wp.k_weight + head * wp.k_weight_head : wp.q_weight + head * wp.q_weight_head, r.c0, r.c1, wp.eps);
      if (r.rotate) rotate16(x, cs, sn, p.pairs);
      if (HELD && n == 0) {
        const uint32_t e = row_byte<LPR>(x);
        const uint4 code = row_codes(x, e);
        if (mine && ok) {
          uint2* kd = reinterpret_cast<uint2*>(static_cast<char*>(p.k) + at);
          kd[r.c0] = make_uint2(code.x, code.y);
          kd[r.c1] = make_uint2(code.z, code.w);
          if (l == 0) wp.held.k_scales[scale_at] = (uint8_t)e;
        }
      } else if (mine && (n > 0 || ok)) {
        char* to = n == 0 ? static_cast<char*>(p.k) + at * 2 : static_cast<char*>(p.q_out) + ((size_t)tok * p.q_out_token + (size_t)head * p.q_out_head) * 2;
        put_pieces(to, r.c0, r.c1, false, pack_piece<T>(x), pack_piece<T>(x + 8));
      }
    }
    if (p.bounds && __any_sync(0xffffffffu, again & 1u)) {
      __syncwarp();
      uint4 a = make_uint4(0, 0, 0, 0), c = a;
      if (in && ok) held_key<T, HELD>(wp, at, scale_at, r.c0, r.c1, a, c);
      warp_bounds<T, LPR>(in, a, c, r.c0, r.c1, s_red[(r0 + warp * RPW) / RPW]);
    }
  }
}

// An item is one KV head of 64 aligned cache positions (128 where the page is that long): whole pages, so that their
// bounds need no other CTA.
template <typename T, int D, int NT, bool HELD>
__global__ void __launch_bounds__(NT, NT == 128 ? 4 : 2) paged_write_kernel(const __grid_constant__ WriteProblem wp) {
  constexpr int LPR = D / 16;                  // lanes of a row
  constexpr int RPW = 32 / LPR;                // rows of a warp
  constexpr int RPP = NT / LPR;                // rows of one pass of the CTA
  constexpr size_t es = 2;
  const AppendProblem& p = wp.a;
  __shared__ long long s_find[4];              // sequence, its first token row, cache length, first new position
  __shared__ int s_item;
  __shared__ Turn s_turn[D / 2];
  __shared__ uint4 s_red[128 / RPW][2][2 * LPR];     // a warp's rows: their minimum and maximum
  __shared__ uint32_t s_again[T::kBf16 ? 128 : 1];   // of a new row of the item: heads to be written once more
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  if (T::kBf16 && tid < 128) s_again[tid] = 0;
  const int h = blockIdx.y, span_shift = p.page_shift > 6 ? p.page_shift : 6;
  pdl_wait();
  pdl_launch_next();
  // The product of a pair's turns with a position drops whole turns by itself, exactly: the angle is off by position * 2^-64 turns,
  // and by the product's rounding to 2^-53 of inv_freq.
  if (tid >= NT / 2 && tid - NT / 2 < p.rot / 2) {
    const float freq = __ldg(p.inv_freq + tid - NT / 2);
    const double t = (double)freq * 0.15915494309189533577;
    // (the pairs of one place in all lanes beside each other, so that a warp's reads of them spread over the banks)
    s_turn[(tid & 7) * LPR + (tid - NT / 2) / 8] = Turn{__double2ull_rz((t - floor(t)) * 18446744073709551616.0),
                                fabsf(freq) < INFINITY ? 1.46291807926715968e-9f : __uint_as_float(0x7fc00000u)};
  }

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
  // (in the form for many rows: where latency counts, the choice costs more than it gives)
  const bool wide = NT == 128 && wp.wide && c1 == c0 + 1;
  const float* kw = wp.k_weight ? wp.k_weight + h * wp.k_weight_head : nullptr;
  // page ids one pass ahead
  auto page_of = [&](int r0) {
    const int row = r0 + tid / LPR;
    return row >= first && row < hi ? __ldg(table + (row >> p.page_shift)) : -1;
  };
  const int r_begin = first / RPP * RPP;
  int page_next = page_of(r_begin);
  bool any_again = false;
  for (int r0 = r_begin; r0 < hi; r0 += RPP) {
    const int row = r0 + tid / LPR;
    const bool in = row >= first && row < hi, fresh = in && row >= lo;
    uint4 a = make_uint4(0, 0, 0, 0), c = a;              // the held key, as 16-bit pieces, for the bounds
    int phys = page_next;
    page_next = page_of(r0 + RPP);
    // a page id outside the cache: its rows are dropped, the queries of its tokens are written all the same
    const bool ok = phys >= 0 && phys < p.n_pages;
    const bool bad = in && !ok && l == 0;
    phys = ok ? phys : 0;
    const size_t at = (size_t)phys * p.stride_page + (size_t)h * p.stride_head + (size_t)(row & (ps - 1)) * p.stride_token;
    const size_t scale_at = ((size_t)phys * p.hkv + h) * ps + (row & (ps - 1));
    if (__any_sync(0xffffffffu, fresh)) {
      const long long t = t0 + row, tok = fresh ? tok0 + (t - begin) : tok0;
      const uint4* ks = reinterpret_cast<const uint4*>(static_cast<const char*>(p.k_new) + ((size_t)tok * p.k_new_token + (size_t)h * p.k_new_head) * es);
      const uint4* vs = reinterpret_cast<const uint4*>(static_cast<const char*>(p.v_new) + ((size_t)tok * p.v_new_token + (size_t)h * p.v_new_head) * es);
      uint4 ka = a, kc = a, v0 = a, v1 = a;
      const char* qs = static_cast<const char*>(p.q) + ((size_t)tok * p.q_token + (size_t)h * p.group * p.q_head) * es;
      char* qd = static_cast<char*>(p.q_out) + ((size_t)tok * p.q_out_token + (size_t)h * p.group * p.q_out_head) * es;
      uint4 u[4], w[4];
      auto load_queries = [&](int g) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          u[i] = w[i] = make_uint4(0, 0, 0, 0);
          if (g + i < p.group && fresh) {
            const uint4* s = reinterpret_cast<const uint4*>(qs + (size_t)(g + i) * p.q_head * es);
            u[i] = s[c0];
            w[i] = s[c1];
          }
        }
      };
      float cs[8], sn[8];
      if (fresh) {
        ka = __ldg(ks + c0);
        kc = __ldg(ks + c1);
        v0 = __ldg(vs + 2 * l);
        v1 = __ldg(vs + 2 * l + 1);
      }
      if (p.q) load_queries(0);
      if (fresh) {
        if (rotate) {
          const unsigned long long x = (unsigned long long)(p.positions ? __ldg(p.positions + tok) : t);
          row_angles<LPR>(cs, sn, x, s_turn + l);
        }
      }
      float x[16];
      unpack_piece<T>(ka, x);
      unpack_piece<T>(kc, x + 8);
      uint32_t again = 0;                                 // heads whose norm needs scaled squares: the key, the group's queries
      if (kw && norm16<T, LPR>(x, kw, c0, c1, wp.eps)) again = 1;
      if (fresh && rotate) rotate16(x, cs, sn, p.pairs);
      if (HELD) {
        const uint32_t ke = row_byte<LPR>(x);
        const uint4 kcode = row_codes(x, ke);
        float y[16];
        unpack_piece<T>(v0, y);
        unpack_piece<T>(v1, y + 8);
        const uint32_t ve = row_byte<LPR>(y);
        if (ok && fresh) {
          uint2* kd = reinterpret_cast<uint2*>(static_cast<char*>(p.k) + at);
          kd[c0] = make_uint2(kcode.x, kcode.y);
          kd[c1] = make_uint2(kcode.z, kcode.w);
          reinterpret_cast<uint4*>(static_cast<char*>(p.v) + at)[l] = row_codes(y, ve);
          if (l == 0) {
            wp.held.k_scales[scale_at] = (uint8_t)ke;
            wp.held.v_scales[scale_at] = (uint8_t)ve;
          }
        }
        if (p.bounds && fresh) {
          const float s = held_scale(ke);
          const uint2 w0 = held_values<T>(kcode.x, s), w1 = held_values<T>(kcode.y, s);
          const uint2 w2 = held_values<T>(kcode.z, s), w3 = held_values<T>(kcode.w, s);
          a = make_uint4(w0.x, w0.y, w1.x, w1.y);
          c = make_uint4(w2.x, w2.y, w3.x, w3.y);
        }
      } else if (fresh) {
        a = pack_piece<T>(x);
        c = pack_piece<T>(x + 8);
        if (ok) {
          put_pieces(static_cast<char*>(p.k) + at * es, c0, c1, wide, a, c);
          put_pieces(static_cast<char*>(p.v) + at * es, 2 * l, 2 * l + 1, NT == 128 && wp.wide, v0, v1);
        }
      }
      if (p.q) {
        // four heads at a time, all loads before the stores (plain loads: q_out may be q itself)
        for (int g = 0; g < p.group; g += 4) {
          if (g > 0) load_queries(g);
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if (g + i < p.group) {
              float z[16];
              unpack_piece<T>(u[i], z);
              unpack_piece<T>(w[i], z + 8);
              // (such a head stays as it is for now: q_out may be q itself)
              const bool scale = wp.q_weight && norm16<T, LPR>(z, wp.q_weight + (h * p.group + g + i) * wp.q_weight_head, c0, c1, wp.eps);
              if (scale) again |= 2u << (g + i);
              if (fresh && !scale) {
                if (rotate) rotate16(z, cs, sn, p.pairs);
                put_pieces(qd + (size_t)(g + i) * p.q_out_head * es, c0, c1, wide, pack_piece<T>(z), pack_piece<T>(z + 8));
              }
            }
        }
      }
      if (T::kBf16 && fresh && again) {
        any_again = true;
        if (l == 0) s_again[row] = again;
      }
    }
    if (bad) atomicExch(p.status, kStatusBadPage);
    if (in && !fresh) {                                   // a row of an earlier call
      held_key<T, HELD>(wp, at, scale_at, c0, c1, a, c);
    }
    if (p.bounds) {
      warp_bounds<T, LPR>(in, a, c, c0, c1, s_red[(r0 + warp * RPW) / RPW]);
    }
  }
  if (T::kBf16 && __any_sync(0xffffffffu, any_again)) {
    const AgainRows r{h, c0, c1, rotate, b, tok0, begin, t0, first, lo, hi};
    write_again<T, D, NT, HELD>(wp, r, s_again, s_turn, s_red);
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

// 256 threads per CTA where items hold few new rows (decoding: a single pass, all latency), 128 otherwise.
template <typename T, int D, bool HELD>
static cudaError_t launch_write_t(const WriteProblem& p, cudaStream_t st) {
  const dim3 grid(p.a.items, p.a.hkv);
  return p.a.total_q <= 16ll * p.a.items ? launch_pdl(paged_write_kernel<T, D, 256, HELD>, grid, dim3(256), 0, st, p)
                                         : launch_pdl(paged_write_kernel<T, D, 128, HELD>, grid, dim3(128), 0, st, p);
}
template <typename T, int D>
static cudaError_t launch_write_d(const WriteProblem& p, cudaStream_t st) {
  return p.held.k_scales ? launch_write_t<T, D, true>(p, st) : launch_write_t<T, D, false>(p, st);
}

cudaError_t launch_paged_write(const WriteProblem& q, bool bf16, cudaStream_t st) {
  WriteProblem p = q;
  const AppendProblem& a = p.a;
  uintptr_t bits = reinterpret_cast<uintptr_t>(a.q_out);
  long long strides = a.q ? a.q_out_token | a.q_out_head : 0;
  if (!p.held.k_scales) {
    bits |= reinterpret_cast<uintptr_t>(a.k) | reinterpret_cast<uintptr_t>(a.v);
    strides |= a.stride_page | a.stride_head | a.stride_token;
  }
  p.wide = (bits & 31u) == 0 && (strides & 15) == 0;
  if (p.a.d == 64) return bf16 ? launch_write_d<Bf16, 64>(p, st) : launch_write_d<Fp16, 64>(p, st);
  return bf16 ? launch_write_d<Bf16, 128>(p, st) : launch_write_d<Fp16, 128>(p, st);
}

}  // namespace tkphi
