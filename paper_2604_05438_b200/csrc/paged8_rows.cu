// Attention of few query rows over an 8-bit paged cache: sequences with at most 16 rows (tokens x query heads of a KV head),
// and the page-selected form, where every token of a KV head reads a page list of its own.
//
//   y = sum_t p_t v_t / sum_t p_t,  p_t = exp(scale * q.k_t - m),  lse = m + log sum_t p_t   over the visible keys t
//   k_t = a_t * (its codes),  v_t = b_t * (its codes),  a_t and b_t powers of two
//
// in one pass with the running maximum m and sum.  Work is dealt out and joined as over a 16-bit cache (paged_walk.cuh), in
// tiles of 128 keys.  Bound: memory, 2 * (head_dim + 1) bytes per key against 16 rows of work; with half the bytes of a
// 16-bit cache the instructions per key count, too.  So:
//   - both products run as fp16 products of the codes, which fp16 holds exactly: one conversion instruction per two codes.
//     The dims of a code word are dealt to the operand's registers in the order in which the conversion leaves them, and the
//     queries (first product) and outputs (second) are laid out to match, so that nothing is rearranged but one byte
//     permutation per word of values.
//   - a key's power of two multiplies its score; a value's multiplies its probability, relative to the largest of the
//     values that the warp has met (the outputs are rescaled when that grows), so that the fp16 operand stays in range.
//   - bf16 queries are brought into fp16's range by a power of two per row, which the softmax scale takes back; elements
//     below 2^-39 of the row's largest vanish.
//   - a warp takes 32 keys of a tile with a running softmax of its own; rows are rescaled only when a maximum moved.
// Probabilities are scaled by 2^14 (the largest is then 2^14 or less: fp16 has few exponents) and rounded to fp16: bf16
// outputs take that single rounding, an eighth of the output's own; fp16 ones enter as hi + lo pairs of numbers, 2^-22.
#include <type_traits>

#include "held8.cuh"
#include "paged_walk.cuh"

namespace tkphi {

template <int D, bool SPLIT>
struct HeldRowCfg {
  static constexpr int WARPS = SPLIT ? 8 : 4;               // (cluster form: four warps for the even, four for the odd tiles)
  static constexpr int THREADS = (WARPS + 1) * 32;
  static constexpr int CTAS = SPLIT ? 1 : D == 64 ? 3 : 2;  // per multiprocessor
  static constexpr int TILE = kHeldKeys * D;                // codes of a tile's keys or values
  static constexpr int STAGE = 2 * TILE;
  static constexpr int NS = D == 128 ? (SPLIT ? 5 : 3) : (SPLIT ? 10 : 3);
  static constexpr size_t scales = (size_t)NS * STAGE;      // [NS][2][128] scale bytes
  static constexpr size_t frags = scales + NS * 2 * kHeldKeys;      // [D / 16][32 lanes] queries as the lanes take them
  static constexpr size_t red = frags + D * kRowTile * 2;           // [warps][16 rows][32 dims] fp32
  static constexpr size_t stat = red + WARPS * kRowTile * 32 * 4;   // [warps][16][2]
  static constexpr size_t bars = stat + WARPS * kRowTile * 2 * 4;
  static constexpr size_t total = bars + (2 * NS) * 8 + 16;
  static constexpr size_t keep = 0;                         // cluster form: this CTA's piece, over the ring's first tiles
  static_assert(kRowTile * (D + 2) * 4 <= NS * STAGE, "piece");
  static_assert(CTAS * (total + 1024) <= 228 * 1024, "shared memory of a multiprocessor");
};

// Place of 16-byte chunk `chunk` of a row in a tile of rows of D bytes, as the TMA box with the swizzle of that width lies.
template <int D>
__device__ __forceinline__ uint32_t held_at(uint32_t row, uint32_t chunk) {
  return D == 128 ? swz128(row, chunk) : row * 64u + ((chunk ^ ((row >> 1) & 3u)) << 4);
}
// The high bits of the bytes that are NaN codes.
__device__ __forceinline__ uint32_t nan_codes(uint32_t w) { return ((w & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u; }

template <typename T, int D, bool BLOCK, bool SPLIT>
__global__ void __launch_bounds__(HeldRowCfg<D, SPLIT>::THREADS, HeldRowCfg<D, SPLIT>::CTAS)
paged8_rows_kernel(const __grid_constant__ CUtensorMap tmap_k, const __grid_constant__ CUtensorMap tmap_v,
                   const __grid_constant__ PagedProblem p, const __grid_constant__ HeldCache held) {
  using C = HeldRowCfg<D, SPLIT>;
  using Walk = RowWalk<BLOCK, SPLIT, kHeldKeys>;
  constexpr int WARPS = C::WARPS, NS = C::NS;
  constexpr float kShift = 14.f;                            // p = 2^kShift exp2(..)
  constexpr bool kPairs = !T::kBf16;
  extern __shared__ __align__(1024) unsigned char smem[];
  uint4* q_frags = reinterpret_cast<uint4*>(smem + C::frags);
  float* red = reinterpret_cast<float*>(smem + C::red);
  float* stat = reinterpret_cast<float*>(smem + C::stat);
  uint64_t* full = reinterpret_cast<uint64_t*>(smem + C::bars);
  uint64_t* empty = full + NS;
  volatile int* s_abort = reinterpret_cast<int*>(empty + NS);
  float* keep = reinterpret_cast<float*>(smem + C::keep);
  float* keep_stat = keep + kRowTile * D;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int cta = blockIdx.x;

  if (tid == 0) {
    for (int s = 0; s < NS; ++s) { mbar_init(&full[s], 1); mbar_init(&empty[s], 4); }
    mbar_fence_init();
    *s_abort = 0;
  }
  __syncthreads();
  // Inputs of the call may be read once all work before the call is complete.  The block form follows the selection,
  // which begins only then: the page lists alone remain to be waited for, by the producer.
  if (!BLOCK && !p.beside) pdl_wait();
  pdl_launch_next();

  if (warp == WARPS) {
    // ================================================================ TMA producer
    Walk w(p, cta);
    if (BLOCK) pdl_wait();
    const int ps = 1 << p.page_shift;
    const int npg = kHeldKeys >> p.page_shift;                                // pages of a tile: 1 to 8
    // lane: codes of keys, of values, scales of keys, of values, of one page each
    const int which = lane / npg, pg = lane % npg;
    const CUtensorMap* tm = which & 1 ? &tmap_v : &tmap_k;
    const uint8_t* scales = which & 1 ? held.v_scales : held.k_scales;
    const uint64_t pol = BLOCK ? l2_policy_normal() : l2_policy_evict_first();
    int it = 0;
    bool ok = true;
    int issued[NS];
#pragma unroll
    for (int s = 0; s < NS; ++s) issued[s] = -1;
    while (ok && w.next()) {
      const int n_pages_unit = BLOCK ? w.n_list : (w.len + ps - 1) >> p.page_shift;
      const int* list = BLOCK ? p.page_list + (size_t)w.unit * p.n_keep : p.table + (size_t)w.b * p.max_pages;
      auto id_at = [&](int i) { return i < n_pages_unit ? (BLOCK ? __ldcg(list + i) : __ldg(list + i)) : p.n_pages; };
      int batch0 = (int)(((long long)w.t0 * kHeldKeys) >> p.page_shift) & ~31;
      int id = id_at(batch0 + lane), id_next = id_at(batch0 + 32 + lane);
      for (int t = w.t0; t < w.t1; ++t, ++it) {
        const int stage = it % NS;
        const int first = (t * kHeldKeys) >> p.page_shift;
        if (first >= batch0 + 32) {
          batch0 += 32;
          id = id_next;
          id_next = id_at(batch0 + 32 + lane);
        }
        int page = __shfl_sync(0xffffffffu, id, (first + pg) & 31);
        if (page < 0 || page > p.n_pages || (page == p.n_pages && first + pg < n_pages_unit)) {
          if (lane < npg) atomicExch(p.status, kStatusBadPage);
          page = p.n_pages;                     // a box outside the tensor arrives as zeros
        }
        ok = __all_sync(0xffffffffu, mbar_wait(&empty[stage], ((uint32_t)(it / NS) & 1u) ^ 1u, s_abort));
        if (!ok) break;
        if (lane == 0) mbar_expect_tx(&full[stage], C::STAGE + 2 * kHeldKeys);
        __syncwarp();
        if (which < 2) {
          tma_load_4d(smem + (size_t)stage * C::STAGE + which * C::TILE + pg * ps * D, tm, &full[stage], 0, 0, w.h, page, pol);
        } else if (which < 4) {
          // (scales of a page outside: those of another, they belong to codes 0 or to keys that nothing sees)
          const size_t at = ((size_t)(page < p.n_pages ? page : 0) * p.hkv + w.h) << p.page_shift;
          bulk_load(smem + C::scales + (stage * 2 + (which & 1)) * kHeldKeys + pg * ps, scales + at, (uint32_t)ps, &full[stage]);
        }
#pragma unroll
        for (int s = 0; s < NS; ++s)
          if (s == stage) issued[s] = it;
      }
    }
    if (*s_abort) {
      // every copy that was issued must land before shared memory is released
#pragma unroll
      for (int s = 0; s < NS; ++s)
        for (uint32_t n = 0; issued[s] >= 0 && n < kWaitPolls; ++n) {
          if (mbar_try_wait(&full[s], (uint32_t)(issued[s] / NS) & 1u)) break;
          __nanosleep(64);
        }
    }
  } else {
    // ================================================================ compute
    Walk w(p, cta);
    const int ps = 1 << p.page_shift;
    const int rA = lane >> 2, rB = rA + 8, cj = lane & 3, cc = 2 * cj;
    const int kg = (warp & 3) * 32;                          // this warp's keys of a tile
    bool ok = true;
    int it = 0;
    while (w.next()) {
      // ---- the unit's queries as A operands in fp16.  Operand columns 2j, 2j+1, 2j+8, 2j+9 of a group of 16 are dims 4j .. 4j+3.
      // They lie in shared memory, as a lane of each warp takes them: 2 or 4 KB that registers have no room for.
      float slA = p.scale_log2, slB = p.scale_log2;          // log2 units per unit of (operand q).(codes) * key scale
      {
        const uint2* qa = nullptr;
        const uint2* qb = nullptr;
        const uint2* q = static_cast<const uint2*>(p.q);
        if (rA < w.rows) {
          const int r = w.r_first + rA;
          qa = q + ((size_t)(w.tok0 + r / p.group) * p.hq + w.h * p.group + r % p.group) * (D / 4);
        }
        if (rB < w.rows) {
          const int r = w.r_first + rB;
          qb = q + ((size_t)(w.tok0 + r / p.group) * p.hq + w.h * p.group + r % p.group) * (D / 4);
        }
        uint2 x[D / 16][2];                                  // [group of 16 dims][row]
#pragma unroll
        for (int k = 0; k < D / 16; ++k) {
          x[k][0] = qa ? __ldg(qa + k * 4 + cj) : make_uint2(0, 0);
          x[k][1] = qb ? __ldg(qb + k * 4 + cj) : make_uint2(0, 0);
        }
        float f[2] = {1.f, 1.f};
        if (T::kBf16) {
#pragma unroll
          for (int r = 0; r < 2; ++r) {
            float most = 0.f;                                // the largest finite magnitude
#pragma unroll
            for (int k = 0; k < D / 16; ++k)
#pragma unroll
              for (int i = 0; i < 4; ++i) {
                const uint32_t w = i < 2 ? x[k][r].x : x[k][r].y;
                const float v = fabsf(i & 1 ? T::hi(w) : T::lo(w));
                if (v < INFINITY) most = fmaxf(most, v);
              }
#pragma unroll
            for (int d = 1; d < 4; d <<= 1) most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, d));
            // the largest goes to [2^14, 2^15); the exponent that is taken off is at least -100
            const int e = max((int)(__float_as_uint(most) >> 23) - 127 - 14, -100);
            f[r] = __uint_as_float((uint32_t)(127 - e) << 23);
            (r ? slB : slA) *= __uint_as_float((uint32_t)(127 + e) << 23);
          }
        }
#pragma unroll
        for (int k = 0; k < D / 16; ++k) {
          if (k % WARPS != warp) continue;                   // the warps share the work
          uint4 v = make_uint4(x[k][0].x, x[k][1].x, x[k][0].y, x[k][1].y);
          if (T::kBf16)
            v = make_uint4(Fp16::pack(T::lo(v.x) * f[0], T::hi(v.x) * f[0]), Fp16::pack(T::lo(v.y) * f[1], T::hi(v.y) * f[1]),
                           Fp16::pack(T::lo(v.z) * f[0], T::hi(v.z) * f[0]), Fp16::pack(T::lo(v.w) * f[1], T::hi(v.w) * f[1]));
          q_frags[k * 32 + lane] = v;
        }
      }
      named_barrier(1, WARPS * 32);
      // last visible position of this thread's rows; -1: no such row
      int limA = -1, limB = -1;
      if (rA < w.rows) limA = BLOCK ? w.pos0 : p.causal ? w.pos0 + (w.r_first + rA) / p.group : w.len - 1;
      if (rB < w.rows) limB = BLOCK ? w.pos0 : p.causal ? w.pos0 + (w.r_first + rB) / p.group : w.len - 1;
      // keys up to lim_all are visible to every row of the unit, keys behind lim_last to none
      const int lim_all = BLOCK ? w.pos0 : p.causal ? w.pos0 + w.r_first / p.group : w.len - 1;
      const int lim_last = BLOCK ? w.pos0 : p.causal ? w.pos0 + (w.r_first + w.rows - 1) / p.group : w.len - 1;
      // outputs: o[2x], o[2x+1] hold dims 16 x + 4 j, + 2 and 16 x + 4 j + 1, + 3 of rows A and B
      float o[D / 8][4];
#pragma unroll
      for (int n = 0; n < D / 8; ++n) { o[n][0] = o[n][1] = o[n][2] = o[n][3] = 0.f; }
      float mA = -INFINITY, mB = -INFINITY, lA = 0.f, lB = 0.f;
      int top = 0;                                           // the outputs' unit is 2^(top - 127)

      for (int t = w.t0; t < w.t1; ++t, ++it) {
        if (SPLIT && (it & 1) != warp >> 2) continue;
        const int stage = it % NS;
        if (ok) ok = __all_sync(0xffffffffu, mbar_wait(&full[stage], (uint32_t)(it / NS) & 1u, s_abort));
        if (!ok) continue;                                // the barriers below are still met
        unsigned char* ks = smem + (size_t)stage * C::STAGE;
        unsigned char* vs = ks + C::TILE;
        const unsigned char* ke = smem + C::scales + stage * 2 * kHeldKeys + kg;
        const unsigned char* ve = ke + kHeldKeys;
        // positions of this warp's two groups of 16 keys (a group never straddles a page); in the block form only the last
        // page of a list can be partly visible, everything before it is
        int key0[2];
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          key0[x] = t * kHeldKeys + kg + x * 16;
          if (BLOCK) {
            const int entry = key0[x] >> p.page_shift;
            if (entry < w.n_list - 1) key0[x] = 0 - 16;                          // all visible
            else if (entry == w.n_list - 1) key0[x] = ((w.pos0 >> p.page_shift) << p.page_shift) + (key0[x] & (ps - 1));
            else key0[x] = w.len;                                                // past the list
          }
        }
        // (two copies: with keys that some row does not see, and without any)
        auto step = [&](auto tag) {
          constexpr bool careful = decltype(tag)::value;
          bool odd_values = false;                          // NaN codes that not every row sees
          float s[4][4];
          // Scores of group x in s[2x], s[2x+1]: column 2j + e of s[2x + n] is key 4j + 2n + e of the group, so that a thread's
          // four keys lie beside each other.
#pragma unroll
          for (int n = 0; n < 4; ++n) s[n][0] = s[n][1] = s[n][2] = s[n][3] = 0.f;
          const int kr = lane & 7, krow = kg + ((kr >> 1) << 2) + ((lane >> 4) << 1) + (kr & 1), ksub = (lane >> 3) & 1;
          const uint32_t k_at[2] = {smem_u32(ks) + held_at<D>(krow, ksub), smem_u32(ks) + held_at<D>(krow + 16, ksub)};
#pragma unroll
          for (int k = 0; k < D / 32; ++k) {
            uint32_t b0[2][4], b1[2][4];                    // words: (n = 0, dims 0-15), (0, 16-31), (1, 0-15), (1, 16-31)
#pragma unroll
            for (int x = 0; x < 2; ++x) {
              uint32_t c[4];
              ldmatrix_x4(c, k_at[x] ^ (k << 5));
#pragma unroll
              for (int i = 0; i < 4; ++i) unpack_codes(c[i], b0[x][i], b1[x][i]);
            }
#pragma unroll
            for (int y = 0; y < 2; ++y) {
              const uint4 q4 = q_frags[(2 * k + y) * 32 + lane];
              const uint32_t qf[4] = {q4.x, q4.y, q4.z, q4.w};
#pragma unroll
              for (int n = 0; n < 4; ++n) Fp16::mma(s[n], qf, b0[n >> 1][2 * (n & 1) + y], b1[n >> 1][2 * (n & 1) + y]);
            }
          }
          // this thread's keys: scale bytes of four at a time
          uint32_t vw[2];
#pragma unroll
          for (int x = 0; x < 2; ++x) {
            const uint32_t kw = *reinterpret_cast<const uint32_t*>(ke + x * 16 + 4 * cj);
            vw[x] = *reinterpret_cast<const uint32_t*>(ve + x * 16 + 4 * cj);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              // (byte 255 gives infinity here, less itself no number; byte 0 gives 0 for 2^-127)
              const float f = __uint_as_float((i == 3 ? kw >> 1 : kw << (23 - 8 * i)) & 0x7f800000u), z = f - f;
              float (&a)[4] = s[2 * x + (i >> 1)];
              a[i & 1] = fmaf(a[i & 1], f, z);
              a[2 + (i & 1)] = fmaf(a[2 + (i & 1)], f, z);
            }
          }
          if (careful) {
#pragma unroll
            for (int x = 0; x < 2; ++x)
#pragma unroll
              for (int i = 0; i < 4; ++i) {
                const int key = key0[x] + 4 * cj + i;
                if (key > limA) s[2 * x + (i >> 1)][i & 1] = -INFINITY;
                if (key > limB) s[2 * x + (i >> 1)][2 + (i & 1)] = -INFINITY;
                if (key > lim_last) vw[x] &= ~(0xffu << (8 * i));
              }
            // Values that no row sees may be anything (behind the sequence's end they may be left-overs): 0 times them must
            // not reach the product.  Those that some rows see are looked through.
            constexpr int CPR = D / 16;                     // 16-byte chunks of a row
#pragma unroll
            for (int x = 0; x < 2; ++x) {
              const int seen = max(lim_last + 1 - key0[x], 0);
              for (int i = lane; i < (16 - seen) * CPR; i += 32)
                *reinterpret_cast<uint4*>(vs + held_at<D>(kg + x * 16 + seen + i / CPR, i % CPR)) = make_uint4(0, 0, 0, 0);
            }
            fence_proxy_async_smem();                       // before the slot's next copy
            __syncwarp();
            if (!BLOCK && lim_all < lim_last) {
              uint32_t bad = 0;
              for (int i = lane; i < 32 * CPR; i += 32) {
                const uint4 c = *reinterpret_cast<const uint4*>(vs + held_at<D>(kg + i / CPR, i % CPR));
                bad |= nan_codes(c.x) | nan_codes(c.y) | nan_codes(c.z) | nan_codes(c.w);
              }
              odd_values = __any_sync(0xffffffffu, bad != 0);
            }
          }
          // the largest value scale so far; the outputs follow when it grows.  Bytes as pairs of 16 bits, keys 0, 2 and 1, 3.
          uint32_t v2[4] = {vw[0] & 0x00ff00ffu, vw[0] >> 8 & 0x00ff00ffu, vw[1] & 0x00ff00ffu, vw[1] >> 8 & 0x00ff00ffu};
          auto largest = [&]() {
            const uint32_t m = __vmaxu2(__vmaxu2(v2[0], v2[1]), __vmaxu2(v2[2], v2[3]));
            return __reduce_max_sync(0xffffffffu, max(m & 0xffffu, m >> 16));
          };
          uint32_t most = largest();
          const bool bad_scale = most == 255u;
          if (bad_scale) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              if ((v2[i] & 0xffffu) == 255u) v2[i] &= 0xffff0000u;
              if (v2[i] >> 16 == 255u) v2[i] &= 0xffffu;
            }
            most = largest();
          }
          if ((int)most > top) {
            const int d = 127 + top - (int)most;
            const float f = d > 0 ? __uint_as_float((uint32_t)d << 23) : 0.f;
#pragma unroll
            for (int n = 0; n < D / 8; ++n) { o[n][0] *= f; o[n][1] *= f; o[n][2] *= f; o[n][3] *= f; }
            top = (int)most;
          }
          // exponent fields of the values' scales over the largest: 127 + byte - top, 0 if that is less
          const uint32_t least = (uint32_t)max(top - 127, 0) * 0x00010001u, shift = (uint32_t)(127 - top) * 0x00010001u;
#pragma unroll
          for (int i = 0; i < 4; ++i) v2[i] = __vmaxu2(v2[i], least) + shift;
          float tA = fmaxf(fmaxf(s[0][0], s[0][1]), fmaxf(s[1][0], s[1][1])), tB = fmaxf(fmaxf(s[0][2], s[0][3]), fmaxf(s[1][2], s[1][3]));
          tA = fmaxf(tA, fmaxf(fmaxf(s[2][0], s[2][1]), fmaxf(s[3][0], s[3][1])));
          tB = fmaxf(tB, fmaxf(fmaxf(s[2][2], s[2][3]), fmaxf(s[3][2], s[3][3])));
#pragma unroll
          for (int d = 1; d < 4; d <<= 1) {
            tA = fmaxf(tA, __shfl_xor_sync(0xffffffffu, tA, d));
            tB = fmaxf(tB, __shfl_xor_sync(0xffffffffu, tB, d));
          }
          // (maxima are kept before the scale: the largest score less the maximum is then exactly 0)
          const float nA = fmaxf(mA, tA), nB = fmaxf(mB, tB);
          if (__any_sync(0xffffffffu, nA > mA || nB > mB)) {
            const float fA = nA > mA ? ex2_approx((mA - nA) * slA) : 1.f, fB = nB > mB ? ex2_approx((mB - nB) * slB) : 1.f;
            lA *= fA; lB *= fB;
#pragma unroll
            for (int n = 0; n < D / 8; ++n) { o[n][0] *= fA; o[n][1] *= fA; o[n][2] *= fB; o[n][3] *= fB; }
            mA = nA; mB = nB;
          }
          // a row that has seen nothing yet: every term exp2(-inf - 0) = 0
          const float uA = mA == -INFINITY ? 0.f : mA, uB = mB == -INFINITY ? 0.f : mB;
#pragma unroll
          for (int x = 0; x < 2; ++x)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              float& sa = s[2 * x + (i >> 1)][i & 1];
              float& sb = s[2 * x + (i >> 1)][2 + (i & 1)];
              const float a = ex2_approx(fmaf(sa - uA, slA, kShift)), b = ex2_approx(fmaf(sb - uB, slB, kShift));
              lA += a;
              lB += b;
              const uint32_t e = v2[2 * x + (i & 1)];
              const float f = __uint_as_float(i < 2 ? e << 23 : e << 7 & 0x7f800000u);
              sa = a * f;
              sb = b * f;
            }
          if (bad_scale || careful) {
#pragma unroll
            for (int x = 0; x < 2; ++x)
#pragma unroll
              for (int i = 0; i < 4; ++i) {
                float& sa = s[2 * x + (i >> 1)][i & 1];
                float& sb = s[2 * x + (i >> 1)][2 + (i & 1)];
                const int key = key0[x] + 4 * cj + i;
                if ((vw[x] >> (8 * i) & 255u) == 255u) sa = sb = __uint_as_float(0x7fc00000u);
                if (key > limA) sa = 0.f;                    // (unseen, whatever its scale)
                if (key > limB) sb = 0.f;
              }
          }
          if (careful && !BLOCK && odd_values) {
            // added to the rows that see them, and taken out of the product, where 0 times them would reach the others
            const float none = __uint_as_float(0x7fc00000u);
#pragma unroll 1
            for (int k = 0; k < 32; ++k) {
              const int key = key0[k >> 4] + (k & 15);
              const bool a = key <= limA, b = key <= limB;
#pragma unroll
              for (int x = 0; x < D / 16; ++x) {
                const uint32_t c = nan_codes(*reinterpret_cast<const uint32_t*>(vs + held_at<D>(kg + k, x) + 4 * cj));
                if (c & 0x80u) { if (a) o[2 * x][0] = none; if (b) o[2 * x][2] = none; }
                if (c & 0x8000u) { if (a) o[2 * x + 1][0] = none; if (b) o[2 * x + 1][2] = none; }
                if (c & 0x800000u) { if (a) o[2 * x][1] = none; if (b) o[2 * x][3] = none; }
                if (c >> 31) { if (a) o[2 * x + 1][1] = none; if (b) o[2 * x + 1][3] = none; }
              }
            }
            __syncwarp();
            for (int i = lane; i < 32 * (D / 4); i += 32) {
              uint32_t* c = reinterpret_cast<uint32_t*>(vs + held_at<D>(kg + i / (D / 4), (i % (D / 4)) >> 2) + (i & 3) * 4);
              *c &= ~((nan_codes(*c) >> 7) * 0xffu);
            }
            fence_proxy_async_smem();
            __syncwarp();
          }
#pragma unroll
          for (int x = 0; x < 2; ++x) {
            uint32_t ph[4], pl[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {                    // A operand: (row, keys 0-7), (row + 8, 0-7), (row, 8-15), (row + 8, 8-15)
              const float u = s[2 * x + (j >> 1)][(j & 1) * 2], v = s[2 * x + (j >> 1)][(j & 1) * 2 + 1];
              ph[j] = Fp16::pack(u, v);
              if (kPairs) pl[j] = Fp16::pack(u - Fp16::lo(ph[j]), v - Fp16::hi(ph[j]));
            }
            const int r = lane & 7, row = kg + x * 16 + ((r >> 1) << 2) + (((lane >> 3) & 1) << 1) + (r & 1);
            const uint32_t v_at = smem_u32(vs) + held_at<D>(row, lane >> 4);
#pragma unroll
            for (int n = 0; n < D / 32; ++n) {
              uint32_t c[4], b0[4], b1[4];                   // c: (columns 0-7, dims 0-15), (8-15, 0-15), (0-7, 16-31), (8-15, 16-31)
              ldmatrix_x4_trans(c, v_at ^ (n << 5));
              // a word: column 2j's dims 2g, 2g+1, then column 2j+1's; the two keys of a dim beside each other
#pragma unroll
              for (int i = 0; i < 4; ++i) unpack_codes(__byte_perm(c[i], 0, 0x3120), b0[i], b1[i]);
#pragma unroll
              for (int y = 0; y < 2; ++y) {
                Fp16::mma(o[4 * n + 2 * y], ph, b0[2 * y], b0[2 * y + 1]);
                Fp16::mma(o[4 * n + 2 * y + 1], ph, b1[2 * y], b1[2 * y + 1]);
                if (kPairs) {
                  Fp16::mma(o[4 * n + 2 * y], pl, b0[2 * y], b0[2 * y + 1]);
                  Fp16::mma(o[4 * n + 2 * y + 1], pl, b1[2 * y], b1[2 * y + 1]);
                }
              }
            }
          }
        };
        if (key0[0] + 15 <= lim_all && key0[1] + 15 <= lim_all) step(std::false_type());
        else if (key0[0] <= lim_last || key0[1] <= lim_last) step(std::true_type());
        __syncwarp();
        if (lane == 0) mbar_arrive(&empty[stage]);
      }

      // ---- the warps' softmaxes joined; a thread ends up with PER of 32 dims of one row
      mA = mA * slA - kShift; mB = mB * slB - kShift;
#pragma unroll
      for (int d = 1; d < 4; d <<= 1) {
        lA += __shfl_xor_sync(0xffffffffu, lA, d);
        lB += __shfl_xor_sync(0xffffffffu, lB, d);
      }
      if (cj == 0) {
        stat[(warp * kRowTile + rA) * 2] = mA; stat[(warp * kRowTile + rA) * 2 + 1] = lA;
        stat[(warp * kRowTile + rB) * 2] = mB; stat[(warp * kRowTile + rB) * 2 + 1] = lB;
      }
      named_barrier(1, WARPS * 32);
      float MA = -INFINITY, MB = -INFINITY;
#pragma unroll
      for (int i = 0; i < WARPS; ++i) {
        MA = fmaxf(MA, stat[(i * kRowTile + rA) * 2]);
        MB = fmaxf(MB, stat[(i * kRowTile + rB) * 2]);
      }
      // (a warp that has seen nothing has the sum 0; one that has seen no numbers alone has no maximum, but no 0 either)
      const float unit = held_scale((uint32_t)top);
      const float sA = lA == 0.f ? 0.f : ex2_approx(mA - MA) * unit, sB = lB == 0.f ? 0.f : ex2_approx(mB - MB) * unit;
      constexpr int PER = 16 / WARPS, TPR = 32 / PER;          // dims of a thread, threads of a row
      const int row = tid / TPR, dp = tid % TPR * PER;
      float M = -INFINITY, L = 0.f;
#pragma unroll
      for (int i = 0; i < WARPS; ++i) M = fmaxf(M, stat[(i * kRowTile + row) * 2]);
#pragma unroll
      for (int i = 0; i < WARPS; ++i) {
        const float l = stat[(i * kRowTile + row) * 2 + 1];
        if (l != 0.f) L += l * ex2_approx(stat[(i * kRowTile + row) * 2] - M);
      }
      const bool fin = w.whole();              // in a cluster: the unit is this CTA's alone
      const int slot = w.slot(cta);
      const int r = w.r_first + row;
      const size_t out_row = (size_t)(w.tok0 + r / p.group) * p.hq + w.h * p.group + r % p.group;
      const float inv = L != 0.f ? 1.f / L : 0.f;
#pragma unroll
      for (int x = 0; x < D / 32; ++x) {
        // rows of 32 floats, 4-float pieces shifted by four in odd rows so that the accesses spread over the banks
        float* mine = red + warp * kRowTile * 32;
#pragma unroll
        for (int n = 0; n < 2; ++n) {
          const int at = ((4 * n + cj + 4 * (rA & 1)) & 7) * 4;
          const float (&e)[4] = o[4 * x + 2 * n];
          const float (&f)[4] = o[4 * x + 2 * n + 1];
          *reinterpret_cast<float4*>(mine + rA * 32 + at) = make_float4(e[0] * sA, f[0] * sA, e[1] * sA, f[1] * sA);
          *reinterpret_cast<float4*>(mine + rB * 32 + at) = make_float4(e[2] * sB, f[2] * sB, e[3] * sB, f[3] * sB);
        }
        named_barrier(1, WARPS * 32);
        float a[PER];
#pragma unroll
        for (int e = 0; e < PER; ++e) a[e] = 0.f;
#pragma unroll
        for (int i = 0; i < WARPS; ++i)
#pragma unroll
          for (int e = 0; e < PER; e += 2) {
            const float2 u = *reinterpret_cast<const float2*>(red + (i * kRowTile + row) * 32 + ((((dp >> 2) + 4 * (row & 1)) & 7) * 4) + (dp & 3) + e);
            a[e] += u.x; a[e + 1] += u.y;
          }
        if (row < w.rows) {
          float* part = (SPLIT ? keep + (size_t)row * D : p.row_part + ((size_t)slot * kRowTile + row) * D) + x * 32 + dp;
          uint32_t* y = reinterpret_cast<uint32_t*>(static_cast<uint16_t*>(p.y) + out_row * D + x * 32 + dp);
#pragma unroll
          for (int e = 0; e < PER; e += 2) {
            if (fin) y[e >> 1] = T::pack(a[e] * inv, a[e + 1] * inv);
            else *reinterpret_cast<float2*>(part + e) = make_float2(a[e], a[e + 1]);
          }
        }
        named_barrier(1, WARPS * 32);
      }
      if (tid % TPR == 0 && row < w.rows) {
        if (fin) {
          if (p.lse) p.lse[out_row] = L != 0.f ? (M + log2f(L)) * 0.6931471805599453f : -INFINITY;
        } else {
          float* st = SPLIT ? keep_stat + row * 2 : p.row_stat + ((size_t)slot * kRowTile + row) * 2;
          st[0] = M;
          st[1] = L;
        }
      }
    }
  }
  if (SPLIT && p.n_split > 1) join_cluster<T, D, BLOCK, kHeldKeys, WARPS>(p, cta, keep, keep_stat);
  __syncthreads();
  if (*s_abort && tid == 0) atomicExch(p.status, kStatusTimeout);
  // (beside a tile-kernel launch this grid may run next to it: it must not be complete before that one is, because the
  // joins that follow wait for this grid only)
  if (p.beside) pdl_wait();
}

template <typename T, int D, bool BLOCK, bool SPLIT>
static cudaError_t launch_rows_s(const PagedProblem& p, const HeldCache& held, const CUtensorMap& tk, const CUtensorMap& tv, int grid,
                                 cudaStream_t st) {
  using C = HeldRowCfg<D, SPLIT>;
  static PerDeviceFlag configured;
  const cudaError_t e = set_max_dynamic_smem(configured, reinterpret_cast<const void*>(paged8_rows_kernel<T, D, BLOCK, SPLIT>), C::total);
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(grid);
  cfg.blockDim = dim3(C::THREADS);
  cfg.dynamicSmemBytes = C::total;
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = p.n_split; attr[1].val.clusterDim.y = 1; attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = SPLIT && p.n_split > 1 ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, paged8_rows_kernel<T, D, BLOCK, SPLIT>, tk, tv, p, held);
}

#define TKPHI_BY_TYPE(call)                                                          \
  (d == 64 ? (bf16 ? (block ? call(Bf16, 64, true) : call(Bf16, 64, false))           \
                   : (block ? call(Fp16, 64, true) : call(Fp16, 64, false)))          \
           : (bf16 ? (block ? call(Bf16, 128, true) : call(Bf16, 128, false))         \
                   : (block ? call(Fp16, 128, true) : call(Fp16, 128, false))))

int paged8_row_ctas(int d) { return d == 64 ? HeldRowCfg<64, false>::CTAS : HeldRowCfg<128, false>::CTAS; }

cudaError_t launch_paged8_rows(const PagedProblem& p, const HeldCache& held, const CUtensorMap& tk, const CUtensorMap& tv, int d,
                               bool bf16, bool block, bool split, int grid, cudaStream_t st) {
#define ROWS(T, D, B) (split ? launch_rows_s<T, D, B, true>(p, held, tk, tv, grid, st) : launch_rows_s<T, D, B, false>(p, held, tk, tv, grid, st))
  return TKPHI_BY_TYPE(ROWS);
#undef ROWS
}

cudaError_t launch_paged8_rows_merge(const PagedProblem& p, int d, bool bf16, bool block, int units, int max_rows, cudaStream_t st) {
#define MERGE(T, D, B) \
  launch_pdl(paged_rows_merge_kernel<T, D, B, kHeldKeys>, dim3(units, max_rows), dim3(kMergeThreads), 0, st, p)
  return TKPHI_BY_TYPE(MERGE);
#undef MERGE
}

}  // namespace tkphi
