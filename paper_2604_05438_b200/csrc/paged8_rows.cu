// Attention of few query rows over an 8-bit paged cache: sequences with at most 64 rows (tokens x query heads of a KV head),
// and the page-selected form, where every token of a KV head reads a page list of its own.
//
//   y = sum_t p_t v_t / sum_t p_t,  p_t = exp(scale * q.k_t - m),  lse = m + log sum_t p_t   over the visible keys t
//   k_t = a_t * (its codes),  v_t = b_t * (its codes),  a_t and b_t powers of two
//
// in one pass with the running maximum m and sum.  Work is dealt out and joined as over a 16-bit cache (paged_walk.cuh), in
// tiles of 128 keys.  Bound: memory, 2 * (head_dim + 1) bytes per key against 8 or 16 rows of work; with half the bytes of a
// 16-bit cache the instructions per key count as much.  So:
//   - both products have the keys or dims of the cache as the 16 rows of the matrix instruction and 8 query rows as its
//     columns (S^T = K Q^T, O^T = V^T P^T), once or twice: a single token of a group of up to 8 heads pays for 8 rows, where
//     queries as the instruction's rows would pay for 16, in products, exponentials and registers.  P^T changes from
//     accumulator to operand by a transpose of 8 x 8 blocks between lanes.
//   - the products are fp16 products of the codes, which fp16 holds exactly: one conversion instruction per two codes.  The
//     dims of a code word are dealt to the operand's registers in the order in which the conversion leaves them, and queries
//     and outputs are laid out to match, so that nothing is rearranged but one byte permutation per word of values.
//     (e4m3 instructions for the first product, with queries as sums of two or three codes, need no conversion of keys, but
//     took 1.2x the time: they issue as more instructions.)
//   - a key's power of two multiplies its score; a value's multiplies its probability, in units of the row's reference: a power
//     of two that the row's largest product of the two does not exceed and is at most 2^10 below, so that the products that
//     count are normal numbers of the fp16 operand, whatever the sizes of values that nothing attends to or of later tokens'
//     values.  Scales below the reference change nothing in that, unless a maximum moves to a key with a very small one.  So a
//     warp, whose rows have one reference as a rule, looks for scales above it only; where there is one, each row takes the
//     reference that its own keys allow, with room for larger scales, and its outputs follow.
//   - bf16 queries are brought into fp16's range by a power of two per row, which the softmax scale takes back; elements
//     below 2^-39 of the row's largest vanish.
//   - a warp takes 32 keys of a tile with a running softmax of its own; rows are rescaled only when a maximum moved.
// Probabilities are scaled by 2^14 (a row's largest product is then from 2^4 to 2^15: fp16 has few exponents) and rounded to
// fp16 once, 2^-12: an eighth of a bf16 output's own rounding, as much as an fp16 one's.  Products below 2^-29 of the row's
// largest vanish.
// Measured: 32 sequences of 8K to 64K, 24 / 8 heads of 128: 330-345 us, 6.3-6.5 TB/s of codes and scales (16-bit operands in the
// other order, queries as the rows: 435; scales looked at on both sides of the reference and references tracked row by row in
// every tile: 395-445).  Scales spread by a standard deviation of 12 powers instead of 1: 204 against 198 us for 32 sequences of
// 16K; with two row tiles and a deviation of 4, 157 against 72 for eight of 32K, because each row then keeps a reference of its own.  A token over 4096 keys, 32 / 8 heads of 64: 8.0 us; with sixteen warps instead of
// eight in the cluster form 9.1.  Three CTAs per multiprocessor instead of two at head_dim 128: no faster (registers spill).
#include <cfloat>
#include <type_traits>

#include "held8.cuh"
#include "paged_walk.cuh"

namespace tkphi {

template <int D, bool SPLIT, int NT>
struct HeldRowCfg {
  static constexpr int ROWS = 8 * NT;                       // query rows of a unit, at most
  static constexpr int WARPS = SPLIT ? 8 : 4;               // (cluster form: four warps for the even, four for the odd tiles)
  static constexpr int THREADS = (WARPS + 1) * 32;
  static constexpr int CTAS = SPLIT ? 1 : D == 128 ? 2 : NT == 1 ? 4 : 3;  // per multiprocessor
  static constexpr int TILE = kHeldKeys * D;                // codes of a tile's keys or values
  static constexpr int STAGE = 2 * TILE;
  static constexpr int NS = D == 128 ? (SPLIT ? 5 : 3) : SPLIT ? 10 : NT == 1 ? 2 : 3;
  static constexpr size_t scales = (size_t)NS * STAGE;      // [NS][2][128] scale bytes
  static constexpr size_t frags = scales + NS * 2 * kHeldKeys;      // [D / 16][32 lanes][NT] queries as the lanes take them
  static constexpr int CHUNK = 512 / ROWS;                  // dims of a row that are joined at a time
  static constexpr size_t red = frags + D * ROWS * 2;       // [warps][ROWS][CHUNK] fp32
  static constexpr size_t stat = red + WARPS * ROWS * CHUNK * 4;    // [warps][ROWS][2]
  static constexpr size_t bars = stat + WARPS * ROWS * 2 * 4;
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
// Transpose of an 8 x 8 matrix of 16-bit elements: lane (g, j) gives elements (g, 2j), (g, 2j + 1) and gets (2j, g), (2j + 1, g).
__device__ __forceinline__ uint32_t transpose_8x8(uint32_t a) {
  uint32_t d;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(d) : "r"(a));
  return d;
}
// The high bits of the bytes that are NaN codes.
__device__ __forceinline__ uint32_t nan_codes(uint32_t w) { return ((w & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u; }

template <typename T, int D, bool BLOCK, bool SPLIT, int NT>
__global__ void __launch_bounds__(HeldRowCfg<D, SPLIT, NT>::THREADS, HeldRowCfg<D, SPLIT, NT>::CTAS)
paged8_rows_kernel(const __grid_constant__ CUtensorMap tmap_k, const __grid_constant__ CUtensorMap tmap_v,
                   const __grid_constant__ PagedProblem p, const __grid_constant__ HeldCache held) {
  using C = HeldRowCfg<D, SPLIT, NT>;
  using Walk = RowWalk<BLOCK, SPLIT, kHeldKeys>;
  constexpr int WARPS = C::WARPS, NS = C::NS, ROWS = C::ROWS;
  constexpr float kShift = 14.f;                            // p = 2^kShift exp2(..)
  constexpr int kLoose = 10;                                // powers of two that a row's reference may be above its largest product
  constexpr int kRoom = 3;                                  // .. and is above the scales where that allows it
  constexpr int kNone = -10000;
  extern __shared__ __align__(1024) unsigned char smem[];
  uint2* q_frags = reinterpret_cast<uint2*>(smem + C::frags);
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
    const int g = lane >> 2, j = lane & 3;                   // query rows of this thread: 8 t + 2 j + i, i = 0, 1
    const int kg = (warp & 3) * 32;                          // this warp's keys of a tile
    // the key row and the piece of it that this lane gives to ldmatrix, of the first group of 16 keys: even keys, odd ones
    const int frag_row = kg + 2 * (lane & 7) + ((lane >> 3) & 1), frag_piece = lane >> 4;
    bool ok = true;
    int it = 0;
    while (w.next()) {
      // ---- the unit's queries as operands in fp16.  Operand rows 2j, 2j+1, 2j+8, 2j+9 of a group of 16 dims are dims 4j .. 4j+3.
      // They lie in shared memory, as a lane of each warp takes them.
      float sl[NT][2];                                       // log2 units per unit of (operand q).(codes) * key scale * key_unit
      float key_unit = 1.f;
      int e_row[NT], e_top = 0;                              // powers of two taken off the rows, the largest of the unit's
      if (T::kBf16) e_top = -126;
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        const int r = w.r_first + 8 * t + g;
        uint2 x[D / 16];
#pragma unroll
        for (int k = 0; k < D / 16; ++k)
          x[k] = 8 * t + g < w.rows
                     ? __ldg(static_cast<const uint2*>(p.q) + ((size_t)(w.tok0 + r / p.group) * p.hq + w.h * p.group + r % p.group) * (D / 4) + k * 4 + j)
                     : make_uint2(0, 0);
        float f = 1.f;
        e_row[t] = 0;
        if (T::kBf16) {
          float most = 0.f;                                  // the largest finite magnitude
#pragma unroll
          for (int k = 0; k < D / 16; ++k)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const uint32_t u = i < 2 ? x[k].x : x[k].y;
              const float v = fabsf(i & 1 ? T::hi(u) : T::lo(u));
              if (v < INFINITY) most = fmaxf(most, v);
            }
#pragma unroll
          for (int d = 1; d < 4; d <<= 1) most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, d));
          // the largest goes to [2^14, 2^15); the exponent that is taken off is at least -126
          const int e = max((int)(__float_as_uint(most) >> 23) - 127 - 14, -126);
          f = __uint_as_float((uint32_t)(127 - e) << 23);
          e_row[t] = e;
          e_top = max(e_top, __reduce_max_sync(0xffffffffu, e));
        }
#pragma unroll
        for (int k = 0; k < D / 16; ++k) {
          if (k % WARPS != warp) continue;                   // the warps share the work
          if (T::kBf16) x[k] = make_uint2(Fp16::pack(T::lo(x[k].x) * f, T::hi(x[k].x) * f), Fp16::pack(T::lo(x[k].y) * f, T::hi(x[k].y) * f));
          q_frags[(k * 32 + lane) * NT + t] = x[k];
        }
      }
      // Small queries scaled up times large keys would leave fp32's range where their products do not: up to 2^32 of what the
      // queries gained comes off the keys' scales (products below 2^31 * 2^(127 - 32); the keys that vanish then are below
      // 2^-86, of queries below 2^-16).
      const int off = min(max(-e_top, 0), 32);
      key_unit = __uint_as_float((uint32_t)(127 - off) << 23);
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        // (not 0, not infinite: either would make no numbers of infinite and of equal scores)
        const float back = fminf(fmaxf(p.scale_log2 * __uint_as_float((uint32_t)max(127 + e_row[t] + off, 1) << 23), FLT_TRUE_MIN), FLT_MAX);
#pragma unroll
        for (int i = 0; i < 2; ++i) sl[t][i] = __shfl_sync(0xffffffffu, back, 8 * j + 4 * i);
      }
      named_barrier(1, WARPS * 32);
      // last visible position of this thread's rows; -1: no such row
      int lim[NT][2];
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const int r = 8 * t + 2 * j + i;
          lim[t][i] = r >= w.rows ? -1 : BLOCK ? w.pos0 : p.causal ? w.pos0 + (w.r_first + r) / p.group : w.len - 1;
        }
      // keys up to lim_all are visible to every row of the unit, keys behind lim_last to none
      const int lim_all = BLOCK ? w.pos0 : p.causal ? w.pos0 + w.r_first / p.group : w.len - 1;
      const int lim_last = BLOCK ? w.pos0 : p.causal ? w.pos0 + (w.r_first + w.rows - 1) / p.group : w.len - 1;
      // outputs: o[t][b][0], [1] are dim 16 b + 2 g of this thread's rows, [2], [3] the dim behind it
      float o[NT][D / 16][4];
      float m[NT][2], l[NT][2];
#pragma unroll
      for (int t = 0; t < NT; ++t) {
#pragma unroll
        for (int b = 0; b < D / 16; ++b) { o[t][b][0] = o[t][b][1] = o[t][b][2] = o[t][b][3] = 0.f; }
        m[t][0] = m[t][1] = -INFINITY;
        l[t][0] = l[t][1] = 0.f;
      }
      // A row's outputs are in units of 2^(reference - 127), and so are the values' scales in its probabilities' operands: `top`
      // for all rows, or (mixed) one for each, of which it is the largest (in this warp's part of stat, since it is seldom used).
      // Each row's largest product so far is 2^(low - 127) at least, top - kLoose <= low (mixed: 2^(its reference - kLoose - 127)).
      int top = 0, low = 0;
      bool mixed = false, fresh = true;                      // fresh: no keys yet
      int* refs = reinterpret_cast<int*>(stat) + (warp * ROWS + 2 * j) * 2;      // this thread's rows: [16 t + 2 i]

      for (int tile = w.t0; tile < w.t1; ++tile, ++it) {
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
          key0[x] = tile * kHeldKeys + kg + x * 16;
          if (BLOCK) {
            const int entry = key0[x] >> p.page_shift;
            if (entry < w.n_list - 1) key0[x] = 0 - 16;                          // all visible
            else if (entry == w.n_list - 1) key0[x] = ((w.pos0 >> p.page_shift) << p.page_shift) + (key0[x] & (ps - 1));
            else key0[x] = w.len;                                                // past the list
          }
        }
        // the scale bytes of this thread's values, two keys of each group, as pairs of 16 bits
        const bool all_seen = key0[0] + 15 <= lim_all && key0[1] + 15 <= lim_all;
        uint32_t v2[2];
#pragma unroll
        for (int x = 0; x < 2; ++x) v2[x] = __byte_perm(*reinterpret_cast<const uint16_t*>(ve + x * 16 + 2 * g), 0, 0x4140);
        auto smallest = [](uint32_t a, uint32_t b) {
          const uint32_t u = __vminu2(a, b);
          return (int)__reduce_min_sync(0xffffffffu, min(u & 0xffffu, u >> 16));
        };
        auto above_top = [&]() { const uint32_t u = (uint32_t)top * 0x00010001u; return __any_sync(0xffffffffu, __vmaxu2(__vmaxu2(v2[0], v2[1]), u) != u); };
        bool plain = all_seen && !mixed;
        if (plain && fresh) {
          // the first keys: in most cases one reference does for all rows
          const uint32_t u = __vmaxu2(v2[0], v2[1]);
          const int most = (int)__reduce_max_sync(0xffffffffu, max(u & 0xffffu, u >> 16));
          low = smallest(v2[0], v2[1]);
          plain = most < 255 && most - low <= kLoose;
          if (plain) { top = min(min(most + kRoom, low + kLoose), 254); fresh = false; }
        } else if (plain) {
          plain = !above_top();
        }
        // (two copies: with keys that some row does not see or scales that need other references, and without any.  The latter
        // is the false one, and returns whether the other has to do the tile: nothing has changed then.)
        auto step = [&](auto tag) -> bool {
          constexpr bool careful = decltype(tag)::value;
          int least = 0;                                    // the smallest scale byte of the keys that some row sees
          bool other = mixed || fresh;                      // other references are needed
          bool odd_values = false;                          // NaN codes that not every row sees
          // s[x][t][2 e + i]: key 16 x + 2 g + e of the warp's, row i of this thread's in row tile t
          float s[2][NT][4];
#pragma unroll
          for (int x = 0; x < 2; ++x)
#pragma unroll
            for (int t = 0; t < NT; ++t) s[x][t][0] = s[x][t][1] = s[x][t][2] = s[x][t][3] = 0.f;
          {
            const uint32_t at[2] = {smem_u32(ks) + held_at<D>(frag_row, frag_piece), smem_u32(ks) + held_at<D>(frag_row + 16, frag_piece)};
#pragma unroll
            for (int k = 0; k < D / 32; ++k) {
              uint32_t a[2][2][4];                          // [x][group of 16 dims]: (even keys, dims 4j, 4j+1), (odd ..), (.., 4j+2, 4j+3)
#pragma unroll
              for (int x = 0; x < 2; ++x) {
                uint32_t c[4];                              // (even, dims 0-15), (odd, 0-15), (even, 16-31), (odd, 16-31)
                ldmatrix_x4(c, at[x] ^ (k << 5));
#pragma unroll
                for (int i = 0; i < 4; ++i) unpack_codes(c[i], a[x][i >> 1][i & 1], a[x][i >> 1][2 + (i & 1)]);
              }
#pragma unroll
              for (int y = 0; y < 2; ++y)
#pragma unroll
                for (int t = 0; t < NT; ++t) {
                  const uint2 q = q_frags[((2 * k + y) * 32 + lane) * NT + t];
#pragma unroll
                  for (int x = 0; x < 2; ++x) Fp16::mma(s[x][t], a[x][y], q.x, q.y);
                }
            }
          }
#pragma unroll
          for (int x = 0; x < 2; ++x) {
            const uint32_t kw = *reinterpret_cast<const uint16_t*>(ke + x * 16 + 2 * g);     // this thread's keys' scale bytes
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              // (byte 255 gives infinity here, less itself no number; byte 0 gives 0 for 2^-127)
              const float f = __uint_as_float(kw << (23 - 8 * e) & 0x7f800000u) * key_unit, z = f - f;
#pragma unroll
              for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int i = 0; i < 2; ++i) s[x][t][2 * e + i] = fmaf(s[x][t][2 * e + i], f, z);
            }
          }
          if (careful) {
#pragma unroll
            for (int x = 0; x < 2; ++x)
#pragma unroll
              for (int e = 0; e < 2; ++e) {
                const int key = key0[x] + 2 * g + e;
#pragma unroll
                for (int t = 0; t < NT; ++t)
#pragma unroll
                  for (int i = 0; i < 2; ++i)
                    if (key > lim[t][i]) s[x][t][2 * e + i] = -INFINITY;
              }
            uint32_t unseen[2];
#pragma unroll
            for (int x = 0; x < 2; ++x) {
              unseen[x] = (key0[x] + 2 * g > lim_last ? 0xffffu : 0u) | (key0[x] + 2 * g + 1 > lim_last ? 0xffff0000u : 0u);
              v2[x] &= ~unseen[x];
            }
            least = smallest(v2[0] | unseen[0], v2[1] | unseen[1]);
            if (fresh) {
              // The first keys: where scales are near each other, and the largest is the same for every row that sees a key, one
              // reference does for all rows.
              const uint32_t u = __vmaxu2(v2[0], v2[1]);
              const int hi = (int)__reduce_max_sync(0xffffffffu, max(u & 0xffffu, u >> 16));
              if (hi < 255 && hi - least <= kLoose - kRoom) {
                uint32_t row_most = 0, row_least = 0x7fffu;  // (bytes + 1; 0: no key)
#pragma unroll
                for (int t = 0; t < NT; ++t) {
                  uint32_t w = 0;                            // of the thread's two rows
#pragma unroll
                  for (int x = 0; x < 2; ++x)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                      const int key = key0[x] + 2 * g + e;
                      const uint32_t b = (e ? v2[x] >> 16 : v2[x] & 0xffffu) + 1;
                      w = __vmaxu2(w, (key <= lim[t][0] ? b : 0) | (key <= lim[t][1] ? b << 16 : 0));
                    }
#pragma unroll
                  for (int d = 4; d < 32; d <<= 1) w = __vmaxu2(w, __shfl_xor_sync(0xffffffffu, w, d));
#pragma unroll
                  for (int i = 0; i < 2; ++i) {
                    const uint32_t b = i ? w >> 16 : w & 0xffffu;
                    row_most = max(row_most, b);
                    if (b > 0) row_least = min(row_least, b);
                  }
                }
                row_most = __reduce_max_sync(0xffffffffu, row_most);
                row_least = __reduce_min_sync(0xffffffffu, row_least);
                if (row_most == row_least) {
                  top = min((int)row_most - 1 + kRoom, 254);
                  low = least;
                  fresh = other = false;
                }
              }
            } else {
              other |= above_top();
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
            if (!BLOCK && !all_seen && lim_all < lim_last) {
              uint32_t bad = 0;
              for (int i = lane; i < 32 * CPR; i += 32) {
                const uint4 c = *reinterpret_cast<const uint4*>(vs + held_at<D>(kg + i / CPR, i % CPR));
                bad |= nan_codes(c.x) | nan_codes(c.y) | nan_codes(c.z) | nan_codes(c.w);
              }
              odd_values = __any_sync(0xffffffffu, bad != 0);
            }
          }
          // maxima over the warp's keys.  (They are kept before the scale: the largest score less the maximum is then exactly 0.)
          float best[NT][2];
          bool moved = false;
#pragma unroll
          for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
              float u = fmaxf(fmaxf(s[0][t][i], s[0][t][2 + i]), fmaxf(s[1][t][i], s[1][t][2 + i]));
#pragma unroll
              for (int d = 4; d < 32; d <<= 1) u = fmaxf(u, __shfl_xor_sync(0xffffffffu, u, d));
              best[t][i] = fmaxf(m[t][i], u);
              moved |= best[t][i] > m[t][i];
            }
          bool had[NT][2], rose[NT][2];                     // the row had a key before; its maximum moved
#pragma unroll
          for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int i = 0; i < 2; ++i) { had[t][i] = m[t][i] > -INFINITY; rose[t][i] = best[t][i] > m[t][i]; }
          if (__any_sync(0xffffffffu, moved)) {
            // a largest score's key has its value's scale as product
            if (!careful) least = smallest(v2[0], v2[1]);
            if (least < top - kLoose) {
              if (careful) {
                other = true;
              } else {
                // (where that is not another key's)
                least = 1000;
#pragma unroll
                for (int t = 0; t < NT; ++t)
#pragma unroll
                  for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int x = 0; x < 2; ++x)
#pragma unroll
                      for (int e = 0; e < 2; ++e)
                        if (rose[t][i] && lim[t][i] >= 0 && s[x][t][2 * e + i] == best[t][i])
                          least = min(least, (int)(e ? v2[x] >> 16 : v2[x] & 0xffffu));
                least = __reduce_min_sync(0xffffffffu, least);
                if (least < top - kLoose) return true;
              }
            }
            low = min(low, least);
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
              for (int i = 0; i < 2; ++i) {
                const float f = rose[t][i] ? ex2_approx((m[t][i] - best[t][i]) * sl[t][i]) : 1.f;
                l[t][i] *= f;
#pragma unroll
                for (int b = 0; b < D / 16; ++b) { o[t][b][i] *= f; o[t][b][2 + i] *= f; }
                m[t][i] = best[t][i];
              }
          }
#pragma unroll
          for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
              // (a row that has seen nothing yet: every term exp2(-inf - 0) = 0)
              const float u = m[t][i] == -INFINITY ? 0.f : m[t][i];
#pragma unroll
              for (int x = 0; x < 2; ++x)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                  float& a = s[x][t][2 * e + i];
                  a = ex2_approx(fmaf(a - u, sl[t][i], kShift));
                  l[t][i] += a;
                }
            }
          // probabilities times the values' scales
          if (!careful || !other) {
            const uint32_t floor2 = (uint32_t)max(top - 127, 0) * 0x00010001u, shift2 = (uint32_t)(127 - top) * 0x00010001u;
#pragma unroll
            for (int x = 0; x < 2; ++x) {
              const uint32_t w = __vmaxu2(v2[x], floor2) + shift2;      // exponent fields, 0 if that is less
#pragma unroll
              for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int e = 0; e < 2; ++e)
#pragma unroll
                  for (int i = 0; i < 2; ++i) s[x][t][2 * e + i] *= __uint_as_float(e ? w << 7 & 0x7f800000u : w << 23);
            }
          } else {
            int most[NT][2], product[NT][2], mine[NT][2];    // of the keys that a row sees: largest byte, largest product; its own `low`
            int all_product = 0, all_most = -1, all_low = 1000;
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
              for (int i = 0; i < 2; ++i) {
                const int ref = mixed ? refs[16 * t + 2 * i] : top;
                int u = -1, v = kNone;
#pragma unroll
                for (int x = 0; x < 2; ++x)
#pragma unroll
                  for (int e = 0; e < 2; ++e) {
                    const int byte = (int)(e ? v2[x] >> 16 : v2[x] & 0xffffu), field = (int)(__float_as_uint(s[x][t][2 * e + i]) >> 23);
                    if (byte < 255 && key0[x] + 2 * g + e <= lim[t][i]) {
                      u = max(u, byte);
                      if (field > 0) v = max(v, field - 127 - (int)kShift + byte);     // (0, or below what 32 bits hold well)
                    }
                  }
#pragma unroll
                for (int d = 4; d < 32; d <<= 1) {
                  u = max(u, __shfl_xor_sync(0xffffffffu, u, d));
                  v = max(v, __shfl_xor_sync(0xffffffffu, v, d));
                }
                most[t][i] = u;
                product[t][i] = v;
                // (a new maximum is among the products)
                mine[t][i] = max(v, rose[t][i] && u >= 0 ? kNone : mixed ? ref - kLoose : low);
                if (lim[t][i] >= 0 && m[t][i] > -INFINITY) {
                  all_product = max(all_product, v);
                  all_most = max(all_most, u);
                  all_low = min(all_low, mine[t][i]);
                }
              }
            // One reference for all rows if there is one that their largest products allow, with room for larger scales, so that it
            // seldom moves.  (Not where some rows do not see all keys: those must not matter to them.)
            all_most = __reduce_max_sync(0xffffffffu, all_most);
            all_product = max((int)__reduce_max_sync(0xffffffffu, all_product), all_most);
            all_low = __reduce_min_sync(0xffffffffu, all_low);
            const int common = min(all_low + kLoose, max(fresh ? 0 : top, all_most + kRoom));
            const bool same = all_seen && common >= all_product && common <= 254;
            int ref_max = -1, ref_min = 1000;
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
              for (int i = 0; i < 2; ++i) {
                int ref = mixed ? refs[16 * t + 2 * i] : top;
                if (most[t][i] >= 0) {
                  const int want = !had[t][i] ? most[t][i] + kRoom : mixed || most[t][i] > ref ? max(top, most[t][i] + kRoom) : top;
                  const int own = min(max(max(product[t][i], 0), min(mine[t][i] + kLoose, want)), 254), to = same ? common : own;
                  const int by = ref - to, half = by / 2;
                  const float f0 = __uint_as_float((uint32_t)(127 + half) << 23), f1 = __uint_as_float((uint32_t)(127 + by - half) << 23);
#pragma unroll
                  for (int b = 0; b < D / 16; ++b) { o[t][b][i] = o[t][b][i] * f0 * f1; o[t][b][2 + i] = o[t][b][2 + i] * f0 * f1; }
                  ref = to;
                }
                __syncwarp();
                refs[16 * t + 2 * i] = ref;                  // (the same from all lanes of the row)
                if (lim[t][i] >= 0 && m[t][i] > -INFINITY) {
                  ref_max = max(ref_max, ref);
                  ref_min = min(ref_min, ref);
                }
#pragma unroll
                for (int x = 0; x < 2; ++x)
#pragma unroll
                  for (int e = 0; e < 2; ++e) {
                    const int byte = (int)(e ? v2[x] >> 16 : v2[x] & 0xffffu);
                    s[x][t][2 * e + i] *= __uint_as_float((uint32_t)min(max(127 + byte - ref, 0), 254) << 23);
                  }
              }
            ref_max = __reduce_max_sync(0xffffffffu, ref_max);
            ref_min = __reduce_min_sync(0xffffffffu, ref_min);
            low = all_low;
            if (ref_max >= 0) {                              // (some row has a key)
              mixed = ref_max != ref_min;
              top = ref_max;
              fresh = false;
            }
          }
          if (careful) {
#pragma unroll
            for (int x = 0; x < 2; ++x)
#pragma unroll
              for (int e = 0; e < 2; ++e) {
                const int key = key0[x] + 2 * g + e;
                const bool none = (v2[x] >> (16 * e) & 0xffffu) == 255u;
#pragma unroll
                for (int t = 0; t < NT; ++t)
#pragma unroll
                  for (int i = 0; i < 2; ++i) {
                    if (none) s[x][t][2 * e + i] = __uint_as_float(0x7fc00000u);
                    if (key > lim[t][i]) s[x][t][2 * e + i] = 0.f;       // (unseen, whatever its scale)
                  }
              }
          }
          if (careful && !BLOCK && odd_values) {
            // added to the rows that see them, and taken out of the product, where 0 times them would reach the others
#pragma unroll 1
            for (int k = 0; k < 32; ++k) {
              const int key = key0[k >> 4] + (k & 15);
#pragma unroll
              for (int b = 0; b < D / 16; ++b) {
                const uint32_t c = nan_codes(*reinterpret_cast<const uint16_t*>(vs + held_at<D>(kg + k, b) + 2 * g));
#pragma unroll
                for (int t = 0; t < NT; ++t)
#pragma unroll
                  for (int i = 0; i < 2; ++i) {
                    if ((c & 0x80u) && key <= lim[t][i]) o[t][b][i] = __uint_as_float(0x7fc00000u);
                    if ((c & 0x8000u) && key <= lim[t][i]) o[t][b][2 + i] = __uint_as_float(0x7fc00000u);
                  }
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
            uint32_t pt[NT][2];                              // P^T: even keys, odd keys of the group by rows
#pragma unroll
            for (int t = 0; t < NT; ++t) {
              pt[t][0] = transpose_8x8(Fp16::pack(s[x][t][0], s[x][t][1]));
              pt[t][1] = transpose_8x8(Fp16::pack(s[x][t][2], s[x][t][3]));
            }
            const uint32_t at = smem_u32(vs) + held_at<D>(frag_row + 16 * x, frag_piece);
#pragma unroll
            for (int n = 0; n < D / 32; ++n) {
              uint32_t c[4];                                 // (even keys, dims 0-15), (odd, 0-15), (even, 16-31), (odd, 16-31)
              ldmatrix_x4_trans(c, at ^ (n << 5));
#pragma unroll
              for (int y = 0; y < 2; ++y) {
                // a word: one key's dims 2g, 2g+1, then the next key's; the two keys of a dim beside each other
                uint32_t a[4];
                unpack_codes(__byte_perm(c[2 * y], 0, 0x3120), a[0], a[1]);
                unpack_codes(__byte_perm(c[2 * y + 1], 0, 0x3120), a[2], a[3]);
#pragma unroll
                for (int t = 0; t < NT; ++t) Fp16::mma(o[t][2 * n + y], a, pt[t][0], pt[t][1]);
              }
            }
          }
          return false;
        };
        if (plain) plain = !step(std::false_type());
        if (!plain && (key0[0] <= lim_last || key0[1] <= lim_last)) step(std::true_type());
        __syncwarp();
        if (lane == 0) mbar_arrive(&empty[stage]);
      }

      // ---- the warps' softmaxes joined; a thread ends up with PER dims of a chunk of one row
      float unit[NT][2];
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int i = 0; i < 2; ++i) unit[t][i] = held_scale((uint32_t)(mixed ? refs[16 * t + 2 * i] : top)) * (1.f / (1 << (int)kShift));
      __syncwarp();
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          m[t][i] *= sl[t][i];                               // (from here on without the 2^kShift)
          l[t][i] *= 1.f / (1 << (int)kShift);
#pragma unroll
          for (int d = 4; d < 32; d <<= 1) l[t][i] += __shfl_xor_sync(0xffffffffu, l[t][i], d);
          if (g == 0) {
            stat[(warp * ROWS + 8 * t + 2 * j + i) * 2] = m[t][i];
            stat[(warp * ROWS + 8 * t + 2 * j + i) * 2 + 1] = l[t][i];
          }
        }
      named_barrier(1, WARPS * 32);
      // (a warp that has seen nothing has the sum 0; one that has seen no numbers alone has no maximum, but no 0 either)
      float f[NT][2];
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          float M = -INFINITY;
#pragma unroll
          for (int k = 0; k < WARPS; ++k) M = fmaxf(M, stat[(k * ROWS + 8 * t + 2 * j + i) * 2]);
          f[t][i] = l[t][i] == 0.f ? 0.f : ex2_approx(m[t][i] - M) * unit[t][i];
        }
      constexpr int PER = 16 / WARPS, TPR = C::CHUNK / PER;    // dims of a thread, threads of a row
      const int row = tid / TPR, dp = tid % TPR * PER;
      float M = -INFINITY, L = 0.f;
#pragma unroll
      for (int k = 0; k < WARPS; ++k) M = fmaxf(M, stat[(k * ROWS + row) * 2]);
#pragma unroll
      for (int k = 0; k < WARPS; ++k) {
        const float x = stat[(k * ROWS + row) * 2 + 1];
        if (x != 0.f) L += x * ex2_approx(stat[(k * ROWS + row) * 2] - M);
      }
      const bool fin = w.whole();              // in a cluster: the unit is this CTA's alone
      const int slot = w.slot(cta);
      const int r = w.r_first + row;
      const size_t out_row = (size_t)(w.tok0 + r / p.group) * p.hq + w.h * p.group + r % p.group;
      const float inv = L != 0.f ? 1.f / L : 0.f;
      // rows of CHUNK floats, each pair of rows turned by eight more, so that the accesses spread over the banks
      auto place = [](int row, int dim) { return row * C::CHUNK + ((dim + 8 * (row >> 1)) & (C::CHUNK - 1)); };
#pragma unroll
      for (int c = 0; c < D / C::CHUNK; ++c) {
        float* mine = red + warp * 512;
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
          for (int b = 0; b < C::CHUNK / 16; ++b) {
            const float (&x)[4] = o[t][c * (C::CHUNK / 16) + b];
#pragma unroll
            for (int i = 0; i < 2; ++i)
              *reinterpret_cast<float2*>(mine + place(8 * t + 2 * j + i, 16 * b + 2 * g)) = make_float2(x[i] * f[t][i], x[2 + i] * f[t][i]);
          }
        named_barrier(1, WARPS * 32);
        float a[PER];
#pragma unroll
        for (int e = 0; e < PER; ++e) a[e] = 0.f;
#pragma unroll
        for (int k = 0; k < WARPS; ++k)
#pragma unroll
          for (int e = 0; e < PER; e += 2) {
            const float2 u = *reinterpret_cast<const float2*>(red + k * 512 + place(row, dp) + e);
            a[e] += u.x; a[e + 1] += u.y;
          }
        if (row < w.rows) {
          float* part = (SPLIT ? keep + (size_t)row * D : p.row_part + ((size_t)slot * kRowTile + row) * D) + c * C::CHUNK + dp;
          uint32_t* y = reinterpret_cast<uint32_t*>(static_cast<uint16_t*>(p.y) + out_row * D + c * C::CHUNK + dp);
#pragma unroll
          for (int e = 0; e < PER; e += 2) {
            if (fin) y[e >> 1] = OutOfHeld<T>::type::pack(a[e] * inv, a[e + 1] * inv);
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
  if (SPLIT && p.n_split > 1) join_cluster<typename OutOfHeld<T>::type, D, BLOCK, kHeldKeys, WARPS>(p, cta, keep, keep_stat);
  __syncthreads();
  if (*s_abort && tid == 0) atomicExch(p.status, kStatusTimeout);
  // (beside a tile-kernel launch this grid may run next to it: it must not be complete before that one is, because the
  // joins that follow wait for this grid only)
  if (p.beside) pdl_wait();
}

template <typename T, int D, bool BLOCK, bool SPLIT, int NT>
static cudaError_t launch_rows_n(const PagedProblem& p, const HeldCache& held, const CUtensorMap& tk, const CUtensorMap& tv, int grid,
                                 cudaStream_t st) {
  using C = HeldRowCfg<D, SPLIT, NT>;
  static PerDeviceFlag configured;
  const cudaError_t e = set_max_dynamic_smem(configured, reinterpret_cast<const void*>(paged8_rows_kernel<T, D, BLOCK, SPLIT, NT>), C::total);
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
  return cudaLaunchKernelEx(&cfg, paged8_rows_kernel<T, D, BLOCK, SPLIT, NT>, tk, tv, p, held);
}

// Units of at most 8 rows by the kernel of one row tile, others by that of two.
template <typename T, int D, bool BLOCK, bool SPLIT>
static cudaError_t launch_rows_s(const PagedProblem& p, const HeldCache& held, const CUtensorMap& tk, const CUtensorMap& tv, int max_rows,
                                 int grid, cudaStream_t st) {
  return max_rows <= 8 ? launch_rows_n<T, D, BLOCK, SPLIT, 1>(p, held, tk, tv, grid, st)
                       : launch_rows_n<T, D, BLOCK, SPLIT, 2>(p, held, tk, tv, grid, st);
}

#define TKPHI_BY_TYPE(call)                                                          \
  (d == 64 ? (bf16 ? (block ? call(Bf16, 64, true) : call(Bf16, 64, false))           \
                   : (block ? call(Fp16, 64, true) : call(Fp16, 64, false)))          \
           : (bf16 ? (block ? call(Bf16, 128, true) : call(Bf16, 128, false))         \
                   : (block ? call(Fp16, 128, true) : call(Fp16, 128, false))))

int paged8_row_ctas(int d, int max_rows) {
  return d == 64 ? (max_rows <= 8 ? HeldRowCfg<64, false, 1>::CTAS : HeldRowCfg<64, false, 2>::CTAS)
                 : (max_rows <= 8 ? HeldRowCfg<128, false, 1>::CTAS : HeldRowCfg<128, false, 2>::CTAS);
}

cudaError_t launch_paged8_rows(const PagedProblem& p, const HeldCache& held, const CUtensorMap& tk, const CUtensorMap& tv, int d,
                               bool bf16, bool block, bool split, int max_rows, int grid, cudaStream_t st) {
#define ROWS(T, D, B) \
  (split ? launch_rows_s<T, D, B, true>(p, held, tk, tv, max_rows, grid, st) : launch_rows_s<T, D, B, false>(p, held, tk, tv, max_rows, grid, st))
  return TKPHI_BY_TYPE(ROWS);
#undef ROWS
}

cudaError_t launch_paged8_rows_merge(const PagedProblem& p, int d, bool bf16, bool block, int units, int max_rows, cudaStream_t st) {
#define MERGE(T, D, B) \
  launch_pdl(paged_rows_merge_kernel<OutOfHeld<T>::type, D, B, kHeldKeys>, dim3(units, max_rows), dim3(kMergeThreads), 0, st, p)
  return TKPHI_BY_TYPE(MERGE);
#undef MERGE
}

}  // namespace tkphi
