// Attention of many query rows over a paged cache (prefill, chunks of a prompt): the two products on tcgen05.
//
//   S = Q K^T (fp32, tensor memory), P = exp2(scale_log2 S - m) (16 bits), O = O + P V (fp32, tensor memory)
//
// with a reference m and the running sum of each row; y = O / sum.  A CTA owns 256 query rows of one KV head (tokens x
// query heads of the group, so that the group's heads share every key and value tile) as two MMA tiles of up to 128 rows
// (whole tokens), and a range of keys.  While the softmax warps of one tile work on its scores, the tensor pipe runs the
// other tile's products.  Per tile of 128 keys and 128 rows: 2 * 128 * 128 * head_dim FMAs of tensor work against 16384
// exponentials, at 16 per clock and SM as long as the tensor work at head_dim 128 and twice as long at 64.
//   warps 0-3, 4-7  softmax of row tile 0, 1: thread = row = tensor-memory lane, so that a row's sum needs no exchange.
//                   P is written over the scores it came from and read from there as the A operand.
//                   The reference m of a row need not be its maximum, it only has to keep P in range: it is the
//                   maximum of the first tile, and later tiles go straight from the score to exp2(score - m) without
//                   looking for theirs.  A tile whose row sum passes a limit (2^40; fp16: 61440, below which no term
//                   can overflow the type) or is no number is redone with its maximum as the new reference and O
//                   rescaled.  Both ways of computing exp2 let a term that is out of range fail that limit.
//                   At head_dim 64 a quarter of the exponentials are computed on the FMA pipes (exp2_pair).
//   warp 8          issues the MMAs: P V of a row tile as soon as its P is stored, then the next S into the same buffer.
//   warp 9          TMA producer: the queries, then page boxes of keys and values into one ring, in the order of their use.
//   warps 10, 11    look through the value tiles that not every row of the CTA sees whole (three at most), because 0 times an
//                   infinity or NaN would reach the rows that do not see it: value rows that no row sees are zeroed (behind
//                   the sequence's end they may hold anything), other elements that are not finite are zeroed and noted with
//                   the first key that has one in their dim, and added at the end to the rows that see that key.
// Rounding P to 16 bits (the kernel for few rows does not) is the only rounding besides the output's: per term it is that of
// one 16-bit rounding, and it averages out over the terms; bf16 outputs are off by 0.0022 (norm, against 0.0017 from their
// own rounding alone).  The sum is of the unrounded values.  fp16: P is scaled by 2^7 and the sum with it, because without it
// probabilities below 2^-24 of the maximum vanish, and a long context is made of those; with it they have all their bits down
// to 2^-21 of the reference and are off by 2^-32 of it below that.
// Keys are cut into chunks when there are too few row tiles to fill the SMs evenly; partial outputs are joined in key
// order by a second, dependent kernel.
// What it measured (24 / 8 heads of 128, 2048 tokens at the end of 32K; 32 / 8 heads of 64, 4096 at the end of 32K):
//   first version 954 / 565 TFLOP/s: the issuing thread needed 75 cycles per MMA, see there
//   convergent issue 1218 / 701; three score buffers at head_dim 64, a burst of MMAs per step, fewer commits 1203 / 868
//   queries by TMA, join in runs of rows 1190 / 896 (a group of 3 fills 126 of the 128 rows)
//   exponentials cut at both ends, values that not every row sees looked through, far references 1176 / 865-884
// Bound now: at head_dim 128 the chain of a row tile (scores, softmax, product) where the other row tile does not cover it
// (tensor pipe active 59%), under the power limit (the sustained library rate is 1344 TFLOP/s); at 64 the softmax warps'
// issue and special-function rate.  A CTA's set-up and its output take about 12K cycles, which shows where contexts are short
// (5K-8K prompts: 700-735 TFLOP/s).  Two issuing warps were slower (1005 / 631): the row tiles then run in phase and wait
// together.
#include <climits>

#include "paged.cuh"

namespace tkphi {

constexpr int kTileThreads = 384;
constexpr int kWarpMma = 8, kWarpTma = 9;
constexpr uint32_t kTileTmemCols = 512;      // S / P buffers of 128 columns, then the two outputs
// References in log2 units (and the -inf of a row that has seen nothing) beyond which every tile is done carefully: scale *
// score - scaled reference in one FMA carries the rounding of the reference, 2^-2 here, which beyond 2^31 would push the
// largest term out of range.  Carefully, the reference is taken off before the scale.
constexpr float kFarReference = 4194304.f;
constexpr float kGrow = 1.f;                 // log2: how far a tile's maximum passes the reference before it replaces it

// Two fp32 values as one operand of the packed FMA instructions.
__device__ __forceinline__ uint64_t pack2(float a, float b) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ void unpack2(uint64_t v, float& a, float& b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(v)); }
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
// exp2 of two values on the FMA and integer pipes: x = n + f with n the nearest integer, |f| <= 1/2, 2^f by the
// Chebyshev interpolation polynomial of degree 5 (relative error below 2^-22: the terms of the series beyond it,
// (ln 2 / 2)^6 / 6! = 2.4e-6, shrink by 2^5 when the six nodes are Chebyshev's), n added to the exponent field.
// Below -126 the result is 2^-126.  Above 127, where n would run into the sign, it is 2^127, which fails a row sum's limit
// (2^40 or less), so that the tile is redone with its maximum as the reference.  What is no number stays none until the
// integer addition, which makes a number near 2^128 of it: that fails the limit as well, and the redone sum is none.
__device__ __forceinline__ float exp2_range(float x) {
  float r;
  asm("max.NaN.f32 %0, %1, 0fC2FC0000;\n\tmin.NaN.f32 %0, %0, 0f42FE0000;" : "=f"(r) : "f"(x));      // [-126, 127]
  return r;
}
__device__ __forceinline__ uint64_t exp2_pair(uint64_t x2) {
  constexpr float c0 = 1.000000075e+00f, c1 = 6.931471880e-01f, c2 = 2.402210749e-01f, c3 = 5.550357114e-02f, c4 = 9.676031918e-03f, c5 = 1.339086336e-03f;
  float x, y;
  unpack2(x2, x, y);
  x2 = pack2(exp2_range(x), exp2_range(y));
  const uint64_t magic = pack2(12582912.f, 12582912.f), minus = pack2(-1.f, -1.f);      // 1.5 * 2^23: the sum's low bits are n
  const uint64_t t = add2(x2, magic);
  const uint64_t n = add2(t, pack2(-12582912.f, -12582912.f));
  const uint64_t f = fma2(n, minus, x2);
  uint64_t r = fma2(f, pack2(c5, c5), pack2(c4, c4));
  r = fma2(r, f, pack2(c3, c3));
  r = fma2(r, f, pack2(c2, c2));
  r = fma2(r, f, pack2(c1, c1));
  r = fma2(r, f, pack2(c0, c0));
  float a, b, ta, tb;
  unpack2(r, a, b);
  unpack2(t, ta, tb);
  return pack2(__int_as_float(__float_as_int(a) + (__float_as_int(ta) << 23)),
               __int_as_float(__float_as_int(b) + (__float_as_int(tb) << 23)));
}
// Which of the 16 pairs of a 32-column piece go through exp2_pair: a quarter at head_dim 64, where the special-function
// unit is the bound (4096 x 32K tokens, 32 / 8 heads, fp16: 1320 us with none, 1237 with an eighth, 1192 with a quarter, 1256
// with three eighths, 1430 with a half); none at 128, where it is not (2048 x 32K, 24 / 8 heads: 664 us with none or a
// quarter, 714 with a half).
template <int D>
__device__ __forceinline__ constexpr bool emulated(int e) { return D == 64 && e % 4 == 0; }
__device__ __forceinline__ bool elect_one() {
  uint32_t e;
  asm volatile("{\n .reg .pred p;\n elect.sync _|p, 0xffffffff;\n selp.b32 %0, 1, 0, p;\n}\n" : "=r"(e));
  return e != 0;
}
// Waits for this thread's tensor-memory loads; the values are tied to the wait.
__device__ __forceinline__ void tc_wait_ld_x32(float (&v)[32]) {
  asm volatile("tcgen05.wait::ld.sync.aligned;"
               : "+f"(v[0]), "+f"(v[1]), "+f"(v[2]), "+f"(v[3]), "+f"(v[4]), "+f"(v[5]), "+f"(v[6]), "+f"(v[7]),
                 "+f"(v[8]), "+f"(v[9]), "+f"(v[10]), "+f"(v[11]), "+f"(v[12]), "+f"(v[13]), "+f"(v[14]), "+f"(v[15]),
                 "+f"(v[16]), "+f"(v[17]), "+f"(v[18]), "+f"(v[19]), "+f"(v[20]), "+f"(v[21]), "+f"(v[22]), "+f"(v[23]),
                 "+f"(v[24]), "+f"(v[25]), "+f"(v[26]), "+f"(v[27]), "+f"(v[28]), "+f"(v[29]), "+f"(v[30]), "+f"(v[31])
               :
               : "memory");
}

template <int D>
struct TileCfg {
  static constexpr int HALVES = D / 64;
  static constexpr int BOX = 128 * 128;                      // bytes of one 64-dim half of 128 rows
  static constexpr int TILE = HALVES * BOX;
  static constexpr int NS = D == 128 ? 5 : 10;               // ring slots
  // Score buffers of 128 columns: as many as tensor memory has room for beside the two outputs.  With three, the next
  // scores of a row tile are computed while its softmax warps still work on the ones before.
  static constexpr int NB = D == 128 ? 2 : 3;
  static constexpr int O_COL = NB * 128;
  static constexpr int NV = 8;                               // more than the value tiles that the ring can hold
  static_assert(NV > NS / 2 + 2, "a phase of v_free may not come round while the producer waits for it");
  static constexpr size_t q = 0;
  static constexpr size_t ring = 2 * TILE;
  static constexpr size_t bars = ring + (size_t)NS * TILE;
  static constexpr size_t bar_bytes = 512;                   // barriers and four words
  static_assert((NS + NV + 3 * NB + 4 + 2 * 3) * 8 + 12 + 11 * 4 <= bar_bytes, "barriers");
  static constexpr size_t odd = bars + bar_bytes;            // [3][D] per dim the first key whose value is inf, -inf, NaN
  static constexpr size_t total = odd + 3 * D * sizeof(int);
};
constexpr int kMostMixed = 3;                // value tiles that some rows of a CTA see in part: 255 tokens touch three

__device__ __forceinline__ void tmem_st_x32(uint32_t taddr, const uint32_t* r) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], "
      "{%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, "
      "%17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31, %32};" ::"r"(taddr),
      "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]),
      "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]), "r"(r[17]), "r"(r[18]),
      "r"(r[19]), "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]),
      "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31])
      : "memory");
}
// 32 bytes, a whole sector (dst 32-byte aligned).
__device__ __forceinline__ void st_global_32(float* dst, const float* v) {
  asm volatile("st.global.v8.f32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(dst), "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]),
               "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7]) : "memory");
}
// kind::f16 instruction descriptor with both operands of one 16-bit type (1: bf16, 0: f16)
__host__ __device__ constexpr uint32_t umma_idesc_16(int bf16, int M, int N, int a_mn, int b_mn) {
  return (1u << 4) | ((uint32_t)bf16 << 7) | ((uint32_t)bf16 << 10) | ((uint32_t)a_mn << 15) | ((uint32_t)b_mn << 16) |
         ((uint32_t)(N >> 3) << 17) | ((uint32_t)(M >> 4) << 24);
}

// CTAs of a sequence: KV heads x key chunks x row tiles (pairs of MMA tiles).
struct TileSeq {
  int rows, len, chunks, row_tiles;
};
__device__ __forceinline__ TileSeq tile_seq_of(const PagedProblem& p, int b) {
  TileSeq s{0, 0, 1, 0};
  if (b >= p.batch) return s;
  const int q = paged_q_len(p, b);
  s.len = paged_kv_len(p, b);
  s.rows = q > 0 ? q * p.group : 0;
  if (s.rows <= p.rows_limit) s.rows = 0;
  const int pair = 2 * tile_rows(p.group);
  s.row_tiles = (s.rows + pair - 1) / pair;
  s.chunks = s.len > p.chunk ? (s.len + p.chunk - 1) / p.chunk : 1;
  return s;
}

// What a CTA works on.
struct TileWork {
  int seq;                                 // -1: nothing
  int h, c0, row0, rows, len, q_len, tok0, chunks;
  int n, tiles;                            // key tiles, row tiles
};

template <typename T, int D>
__global__ void __launch_bounds__(kTileThreads, 1)
paged_tiles_kernel(const __grid_constant__ CUtensorMap tmap_k, const __grid_constant__ CUtensorMap tmap_v,
                   const __grid_constant__ CUtensorMap tmap_q, const __grid_constant__ PagedProblem p) {
  using C = TileCfg<D>;
  constexpr int NS = C::NS, NV = C::NV;
  constexpr float kShift = T::kBf16 ? 0.f : 7.f;             // P = 2^kShift exp2(..)
  constexpr float kSumLimit = T::kBf16 ? 1.099511627776e12f : 61440.f;
  extern __shared__ __align__(1024) unsigned char smem[];
  unsigned char* qs = smem + C::q;
  unsigned char* ring = smem + C::ring;
  uint64_t* full = reinterpret_cast<uint64_t*>(smem + C::bars);   // [NS] tile landed
  uint64_t* v_free = full + NS;            // [NV] products of a key tile complete (key tile j: j % NV)
  uint64_t* s_full = v_free + NV;          // [NB] scores complete
  uint64_t* p_ready = s_full + C::NB;      // [NB] P stored
  uint64_t* o_full = p_ready + C::NB;      // [2]  last product of the row tile complete
  uint64_t* pv_done = o_full + 2;          // [NB] products whose completion no scores tell (more score buffers than row tiles)
  uint64_t* q_ready = pv_done + C::NB;     // [1]
  uint64_t* v_issued = q_ready + 1;        // [3]  copy of a mixed value tile issued
  uint64_t* v_fixed = v_issued + kMostMixed;   // [3]  that tile looked through
  uint64_t* drained = v_fixed + kMostMixed;    // [1]  after a wait that ran out: the MMAs issued so far are complete
  int* misc = reinterpret_cast<int*>(drained + 1);
  volatile int* s_abort = misc;
  uint32_t* s_tmem = reinterpret_cast<uint32_t*>(misc + 1);
  volatile int* s_odd = misc + 2;
  TileWork* s_work = reinterpret_cast<TileWork*>(misc + 3);
  int* odd_key = reinterpret_cast<int*>(smem + C::odd);
  const int tid = threadIdx.x, lane = tid & 31, warp = __shfl_sync(0xffffffffu, tid >> 5, 0);
  const int cta = blockIdx.x;

  pdl_wait();
  pdl_launch_next();
  if (warp == 0) {
    int base = 0;
    if (lane == 0) s_work->seq = -1;
    for (int s = 0; s < p.batch; s += 32) {
      const TileSeq q = tile_seq_of(p, s + lane);
      const int w = q.row_tiles * q.chunks * p.hkv, incl = warp_inclusive_scan(w) + base;
      if (incl > cta && incl - w <= cta) {             // one lane
        const int b = s + lane;
        int i = cta - (incl - w);
        TileWork k;
        k.seq = b;
        k.q_len = paged_q_len(p, b);
        k.tok0 = (int)__ldg(p.cu_q + b);
        k.row0 = (q.row_tiles - 1 - i % q.row_tiles) * 2 * tile_rows(p.group);       // the rows that see most first
        i /= q.row_tiles;
        k.c0 = (i % q.chunks) * p.chunk;
        k.h = i / q.chunks;
        k.rows = q.rows; k.len = q.len; k.chunks = q.chunks;
        const int pair = 2 * tile_rows(p.group), rows = q.rows - k.row0 < pair ? q.rows - k.row0 : pair;
        k.tiles = rows > pair / 2 ? 2 : 1;
        // up to the last key that the last row sees; both row tiles take all of these (the first one may see less: masked)
        int end = p.causal ? q.len - k.q_len + (k.row0 + rows - 1) / p.group + 1 : q.len;
        if (end > k.c0 + p.chunk) end = k.c0 + p.chunk;
        k.n = end > k.c0 ? (end - k.c0 + kTileKeys - 1) / kTileKeys : 0;
        *s_work = k;
      }
      base = __shfl_sync(0xffffffffu, incl, 31);
      if (base > cta) break;
    }
  } else if (warp == 1) {
    tmem_alloc(s_tmem, kTileTmemCols);
  } else if (tid == 64) {
    for (int s = 0; s < NS; ++s) mbar_init(&full[s], 1);
    for (int s = 0; s < NV; ++s) mbar_init(&v_free[s], 1);
    for (int i = 0; i < C::NB; ++i) { mbar_init(&s_full[i], 1); mbar_init(&p_ready[i], 4); }
    mbar_init(&o_full[0], 1); mbar_init(&o_full[1], 1);
    for (int i = 0; i < C::NB; ++i) mbar_init(&pv_done[i], 1);
    mbar_init(q_ready, 1);
    for (int i = 0; i < kMostMixed; ++i) { mbar_init(&v_issued[i], 1); mbar_init(&v_fixed[i], 2); }
    mbar_init(drained, 1);
    mbar_fence_init();
    *s_abort = 0;
    *s_odd = 0;
  } else if (warp >= 8) {
    for (int i = tid - 256; i < 3 * D; i += 128) odd_key[i] = INT_MAX;
  }
  tc_fence_before_sync();
  __syncthreads();
  tc_fence_after_sync();
  const uint32_t tmem = *s_tmem;
  const TileWork k = *s_work;
  const int b = k.seq, n = b >= 0 ? k.n : 0, tiles = b >= 0 ? k.tiles : 1;
  const int h = k.h, c0 = k.c0, row0 = k.row0, q_len = k.q_len, t_rows = tile_rows(p.group);
  // Keys up to vis0 are visible to every row of the CTA, from vis1 on to none.  Value tiles from `mixed` on are neither.
  // (A CTA without work, as in a replay with shorter lengths, has n = 0 and nothing else in k that means anything.)
  const int pair_rows = k.rows - row0 < 2 * t_rows ? k.rows - row0 : 2 * t_rows;
  const int vis0 = p.causal ? k.len - q_len + row0 / p.group + 1 : k.len;
  const int vis1 = p.causal ? k.len - q_len + (row0 + pair_rows - 1) / p.group + 1 : k.len;
  const int mixed = n == 0 || vis0 <= c0 ? 0 : (vis0 - c0) / kTileKeys < n ? (vis0 - c0) / kTileKeys : n;
  // Scores, P and products run through one sequence: number i = key tile * tiles + row tile, buffer i % NB.  Keys are
  // used `lead` tiles ahead of values: the ring holds K 0 .. K lead-1, V 0, K lead, V 1, ..
  const int lead = (C::NB + tiles - 1) / tiles;

  if (warp < 8) {
    // ================================================================ softmax: thread = row
    asm volatile("setmaxnreg.inc.sync.aligned.u32 208;");
    const int t = warp >> 2, quad = warp & 3;
    const int nt = t < tiles ? n : 0;
    // The row's place: computed here and again at the end (the loop between has no registers to spare).
    auto row_of = [&](int& row) {
      const volatile TileWork* w = s_work;
      const int r = tid & 127;
      row = w->row0 + t * t_rows + r;
      return w->seq >= 0 && r < t_rows && row < w->rows;
    };
    int row;
    const bool live = row_of(row);
    // last visible key; rows without a query (their tile rows hold anything) run along, have no say and are not stored
    const int lim = !live ? INT_MAX : p.causal ? k.len - q_len + row / p.group : k.len - 1;
    const uint32_t o_addr = tmem_addr(tmem, quad * 32, C::O_COL + t * D);
    int buf = t;
    uint32_t phase = 0;
    float m = -INFINITY, l = 0.f;                              // the reference (a score, before the scale) and the sum
    bool ok = true;
    for (int j = 0; j < nt; ++j) {
      ok = __all_sync(0xffffffffu, mbar_wait(&s_full[buf], phase, s_abort));
      if (!ok) break;
      tc_fence_after_sync();
      const uint32_t s_addr = tmem_addr(tmem, quad * 32, buf * 128);
      const int key0 = c0 + j * kTileKeys;
      uint32_t w[64];
      bool careful = j == 0 || __any_sync(0xffffffffu, live && (key0 + kTileKeys - 1 > lim || !(fabsf(m * p.scale_log2) < kFarReference)));
      if (!careful) {
        const float off = fmaf(-m, p.scale_log2, kShift);
        const uint64_t scale2 = pack2(p.scale_log2, p.scale_log2), off2 = pack2(off, off);
        uint64_t sum2[2] = {0, 0};
        float u[32], v[32];
        // pairs of a 32-column piece: the first kEmulated on the FMA pipes, spread between the others
        auto piece = [&](const float (&x)[32], int c) {
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            const uint64_t y = fma2(pack2(x[2 * e], x[2 * e + 1]), scale2, off2);
            uint64_t r;
            if (emulated<D>(e)) {
              r = exp2_pair(y);
            } else {
              float a, d;
              unpack2(y, a, d);
              r = pack2(ex2_approx(a), ex2_approx(d));
            }
            sum2[e & 1] = add2(sum2[e & 1], r);
            float a, d;
            unpack2(r, a, d);
            w[c * 16 + e] = T::pack(a, d);
          }
        };
        tmem_ld_x32(s_addr, u);
        tc_wait_ld_x32(u);
        tmem_ld_x32(s_addr + 32, v);
        piece(u, 0);
        tc_wait_ld_x32(v);
        tmem_ld_x32(s_addr + 64, u);
        piece(v, 1);
        tc_wait_ld_x32(u);
        tmem_ld_x32(s_addr + 96, v);
        piece(u, 2);
        tc_wait_ld_x32(v);
        piece(v, 3);
        float a, d;
        unpack2(add2(sum2[0], sum2[1]), a, d);
        careful = __any_sync(0xffffffffu, live && !(a + d < kSumLimit));
        if (!careful) l += a + d;
      }
      if (careful) {
        float s[4][32];
#pragma unroll
        for (int c = 0; c < 4; ++c) tmem_ld_x32(s_addr + c * 32, s[c]);
        tc_wait_ld();
        if (__any_sync(0xffffffffu, key0 + kTileKeys - 1 > lim)) {
#pragma unroll
          for (int c = 0; c < 4; ++c)
#pragma unroll
            for (int e = 0; e < 32; ++e)
              if (key0 + c * 32 + e > lim) s[c][e] = -INFINITY;
        }
        float mx[4];
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          mx[c] = fmaxf(s[c][0], s[c][1]);
#pragma unroll
          for (int e = 2; e < 32; e += 2) mx[c] = fmaxf(mx[c], fmaxf(s[c][e], s[c][e + 1]));
        }
        const float cand = fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3]));
        const bool grow = live && (cand - m) * p.scale_log2 > kGrow;
        if (__any_sync(0xffffffffu, grow)) {
          const float f = grow ? ex2_approx((m - cand) * p.scale_log2) : 1.f;   // m = -inf: 0
          if (j > 0) {
            // The product before this one must be complete.  With as many score buffers as row tiles these scores were
            // issued after it.  With three buffers and two row tiles the next scores were (or, where there are none, it
            // has a barrier of its own); with one row tile every product tells its buffer's barrier.  (One barrier for all
            // would not do: up to three products may be pending here, and two phases look alike.)
            if (tiles == 1) {
              ok = __all_sync(0xffffffffu, mbar_wait(&pv_done[(j - 1) % C::NB], (uint32_t)((j - 1) / C::NB) & 1u, s_abort));
              tc_fence_after_sync();
            } else if (C::NB == 3) {
              const int nb = buf + 1 == C::NB ? 0 : buf + 1;
              ok = __all_sync(0xffffffffu, 2 * j + t + 1 < 2 * n ? mbar_wait(&s_full[nb], nb ? phase : phase ^ 1u, s_abort)
                                                                 : mbar_wait(&pv_done[0], 0, s_abort));
              tc_fence_after_sync();
            }
#pragma unroll
            for (int c = 0; c < D / 32; ++c) {
              float o[32];
              tmem_ld_x32(o_addr + c * 32, o);
              tc_wait_ld();
              uint32_t x[32];
#pragma unroll
              for (int e = 0; e < 32; ++e) x[e] = __float_as_uint(o[e] * f);
              tmem_st_x32(o_addr + c * 32, x);
            }
          }
          l *= f;
          if (grow) m = cand;
        }
        const float ref = m == -INFINITY ? 0.f : m, off = fmaf(-ref, p.scale_log2, kShift);
        float sum[4] = {0.f, 0.f, 0.f, 0.f};
        auto terms = [&](auto arg) {
#pragma unroll
          for (int c = 0; c < 4; ++c)
#pragma unroll
            for (int e = 0; e < 16; ++e) {
              const float a = ex2_approx(arg(s[c][2 * e])), d = ex2_approx(arg(s[c][2 * e + 1]));
              sum[(c & 1) * 2] += a;
              sum[(c & 1) * 2 + 1] += d;
              w[c * 16 + e] = T::pack(a, d);
            }
        };
        // far: the difference before the scale, exactly 0 for the score that is the reference, whatever its size
        if (__any_sync(0xffffffffu, live && fabsf(off) >= kFarReference)) terms([&](float x) { return fmaf(x - ref, p.scale_log2, kShift); });
        else terms([&](float x) { return fmaf(x, p.scale_log2, off); });
        l += (sum[0] + sum[1]) + (sum[2] + sum[3]);
      }
      tmem_st_x32(s_addr, w);
      tmem_st_x32(s_addr + 32, w + 32);
      tc_wait_st();
      tc_fence_before_sync();
      __syncwarp();
      if (lane == 0) mbar_arrive(&p_ready[buf]);
      buf += tiles;
      if (buf >= C::NB) { buf -= C::NB; phase ^= 1u; }
    }
    if (ok && nt > 0) ok = __all_sync(0xffffffffu, mbar_wait(&o_full[t], 0, s_abort));
    for (int i = 0; i < nt - mixed && ok; ++i) ok = __all_sync(0xffffffffu, mbar_wait(&v_fixed[i], 0, s_abort));
    // the values that are not finite, of the keys that this row sees
    const bool odd = nt > 0 && *s_odd;
    auto add_odd = [&](float (&o)[32], int c) {
      const int* first = odd_key + c * 32;
#pragma unroll
      for (int e = 0; e < 32; ++e) {
        if (first[e] <= lim) o[e] += INFINITY;
        if (first[D + e] <= lim) o[e] -= INFINITY;
        if (first[2 * D + e] <= lim) o[e] = __int_as_float(0x7fffffff);
      }
    };
    if (ok && b >= 0) {
      tc_fence_after_sync();
      const volatile TileWork* w = s_work;
      int row;
      const bool live = row_of(row);
      if (w->chunks == 1) {
        const size_t out_row = live ? ((size_t)w->tok0 + row / p.group) * p.hq + (size_t)w->h * p.group + row % p.group : 0;
        const float inv = l != 0.f ? 1.f / l : 0.f;          // (a sum that is no number: so are y and lse)
        uint4* y = reinterpret_cast<uint4*>(static_cast<uint16_t*>(p.y) + out_row * D);
#pragma unroll
        for (int c = 0; c < D / 32; ++c) {
          float o[32];
          if (nt > 0) {                        // warp-uniform
            tmem_ld_x32(o_addr + c * 32, o);
            tc_wait_ld();
            if (odd) add_odd(o, c);
          }
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            uint4 v = make_uint4(0, 0, 0, 0);
            if (l != 0.f) {
              v.x = T::pack(o[8 * e] * inv, o[8 * e + 1] * inv); v.y = T::pack(o[8 * e + 2] * inv, o[8 * e + 3] * inv);
              v.z = T::pack(o[8 * e + 4] * inv, o[8 * e + 5] * inv); v.w = T::pack(o[8 * e + 6] * inv, o[8 * e + 7] * inv);
            }
            if (live) y[c * 4 + e] = v;
          }
        }
        if (live && p.lse) p.lse[out_row] = l != 0.f ? (m * p.scale_log2 - kShift + log2f(l)) * 0.6931471805599453f : -INFINITY;
      } else {
        const size_t slot_row = (size_t)cta * kTileRows + t * t_rows + (tid & 127);
        if (live) reinterpret_cast<float2*>(p.tile_stat)[slot_row] = make_float2(l != 0.f ? m * p.scale_log2 - kShift : -INFINITY, l);
        if (nt > 0) {
          float* dst = p.tile_part + slot_row * D;
#pragma unroll
          for (int c = 0; c < D / 32; ++c) {
            float o[32];
            tmem_ld_x32(o_addr + c * 32, o);
            tc_wait_ld();
            if (odd) add_odd(o, c);
#pragma unroll
            for (int e = 0; e < 4; ++e)
              if (live) st_global_32(dst + c * 32 + e * 8, &o[e * 8]);
          }
        }
      }
    }
  } else {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 88;");
    if (warp == kWarpTma && n > 0) {
      // ================================================================ TMA producer
      const int ps = 1 << p.page_shift;
      const int box_rows = ps < 64 ? ps : 64, boxes = kTileKeys / box_rows;
      const int copies = C::HALVES * boxes, half = lane / boxes, bx = lane % boxes;
      const int page_off = (bx * box_rows) >> p.page_shift, row_off = (bx * box_rows) & (ps - 1);
      const uint32_t dst_off = half * C::BOX + bx * box_rows * 128;
      const int n_pages_seq = (k.len + ps - 1) >> p.page_shift;
      const int* list = p.table + (size_t)b * p.max_pages;
      const uint64_t pol = l2_policy_normal();
      // page ids of the keys' and of the values' tiles: 32 at a time, the next 32 fetched ahead
      int batch0[2], id[2], id_next[2];
      batch0[0] = batch0[1] = (c0 >> p.page_shift) & ~31;
      id[0] = id[1] = batch0[0] + lane < n_pages_seq ? __ldg(list + batch0[0] + lane) : p.n_pages;
      id_next[0] = id_next[1] = batch0[0] + 32 + lane < n_pages_seq ? __ldg(list + batch0[0] + 32 + lane) : p.n_pages;
      int slot = 0;
      uint32_t phase = 0;
      // the queries: tokens x the group's heads, 64 dims at a time (a second tile of other tokens is not used)
      if (lane == 0) mbar_expect_tx(q_ready, (uint32_t)(tiles * C::HALVES * t_rows * 128));
      __syncwarp();
      if (lane < tiles * C::HALVES)
        tma_load_4d(qs + (lane / C::HALVES) * C::TILE + (lane % C::HALVES) * C::BOX, &tmap_q, q_ready, (lane % C::HALVES) * 64, 0,
                    h, k.tok0 + (row0 + (lane / C::HALVES) * t_rows) / p.group, pol);
      int issued = 0;
      uint32_t pending = 0, parity = 0;                       // slots with a copy issued, and its phase
      bool ok = true;
      auto load = [&](int x, int j) {                         // x: 0 keys, 1 values
        const int first = (c0 + j * kTileKeys) >> p.page_shift;
        if (first >= batch0[x] + 32) {
          batch0[x] += 32;
          id[x] = id_next[x];
          id_next[x] = batch0[x] + 32 + lane < n_pages_seq ? __ldg(list + batch0[x] + 32 + lane) : p.n_pages;
        }
        int page = __shfl_sync(0xffffffffu, id[x], (first + page_off) & 31);
        if (page < 0 || page > p.n_pages || (page == p.n_pages && first + page_off < n_pages_seq)) {
          if (lane < boxes) atomicExch(p.status, kStatusBadPage);
          page = p.n_pages;                                   // a box outside the tensor arrives as zeros
        }
        // The slot's last tile: number issued - NS of the ring's order.  Keys are free when the products of their own
        // tile number (less the keys' lead) are complete, because all scores issued before those are, too.
        const int old = issued++ - NS;
        if (old >= 0) {
          const int oj = old < lead ? 0 : ((old - lead) & 1) ? (old - lead + 1) / 2 : (old - lead) / 2;
          ok = __all_sync(0xffffffffu, mbar_wait(&v_free[oj % NV], (uint32_t)(oj / NV) & 1u, s_abort));
          if (!ok) return;
        }
        if (lane == 0) mbar_expect_tx(&full[slot], C::TILE);
        __syncwarp();
        if (lane < copies)
          tma_load_4d(ring + (size_t)slot * C::TILE + dst_off, x ? &tmap_v : &tmap_k, &full[slot], half * 64, row_off, h,
                      page, pol);
        pending |= 1u << slot;
        parity = (parity & ~(1u << slot)) | (phase << slot);
        if (x && j >= mixed && lane == 0) mbar_arrive(&v_issued[j - mixed]);
        if (++slot == NS) { slot = 0; phase ^= 1u; }
      };
      for (int jk = 0, jv = 0; jv < n && ok;) {
        if (jk < n && jk < jv + lead) load(0, jk++);
        else load(1, jv++);
      }
      if (!ok) {
        // every copy that was issued must land before shared memory is released
        for (uint32_t w = 0; w < kWaitPolls && !mbar_try_wait(q_ready, 0); ++w) __nanosleep(64);
        for (int s = 0; s < NS; ++s)
          for (uint32_t w = 0; (pending >> s & 1u) && w < kWaitPolls; ++w) {
            if (mbar_try_wait(&full[s], parity >> s & 1u)) break;
            __nanosleep(64);
          }
      }
    } else if (warp == kWarpMma && n > 0) {
      // ================================================================ MMA issuer
      // The whole warp runs this code and one elected lane issues: descriptors then stay in uniform registers, where
      // the instruction takes them from.  (In a branch of one lane every MMA cost about 75 cycles of moves to issue, more
      // than it took to execute.)  A wait that runs out raises the abort flag; this warp then issues the rest without
      // waiting long, which touches only this CTA's own memory.
      constexpr int NB = C::NB;
      constexpr uint32_t idesc_s = umma_idesc_16(T::kBf16, 128, kTileKeys, 0, 0);
      constexpr uint32_t idesc_o = umma_idesc_16(T::kBf16, 128, D, 0, 1);
      const uint32_t tm = __shfl_sync(0xffffffffu, tmem, 0), base = __shfl_sync(0xffffffffu, smem_u32(smem), 0);
      const int nu = __shfl_sync(0xffffffffu, n, 0), T2 = __shfl_sync(0xffffffffu, tiles, 0), L = __shfl_sync(0xffffffffu, lead, 0);
      const int mixed_u = __shfl_sync(0xffffffffu, mixed, 0);
      const uint64_t q_desc = umma_smem_desc(base + (uint32_t)C::q, 16, 1024);
      const uint64_t k_desc = umma_smem_desc(base + (uint32_t)C::ring, 16, 1024);
      const uint64_t v_desc = umma_smem_desc(base + (uint32_t)C::ring, C::BOX, 1024);   // MN-major: 64-dim blocks BOX bytes apart
      auto wait_on = [&](uint64_t* bar, uint32_t parity) {
        mbar_wait(bar, parity, s_abort);
        __syncwarp();
      };
      // Ring slots and phases of the next key and value tiles.  In the ring's order a value tile follows every key tile
      // from the lead-th on, until the keys run out.
      int k_slot = 0, v_slot = 0, v_next = 0;
      uint32_t k_phase = 0, v_phase = 0;
      auto advance = [](int& slot, uint32_t& phase, int by) {
        slot += by;
        if (slot >= NS) { slot -= NS; phase ^= 1u; }
      };
      static_assert(NS > 3, "a step of the ring passes its end once at most");
      auto issue_scores = [&](int t, int buf) {                 // (elected lane)
        const uint64_t qd = q_desc + (uint64_t)((t * C::TILE) >> 4), kd = k_desc + (uint64_t)((k_slot * C::TILE) >> 4);
#pragma unroll
        for (int k = 0; k < D / 16; ++k) {
          const uint64_t off = (uint64_t)(((k >> 2) * C::BOX + (k & 3) * 32) >> 4);
          umma_ss(tm + buf * 128, qd + off, kd + off, idesc_s, k ? 1u : 0u);
        }
        tc_commit(&s_full[buf]);
      };
      auto wait_keys = [&](int j) {
        if (j > 0) advance(k_slot, k_phase, j < L ? 1 : 2);
        wait_on(&full[k_slot], k_phase);
      };
      auto wait_values = [&](int j) {
        advance(v_next, v_phase, j == 0 ? (L < nu ? L : nu) : j + L <= nu ? 2 : 1);
        wait_on(&full[v_next], v_phase);
        if (j >= mixed_u) wait_on(&v_fixed[j - mixed_u], 0);
      };
      wait_on(q_ready, 0);
      int sj = 0, st = 0;                                       // next scores to issue
      for (int i = 0; i < NB && sj < nu; ++i) {
        if (st == 0) wait_keys(sj);
        tc_fence_after_sync();
        if (elect_one()) issue_scores(st, i);
        __syncwarp();
        if (++st == T2) { st = 0; ++sj; }
      }
      if (NB == 3) {
        wait_values(0);
        v_slot = v_next;
        if (st == 0 && sj < nu) wait_keys(sj);
      }
      int buf = 0;
      uint32_t phase = 0;
      // One burst per step: the product of a row tile, then its buffer's next scores.  What a burst needs beside P has
      // been waited for after an earlier one, while that one's MMAs ran.
      for (int j = 0; j < nu; ++j) {
        if (NB == 2) {
          wait_values(j);
          v_slot = v_next;
        }
        for (int t = 0; t < T2; ++t) {
          if (NB == 2 && st == 0 && sj < nu) wait_keys(sj);
          wait_on(&p_ready[buf], phase);
          const uint64_t vd = v_desc + (uint64_t)((v_slot * C::TILE) >> 4);
          tc_fence_after_sync();
          if (elect_one()) {
#pragma unroll
            for (int k = 0; k < kTileKeys / 16; ++k)
              umma_ts(tm + C::O_COL + t * D, tm + buf * 128 + k * 8, vd + (uint64_t)((k * 16 * 128) >> 4), idesc_o,
                      (j > 0 || k > 0) ? 1u : 0u);
            if (sj < nu) issue_scores(st, buf);
            if (t + 1 == T2) tc_commit(&v_free[j % NV]);
            if (j + 1 == nu) tc_commit(&o_full[t]);
            if (T2 == 1) tc_commit(&pv_done[buf]);
            else if (NB == 3 && t == 1 && j + 2 == nu) tc_commit(&pv_done[0]);
          }
          __syncwarp();
          if (++st == T2) { st = 0; ++sj; }
          if (NB == 3 && t + 1 == T2 && j + 1 < nu) wait_values(j + 1);
          if (NB == 3 && st == 0 && sj < nu) wait_keys(sj);
          if (++buf == NB) { buf = 0; phase ^= 1u; }
        }
        if (NB == 3) v_slot = v_next;
      }
      if (*s_abort) {                        // tensor memory is released only when no MMA uses it any more
        if (elect_one()) {
          tc_commit(drained);
          for (uint32_t w = 0; w < kWaitPolls && !mbar_try_wait(drained, 0); ++w) __nanosleep(64);
        }
        __syncwarp();
      }
    } else if (warp > kWarpTma) {
      // ================================================================ values that not every row sees
      constexpr int CPR = D / 8;                                // 16-byte pieces of a row
      bool ok = true;
      for (int j = mixed; j < n && ok; ++j) {
        // V j is number min(j + lead, n) + j of the ring.  Its slot's barrier is waited for only once the copy is issued: from
        // then on it is in the phase of this copy until the tile has been used, which needs this warp.
        ok = __all_sync(0xffffffffu, mbar_wait(&v_issued[j - mixed], 0, s_abort));
        const int number = (j + lead < n ? j + lead : n) + j, slot = number % NS;
        if (ok) ok = __all_sync(0xffffffffu, mbar_wait(&full[slot], (uint32_t)(number / NS) & 1u, s_abort));
        if (!ok) break;
        unsigned char* v = ring + (size_t)slot * C::TILE;
        const int key0 = c0 + j * kTileKeys;
        const int seen = vis1 - key0 < kTileKeys ? vis1 - key0 : kTileKeys, from = vis0 > key0 ? vis0 - key0 : 0;
#pragma unroll 2
        for (int x = from * CPR + tid - (kWarpTma + 1) * 32; x < kTileKeys * CPR; x += 64) {
          const int row = x / CPR, c = x % CPR;
          uint4* at = reinterpret_cast<uint4*>(v + (c >> 3) * C::BOX + swz128(row, c & 7));
          uint4 w = *at;
          if (row < seen && not_finite<T>(w)) {
            uint32_t* ws = reinterpret_cast<uint32_t*>(&w);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              uint32_t& word = ws[e >> 1];
              const float f = e & 1 ? T::hi(word) : T::lo(word);
              if (fabsf(f) < INFINITY) continue;
              atomicMin(&odd_key[(f != f ? 2 : f < 0.f ? 1 : 0) * D + c * 8 + e], key0 + row);
              word &= e & 1 ? 0xffffu : 0xffff0000u;
            }
            *s_odd = 1;
            *at = w;
          } else if (row >= seen) {
            *at = make_uint4(0, 0, 0, 0);
          }
        }
        fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) mbar_arrive(&v_fixed[j - mixed]);
      }
    }
  }
  // ---- teardown
  tc_fence_before_sync();
  __syncthreads();
  if (warp == 1) {
    tc_fence_after_sync();
    tmem_dealloc(tmem, kTileTmemCols);
  }
  if (*s_abort && tid == 0) atomicExch(p.status, kStatusTimeout);
}

// Joins the key chunks of a row in key order.  A row is a (token, query head); a warp takes eight in a row, so that the
// look-up of their sequence is paid once (a warp per row spent its time on that: 44 us instead of 26 for 49K rows of three
// chunks), and the chunks of a row are loaded four at a time.
constexpr int kJoinRows = 8;
template <typename T, int D>
__global__ void __launch_bounds__(256) paged_tiles_merge_kernel(const __grid_constant__ PagedProblem p) {
  constexpr int V = D / 32;                  // dims of a lane
  pdl_wait();
  pdl_launch_next();
  const int lane = threadIdx.x & 31;
  int idx = (blockIdx.x * 8 + (threadIdx.x >> 5)) * kJoinRows;
  const int end = idx + kJoinRows < p.total_q * p.hq ? idx + kJoinRows : p.total_q * p.hq;
  if (idx >= end) return;
  int tok = idx / p.hq, head = idx % p.hq, kv_head = head / p.group, g = head % p.group, tok_end = 0, tok_0 = 0;
  const int pair = 2 * tile_rows(p.group);
  TileSeq sq{0, 0, 1, 0};
  size_t before = 0;
  for (; idx < end; ++idx) {
    if (tok >= tok_end) {                    // another sequence
      const int b = paged_seq_of(p, tok);
      sq = tile_seq_of(p, b);
      tok_0 = (int)__ldg(p.cu_q + b);
      tok_end = (int)__ldg(p.cu_q + b + 1);
      int n = 0;
      for (int s = 0; s < b; s += 32) {
        const TileSeq o = tile_seq_of(p, s + lane);
        n += __reduce_add_sync(0xffffffffu, s + lane < b ? o.row_tiles * o.chunks * p.hkv : 0);
      }
      before = n;
    }
    if (sq.rows > 0 && sq.chunks > 1) {
      const int row = (tok - tok_0) * p.group + g, i = row / pair;
      const size_t first = (before + (size_t)kv_head * sq.chunks * sq.row_tiles + (sq.row_tiles - 1 - i)) * kTileRows + (row - i * pair);
      const size_t step = (size_t)sq.row_tiles * kTileRows;
      float M = -INFINITY, L = 0.f, a[V];
#pragma unroll
      for (int e = 0; e < V; ++e) a[e] = 0.f;
      for (int c = 0; c < sq.chunks; c += 4) {
        float2 st[4];
        float v[4][V];
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          st[x] = make_float2(-INFINITY, 0.f);
          if (c + x < sq.chunks) {
            st[x] = __ldcg(reinterpret_cast<const float2*>(p.tile_stat) + first + (c + x) * step);
            const float* src = p.tile_part + (first + (c + x) * step) * D + lane * V;
            if (V == 4) {
              const float4 w = __ldcg(reinterpret_cast<const float4*>(src));
              v[x][0] = w.x; v[x][1] = w.y; v[x][V - 2] = w.z; v[x][V - 1] = w.w;
            } else {
              const float2 w = __ldcg(reinterpret_cast<const float2*>(src));
              v[x][0] = w.x; v[x][1] = w.y;
            }
          }
        }
        const float m = fmaxf(fmaxf(fmaxf(st[0].x, st[1].x), fmaxf(st[2].x, st[3].x)), M);
        const float keep = M == -INFINITY ? 0.f : ex2_approx(M - m);
        L *= keep;
#pragma unroll
        for (int e = 0; e < V; ++e) a[e] *= keep;
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          if (st[x].y == 0.f) continue;                   // (nothing seen: its partial output was not written)
          const float f = ex2_approx(st[x].x - m);
          L += st[x].y * f;
#pragma unroll
          for (int e = 0; e < V; ++e) a[e] = fmaf(v[x][e], f, a[e]);
        }
        M = m;
      }
      const float inv = L != 0.f ? 1.f / L : 0.f;
      uint32_t* y = static_cast<uint32_t*>(p.y) + (size_t)idx * (D / 2) + lane * (V / 2);
      y[0] = T::pack(a[0] * inv, a[1] * inv);
      if (V == 4) y[1] = T::pack(a[V - 2] * inv, a[V - 1] * inv);
      if (lane == 0 && p.lse) p.lse[idx] = L != 0.f ? (M + log2f(L)) * 0.6931471805599453f : -INFINITY;
    }
    if (++g == p.group) { g = 0; ++kv_head; }
    if (++head == p.hq) { head = 0; kv_head = 0; g = 0; ++tok; }
  }
}

template <typename T, int D>
static cudaError_t launch_tiles_t(const PagedProblem& p, const CUtensorMap& tk, const CUtensorMap& tv, const CUtensorMap& tq, int grid,
                                  cudaStream_t st) {
  static PerDeviceFlag configured;
  const cudaError_t e = set_max_dynamic_smem(configured, reinterpret_cast<const void*>(paged_tiles_kernel<T, D>), TileCfg<D>::total);
  if (e != cudaSuccess) return e;
  return launch_pdl(paged_tiles_kernel<T, D>, dim3(grid), dim3(kTileThreads), TileCfg<D>::total, st, tk, tv, tq, p);
}

cudaError_t launch_paged_tiles(const PagedProblem& p, const CUtensorMap& tk, const CUtensorMap& tv, const CUtensorMap& tq, int d,
                               bool bf16, int grid, cudaStream_t st) {
  if (d == 64) return bf16 ? launch_tiles_t<Bf16, 64>(p, tk, tv, tq, grid, st) : launch_tiles_t<Fp16, 64>(p, tk, tv, tq, grid, st);
  return bf16 ? launch_tiles_t<Bf16, 128>(p, tk, tv, tq, grid, st) : launch_tiles_t<Fp16, 128>(p, tk, tv, tq, grid, st);
}

cudaError_t launch_paged_tiles_merge(const PagedProblem& p, int d, bool bf16, cudaStream_t st) {
  const dim3 grid((p.total_q * p.hq + 8 * kJoinRows - 1) / (8 * kJoinRows)), block(256);
  if (d == 64)
    return bf16 ? launch_pdl(paged_tiles_merge_kernel<Bf16, 64>, grid, block, 0, st, p)
                : launch_pdl(paged_tiles_merge_kernel<Fp16, 64>, grid, block, 0, st, p);
  return bf16 ? launch_pdl(paged_tiles_merge_kernel<Bf16, 128>, grid, block, 0, st, p)
              : launch_pdl(paged_tiles_merge_kernel<Fp16, 128>, grid, block, 0, st, p);
}

}  // namespace tkphi
