// Decoding-stage attention over a KV cache in 4 bits (the format of
// apb_cache4.hip), for gfx950.
//
// Rows are (query head, new token) pairs; the rows of one GQA group share a KV head.
// The work is a read of the cache: a CU's share of the HBM rate is a 32-key
// block of K and V (4352 bytes at d = 128) in about 450 cycles, which leaves each
// SIMD 450 vector instructions of a wave a block to turn codes into operands and
// to form the softmax.  So:
//  * A wave owns 16 * RB rows and walks 32-key blocks of its own; the waves of a
//    workgroup take a split's blocks in turn and meet in LDS at its end, so that a
//    split is one partial.  The next block's loads are in flight while one is computed.
//  * S^T = K Q^T on v_mfma_f32_16x16x32_bf16 (keys on M, rows on N).  A product over
//    the head size may take it in any order that both operands share, so a lane takes
//    the d / 4 elements of its key that lie together (16 or 8 bytes of codes and one
//    scale) and K goes from memory to the operand registers without LDS;
//    v_cvt_scalef32_pk_bf16_fp4 makes two elements at a time.  A code times its scale
//    is exact in bf16.
//  * O^T = V^T P^T needs 8 keys of one element in a lane: V is made bf16 the same
//    way, its scales applied, goes to LDS row by row and comes back through
//    transposing reads (ds_read_b64_tr_b16).  The wave has the tile to itself, so
//    there is no barrier in the loop.  Rows are swizzled so that reads and writes
//    touch every bank once.
//  * The probabilities are three bf16 each, the top, middle and lowest 8 bits of
//    their fp32 significand: three products in place of one, no rounding at all.
//    (Two would leave 2^-17, and o 2.3e-6 off; the matrix cores have the time.)
//  * Online softmax in base 2 in fp32 with a lazily moved maximum, as in the decode
//    kernels over bf16: the maximum and O's rescale only when a lane's sum of a block
//    passes 2^13.
#include <math.h>

#include <type_traits>

#include "apb_internal.h"
#include "apb_plan.h"

namespace apb {
namespace {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short i16x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
typedef __attribute__((address_space(3))) i16x4 lds_i16x4;
typedef __attribute__((address_space(3))) u32x4 lds_u32x4;

constexpr float kSumLimit = 8192.f;  // largest lane sum of a block against a stale maximum

struct Dec4Params {
  const uint16_t* q;
  const uint8_t* k_codes;
  const uint8_t* k_scales;
  const uint8_t* v_codes;
  const uint8_t* v_scales;
  float* part_o;    // [n_split][rows_total][d]: not yet divided by l
  float* part_m;    // [n_split][rows_total]: maximum, base 2
  float* part_l;    // [n_split][rows_total]: sum against it
  float* o;         // one split: the result
  float* lse;
  int capacity, Lc, n_new, causal, n_kv, R, rows_total, n_split, n_rb, blocks_per_split;
  float scale_log2;
};

// The codes and scale bytes that a lane takes of a 32-key block.
template <int D>
struct Block4 {
  static constexpr int KW = D / 32;  // words of codes of one key in a lane: 8 elements each
  static constexpr int VL = D / 64;  // 32-element groups of V in a lane
  unsigned kw[2][KW], kb[2];
  u32x4 vw[VL];
  unsigned vb[VL];
};

// 8 elements of codes in a word, as a bf16 operand.
__device__ __forceinline__ u32x4 elements(unsigned w, float scale) {
  u32x4 x;
  x[0] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 0));
  x[1] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 1));
  x[2] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 2));
  x[3] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 3));
  return x;
}

__device__ __forceinline__ bf16x8 as_bf16(u32x4 x) { return __builtin_bit_cast(bf16x8, x); }

// Chunk (16 bytes) c of row r of a V tile sits at chunk c ^ v_swz(r): a transposing
// read serves 8 rows x 32 bytes a clock, which fall on all 64 banks, and 16 lanes'
// writes do (see v_flip).
template <int D>
__device__ __forceinline__ int v_swz(int r) { return D == 128 ? 2 * (r & 7) : 2 * ((r >> 1) & 3); }
// A lane writes its four chunks in the order j ^ v_flip(r).
template <int D>
__device__ __forceinline__ int v_flip(int r) { return D == 128 ? (r >> 1) & 1 : (r >> 2) & 1; }

// K, for reads of a chunk of 16 rows at once.
template <int D>
__device__ __forceinline__ int k_swz(int r) { return D == 128 ? r & 15 : (r >> 1) & 7; }

// A lane's first transposing read of a V tile: rows 4 lg .. 4 lg + 3 of dims 0 .. 15
// between the 16 lanes of a group (dim block db is 32 db away by exclusive or, rows 16 on
// 16 rows); the lane then has element li of its group's four rows.
template <int D>
__device__ __forceinline__ uint32_t v_lane(int li, int lg) {
  const int row = 4 * lg + (li >> 2);
  return (uint32_t)(row * 2 * D + 16 * (((li & 3) >> 1) ^ v_swz<D>(row)) + 8 * (li & 1));
}

// The V operand of dim block db: 32 keys, the lane's eight those of its P operand.
template <int D>
__device__ __forceinline__ bf16x8 v_operand(uint32_t v_get, int db) {
  i16x4 part[2];
#pragma unroll
  for (int rd = 0; rd < 2; ++rd)
    part[rd] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
        (lds_i16x4*)(uintptr_t)((v_get ^ (32u * db)) + (uint32_t)(16 * rd * 2 * D)));
  return __builtin_bit_cast(bf16x8,
                            __builtin_shufflevector(part[0], part[1], 0, 1, 2, 3, 4, 5, 6, 7));
}

// A group's 32 elements into its row's four chunks.  A group of NaN goes there as zeros
// where it is V's: in a product a zero probability would not keep it out.
__device__ __forceinline__ void put_group(uint32_t at, u32x4 codes, unsigned b, bool flip, bool v) {
  const bool bad = v && b == 255;
  const float scale = __uint_as_float(bad ? 0u : b << 23);
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const unsigned there = codes[j ^ 1], here = codes[j];
    *(lds_u32x4*)(uintptr_t)(at ^ (16u * j)) = elements(bad ? 0u : flip ? there : here, scale);
  }
}

__device__ __forceinline__ float across_groups_max(float x) {
  x = fmaxf(x, __shfl_xor(x, 16));
  return fmaxf(x, __shfl_xor(x, 32));
}

// Where workgroup `id` works.  Its XCD is id % 8: the row blocks of one split of one KV
// head, which read the same keys, go to one XCD and so to one L2.
struct Place4 {
  int split, row_block, kvh;
};

__device__ __forceinline__ Place4 place4(int n_split, int n_rb, int n_kv) {
  const unsigned id = blockIdx.x, pairs = (unsigned)n_split * n_kv, full = pairs / 8 * 8 * n_rb;
  unsigned rb, u;
  if (id < full) {
    rb = id % (8 * n_rb) / 8;
    u = id / (8 * n_rb) * 8 + id % 8;
  } else {
    const unsigned rest = pairs % 8;
    rb = (id - full) / rest;
    u = pairs / 8 * 8 + (id - full) % rest;
  }
  return Place4{(int)(u % n_split), (int)rb, (int)(u / n_split)};
}

// A wave's state: 16 * RB rows, row li of each block in the four lanes li + 16 lg.
template <int D, int RB>
struct Rows4 {
  static constexpr int NDB = D / 16, KW = D / 32;
  int vis[RB];            // keys that the lane's rows see
  bf16x8 q[RB][KW];
  f32x4 oacc[RB][NDB];    // element r of dim block db: O^T[16 db + 4 lg + r][row li]
  float m_run[RB], l_run[RB];

  // Rows from row0 on of KV head kvh; q's dims of product j from dim(j) on.
  template <typename Dim>
  __device__ __forceinline__ void start(const Dec4Params& p, int kvh, int row0, Dim dim) {
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
      const int rho = row0 + 16 * rb + (threadIdx.x & 15);
      const bool ok = rho < p.R;
      vis[rb] = p.causal ? p.Lc - p.n_new + (ok ? rho % p.n_new : 0) + 1 : p.Lc;
      const uint16_t* row = p.q + ((size_t)kvh * p.R + (ok ? rho : 0)) * D;
#pragma unroll
      for (int j = 0; j < KW; ++j)
        q[rb][j] = as_bf16(*reinterpret_cast<const u32x4*>(row + dim(j)) & (ok ? ~0u : 0u));
      m_run[rb] = -INFINITY;
      l_run[rb] = 0.f;
#pragma unroll
      for (int db = 0; db < NDB; ++db) oacc[rb][db] = f32x4{};
    }
  }

  // Keys that the rows do not see, of the 32 from c0 on.
  __device__ __forceinline__ void mask(f32x4 (&s)[2][RB], int c0, int lg) const {
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int rb = 0; rb < RB; ++rb)
#pragma unroll
        for (int r = 0; r < 4; ++r)
          if (c0 + 16 * i + 4 * lg + r >= vis[rb]) s[i][rb][r] = -INFINITY;
  }

  // Logits of SUB 32-key blocks (element r of tile i: key 16 i + 4 lg + r) to
  // probabilities, in their three parts as the P operand, and the running maximum and sum.
  // All of them against one maximum: O is rescaled when that rises, and their values are
  // not in it yet.
  template <int SUB>
  __device__ __forceinline__ void softmax(const f32x4 (&s)[SUB][2][RB], float scale,
                                          u32x4 (&pr)[SUB][RB][3]) {
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
      constexpr int N = 8 * SUB;
      auto logit = [&](int i) __attribute__((always_inline)) { return s[i >> 3][(i >> 2) & 1][rb][i & 3]; };
      float e[N], sum;
      auto exps = [&]() __attribute__((always_inline)) {
        sum = 0.f;
#pragma unroll
        for (int i = 0; i < N; ++i)
          e[i] = __builtin_amdgcn_exp2f(fmaf(logit(i), scale, -m_run[rb]));
#pragma unroll
        for (int i = 0; i < N; i += 8)
          sum += ((e[i] + e[i + 1]) + (e[i + 2] + e[i + 3])) + ((e[i + 4] + e[i + 5]) + (e[i + 6] + e[i + 7]));
      };
      exps();
      if (__any(!(sum <= kSumLimit))) {
        float mx = logit(0);
#pragma unroll
        for (int i = 1; i < N; ++i) mx = fmaxf(mx, logit(i));
        const float m_new = fmaxf(m_run[rb], across_groups_max(mx) * scale);
        if (m_new == -INFINITY) {
          // nothing but keys that the row does not see, and NaN, which stays
          sum = 0.f;
#pragma unroll
          for (int i = 0; i < N; ++i) {
            const float y = logit(i);
            e[i] = y == -INFINITY ? 0.f : y;
            sum += e[i];
          }
        } else {
          const float alpha = __builtin_amdgcn_exp2f(m_run[rb] - m_new);  // from -inf: 0
          m_run[rb] = m_new;
          l_run[rb] *= alpha;
#pragma unroll
          for (int db = 0; db < NDB; ++db) oacc[rb][db] *= alpha;
          exps();
        }
      }
      l_run[rb] += sum;
#pragma unroll
      for (int i = 0; i < N / 2; ++i) {
        unsigned hi[2], mid[2], lo[2];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          hi[t] = __float_as_uint(e[2 * i + t]);
          const float r1 = e[2 * i + t] - __uint_as_float(hi[t] & 0xFFFF0000u);
          mid[t] = __float_as_uint(r1);
          lo[t] = __float_as_uint(r1 - __uint_as_float(mid[t] & 0xFFFF0000u));
        }
        u32x4(&out)[3] = pr[i >> 2][rb];
        out[0][i & 3] = __builtin_amdgcn_perm(hi[1], hi[0], 0x07060302u);
        out[1][i & 3] = __builtin_amdgcn_perm(mid[1], mid[0], 0x07060302u);
        out[2][i & 3] = __builtin_amdgcn_perm(lo[1], lo[0], 0x07060302u);
      }
    }
  }

  // O^T += V^T P^T of one dim block, v its V operand: product t of 3 * RB.
  __device__ __forceinline__ void value_product(const bf16x8& v, const u32x4 (&pr)[RB][3], int db, int t) {
    f32x4& o = oacc[t % RB][db];
    o = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, as_bf16(pr[t % RB][t / RB]), o, 0, 0, 0);
  }

  // Values of group g (dims 32 g ..) of key c are NaN: so is O of the rows that see it.
  __device__ __forceinline__ void not_a_number(int g, int c) {
#pragma unroll
    for (int rb = 0; rb < RB; ++rb)
#pragma unroll
      for (int db = 0; db < NDB; ++db)
        if (db / 2 == g && c < vis[rb]) oacc[rb][db] = f32x4{} + NAN;
  }

  // The parts of WK waves over the same rows (this one the wk-th) meet in LDS: at o_lds, 1
  // KiB for each row block, dim block and wave, and ml_lds.  Then the waves take the
  // rows in turn, whole ones: a store is 1 KiB that lies together.  Chunk 4 db + lg of row li
  // sits at chunk li ^ (that & 15) of its KiB's quarter lg, on a bank of its own in both
  // directions.
  template <int WK, bool WHOLE>
  __device__ __forceinline__ void finish(const Dec4Params& p, const Place4& at, int row0, int wk,
                                         uint8_t* o_lds, float (*ml_lds)[WK][RB][16]) {
    constexpr int OUT = RB * NDB * 1024;          // bytes of a wave's O
    constexpr int CH = D / 4, RPI = 64 / CH;      // chunks of a row, rows of a store
    constexpr int ROWS = 16 * RB, TURNS = (ROWS + RPI * WK - 1) / (RPI * WK);
    const int lane = threadIdx.x & 63, li = lane & 15, lg = lane >> 4;
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {  // sums over the four lanes of a row
      l_run[rb] += __shfl_xor(l_run[rb], 16);
      l_run[rb] += __shfl_xor(l_run[rb], 32);
    }
    __syncthreads();  // the tiles are done with
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
#pragma unroll
      for (int db = 0; db < NDB; ++db)
        *reinterpret_cast<f32x4*>(o_lds + wk * OUT + 1024 * (rb * NDB + db) + 256 * lg +
                                  16 * (li ^ ((4 * db + lg) & 15))) = oacc[rb][db];
      if (lg == 0) {
        ml_lds[0][wk][rb][li] = m_run[rb];
        ml_lds[1][wk][rb][li] = l_run[rb];
      }
    }
    __syncthreads();
    const int c = lane % CH;
#pragma unroll
    for (int it = 0; it < TURNS; ++it) {
      const int r = (it * WK + wk) * RPI + lane / CH, rb = r / 16, ri = r % 16;
      if (r >= ROWS || row0 + r >= p.R) continue;
      float m = -INFINITY, l = 0.f;
#pragma unroll
      for (int k = 0; k < WK; ++k) m = fmaxf(m, ml_lds[0][k][rb][ri]);
      f32x4 y = {};
#pragma unroll
      for (int k = 0; k < WK; ++k) {
        const float lk = ml_lds[1][k][rb][ri];  // (0: no key; NaN stays)
        const float w = lk == 0.f ? 0.f : __builtin_amdgcn_exp2f(ml_lds[0][k][rb][ri] - m);
        l = fmaf(w, lk, l);
        y += w * *reinterpret_cast<const f32x4*>(o_lds + k * OUT + 1024 * (rb * NDB + c / 4) +
                                                 256 * (c & 3) + 16 * (ri ^ (c & 15)));
      }
      const size_t row = (size_t)at.kvh * p.R + row0 + r;
      if constexpr (WHOLE) {
        *reinterpret_cast<f32x4*>(p.o + row * D + 4 * c) = y * (l == 0.f ? 0.f : 1.f / l);
        if (c == 0)
          p.lse[row] = l == 0.f ? -INFINITY : 0.69314718055994531f * (m + log2f(l));
      } else {
        const size_t part = (size_t)at.split * p.rows_total + row;
        *reinterpret_cast<f32x4*>(p.part_o + part * D + 4 * c) = y;
        if (c == 0) {
          p.part_m[part] = m;
          p.part_l[part] = l;
        }
      }
    }
  }
};

// Up to 32 rows of a KV head: WK waves, each with 32-key blocks of its own.
template <int D, int RB, int WK, bool WHOLE>
__global__ void __launch_bounds__(64 * WK, 2) decode4_kernel(Dec4Params p) {
  using Rows = Rows4<D, RB>;
  constexpr int KW = Block4<D>::KW, VL = Block4<D>::VL;
  constexpr int TILE = 32 * D * 2, OUT = RB * D * 64;  // bytes of a V tile, of a wave's O
  __shared__ __attribute__((aligned(256))) uint8_t lds[WK * (OUT > TILE ? OUT : TILE)];
  __shared__ float ml_lds[2][WK][RB][16];

  const int lane = threadIdx.x & 63, li = lane & 15, lg = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const Place4 at = place4(p.n_split, p.n_rb, p.n_kv);
  const int nblk = (p.Lc + 31) / 32;
  const int b0 = at.split * p.blocks_per_split, b1 = min(b0 + p.blocks_per_split, nblk);
  const int vis_all = p.causal ? p.Lc - p.n_new + 1 : p.Lc;  // keys that every row sees

  // V: lane -> (key, group) of each 16-byte load, and its place in the tile.
  constexpr int G = D / 32;
  const uint32_t tile = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t*)lds +
                        (uint32_t)(wave * TILE);
  uint32_t v_put[VL];
#pragma unroll
  for (int v = 0; v < VL; ++v) {
    const int key = (64 * v + lane) / G, g = lane % G;
    v_put[v] = tile + (uint32_t)(key * 2 * D + 16 * ((4 * g) ^ v_swz<D>(key) ^ v_flip<D>(key)));
  }
  const bool flip = v_flip<D>(lane / G) != 0;  // (the same for every v: 64 / G keys apart)
  const uint32_t v_get = tile + v_lane<D>(li, lg);

  auto load = [&](int b) __attribute__((always_inline)) {
    Block4<D> x;
    const int c0 = min(32 * b, p.Lc - 1), last = p.Lc - 1 - c0;  // rows past the last key repeat it
    const size_t r0 = (size_t)at.kvh * p.capacity + c0;
    const uint8_t* kc = p.k_codes + r0 * (D / 2);
    const uint8_t* ks = p.k_scales + r0 * G;
    const uint8_t* vc = p.v_codes + r0 * (D / 2);
    const uint8_t* vs = p.v_scales + r0 * G;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const uint32_t key = (uint32_t)min(16 * i + li, last);
      if constexpr (D == 128) {
        const u32x4 w = *reinterpret_cast<const u32x4*>(kc + (key * (D / 2) + 16u * lg));
        x.kw[i][0] = w[0]; x.kw[i][1] = w[1]; x.kw[i][2] = w[2]; x.kw[i][3] = w[3];
        x.kb[i] = ks[key * G + lg];
      } else {
        const u32x2 w = *reinterpret_cast<const u32x2*>(kc + (key * (D / 2) + 8u * lg));
        x.kw[i][0] = w[0]; x.kw[i][1] = w[1];
        x.kb[i] = ks[key * G + lg / 2];
      }
    }
#pragma unroll
    for (int v = 0; v < VL; ++v) {
      const uint32_t key = (uint32_t)min((64 * v + lane) / G, last), g = lane % G;
      x.vw[v] = *reinterpret_cast<const u32x4*>(vc + (key * (D / 2) + 16u * g));
      x.vb[v] = vs[key * G + g];
    }
    return x;
  };

  Rows rows;
  const int row0 = 16 * RB * at.row_block;
  // (a lane's d / 4 elements of its key lie together)
  rows.start(p, at.kvh, row0, [&](int j) { return lg * (D / 4) + 8 * j; });

  // Block b from x, which takes the wave's next block as soon as it is done with, whatever
  // b1 (past the last key the loads repeat it).  A second block in flight per wave gained
  // nothing (16385 keys of 8 heads 11.4 against 12.3 us, 524289 110.8 against 112.2): eight
  // waves of a CU have 35 KiB under way.
  auto block = [&](Block4<D>& x, int b) __attribute__((always_inline)) {
    const int c0 = 32 * b;
    f32x4 s[1][2][RB];  // S^T: element r of tile i is key c0 + 16 i + 4 lg + r
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const float scale = __uint_as_float(x.kb[i] << 23);  // b = 255: NaN elements
#pragma unroll
      for (int j = 0; j < KW; ++j) {
        const bf16x8 k = as_bf16(elements(x.kw[i][j], scale));
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) {
          const f32x4 zero = {};
          s[0][i][rb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k, rows.q[rb][j],
                                                                j == 0 ? zero : s[0][i][rb], 0, 0, 0);
        }
      }
    }

    // V -> LDS; a group of NaN goes into O by hand, for the rows that see it: the first
    // key of each.
    int first[G];
    bool bad = false;
#pragma unroll
    for (int v = 0; v < VL; ++v) {
      put_group(v_put[v], x.vw[v], x.vb[v], flip, true);
      bad |= x.vb[v] == 255;
    }
    const bool any_bad = __any(bad);
    if (any_bad) {
#pragma unroll
      for (int g = 0; g < G; ++g) {
        first[g] = 32;
#pragma unroll
        for (int v = 0; v < VL; ++v) {
          const unsigned long long hit = __ballot(x.vb[v] == 255 && (int)(lane % G) == g);
          if (hit) first[g] = min(first[g], (64 * v + (int)__builtin_ctzll(hit)) / G);
        }
      }
    }
    x = load(b + WK);
    // (a wave's LDS accesses are in order; the reads land during the softmax)
    bf16x8 v[Rows::NDB];
#pragma unroll
    for (int db = 0; db < Rows::NDB; ++db) v[db] = v_operand<D>(v_get, db);
    __builtin_amdgcn_sched_barrier(0);

    if (c0 + 32 > vis_all) rows.mask(s[0], c0, lg);
    u32x4 pr[1][RB][3];
    rows.softmax(s, p.scale_log2, pr);
#pragma unroll
    for (int db = 0; db < Rows::NDB; ++db)
#pragma unroll
      for (int t = 0; t < 3 * RB; ++t) rows.value_product(v[db], pr[0], db, t);
    if (any_bad) {
#pragma unroll
      for (int g = 0; g < G; ++g)
        if (first[g] < 32) rows.not_a_number(g, c0 + first[g]);
    }
  };
  if (b0 + wave < b1) {
    Block4<D> x = load(b0 + wave);
    for (int b = b0 + wave; b < b1; b += WK) block(x, b);
  }
  rows.template finish<WK, WHOLE>(p, at, row0, wave, lds, ml_lds);
}

// More rows: eight waves, WR of them with 32 rows each and WK = 8 / WR such sets, which
// share a split's keys.  A step is 128 keys: all threads make its codes bf16 and put K
// and V into LDS, where each set reads 128 / WK of them, so that the work of a conversion
// is shared by 32 * WR rows.
// Products and vector work are about even here (a 32-key block of 32 rows: 64 products of
// 16 cycles; 200 vector instructions of 4 and 16 exponentials of 16), and eight waves in
// step would wait for each other's turns at both.  So the waves form two groups, one wave
// of each on every SIMD, and a barrier ends every phase:
//   phase    group A                       group B
//   2 t      S(t) = Q K(t), O += P V(t-1)  softmax(t-1); K(t+1), V(t) -> LDS
//   2 t + 1  softmax(t); K(t+1), V(t)      S(t), O += P V(t-1)
//            -> LDS
// K(t) and V(t-1) are read in both phases while K(t+1) and V(t) are written: two buffers
// of each.  The codes of the writes after those are in flight meanwhile.
template <int D, int WR, bool WHOLE>
__global__ void __launch_bounds__(512, 2) decode4_shared_kernel(Dec4Params p) {
  constexpr int RB = 2, WK = 8 / WR, SUB = 4 / WK;  // 32-key blocks of a step and set
  using Rows = Rows4<D, RB>;
  constexpr int KW = D / 32, G = D / 32, TILE = 32 * D * 2;
  __shared__ __attribute__((aligned(256))) uint8_t lds[2][2][4][TILE];  // K or V, buffer, block
  __shared__ float ml_lds[WR][2][WK][RB][16];
  // First key (of 32) whose values of a group are NaN, and whether there is one, by step % 3:
  // cleared in the step before it is set, read in the one after.
  __shared__ int nan_lds[3][4][4], any_lds[3];

  const int tid = threadIdx.x, lane = tid & 63, li = lane & 15, lg = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), wr = wave / WK, wk = wave % WK;
  const bool group_b = wave >= 4;
  const Place4 at = place4(p.n_split, p.n_rb, p.n_kv);
  const int nblk = (p.Lc + 31) / 32;
  const int b0 = at.split * p.blocks_per_split, b1 = min(b0 + p.blocks_per_split, nblk);
  const int steps = (b1 - b0 + 3) / 4;
  const int vis_all = min(p.causal ? p.Lc - p.n_new + 1 : p.Lc, 32 * b1);

  // This thread's groups of a step: (key, g) of K and of V (d = 128), or of one of them by
  // wave (d = 64).  Every load and write is made, whatever the step: past the split's end
  // they repeat its last key and go where nothing is read any more.  (Where some are
  // left out, the compiler waits for all that are in flight before the first is used.)
  constexpr int NU = D / 64;
  const int unit = D == 128 ? tid : (tid & 63) + (tid >> 7) * 64, key = unit / G, g = unit % G;
  const uint32_t base = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t*)lds;
  constexpr uint32_t BUF = 4 * TILE, V = 2 * BUF;
  bool is_v[NU], flip[NU];
  uint32_t put_at[NU];
#pragma unroll
  for (int u = 0; u < NU; ++u) {
    is_v[u] = D == 128 ? u == 1 : (wave & 1) != 0;
    flip[u] = is_v[u] && v_flip<D>(key) != 0;
    const int swz = is_v[u] ? v_swz<D>(key) ^ v_flip<D>(key) : k_swz<D>(key);
    put_at[u] = base + (is_v[u] ? V : 0) + (uint32_t)(key * 2 * D) + 16u * ((4 * g) ^ swz);
  }

  struct Unit {
    u32x4 w;
    unsigned b;
  };
  // The codes of K(step) and V(step - 1), and their way into LDS.
  auto load = [&](int step, Unit (&x)[NU]) __attribute__((always_inline)) {
#pragma unroll
    for (int u = 0; u < NU; ++u) {
      const int c0 = min(32 * (b0 + 4 * max(step - (is_v[u] ? 1 : 0), 0)), p.Lc - 1);
      const uint32_t k = (uint32_t)min(key, p.Lc - 1 - c0);
      const size_t r0 = (size_t)at.kvh * p.capacity + c0;
      const uint8_t* codes = (is_v[u] ? p.v_codes : p.k_codes) + r0 * (D / 2);
      const uint8_t* scales = (is_v[u] ? p.v_scales : p.k_scales) + r0 * G;
      x[u].w = *reinterpret_cast<const u32x4*>(codes + (k * (D / 2) + 16u * g));
      x[u].b = scales[k * G + g];
    }
  };
  auto put = [&](int step, const Unit (&x)[NU]) __attribute__((always_inline)) {
#pragma unroll
    for (int u = 0; u < NU; ++u) {
      const int of = step - (is_v[u] ? 1 : 0);
      put_group(put_at[u] + (of & 1 ? BUF : 0), x[u].w, x[u].b, flip[u], is_v[u]);
      if (is_v[u] && x[u].b == 255 && of < steps) {
        atomicMin(&nan_lds[of % 3][key / 32][g], key % 32);
        any_lds[of % 3] = 1;
      }
    }
  };
  auto put_keys = [&](const Unit (&x)[NU]) __attribute__((always_inline)) {  // K(0)
#pragma unroll
    for (int u = 0; u < NU; ++u)
      if (!is_v[u]) put_group(put_at[u], x[u].w, x[u].b, false, false);
  };
  auto clear = [&](int step) __attribute__((always_inline)) {  // by group B
    if (tid >= 256 && tid < 272) nan_lds[step % 3][(tid & 15) / 4][tid & 3] = 32;
    if (tid == 272) any_lds[step % 3] = 0;
  };

  Rows rows;
  const int row0 = 32 * (WR * at.row_block + wr);
  Unit codes[NU], first[NU];
  if (steps > 0) {
    load(0, first);
    load(1, codes);
  }
  rows.start(p, at.kvh, row0, [&](int j) { return 32 * j + 8 * lg; });
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) rows.vis[rb] = min(rows.vis[rb], 32 * b1);
  const uint32_t k_get = base + (uint32_t)(li * 2 * D) + 16u * (lg ^ k_swz<D>(li)) + wk * SUB * TILE;
  const uint32_t v_get = base + V + v_lane<D>(li, lg) + wk * SUB * TILE;

  clear(0);
  if (steps > 0) put_keys(first);
  __syncthreads();
  if (group_b && steps > 0) {
    put(1, codes);
    load(2, codes);
    clear(1);
  }
  f32x4 s[SUB][2][RB];
  u32x4 pr[SUB][RB][3];
  // A phase of products, in turns of two dim blocks of O (twelve, on four accumulators) and
  // two operands of S (four): a turn's operands are read while the one before it goes on.
  auto products = [&](int step, auto with_s, auto with_o) __attribute__((always_inline)) {
    constexpr bool S = decltype(with_s)::value, O = decltype(with_o)::value;
    constexpr int N = Rows::NDB * SUB / 2;
    static_assert(Rows::NDB == 2 * KW, "as many dim blocks as operands of K");
    const uint32_t kt = k_get + (step & 1 ? BUF : 0), vt = v_get + (step & 1 ? 0 : BUF);
    bf16x8 k[2][2], v[2][2];
    auto read = [&](int n) __attribute__((always_inline)) {
      const int t = 2 * n / Rows::NDB, m = 2 * n % Rows::NDB;
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        if constexpr (O) v[n & 1][i] = v_operand<D>(vt + t * TILE, m + i);
        if constexpr (S)
          k[n & 1][i] = as_bf16(*(lds_u32x4*)(uintptr_t)((kt ^ (64u * (m / 2))) +
                                                        (uint32_t)(t * TILE + 16 * i * 2 * D)));
      }
    };
    read(0);
#pragma unroll
    for (int n = 0; n < N; ++n) {
      const int t = 2 * n / Rows::NDB, m = 2 * n % Rows::NDB, j = m / 2;
      if (n + 1 < N) read(n + 1);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int u = 0; u < 3; ++u) {
        if constexpr (O) {
#pragma unroll
          for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int rb = 0; rb < RB; ++rb) rows.value_product(v[n & 1][i], pr[t], m + i, RB * u + rb);
        }
        if constexpr (S) {
          if (u < 2) {
#pragma unroll
            for (int rb = 0; rb < RB; ++rb) {
              const f32x4 zero = {};
              s[t][u][rb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                  k[n & 1][u], rows.q[rb][j], j == 0 ? zero : s[t][u][rb], 0, 0, 0);
            }
          }
        }
      }
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  auto not_numbers = [&](int step, int any) __attribute__((always_inline)) {
    if (any == 0) return;
    for (int t = 0; t < SUB; ++t)
      for (int n = 0; n < G; ++n) {
        const int blk = wk * SUB + t, first = nan_lds[step % 3][blk][n];
        if (first < 32) rows.not_a_number(n, 32 * (b0 + 4 * step + blk) + first);
      }
  };
  auto turn = [&](int step, auto more) __attribute__((always_inline)) {
#pragma unroll
    for (int t = 0; t < SUB; ++t) {
      const int c0 = 32 * (b0 + 4 * step + wk * SUB + t);
      if (c0 + 32 > vis_all) rows.mask(s[t], c0, lg);
    }
    rows.softmax(s, p.scale_log2, pr);
    put(step + (group_b ? 2 : 1), codes);
    load(step + (group_b ? 3 : 2), codes);
    if (group_b) clear(step + 2);
    if (!group_b) __syncthreads();
    const int any = any_lds[step % 3];
    __builtin_amdgcn_s_setprio(1);
    products(step + 1, more, std::true_type{});
    __builtin_amdgcn_s_setprio(0);
    not_numbers(step, any);
    if (decltype(more)::value && group_b) __syncthreads();
  };
  if (steps > 0) {
    products(0, std::true_type{}, std::false_type{});
    if (group_b) __syncthreads();
    for (int step = 0; step + 1 < steps; ++step) turn(step, std::true_type{});
    turn(steps - 1, std::false_type{});
  }
  rows.template finish<WK, WHOLE>(p, at, row0, wk, &lds[0][0][0][0] + wr * WK * RB * D * 64, ml_lds[wr]);
}

// The splits of a row: O = sum_s 2^(m_s - m) O_s / l, l = sum_s 2^(m_s - m) l_s, with m
// the largest m_s; lse = ln 2 (m + log2 l).  Parts keep O undivided, and m apart from
// log l: a sum of the two would lose l's digits beside a large m.  16 bytes of O a
// thread; its G thread groups take every G-th split, eight at a time against their own
// maximum, so that all a thread reads is one trip to memory, and meet in LDS.  (Two
// groups and four rows a workgroup: no faster at 2048 rows and 16 splits.)
constexpr int kMergeThreads = 256;

template <int D>
__global__ void __launch_bounds__(kMergeThreads) decode4_merge_kernel(
    int n_split, int rows, const float* __restrict__ part_o, const float* __restrict__ part_m,
    const float* __restrict__ part_l, float* __restrict__ o, float* __restrict__ lse) {
  constexpr int TPR = D / 4, G = kMergeThreads / TPR, U = 8;
  __shared__ f32x4 acc_lds[kMergeThreads];
  __shared__ float m_lds[G], l_lds[G];
  const int tid = threadIdx.x, row = blockIdx.x, grp = tid / TPR, c = tid % TPR;
  f32x4 acc = {};
  float m = -INFINITY, l = 0.f;
  for (int s0 = grp; s0 < n_split; s0 += U * G) {
    float ms[U], ls[U];
    f32x4 x[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int s = s0 + u * G;
      const size_t at = (size_t)min(s, n_split - 1) * rows + row;
      ms[u] = part_m[at];
      ls[u] = s < n_split ? part_l[at] : 0.f;
      x[u] = *reinterpret_cast<const f32x4*>(part_o + at * D + 4 * c);
    }
    float m_new = m;
#pragma unroll
    for (int u = 0; u < U; ++u) m_new = fmaxf(m_new, ms[u]);
    const float alpha = l == 0.f ? 0.f : __builtin_amdgcn_exp2f(m - m_new);
    acc *= alpha;
    l *= alpha;
    m = m_new;
#pragma unroll
    for (int u = 0; u < U; ++u) {  // (l = 0: no key; NaN stays)
      if (ls[u] == 0.f) continue;
      const float w = __builtin_amdgcn_exp2f(ms[u] - m);
      acc += w * x[u];
      l = fmaf(w, ls[u], l);
    }
  }
  acc_lds[tid] = acc;
  if (c == 0) {
    m_lds[grp] = m;
    l_lds[grp] = l;
  }
  __syncthreads();
  if (grp != 0) return;
  m = m_lds[0];
#pragma unroll
  for (int k = 1; k < G; ++k) m = fmaxf(m, m_lds[k]);
  acc = f32x4{};
  l = 0.f;
#pragma unroll
  for (int k = 0; k < G; ++k) {
    const float lk = l_lds[k];
    const float w = lk == 0.f ? 0.f : __builtin_amdgcn_exp2f(m_lds[k] - m);
    acc += w * acc_lds[k * TPR + tid];
    l = fmaf(w, lk, l);
  }
  *reinterpret_cast<f32x4*>(o + (size_t)row * D + 4 * c) = acc * (l == 0.f ? 0.f : 1.f / l);
  if (tid == 0) lse[row] = l == 0.f ? -INFINITY : 0.69314718055994531f * (m + log2f(l));
}

template <int D, bool WHOLE>
void launch_splits(const Dec4Params& p, const Decode4Plan& pl, dim3 grid, hipStream_t stream) {
  if (pl.rows == 16 && pl.waves == 8)
    hipLaunchKernelGGL((decode4_kernel<D, 1, 8, WHOLE>), grid, dim3(512), 0, stream, p);
  else if (pl.rows == 16)
    hipLaunchKernelGGL((decode4_kernel<D, 1, 4, WHOLE>), grid, dim3(256), 0, stream, p);
  else if (pl.rows == 32 && WHOLE && pl.waves == 8)  // (splits of 32 rows have four)
    hipLaunchKernelGGL((decode4_kernel<D, 2, 8, true>), grid, dim3(512), 0, stream, p);
  else if (pl.rows == 32)
    hipLaunchKernelGGL((decode4_kernel<D, 2, 4, WHOLE>), grid, dim3(256), 0, stream, p);
  else if (pl.rows == 64)
    hipLaunchKernelGGL((decode4_shared_kernel<D, 2, WHOLE>), grid, dim3(512), 0, stream, p);
  else
    hipLaunchKernelGGL((decode4_shared_kernel<D, 4, WHOLE>), grid, dim3(512), 0, stream, p);
}

template <int D>
hipError_t launch_d(const Dec4Params& p, const Decode4Plan& pl, hipStream_t stream) {
  const dim3 grid((unsigned)((int64_t)pl.n_split * pl.row_blocks * p.n_kv));
  if (pl.n_split == 1) launch_splits<D, true>(p, pl, grid, stream);
  else launch_splits<D, false>(p, pl, grid, stream);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || pl.n_split == 1) return e;
  hipLaunchKernelGGL((decode4_merge_kernel<D>), dim3((unsigned)p.rows_total), dim3(kMergeThreads), 0,
                     stream, p.n_split, p.rows_total, p.part_o, p.part_m, p.part_l, p.o, p.lse);
  return hipGetLastError();
}

Decode4Plan plan(const Decode4Args& a) {
  return plan_decode4(a.n_q, a.n_kv, a.head_dim, a.Lc, a.n_new);
}

}  // namespace

uint64_t decode4_workspace_bytes(const Decode4Args& a) { return plan(a).workspace_bytes; }

hipError_t launch_decode4(const Decode4Args& a, hipStream_t stream) {
  const Decode4Plan pl = plan(a);
  Dec4Params p;
  p.q = a.q;
  p.k_codes = a.k_codes; p.k_scales = a.k_scales; p.v_codes = a.v_codes; p.v_scales = a.v_scales;
  const int64_t rows = (int64_t)a.n_q * a.n_new;
  const size_t parts = (size_t)pl.n_split * rows;
  p.part_o = a.workspace;
  p.part_m = p.part_o + parts * a.head_dim;
  p.part_l = p.part_m + parts;
  p.o = a.o; p.lse = a.lse;
  p.capacity = a.capacity; p.Lc = a.Lc; p.n_new = a.n_new; p.causal = a.causal; p.n_kv = a.n_kv;
  p.R = a.n_q / a.n_kv * a.n_new;
  p.rows_total = (int)rows;
  p.n_split = pl.n_split; p.n_rb = pl.row_blocks; p.blocks_per_split = pl.blocks_per_split;
  p.scale_log2 = a.scale_log2;
  return a.head_dim == 128 ? launch_d<128>(p, pl, stream)
                           : launch_d<64>(p, pl, stream);
}

}  // namespace apb
