// Decoding-stage attention over a KV cache in 4 bits (the format of
// apb_cache4.hip), for gfx950.
//
// Rows are (query head, new token) pairs; the rows of one GQA group share a KV head.
// Few rows: the work is a read of the cache.  A CU's share of the HBM rate is a 32-key
// block of K and V (4352 bytes at d = 128) in about 450 cycles, which leaves each SIMD 450
// vector instructions a block to turn codes into operands and to form the softmax.
// Many rows: the SIMDs' vector instructions, of which a matrix product takes up as
// much as two (8 cycles of issue whatever its size, 4.7 for an instruction, 8 for a
// conversion of two codes, 16 for an exponential).  A block of 32 rows has 32 products, 64
// conversions, 16 exponentials and 140 others: 1700 cycles, the matrix pipe busy in 1000 of
// them, and takes a SIMD's two waves 2250 (512 rows of 8 heads x 16385 keys).  So:
//  * A wave owns N = 16 or 32 rows and takes 32-key blocks; the waves of a workgroup
//    share a split's blocks and meet in LDS at its end, so that a split is one partial.
//  * S^T = K Q^T on v_mfma_f32_16x16x32_bf16 or v_mfma_f32_32x32x16_bf16 (keys on M,
//    rows on N).  The 32-row product does twice the work for its 8 cycles.
//  * v_cvt_scalef32_pk_bf16_fp4 makes two elements at a time, scale applied: exact.
//  * O^T = V^T P^T needs 8 keys of one element in a lane: V goes to LDS row by row and
//    comes back through transposing reads (ds_read_b64_tr_b16).
//  * The probabilities are three bf16 each, the top, middle and lowest 8 bits of
//    their fp32 significand: three products in place of one, no rounding, whatever their
//    size beside the row's largest.  Two bf16 parts leave 2^-17, and o 2.3e-6 off.  Two
//    fp16 parts cost half the instructions (64 tokens of 32 / 8 heads x 16448 keys 35.6 us
//    against 40.5) but end at 2^-24: behind a key 14 nats above the others, with values
//    of zero, o is 1e-4 off, at 22 nats gone.
//  * Online softmax in base 2 in fp32 with a lazily moved maximum, as in the decode
//    kernels over bf16: the maximum and O's rescale only when a lane's sum of a block
//    passes 2^13.
#include <math.h>

#include <type_traits>

#include "apb_internal.h"
#include "apb_plan.h"

namespace apb {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short i16x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
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

__device__ __forceinline__ f32x4 product(const bf16x8& a, const bf16x8& b, const f32x4& c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ f32x16 product(const bf16x8& a, const bf16x8& b, const f32x16& c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}

// A V tile of 32 keys in LDS, bf16 row by row, chunk (16 bytes) c of key r at chunk c ^ swz(r).
// A clock serves 16 lanes' 16 bytes or 32 lanes' transposing reads, on 64 banks (256 bytes,
// one row of d = 128, two of 64).
// Transposing reads take 8 keys x 32 bytes (N = 16) or 4 keys x 64 bytes (N = 32).
template <int D, int N>
__device__ __forceinline__ int v_swz(int r) {
  if (N == 16) return (D == 128 ? 2 * (r & 7) : 2 * ((r >> 1) & 3)) ^ ((r >> 3) & 1);
  return (D == 128 ? 4 * (r & 3) : 4 * ((r >> 1) & 1)) ^ ((r >> 2) & 3);
}
// Its writes go without conflicts where 16 lanes' keys differ in the bits of r that move
// their chunks j: key x of 32 (the group's lanes neighbours, then keys in this order).
template <int D, int N>
__device__ __forceinline__ int v_key(int x) {
  const int hi = x & ~15;
  if (D == 128)
    return N == 16 ? hi | (x & 1) | (x & 2) << 2 | (x & 12) >> 1    // r0, r3, then r1, r2
                   : hi | (x & 3) << 2 | (x & 12) >> 2;             // r2, r3, then r0, r1
  return N == 16 ? hi | (x & 3) | (x & 4) << 1 | (x & 8) >> 1       // r0, r1, r3, then r2
                 : hi | (x & 1) | (x & 6) << 1 | (x & 8) >> 2;      // r0, r2, r3, then r1
}

// Scale bytes whose groups the products do not take: of 253 on 6 * 2^(b - 127) is infinite.
__device__ __forceinline__ bool not_finite(unsigned b) { return b > 252; }

// A group's 32 elements into its row's four chunks at `at` (exclusive or 16 j).
__device__ __forceinline__ void put_group(uint32_t at, const u32x4& codes, unsigned b) {
  const float scale = __uint_as_float(b << 23);
#pragma unroll
  for (int j = 0; j < 4; ++j) *(lds_u32x4*)(uintptr_t)(at ^ (16u * j)) = elements(codes[j], scale);
}

__device__ __forceinline__ uint32_t lds_base(const void* p) {
  return (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const uint8_t*)p;
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

// A wave's state: N rows, row lane % N in the 64 / N lanes of group lane / N each.
template <int D, int N>
struct Rows4 {
  static constexpr bool kWide = N == 32;
  using Acc = typename std::conditional<kWide, f32x16, f32x4>::type;
  static constexpr int TILES = 32 / N;      // products of N keys make a block's S
  static constexpr int KS = D * N / 512;    // products along the head size: 512 / N dims each
  static constexpr int NS = N / 2;          // logits of a block in a lane
  static constexpr int PS = NS / 8;         // P operands of a block, 8 keys of a lane each
  static constexpr int NDB = D / N;         // dim blocks of O
  static constexpr int QUADS = N * N / 256; // runs of four dims in an accumulator
  static constexpr int OUT = N * D * 4;     // bytes of O

  int vis;              // keys that the lane's row sees
  bf16x8 q[KS];
  Acc oacc[NDB];        // O^T of N dims: element r of group lg is dim dim_of(r / 4, lg) + r % 4
  float m_run, l_run;

  static __device__ __forceinline__ int lane_row() { return threadIdx.x % N; }
  static __device__ __forceinline__ int group() { return (threadIdx.x & 63) / N; }
  static __device__ __forceinline__ int dim_of(int quad, int lg) { return kWide ? 8 * quad + 4 * lg : 4 * lg; }
  // Key (of 32) of logit i: the keys of a P operand are those of the lane's own logits.
  static __device__ __forceinline__ int key_of(int i, int lg) {
    return (kWide ? 8 : 16) * (i >> 2) + 4 * lg + (i & 3);
  }
  static __device__ __forceinline__ float logit(const Acc (&s)[TILES], int i) {
    if constexpr (kWide) return s[0][i];
    else return s[i >> 2][i & 3];
  }

  // Rows from row0 on of KV head kvh; q's dims of product j from dim(j) on.
  template <typename Dim>
  __device__ __forceinline__ void start(const Dec4Params& p, int kvh, int row0, Dim dim) {
    const int rho = row0 + lane_row();
    const bool ok = rho < p.R;
    vis = p.causal ? p.Lc - p.n_new + (ok ? rho % p.n_new : 0) + 1 : p.Lc;
    const uint16_t* row = p.q + ((size_t)kvh * p.R + (ok ? rho : 0)) * D;
#pragma unroll
    for (int j = 0; j < KS; ++j)
      q[j] = as_bf16(*reinterpret_cast<const u32x4*>(row + dim(j)) & (ok ? ~0u : 0u));
    m_run = -INFINITY;
    l_run = 0.f;
#pragma unroll
    for (int db = 0; db < NDB; ++db) oacc[db] = Acc{};
  }

  // S of a tile: product j of KS.
  __device__ __forceinline__ void logits(Acc& s, const bf16x8& k, int j) const {
    const Acc zero = {};
    s = product(k, q[j], j == 0 ? zero : s);
  }

  // Keys that the row does not see, of the 32 from c0 on.
  __device__ __forceinline__ void mask(Acc (&s)[TILES], int c0) const {
    const int lg = group();
#pragma unroll
    for (int i = 0; i < NS; ++i)
      if (c0 + key_of(i, lg) >= vis) {
        if constexpr (kWide) s[0][i] = -INFINITY;
        else s[i >> 2][i & 3] = -INFINITY;
      }
  }

  // Logits of a block to probabilities, and the running maximum and sum.
  __device__ __forceinline__ void softmax(const Acc (&s)[TILES], float scale, float (&e)[NS]) {
    float sum;
    auto exps = [&]() __attribute__((always_inline)) {
      sum = 0.f;
#pragma unroll
      for (int i = 0; i < NS; ++i) e[i] = __builtin_amdgcn_exp2f(fmaf(logit(s, i), scale, -m_run));
#pragma unroll
      for (int i = 0; i < NS; i += 8)
        sum += ((e[i] + e[i + 1]) + (e[i + 2] + e[i + 3])) + ((e[i + 4] + e[i + 5]) + (e[i + 6] + e[i + 7]));
    };
    exps();
    if (__any(!(sum <= kSumLimit))) {
      float mx = logit(s, 0);
#pragma unroll
      for (int i = 1; i < NS; ++i) mx = fmaxf(mx, logit(s, i));
#pragma unroll
      for (int off = N; off < 64; off *= 2) mx = fmaxf(mx, __shfl_xor(mx, off));
      const float m_new = fmaxf(m_run, mx * scale);
      if (m_new == -INFINITY) {
        // nothing but keys that the row does not see, and NaN, which stays
        sum = 0.f;
#pragma unroll
        for (int i = 0; i < NS; ++i) {
          const float y = logit(s, i);
          e[i] = y == -INFINITY ? 0.f : y;
          sum += e[i];
        }
      } else {
        const float alpha = __builtin_amdgcn_exp2f(m_run - m_new);  // from -inf: 0
        m_run = m_new;
        l_run *= alpha;
#pragma unroll
        for (int db = 0; db < NDB; ++db) oacc[db] *= alpha;
        exps();
      }
    }
    l_run += sum;
  }

  // The probabilities as P operands, in their three parts.
  static __device__ __forceinline__ void parts(const float (&e)[NS], u32x4 (&pr)[PS][3]) {
#pragma unroll
    for (int i = 0; i < NS / 2; ++i) {
      unsigned hi[2], mid[2], lo[2];
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        hi[t] = __float_as_uint(e[2 * i + t]);
        const float r1 = e[2 * i + t] - __uint_as_float(hi[t] & 0xFFFF0000u);
        mid[t] = __float_as_uint(r1);
        lo[t] = __float_as_uint(r1 - __uint_as_float(mid[t] & 0xFFFF0000u));
      }
      u32x4(&out)[3] = pr[i / 4];
      out[0][i & 3] = __builtin_amdgcn_perm(hi[1], hi[0], 0x07060302u);
      out[1][i & 3] = __builtin_amdgcn_perm(mid[1], mid[0], 0x07060302u);
      out[2][i & 3] = __builtin_amdgcn_perm(lo[1], lo[0], 0x07060302u);
    }
  }

  // The lane's first transposing read of a V tile at `tile`: four keys of 16 lanes'
  // N dims; the lane then has its dim's element of them.
  static __device__ __forceinline__ uint32_t v_lane(uint32_t tile) {
    const int lane = threadIdx.x & 63, sl = lane & 15;
    const int key = kWide ? 4 * (lane >> 5) + (sl >> 2) : 4 * (lane >> 4) + (sl >> 2);
    const int chunk = (kWide ? 2 * (lane >> 4 & 1) : 0) + ((sl & 3) >> 1);
    return tile + (uint32_t)(key * 2 * D + 16 * (chunk ^ v_swz<D, N>(key)) + 8 * (sl & 1));
  }
  // The V operand of dim block db and P operand ps: two of them, 8 or 16 keys apart.
  static __device__ __forceinline__ bf16x8 v_operand(uint32_t v_get, int db, int ps) {
    i16x4 part[2];
#pragma unroll
    for (int rd = 0; rd < 2; ++rd) {
      // (N = 32: key + 8 moves bit 1 of the swizzle)
      const uint32_t a = v_get ^ (uint32_t)(2 * N * db ^ (kWide ? 32 * rd : 0));
      part[rd] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
          (lds_i16x4*)(uintptr_t)(a + (uint32_t)((16 * ps + (kWide ? 8 : 16) * rd) * 2 * D)));
    }
    return __builtin_bit_cast(bf16x8,
                              __builtin_shufflevector(part[0], part[1], 0, 1, 2, 3, 4, 5, 6, 7));
  }
  // O^T += V^T P^T: one part of one P operand, one dim block.
  __device__ __forceinline__ void values(int db, const bf16x8& v, const u32x4& p) {
    oacc[db] = product(v, as_bf16(p), oacc[db]);
  }

  // Values of group g (dims 32 g ..) of key c are NaN: so is O of the row if it sees it.
  __device__ __forceinline__ void not_a_number(int g, int c) {
#pragma unroll
    for (int db = 0; db < NDB; ++db)
      if (db * N / 32 == g && c < vis) oacc[db] = Acc{} + NAN;
  }

  // The parts of WK waves over the same rows (this one the wk-th) meet in LDS: at o_lds,
  // OUT bytes each, and ml_lds.  Then the waves take the rows in turn, whole ones: a store
  // is 1 KiB that lies together.  Chunk c (four dims) of row r sits at chunk c ^ (r & 15)
  // of its row, on a bank of its own in both directions.
  template <int WK, bool WHOLE>
  __device__ __forceinline__ void finish(const Dec4Params& p, const Place4& at, int row0, int wk,
                                         uint8_t* o_lds, float (*ml_lds)[WK][N]) {
    constexpr int CH = D / 4, RPI = 64 / CH;      // chunks of a row, rows of a store
    constexpr int TURNS = (N + RPI * WK - 1) / (RPI * WK);
    const int lane = threadIdx.x & 63, r0 = lane_row(), lg = group();
#pragma unroll
    for (int off = N; off < 64; off *= 2) l_run += __shfl_xor(l_run, off);
    __syncthreads();  // the tiles are done with
#pragma unroll
    for (int db = 0; db < NDB; ++db)
#pragma unroll
      for (int k = 0; k < QUADS; ++k) {
        f32x4 y;
#pragma unroll
        for (int i = 0; i < 4; ++i) y[i] = oacc[db][4 * k + i];
        const int c = (N * db + dim_of(k, lg)) / 4;
        *reinterpret_cast<f32x4*>(o_lds + wk * OUT + r0 * (4 * D) + 16 * (c ^ (r0 & 15))) = y;
      }
    if (lg == 0) {
      ml_lds[0][wk][r0] = m_run;
      ml_lds[1][wk][r0] = l_run;
    }
    __syncthreads();
    const int c = lane % CH;
#pragma unroll
    for (int it = 0; it < TURNS; ++it) {
      const int r = (it * WK + wk) * RPI + lane / CH;
      if (r >= N || row0 + r >= p.R) continue;
      float m = -INFINITY, l = 0.f;
#pragma unroll
      for (int k = 0; k < WK; ++k) m = fmaxf(m, ml_lds[0][k][r]);
      f32x4 y = {};
#pragma unroll
      for (int k = 0; k < WK; ++k) {
        const float lk = ml_lds[1][k][r];  // (0: no key; NaN stays)
        const float w = lk == 0.f ? 0.f : __builtin_amdgcn_exp2f(ml_lds[0][k][r] - m);
        l = fmaf(w, lk, l);
        y += w * *reinterpret_cast<const f32x4*>(o_lds + k * OUT + r * (4 * D) + 16 * (c ^ (r & 15)));
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

// N rows of a KV head: WK waves, each with 32-key blocks of its own.  A product
// over the head size may take it in any order that both operands share, so a lane takes
// the part of its key that lies together and K goes from memory to the operand
// registers without LDS; a wave has its V tile to itself, so that the loop has no barrier.
template <int D, int N, int WK, bool WHOLE>
__global__ void __launch_bounds__(64 * WK, 2) decode4_kernel(Dec4Params p) {
  using Rows = Rows4<D, N>;
  constexpr int G = D / 32, TILE = 32 * D * 2, OUT = Rows::OUT;
  constexpr int RUN = D * N / 64;            // elements of a key in a lane, of TILES keys
  constexpr int KW = RUN / 8, KB = RUN > 32 ? 2 : 1, VL = D / 64;
  __shared__ __attribute__((aligned(256))) uint8_t lds[WK * (OUT > TILE ? OUT : TILE)];
  __shared__ float ml_lds[2][WK][N];

  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const Place4 at = place4(p.n_split, p.n_rb, p.n_kv);
  const int nblk = (p.Lc + 31) / 32;
  const int b0 = at.split * p.blocks_per_split, b1 = min(b0 + p.blocks_per_split, nblk);
  const int vis_all = p.causal ? p.Lc - p.n_new + 1 : p.Lc;  // keys that every row sees
  const uint32_t tile = lds_base(lds) + (uint32_t)(wave * TILE);

  // Where a lane works in a block: of K it takes its part of each tile's key, of V whole
  // groups, of keys v_of.
  const int lane = threadIdx.x & 63, lr = Rows::lane_row(), lg = Rows::group(), g = lane % G;
  int v_of[VL];
  uint32_t v_put[VL];
#pragma unroll
  for (int v = 0; v < VL; ++v) {
    v_of[v] = v_key<D, N>((64 * v + lane) / G);
    v_put[v] = tile + (uint32_t)(v_of[v] * 2 * D + 16 * ((4 * g) ^ v_swz<D, N>(v_of[v])));
  }
  const uint32_t v_get = Rows::v_lane(tile);
  // The codes and scale bytes that a lane takes of a block.
  struct Block {
    unsigned kw[Rows::TILES][KW], kb[Rows::TILES][KB];
    u32x4 vw[VL];
    unsigned vb[VL];
  };

  auto load = [&](int b) __attribute__((always_inline)) {
    Block x;
    // (past the split's last block that again, past the last key that)
    const int c0 = 32 * min(b, b1 - 1), last = p.Lc - 1 - c0;
    const size_t r0 = (size_t)at.kvh * p.capacity + c0;
    const uint8_t* kc = p.k_codes + r0 * (D / 2);
    const uint8_t* ks = p.k_scales + r0 * G;
    const uint8_t* vc = p.v_codes + r0 * (D / 2);
    const uint8_t* vs = p.v_scales + r0 * G;
#pragma unroll
    for (int i = 0; i < Rows::TILES; ++i) {
      const uint32_t key = (uint32_t)min(N * i + lr, last);
      if constexpr (RUN >= 32) {
#pragma unroll
        for (int h = 0; h < KB; ++h) {
          const u32x4 w = *reinterpret_cast<const u32x4*>(kc + (key * (D / 2) + (RUN / 2) * lg + 16u * h));
          x.kw[i][4 * h] = w[0]; x.kw[i][4 * h + 1] = w[1];
          x.kw[i][4 * h + 2] = w[2]; x.kw[i][4 * h + 3] = w[3];
          x.kb[i][h] = ks[key * G + KB * lg + h];
        }
      } else {
        const u32x2 w = *reinterpret_cast<const u32x2*>(kc + (key * (D / 2) + (RUN / 2) * lg));
        x.kw[i][0] = w[0]; x.kw[i][1] = w[1];
        x.kb[i][0] = ks[key * G + RUN * lg / 32];
      }
    }
#pragma unroll
    for (int v = 0; v < VL; ++v) {
      const uint32_t key = (uint32_t)min(v_of[v], last);
      x.vw[v] = *reinterpret_cast<const u32x4*>(vc + (key * (D / 2) + 16u * g));
      x.vb[v] = vs[key * G + g];
    }
    return x;
  };

  Rows rows;
  const int row0 = N * at.row_block;
  rows.start(p, at.kvh, row0, [&](int j) { return RUN * lg + 8 * j; });

  // Block b from x, which takes the wave's next block as soon as it is done with; past the
  // split's end it asks for its last block, which is on the way anyway (the next split's
  // would be 26.3 MB of reads in place of 18.1 with one token over 16385 keys of 8 heads).  A
  // second block in flight per wave gained nothing (those 11.4 against 12.3 us, 524289 keys
  // 110.8 against 112.2): eight waves of a CU have 35 KiB under way.
  auto block = [&](Block& x, int b) __attribute__((always_inline)) {
    const int c0 = 32 * b;
    typename Rows::Acc s[Rows::TILES];
#pragma unroll
    for (int i = 0; i < Rows::TILES; ++i)
#pragma unroll
      for (int j = 0; j < KW; ++j) {
        const float scale = __uint_as_float(x.kb[i][j / 4 % KB] << 23);  // b = 255: NaN elements
        rows.logits(s[i], as_bf16(elements(x.kw[i][j], scale)), j);
      }

    // A group that is not finite (NaN, or under a scale past bf16's numbers) goes into O by
    // hand, for the rows that see the first key of it, and into the tile as zeros: in a
    // product a zero probability would not keep it out.
    bool bad = false;
#pragma unroll
    for (int v = 0; v < VL; ++v) bad |= not_finite(x.vb[v]);
    if (__any(bad)) {
#pragma unroll
      for (int n = 0; n < G; ++n) {
        int f = 32;
#pragma unroll
        for (int v = 0; v < VL; ++v)
          if (not_finite(x.vb[v]) && g == n) f = min(f, v_of[v]);
        for (int off = 1; off < 64; off *= 2) f = min(f, __shfl_xor(f, off));
        f = __builtin_amdgcn_readfirstlane(f);
        if (f < 32) rows.not_a_number(n, c0 + f);
      }
#pragma unroll
      for (int v = 0; v < VL; ++v)
        if (not_finite(x.vb[v])) {
          x.vw[v] = u32x4{};
          x.vb[v] = 127;
        }
    }
#pragma unroll
    for (int v = 0; v < VL; ++v) put_group(v_put[v], x.vw[v], x.vb[v]);
    x = load(b + WK);
    // (a wave's LDS accesses are in order; the reads land during the softmax)
    bf16x8 v[Rows::NDB][Rows::PS];
#pragma unroll
    for (int db = 0; db < Rows::NDB; ++db)
#pragma unroll
      for (int ps = 0; ps < Rows::PS; ++ps) v[db][ps] = Rows::v_operand(v_get, db, ps);
    __builtin_amdgcn_sched_barrier(0);

    if (c0 + 32 > vis_all) rows.mask(s, c0);
    float e[Rows::NS];
    rows.softmax(s, p.scale_log2, e);
    u32x4 pr[Rows::PS][3];
    Rows::parts(e, pr);
#pragma unroll
    for (int ps = 0; ps < Rows::PS; ++ps)
#pragma unroll
      for (int t = 0; t < 3; ++t)
#pragma unroll
        for (int db = 0; db < Rows::NDB; ++db) rows.values(db, v[db][ps], pr[ps][t]);
  };
  if (b0 + wave < b1) {
    Block x = load(b0 + wave);
    for (int b = b0 + wave; b < b1; b += WK) block(x, b);
  }
  rows.template finish<WK, WHOLE>(p, at, row0, wave, lds, ml_lds);
}

// The splits of a row: O = sum_s 2^(m_s - m) O_s / l, l = sum_s 2^(m_s - m) l_s, with m
// the largest m_s; lse = ln 2 (m + log2 l).  Parts keep O undivided, and m apart from
// log l: a sum of the two would lose l's digits beside a large m.  16 bytes of O a
// thread; a row's G thread groups take every G-th split, eight at a time against their own
// maximum, so that all a thread reads is one trip to memory, and meet in LDS.  With up to
// 8 or 16 splits one or two groups a row do, and a workgroup has several rows: 256 rows of
// a KV head, 8 heads x 16448 keys, 4 splits 41.2 -> 40.0 us in all, 128 rows x 4000 keys
// 14.9 -> 14.0, one row x 1000 7.0 -> 6.3, 40 rows of 2 heads of d = 64 x 1000 7.3 -> 6.4.
constexpr int kMergeThreads = 256;

template <int D, int G>
__global__ void __launch_bounds__(kMergeThreads) decode4_merge_kernel(
    int n_split, int rows, const float* __restrict__ part_o, const float* __restrict__ part_m,
    const float* __restrict__ part_l, float* __restrict__ o, float* __restrict__ lse) {
  constexpr int TPR = D / 4, RPW = kMergeThreads / (TPR * G), U = 8;
  __shared__ f32x4 acc_lds[kMergeThreads];
  __shared__ float m_lds[kMergeThreads / TPR], l_lds[kMergeThreads / TPR];
  const int tid = threadIdx.x, grp = tid / TPR % G, c = tid % TPR, wg_row = tid / (TPR * G);
  const int my_row = (int)blockIdx.x * RPW + wg_row, row = min(my_row, rows - 1);
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
    for (int u = 0; u < U; ++u) {  // (l = 0: no key with weight; a NaN of V stays)
      const float w = ls[u] == 0.f ? 0.f : __builtin_amdgcn_exp2f(ms[u] - m);
      acc += w * x[u];
      l = fmaf(w, ls[u], l);
    }
  }
  if constexpr (G > 1) {
    const int first = G * wg_row;
    acc_lds[tid] = acc;
    if (c == 0) {
      m_lds[first + grp] = m;
      l_lds[first + grp] = l;
    }
    __syncthreads();
    if (grp != 0) return;
    m = m_lds[first];
#pragma unroll
    for (int k = 1; k < G; ++k) m = fmaxf(m, m_lds[first + k]);
    acc = f32x4{};
    l = 0.f;
#pragma unroll
    for (int k = 0; k < G; ++k) {
      const float lk = l_lds[first + k];
      const float w = lk == 0.f ? 0.f : __builtin_amdgcn_exp2f(m_lds[first + k] - m);
      acc += w * acc_lds[k * TPR + tid];
      l = fmaf(w, lk, l);
    }
  }
  if (my_row >= rows) return;
  *reinterpret_cast<f32x4*>(o + (size_t)row * D + 4 * c) = acc * (l == 0.f ? 0.f : 1.f / l);
  if (c == 0) lse[row] = l == 0.f ? -INFINITY : 0.69314718055994531f * (m + log2f(l));
}

template <int D, int N, bool WHOLE>
void launch_rows(const Dec4Params& p, const Decode4Plan& pl, dim3 grid, hipStream_t stream) {
  if (pl.waves == 8)
    hipLaunchKernelGGL((decode4_kernel<D, N, 8, WHOLE>), grid, dim3(512), 0, stream, p);
  else
    hipLaunchKernelGGL((decode4_kernel<D, N, 4, WHOLE>), grid, dim3(256), 0, stream, p);
}

template <int D, bool WHOLE>
void launch_splits(const Dec4Params& p, const Decode4Plan& pl, dim3 grid, hipStream_t stream) {
  if (pl.rows == 16) launch_rows<D, 16, WHOLE>(p, pl, grid, stream);
  else launch_rows<D, 32, WHOLE>(p, pl, grid, stream);
}

template <int D>
hipError_t launch_d(const Dec4Params& p, const Decode4Plan& pl, hipStream_t stream) {
  const dim3 grid((unsigned)((int64_t)pl.n_split * pl.row_blocks * p.n_kv));
  if (pl.n_split == 1) launch_splits<D, true>(p, pl, grid, stream);
  else launch_splits<D, false>(p, pl, grid, stream);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || pl.n_split == 1) return e;
  auto merge = [&](auto groups) {
    constexpr int G = decltype(groups)::value, RPW = kMergeThreads / (D / 4 * G);
    hipLaunchKernelGGL((decode4_merge_kernel<D, G>), dim3((unsigned)((p.rows_total + RPW - 1) / RPW)),
                       dim3(kMergeThreads), 0, stream, p.n_split, p.rows_total, p.part_o, p.part_m,
                       p.part_l, p.o, p.lse);
  };
  if (pl.n_split <= 8) merge(std::integral_constant<int, 1>{});
  else if (pl.n_split <= 16) merge(std::integral_constant<int, 2>{});
  else merge(std::integral_constant<int, kMergeThreads / (D / 4)>{});
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
