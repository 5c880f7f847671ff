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
  int capacity, Lc, n_new, causal, R, rows_total, n_split, n_rb, blocks_per_split;
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

__device__ __forceinline__ float across_groups_max(float x) {
  x = fmaxf(x, __shfl_xor(x, 16));
  return fmaxf(x, __shfl_xor(x, 32));
}

// Workgroup: split (fastest), row block, KV head.
template <int D, int RB, int WK, bool WHOLE>
__global__ void __launch_bounds__(64 * WK, RB == 4 ? 1 : 2) decode4_kernel(Dec4Params p) {
  constexpr int NDB = D / 16, KW = Block4<D>::KW, VL = Block4<D>::VL;
  constexpr int TILE = 32 * D * 2;            // bytes of a V tile
  constexpr int OUT = RB * NDB * 4 * 64 * 4;  // bytes of a wave's O
  constexpr int LDS = WK * (OUT > TILE && WK > 1 ? OUT : TILE);
  __shared__ __attribute__((aligned(256))) uint8_t lds[LDS];
  __shared__ float ml_lds[2][WK][RB][16];

  const int lane = threadIdx.x & 63, li = lane & 15, lg = lane >> 4;
  const int wave = WK == 1 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int split = blockIdx.x % p.n_split;
  const int rb0 = (int)(blockIdx.x / p.n_split) % p.n_rb * RB;
  const int kvh = (int)(blockIdx.x / p.n_split) / p.n_rb;
  const int nblk = (p.Lc + 31) / 32;
  const int b0 = split * p.blocks_per_split, b1 = min(b0 + p.blocks_per_split, nblk);

  // This lane's rows (MFMA column li of every row block) and the keys they see.
  int vis[RB];
  bf16x8 q[RB][KW];
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) {
    const int rho = (rb0 + rb) * 16 + li;
    const bool ok = rho < p.R;
    vis[rb] = p.causal ? p.Lc - p.n_new + (ok ? rho % p.n_new : 0) + 1 : p.Lc;
    const uint16_t* row = p.q + ((size_t)kvh * p.R + (ok ? rho : 0)) * D + lg * (D / 4);
#pragma unroll
    for (int j = 0; j < KW; ++j)
      q[rb][j] = as_bf16(*reinterpret_cast<const u32x4*>(row + 8 * j) & (ok ? ~0u : 0u));
  }
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
  uint32_t v_get;
  {
    const int row = 4 * lg + (li >> 2);
    v_get = tile + (uint32_t)(row * 2 * D + 16 * (((li & 3) >> 1) ^ v_swz<D>(row)) + 8 * (li & 1));
  }

  auto load = [&](int b) __attribute__((always_inline)) {
    Block4<D> x;
    const int c0 = 32 * b, last = p.Lc - 1 - c0;  // rows past the last key repeat it
    const size_t r0 = (size_t)kvh * p.capacity + c0;
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

  f32x4 oacc[RB][NDB];
  float m_run[RB], l_run[RB];
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) {
    m_run[rb] = -INFINITY;
    l_run[rb] = 0.f;
#pragma unroll
    for (int db = 0; db < NDB; ++db) oacc[rb][db] = f32x4{};
  }

  Block4<D> next;
  if (b0 + wave < b1) next = load(b0 + wave);
  for (int b = b0 + wave; b < b1; b += WK) {
    const Block4<D> x = next;
    if (b + WK < b1) next = load(b + WK);
    const int c0 = 32 * b;

    // S^T: element r of tile i of this lane is key c0 + 16 i + 4 lg + r
    f32x4 s[2][RB];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const float scale = __uint_as_float(x.kb[i] << 23);  // b = 255: NaN elements
#pragma unroll
      for (int j = 0; j < KW; ++j) {
        const bf16x8 k = as_bf16(elements(x.kw[i][j], scale));
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) {
          const f32x4 zero = {};
          s[i][rb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k, q[rb][j], j == 0 ? zero : s[i][rb],
                                                             0, 0, 0);
        }
      }
    }

    // V -> LDS.  A group of NaN goes there as zeros, and into O by hand, for the
    // rows that see it: in a product a zero probability would not keep it out.
    bool bad = false;
#pragma unroll
    for (int v = 0; v < VL; ++v) bad |= x.vb[v] == 255;
    const bool any_bad = __any(bad);
#pragma unroll
    for (int v = 0; v < VL; ++v) {
      unsigned w[4] = {x.vw[v][0], x.vw[v][1], x.vw[v][2], x.vw[v][3]};
      float scale = __uint_as_float(x.vb[v] << 23);
      if (any_bad && x.vb[v] == 255) {
        w[0] = w[1] = w[2] = w[3] = 0;
        scale = 1.f;
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const unsigned mine = flip ? w[j ^ 1] : w[j];
        *(lds_u32x4*)(uintptr_t)(v_put[v] ^ (16u * j)) = elements(mine, scale);
      }
    }

    if (c0 + 32 > vis_all) {
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int rb = 0; rb < RB; ++rb)
#pragma unroll
          for (int r = 0; r < 4; ++r)
            if (c0 + 16 * i + 4 * lg + r >= vis[rb]) s[i][rb][r] = -INFINITY;
    }

    u32x4 pr[RB][3];  // the probabilities' three parts, as the P operand
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
      float e[8], sum;
      auto exps = [&]() __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < 8; ++i)
          e[i] = __builtin_amdgcn_exp2f(fmaf(s[i >> 2][rb][i & 3], p.scale_log2, -m_run[rb]));
        sum = ((e[0] + e[1]) + (e[2] + e[3])) + ((e[4] + e[5]) + (e[6] + e[7]));
      };
      exps();
      if (__any(!(sum <= kSumLimit))) {
        float mx = s[0][rb][0];
#pragma unroll
        for (int i = 1; i < 8; ++i) mx = fmaxf(mx, s[i >> 2][rb][i & 3]);
        const float m_new = fmaxf(m_run[rb], across_groups_max(mx) * p.scale_log2);
        if (m_new == -INFINITY) {
          // nothing but keys that the row does not see, and NaN, which stays
          sum = 0.f;
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const float y = s[i >> 2][rb][i & 3];
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
      for (int i = 0; i < 4; ++i) {
        unsigned hi[2], mid[2], lo[2];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          hi[t] = __float_as_uint(e[2 * i + t]);
          const float r1 = e[2 * i + t] - __uint_as_float(hi[t] & 0xFFFF0000u);
          mid[t] = __float_as_uint(r1);
          lo[t] = __float_as_uint(r1 - __uint_as_float(mid[t] & 0xFFFF0000u));
        }
        pr[rb][0][i] = __builtin_amdgcn_perm(hi[1], hi[0], 0x07060302u);
        pr[rb][1][i] = __builtin_amdgcn_perm(mid[1], mid[0], 0x07060302u);
        pr[rb][2][i] = __builtin_amdgcn_perm(lo[1], lo[0], 0x07060302u);
      }
    }

    // O^T += V^T P^T
#pragma unroll
    for (int db = 0; db < NDB; ++db) {
      i16x4 part[2];
#pragma unroll
      for (int rd = 0; rd < 2; ++rd)
        part[rd] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
            (lds_i16x4*)(uintptr_t)((v_get ^ (32u * db)) + (uint32_t)(16 * rd * 2 * D)));
      const bf16x8 v = __builtin_bit_cast(
          bf16x8, __builtin_shufflevector(part[0], part[1], 0, 1, 2, 3, 4, 5, 6, 7));
#pragma unroll
      for (int t = 0; t < 3; ++t)
#pragma unroll
        for (int rb = 0; rb < RB; ++rb)
          oacc[rb][db] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, as_bf16(pr[rb][t]), oacc[rb][db],
                                                                 0, 0, 0);
    }

    if (any_bad) {  // the first key of each group's NaN
#pragma unroll
      for (int g = 0; g < G; ++g) {
        int first = 32;
#pragma unroll
        for (int v = 0; v < VL; ++v) {
          const unsigned long long hit = __ballot(x.vb[v] == 255 && (int)(lane % G) == g);
          if (hit) first = min(first, (64 * v + (int)__builtin_ctzll(hit)) / G);
        }
#pragma unroll
        for (int rb = 0; rb < RB; ++rb)
          if (first < 32 && c0 + first < vis[rb])
            oacc[rb][2 * g] = oacc[rb][2 * g + 1] = f32x4{} + NAN;
      }
    }
  }

  // sums over the four lanes of a row
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) {
    l_run[rb] += __shfl_xor(l_run[rb], 16);
    l_run[rb] += __shfl_xor(l_run[rb], 32);
  }
  // the waves' parts: O, maximum and sum through LDS, then dim block db to wave db % WK
  float w[RB][WK], m_all[RB], l_all[RB];
  float* const mine = reinterpret_cast<float*>(lds + (WK > 1 ? wave * OUT : 0)) + 4 * lane;
  if constexpr (WK > 1) {
    __syncthreads();  // the tiles are done with (a wave's O may lie over another's)
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
#pragma unroll
      for (int db = 0; db < NDB; ++db)
        *reinterpret_cast<f32x4*>(mine + 256 * (rb * NDB + db)) = oacc[rb][db];
      if (lg == 0) {
        ml_lds[0][wave][rb][li] = m_run[rb];
        ml_lds[1][wave][rb][li] = l_run[rb];
      }
    }
    __syncthreads();
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
      m_all[rb] = -INFINITY;
      l_all[rb] = 0.f;
#pragma unroll
      for (int k = 0; k < WK; ++k) m_all[rb] = fmaxf(m_all[rb], ml_lds[0][k][rb][li]);
#pragma unroll
      for (int k = 0; k < WK; ++k) {
        const float l = ml_lds[1][k][rb][li];  // (0: no key; NaN stays)
        w[rb][k] = l == 0.f ? 0.f : __builtin_amdgcn_exp2f(ml_lds[0][k][rb][li] - m_all[rb]);
        l_all[rb] = fmaf(w[rb][k], l, l_all[rb]);
      }
    }
  } else {
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
      m_all[rb] = m_run[rb];
      l_all[rb] = l_run[rb];
    }
  }
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) {
    const int rho = (rb0 + rb) * 16 + li;
    if (rho >= p.R) continue;
    const size_t row = (size_t)kvh * p.R + rho;
    const float inv = !WHOLE ? 1.f : l_all[rb] == 0.f ? 0.f : 1.f / l_all[rb];
    float* out = (WHOLE ? p.o : p.part_o + (size_t)split * p.rows_total * D) + row * D + 4 * lg;
#pragma unroll
    for (int db = 0; db < NDB; ++db) {
      if (WK > 1 && db % WK != wave) continue;
      f32x4 y = {};
      if constexpr (WK > 1) {
#pragma unroll
        for (int k = 0; k < WK; ++k)
          y += w[rb][k] * *reinterpret_cast<const f32x4*>(
                              reinterpret_cast<float*>(lds + k * OUT) + 4 * lane + 256 * (rb * NDB + db));
      } else {
        y = oacc[rb][db];
      }
      *reinterpret_cast<f32x4*>(out + 16 * db) = y * inv;
    }
    if (wave == 0 && lg == 0) {
      if constexpr (WHOLE) {
        p.lse[row] = l_all[rb] == 0.f ? -INFINITY
                                      : 0.69314718055994531f * (m_all[rb] + log2f(l_all[rb]));
      } else {
        p.part_m[(size_t)split * p.rows_total + row] = m_all[rb];
        p.part_l[(size_t)split * p.rows_total + row] = l_all[rb];
      }
    }
  }
}

// The splits of a row: O = sum_s 2^(m_s - m) O_s / l, l = sum_s 2^(m_s - m) l_s, with m
// the largest m_s; lse = ln 2 (m + log2 l).  Parts keep O undivided, and m apart from
// log l: a sum of the two would lose l's digits beside a large m.  A workgroup per row,
// 16 bytes a thread, thread groups taking every G-th split.
constexpr int kMergeThreads = 256;

template <int D>
__global__ void __launch_bounds__(kMergeThreads) decode4_merge_kernel(
    int n_split, int rows, const float* __restrict__ part_o, const float* __restrict__ part_m,
    const float* __restrict__ part_l, float* __restrict__ o, float* __restrict__ lse) {
  constexpr int TPR = D / 4, G = kMergeThreads / TPR;
  __shared__ f32x4 acc_lds[kMergeThreads];
  __shared__ float red[kMergeThreads / 64], l_lds[G];
  const int tid = threadIdx.x, row = blockIdx.x, grp = tid / TPR, c = tid % TPR;
  float m = -INFINITY;
  for (int s = tid; s < n_split; s += kMergeThreads) m = fmaxf(m, part_m[(size_t)s * rows + row]);
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) m = fmaxf(m, __shfl_xor(m, off));
  if (tid % 64 == 0) red[tid / 64] = m;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kMergeThreads / 64; ++w) m = fmaxf(m, red[w]);
  f32x4 acc = {};
  float l = 0.f;
#pragma unroll 4
  for (int s = grp; s < n_split; s += G) {
    const size_t at = (size_t)s * rows + row;
    const float ls = part_l[at];
    const float w = ls == 0.f ? 0.f : __builtin_amdgcn_exp2f(part_m[at] - m);
    acc += w * *reinterpret_cast<const f32x4*>(part_o + at * D + 4 * c);
    l = fmaf(w, ls, l);
  }
  acc_lds[tid] = acc;
  if (c == 0) l_lds[grp] = l;
  __syncthreads();
  if (grp != 0) return;
#pragma unroll
  for (int k = 1; k < G; ++k) {
    acc += acc_lds[k * TPR + tid];
    l += l_lds[k];
  }
  *reinterpret_cast<f32x4*>(o + (size_t)row * D + 4 * c) = acc * (l == 0.f ? 0.f : 1.f / l);
  if (tid == 0) lse[row] = l == 0.f ? -INFINITY : 0.69314718055994531f * (m + log2f(l));
}

template <int D, int RB>
void launch_rows(const Dec4Params& p, unsigned grid, hipStream_t stream) {
  constexpr int WK = 4;
  if (p.n_split == 1)
    hipLaunchKernelGGL((decode4_kernel<D, RB, WK, true>), dim3(grid), dim3(64 * WK), 0, stream, p);
  else
    hipLaunchKernelGGL((decode4_kernel<D, RB, WK, false>), dim3(grid), dim3(64 * WK), 0, stream, p);
}

template <int D>
hipError_t launch_d(const Dec4Params& p, const Decode4Plan& pl, int n_kv, hipStream_t stream) {
  const unsigned grid = (unsigned)((int64_t)pl.n_split * pl.row_blocks * n_kv);
  if (pl.rb == 1) launch_rows<D, 1>(p, grid, stream);
  else if (pl.rb == 2) launch_rows<D, 2>(p, grid, stream);
  else launch_rows<D, 4>(p, grid, stream);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || pl.n_split == 1) return e;
  hipLaunchKernelGGL((decode4_merge_kernel<D>), dim3((unsigned)p.rows_total), dim3(kMergeThreads), 0,
                     stream, pl.n_split, p.rows_total, p.part_o, p.part_m, p.part_l, p.o, p.lse);
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
  p.capacity = a.capacity; p.Lc = a.Lc; p.n_new = a.n_new; p.causal = a.causal;
  p.R = a.n_q / a.n_kv * a.n_new;
  p.rows_total = (int)rows;
  p.n_split = pl.n_split; p.n_rb = pl.row_blocks; p.blocks_per_split = pl.blocks_per_split;
  p.scale_log2 = a.scale_log2;
  return a.head_dim == 128 ? launch_d<128>(p, pl, a.n_kv, stream)
                           : launch_d<64>(p, pl, a.n_kv, stream);
}

}  // namespace apb
