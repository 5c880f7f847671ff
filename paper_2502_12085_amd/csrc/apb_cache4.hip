// KV cache in 4 bits for gfx950: rows of bf16 K and V quantised into it, and read
// back.  Groups of 32 elements along the head size share a power of two 2^(b - 127);
// an element is e2m1 (0, 0.5, 1, 1.5, 2, 3, 4, 6 and their negatives), two to a
// byte.
//
// Scale.  A group with largest magnitude a takes the smallest e with a <= 7 * 2^e.
// Past 6 a magnitude becomes 6; up to 7 that is off by no more than the half step of
// 1 that rounding between 4 and 6 costs anyway.  Signal to error power of N(0, 1)
// rows: 19.0 dB (with a <= 6 * 2^e 18.8, with a < 8 * 2^e 18.8); with 2% of channels
// 8 times as large 16.2 (15.4, 16.2).  For a bf16 a = (1 + M / 128) 2^(E - 127) that is
// b = e + 127 = E - 2 + (M > 96), one addition and shift of its bits.  Held to 7 .. 252
// every value of the cache is a normal bf16 number, so that reading back and the
// products with it are exact.  Powers of two make the division by the scale exact
// too: the codes are a function of the row alone, with one rounding, to nearest even,
// which v_cvt_scalef32_pk_fp4_bf16 does.
//
// Both directions are bound by HBM: 2 bytes of bf16 and 17 / 32 of cache an element.
// A thread takes 8 elements (16 bytes of bf16, 4 of codes), a group is four threads.
// The bf16 side passes the caches by, which leaves them to the cache's codes.  131072 rows
// of 8 heads of d = 128 (679 MB), four sets of tensors in turn: write 122 -> 116 us (5.9
// TB/s), read 123 -> 107 (6.4), against four rows a thread and plain loads and stores;
// eight rows 120 and 121, one 116 and 128.  (A write and a read of the same rows in turn
// take 104 and 93: part of the codes is still in the Infinity Cache.)  A few rows are one
// launch's latency, 1.6 us.
#include "apb_internal.h"

namespace apb {
namespace {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));

constexpr int kThreads = 256;
constexpr int kSteps = 2;  // rows a thread moves, their loads in flight together

constexpr int rows_per_block(int d) { return kThreads / (d / 8) * kSteps; }

// Workgroup blockIdx.x: row block, then K or V, then head, the row block fastest.
struct Place {
  int which, row, col;   // K or V, first row of the thread, its 8-element column
  size_t bf16, cache;    // row index of row 0 of the call in either tensor
};

template <int D>
__device__ __forceinline__ Place place(const Cache4Args& a) {
  const unsigned nb = (unsigned)(((int64_t)a.n_rows + rows_per_block(D) - 1) / rows_per_block(D));
  const unsigned blk = blockIdx.x % nb, hw = blockIdx.x / nb;
  Place p;
  p.which = (int)(hw & 1);
  p.row = (int)blk * rows_per_block(D) + (int)threadIdx.x / (D / 8);
  p.col = (int)threadIdx.x % (D / 8);
  p.bf16 = (size_t)(hw >> 1) * a.bf16_rows + a.bf16_first;
  p.cache = (size_t)(hw >> 1) * a.capacity + a.first_row;
  return p;
}

// The four lanes of a group are neighbours: largest value over them.
__device__ __forceinline__ unsigned quad_max(unsigned x) {
  x = max(x, (unsigned)__builtin_amdgcn_update_dpp(0, (int)x, 0xB1, 0xF, 0xF, true));  // lane ^ 1
  return max(x, (unsigned)__builtin_amdgcn_update_dpp(0, (int)x, 0x4E, 0xF, 0xF, true));  // lane ^ 2
}

// Byte BYTE of `code` from the two elements in w.  (By value: a bit cast of an
// element of a vector takes the vector's first.)
template <int BYTE>
__device__ __forceinline__ unsigned pack_pair(unsigned code, unsigned w, float scale) {
  return __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(code, __builtin_bit_cast(bf16x2, w), scale, BYTE);
}

template <int D>
__global__ void __launch_bounds__(kThreads) cache4_write_kernel(Cache4Args a) {
  const Place p = place<D>(a);
  const uint16_t* src = a.rows[p.which] + p.bf16 * D + 8 * p.col;
  uint8_t* codes = a.codes[p.which] + p.cache * (D / 2) + 4 * p.col;
  uint8_t* scales = a.scales[p.which] + p.cache * (D / 32) + p.col / 4;
  constexpr int STEP = kThreads / (D / 8);
  u32x4 x[kSteps];
#pragma unroll
  for (int i = 0; i < kSteps; ++i) {
    const int r = p.row + i * STEP;
    x[i] = u32x4{};
    if (r < a.n_rows) x[i] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(src + (size_t)r * D));
  }
#pragma unroll
  for (int i = 0; i < kSteps; ++i) {
    const int r = p.row + i * STEP;
    // magnitudes of bf16 order as their bits do, infinities and NaN on top
    u16x2 top = {};
#pragma unroll
    for (int j = 0; j < 4; ++j)
      top = __builtin_elementwise_max(top, __builtin_bit_cast(u16x2, x[i][j] & 0x7FFF7FFFu));
    const unsigned m = quad_max(max(top[0], top[1]));
    const int b = min(max((int)((m + 31) >> 7) - 2, 7), 252);
    const float scale = __uint_as_float((unsigned)b << 23);
    unsigned code = 0;
    code = pack_pair<0>(code, x[i][0], scale);
    code = pack_pair<1>(code, x[i][1], scale);
    code = pack_pair<2>(code, x[i][2], scale);
    code = pack_pair<3>(code, x[i][3], scale);
    const bool bad = m >= 0x7F80u;  // an infinity or a NaN
    if (r < a.n_rows) {
      *reinterpret_cast<unsigned*>(codes + (size_t)r * (D / 2)) = bad ? 0u : code;
      if (p.col % 4 == 0) scales[(size_t)r * (D / 32)] = (uint8_t)(bad ? 255 : b);
    }
  }
}

template <int D>
__global__ void __launch_bounds__(kThreads) cache4_read_kernel(Cache4Args a) {
  const Place p = place<D>(a);
  uint16_t* dst = a.rows[p.which] + p.bf16 * D + 8 * p.col;
  const uint8_t* codes = a.codes[p.which] + p.cache * (D / 2) + 4 * p.col;
  const uint8_t* scales = a.scales[p.which] + p.cache * (D / 32) + p.col / 4;
  constexpr int STEP = kThreads / (D / 8);
  unsigned code[kSteps], b[kSteps];
#pragma unroll
  for (int i = 0; i < kSteps; ++i) {
    const int r = p.row + i * STEP;
    code[i] = b[i] = 0;
    if (r < a.n_rows) {
      code[i] = *reinterpret_cast<const unsigned*>(codes + (size_t)r * (D / 2));
      b[i] = scales[(size_t)r * (D / 32)];
    }
  }
#pragma unroll
  for (int i = 0; i < kSteps; ++i) {
    const int r = p.row + i * STEP;
    const float scale = __uint_as_float(b[i] << 23);  // b = 255: the conversions give NaN
    u32x4 y;
    y[0] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code[i], scale, 0));
    y[1] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code[i], scale, 1));
    y[2] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code[i], scale, 2));
    y[3] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code[i], scale, 3));
    if (r < a.n_rows) __builtin_nontemporal_store(y, reinterpret_cast<u32x4*>(dst + (size_t)r * D));
  }
}

}  // namespace

int64_t cache4_blocks(const Cache4Args& a) {
  const int64_t rb = rows_per_block(a.head_dim);
  return ((int64_t)a.n_rows + rb - 1) / rb * 2 * a.n_kv;
}

hipError_t launch_cache4_write(const Cache4Args& a, hipStream_t stream) {
  const dim3 grid((unsigned)cache4_blocks(a));
  if (a.head_dim == 128) hipLaunchKernelGGL((cache4_write_kernel<128>), grid, dim3(kThreads), 0, stream, a);
  else hipLaunchKernelGGL((cache4_write_kernel<64>), grid, dim3(kThreads), 0, stream, a);
  return hipGetLastError();
}

hipError_t launch_cache4_read(const Cache4Args& a, hipStream_t stream) {
  const dim3 grid((unsigned)cache4_blocks(a));
  if (a.head_dim == 128) hipLaunchKernelGGL((cache4_read_kernel<128>), grid, dim3(kThreads), 0, stream, a);
  else hipLaunchKernelGGL((cache4_read_kernel<64>), grid, dim3(kThreads), 0, stream, a);
  return hipGetLastError();
}

}  // namespace apb
