// The values of an e4m3 cache in bf16 (exact: scales are powers of two), for attention launches that read each of them often enough.
// HBM-bound, 6 bytes moved for each pair of K and V (about 6 TB/s, and 2 us a launch): a lane turns 16 codes of K and the 16 of V beside
// them into 32 bytes each.
#include "kvra_lowbit_device.h"

namespace kvra {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));

struct UnpackQ8Args {
  const u32x4* k;                // [rows, Hkv, D / 16]
  const u32x4* v;
  const unsigned char* k_scale;
  const unsigned char* v_scale;
  u32x4* k_out;                  // [rows, Hkv, D / 8]
  u32x4* v_out;
  long long pieces;              // rows Hkv D / 16
  unsigned Hkv;
  unsigned hidden_from;          // first row that a query does not see
};

template <int D>
__global__ __launch_bounds__(256) void unpack_q8_kernel(UnpackQ8Args a) {
  constexpr unsigned CPR = D / 16;
  const long long i = static_cast<long long>(blockIdx.x) * 256 + threadIdx.x;
  if (i >= a.pieces) return;                              // (the lanes of a row stay together)
  const unsigned long long line = static_cast<unsigned long long>(i) / CPR;   // row Hkv + head: below 2^32, see the launch
  const unsigned row = static_cast<unsigned>(line) / a.Hkv, head = static_cast<unsigned>(line) - row * a.Hkv;
  u32x4 codes[2] = {a.k[i], a.v[i]};
  const long long scale_at = static_cast<long long>(row / 64) * a.Hkv + head;
  const float factor[2] = {scale_factor(a.k_scale[scale_at]), scale_factor(a.v_scale[scale_at])};
  // A NaN in a row of V must not reach the queries it is hidden from (a weight of zero times NaN), nor be lost for those that see
  // it: it becomes a zero and its key's K NaN, and so the scores.
  unsigned bad = 0;
  if (row >= a.hidden_from) {
#pragma unroll
    for (int e = 0; e < 4; ++e) bad |= nan_bytes(codes[1][e]);
  }
#pragma unroll
  for (unsigned m = 1; m < CPR; m *= 2) bad |= __shfl_xor(bad, m);
  if (bad != 0) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      codes[0][e] = 0x7F7F7F7Fu;
      codes[1][e] &= ~((nan_bytes(codes[1][e]) >> 7) * 255u);
    }
  }
#pragma unroll
  for (int which = 0; which < 2; ++which) {
    u32x4 w[2];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      w[e / 2][2 * (e % 2)] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes[which][e], factor[which], false));
      w[e / 2][2 * (e % 2) + 1] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes[which][e], factor[which], true));
    }
    u32x4* const out = (which == 0 ? a.k_out : a.v_out) + 2 * i;
    out[0] = w[0];
    out[1] = w[1];
  }
}

int launch_unpack_q8(const Q8Cache& cache, int64_t rows, int64_t hidden_from, int n_kv_heads, int head_dim, void* k, void* v, hipStream_t stream) {
  UnpackQ8Args a;
  a.k = static_cast<const u32x4*>(cache.k);
  a.v = static_cast<const u32x4*>(cache.v);
  a.k_scale = static_cast<const unsigned char*>(cache.k_scale);
  a.v_scale = static_cast<const unsigned char*>(cache.v_scale);
  a.k_out = static_cast<u32x4*>(k);
  a.v_out = static_cast<u32x4*>(v);
  a.pieces = rows * n_kv_heads * (head_dim / 16);
  a.Hkv = static_cast<unsigned>(n_kv_heads);
  a.hidden_from = static_cast<unsigned>(hidden_from);
  if (rows * n_kv_heads > int64_t(0xFFFFFFFF) || (a.pieces + 255) / 256 > 0xFFFFFF) return KVRA_EUNSUPPORTED;
  const dim3 grid(static_cast<unsigned>((a.pieces + 255) / 256));
  return head_dim == 128 ? launch_kernel(unpack_q8_kernel<128>, grid, dim3(256), a, stream) : launch_kernel(unpack_q8_kernel<64>, grid, dim3(256), a, stream);
}

}  // namespace kvra
