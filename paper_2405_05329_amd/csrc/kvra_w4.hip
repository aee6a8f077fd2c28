// Linear layers with 4-bit weights:  out[m, n] = sum_k x[m, k] * w[n, k],  w = e2m1 value * 2^(scale of its group of 32 along k).
// The weights of a layer are most of what a token's step reads; at 4.25 bits they are 3.8 times less than in bf16.
// Products are those of kvra_linear on the same weights in bf16: an e2m1 value times a power of two is an exact bf16 number, and
// v_cvt_scalef32_pk_bf16_fp4 makes two of them, scale included, per instruction.
#include "kvra_attn_device.h"
#include "kvra_lowbit_device.h"

#include <algorithm>

namespace kvra {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef unsigned short u16x8 __attribute__((ext_vector_type(8)));

// ---- the format --------------------------------------------------------------------------------------------------------
struct PackW4Args {
  const unsigned short* w;       // [n, k] bf16
  unsigned* codes;               // [n, k / 8] words of eight codes, element 0 in the lowest four bits
  unsigned char* scales;         // [n, k / 32]
  long long words;               // n k / 8
};

// HBM-bound.  A lane has eight values (16 bytes in, 4 out), four neighbouring lanes a group: its largest value is found with two
// exchanges.  A group that holds an infinity or a NaN becomes NaN as a whole (scale 255): e2m1 has no code for either.
__global__ __launch_bounds__(256) void pack_w4_kernel(PackW4Args a) {
  const long long step = static_cast<long long>(gridDim.x) * 256;
  // (all lanes of a group are in or out together: words is a multiple of 4)
  for (long long i = static_cast<long long>(blockIdx.x) * 256 + threadIdx.x; i < a.words; i += step) {
    const u16x8 raw = *reinterpret_cast<const u16x8*>(a.w + 8 * i);
    float x[8], peak = 0.0f;
    bool finite = true;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      x[e] = __uint_as_float(static_cast<unsigned>(raw[e]) << 16);
      finite &= fabsf(x[e]) < INFINITY;
      peak = fmaxf(peak, fabsf(x[e]));
    }
    if (!finite) peak = INFINITY;
    peak = fmaxf(peak, __shfl_xor(peak, 1));
    peak = fmaxf(peak, __shfl_xor(peak, 2));
    const bool good = peak < INFINITY;
    const int e = good ? scale_exponent<6>(peak) : 128;
    unsigned word = 0;
    if (good) {
      const float factor = power_of_two(e);
      word = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(word, x[0], x[1], factor, 0);
      word = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(word, x[2], x[3], factor, 1);
      word = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(word, x[4], x[5], factor, 2);
      word = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(word, x[6], x[7], factor, 3);
    }
    a.codes[i] = word;
    if ((threadIdx.x & 3) == 0) a.scales[i / 4] = static_cast<unsigned char>(e + 127);
  }
}

// eight codes -> bf16, times the group's scale
__device__ __forceinline__ bf16x8 dequant8(unsigned word, float factor) {
  const bf16x2 x[4] = {__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(word, factor, 0), __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(word, factor, 1),
                       __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(word, factor, 2), __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(word, factor, 3)};
  return bf16x8{x[0][0], x[0][1], x[1][0], x[1][1], x[2][0], x[2][1], x[3][0], x[3][1]};
}

struct UnpackW4Args {
  const unsigned* codes;
  const unsigned char* scales;
  __bf16* w;
  long long words;
};

__global__ __launch_bounds__(256) void unpack_w4_kernel(UnpackW4Args a) {
  const long long step = static_cast<long long>(gridDim.x) * 256;
  for (long long i = static_cast<long long>(blockIdx.x) * 256 + threadIdx.x; i < a.words; i += step)
    *reinterpret_cast<bf16x8*>(a.w + 8 * i) = dequant8(a.codes[i], scale_factor(a.scales[i / 4]));
}

static unsigned stream_grid(int64_t words) { return static_cast<unsigned>(std::min<int64_t>((words + 255) / 256, 256 * 32)); }

int launch_pack_w4(const void* w, void* codes, void* scales, int64_t n, int64_t k, hipStream_t stream) {
  PackW4Args a{static_cast<const unsigned short*>(w), static_cast<unsigned*>(codes), static_cast<unsigned char*>(scales), n * k / 8};
  return launch_kernel(pack_w4_kernel, dim3(stream_grid(a.words)), dim3(256), a, stream);
}

int launch_unpack_w4(const void* codes, const void* scales, void* w, int64_t n, int64_t k, hipStream_t stream) {
  UnpackW4Args a{static_cast<const unsigned*>(codes), static_cast<const unsigned char*>(scales), static_cast<__bf16*>(w), n * k / 8};
  return launch_kernel(unpack_w4_kernel, dim3(stream_grid(a.words)), dim3(256), a, stream);
}

// ---- few tokens --------------------------------------------------------------------------------------------------------
struct LinearW4Args {
  const __bf16* x;               // [m, k]
  const unsigned char* w;        // [n, k / 2]
  const unsigned char* ws;       // [n, k / 32]
  const unsigned char* w2;       // SwiGLU: the up projection; else null
  const unsigned char* ws2;
  const __bf16* res;             // [m, n] or null
  __bf16* out;                   // [m, n]
  int m;
  int n;
  int k;
};

// Weights straight from memory into the A operand of v_mfma_f32_16x16x32_bf16: a lane loads 32 codes (16 bytes: one group of one
// row) and feeds them to four products, whose contraction slots are therefore components 32 g + 8 i .. of 128.  The waves of a
// workgroup share out k and meet in LDS.
template <bool DUAL, int RB, int TB, int WAVES>
__global__ __launch_bounds__(64 * WAVES) void linear_w4_rows_kernel(LinearW4Args a) {
  static_assert(!DUAL || RB % 2 == 0, "gate and up rows side by side");
  constexpr int OB = DUAL ? RB / 2 : RB;         // 16-row blocks of output columns
  extern __shared__ f32x4 sums[];                // [wave][row block][token block][lane]
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int r16 = lane & 15, g4 = lane >> 4;
  const int n0 = blockIdx.x * 16 * OB;
  const int tok0 = blockIdx.y * 16 * TB;
  const int chunks = (a.k + 127) / 128;
  const int c0 = chunks * wave / WAVES, c1 = chunks * (wave + 1) / WAVES;

  const unsigned char* w_row[RB];
  const unsigned char* s_row[RB];
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) {
    const long long row = n0 + 16 * (DUAL ? rb / 2 : rb) + r16;
    const bool up = DUAL && rb % 2 == 1;
    w_row[rb] = (up ? a.w2 : a.w) + row * (a.k / 2) + 16 * g4;
    s_row[rb] = (up ? a.ws2 : a.ws) + row * (a.k / 32) + g4;
  }
  const __bf16* x_row[TB];
#pragma unroll
  for (int tb = 0; tb < TB; ++tb) x_row[tb] = a.x + static_cast<long long>(min(tok0 + 16 * tb + r16, a.m - 1)) * a.k + 32 * g4;

  f32x4 acc[RB][TB];
#pragma unroll
  for (int rb = 0; rb < RB; ++rb)
#pragma unroll
    for (int tb = 0; tb < TB; ++tb) acc[rb][tb] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};

  for (int c = c0; c < c1; ++c) {
    u32x4 w[RB];
    unsigned s[RB];
    bf16x8 xf[TB][4];
    if (128 * c + 32 * g4 < a.k) {
#pragma unroll
      for (int rb = 0; rb < RB; ++rb) {
        w[rb] = *reinterpret_cast<const u32x4*>(w_row[rb] + 64 * static_cast<long long>(c));
        s[rb] = s_row[rb][4 * c];
      }
#pragma unroll
      for (int tb = 0; tb < TB; ++tb)
#pragma unroll
        for (int i = 0; i < 4; ++i) xf[tb][i] = *reinterpret_cast<const bf16x8*>(x_row[tb] + 128 * static_cast<long long>(c) + 8 * i);
    } else {                                     // behind the end of the rows
#pragma unroll
      for (int rb = 0; rb < RB; ++rb) {
        w[rb] = u32x4{0u, 0u, 0u, 0u};
        s[rb] = 127;
      }
#pragma unroll
      for (int tb = 0; tb < TB; ++tb)
#pragma unroll
        for (int i = 0; i < 4; ++i) xf[tb][i] = bf16x8{};
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int rb = 0; rb < RB; ++rb) {
        const bf16x8 wf = dequant8(w[rb][i], scale_factor(s[rb]));
#pragma unroll
        for (int tb = 0; tb < TB; ++tb) acc[rb][tb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wf, xf[tb][i], acc[rb][tb], 0, 0, 0);
      }
  }
#pragma unroll
  for (int rb = 0; rb < RB; ++rb)
#pragma unroll
    for (int tb = 0; tb < TB; ++tb) sums[((wave * RB + rb) * TB + tb) * 64 + lane] = acc[rb][tb];
  __syncthreads();

  // register e of a block is weight row 4 g4 + e of token r16
  for (int u = tid; u < OB * TB * 64; u += 64 * WAVES) {
    const int ln = u & 63, tb = u / 64 % TB, ob = u / 64 / TB;
    f32x4 y[DUAL ? 2 : 1];
#pragma unroll
    for (int j = 0; j < (DUAL ? 2 : 1); ++j) {
      y[j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int v = 0; v < WAVES; ++v) y[j] += sums[((v * RB + (DUAL ? 2 * ob + j : ob)) * TB + tb) * 64 + ln];
    }
    const int token = tok0 + 16 * tb + (ln & 15);
    if (token >= a.m) continue;
    const long long at = static_cast<long long>(token) * a.n + n0 + 16 * ob + 4 * (ln >> 4);
    f32x4 o = y[0];
    if constexpr (DUAL) {
#pragma unroll
      for (int e = 0; e < 4; ++e) o[e] = y[0][e] / (1.0f + __builtin_amdgcn_exp2f(-1.4426950408889634f * y[0][e])) * y[1][e];
    } else if (a.res != nullptr) {
      const bf16x4 r = *reinterpret_cast<const bf16x4*>(a.res + at);
#pragma unroll
      for (int e = 0; e < 4; ++e) o[e] += static_cast<float>(r[e]);
    }
    bf16x4 b;
#pragma unroll
    for (int e = 0; e < 4; ++e) b[e] = static_cast<__bf16>(o[e]);
    *reinterpret_cast<bf16x4*>(a.out + at) = b;
  }
}

// ---- many tokens -------------------------------------------------------------------------------------------------------
// MFMA-bound.  A wave owns 64 weight rows x 64 tokens: per 128 of k it converts 64 x 128 codes (64 conversions, on the vector
// pipe) for 64 matrix products.  Codes go from memory to registers in operand order as above, one stage ahead; tokens go to LDS
// (16 KB a stage, loaded straight to it, two stages), where the WN waves of a workgroup that have the same k share them.  WK waves share
// the k of a tile and meet in LDS at the end, so that a launch of few tiles still fills the chip.
constexpr int kTileStage = 64 * 256;      // bytes: 64 tokens x 128 of k

template <bool DUAL, int WN, int WK>
__global__ __launch_bounds__(64 * WN * WK, 2) void linear_w4_tile_kernel(LinearW4Args a) {
  constexpr int TK = 128;                 // k of a stage
  extern __shared__ u32x4 smem[];         // [wk][2 stages]; at the end the sums of the waves with wk > 0
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wn = wave % WN, wk = wave / WN;
  const int r16 = lane & 15, g4 = lane >> 4;
  constexpr int COLS = DUAL ? 32 : 64;    // output columns of a wave
  // ids go round-robin over the 8 XCDs: each takes a run of the order "token tile fastest"
  const int token_tiles = (a.m + 63) / 64, col_tiles = (a.n + COLS * WN - 1) / (COLS * WN), tiles = token_tiles * col_tiles;
  const int per = (tiles + 7) / 8, tile = (blockIdx.x & 7) * per + (blockIdx.x >> 3);
  if ((blockIdx.x >> 3) >= static_cast<unsigned>(per) || tile >= tiles) return;   // the whole workgroup
  const int tok0 = tile % token_tiles * 64, n0 = tile / token_tiles * (COLS * WN) + wn * COLS;

  const int stages_all = (a.k + TK - 1) / TK;
  const int s0 = stages_all * wk / WK, s1 = stages_all * (wk + 1) / WK, stages = (stages_all + WK - 1) / WK;   // (of the longest share)

  // weights: row blocks 0..3; SwiGLU: gate rows in 0 and 1, the same rows of up in 2 and 3.  Rows past the end repeat the last.
  const unsigned char* w_row[4];
  const unsigned char* s_row[4];
#pragma unroll
  for (int rb = 0; rb < 4; ++rb) {
    const bool up = DUAL && rb >= 2;
    const long long row = min(n0 + 16 * (DUAL ? rb % 2 : rb) + r16, a.n - 1);
    w_row[rb] = (up ? a.w2 : a.w) + row * (a.k / 2) + 16 * g4;
    s_row[rb] = (up ? a.ws2 : a.ws) + row * (a.k / 32) + g4;
  }
  u32x4 w[4];
  unsigned ws[4];
  auto load_w = [&](int st) __attribute__((always_inline)) {
    const bool in = TK * st + 32 * g4 < a.k;      // (the last stage of k = 64 mod 128 has half of it)
#pragma unroll
    for (int rb = 0; rb < 4; ++rb) {
      w[rb] = u32x4{0u, 0u, 0u, 0u};
      ws[rb] = 127;
      if (in) {
        w[rb] = *reinterpret_cast<const u32x4*>(w_row[rb] + 64 * static_cast<long long>(st));
        ws[rb] = s_row[rb][4 * st];
      }
    }
  };

  // tokens: a row of a stage is 16 pieces of 16 bytes; slot = piece ^ (row % 16), so that 16 rows of one piece meet no bank twice
  const unsigned long long x_at = reinterpret_cast<unsigned long long>(a.x) + static_cast<unsigned long long>(tok0) * a.k * 2;
  const unsigned long long x_left = static_cast<unsigned long long>(a.m - tok0) * a.k * 2;   // (below 4 GiB); beyond: zeros
  const u32x4 x_res = {static_cast<unsigned>(__builtin_amdgcn_readfirstlane(static_cast<int>(x_at))),
                       static_cast<unsigned>(__builtin_amdgcn_readfirstlane(static_cast<int>(x_at >> 32))) & 0xFFFFu,
                       static_cast<unsigned>(__builtin_amdgcn_readfirstlane(static_cast<int>(x_left))), 0x00020000u};
  const unsigned lds0 = static_cast<unsigned>(reinterpret_cast<uintptr_t>((lds_void*)smem)) + wk * 2 * kTileStage;
  constexpr int LOADS = 16 / WN;          // of this wave, 4 rows each
  const unsigned x_row = static_cast<unsigned>(4 * wn + (lane >> 4)) * a.k * 2, x_piece = static_cast<unsigned>((lane & 15) ^ (lane >> 4)) * 16;
  auto load_x = [&](int st) __attribute__((always_inline)) {
    unsigned row = x_row + static_cast<unsigned>(st) * 256, piece = x_piece, step = 4 * WN * static_cast<unsigned>(a.k) * 2;
    asm volatile("" : "+v"(row), "+v"(piece), "+s"(step));   // (opaque, so that nothing is formed ahead and kept)
#pragma unroll
    for (int i = 0; i < LOADS; ++i)
      lds_dma16(x_res, (piece ^ 64u * ((i * WN + wn) & 3)) + row + i * step, lds0 + (st & 1) * kTileStage + (i * WN + wn) * 1024);
  };
  unsigned x_addr[4];                     // of product i: token r16's piece 4 g4 + i
#pragma unroll
  for (int i = 0; i < 4; ++i) x_addr[i] = lds0 + r16 * 256 + ((4 * g4 + i) ^ r16) * 16;

  f32x4 acc[4][4];
#pragma unroll
  for (int rb = 0; rb < 4; ++rb)
#pragma unroll
    for (int tb = 0; tb < 4; ++tb) acc[rb][tb] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};

  if (s0 < s1) {
    load_x(s0);
    load_w(s0);
  }
  for (int j = 0; j < stages; ++j) {
    const int st = s0 + j;
    u32x4 wc[4];
    float wf[4];
#pragma unroll
    for (int rb = 0; rb < 4; ++rb) {
      wc[rb] = w[rb];
      wf[rb] = scale_factor(ws[rb]);
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();                      // the stage is there for all its waves, and all have read the one before
    if (st + 1 < s1) {
      load_x(st + 1);
      load_w(st + 1);
    }
    if (st < s1) {
      const unsigned slot = (st & 1) * kTileStage;
      const bool in = TK * st + 32 * g4 < a.k;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        bf16x8 x[4];
#pragma unroll
        for (int tb = 0; tb < 4; ++tb) {
          x[tb] = *(lds_bf16x8*)static_cast<uintptr_t>(x_addr[i] + slot + tb * 16 * 256);
          if (!in) x[tb] = bf16x8{};      // (what lies behind the end of a row belongs to the next token)
        }
#pragma unroll
        for (int rb = 0; rb < 4; ++rb) {
          const bf16x8 wx = dequant8(wc[rb][i], wf[rb]);
#pragma unroll
          for (int tb = 0; tb < 4; ++tb) acc[rb][tb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wx, x[tb], acc[rb][tb], 0, 0, 0);
        }
      }
    }
  }

  if constexpr (WK > 1) {
    __syncthreads();
    f32x4* const sums = reinterpret_cast<f32x4*>(smem);     // [wk - 1][wn][block][lane]
    if (wk > 0) {
#pragma unroll
      for (int b = 0; b < 16; ++b) sums[(((wk - 1) * WN + wn) * 16 + b) * 64 + lane] = acc[b / 4][b % 4];
    }
    __syncthreads();
    if (wk > 0) return;
#pragma unroll
    for (int v = 0; v < WK - 1; ++v)
#pragma unroll
      for (int b = 0; b < 16; ++b) acc[b / 4][b % 4] += sums[((v * WN + wn) * 16 + b) * 64 + lane];
  }

  // register e of a block is weight row 4 g4 + e of token r16
#pragma unroll
  for (int tb = 0; tb < 4; ++tb) {
    const int token = tok0 + 16 * tb + r16;
    if (token >= a.m) continue;
#pragma unroll
    for (int ob = 0; ob < COLS / 16; ++ob) {
      const int col = n0 + 16 * ob + 4 * g4;
      if (n0 + 16 * ob >= a.n) continue;
      const long long at = static_cast<long long>(token) * a.n + col;
      f32x4 o = acc[ob][tb];
      if constexpr (DUAL) {
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] = o[e] / (1.0f + __builtin_amdgcn_exp2f(-1.4426950408889634f * o[e])) * acc[ob + 2][tb][e];
      } else if (a.res != nullptr) {
        const bf16x4 r = *reinterpret_cast<const bf16x4*>(a.res + at);
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] += static_cast<float>(r[e]);
      }
      bf16x4 b;
#pragma unroll
      for (int e = 0; e < 4; ++e) b[e] = static_cast<__bf16>(o[e]);
      *reinterpret_cast<bf16x4*>(a.out + at) = b;
    }
  }
}

namespace {

template <bool DUAL, int RB, int TB, int WAVES>
int launch_rows(LinearW4Args& a, hipStream_t stream) {
  const int64_t tiles = (a.m + 16 * TB - 1) / (16 * TB);
  if (tiles > 65535) return KVRA_EUNSUPPORTED;
  return launch_kernel(linear_w4_rows_kernel<DUAL, RB, TB, WAVES>, dim3(static_cast<unsigned>(a.n / (DUAL ? 8 * RB : 16 * RB)), static_cast<unsigned>(tiles)),
                       dim3(64 * WAVES), a, stream, WAVES * RB * TB * 64u * 16u);
}

template <bool DUAL, int WN, int WK>
int launch_tile(LinearW4Args& a, hipStream_t stream) {
  const int64_t token_tiles = (a.m + 63) / 64, cols = (DUAL ? 32 : 64) * WN, tiles = token_tiles * ((a.n + cols - 1) / cols);
  const int64_t grid = (tiles + 7) / 8 * 8;
  if (grid > INT32_MAX) return KVRA_EUNSUPPORTED;
  const unsigned smem = std::max(WK * 2 * kTileStage, (WK - 1) * WN * 16 * 1024);
  return launch_kernel(linear_w4_tile_kernel<DUAL, WN, WK>, dim3(static_cast<unsigned>(grid)), dim3(64 * WN * WK), a, stream, smem);
}

template <bool DUAL>
int launch_many(LinearW4Args& a, hipStream_t stream) {
  const int64_t tiles = static_cast<int64_t>((a.m + 63) / 64) * ((a.n + (DUAL ? 31 : 63)) / (DUAL ? 32 : 64));   // of one wave
  if (tiles >= 4 * 384) return launch_tile<DUAL, 4, 1>(a, stream);
  if (tiles >= 2 * 256) return launch_tile<DUAL, 2, 2>(a, stream);
  return launch_tile<DUAL, 1, 4>(a, stream);
}

}  // namespace

int launch_linear_w4(const void* x, const void* w, const void* ws, const void* w2, const void* ws2, const void* residual, void* out,
                     int64_t m, int64_t n, int64_t k, hipStream_t stream) {
  LinearW4Args a;
  a.x = static_cast<const __bf16*>(x);
  a.w = static_cast<const unsigned char*>(w);
  a.ws = static_cast<const unsigned char*>(ws);
  a.w2 = static_cast<const unsigned char*>(w2);
  a.ws2 = static_cast<const unsigned char*>(ws2);
  a.res = static_cast<const __bf16*>(residual);
  a.out = static_cast<__bf16*>(out);
  a.m = static_cast<int>(m);
  a.n = static_cast<int>(n);
  a.k = static_cast<int>(k);
  if (m > 64) return w2 != nullptr ? launch_many<true>(a, stream) : launch_many<false>(a, stream);
  if (w2 != nullptr) return m <= 16 ? launch_rows<true, 2, 1, 8>(a, stream) : launch_rows<true, 2, 4, 8>(a, stream);
  return m <= 16 ? launch_rows<false, 1, 1, 8>(a, stream) : launch_rows<false, 1, 4, 8>(a, stream);
}

}  // namespace kvra
