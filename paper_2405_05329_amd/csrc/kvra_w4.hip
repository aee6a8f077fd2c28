// Linear layers with 4-bit weights:  out[m, n] = sum_k x[m, k] * w[n, k],  w = e2m1 value * 2^(scale of its group of 32 along k).
// The weights of a layer are most of what a token's step reads; at 4.25 bits they are 3.8 times less than in bf16.
// Products are those of kvra_linear on the same weights in bf16: an e2m1 value times a power of two is an exact bf16 number, and
// v_cvt_scalef32_pk_bf16_fp4 makes two of them, scale included, per instruction.
#include "kvra_attn_device.h"
#include "kvra_lowbit_device.h"

#include <algorithm>
#include <type_traits>

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

// HBM-bound (4096 x 11008 there and back 44.4 us, 5.1 TB/s).  A lane has eight values (16 bytes in, 4 out), four neighbouring lanes a group: its largest value is found with two
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
// Lanes of one wave hand data to each other through LDS.  The hardware carries out a wave's LDS operations in their order, so there is
// nothing to wait for; this holds the compiler to that order too (to which each lane's own stores and loads are unrelated).
__device__ __forceinline__ void wave_exchange() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

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

// HBM-bound, and before that bound by the address unit: in the order of the A operand of v_mfma_f32_16x16x32_bf16, 16 neighbouring
// lanes ask for 16 different rows, 64 lookups an instruction, and the weights came at 2.4 TB/s.  So four neighbouring lanes load
// 64 bytes of a row, 128 of k, and a buffer of the wave in LDS turns them into operand order (no workgroup barrier: see wave_exchange); the tokens go the same way, 256 bytes of a row to 16 lanes.  A lane's 16 bytes of codes are one group of one
// row and feed four products, whose contraction slots are components 32 g + 8 i .. of the 128.  The waves of a workgroup share out k
// and meet in LDS.  XL: loads of four tokens each.  1 token x 4096 x 4096: 3.7 us (bf16 weights 8.3); 12288 x 4096: 7.1 to 7.7, 3.5 TB/s (19.6);
// 13 tokens x 11008 x 4096, SwiGLU: 14 us (41.5).  Tried: more chunks ahead in fewer waves: slower.
template <bool DUAL, int RB, int TB, int XL, int WAVES>
__global__ __launch_bounds__(64 * WAVES) void linear_w4_rows_kernel(LinearW4Args a) {
  static_assert(!DUAL || RB % 2 == 0, "gate and up rows side by side");
  static_assert(XL <= 4 * TB, "");
  constexpr int OB = DUAL ? RB / 2 : RB;         // 16-row blocks of output columns
  constexpr int BUF = (RB + 4 * TB) * 64;        // 16-byte pieces of a wave's buffer: codes, tokens
  extern __shared__ u32x4 smem[];                // the waves' buffers; then [wave][row block][token block][lane]
  f32x4* const sums = reinterpret_cast<f32x4*>(smem);
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int r16 = lane & 15, g4 = lane >> 4;
  const int n0 = blockIdx.x * 16 * OB;
  const int tok0 = blockIdx.y * 16 * TB;
  const int chunks = (a.k + 127) / 128;
  const int c0 = chunks * wave / WAVES, c1 = chunks * (wave + 1) / WAVES;

  // loading: lane / 4 is the row of a block and lane % 4 the group of a chunk; for tokens lane / 16 and lane % 16.  Through buffer
  // resources: one lane-constant offset a block, the chunk's in a scalar register, zeros behind the last row.
  constexpr int MATS = DUAL ? 2 : 1;
  auto resource = [](const void* at, unsigned bytes) __attribute__((always_inline)) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(at), 0, static_cast<int>(bytes), 0x00020000);
  };
  const unsigned w_ld = static_cast<unsigned>(a.k) / 2, s_ld = static_cast<unsigned>(a.k) / 32, x_ld = static_cast<unsigned>(a.k) * 2;
  const __amdgpu_buffer_rsrc_t w_res[2] = {resource(a.w + static_cast<long long>(n0) * w_ld, 16 * OB * w_ld), resource((DUAL ? a.w2 : a.w) + static_cast<long long>(n0) * w_ld, 16 * OB * w_ld)};
  const __amdgpu_buffer_rsrc_t s_res[2] = {resource(a.ws + static_cast<long long>(n0) * s_ld, 16 * OB * s_ld), resource((DUAL ? a.ws2 : a.ws) + static_cast<long long>(n0) * s_ld, 16 * OB * s_ld)};
  const __amdgpu_buffer_rsrc_t x_res = resource(a.x + static_cast<long long>(tok0) * a.k, static_cast<unsigned>(a.m - tok0) * x_ld);
  const unsigned w_off = static_cast<unsigned>(lane >> 2) * w_ld + 16 * (lane & 3), s_off = static_cast<unsigned>(lane >> 2) * s_ld;
  const unsigned x_off = static_cast<unsigned>(lane >> 4) * x_ld + 16 * (lane & 15);
  // a chunk's four scales are a word, at an address that a load of one may have (the tensors are bound to 2 bytes only)
  const bool words = ((s_ld | static_cast<unsigned>(reinterpret_cast<uintptr_t>(a.ws)) | static_cast<unsigned>(reinterpret_cast<uintptr_t>(a.ws2))) & 3) == 0;
  struct Chunk {
    u32x4 w[RB], x[XL];
  };
  // (A chunk behind the wave's share is loaded and left; one behind the rows' end is the last again: a scalar offset has to stay inside
  // the resource, the lanes' offsets are compared with what is left of it.)
  auto load = [&](Chunk& b, int c) __attribute__((always_inline)) {
    c = min(c, chunks - 1);
#pragma unroll
    for (int rb = 0; rb < RB; ++rb)
      b.w[rb] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(w_res[rb % MATS], static_cast<int>(w_off + rb / MATS * 16 * w_ld), 64 * c, 0));
#pragma unroll
    for (int i = 0; i < XL; ++i)
      b.x[i] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(x_res, static_cast<int>(x_off + 4 * i * x_ld), 256 * c, 0));
  };
  // The four scales of chunk c + lane % 4 of a row.  (Behind the end of the row: the row's last, so that what the half chunk's
  // zeros are multiplied with is NaN only where the row is.)
  struct Four {
    unsigned lo, hi;
  };
  auto load_scales = [&](int rb, int c) __attribute__((always_inline)) -> Four {
    const int at = 4 * (c + (lane & 3)), row = static_cast<int>(s_off + rb / MATS * 16 * s_ld);
    if (words) return {__builtin_amdgcn_raw_buffer_load_b32(s_res[rb % MATS], row + min(at, static_cast<int>(s_ld) - 4), 0, 0), 0u};
    const int last = static_cast<int>(s_ld) - 2;   // (rows are an even number of bytes)
    return {__builtin_amdgcn_raw_buffer_load_b16(s_res[rb % MATS], row + min(at, last), 0, 0),
            __builtin_amdgcn_raw_buffer_load_b16(s_res[rb % MATS], row + min(at + 2, last), 0, 0)};
  };

  // the wave's buffer.  Slot of a row's piece: codes piece ^ f, f = 0, 3, 2, 1 for rows 0, 4, 8, 12 on; tokens piece ^ (row - 4) % 16: so
  // that the eight lanes that read in one cycle ({0..3, 12..15} of a 16-lane row with {4..11} of the next) meet no bank twice
  u32x4* const buf = smem + wave * BUF;
  const int w_put = (lane >> 2) * 4 + ((lane & 3) ^ (-(lane >> 4) & 3));
  const int x_put = (lane >> 4) * 16, x_get = RB * 64 + r16 * 16;
  const int w_get = r16 * 4 + (g4 ^ (-(r16 >> 2) & 3));

  f32x4 acc[RB][TB];
#pragma unroll
  for (int rb = 0; rb < RB; ++rb)
#pragma unroll
    for (int tb = 0; tb < TB; ++tb) acc[rb][tb] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  Chunk b;                                       // one chunk ahead: more waves on a CU beat more loads in a wave
  Four scales[RB];
  load(b, c0);
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) scales[rb] = load_scales(rb, c0);

  for (int c = c0; c < c1; c += 4) {
    Four next[RB];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      if (c + u >= c1) break;
      if (128 * (c + u) + 128 > a.k && (lane & 15) >= 8) {   // the half chunk: what follows is the next token's
#pragma unroll
        for (int i = 0; i < XL; ++i) b.x[i] = u32x4{0u, 0u, 0u, 0u};
      }
      wave_exchange();                           // the reads of the chunk before
#pragma unroll
      for (int rb = 0; rb < RB; ++rb) buf[rb * 64 + w_put] = b.w[rb];
#pragma unroll
      for (int i = 0; i < XL; ++i) buf[RB * 64 + i * 64 + x_put + ((lane & 15) ^ ((4 * i + (lane >> 4) - 4) & 15))] = b.x[i];
      load(b, c + u + 1);
      if (u == 0)
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) next[rb] = load_scales(rb, c + 4);
      wave_exchange();
      u32x4 w[RB];
      float factor[RB];
#pragma unroll
      for (int rb = 0; rb < RB; ++rb) {
        w[rb] = buf[rb * 64 + w_get];
        const unsigned four = static_cast<unsigned>(__builtin_amdgcn_ds_bpermute(4 * (4 * r16 + u), static_cast<int>(scales[rb].lo | scales[rb].hi << 16)));
        factor[rb] = scale_factor(four >> (8 * g4) & 255u);
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        bf16x8 x[TB];
#pragma unroll
        for (int tb = 0; tb < TB; ++tb) x[tb] = __builtin_bit_cast(bf16x8, buf[x_get + tb * 256 + ((4 * g4 + i) ^ ((r16 - 4) & 15))]);
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) {
          const bf16x8 wx = dequant8(w[rb][i], factor[rb]);
#pragma unroll
          for (int tb = 0; tb < TB; ++tb) acc[rb][tb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wx, x[tb], acc[rb][tb], 0, 0, 0);
        }
      }
    }
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) scales[rb] = next[rb];
  }
  __syncthreads();
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
// MFMA-bound.  A wave owns 64 weight rows x 64 tokens: per stage of 128 of k it converts 64 x 128 codes (64 conversions, on the
// vector pipe, beside the products) for 64 matrix products.  Codes and tokens go straight to LDS, the codes to the wave's own (4 KB a
// stage, two stages), the tokens to a ring of three stages of 16 KB that the four waves with the same k share.  A
// stage is 16 steps of four products; between them lie, each a step or more ahead of its use: one operand read, the conversion of one
// weight operand, the loads of the next stages, and the one barrier, past which a stage's reads begin three quarters of a stage later.
// WK groups of four waves share the k of a tile and meet in LDS at the end, so that one workgroup per CU has two waves per SIMD.
// 4096 x 4096 x 4096: 118 us, 1160 TFLOP/s (bf16 weights 108; without its loads 95); 777 x 4096 x 11008: 78 us (97).  Tried: the
// conversions between single products, equal; a ring that waits a stage later, 128 us.
constexpr int kTileStage = 64 * 256;      // bytes: 64 tokens x 128 of k
constexpr int kTileRing = 3;
constexpr int kTileCodes = 64 * 64;       // of a wave: 64 rows x 128 of k

template <bool DUAL, int WK>
__global__ __launch_bounds__(256 * WK, 2) void linear_w4_tile_kernel(LinearW4Args a) {
  constexpr int TK = 128, WN = 4;         // k of a stage; waves along the weight rows
  extern __shared__ u32x4 smem[];         // [wk][ring]; at the end the sums of the waves with wk > 0
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wn = wave % WN, wk = wave / WN;
  const int r16 = lane & 15, g4 = lane >> 4;
  constexpr int COLS = DUAL ? 32 : 64;    // output columns of a wave
  // ids go round-robin over the 8 XCDs: each takes a run of the order "bands of token tiles, in a band token tile fastest", so
  // that what an XCD runs together shares its tokens and weights in the L2
  const int token_tiles = (a.m + 63) / 64, col_tiles = (a.n + COLS * WN - 1) / (COLS * WN), tiles = token_tiles * col_tiles;
  const int per = (tiles + 7) / 8, tile = (blockIdx.x & 7) * per + (blockIdx.x >> 3);
  if ((blockIdx.x >> 3) >= static_cast<unsigned>(per) || tile >= tiles) return;   // the whole workgroup
  const int tall = token_tiles >= 32 ? 8 : 16;   // (4096 tokens x 4096 x 4096: 118.6 us in 16s, 114.7 in 8s; 777 x 4096 x 11008: 76.0 and 78.4)
  const int band = tile / (tall * col_tiles), in_band = tile - band * tall * col_tiles, high = min(tall, token_tiles - tall * band);
  const int tok0 = (tall * band + in_band % high) * 64, n0 = in_band / high * (COLS * WN) + wn * COLS;

  // this group's stages [s0, s1), of which the last of all may be half a one (k = 64 mod 128): `whole` stages and then that
  const int stages = (a.k + TK - 1) / TK;
  const int s0 = stages * wk / WK, s1 = stages * (wk + 1) / WK, whole = min(s1, a.k / TK) - s0, longest = (stages + WK - 1) / WK;

  // weights: row blocks 0..3; SwiGLU: gate rows in 0 and 1, the same rows of up in 2 and 3.  Rows past the end repeat the last.
  // Loads as in the kernel for few tokens, four neighbouring lanes to 64 bytes of a row, but straight to the wave's LDS (two stages);
  // scales by lane = row, 16 bytes for four stages, and from lane to lane.
  auto row_of = [&](int rb, int r) __attribute__((always_inline)) -> long long { return min(n0 + 16 * (DUAL ? rb % 2 : rb) + r, a.n - 1); };
  auto resource = [](const void* at, unsigned long long bytes) __attribute__((always_inline)) -> u32x4 {
    const unsigned long long p = reinterpret_cast<unsigned long long>(at);
    return u32x4{static_cast<unsigned>(__builtin_amdgcn_readfirstlane(static_cast<int>(p))),
                 static_cast<unsigned>(__builtin_amdgcn_readfirstlane(static_cast<int>(p >> 32))) & 0xFFFFu,
                 static_cast<unsigned>(__builtin_amdgcn_readfirstlane(static_cast<int>(bytes))), 0x00020000u};
  };
  const u32x4 w_res = resource(a.w, static_cast<unsigned long long>(a.n) * (a.k / 2)), w2_res = DUAL ? resource(a.w2, static_cast<unsigned long long>(a.n) * (a.k / 2)) : w_res;
  unsigned w_off[4];
#pragma unroll
  for (int rb = 0; rb < 4; ++rb) w_off[rb] = static_cast<unsigned>(row_of(rb, lane >> 2) * (a.k / 2)) + 16 * ((lane & 3) ^ (-(lane >> 4) & 3));
  const unsigned lds_w = static_cast<unsigned>(reinterpret_cast<uintptr_t>((lds_void*)smem)) + WK * kTileRing * kTileStage + wave * 2 * kTileCodes;
  auto load_w = [&](int rb, int st, unsigned half) __attribute__((always_inline)) {
    lds_dma16(DUAL && rb >= 2 ? w2_res : w_res, w_off[rb] + 64 * static_cast<unsigned>(st), lds_w + half + rb * 1024);
  };
  const unsigned w_addr = lds_w + r16 * 64 + (g4 ^ (-(r16 >> 2) & 3)) * 16;
  auto read_w = [&](int rb, unsigned half) __attribute__((always_inline)) -> u32x4 {
    return *(lds_u32x4*)static_cast<uintptr_t>(w_addr + half + rb * 1024);
  };
  const unsigned char* const s_row = (DUAL && lane >= 32 ? a.ws2 : a.ws) + row_of(lane >> 4, r16) * (a.k / 32);
  u32x4 scales, scales_next;
  auto load_scales = [&](int st) __attribute__((always_inline)) -> u32x4 {
    u32x4 v;
    __builtin_memcpy(&v, s_row + min(16 * (st >> 2), a.k / 32 - 16), 16);
    return v;
  };
  // the factor of row block rb in stage st: byte g4 of the four that lane 16 rb + r16 holds for the stage
  auto stage_scales = [&](const u32x4& v, int st) __attribute__((always_inline)) -> unsigned {
    const int at = 4 * st - min(16 * (st >> 2), a.k / 32 - 16);
    const unsigned lo = at & 8 ? (at & 4 ? v[3] : v[2]) : (at & 4 ? v[1] : v[0]), hi = at & 8 ? v[3] : (at & 4 ? v[2] : v[1]);
    return at & 2 ? lo >> 16 | hi << 16 : lo;    // (k = 64 mod 128: the last stages' begin between two words)
  };
  auto factor_of = [&](int rb, unsigned four) __attribute__((always_inline)) -> float {
    return scale_factor(static_cast<unsigned>(__builtin_amdgcn_ds_bpermute(4 * (16 * rb + r16), static_cast<int>(four))) >> (8 * g4) & 255u);
  };

  // tokens: a row of a stage is 16 pieces of 16 bytes; slot = piece ^ (row - 4) % 16, for the banks' sake
  const u32x4 x_res = resource(a.x + static_cast<long long>(tok0) * a.k, static_cast<unsigned long long>(a.m - tok0) * a.k * 2);   // beyond: zeros
  const unsigned lds0 = static_cast<unsigned>(reinterpret_cast<uintptr_t>((lds_void*)smem)) + wk * kTileRing * kTileStage;
  // load i of this wave: rows 16 i + 4 wn ..
  const unsigned x_row = static_cast<unsigned>(4 * wn + (lane >> 4)) * a.k * 2 +
                         (static_cast<unsigned>((lane & 15) ^ (lane >> 4)) * 16 ^ 64u * ((wn + 3) & 3)), x_step = 16 * static_cast<unsigned>(a.k) * 2;
  auto load_x = [&](int i, int st, unsigned slot) __attribute__((always_inline)) {
    lds_dma16(x_res, x_row + i * x_step + static_cast<unsigned>(st) * 256, lds0 + slot + (i * WN + wn) * 1024);
  };
  unsigned x_addr[4];                     // of product i: token r16's piece 4 g4 + i
#pragma unroll
  for (int i = 0; i < 4; ++i) x_addr[i] = lds0 + r16 * 256 + ((4 * g4 + i) ^ ((r16 - 4) & 15)) * 16;
  auto read_x = [&](int i, int tb, unsigned slot) __attribute__((always_inline)) -> bf16x8 {
    return *(lds_bf16x8*)static_cast<uintptr_t>(x_addr[i] + slot + tb * 16 * 256);
  };

  f32x4 acc[4][4];
#pragma unroll
  for (int rb = 0; rb < 4; ++rb)
#pragma unroll
    for (int tb = 0; tb < 4; ++tb) acc[rb][tb] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};

  u32x4 w[2][4];
  float f[2][4];
  bf16x8 x[2][4], wx[2];
  unsigned slot = 0, slot1 = kTileStage, slot2 = 2 * kTileStage;   // of this stage's tokens, the next one's, those after
  if (s0 < s1) {
    scales = load_scales(s0);
    scales_next = load_scales(min(s0 + 4, s1 - 1));
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      load_x(i, s0, slot);
      load_x(i, min(s0 + 1, s1 - 1), slot1);
      load_w(i, s0, 0);
      load_w(i, min(s0 + 1, s1 - 1), kTileCodes);
    }
  }
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[0][i] = read_x(0, i, slot);
    w[0][i] = read_w(i, 0);
    f[0][i] = factor_of(i, stage_scales(scales, s0));
  }
  wx[0] = dequant8(w[0][0][0], f[0][0]);

  // One whole stage, the H-th of a pair: its weights are in w[H]; the next one's are read to the other.
  auto stage = [&](int st, auto half_tag) __attribute__((always_inline)) {
    constexpr int H = decltype(half_tag)::value;
    constexpr unsigned HERE = H * kTileCodes, OTHER = kTileCodes - HERE;
    const int st1 = min(st + 1, s1 - 1), st2 = min(st + 2, s1 - 1);   // (past the end: loaded again, to where nobody looks)
    unsigned four = 0;
#pragma unroll
    for (int q = 0; q < 16; ++q) {
      const int i = q / 4, rb = q % 4;
      __builtin_amdgcn_sched_barrier(0);
      x[(i + 1) % 2][rb] = i < 3 ? read_x(i + 1, rb, slot) : read_x(0, rb, slot1);
      if (q == 10) four = stage_scales(scales, st1);
      if (q >= 11 && q < 15) {
        if (q == 11) asm volatile("s_waitcnt vmcnt(8)" ::: "memory");   // the next stage's codes: all but this stage's loads
        w[1 - H][q - 11] = read_w(q - 11, OTHER);
        f[1 - H][q - 11] = factor_of(q - 11, four);
      }
      const int q1 = (q + 1) % 16, from = q < 15 ? H : 1 - H;
      wx[q1 % 2] = dequant8(w[from][q1 % 4][q1 / 4], f[from][q1 % 4]);
      if (q == 1) {   // every wave of the group is done with the stage before, and the next one's tokens are there
        asm volatile("s_waitcnt vmcnt(4)" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        // (The wait for this drains what was sent before it: here that is the next stage's codes alone.)
        if ((st1 & 3) == 0 && st1 != st) {
          scales = scales_next;
          scales_next = load_scales(min(st1 + 4, s1 - 1));
        }
      }
      if (q >= 2 && q < 6) load_x(q - 2, st2, slot2);
      if (q >= 6 && q < 10) load_w(q - 6, st2, HERE);
#pragma unroll
      for (int tb = 0; tb < 4; ++tb) acc[rb][tb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wx[q % 2], x[i % 2][tb], acc[rb][tb], 0, 0, 0);
    }
    __builtin_amdgcn_sched_barrier(0);
    const unsigned done = slot;
    slot = slot1;
    slot1 = slot2;
    slot2 = done;
  };
  int j = 0;
  for (; j + 2 <= whole; j += 2) {
    stage(s0 + j, std::integral_constant<int, 0>{});
    stage(s0 + j + 1, std::integral_constant<int, 1>{});
  }
  if (j < whole) {
    stage(s0 + j, std::integral_constant<int, 0>{});
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      w[0][i] = w[1][i];
      f[0][i] = f[1][i];
    }
    ++j;
  }
  for (int b = j; b < longest; ++b) __builtin_amdgcn_s_barrier();     // (as many barriers for every group)
  if (whole < s1 - s0) {                  // the half stage
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int tb = 0; tb < 4; ++tb) {
        // what lies behind the end of a row belongs to the next token
        const bf16x8 xt = g4 < 2 ? read_x(i, tb, slot) : bf16x8{};
#pragma unroll
        for (int rb = 0; rb < 4; ++rb)
          acc[rb][tb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(dequant8(g4 < 2 ? w[0][rb][i] : 0u, g4 < 2 ? f[0][rb] : 1.0f), xt,
                                                                acc[rb][tb], 0, 0, 0);
      }
  }

  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
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

template <bool DUAL, int RB, int TB, int XL, int WAVES>
int launch_rows(LinearW4Args a, hipStream_t stream) {
  constexpr int64_t MOST = 65535 * int64_t(16 * TB);     // tokens of a launch: a grid's second dimension ends there
  for (int64_t left = a.m; left > 0; left -= MOST) {
    a.m = static_cast<int>(std::min(left, MOST));
    const int rc = launch_kernel(linear_w4_rows_kernel<DUAL, RB, TB, XL, WAVES>,
                                 dim3(static_cast<unsigned>(a.n / (DUAL ? 8 * RB : 16 * RB)), static_cast<unsigned>((a.m + 16 * TB - 1) / (16 * TB))),
                                 dim3(64 * WAVES), a, stream, WAVES * (RB + 4 * TB) * 1024u);
    if (rc != KVRA_OK) return rc;
    a.x += MOST * a.k;
    a.out += MOST * a.n;
    if (a.res != nullptr) a.res += MOST * a.n;
  }
  return KVRA_OK;
}

template <bool DUAL>
int launch_few(LinearW4Args& a, hipStream_t stream) {
  constexpr int RB = DUAL ? 2 : 1;
  if (a.m <= 4) return launch_rows<DUAL, RB, 1, 1, 8>(a, stream);
  if (a.m <= 16) return launch_rows<DUAL, RB, 1, 4, 8>(a, stream);
  if (a.m <= 32) return launch_rows<DUAL, 2, 2, 8, 8>(a, stream);
  return launch_rows<DUAL, 2, 4, 16, 8>(a, stream);
}

template <bool DUAL, int WK>
int launch_tile(LinearW4Args& a, hipStream_t stream) {
  const int64_t token_tiles = (a.m + 63) / 64, cols = DUAL ? 128 : 256, tiles = token_tiles * ((a.n + cols - 1) / cols);
  const int64_t grid = (tiles + 7) / 8 * 8;
  if (grid > INT32_MAX) return KVRA_EUNSUPPORTED;
  return launch_kernel(linear_w4_tile_kernel<DUAL, WK>, dim3(static_cast<unsigned>(grid)), dim3(256 * WK), a, stream,
                       WK * (kTileRing * kTileStage + 4 * 2 * kTileCodes));
}

// Which kernel.  Both take about k times a constant per round of workgroups on the chip's 256 CUs, whatever the round holds: the
// one for few tokens, 32 rows (SwiGLU 16) x 64 tokens a workgroup, 2.45 us per 1000 of k; the other, 256 rows (128) x 64 tokens, 7.0 us
// with two groups of waves along k and one workgroup a CU, 12.5 us with one group and two workgroups a CU.  Timed on 100 shapes, n 1024 to
// 12288, k 1024 to 11008, 40 to 1500 tokens; 4096 x 4096 (in a graph): 128 tokens 12.1 us here, 30.9 there; 300 tokens 29.8 and 31.0; 512 tokens
// 40.1 and 32.0.
template <bool DUAL>
int launch_any(LinearW4Args& a, hipStream_t stream) {
  const int64_t token_tiles = (a.m + 63) / 64, tiles = token_tiles * ((a.n + (DUAL ? 127 : 255)) / (DUAL ? 128 : 256));
  const int64_t few_rounds = (token_tiles * (a.n / (DUAL ? 16 : 32)) + 255) / 256;
  const double few = 2.45 * static_cast<double>(few_rounds), many = tiles <= 256 ? 7.0 : 12.5 * static_cast<double>((tiles + 511) / 512);
  if (a.m <= 64 || a.k < 512 || few <= many) return launch_few<DUAL>(a, stream);
  return tiles <= 256 ? launch_tile<DUAL, 2>(a, stream) : launch_tile<DUAL, 1>(a, stream);
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
  return w2 != nullptr ? launch_any<true>(a, stream) : launch_any<false>(a, stream);
}

}  // namespace kvra
