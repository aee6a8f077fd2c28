// kvra_append_kv_q8: rotary embedding, and cache population in e4m3 with a power-of-two scale for each block of 64 tokens and
// head.  HBM-bound: K, V and Q are read once (2 bytes an element), K and V written as bytes.  5824 tokens of 32 heads x 128: 50 us, 4.8 TB/s
// (a large copy: 5.2); a token 4.6 us, a launch and two trips to memory.
//
// A block's scale needs the largest of its 64 x head_dim values before the first can be written, so a workgroup owns a
// (block, few heads) pair, holds a head's K and V rows of the block in registers (16 elements of each per thread) and meets
// once per head for the two maxima.  A thread keeps its token and its frequencies from head to head, so the angles are formed
// once per workgroup: two sets of 8 by angle addition (position = 8 i + o) instead of 64, in fp64, and stay in registers.
//
// K is rotated in fp64 and goes to fp32 by rounding to odd (a last bit that stands for everything below it), so that the one
// rounding to e4m3 is that of the exact product sums: with fp32 in between, one value in 10^5 lands on the other side of a tie.
//
// A chunk that starts inside a block finds rows there.  The block's scale then only grows, and where it does the rows are
// rescaled: by a power of two, which an e4m3 value takes without loss unless it falls below the smallest normal one.
#include "kvra_lowbit_device.h"
#include "kvra_rope_device.h"

namespace kvra {

typedef unsigned short u16x8 __attribute__((ext_vector_type(8)));
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));

struct AppendQ8Args {
  const unsigned short* k_in;
  const unsigned short* v_in;
  const unsigned short* q_in;   // may be null
  unsigned short* q_out;
  unsigned char* k_cache;
  unsigned char* v_cache;
  unsigned char* k_scale;
  unsigned char* v_scale;
  long long prefix_len;
  int chunk_len;
  int n_q_heads;
  int n_kv_heads;
  int use_rope;
  int heads_per_wg;             // kv heads a workgroup works through
  int head_groups;
  int kv_groups;                // workgroups [0, kv_groups) append, the others rotate Q
  int q_tokens;                 // tokens of one of those
  double inv_freq[64];
};

__device__ __forceinline__ float widen(unsigned short b) { return __uint_as_float(static_cast<unsigned>(b) << 16); }

__device__ __forceinline__ unsigned short round_bf16(float x) {
  const __bf16 b = static_cast<__bf16>(x);
  return __builtin_bit_cast(unsigned short, b);
}

// x in fp32, rounded to odd: cut to 24 bits, the last of which also stands for everything cut off, so that no later tie can
// fall on it.  In integers (fp64 instructions are slow): the bits from the exponent on are x's, moved by 29, its bias by 896.
__device__ __forceinline__ float round_odd(double x) {
  const unsigned long long bits = __builtin_bit_cast(unsigned long long, x);
  const unsigned lo = static_cast<unsigned>(bits), hi = static_cast<unsigned>(bits >> 32), mag = hi & 0x7FFFFFFFu;
  unsigned u = __builtin_amdgcn_alignbit(hi, lo, 29) + 0x40000000u;
  u |= min(lo & 0x1FFFFFFFu, 1u);
  if (mag - 0x38100000u >= 0x47F00000u - 0x38100000u)   // outside fp32's normal numbers: below them zero, above the largest, or not finite
    u = mag < 0x38100000u ? 0u : mag < 0x7FF00000u ? 0x7F7FFFFFu : 0x7FC00000u;
  return __uint_as_float(u | (hi & 0x80000000u));
}

__device__ __forceinline__ float finite_abs(float x) {
  const float a = fabsf(x);
  return a < INFINITY ? a : 0.0f;
}

// Finite values beyond the cache's largest, to that: a magnitude's bits rise with it.  (Only a block with the largest scale can meet one.)
__device__ __forceinline__ float within_cache(float x) {
  const unsigned u = __float_as_uint(x), mag = u & 0x7FFFFFFFu;
  return mag < 0x7F800000u ? __uint_as_float(min(mag, kCacheMost << 16) | (u & 0x80000000u)) : x;
}

__device__ __forceinline__ u16x8 within_cache(u16x8 b) {
#pragma unroll
  for (int e = 0; e < 8; ++e) b[e] = static_cast<unsigned short>(__float_as_uint(within_cache(widen(b[e]))) >> 16);
  return b;
}

__device__ __forceinline__ unsigned pack4(float a, float b, float c, float d) {
  unsigned r = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  return __builtin_amdgcn_cvt_pk_fp8_f32(c, d, r, true);
}

__device__ __forceinline__ u32x2 pack8(const float* x, float factor) {
  return u32x2{pack4(x[0] * factor, x[1] * factor, x[2] * factor, x[3] * factor), pack4(x[4] * factor, x[5] * factor, x[6] * factor, x[7] * factor)};
}

__device__ __forceinline__ u32x2 pack8(const u16x8& b, float factor) {
  const float x[8] = {widen(b[0]), widen(b[1]), widen(b[2]), widen(b[3]), widen(b[4]), widen(b[5]), widen(b[6]), widen(b[7])};
  return pack8(x, factor);
}

__device__ __forceinline__ unsigned rescale4(unsigned codes, float factor) {
  const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8(codes, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(codes, true);
  return pack4(lo[0] * factor, lo[1] * factor, hi[0] * factor, hi[1] * factor);
}

template <int D>
__global__ __launch_bounds__(4 * D) void append_q8_kernel(AppendQ8Args a) {
  constexpr int HALF = D / 2, NT = 4 * D, WAVES = NT / 64;
  constexpr int UNITS = D / 16;                    // units of 16 elements in a head row
  __shared__ double cos_s[2][8][HALF], sin_s[2][8][HALF];
  __shared__ float peak[2][2][WAVES];
  const int tid = threadIdx.x;

  if (static_cast<int>(blockIdx.x) >= a.kv_groups) {
    // ---- Q: as kvra_append_kv rotates it (fp32, one rounding to bf16)
    float* const cs = reinterpret_cast<float*>(&cos_s[0][0][0]);
    float* const sn = reinterpret_cast<float*>(&sin_s[0][0][0]);
    const long long tok0 = static_cast<long long>(blockIdx.x - a.kv_groups) * a.q_tokens;
    const int ntok = static_cast<int>(min(static_cast<long long>(a.q_tokens), a.chunk_len - tok0));
    if (a.use_rope && tid < ntok * HALF) rope_angle(static_cast<double>(a.prefix_len + tok0 + tid / HALF) * a.inv_freq[tid % HALF], cs + tid, sn + tid);
    __syncthreads();
    const int per_tok = a.n_q_heads * UNITS;
    for (int u = tid; u < ntok * per_tok; u += NT) {
      const int t = u / per_tok, rem = u - t * per_tok, j = rem % UNITS;
      const long long at = ((tok0 + t) * a.n_q_heads + rem / UNITS) * D + 8 * j;
      const u16x8 lo = *reinterpret_cast<const u16x8*>(a.q_in + at), hi = *reinterpret_cast<const u16x8*>(a.q_in + at + HALF);
      u16x8 olo = lo, ohi = hi;
      if (a.use_rope) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float c = cs[t * HALF + 8 * j + e], s = sn[t * HALF + 8 * j + e], x0 = widen(lo[e]), x1 = widen(hi[e]);
          olo[e] = round_bf16(fmaf(x0, c, -(x1 * s)));
          ohi[e] = round_bf16(fmaf(x1, c, x0 * s));
        }
      }
      *reinterpret_cast<u16x8*>(a.q_out + at) = olo;
      *reinterpret_cast<u16x8*>(a.q_out + at + HALF) = ohi;
    }
    return;
  }

  // ---- K and V of one block and a few heads
  const int block = blockIdx.x / a.head_groups, h0 = blockIdx.x % a.head_groups * a.heads_per_wg;
  const int h1 = min(h0 + a.heads_per_wg, a.n_kv_heads);
  const long long first = (a.prefix_len / 64 + block) * 64;           // the block's first row
  const int held = static_cast<int>(max(0LL, a.prefix_len - first));    // rows it holds already
  const int end = static_cast<int>(min(64LL, a.prefix_len + a.chunk_len - first));
  const int t = tid / UNITS, j = tid % UNITS;
  const bool fresh = t >= held && t < end;

  // A head's rows of the block, and the scales found: on their way while the angles, or the head before, are worked on.
  struct Rows {
    u16x8 lo, hi, v0, v1;
    int k_old, v_old;
  };
  auto load = [&](int h) __attribute__((always_inline)) -> Rows {
    Rows r;
    r.k_old = r.v_old = kScaleMin + 127;
    r.lo = r.hi = r.v0 = r.v1 = u16x8{};
    if (fresh) {
      const long long in_row = ((first + t - a.prefix_len) * a.n_kv_heads + h) * D;
      r.lo = *reinterpret_cast<const u16x8*>(a.k_in + in_row + 8 * j);
      r.hi = *reinterpret_cast<const u16x8*>(a.k_in + in_row + HALF + 8 * j);
      r.v0 = *reinterpret_cast<const u16x8*>(a.v_in + in_row + 16 * j);
      r.v1 = *reinterpret_cast<const u16x8*>(a.v_in + in_row + 16 * j + 8);
    }
    if (held > 0) {
      const long long scale_at = (first / 64) * a.n_kv_heads + h;
      r.k_old = a.k_scale[scale_at];
      r.v_old = a.v_scale[scale_at];
    }
    return r;
  };
  Rows now = load(h0);

  double c8[8], s8[8];
  if (a.use_rope) {
    const int row = tid / HALF, f = tid % HALF;
    const double freq = a.inv_freq[f];
    auto angle = [&](double position, int set) __attribute__((always_inline)) {
      const double phi = position * freq;
      double s, c;
      if (phi < 67108864.0) sincos_reduced(phi, &s, &c);
      else sincos(phi, &s, &c);
      cos_s[set][row][f] = c;
      sin_s[set][row][f] = s;
    };
    if (end - held <= 8) {                       // (a step's one token, a few: an angle each is all there is)
      angle(static_cast<double>(first + held + row), 0);
      __syncthreads();
      if (fresh) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          c8[e] = cos_s[0][t - held][8 * j + e];
          s8[e] = sin_s[0][t - held][8 * j + e];
        }
      }
    } else {
      angle(static_cast<double>(first + 8 * row), 0);
      angle(static_cast<double>(row), 1);
      __syncthreads();
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const double ca = cos_s[0][t / 8][8 * j + e], sa = sin_s[0][t / 8][8 * j + e], cb = cos_s[1][t % 8][8 * j + e], sb = sin_s[1][t % 8][8 * j + e];
        c8[e] = fma(ca, cb, -(sa * sb));
        s8[e] = fma(sa, cb, ca * sb);
      }
    }
  }

  for (int h = h0; h < h1; ++h) {
    const long long row = ((first + t) * a.n_kv_heads + h) * D;
    const long long scale_at = (first / 64) * a.n_kv_heads + h;
    u16x8 v0 = now.v0, v1 = now.v1;
    float k[16];
    float kmax = 0.0f, vmax = 0.0f;
    const int k_old = now.k_old - 127, v_old = now.v_old - 127;
    if (fresh) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float x0 = widen(now.lo[e]), x1 = widen(now.hi[e]);
        k[e] = x0;
        k[8 + e] = x1;
        if (a.use_rope) {
          const double d0 = x0, d1 = x1;
          k[e] = round_odd(fma(d0, c8[e], -(d1 * s8[e])));
          k[8 + e] = round_odd(fma(d1, c8[e], d0 * s8[e]));
        }
        kmax = fmaxf(kmax, fmaxf(fabsf(k[e]), fabsf(k[8 + e])));      // (fmaxf takes the number beside a NaN)
        vmax = fmaxf(vmax, fmaxf(fabsf(widen(v0[e])), fabsf(widen(v1[e]))));
      }
      if (!(fmaxf(kmax, vmax) < INFINITY)) {
        kmax = vmax = 0.0f;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          kmax = fmaxf(kmax, fmaxf(finite_abs(k[e]), finite_abs(k[8 + e])));
          vmax = fmaxf(vmax, fmaxf(finite_abs(widen(v0[e])), finite_abs(widen(v1[e]))));
        }
      }
    }
    if (h + 1 < h1) now = load(h + 1);
#pragma unroll
    for (int m = 1; m < 64; m *= 2) {
      kmax = fmaxf(kmax, __shfl_xor(kmax, m));
      vmax = fmaxf(vmax, __shfl_xor(vmax, m));
    }
    float (*const meet)[WAVES] = peak[(h - h0) & 1];
    if ((tid & 63) == 0) {
      meet[0][tid >> 6] = kmax;
      meet[1][tid >> 6] = vmax;
    }
    __syncthreads();
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
      kmax = fmaxf(kmax, meet[0][w]);
      vmax = fmaxf(vmax, meet[1][w]);
    }
    // (a scale byte outside the bounds is none that this kernel wrote: taken to the nearest that is)
    const int ke = max(scale_exponent<448>(kmax), min(k_old, kScaleMax)), ve = max(scale_exponent<448>(vmax), min(v_old, kScaleMax));
    if (t < held) {                            // 16 codes of a row that was there
      if (ke > k_old) {
        u32x4* const p = reinterpret_cast<u32x4*>(a.k_cache + row + 16 * j);
        const float factor = ldexpf(1.0f, k_old - ke);
        u32x4 w = *p;
#pragma unroll
        for (int e = 0; e < 4; ++e) w[e] = rescale4(w[e], factor);
        *p = w;
      }
      if (ve > v_old) {
        u32x4* const p = reinterpret_cast<u32x4*>(a.v_cache + row + 16 * j);
        const float factor = ldexpf(1.0f, v_old - ve);
        u32x4 w = *p;
#pragma unroll
        for (int e = 0; e < 4; ++e) w[e] = rescale4(w[e], factor);
        *p = w;
      }
    } else if (fresh) {
      const float kf = power_of_two(-ke), vf = power_of_two(-ve);
      if (__builtin_expect(ke == kScaleMax, 0)) {
#pragma unroll
        for (int e = 0; e < 16; ++e) k[e] = within_cache(k[e]);
      }
      if (__builtin_expect(ve == kScaleMax, 0)) {
        v0 = within_cache(v0);
        v1 = within_cache(v1);
      }
      *reinterpret_cast<u32x2*>(a.k_cache + row + 8 * j) = pack8(k, kf);
      *reinterpret_cast<u32x2*>(a.k_cache + row + HALF + 8 * j) = pack8(k + 8, kf);
      const u32x2 w0 = pack8(v0, vf), w1 = pack8(v1, vf);
      *reinterpret_cast<u32x4*>(a.v_cache + row + 16 * j) = u32x4{w0[0], w0[1], w1[0], w1[1]};
    }
    if (tid == 0) {
      a.k_scale[scale_at] = static_cast<unsigned char>(ke + 127);
      a.v_scale[scale_at] = static_cast<unsigned char>(ve + 127);
    }
  }
}

int launch_append_kv_q8(const void* k_in, const void* v_in, const void* q_in, void* q_out, void* k_cache, void* v_cache,
                        void* k_scale, void* v_scale, int64_t prefix_len, int64_t chunk_len, int n_q_heads, int n_kv_heads,
                        int head_dim, float rope_base, hipStream_t stream) {
  AppendQ8Args a;
  a.k_in = static_cast<const unsigned short*>(k_in);
  a.v_in = static_cast<const unsigned short*>(v_in);
  a.q_in = static_cast<const unsigned short*>(q_in);
  a.q_out = static_cast<unsigned short*>(q_out);
  a.k_cache = static_cast<unsigned char*>(k_cache);
  a.v_cache = static_cast<unsigned char*>(v_cache);
  a.k_scale = static_cast<unsigned char*>(k_scale);
  a.v_scale = static_cast<unsigned char*>(v_scale);
  a.prefix_len = prefix_len;
  a.chunk_len = static_cast<int>(chunk_len);
  a.n_q_heads = n_q_heads;
  a.n_kv_heads = n_kv_heads;
  a.use_rope = rope_base > 0.0f ? 1 : 0;
  const double* const inv = rope_frequencies(rope_base, head_dim);
  for (int i = 0; i < 64; ++i) a.inv_freq[i] = inv[i];
  const int64_t blocks = (prefix_len + chunk_len + 63) / 64 - prefix_len / 64;
  // heads per workgroup: up to 8 where a workgroup and a half per CU are left, so that the angles are formed less often (5824 tokens of
  // 32 x 128: 61.8 us with one, 52.4 with four, 50.0 with eight); a step of few blocks wants them all at once (1 token 4.6 and 16)
  int64_t per = blocks * n_kv_heads / 360;
  per = per < 1 ? 1 : per > 8 ? 8 : per;
  a.heads_per_wg = static_cast<int>(per);
  a.head_groups = static_cast<int>((n_kv_heads + per - 1) / per);
  const int64_t kv_groups = blocks * a.head_groups;
  // Q: tokens per workgroup, at most one angle per thread (8), fewer while the grid is small
  a.q_tokens = 8;
  while (a.q_tokens > 1 && (chunk_len + a.q_tokens - 1) / a.q_tokens < 1024) a.q_tokens >>= 1;
  const int64_t q_groups = q_in != nullptr && (q_in != q_out || a.use_rope) ? (chunk_len + a.q_tokens - 1) / a.q_tokens : 0;
  if (kv_groups + q_groups > INT32_MAX) return KVRA_EUNSUPPORTED;
  a.kv_groups = static_cast<int>(kv_groups);
  const dim3 grid(static_cast<unsigned>(kv_groups + q_groups)), block(static_cast<unsigned>(4 * head_dim));
  return head_dim == 128 ? launch_kernel(append_q8_kernel<128>, grid, block, a, stream)
                         : launch_kernel(append_q8_kernel<64>, grid, block, a, stream);
}

}  // namespace kvra
