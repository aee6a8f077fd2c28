// Attention over an e4m3 cache with a power-of-two scale for each block of 64 tokens and head, for launches of few rows: a
// token behind a long prompt, a follow-up turn, a short prompt.  The split of the work is that of the bf16 kernel for few rows
// (kvra_attn_rows.hip): a workgroup owns one slice of virtual rows (token * G + head in group), its eight waves share out the
// key tiles and meet at the end, workgroups that share a slice meet through the workspace.
//
// What bounds it: the cache is read once, as bytes.  A tile of 64 keys (which is one block of the cache: one scale each for K
// and V) goes from memory straight into the wave's own LDS, K and V 4 to 8 KB each, as it is; 64 to 128 KB per CU are on their
// way together.  K is read from there in operand order, V transposed (ds_read_b64_tr_b8), and both become bf16 in registers
// on the way to the matrix pipe, two values an instruction, scale included: exact, since a scale is a power of two.  (Half the
// LDS traffic and half the bytes in flight of bf16 tiles; the conversions, 128 a tile and wave at head_dim 128, overlap with the loads.)
// A slice is 16 rows where a head has no more - a token with up to 16 heads in a group - else 32.
//
// us on one MI355X, and those of the bf16 kernel over twice the bytes: 1 token behind 16383, 32 heads x 128: 33.6 over four caches in turn
// (4.0 TB/s; the same loads alone 27.7; as 256 heads behind 2047, without a merge, 29.5) and 54; 32 heads on 8: 14 and 25; 77 behind 5824, 32 on 8: 20 and 25; 160 tokens, 2 heads x 64: 5.0 and 5.1.  Of a short
// launch half is start, first trip to memory and merge.
// Tried: K straight to the fp8 matrix instruction, Q in two e4m3 parts that add up to it: half the conversions, the same loop times, and
// 1 us more ahead of the first tile (77 tokens 23 us).
//
// Roundings: Q is used as it came (the softmax scale goes onto the fp32 scores), P is rounded to bf16 for the product with V,
// the row sums add the unrounded fp32 weights.  P is rounded because it is an operand of the bf16 matrix instruction: in two bf16 parts it would
// take twice the products with V.  Against fp64 that is sqrt(2) times the error of rounding the output alone (2.3e-3 and 1.7e-3, relative 2-norm).
#include "kvra_attn_device.h"
#include "kvra_lowbit_device.h"

#include <algorithm>

namespace kvra {

constexpr int kQ8Waves = 8;
constexpr int kQ8Threads = 64 * kQ8Waves;

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
typedef int i32x2 __attribute__((ext_vector_type(2)));
typedef __attribute__((address_space(3))) i32x2 lds_i32x2;

struct RowsQ8Args {
  const __bf16* q;
  const unsigned char* k;
  const unsigned char* v;
  const unsigned char* k_scale;
  const unsigned char* v_scale;
  __bf16* out;
  int prefix;
  int chunk;
  int H;
  int Hkv;
  int G;
  int slices;        // slices of 16 QB virtual rows per kv head
  int splits;        // workgroups that share the key tiles of a slice
  float c_log2;      // scale * log2(e)
  float* partial;    // splits > 1: rows_q8_slot_floats(D, QB) per workgroup
  int* counters;     // splits > 1: pieces counted so far, one per slice; all zero between launches
};

constexpr int rows_q8_slot_floats(int D, int QB) { return D / 16 * QB * 4 * 64 + 32 * QB; }

template <int D, int QB>
__global__ __launch_bounds__(kQ8Threads, 2) void attn_rows_q8_kernel(RowsQ8Args a) {
  constexpr int BN = 64;                   // keys of a tile: a block of the cache
  constexpr int KB = BN / 16;              // 16-key blocks of a tile
  constexpr int CPR = D / 16;              // 16-byte pieces per K/V row
  constexpr int KS = D / 32;               // contraction steps of S^T = K Q^T
  constexpr int DB = D / 16;               // 16-row blocks of O^T
  constexpr int RPB = 256 / D;             // rows per 256-byte LDS bank span
  constexpr int TILE_BYTES = BN * D;
  constexpr int LOADS = TILE_BYTES / 1024; // wave loads per tile
  constexpr int RPL = 64 / CPR;            // rows one wave load moves
  constexpr int ROWS = 16 * QB;
  constexpr int R = DB * QB * 4;           // registers of O per lane
  constexpr int RW = R / kQ8Waves;         // of which a wave merges this many
  constexpr int RE = RW < 4 ? RW : 4;      // of one accumulator block
  constexpr int ML = 2 * ROWS;             // floats: m and l of the rows
  static_assert(R * 256 <= 2 * TILE_BYTES, "a wave's O takes the place of its tiles");
  // LDS: [wave][K tile, V tile], then [wave][m, l], then a flag
  extern __shared__ u32x4 smem[];
  char* const lds = reinterpret_cast<char*>(smem);
  float* const lds_ml = reinterpret_cast<float*>(lds + kQ8Waves * 2 * TILE_BYTES);
  int* const last_flag = reinterpret_cast<int*>(lds_ml + kQ8Waves * ML);

  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);   // wave-uniform by construction
  const int n = lane & 15, g4 = lane >> 4;

  // grid (kv heads, splits, slices), so that nothing has to be divided; ids go round-robin over the 8 XCDs, which so read apart by
  // head (27 against 29.5 us for the bytes of 16384 x 32 x 128 alone).  Last slices first: they see the most keys.
  const int g = blockIdx.x, split = blockIdx.y, slice = a.slices - 1 - static_cast<int>(blockIdx.z);

  const int VR = a.chunk * a.G, total = a.prefix + a.chunk;
  const int v0 = slice * ROWS, row_hi = min(v0 + ROWS, VR);
  // (a division is some 20 instructions, and a step of one token waits for each of them)
  auto token_of = [&](int vr) __attribute__((always_inline)) -> int { return a.chunk == 1 ? 0 : static_cast<int>(static_cast<unsigned>(vr) / static_cast<unsigned>(a.G)); };
  const int wmin = a.prefix + token_of(v0);             // last visible key of the slice's first and last row
  const int wmax = a.prefix + token_of(row_hi - 1);
  const int tiles = wmax / BN + 1;
  // (at most 2^19 tiles and 32 splits)
  const int t_lo = a.splits == 1 ? 0 : static_cast<int>(static_cast<unsigned>(tiles * split) / static_cast<unsigned>(a.splits));
  const int t_hi = a.splits == 1 ? tiles : static_cast<int>(static_cast<unsigned>(tiles * (split + 1)) / static_cast<unsigned>(a.splits));

  // Piece p = 64 i + lane of a tile = (row p / CPR, slot p % CPR); the lane that owns slot (row, slot) fetches column piece
  // slot ^ f(row), so that the reads below are free of bank conflicts: K is read 16 bytes a lane down 16 rows of one column
  // piece (f = row / RPB), V 8 bytes a lane over rows 4 g + {0..3} and 16 on of one piece (f also takes half of CPR in
  // every second group of 16 rows).  Only the offsets of the first load are kept: those of load i differ by an XOR and i row steps.
  const unsigned row_bytes = static_cast<unsigned>(a.Hkv) * D;
  const unsigned f_load = static_cast<unsigned>(lane / CPR / RPB);
  const unsigned off0 = static_cast<unsigned>(lane / CPR) * row_bytes + (static_cast<unsigned>(lane % CPR) ^ f_load) * 16;
  auto k_xor = [](int i) -> unsigned { return D == 128 ? 64u * (i & 1) : 0u; };
  auto v_xor = [](int i) -> unsigned { return D == 128 ? 64u * ((i ^ i >> 1) & 1) : 32u * (i & 1); };
  const unsigned lds_k = static_cast<unsigned>(reinterpret_cast<uintptr_t>((lds_void*)smem)) + wave * 2 * TILE_BYTES;
  const unsigned lds_v = lds_k + TILE_BYTES;
  const unsigned k_addr = lds_k + static_cast<unsigned>(n * CPR + (g4 ^ n / RPB % CPR)) * 16;
  // lane i of a 16-lane block names half of a row for the transposing read: row i / 2 of the eight {0..3, 16..19} + 4 g
  const int v_row = 4 * g4 + 16 * (n >> 3) + (n >> 1 & 3);
  const unsigned v_f = static_cast<unsigned>(v_row / RPB % CPR ^ (CPR / 2) * (v_row >> 4 & 1));
  const unsigned v_addr = lds_v + static_cast<unsigned>(v_row) * D + v_f * 16 + (n & 1) * 8;

  auto uniform = [](unsigned x) __attribute__((always_inline)) -> unsigned {
    return static_cast<unsigned>(__builtin_amdgcn_readfirstlane(static_cast<int>(x)));
  };
  auto load_tile = [&](const unsigned char* cache, int t, unsigned dst, auto xor_of) __attribute__((always_inline)) {
    const unsigned long long at = reinterpret_cast<unsigned long long>(cache + static_cast<long long>(g) * D) +
                                  static_cast<unsigned long long>(t) * BN * row_bytes;
    // to the end of the rows that exist: lanes beyond get zeros
    const u32x4 res = {uniform(static_cast<unsigned>(at)), uniform(static_cast<unsigned>(at >> 32) & 0xFFFFu),
                       uniform(min(total - t * BN, BN) * row_bytes - static_cast<unsigned>(g) * D), 0x00020000u};
    unsigned off = off0, step = RPL * row_bytes;
    asm volatile("" : "+v"(off), "+s"(step));   // (opaque, so that nothing is formed ahead and kept through the loop)
#pragma unroll
    for (int i = 0; i < LOADS; ++i) lds_dma16(res, (off ^ xor_of(i)) + i * step, dst + i * 1024);
  };

  // lane i holds the scales of this wave's next 64 tiles
  unsigned scales_k = 0, scales_v = 0;
  auto load_scales = [&](int from) __attribute__((always_inline)) {
    const long long tile = static_cast<long long>(from) + kQ8Waves * lane;
    if (tile < t_hi) {
      scales_k = a.k_scale[tile * a.Hkv + g];
      scales_v = a.v_scale[tile * a.Hkv + g];
    }
  };

  int t = t_lo + wave;
  if (t < t_hi) {
    load_tile(a.k, t, lds_k, k_xor);
    load_tile(a.v, t, lds_v, v_xor);
    load_scales(t);
  }

  // Q fragments: B operand of S^T.  The lanes of a 16-lane row g take pieces g and g + 4 of a key's row, so contraction
  // slots 8 g .. of step ks are components 16 (g + 4 (ks / 2)) + 8 (ks % 2) ..  Rows past the end repeat the last one.
  bf16x8 qf[KS][QB];
  int qpos[QB];
#pragma unroll
  for (int qb = 0; qb < QB; ++qb) {
    const int vr = min(v0 + 16 * qb + n, row_hi - 1), r = token_of(vr), h = g * a.G + (vr - r * a.G);
    qpos[qb] = a.prefix + r;
    const __bf16* qrow = a.q + (static_cast<long long>(r) * a.H + h) * D;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) qf[ks][qb] = *reinterpret_cast<const bf16x8*>(qrow + 16 * (g4 + 4 * (ks / 2)) + 8 * (ks % 2));
  }

  f32x4 o[DB][QB];
  float m[QB], l[QB];   // l: of this lane's quarter of the keys
#pragma unroll
  for (int qb = 0; qb < QB; ++qb) {
    m[qb] = kNoKeyYet;
    l[qb] = 0.0f;
#pragma unroll
    for (int db = 0; db < DB; ++db) o[db][qb] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  }

  // eight e4m3 codes -> bf16, times the block's scale
  auto dequant = [](unsigned lo, unsigned hi, float factor) __attribute__((always_inline)) -> bf16x8 {
    const bf16x2 x[4] = {__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, factor, false), __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, factor, true),
                         __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, factor, false), __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, factor, true)};
    return bf16x8{x[0][0], x[0][1], x[1][0], x[1][1], x[2][0], x[2][1], x[3][0], x[3][1]};
  };

  bool referenced = false;   // the wave's rows have an exponent reference (those that have met a visible key)
  for (int i = 0; t < t_hi; t += kQ8Waves, ++i) {
    const bool more = t + kQ8Waves < t_hi;
    if (i > 0 && (i & 63) == 0) load_scales(t);
    const float sk = scale_factor(static_cast<unsigned>(__builtin_amdgcn_readlane(static_cast<int>(scales_k), i & 63)));
    const float sv = scale_factor(static_cast<unsigned>(__builtin_amdgcn_readlane(static_cast<int>(scales_v), i & 63)));
    // the K tile has landed; the V tile sent for behind it may still be on its way
    asm volatile("s_waitcnt vmcnt(%0)" :: "n"(LOADS) : "memory");
    __builtin_amdgcn_sched_barrier(0);
    f32x4 s[KB][QB];
    unsigned ka = k_addr, va = v_addr;
    asm volatile("" : "+v"(ka), "+v"(va));
#pragma unroll
    for (int kb = 0; kb < KB; ++kb)
#pragma unroll
      for (int p = 0; p < KS / 2; ++p) {
        const u32x4 w = *(lds_u32x4*)static_cast<uintptr_t>((ka ^ 64u * p) + 16 * kb * D);
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          const bf16x8 kf = dequant(w[2 * half], w[2 * half + 1], sk);
#pragma unroll
          for (int qb = 0; qb < QB; ++qb)
            s[kb][qb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, qf[2 * p + half][qb], p + half == 0 ? f32x4{0.0f, 0.0f, 0.0f, 0.0f} : s[kb][qb], 0, 0, 0);
        }
      }
    // every read of this K tile is back before the next one is sent to its place
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    if (more) load_tile(a.k, t + kQ8Waves, lds_k, k_xor);

    auto wait_v = [&]() __attribute__((always_inline)) {   // V has landed; the next K may be on its way
      if (more) asm volatile("s_waitcnt vmcnt(%0)" :: "n"(LOADS) : "memory");
      else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
      __builtin_amdgcn_sched_barrier(0);
    };
    // register e of block (kb, qb) is key  t*BN + 16 kb + 4 g4 + e  of query 16 qb + n
    if (t * BN + BN - 1 > wmin) {
      if (wmin + 1 < total) {
        // A NaN in a row of V must not reach the rows it is hidden from (a weight of zero times NaN), nor be lost for those
        // that see it: it becomes a zero, and the scores of its key NaN.  Lane = key; one tile in 64 tokens comes here.
        wait_v();
        unsigned bad = 0;
#pragma unroll
        for (int i = 0; i < CPR; ++i) {
          const u32x4 w = *(lds_u32x4*)static_cast<uintptr_t>(lds_v + lane * D + (i ^ lane / RPB % CPR) * 16);
#pragma unroll
          for (int e = 0; e < 4; ++e) bad |= nan_bytes(w[e]);
        }
        const unsigned long long bad_keys = __builtin_amdgcn_ballot_w64(bad != 0);
        if (bad_keys != 0) {
          if (bad != 0)
            for (int i = 0; i < D / 4; ++i) {
              unsigned* const p = reinterpret_cast<unsigned*>(lds + wave * 2 * TILE_BYTES + TILE_BYTES + lane * D) + i;
              *p &= ~((nan_bytes(*p) >> 7) * 255u);
            }
#pragma unroll
          for (int kb = 0; kb < KB; ++kb)
#pragma unroll
            for (int e = 0; e < 4; ++e)
              if (bad_keys >> (16 * kb + 4 * g4 + e) & 1)
#pragma unroll
                for (int qb = 0; qb < QB; ++qb) s[kb][qb][e] = __builtin_nanf("");
          asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        }
      }
#pragma unroll
      for (int qb = 0; qb < QB; ++qb) {
        const int rel = qpos[qb] - t * BN - 4 * g4;   // largest still-visible key offset (minus 4 g4)
#pragma unroll
        for (int kb = 0; kb < KB; ++kb)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (16 * kb + e > rel) s[kb][qb][e] = -INFINITY;
      }
    }
    // Weights relative to the exponent reference in force, without looking for the largest score; where a lane's sum gets out of hand
    // (scores that outgrew the reference by about 2^20), and on the wave's first tile, the reference moves to the row's maximum,
    // what has been summed up follows, and the weights are formed again.
    u32x4 pf[KB / 2][QB];
    float psum[QB];
    for (bool again = false;;) {
      if (again || referenced) {
        bool out_of_hand = false;
#pragma unroll
        for (int qb = 0; qb < QB; ++qb) {
          psum[qb] = 0.0f;
#pragma unroll
          for (int kb = 0; kb < KB; ++kb)
#pragma unroll
            for (int e = 0; e < 4; e += 2) {
              const float p0 = __builtin_amdgcn_exp2f(fmaf(s[kb][qb][e], a.c_log2, -m[qb])), p1 = __builtin_amdgcn_exp2f(fmaf(s[kb][qb][e + 1], a.c_log2, -m[qb]));
              psum[qb] += p0 + p1;
              const bf16x2 pp = {static_cast<__bf16>(p0), static_cast<__bf16>(p1)};
              pf[kb / 2][qb][2 * (kb % 2) + e / 2] = __builtin_bit_cast(unsigned, pp);
            }
          out_of_hand |= !(psum[qb] < 1048576.0f);
        }
        if (again || __builtin_amdgcn_ballot_w64(out_of_hand) == 0) break;
      }
      again = referenced = true;
#pragma unroll
      for (int qb = 0; qb < QB; ++qb) {
        float tmax = s[0][qb][0];
#pragma unroll
        for (int kb = 0; kb < KB; ++kb)
#pragma unroll
          for (int e = 0; e < 4; ++e) tmax = fmaxf(tmax, s[kb][qb][e]);
        tmax = fmaxf(tmax, other_half(tmax));
        tmax = fmaxf(tmax, other_row(tmax));
        const float mn = fmaxf(m[qb], tmax * a.c_log2);    // a row that has met no visible key stays at kNoKeyYet: weights 0
        const float alpha = __builtin_amdgcn_exp2f(m[qb] - mn);
        m[qb] = mn;
        l[qb] *= alpha;
#pragma unroll
        for (int db = 0; db < DB; ++db)
#pragma unroll
          for (int e = 0; e < 4; ++e) o[db][qb][e] *= alpha;
      }
    }
#pragma unroll
    for (int qb = 0; qb < QB; ++qb) l[qb] += psum[qb];
    wait_v();
    // contraction slot 8 g4 + 4 b + u of step kk is key 32 kk + 16 b + 4 g4 + u on both operands
#pragma unroll
    for (int kk = 0; kk < KB / 2; ++kk)
#pragma unroll
      for (int db = 0; db < DB; ++db) {
        const i32x2 w = __builtin_amdgcn_ds_read_tr8_b64_v2i32((lds_i32x2*)static_cast<uintptr_t>((va ^ 16u * db) + 32 * kk * D));
        const bf16x8 vf = dequant(static_cast<unsigned>(w[0]), static_cast<unsigned>(w[1]), sv);
#pragma unroll
        for (int qb = 0; qb < QB; ++qb)
          o[db][qb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, __builtin_bit_cast(bf16x8, pf[kk][qb]), o[db][qb], 0, 0, 0);
      }
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    if (more) load_tile(a.v, t + kQ8Waves, lds_v, v_xor);
  }

  // ---- the eight waves' results meet in LDS: wave w merges registers RW w .. of all of them ------------------------
#pragma unroll
  for (int qb = 0; qb < QB; ++qb) {        // the whole row's sum, in each of the row's four lanes
    l[qb] += other_half(l[qb]);
    l[qb] += other_row(l[qb]);
    if (g4 == qb) {
      lds_ml[wave * ML + 16 * qb + n] = m[qb];
      lds_ml[wave * ML + ROWS + 16 * qb + n] = l[qb];
    }
  }
  float* const lds_o = reinterpret_cast<float*>(smem);   // [wave][register][lane]: a wave's own part lies in its own tiles
  constexpr int OS = 2 * TILE_BYTES / 4;                 // floats from wave to wave
#pragma unroll
  for (int i = 0; i < R; ++i) lds_o[wave * OS + i * 64 + lane] = o[i / (4 * QB)][i / 4 % QB][i % 4];
  __syncthreads();
  const int r0 = wave * RW;                              // register (db * QB + qb) * 4 + e
  constexpr int QW = (RW + 3) / 4 < QB ? 1 : QB;         // query blocks this wave's registers belong to
  static_assert(RW <= 4 * QW, "");
  const int qb0 = QW == QB ? 0 : r0 / 4 % QB;
  float acc[RW], am[QW], al[QW];
#pragma unroll
  for (int j = 0; j < QW; ++j) {
    const int row = 16 * (qb0 + j) + n;
    float mw[kQ8Waves];
    am[j] = kNoKeyYet;
    al[j] = 0.0f;
#pragma unroll
    for (int w = 0; w < kQ8Waves; ++w) {
      mw[w] = lds_ml[w * ML + row];
      am[j] = fmaxf(am[j], mw[w]);
    }
#pragma unroll
    for (int i = 0; i < RE; ++i) acc[RE * j + i] = 0.0f;
#pragma unroll
    for (int w = 0; w < kQ8Waves; ++w) {
      const float weight = __builtin_amdgcn_exp2f(mw[w] - am[j]);
      al[j] = fmaf(lds_ml[w * ML + ROWS + row], weight, al[j]);
#pragma unroll
      for (int i = 0; i < RE; ++i) acc[RE * j + i] = fmaf(lds_o[w * OS + (r0 + RE * j + i) * 64 + lane], weight, acc[RE * j + i]);
    }
  }

  if (a.splits > 1) {
    // device-coherent stores, acknowledged before the piece is counted; the piece that completes the count merges all of
    // them in their order, so the result does not depend on which one that is
    const int unit = g * a.slices + slice, live = row_hi - v0;   // (rows that are not there are neither stored nor merged)
    constexpr int SLOT = rows_q8_slot_floats(D, QB);
    float* const slots = a.partial + static_cast<long long>(unit) * a.splits * SLOT;
    float* const mine = slots + static_cast<long long>(split) * SLOT;
#pragma unroll
    for (int j = 0; j < QW; ++j)
      if (16 * (qb0 + j) + n < live)
#pragma unroll
        for (int i = 0; i < RE; ++i) store_coherent(mine + (r0 + RE * j + i) * 64 + lane, acc[RE * j + i]);
#pragma unroll
    for (int j = 0; j < QW; ++j)
      if (r0 < 4 * QB && g4 == 0 && 16 * (qb0 + j) + n < live) {         // the waves that hold the first of a query block's registers write its m and l
        store_coherent(mine + R * 64 + 16 * (qb0 + j) + n, am[j]);
        store_coherent(mine + R * 64 + ROWS + 16 * (qb0 + j) + n, al[j]);
      }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    if (tid == 0) *last_flag = atomicAdd(a.counters + unit, 1) == a.splits - 1 ? 1 : 0;
    __syncthreads();
    if (*last_flag == 0) return;
    if (tid == 0) a.counters[unit] = 0;     // ready for the next launch
#pragma unroll
    for (int j = 0; j < QW; ++j) {
      am[j] = kNoKeyYet;
      al[j] = 0.0f;
    }
#pragma unroll
    for (int i = 0; i < RW; ++i) acc[i] = 0.0f;
    // Where a 16-row block has few rows its 16 lanes share out the workgroups' results: lane n has row n % span and every 16 / span-th
    // result from n / span on, and they meet at the end.
    int log_span = 4;
    while (log_span > 0 && live <= 1 << (log_span - 1)) --log_span;
    const int span = 1 << log_span, row = n & (span - 1), shares = 16 >> log_span;
    constexpr int AHEAD = 8;                // of a lane's results on their way together
#pragma unroll 1
    for (int p0 = n >> log_span; p0 < a.splits; p0 += AHEAD * shares) {
      float pv[AHEAD][RW], pm[AHEAD][QW], pl[AHEAD][QW];
#pragma unroll
      for (int u = 0; u < AHEAD; ++u) {
        const float* p = slots + static_cast<long long>(min(p0 + u * shares, a.splits - 1)) * SLOT;
#pragma unroll
        for (int j = 0; j < QW; ++j) {
          const bool is_row = 16 * (qb0 + j) + row < live;
#pragma unroll
          for (int i = 0; i < RE; ++i) pv[u][RE * j + i] = is_row ? load_coherent(p + (r0 + RE * j + i) * 64 + 16 * g4 + row) : 0.0f;
          pm[u][j] = is_row ? load_coherent(p + R * 64 + 16 * (qb0 + j) + row) : kNoKeyYet;
          pl[u][j] = is_row ? load_coherent(p + R * 64 + ROWS + 16 * (qb0 + j) + row) : 0.0f;
        }
      }
#pragma unroll
      for (int u = 0; u < AHEAD; ++u)
#pragma unroll
        for (int j = 0; j < QW; ++j) {
          const bool there = p0 + u * shares < a.splits;   // (past the last it is loaded again, and weighs nothing)
          const float mn = there ? fmaxf(am[j], pm[u][j]) : am[j];
          const float wa = __builtin_amdgcn_exp2f(am[j] - mn), wb = there ? __builtin_amdgcn_exp2f(pm[u][j] - mn) : 0.0f;
          am[j] = mn;
          al[j] = fmaf(pl[u][j], wb, al[j] * wa);
#pragma unroll
          for (int i = 0; i < RE; ++i) acc[RE * j + i] = fmaf(there ? pv[u][RE * j + i] : 0.0f, wb, acc[RE * j + i] * wa);
        }
    }
#pragma unroll 1
    for (int step = span; step < 16; step *= 2)
#pragma unroll
      for (int j = 0; j < QW; ++j) {
        const float om = __shfl_xor(am[j], step), ol = __shfl_xor(al[j], step), mn = fmaxf(am[j], om);
        const float wa = __builtin_amdgcn_exp2f(am[j] - mn), wb = __builtin_amdgcn_exp2f(om - mn);
        am[j] = mn;
        al[j] = al[j] * wa + ol * wb;
#pragma unroll
        for (int i = 0; i < RE; ++i) acc[RE * j + i] = acc[RE * j + i] * wa + __shfl_xor(acc[RE * j + i], step) * wb;
      }
  }

  // register e of block (db, qb) is column 16 db + 4 g4 + e of row n
  typedef __bf16 out_t __attribute__((ext_vector_type(RE)));
#pragma unroll
  for (int j = 0; j < QW; ++j) {
    const int vr = v0 + 16 * (qb0 + j) + n, db = r0 / (4 * QB), e0 = r0 % 4;
    if (vr >= row_hi) continue;
    const int r = token_of(vr), h = g * a.G + (vr - r * a.G);
    const float inv = 1.0f / al[j];
    out_t w;
#pragma unroll
    for (int e = 0; e < RE; ++e) w[e] = static_cast<__bf16>(acc[RE * j + e] * inv);
    *reinterpret_cast<out_t*>(a.out + (static_cast<long long>(r) * a.H + h) * D + 16 * db + 4 * g4 + e0) = w;
  }
}

int64_t attn_rows_q8_slot_bytes(int head_dim, int rows) { return static_cast<int64_t>(rows_q8_slot_floats(head_dim, rows / 16)) * sizeof(float); }

int launch_attn_rows_q8(const Q8Cache& cache, const void* q, int64_t prefix_len, int64_t chunk_len, int n_q_heads, int n_kv_heads,
                        int head_dim, float scale, void* out, int rows, int splits, float* partial, int* counters,
                        hipStream_t stream) {
  RowsQ8Args a;
  a.q = static_cast<const __bf16*>(q);
  a.k = static_cast<const unsigned char*>(cache.k);
  a.v = static_cast<const unsigned char*>(cache.v);
  a.k_scale = static_cast<const unsigned char*>(cache.k_scale);
  a.v_scale = static_cast<const unsigned char*>(cache.v_scale);
  a.out = static_cast<__bf16*>(out);
  a.prefix = static_cast<int>(prefix_len);
  a.chunk = static_cast<int>(chunk_len);
  a.H = n_q_heads;
  a.Hkv = n_kv_heads;
  a.G = n_q_heads / n_kv_heads;
  a.slices = static_cast<int>((chunk_len * a.G + rows - 1) / rows);
  a.splits = splits;
  a.c_log2 = scale * 1.4426950408889634f;
  a.partial = partial;
  a.counters = counters;
  if (a.slices > 65535) return KVRA_EUNSUPPORTED;
  const dim3 grid(static_cast<unsigned>(n_kv_heads), static_cast<unsigned>(splits), static_cast<unsigned>(a.slices)), block(kQ8Threads);
  const unsigned smem = kQ8Waves * (2 * 64 * static_cast<unsigned>(head_dim) + 8u * static_cast<unsigned>(rows)) + 16u;   // tiles, m and l, flag
  if (head_dim == 128)
    return rows == 16 ? launch_kernel(attn_rows_q8_kernel<128, 1>, grid, block, a, stream, smem)
                      : launch_kernel(attn_rows_q8_kernel<128, 2>, grid, block, a, stream, smem);
  return rows == 16 ? launch_kernel(attn_rows_q8_kernel<64, 1>, grid, block, a, stream, smem)
                    : launch_kernel(attn_rows_q8_kernel<64, 2>, grid, block, a, stream, smem);
}

}  // namespace kvra
