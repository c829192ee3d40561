// Attention of a few queries a sequence over the paged 4-bit cache.
//
// The mathematics.  With codes u, scales s and zeros z of a token j and group n of 64 channels
//     q . k_j = sum_n s_jn (sum_c q_c u_jc) + z_jn (sum_c q_c)          c over the channels of group n
//     sum_j p_j v_jc = sum_j (p_j s_jn) u_jc + sum_j p_j z_jn
// so the tensor cores multiply by the codes, which are small integers and exact in fp16, and scales and zeros are applied to a
// score or a weight, once a group instead of once a channel.  A nibble becomes fp16 by one AND: with the other bits zero it is the
// subnormal u 2^-24, or 16 u 2^-24 for a nibble four bits up; the powers of two come back in the row's factor.  Four ANDs and a
// shift unpack eight values.
//
// Layout.  mma.m16n8k16 with 16 tokens (S^T = K Q^T) and then 16 channels (O^T = V^T P^T) as its rows and 8 query rows as its
// columns: the rows of a group's heads and of several new tokens share what is read.  The cache holds K and V in the order of the A
// operand, so a lane's operands are single 16-byte reads, and S^T becomes P^T by movmatrix in registers.  mma.sync and not
// tcgen05: the operands have to pass through registers to be unpacked, and 8 columns are all there is to multiply by.
//
// Work.  Segments (sequence, head, tile of 8 rows) stand one behind the other in steps of 32 tokens, each with what beginning and
// ending it costs, and are dealt out in equal shares to all warps, whatever the lengths, which are read on the device.  (Tiles are counted
// from seq_q, not from each sequence's queries: those that have no rows take shares and do nothing with them.)  A warp goes
// through its share alone, with a ring of bulk copies of its own and no barrier, and writes the rows of segments that lie within
// it.  Pieces of a segment in several warps of a CTA meet in shared memory, parts of one in several CTAs in global memory: the CTA
// that ends the segment waits for the others' and puts them together in their order, so that the result does not depend on timing.
//
// What bounds it (B200, 296 CTAs of 8 warps): large batches the memory, at 4.5 bits a value, with about 545 instructions a warp
// and step beside it (of which 160 unpack and 32 are products): 64 sequences of 2K to 32K tokens, 826 MB, in 143 to 156 us, 0.81
// to 0.88 of the measured copy rate (164 us where the power limit holds).  Small ones the latency of what follows one another: slot,
// length, page, copy (6 us until the first products), the pieces' meeting (2 to 3 us), the joining of parts (2 to 4 us): 8 x 6001
// tokens in 22.7 us, of which the memory takes 8.5.
//
// Exactness.  Scores, statistics and sums are in 32 bits; Q is exact in fp16 after a power of two per row (what lies 2^-28 below a
// row's largest entry is rounded).  P times a group's scale is rounded to fp16: 2^-11 of each product, against 2^-8 of the bf16 result.  The
// power of two that keeps these products in fp16's range is a row's own, for each group of channels, and comes from the products and not from the
// scales: a loud value that the row does not see or hardly weighs takes nothing from the others (one power for all rows, from the
// scales: values of 1e-4 beside an unseen one of 65504 were off by 13 %).  The row's reference is a maximum, rounded up to a whole number, that is
// renewed only when a score exceeds it by 6 in the exponent of 2.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "sm100_ptx.cuh"
#include "steel_cache.cuh"
#include "steel_cache_wait.cuh"

namespace steel {

namespace {

constexpr int kStepTokens = 32;
// Sixteen warps an SM with 128 registers a thread, 8 query rows a tile.  Unpacking K and V once for 16 rows was slower at any number of rows
// (16 sequences of 12 to 40 rows: 24.7 against 28.8 us with 8 x 20 rows at head_dim 64, 36.9 against 43 at 128): it takes twice the registers of the sums,
// and with half the warps too little latency is hidden.
constexpr int kWarps = 8, kThreads = kWarps * 32, kCtasPerSm = 2, kRows = 8;
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr float kMostWeight = 64.f;      // how far a weight may exceed 1 before the reference is renewed
constexpr float kMostProduct = 32768.f;  // the same for weights times scales, which are to be fp16 numbers
// log2 of a row's power of two before its first product, and at most: the smallest scale with a weight of 2^-25 exceeds kMostProduct, and zeros
// that have joined the sums stay in range
constexpr int kMostDown = 64;
constexpr int kSegmentCost = 2;        // what beginning and ending a segment costs, in steps
constexpr float kFloor = -3e38f;       // the reference before any key has been seen: below any score

// n / divisor for 0 <= n < 2^31 by a multiplication.
struct FastDivisor {
  uint32_t divisor, factor, shift;
};
FastDivisor fast_divisor(int d) {
  uint32_t log = 0;
  while ((1ll << log) < d) ++log;
  return FastDivisor{uint32_t(d), d == 1 ? 0u : uint32_t(((1ull << (31 + log)) + d - 1) / d), log - 1};
}
__device__ __forceinline__ int divide(int n, const FastDivisor &d) {
  return d.divisor == 1 ? n : int(__umulhi(uint32_t(n), d.factor) >> d.shift);
}

struct AttendKernelParams {
  CacheView c;
  CacheBatch b;
  Rows q;
  __nv_bfloat16 *o;
  float *lse;
  float *parts;      // [grid][rows][head_dim], then reference and sum of each row: a segment's part in a CTA that does not end it
  uint64_t *flags;   // [grid][rows]: `token` once the row is there
  uint64_t token;    // of this launch alone
  long long wait_cycles;  // the bound of a wait for another CTA's part
  int32_t group, seq_q, row_tiles, window, mask;
  float scale_log2;
  FastDivisor by_group, by_row_tiles, by_warps;
};

// one part: rows x (unnormalised O, reference, sum)
__host__ __device__ constexpr int64_t part_floats(int rows, int head_dim) { return int64_t(rows) * (head_dim + 2); }

__device__ __forceinline__ void mma(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma_first(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                          uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%10, %10, %10, %10};"
      : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.f));
}
__device__ __forceinline__ uint32_t transpose8x8(uint32_t a) {
  uint32_t d;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(d) : "r"(a));
  return d;
}
__device__ __forceinline__ uint32_t pack_half2(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}
__device__ __forceinline__ float2 half2_of(uint32_t w) { return __half22float2(*reinterpret_cast<__half2 *>(&w)); }

// 2^e for -126 <= e <= 127
__device__ __forceinline__ float pow2(int e) { return __int_as_float((e + 127) << 23); }
// floor(log2 x) of a normal positive number
__device__ __forceinline__ int exponent(float x) { return (__float_as_int(x) >> 23) - 127; }

// a / b for powers of two whose quotient is a normal number
__device__ __forceinline__ float over(float a, float b) {
  return __int_as_float(__float_as_int(a) - __float_as_int(b) + (127 << 23));
}

// by shared-memory addresses
__device__ __forceinline__ void bulk_load(uint32_t dst, uint64_t src, uint32_t bytes, uint32_t bar) {
  asm volatile("cp.async.bulk.shared::cta.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst), "l"(src),
               "r"(bytes), "r"(bar)
               : "memory");
}
__device__ __forceinline__ void mbar_expect(uint32_t bar, uint32_t bytes) {
  asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}

// The whole warp waits for a phase, about two seconds at most; the clock is looked at once in 64 polls.
__device__ __forceinline__ bool test_full(uint32_t bar, uint32_t parity) {
  uint32_t ok;
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
      "selp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(ok)
      : "r"(bar), "r"(parity)
      : "memory");
  return ok != 0;
}
__device__ __forceinline__ bool wait_full(uint32_t bar, uint32_t parity) {
  long long since = 0;
  for (uint32_t polls = 1; !__all_sync(0xffffffffu, test_full(bar, parity)); ++polls) {
    if ((polls & 63) == 0) {
      const long long now = clock64();
      if (since == 0) since = now;
      if (__any_sync(0xffffffffu, now - since > kWaitCycles)) return false;
    }
  }
  return true;
}

// The value of lane 0, which the compiler then knows to be the same in all lanes: branches on it need no code for warps that part.
__device__ __forceinline__ int uniform(int x) { return __shfl_sync(0xffffffffu, x, 0); }

// A sequence of the batch: where its tokens are and which steps of 32 tokens its queries see.
struct Sequence {
  int slot, len, count, step_lo, steps;  // steps = 0: no queries
};
// What the device finds for sequence b: slot (-1: none), count and length; then checked and made safe.
__device__ __forceinline__ Sequence read_sequence(const AttendKernelParams &p, int b) {
  Sequence s;
  s.slot = slot_of(p.c, p.b.slots, b);
  s.count = p.b.counts ? p.b.counts[b] : p.seq_q;
  s.len = p.c.lens[max(s.slot, 0)];
  return s;
}
__device__ __forceinline__ bool check_sequence(const AttendKernelParams &p, Sequence &s) {
  const bool good = s.slot >= 0 && s.count >= 0 && s.count <= p.seq_q && s.len >= 0 && s.len <= max_tokens(p.c);
  if (!good) {
    s.slot = max(s.slot, 0);
    s.count = min(max(s.count, 0), p.seq_q);
    s.len = 0;
  }
  const int first = p.mask & STEEL_MASK_WINDOW ? max(0, s.len - s.count - p.window + 1) : 0;
  s.step_lo = first / kStepTokens;
  const int end = (s.len + kStepTokens - 1) / kStepTokens;
  s.steps = s.count == 0 ? 0 : max(1, end - s.step_lo);  // a sequence without keys still has rows to write
  return good;
}

// Keys [lo, hi) that the query at position pos sees.
__device__ __forceinline__ int key_hi(const AttendKernelParams &p, int len, int pos) {
  return p.mask & STEEL_MASK_CAUSAL ? min(len, pos + 1) : len;
}
__device__ __forceinline__ int key_lo(const AttendKernelParams &p, int pos) {
  return p.mask & STEEL_MASK_WINDOW ? pos - p.window + 1 : INT32_MIN;
}

// A warp's ring of steps, and the shared memory of a CTA: the rings, then a place for one piece a warp.
template <int D>
struct Shared {
  static constexpr int kStages = D == 128 ? 2 : 4;  // a power of two
  static constexpr int kStepBytes = 2 * unit_bytes(D), kRingBytes = kStages * kStepBytes;
  static constexpr int kPitch = D + 8;  // floats a row of a piece: 16-byte stores of a warp then miss one another's banks
  static constexpr int kPieceBytes = kRows * kPitch * 4;
  static constexpr int kBytes = kWarps * (kRingBytes + kPieceBytes);
  static_assert(kPieceBytes <= kRingBytes, "a piece lies over its warp's ring");
};

// What a warp holds of a segment: queries as B operands, sums, statistics.
template <int D>
struct Rolling {
  static constexpr int NG = D / kGroup, NC = D / 32;
  uint32_t qf[NC][4];
  float qsum[2][NG], factor[2];  // of this lane's columns, rows 2t and 2t + 1
  float acc[NG][4][4];               // O^T: group, nibble, (channel 8g + i, row 2t), (.., 2t + 1), (8g + 4 + i, 2t), ..
  float zero_sum[2][NG];             // this lane's part of sum_j p_j z_jn, since it last joined acc
  float ref[2], sum[2];          // reference; this lane's part of the sum of weights
  float down[2][NG];                 // a power of two that the row's weights times scales are multiplied by
};

// A warp's place in the work: rows row0 ... row0 + rows - 1 (of the group's heads, position by position) and their keys.
struct Tile {
  int len, pos0, row0, rows;  // pos0: position of the first query
  int any_lo, any_hi;         // keys that some row sees; those that all do
  int all_lo, all_hi;
};

// Reads of shared memory by 32-bit addresses: a register and a constant offset.  Volatile, so that they stay behind the waits.
template <int kOffset>
__device__ __forceinline__ uint4 lds128(uint32_t at) {
  uint4 w;
  asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4 + %5];" : "=r"(w.x), "=r"(w.y), "=r"(w.z), "=r"(w.w) : "r"(at), "n"(kOffset));
  return w;
}
template <int kOffset>
__device__ __forceinline__ void load_pairs(uint32_t at, uint32_t (&sz)[2][2]) {
  const uint4 w = lds128<kOffset>(at);
  sz[0][0] = w.x, sz[0][1] = w.y, sz[1][0] = w.z, sz[1][1] = w.w;
}
template <int kOffset>
__device__ __forceinline__ void load_pairs(uint32_t at, uint32_t (&sz)[2][1]) {
  asm volatile("ld.shared.v2.b32 {%0, %1}, [%2 + %3];" : "=r"(sz[0][0]), "=r"(sz[1][0]) : "r"(at), "n"(kOffset));
}
__device__ __forceinline__ void load_floats(float (&x)[4], const float *src) {
  const float4 v = __ldcg(reinterpret_cast<const float4 *>(src));
  x[0] = v.x, x[1] = v.y, x[2] = v.z, x[3] = v.w;
}
__device__ __forceinline__ void load_floats(float (&x)[2], const float *src) {
  const float2 v = __ldcg(reinterpret_cast<const float2 *>(src));
  x[0] = v.x, x[1] = v.y;
}
__device__ __forceinline__ float max_over_warp(float x) {
#pragma unroll
  for (int bit = 1; bit <= 16; bit <<= 1) x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, bit));
  return x;
}
__device__ __forceinline__ float sum_over_warp(float x) {
#pragma unroll
  for (int bit = 1; bit <= 16; bit <<= 1) x += __shfl_xor_sync(0xffffffffu, x, bit);
  return x;
}
__device__ __forceinline__ float max_over_g(float x) {
  x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 4));
  x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 8));
  return fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 16));
}
__device__ __forceinline__ float sum_over_g(float x) {
  x += __shfl_xor_sync(0xffffffffu, x, 4);
  x += __shfl_xor_sync(0xffffffffu, x, 8);
  return x + __shfl_xor_sync(0xffffffffu, x, 16);
}

// Queries of a tile: row n = g of each tile of 8, channels 32c + 8t ... + 7.
template <int D>
__device__ __forceinline__ void load_queries(const AttendKernelParams &p, int b, int head, const Tile &tile, int lane,
                                             uint4 (&raw)[D / 32]) {
  const unsigned char *src = p.q.data + b * p.q.batch + (lane % 4) * 16;
  const int row = tile.row0 + lane / 4, pos = divide(row, p.by_group);
  const unsigned char *at = src + (head * p.group + row - pos * p.group) * p.q.head + pos * p.q.seq;
#pragma unroll
  for (int c = 0; c < D / 32; ++c)
    raw[c] = lane / 4 < tile.rows ? *reinterpret_cast<const uint4 *>(at + 64 * c) : make_uint4(0, 0, 0, 0);
}

// Queries -> B operands, their sums by group, the rows' factors.
template <int D>
__device__ __forceinline__ void unpack_queries(float scale_log2, const uint4 (&raw)[D / 32], int lane, Rolling<D> &r) {
  constexpr int NG = D / kGroup, NC = D / 32;
  const int t = lane % 4;
  uint32_t big = 0;  // largest magnitude, as bits
#pragma unroll
  for (int c = 0; c < NC; ++c)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t w = (&raw[c].x)[i];
      big = max(big, max(w & 0x7fffu, (w >> 16) & 0x7fffu));
    }
  big = max(big, __shfl_xor_sync(0xffffffffu, big, 1));
  big = max(big, __shfl_xor_sync(0xffffffffu, big, 2));
  // the power of two that brings it to 2^14 ... 2^15 (subnormal ones to less)
  const int up = big == 0 ? 0 : min(14 + 127 - int(big >> 7), 126);
  const float unit = pow2(up);
  float sum[NG];
#pragma unroll
  for (int n = 0; n < NG; ++n) sum[n] = 0.f;
#pragma unroll
  for (int c = 0; c < NC; ++c) {
    float v[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t w = (&raw[c].x)[i];
      v[2 * i] = __uint_as_float(w << 16) * unit;
      v[2 * i + 1] = __uint_as_float(w & 0xffff0000u) * unit;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) sum[c / 2] += v[i];
    // nibbles (0, 4), (1, 5), (2, 6), (3, 7) of a K word; the odd ones stand four bits higher
    r.qf[c][0] = pack_half2(v[0], v[4]);
    r.qf[c][1] = pack_half2(v[1] * 0.0625f, v[5] * 0.0625f);
    r.qf[c][2] = pack_half2(v[2], v[6]);
    r.qf[c][3] = pack_half2(v[3] * 0.0625f, v[7] * 0.0625f);
  }
#pragma unroll
  for (int n = 0; n < NG; ++n) {
    sum[n] += __shfl_xor_sync(0xffffffffu, sum[n], 1);
    sum[n] += __shfl_xor_sync(0xffffffffu, sum[n], 2);
    sum[n] *= pow2(-24);  // in the units of the products with codes
  }
  // in two steps: 2^(24 - up) alone may leave the range
  const float f = fmaxf(scale_log2 * pow2(min(24 - up, 64)) * pow2(max(24 - up - 64, 0)), 1.2e-38f);  // not 0: what is masked is -inf
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    r.factor[j] = __shfl_sync(0xffffffffu, f, (2 * t + j) * 4);
#pragma unroll
    for (int n = 0; n < NG; ++n) r.qsum[j][n] = __shfl_sync(0xffffffffu, sum[n], (2 * t + j) * 4);
  }
}

template <int D>
__device__ __forceinline__ void clear(Rolling<D> &r) {
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    r.ref[j] = kFloor;
    r.sum[j] = 0.f;
#pragma unroll
    for (int n = 0; n < D / kGroup; ++n) {
      r.zero_sum[j][n] = 0.f;
      r.down[j][n] = pow2(kMostDown);
    }
  }
#pragma unroll
  for (int n = 0; n < D / kGroup; ++n)
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) r.acc[n][i][e] = 0.f;
}

// A step: two units of 16 tokens, keys key0 ...  `at` and `at_scales`: shared-memory addresses of the lane's part of the codes and of
// its scales.  `partial`: some row of the tile does not see some key of the step.  Both units go through each stage together: their products
// and exponentials do not wait for one another, and one vote is enough.
template <int D>
__device__ __forceinline__ void attend_step(const AttendKernelParams &p, uint32_t at, uint32_t at_scales, bool partial, int key0,
                                            const Tile &tile, int lane, Rolling<D> &r) {
  constexpr int NG = D / kGroup, UB = unit_bytes(D);
  const int g = lane / 4, t = lane % 4;
  // scores
  float score[2][4];  // [unit]: (token g, row 2t), (g, 2t + 1), (8 + g, 2t), ..
#pragma unroll
  for (int u = 0; u < 2; ++u) {
    float dot[NG][4];
#pragma unroll
    for (int n = 0; n < NG; ++n) {
      const uint4 w = u == 0 ? n == 0 ? lds128<0>(at) : lds128<512>(at) : n == 0 ? lds128<UB>(at) : lds128<UB + 512>(at);
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        uint32_t lo = c ? w.z : w.x, hi = c ? w.w : w.y;
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          const uint32_t *q = &r.qf[2 * n + c][2 * k];
          if (c == 0 && k == 0)
            mma_first(dot[n], lo & 0x000f000fu, hi & 0x000f000fu, lo & 0x00f000f0u, hi & 0x00f000f0u, q[0], q[1]);
          else
            mma(dot[n], lo & 0x000f000fu, hi & 0x000f000fu, lo & 0x00f000f0u, hi & 0x00f000f0u, q[0], q[1]);
          lo >>= 8;
          hi >>= 8;
        }
      }
    }
    uint32_t sz[2][NG];  // (scale, zero) of tokens g and 8 + g
    if (u == 0) load_pairs<NG * 1024>(at_scales, sz);
    else load_pairs<UB + NG * 1024>(at_scales, sz);
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int n = 0; n < NG; ++n) {
        const float2 pair = half2_of(sz[h][n]);
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const float zero = n == 0 ? pair.y * r.qsum[j][n] : fmaf(pair.y, r.qsum[j][n], score[u][2 * h + j]);
          score[u][2 * h + j] = fmaf(pair.x, dot[n][2 * h + j], zero);
        }
      }
  }
  // scales of V
  float vs[2][2][NG], vz[2][2][NG];
#pragma unroll
  for (int u = 0; u < 2; ++u) {
    uint32_t sz[2][NG];
    if (u == 0) load_pairs<NG * 1088>(at_scales, sz);
    else load_pairs<UB + NG * 1088>(at_scales, sz);
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int n = 0; n < NG; ++n) {
        const float2 pair = half2_of(sz[h][n]);
        vs[u][h][n] = pair.x;
        vz[u][h][n] = pair.y;
      }
  }
  if (partial) {
    // Some row does not see some of the keys.  What a row does not see must not reach it even where it is no number: scores
    // become -inf, and scales that are none are taken out here and counted for the rows that do see them.
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int key = key0 + 16 * u + 8 * h + g;
        const bool any = key >= tile.any_lo && key < tile.any_hi;
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const int row = 2 * t + j, pos = tile.pos0 + divide(tile.row0 + row, p.by_group);
          const bool seen = any && row < tile.rows && key >= key_lo(p, pos) && key < key_hi(p, tile.len, pos);
          if (!seen) score[u][2 * h + j] = -INFINITY;
#pragma unroll
          for (int n = 0; n < NG; ++n)
            if (seen && !(fabsf(vs[u][h][n]) + fabsf(vz[u][h][n]) <= 3e38f)) r.zero_sum[j][n] = NAN;
        }
#pragma unroll
        for (int n = 0; n < NG; ++n)
          if (!any || !(fabsf(vs[u][h][n]) + fabsf(vz[u][h][n]) <= 3e38f)) vs[u][h][n] = vz[u][h][n] = 0.f;
      }
  }
  // weights, and times scales in fp16 as B operands; is a reference or a power of two to be renewed?
  float w[2][4], top = 0.f, top_product = 0.f;
  uint32_t pb[2][NG][2];
#pragma unroll
  for (int u = 0; u < 2; ++u) {
#pragma unroll
    for (int e = 0; e < 4; ++e) w[u][e] = ex2_approx(fmaf(score[u][e], r.factor[e & 1], -r.ref[e & 1]));
    top = fmax3(top, w[u][0], w[u][1]);
    top = fmax3(top, w[u][2], w[u][3]);
#pragma unroll
    for (int n = 0; n < NG; ++n) {
      float product[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) product[e] = w[u][e] * r.down[e & 1][n] * vs[u][e / 2][n];
      top_product = fmax3(top_product, product[0], product[1]);
      top_product = fmax3(top_product, product[2], product[3]);
      pb[u][n][0] = pack_half2(product[0], product[1]);
      pb[u][n][1] = pack_half2(product[2], product[3]);
    }
  }
  if (__any_sync(0xffffffffu, top > kMostWeight || top_product > kMostProduct)) {
    // A row's new reference is a whole number, the largest score so far rounded up.  Its power of two follows, so that a value whose weight has
    // become small leaves the room to others; then, if a product is still too large, it is the one that brings the largest of this step
    // to 2^5 ... 2^6: room for later ones to be 2^9 times as large, and a product of 2^-19 of it is a normal number in fp16.
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const float most = fmaxf(fmaxf(score[0][j], score[0][2 + j]), fmaxf(score[1][j], score[1][2 + j]));
      const float now = fmaxf(r.ref[j], ceilf(max_over_g(most * r.factor[j]))), rise = now - r.ref[j], shrink = ex2_approx(-rise);
      r.ref[j] = now;
      r.sum[j] *= shrink;
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int h = 0; h < 2; ++h) w[u][2 * h + j] = ex2_approx(fmaf(score[u][2 * h + j], r.factor[j], -now));
#pragma unroll
      for (int n = 0; n < NG; ++n) {
        r.zero_sum[j][n] *= shrink;
        const float largest = max_over_g(fmaxf(fmaxf(w[0][j] * vs[0][0][n], w[0][2 + j] * vs[0][1][n]),
                                               fmaxf(w[1][j] * vs[1][0][n], w[1][2 + j] * vs[1][1][n])));
        const int was = exponent(r.down[j][n]);
        int is = min(was + int(fminf(rise, 300.f)), kMostDown);
        if (largest * pow2(is) > kMostProduct) is = 5 - exponent(largest);
        r.down[j][n] = pow2(is);
        const float by = ex2_approx(float(is - was) - rise);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          r.acc[n][i][j] *= by;
          r.acc[n][i][2 + j] *= by;
        }
      }
    }
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int n = 0; n < NG; ++n)
#pragma unroll
        for (int h = 0; h < 2; ++h)
          pb[u][n][h] = pack_half2(w[u][2 * h] * r.down[0][n] * vs[u][h][n], w[u][2 * h + 1] * r.down[1][n] * vs[u][h][n]);
  }
#pragma unroll
  for (int u = 0; u < 2; ++u) {
#pragma unroll
    for (int e = 0; e < 4; ++e) r.sum[e & 1] += w[u][e];
#pragma unroll
    for (int n = 0; n < NG; ++n) {
#pragma unroll
      for (int e = 0; e < 4; ++e) r.zero_sum[e & 1][n] = fmaf(w[u][e], vz[u][e / 2][n], r.zero_sum[e & 1][n]);
#pragma unroll
      for (int h = 0; h < 2; ++h) pb[u][n][h] = transpose8x8(pb[u][n][h]);
    }
  }
  // values
#pragma unroll
  for (int u = 0; u < 2; ++u)
#pragma unroll
    for (int n = 0; n < NG; ++n) {
      uint4 v = u == 0 ? n == 0 ? lds128<NG * 512>(at) : lds128<NG * 512 + 512>(at)
                       : n == 0 ? lds128<UB + NG * 512>(at) : lds128<UB + NG * 512 + 512>(at);
#pragma unroll
      for (int i = 0; i < 4; i += 2) {
        mma(r.acc[n][i], v.x & 0x000f000fu, v.y & 0x000f000fu, v.z & 0x000f000fu, v.w & 0x000f000fu, pb[u][n][0], pb[u][n][1]);
        mma(r.acc[n][i + 1], v.x & 0x00f000f0u, v.y & 0x00f000f0u, v.z & 0x00f000f0u, v.w & 0x00f000f0u, pb[u][n][0],
            pb[u][n][1]);
        v.x >>= 8, v.y >>= 8, v.z >>= 8, v.w >>= 8;
      }
    }
}

// The zeros' part joins the codes'.  Codes are 0 ... 15, so their sum alone grows with every token while the zeros take back all but the mean of
// the values; the tensor cores cut their sums off (2^-23.4 of the sum a product, one way, measured over 65536 tokens), which counts against
// what has added up.  Zeros joined only at the end of a chain of 2048 steps left the result off by 12 % (RMS); every 16 steps it
// is what fp16 weights and the bf16 result cost, for 60 instructions in 8500.
constexpr int kJoinSteps = 16;
template <int D>
__device__ __forceinline__ void join_zeros(Rolling<D> &r) {
#pragma unroll
  for (int n = 0; n < D / kGroup; ++n) {
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const float unit = r.down[j][n] * pow2(-24);
      const float z = sum_over_g(r.zero_sum[j][n]);
      r.zero_sum[j][n] = 0.f;
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int y = 0; y < 2; ++y) r.acc[n][i][2 * y + j] = fmaf(z, i & 1 ? 16.f * unit : unit, r.acc[n][i][2 * y + j]);
    }
  }
}

// Channels 64 m + 8 g ... + 7 of row 2t + j, times `by`.
template <int D>
__device__ __forceinline__ void result_of(const Rolling<D> &r, int m, int j, float by, float (&o)[8]) {
  const float a = over(pow2(24), r.down[j][m]) * by, a16 = a * 0.0625f, z = r.zero_sum[j][m] * by;
#pragma unroll
  for (int y = 0; y < 2; ++y)
#pragma unroll
    for (int i = 0; i < 4; ++i) o[4 * y + i] = fmaf(r.acc[m][i][2 * y + j], i & 1 ? a16 : a, z);
}

// A piece of a segment that its warp did not finish alone.
struct Piece {
  int b, segment, rows;  // rows of its tile that exist
  int start;             // where its segment's first step stands in the work of the whole launch
  int first, final;
};

template <int D>
__global__ void __launch_bounds__(kThreads, kCtasPerSm) attend_kernel(const __grid_constant__ AttendKernelParams p) {
  using Sh = Shared<D>;
  constexpr int NG = D / kGroup, UB = unit_bytes(D), S = Sh::kStages, R = kRows, kPitch = Sh::kPitch;
  extern __shared__ __align__(128) unsigned char smem[];
  __shared__ uint64_t full[kWarps][S];
  // pieces: 2 w of a warp's first segment where another follows, 2 w + 1 of its last
  __shared__ Piece pieces[2 * kWarps];
  __shared__ float stat_m[2 * kWarps][R], stat_l[2 * kWarps][R];
  __shared__ union __align__(16) {
    uint64_t source[kWarps][32];  // of units, by warp; read two at a time
    float joint[kWarps][D];       // sums over parts, at the end
  } shared_words;

  const int lane = threadIdx.x % 32, warp = uniform(threadIdx.x / 32), g = lane / 4, t = lane % 4;
  if (lane < S) mbar_init(&full[warp][lane], 1);
  if (lane < 2) pieces[2 * warp + lane].b = -1;
  fence_barrier_init();
  __syncwarp();
  grid_dependency_wait();
  grid_launch_dependents();

  // ---- this warp's share of the work: each warp adds up the whole batch for itself, a run of sequences a lane
  const int hr = p.c.heads_kv * p.row_tiles;  // segments of a sequence
  const int each = (p.b.batch + 31) / 32, b0 = lane * each;
  auto work_of = [&](const Sequence &s) { return s.steps == 0 ? 0 : (s.steps + kSegmentCost) * hr; };
  Sequence held;  // the lane's last sequence: its only one in batches of up to 32
  int mine = 0;   // of all sequences together below 2^31
  constexpr int kAhead = 2;
#pragma unroll 1
  for (int i0 = 0; i0 < each; i0 += kAhead) {
    Sequence s[kAhead];
#pragma unroll
    for (int i = 0; i < kAhead; ++i)
      if (i0 + i < each && b0 + i0 + i < p.b.batch) s[i] = read_sequence(p, b0 + i0 + i);
#pragma unroll
    for (int i = 0; i < kAhead; ++i)
      if (i0 + i < each && b0 + i0 + i < p.b.batch) {
        if (!check_sequence(p, s[i]) && blockIdx.x == 0 && warp == 0) report(p.c.status, STEEL_ERR_INVALID_ARG);
        mine += work_of(s[i]);
        if (i == 0) held = s[0];
      }
  }
  int before = mine;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const int below = __shfl_up_sync(0xffffffffu, before, d);
    if (lane >= d) before += below;
  }
  const int total = __shfl_sync(0xffffffffu, before, 31);
  before -= mine;
  const int share = max(divide(total + int(p.by_warps.divisor) - 1, p.by_warps), kSegmentCost + 1);
  const int cta_begin = min(total, int(min(int64_t(blockIdx.x) * kWarps * share, int64_t(total))));
  if (cta_begin >= total) return;
  const int begin = int(min(int64_t(cta_begin) + warp * share, int64_t(total)));
  int todo = min(share, total - begin), b = 0, offset = 0;
  const int end = begin + todo;
  {
    const bool here = before <= begin && begin < before + mine;  // one lane, or none
    if (here) {
      offset = begin - before;
      b = b0;
      if (each > 1) {
        for (;; ++b) {
          Sequence s = read_sequence(p, b);
          check_sequence(p, s);
          if (offset < work_of(s)) break;
          offset -= work_of(s);
        }
      }
    }
    const int who = max(__ffs(__ballot_sync(0xffffffffu, here)) - 1, 0);
    b = __shfl_sync(0xffffffffu, b, who);
    offset = __shfl_sync(0xffffffffu, offset, who);
  }

  unsigned char *ring = smem + warp * Sh::kRingBytes;
  const uint32_t ring_at = smem_u32(ring), bars_at = smem_u32(full[warp]);
  uint32_t filled = 0;  // steps that this warp has read from its ring since the kernel began
  bool dead = false;    // a wait of this warp has expired
  const int units_a_page = (1 << p.c.page_shift) / kUnitTokens;
  for (; todo > 0; ++b, offset = 0) {
    Sequence seq;
    if (each == 1) {
      seq.slot = __shfl_sync(0xffffffffu, held.slot, b), seq.len = __shfl_sync(0xffffffffu, held.len, b);
      seq.count = __shfl_sync(0xffffffffu, held.count, b);
      seq.step_lo = __shfl_sync(0xffffffffu, held.step_lo, b), seq.steps = __shfl_sync(0xffffffffu, held.steps, b);
    } else {
      seq = read_sequence(p, b);
      seq.slot = uniform(seq.slot), seq.len = uniform(seq.len), seq.count = uniform(seq.count);
      check_sequence(p, seq);
    }
    if (seq.steps == 0) continue;
    const int cost = seq.steps + kSegmentCost;
    int segment = int(uint32_t(offset) / uint32_t(cost)), at = offset - segment * cost;
    for (; todo > 0 && segment < hr; ++segment, at = 0) {
      // ---- a piece: steps [from, to) of the segment (sequence, head, row tile)
      const int n = min(cost - at, todo);
      const int from = max(0, at - kSegmentCost), to = max(0, at + n - kSegmentCost);
      const int start = end - todo - at + kSegmentCost;
      todo -= n;
      if (to <= from) continue;
      const int head = divide(segment, p.by_row_tiles);
      Tile tile;
      tile.len = seq.len;
      tile.pos0 = seq.len - seq.count;
      tile.row0 = (segment - head * p.row_tiles) * R;
      tile.rows = min(R, seq.count * p.group - tile.row0);  // <= 0: none
      const int first_pos = tile.pos0 + divide(tile.row0, p.by_group),
                last_pos = tile.pos0 + divide(tile.row0 + max(tile.rows, 1) - 1, p.by_group);
      tile.any_lo = max(key_lo(p, first_pos), 0), tile.any_hi = key_hi(p, seq.len, last_pos);
      tile.all_lo = key_lo(p, last_pos), tile.all_hi = key_hi(p, seq.len, first_pos);
      const int s0 = max(seq.step_lo + from, tile.any_lo / kStepTokens);
      const int s1 = min(seq.step_lo + to, (tile.any_hi + kStepTokens - 1) / kStepTokens);
      const int steps = dead || tile.rows <= 0 ? 0 : max(0, s1 - s0);

      // ---- pages: lane l looks up where unit l of the next 16 steps lies, or 0.  The first look-up is under way while the queries are
      // asked for.
      const int32_t *table = p.c.table + int64_t(seq.slot) * p.c.max_pages;
      const unsigned char *head_pool = p.c.pool + int64_t(head) * (units_a_page * UB);
      auto page_of = [&](int i0) {  // INT32_MIN: no unit
        const int token = ((s0 + i0) * 2 + lane) * kUnitTokens;
        return i0 + lane / 2 < steps && token < seq.len ? table[token >> p.c.page_shift] : INT32_MIN;
      };
      auto put_sources = [&](int i0, int page) {
        uint64_t from_pool = 0;
        if (page >= 0 && page < p.c.pages)
          from_pool = reinterpret_cast<uint64_t>(head_pool + page * p.c.page_bytes + (((s0 + i0) * 2 + lane) & (units_a_page - 1)) * UB);
        else if (page != INT32_MIN)
          report(p.c.status, STEEL_ERR_INVALID_ARG);
        shared_words.source[warp][lane] = from_pool;
        __syncwarp();
      };
      const int first_page = page_of(0);
      uint4 raw[D / 32];
      load_queries<D>(p, b, head, tile, lane, raw);
      put_sources(0, first_page);
      auto issue = [&](int i) {  // step i into the ring
        if (i > 0 && (i & 15) == 0) put_sources(i, page_of(i));
        if (lane == 0) {
          const uint32_t nth = filled + i, place = ring_at + (nth % S) * Sh::kStepBytes, bar = bars_at + (nth % S) * 8;
          const ulonglong2 source = *reinterpret_cast<const ulonglong2 *>(&shared_words.source[warp][2 * i & 31]);
          if (source.y == source.x + UB) {
            mbar_expect(bar, 2 * UB);
            bulk_load(place, source.x, 2 * UB, bar);
          } else {
            mbar_expect(bar, ((source.x != 0) + (source.y != 0)) * UB);
            if (source.x) bulk_load(place, source.x, UB, bar);
            if (source.y) bulk_load(place + UB, source.y, UB, bar);
          }
        }
        __syncwarp();
      };
      const uint32_t full_steps_from = uint32_t((max(tile.all_lo, 0) + kStepTokens - 1) / kStepTokens),
                     full_steps = uint32_t(max(max(tile.all_hi, 0) / kStepTokens - int(full_steps_from), 0));
      Rolling<D> r;
      // the copy of step i + S is issued behind the work on step i, the first S before any
#pragma unroll 1
      for (int i = -S; i < steps; ++i) {
        if (i == -1) {
          unpack_queries<D>(p.scale_log2, raw, lane, r);
          clear(r);
        }
        if (i >= 0) {
          const uint32_t nth = filled + i;
          if (!wait_full(bars_at + (nth % S) * 8, nth / S & 1)) {
            await_copies<S>(i, steps, [&](int j) { wait_full(bars_at + (filled + j) % S * 8, (filled + j) / S & 1); });
            if (lane == 0) report(p.c.status, STEEL_ERR_TIMEOUT);
            dead = true;
            break;
          }
          const uint32_t place = ring_at + (nth % S) * Sh::kStepBytes, at = place + lane * 16, at_scales = place + g * (8 * NG);
          const int key0 = (s0 + i) * kStepTokens;
          const bool partial = uint32_t(s0 + i) - full_steps_from >= full_steps;
          attend_step<D>(p, at, at_scales, partial, key0, tile, lane, r);
          if ((i & (kJoinSteps - 1)) == kJoinSteps - 1) join_zeros(r);
          __syncwarp();
        }
        if (i + S < steps) issue(i + S);
      }
      filled += steps;

      // ---- the piece's result: rows 2t + j, channels 64 n + 8 g ... + 7 of each
      const bool whole = from == 0 && to == seq.steps;
      const bool last = todo <= kSegmentCost;
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        r.sum[j] = sum_over_g(r.sum[j]);
#pragma unroll
        for (int m = 0; m < NG; ++m) r.zero_sum[j][m] = sum_over_g(r.zero_sum[j][m]);
      }
      if (whole) {
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          if (2 * t + j >= tile.rows) break;
          const float l = r.sum[j], by = l == 0.f ? 0.f : 1.f / l;
          const int row = tile.row0 + 2 * t + j, pos = divide(row, p.by_group);
          const int64_t to_row = (int64_t(b) * (p.c.heads_kv * p.group) + head * p.group + row - pos * p.group) * p.seq_q + pos;
#pragma unroll
          for (int m = 0; m < NG; ++m) {
            float o[8];
            result_of(r, m, j, by, o);
            *reinterpret_cast<uint4 *>(p.o + to_row * D + kGroup * m + 8 * g) =
                make_uint4(pack_bf16x2(o[0], o[1]), pack_bf16x2(o[2], o[3]), pack_bf16x2(o[4], o[5]), pack_bf16x2(o[6], o[7]));
          }
          if (g == 0 && p.lse) p.lse[to_row] = l == 0.f ? -INFINITY : (r.ref[j] + log2f(l)) * kLn2;
        }
        continue;
      }
      // A warp's last piece lies over its ring, which it needs no more; an earlier one (the end of a segment that began in another
      // warp) in a place of its own.  They are put together below.
      float *rows = reinterpret_cast<float *>(last ? ring : smem + kWarps * Sh::kRingBytes + warp * Sh::kPieceBytes) + 8 * g;
#pragma unroll
      for (int j = 0; j < 2; ++j) {
#pragma unroll
        for (int m = 0; m < NG; ++m) {
          float o[8];
          result_of(r, m, j, 1.f, o);
          float4 *to_smem = reinterpret_cast<float4 *>(rows + (2 * t + j) * kPitch + kGroup * m);
          to_smem[0] = make_float4(o[0], o[1], o[2], o[3]);
          to_smem[1] = make_float4(o[4], o[5], o[6], o[7]);
        }
        if (g == 0) {
          stat_m[2 * warp + last][2 * t + j] = r.ref[j];
          stat_l[2 * warp + last][2 * t + j] = r.sum[j];
        }
      }
      if (lane == 0) pieces[2 * warp + last] = Piece{b, segment, tile.rows, start, from == 0, to == seq.steps};
    }
  }
  __syncthreads();

  // ---- runs of pieces of one segment, in the order of the warps.  Lane k looks at piece k; a warp takes a row of a run.  A run
  // that does not end its segment, the last one, is handed to the CTA that does; one that does but began in other CTAs, the first one,
  // comes last here and waits for them.  They have lower numbers and wait for nobody before they have handed over.
  constexpr int V = D / 32;  // a lane's channels
  constexpr int kBatch = 16;  // parts' rows in flight
  const Piece mine_piece = pieces[lane % (2 * kWarps)];
  const uint32_t valid = __ballot_sync(0xffffffffu, lane < 2 * kWarps && mine_piece.b >= 0);
  const uint32_t firsts = __ballot_sync(0xffffffffu, mine_piece.first) & valid;
  const uint32_t finals = __ballot_sync(0xffffffffu, mine_piece.final) & valid;
  // the pieces in front of the first beginning, if they end a segment
  const uint32_t behind = firsts ? (firsts & (0u - firsts)) - 1u : 0xffffffffu;
  const uint32_t joined = finals & behind ? valid & behind : 0u;

  // reference and sum of a row: lane k has those of piece k
  auto row_stats = [&](uint32_t run, int row, float &m, float &sum) {
    const bool in = run >> lane & 1u;
    m = in ? stat_m[lane % (2 * kWarps)][row] : kFloor;
    sum = in ? stat_l[lane % (2 * kWarps)][row] : 0.f;
  };
  auto weight_of = [](float m, float sum, float top) { return m == kFloor && sum == 0.f ? 0.f : ex2_approx(m - top); };
  auto add_pieces = [&](uint32_t run, int row, float weight, float (&o)[V]) {
#pragma unroll 2
    for (uint32_t left = run; left; left &= left - 1) {
      const int k = __ffs(left) - 1;
      const float by = __shfl_sync(0xffffffffu, weight, k);
      const float *src = reinterpret_cast<const float *>(smem + (k & 1 ? k / 2 * Sh::kRingBytes
                                                                       : kWarps * Sh::kRingBytes + k / 2 * Sh::kPieceBytes)) +
                         row * kPitch + lane * V;
#pragma unroll
      for (int c = 0; c < V; ++c) o[c] = fmaf(by, src[c], o[c]);
    }
  };
  auto write_row = [&](const Piece &piece, int row, const float (&o)[V], float l, float top) {
    const int head = divide(piece.segment, p.by_row_tiles), tile_row = (piece.segment - head * p.row_tiles) * R + row;
    const int pos = divide(tile_row, p.by_group);
    const int64_t to_row =
        (int64_t(piece.b) * (p.c.heads_kv * p.group) + head * p.group + tile_row - pos * p.group) * p.seq_q + pos;
    const float inverse = l == 0.f ? 0.f : 1.f / l;
    uint32_t *to = reinterpret_cast<uint32_t *>(p.o + to_row * D + lane * V);
#pragma unroll
    for (int c = 0; c < V / 2; ++c) to[c] = pack_bf16x2(o[2 * c] * inverse, o[2 * c + 1] * inverse);
    if (lane == 0 && p.lse) p.lse[to_row] = l == 0.f ? -INFINITY : (top + log2f(l)) * kLn2;
  };

  int task = 0;  // rows so far: those of the next run go to the warps that follow
  for (uint32_t rest = valid & ~joined, run; rest; rest &= ~run) {
    const uint32_t final_here = finals & rest;
    run = final_here ? rest & ((final_here & (0u - final_here)) * 2u - 1u) : rest;
    const Piece piece = pieces[__ffs(run) - 1];
    const int rows = uniform(min(piece.rows, R));
    for (int row = (warp + kWarps - task % kWarps) % kWarps; row < rows; row += kWarps) {
      float m, l, o[V];
      row_stats(run, row, m, l);
      const float top = max_over_warp(m), weight = weight_of(m, l, top);
      l = sum_over_warp(weight * l);
#pragma unroll
      for (int c = 0; c < V; ++c) o[c] = 0.f;
      add_pieces(run, row, weight, o);
      if (final_here) {
        write_row(piece, row, o, l, top);
      } else {
        float *part = p.parts + int64_t(blockIdx.x) * part_floats(R, D);
#pragma unroll
        for (int c = 0; c < V; ++c) part[row * D + lane * V + c] = o[c];
        if (lane == 0) part[R * D + row] = top, part[R * D + R + row] = l;
        __syncwarp();
        if (lane == 0) hand_over(p.flags + int64_t(blockIdx.x) * R + row, p.token);
      }
    }
    task += max(rows, 0);
  }

  if (joined == 0) return;
  const Piece piece = pieces[__ffs(joined) - 1];
  const int rows = uniform(min(piece.rows, R)), others = int(blockIdx.x) - piece.start / (kWarps * share);  // CTAs with parts
  const int64_t first_other = int64_t(blockIdx.x) - others;
  const float *parts = p.parts + first_other * part_floats(R, D);
  for (int i = threadIdx.x; i < others * rows; i += kThreads) {
    if (!take_over(p.flags + (first_other + i / rows) * R + i % rows, p.token, p.wait_cycles)) report(p.c.status, STEEL_ERR_TIMEOUT);
  }
  __syncthreads();
  const int each_row = max(kWarps / max(rows, 1), 1);  // warps that share a row's parts
  const int turn = warp % each_row;
  float l = 0.f, top = kFloor, o[V];
  for (int row = warp / each_row; row < rows; row += kWarps / each_row) {  // at most once where each_row > 1
    row_stats(joined, row, top, l);
    const float own_top = max_over_warp(top), weight = weight_of(top, l, own_top);
    l *= weight;
    top = own_top;
    float own_scale = 1.f;
#pragma unroll
    for (int c = 0; c < V; ++c) o[c] = 0.f;
    // 32 parts at a time, their statistics and rows asked for together: a round trip to L2 costs more than the sums
#pragma unroll 1
    for (int k0 = 0; k0 < others; k0 += 32) {
      const int here = min(32, others - k0);
      const float *stats = parts + (k0 + min(lane, here - 1)) * part_floats(R, D) + R * D + row;
      float m = __ldcg(stats), sum = __ldcg(stats + R);
      if (lane >= here) m = kFloor, sum = 0.f;
      const float *src = parts + k0 * part_floats(R, D) + row * D + lane * V;
#pragma unroll 1
      for (int first = turn; first == turn || first < here; first += kBatch * each_row) {
        float x[kBatch][V];
#pragma unroll
        for (int j = 0; j < kBatch; ++j) {
          const int k = first + j * each_row;
          if (k < here) load_floats(x[j], src + k * part_floats(R, D));
        }
        if (first == turn) {
          const float now = fmaxf(top, max_over_warp(m)), shrink = ex2_approx(top - now);
          sum *= m = weight_of(m, sum, now);  // m: the part's weight from here on
          l = fmaf(l, shrink, sum);
          own_scale *= shrink;
#pragma unroll
          for (int c = 0; c < V; ++c) o[c] *= shrink;
          top = now;
        }
#pragma unroll
        for (int j = 0; j < kBatch; ++j) {
          const int k = first + j * each_row;
          const float by = __shfl_sync(0xffffffffu, m, k & 31);
          if (k < here) {
#pragma unroll
            for (int c = 0; c < V; ++c) o[c] = fmaf(by, x[j][c], o[c]);
          }
        }
      }
    }
    l = sum_over_warp(l);
    if (turn == 0) add_pieces(joined, row, weight * own_scale, o);
    if (each_row == 1) write_row(piece, row, o, l, top);
  }
  if (each_row > 1) {  // all threads of the CTA come here, or none
#pragma unroll
    for (int c = 0; c < V; ++c) shared_words.joint[warp][lane * V + c] = o[c];
    __syncthreads();
    if (turn == 0 && warp / each_row < rows) {
      for (int w = 1; w < each_row; ++w) {
#pragma unroll
        for (int c = 0; c < V; ++c) o[c] += shared_words.joint[warp + w][lane * V + c];
      }
      write_row(piece, warp / each_row, o, l, top);
    }
  }
}

int64_t flags_bytes(int ctas) { return (int64_t(ctas) * kRows * int64_t(sizeof(uint64_t)) + 127) / 128 * 128; }

}  // namespace

// Steps of all row tiles, heads and sequences are counted in 31 bits.
bool attend_fits(const CacheView &c, int batch, int heads_q, int seq_q) {
  const int64_t rows = int64_t(heads_q / c.heads_kv) * seq_q;
  if (rows > (1 << 24)) return false;
  const int64_t steps = ((int64_t(c.max_pages) << c.page_shift) / kStepTokens + 1 + kSegmentCost) * c.heads_kv * ((rows + kRows - 1) / kRows);
  return steps < (int64_t(1) << 30) && steps * batch < (int64_t(1) << 30);
}

int64_t attend_workspace(int head_dim, int sms) {
  const int ctas = sms * kCtasPerSm;
  return flags_bytes(ctas) + ctas * part_floats(kRows, head_dim) * int64_t(sizeof(float));
}

cudaError_t configure_attend() {
  const cudaError_t e = cudaFuncSetAttribute(attend_kernel<64>, cudaFuncAttributeMaxDynamicSharedMemorySize, Shared<64>::kBytes);
  if (e != cudaSuccess) return e;
  return cudaFuncSetAttribute(attend_kernel<128>, cudaFuncAttributeMaxDynamicSharedMemorySize, Shared<128>::kBytes);
}

cudaError_t launch_attend(const CacheView &c, const AttendProblem &a, int sms, cudaStream_t stream) {
  const int group = a.heads_q / c.heads_kv, grid = sms * kCtasPerSm;
  AttendKernelParams kp{};
  kp.c = c;
  kp.b = a.b;
  kp.q = a.q;
  kp.o = static_cast<__nv_bfloat16 *>(a.o);
  kp.lse = a.lse;
  kp.flags = reinterpret_cast<uint64_t *>(a.workspace);
  kp.parts = reinterpret_cast<float *>(a.workspace + flags_bytes(grid));
  kp.token = next_token();
  kp.wait_cycles = a.wait_cycles;
  kp.group = group;
  kp.seq_q = a.seq_q;
  kp.row_tiles = (group * a.seq_q + kRows - 1) / kRows;
  // a window wider than any sequence hides nothing: within 32 bits
  kp.window = int32_t(a.window < (int64_t(1) << 30) ? a.window : int64_t(1) << 30);
  kp.mask = int32_t(a.flags);
  kp.scale_log2 = a.scale * kLog2e;
  kp.by_group = fast_divisor(group);
  kp.by_row_tiles = fast_divisor(kp.row_tiles);
  kp.by_warps = fast_divisor(grid * kWarps);
  if (a.head_dim == 64)
    return launch_overlapping(attend_kernel<64>, dim3(grid), dim3(kThreads), Shared<64>::kBytes, stream, kp);
  return launch_overlapping(attend_kernel<128>, dim3(grid), dim3(kThreads), Shared<128>::kBytes, stream, kp);
}

}  // namespace steel
