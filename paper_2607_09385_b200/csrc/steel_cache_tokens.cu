// Tokens into the pages of the 4-bit cache and back (include/steel_cache.h has the quantiser and the layout).
//
// Many tokens: a warp takes one unit, 16 tokens of one head.  Lane (g, t) = (lane / 4, lane % 4) holds what it holds of the unit
// in memory: for K the channels 32c + 8t ... + 7 of tokens g and 8 + g, for V the channels 8g ... 8g + 7 of every group of tokens
// 8h + 2t + f.  Codes then move as 16 bytes a lane, 512 bytes a warp and group.  The lanes that share a token reduce its minimum and maximum
// so that each ends with one token's, makes that one's scale and gives it to the others (all scales in all lanes: 28.0 us for what
// then took 26.5, now 26.9).  Memory's part is 4 head_dim bytes of bf16 and 1.125 head_dim of codes and scales a token and head;
// quantising costs 17 instructions a value and lane (2140 a unit at head_dim 128), which is more than that leaves time for: 16K
// tokens x 8 heads take 26.9 us against 13.1 at the measured copy rate, and reading them back 16.2.  The code is kept small, a loop over
// the groups: unrolled, most of the time went into fetching instructions (66 us).
// Few tokens: a warp takes one token of one head, a lane four channels, 16 bits of codes.  Bound by the latency of the reads that follow
// one another (slot, length, page) and by how much code there is to fetch: 64 sequences x 1 token written and read back in 5.0 us, with units
// 10.0.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "sm100_ptx.cuh"
#include "steel_cache.cuh"

namespace steel {

namespace {

constexpr int kWarps = 4;
constexpr int kReadUnits = 2;  // units a warp when reading: 16K x 8 heads at head_dim 128 in 16.4 us, 17.4 with one; 8 x 300 to 6500 at 64 13.2, 15.2

__device__ __forceinline__ float bf16_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }
__device__ __forceinline__ uint4 load16(const void *p) { return *static_cast<const uint4 *>(p); }

__device__ __forceinline__ uint32_t bf16_min2(uint32_t a, uint32_t b) {  // NaN if either is
  uint32_t d;
  asm("min.NaN.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
  return d;
}
__device__ __forceinline__ uint32_t bf16_max2(uint32_t a, uint32_t b) {
  uint32_t d;
  asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
  return d;
}

// Minimum (low half) and negated maximum (high half) of a lane's 8 channels.
__device__ __forceinline__ uint32_t extremes(const uint4 &x) {
  const uint32_t lo = bf16_min2(bf16_min2(x.x, x.y), bf16_min2(x.z, x.w));
  const uint32_t hi = bf16_max2(bf16_max2(x.x, x.y), bf16_max2(x.z, x.w)) ^ 0x80008000u;
  // halves of the same kind side by side
  return bf16_min2(__byte_perm(lo, hi, 0x5410), __byte_perm(lo, hi, 0x7632));
}
// The same over the lanes whose number differs in `bit`, of two tokens: of `a` for the lanes without it, of `b` for those with it.
__device__ __forceinline__ uint32_t extremes_share(uint32_t a, uint32_t b, int bit, int lane) {
  const bool second = lane & bit;
  return bf16_min2(second ? b : a, __shfl_xor_sync(0xffffffffu, second ? a : b, bit));
}
__device__ __forceinline__ uint32_t extremes_over(uint32_t e, int bit) {
  return bf16_min2(e, __shfl_xor_sync(0xffffffffu, e, bit));
}

constexpr float kMost = 65504.f;  // largest fp16
constexpr float kRound = 12582912.f;  // 1.5 * 2^23: adding it rounds to an integer, half to even, in the low bits

// The bits of kRound in every nibble's place, as they add up in a word.
template <int N>
constexpr uint32_t kRoundBits = (0x4B400000u << (4 * (N - 1))) + kRoundBits<N - 1>;
template <>
constexpr uint32_t kRoundBits<0> = 0;

struct Scale {
  uint32_t pair;         // scale and zero in fp16
  float inverse, shift;  // (x - zero) / (15 scale) = x inverse + shift
};
// A quotient further than this from every border between two codes is on the right side of it.
__device__ __forceinline__ float clear_of(float shift) { return 0.5f - (10.f + fabsf(shift)) * (1.f / (1 << 20)); }
__device__ __forceinline__ Scale scale_from(const Scale &s, int lane) {
  return {__shfl_sync(0xffffffffu, s.pair, lane), __shfl_sync(0xffffffffu, s.inverse, lane), __shfl_sync(0xffffffffu, s.shift, lane)};
}

// f32(d / 15): multiplication by the rounded inverse and one FMA correction (division by a constant after Markstein) give the rounded
// quotient for every significand (tried for all 2^23 of them).
__device__ __forceinline__ float fifteenth(float d) {
  constexpr float c = 1.f / 15.f;
  const float q = __fmul_rn(d, c);
  return __fmaf_rn(__fmaf_rn(-15.f, q, d), c, q);
}

// Rare ways are functions of their own: what they cost the others is the code to be fetched.
__device__ __noinline__ float wide_fifteenth(float hi, float lo) {
  return static_cast<float>((static_cast<double>(hi) - static_cast<double>(lo)) / 15.0);
}

__device__ __forceinline__ Scale make_scale(uint32_t e) {
  float lo = bf16_lo(e), hi = -bf16_hi(e);
  Scale s;
  const bool none = lo != lo;  // a NaN: the pair is NaN, codes are 0
  lo = fminf(fmaxf(lo, -kMost), kMost);
  hi = fminf(fmaxf(hi, -kMost), kMost);
  // the difference of two bf16 numbers, and what 32 bits lose of it: nothing unless one is 2^16 times the other
  const float d = __fsub_rn(hi, lo), back = __fsub_rn(d, hi);
  const float rest = __fsub_rn(__fsub_rn(hi, __fsub_rn(d, back)), __fadd_rn(lo, back));
  float wide = fifteenth(d);
  if (rest != 0.f) wide = wide_fifteenth(hi, lo);
  const __half zero = __float2half_rn(lo), scale = __float2half_rn(wide);
  s.pair = none ? 0x7fff7fffu : uint32_t(__half_as_ushort(zero)) << 16 | __half_as_ushort(scale);
  const float by = none ? 0.f : __half2float(scale);
  s.inverse = by > 0.f ? __fdividef(1.f / 15.f, by) : 0.f;
  s.shift = __fmul_rn(-__half2float(zero), s.inverse);
  return s;
}

// The codes of n channels, those next to a border between two codes settled: one value in 2500 lies exactly on it, because bf16 numbers
// and an fp16 scale have few bits.
__device__ __noinline__ uint32_t settle(uint32_t w0, uint32_t w1, uint32_t w2, uint32_t w3, int n, uint32_t scale_zero,
                                        float inverse, float shift, uint32_t word) {
  const float scale = __half2float(__ushort_as_half(uint16_t(scale_zero))), zero = __half2float(__ushort_as_half(uint16_t(scale_zero >> 16)));
  const float clear = clear_of(shift);
  auto channel = [&](int i) {
    const uint32_t pair = i < 2 ? w0 : i < 4 ? w1 : i < 6 ? w2 : w3;
    return i & 1 ? bf16_hi(pair) : bf16_lo(pair);
  };
  auto off_by = [&](float x, int code) { return __fmaf_rn(__saturatef(__fmaf_rn(x, inverse, shift)), 15.f, -float(code)); };
  uint32_t close = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i)
    if (i < n && fabsf(off_by(channel(i), word >> (4 * i) & 15)) > clear) close |= 1u << i;
#pragma unroll 1
  for (; close; close &= close - 1) {
    const int i = __ffs(close) - 1;
    const float x = channel(i);
    int code = word >> (4 * i) & 15;
    const int low = off_by(x, code) > 0.f ? code : code - 1;
    // x - zero against (low + 1/2) scale, which 32 bits hold exactly: the rounded difference and what it lost
    const float d = __fsub_rn(x, zero), back = __fsub_rn(d, x);
    const float rest = __fsub_rn(__fsub_rn(x, __fsub_rn(d, back)), __fadd_rn(zero, back));
    const float side = __fadd_rn(__fsub_rn(d, __fmul_rn(float(low) + 0.5f, scale)), rest);
    code = side > 0.f ? low + 1 : side < 0.f ? low : low + (low & 1);
    word = (word & ~(15u << (4 * i))) | uint32_t(min(max(code, 0), 15)) << (4 * i);
  }
  return word;
}

// Codes of N / 2 words of two channels, nibble i = channel i.  The quotient over 15 in [0, 1], x inverse + shift, is off by at most
// (9 + |shift|) 2^-24: the inverse by 2^-21 of itself (a division of 2 ulp and the constant), the product with zero and the sum by a rounding
// each.  15 times that is less than what `clear` leaves to a border; |shift| is below 2^9, because the numbers of a group that are not equal
// differ by 2^-8 of the largest at least.
template <int N>
__device__ __forceinline__ uint32_t codes_of(const uint32_t (&w)[N / 2], const Scale &s) {
  uint32_t word = 0;
  float far = 0.f, before = 0.f;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const float x = i & 1 ? bf16_hi(w[i / 2]) : bf16_lo(w[i / 2]);
    const float part = __saturatef(__fmaf_rn(x, s.inverse, s.shift));
    const float rounded = __fmaf_rn(part, 15.f, kRound);
    const float off = fabsf(__fmaf_rn(part, 15.f, kRound - rounded));
    if (i & 1) far = fmax3(far, before, off);
    before = off;
    word += __float_as_uint(rounded) << (4 * i);  // the code, and bits of 1.5 * 2^23 that are taken off below
  }
  word -= kRoundBits<N>;
  if (far > clear_of(s.shift))
    word = settle(w[0], w[1], w[N == 8 ? 2 : 0], w[N == 8 ? 3 : 0], N, s.pair, s.inverse, s.shift, word);
  return word;
}
__device__ __forceinline__ uint32_t codes_of(const uint4 &x, const Scale &s) {
  const uint32_t w[4] = {x.x, x.y, x.z, x.w};
  return codes_of<8>(w, s);
}

// What a call finds of sequence i of its batch for writing: the slot's length, or -1 and a report.
__device__ __forceinline__ int checked_length(const CacheView &c, const CacheBatch &b, int i, int seq, int lane, bool tell, int &slot,
                                              int &count) {
  slot = slot_of(c, b.slots, i);
  count = b.counts ? b.counts[i] : seq;
  const int len = c.lens[max(slot, 0)];
  if (slot < 0 || count < 0 || count > seq || len < count || len > max_tokens(c) || slot_taken_before(b.slots, i, slot, lane)) {
    if (tell && lane == 0) report(c.status, STEEL_ERR_INVALID_ARG);
    return -1;
  }
  return len;
}

// The page of a slot's token; of a token that it cannot have, any of its pages.
__device__ __forceinline__ int page_of(const CacheView &c, int slot, int64_t token) {
  return c.table[int64_t(slot) * c.max_pages + min(int(token >> c.page_shift), c.max_pages - 1)];
}

// The unit of tokens `first` ... of a slot, or null and a report.
__device__ __forceinline__ unsigned char *unit_in(const CacheView &c, int page, int first, int head, int bytes, int lane) {
  if (page < 0 || page >= c.pages) {
    if (lane == 0) report(c.status, STEEL_ERR_INVALID_ARG);
    return nullptr;
  }
  const int units = (1 << c.page_shift) / kUnitTokens;
  return c.pool + page * c.page_bytes + (int64_t(head) * units + (first / kUnitTokens & (units - 1))) * bytes;
}

// The same for writing: a page that other entries name too is left alone.
__device__ __forceinline__ unsigned char *own_unit_in(const CacheView &c, int page, int first, int head, int bytes, int lane) {
  unsigned char *unit = unit_in(c, page, first, head, bytes, lane);
  if (unit && c.refs[page] > 1) {
    if (lane == 0) report(c.status, STEEL_ERR_INVALID_ARG);
    return nullptr;
  }
  return unit;
}

template <int D>
__global__ void __launch_bounds__(kWarps * 32, 7) append_kernel(CacheView c, CacheBatch b, int seq, int units_a_head, Rows k, Rows v) {
  constexpr int NG = D / kGroup;
  grid_dependency_wait();
  grid_launch_dependents();
  const int lane = threadIdx.x % 32, g = lane / 4, t = lane % 4;
  const int work = blockIdx.x * kWarps + threadIdx.x / 32;
  const int head = work / units_a_head, nth = work % units_a_head, i = blockIdx.y;
  if (head >= c.heads_kv) return;
  int slot, count;
  const int len = checked_length(c, b, i, seq, lane, work == 0, slot, count);
  const int start = len - count, first = (start / kUnitTokens + nth) * kUnitTokens;
  if (len < 0 || first >= len || count == 0) return;
  const int from = max(start - first, 0), to = min(len - first, kUnitTokens);
  unsigned char *out = own_unit_in(c, page_of(c, slot, first), first, head, unit_bytes(D), lane);
  if (!out) return;
  const bool whole = from == 0 && to == kUnitTokens;

  // keys
  {
    // tokens that are not to be written are read in another's place
    const unsigned char *src = k.data + i * k.batch + head * k.head + (first - start) * k.seq + 16 * t;
    const int64_t row[2] = {min(max(g, from), to - 1) * k.seq, min(max(8 + g, from), to - 1) * k.seq};
    unsigned char *codes = out + lane * 16, *scales = out + NG * 1024 + g * 8 * NG;
#pragma unroll 1
    for (int n = 0; n < NG; ++n, src += kGroup * 2, codes += 512, scales += 4) {
      uint4 x[2][2];  // [c][h]
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int a = 0; a < 2; ++a)
          x[a][h] = load16(src + row[h] + 64 * a);
      uint32_t word[2][2], e[2];
#pragma unroll
      for (int h = 0; h < 2; ++h) e[h] = bf16_min2(extremes(x[0][h]), extremes(x[1][h]));
      const Scale mine = make_scale(extremes_over(extremes_share(e[0], e[1], 1, lane), 2));  // of h = t % 2
      if (t < 2 && (whole || (8 * t + g >= from && 8 * t + g < to))) *reinterpret_cast<uint32_t *>(scales + t * NG * 4) = mine.pair;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const Scale s = scale_from(mine, lane / 4 * 4 + h);
        word[0][h] = codes_of(x[0][h], s);
        word[1][h] = codes_of(x[1][h], s);
      }
      if (whole) {
        *reinterpret_cast<uint4 *>(codes) = make_uint4(word[0][0], word[0][1], word[1][0], word[1][1]);
      } else {
#pragma unroll
        for (int h = 0; h < 2; ++h)
          if (8 * h + g >= from && 8 * h + g < to) {
            *reinterpret_cast<uint32_t *>(codes + h * 4) = word[0][h];
            *reinterpret_cast<uint32_t *>(codes + 8 + h * 4) = word[1][h];
          }
      }
    }
  }
  // values
  {
    const unsigned char *src = v.data + i * v.batch + head * v.head + (first - start) * v.seq + 16 * g;
    int64_t row[2][2];
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int f = 0; f < 2; ++f) row[h][f] = min(max(8 * h + 2 * t + f, from), to - 1) * v.seq;
    unsigned char *codes = out + NG * 512 + lane * 16, *scales = out + NG * 1088 + 2 * t * 8 * NG;
#pragma unroll 1
    for (int n = 0; n < NG; ++n, src += kGroup * 2, codes += 512, scales += 4) {
      uint4 x[2][2];  // [h][f]
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int f = 0; f < 2; ++f) x[h][f] = load16(src + row[h][f]);
      uint32_t e[2];
#pragma unroll
      for (int h = 0; h < 2; ++h) e[h] = extremes_share(extremes(x[h][0]), extremes(x[h][1]), 4, lane);
      const Scale mine = make_scale(extremes_over(extremes_share(e[0], e[1], 8, lane), 16));  // of h = g / 2 % 2, f = g % 2
      {
        const int h = g >> 1, f = g & 1, token = 8 * h + 2 * t + f;
        if (g < 4 && (whole || (token >= from && token < to)))
          *reinterpret_cast<uint32_t *>(scales + (f * 2 + h) * NG * 4) = mine.pair;
      }
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        uint32_t word[2];  // [f]: channels 8g ... 8g + 7 of a token
#pragma unroll
        for (int f = 0; f < 2; ++f) word[f] = codes_of(x[h][f], scale_from(mine, (2 * h + f) * 4 + t));
        // the low and the high four channels of two tokens share a word
        if (whole) {
          *reinterpret_cast<uint2 *>(codes + h * 8) =
              make_uint2(__byte_perm(word[0], word[1], 0x5410), __byte_perm(word[0], word[1], 0x7632));
        } else {
#pragma unroll
          for (int f = 0; f < 2; ++f) {
            const int token = 8 * h + 2 * t + f;
            if (token >= from && token < to) {
              *reinterpret_cast<uint16_t *>(codes + h * 8 + f * 2) = uint16_t(word[f]);
              *reinterpret_cast<uint16_t *>(codes + h * 8 + 4 + f * 2) = uint16_t(word[f] >> 16);
            }
          }
        }
      }
    }
  }
}

// Where the 16 bits of channels 4m ... 4m + 3 of a unit's token stand, in bytes.
template <int NG>
__device__ __forceinline__ int key_place(int token, int m) {
  const int rest = m % 16;
  return (m / 16 * 256 + token % 8 * 32 + rest % 8 / 2 * 8 + rest / 8 * 4 + token / 8 * 2 + rest % 2) * 2;
}
template <int NG>
__device__ __forceinline__ int value_place(int token, int m) {
  const int rest = m % 16;
  return NG * 512 + (m / 16 * 256 + rest / 2 * 32 + token % 8 / 2 * 8 + token / 8 * 4 + rest % 2 * 2 + token % 2) * 2;
}
template <int NG>
__device__ __forceinline__ int scale_place(int token, int group) {
  return NG * 1024 + ((token % 8 * 2 + token / 8) * NG + group) * 4;  // of V: 64 NG further on
}

// One token of one head a warp: lane m has channels 4m ... 4m + 3, of K and then of V; at head_dim 64 half a warp has K and half V.
template <int D>
__global__ void __launch_bounds__(kWarps * 32) append_few_kernel(CacheView c, CacheBatch b, int seq, Rows k, Rows v) {
  constexpr int NG = D / kGroup;
  grid_dependency_wait();
  grid_launch_dependents();
  const int lane = threadIdx.x % 32, work = blockIdx.x * kWarps + threadIdx.x / 32;
  const int j = work / c.heads_kv, head = work % c.heads_kv, i = blockIdx.y;
  if (j >= seq) return;
  int slot, count;
  const int len = checked_length(c, b, i, seq, lane, work == 0, slot, count);
  if (len < 0 || j >= count) return;
  const int pos = len - count + j, token = pos % kUnitTokens, m = lane % (D / 4);
  // under way while the page and its count are looked up
  const unsigned char *rk = k.data + i * k.batch + head * k.head + j * k.seq + m * 8;
  const unsigned char *rv = v.data + i * v.batch + head * v.head + j * v.seq + m * 8;
  constexpr int kPasses = D == 64 ? 1 : 2;
  uint2 x[kPasses];
  if (D == 64) {
    x[0] = *reinterpret_cast<const uint2 *>(lane < 16 ? rk : rv);
  } else {
    x[0] = *reinterpret_cast<const uint2 *>(rk);
    x[kPasses - 1] = *reinterpret_cast<const uint2 *>(rv);
  }
  unsigned char *out = own_unit_in(c, page_of(c, slot, pos), pos, head, unit_bytes(D), lane);
  if (!out) return;
#pragma unroll 1
  for (int pass = 0; pass < kPasses; ++pass) {
    const uint32_t w[2] = {pass ? x[kPasses - 1].x : x[0].x, pass ? x[kPasses - 1].y : x[0].y};
    const uint32_t lo = bf16_min2(w[0], w[1]), hi = bf16_max2(w[0], w[1]) ^ 0x80008000u;
    uint32_t e = bf16_min2(__byte_perm(lo, hi, 0x5410), __byte_perm(lo, hi, 0x7632));
#pragma unroll
    for (int bit = 1; bit <= 8; bit <<= 1) e = extremes_over(e, bit);
    const Scale s = make_scale(e);
    const bool value = D == 64 ? lane >= 16 : pass == 1;
    *reinterpret_cast<uint16_t *>(out + (value ? value_place<NG>(token, m) : key_place<NG>(token, m))) = uint16_t(codes_of<4>(w, s));
    if (m % 16 == 0) *reinterpret_cast<uint32_t *>(out + scale_place<NG>(token, m / 16) + (value ? NG * 64 : 0)) = s.pair;
  }
}

// Nibbles 0, 4 / 1, 5 / 2, 6 / 3, 7 of a word as four pairs of fp16: the subnormals u 2^-24, and u 2^-20 where the nibble stands four
// bits up.
__device__ __forceinline__ void codes_to_half2(uint32_t w, __half2 (&out)[4]) {
  const uint32_t x[4] = {w & 0x000f000fu, w & 0x00f000f0u, w >> 8 & 0x000f000fu, w >> 8 & 0x00f000f0u};
#pragma unroll
  for (int i = 0; i < 4; ++i) out[i] = *reinterpret_cast<const __half2 *>(&x[i]);
}
__device__ __forceinline__ float value_of(float scale, float code, float zero) { return __fmaf_rn(scale, code, zero); }
constexpr float kEven = 16777216.f, kOdd = 1048576.f;  // what a scale is multiplied by for these

// Bound by the latency of what follows one another and by instructions: a warp's units are asked for together.
template <int D>
__global__ void __launch_bounds__(kWarps * 32) read_kernel(CacheView c, const int32_t *slots, const int32_t *begins, int seq,
                                                            int warps_a_head, Rows k, Rows v) {
  constexpr int NG = D / kGroup, U = kReadUnits;
  grid_dependency_wait();
  grid_launch_dependents();
  const int lane = threadIdx.x % 32, g = lane / 4, t = lane % 4;
  const int work = blockIdx.x * kWarps + threadIdx.x / 32;
  const int head = work / warps_a_head, nth = work % warps_a_head, i = blockIdx.y;
  if (head >= c.heads_kv) return;
  const int slot = slot_of(c, slots, i), begin = begins ? begins[i] : 0;
  const int64_t first64 = (int64_t(max(begin, 0)) / kUnitTokens + int64_t(nth) * U) * kUnitTokens;
  const int len = c.lens[max(slot, 0)];  // asked for together with the pages
  int page[U];
#pragma unroll
  for (int u = 0; u < U; ++u) page[u] = page_of(c, max(slot, 0), first64 + u * kUnitTokens);
  if (slot < 0 || begin < 0 || len < 0 || len > max_tokens(c)) {
    if (work == 0 && lane == 0) report(c.status, STEEL_ERR_INVALID_ARG);
    return;
  }
  const int end = int(min(int64_t(len), int64_t(begin) + seq));
  if (first64 >= end) return;

  uint4 ck[U][NG], cv[U][NG];
  __half2 sk[U][2][NG], sv[U][2][2][NG];  // [h][n], [f][h][n]
  bool there[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int first = int(first64) + u * kUnitTokens;
    const unsigned char *in = first < end ? unit_in(c, page[u], first, head, unit_bytes(D), lane) : nullptr;
    there[u] = in != nullptr;
    if (!in) continue;
#pragma unroll
    for (int n = 0; n < NG; ++n) {
      ck[u][n] = load16(in + n * 512 + lane * 16);
      cv[u][n] = load16(in + NG * 512 + n * 512 + lane * 16);
    }
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int n = 0; n < NG; ++n) {
        sk[u][h][n] = *reinterpret_cast<const __half2 *>(in + NG * 1024 + ((g * 2 + h) * NG + n) * 4);
#pragma unroll
        for (int f = 0; f < 2; ++f)
          sv[u][f][h][n] = *reinterpret_cast<const __half2 *>(in + NG * 1088 + (((2 * t + f) * 2 + h) * NG + n) * 4);
      }
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    if (!there[u]) continue;
    const int first = int(first64) + u * kUnitTokens, from = max(begin - first, 0), to = min(end - first, kUnitTokens);
    unsigned char *rk = k.data + i * k.batch + head * k.head + int64_t(first - begin) * k.seq;
    unsigned char *rv = v.data + i * v.batch + head * v.head + int64_t(first - begin) * v.seq;
#pragma unroll
    for (int n = 0; n < NG; ++n) {
      const uint32_t word[2][2] = {{ck[u][n].x, ck[u][n].y}, {ck[u][n].z, ck[u][n].w}};  // [c][h]
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int token = 8 * h + g;
        const float scale = __low2float(sk[u][h][n]), zero = __high2float(sk[u][h][n]), even = scale * kEven, odd = scale * kOdd;
#pragma unroll
        for (int a = 0; a < 2; ++a) {
          __half2 x[4];
          codes_to_half2(word[a][h], x);
          uint32_t o[4];
#pragma unroll
          for (int j = 0; j < 4; ++j) {  // channels 2j, 2j + 1: nibbles 2j % 4 and 2j % 4 + 1 of a half
            const float lo = j < 2 ? __low2float(x[2 * j]) : __high2float(x[2 * j - 4]);
            const float hi = j < 2 ? __low2float(x[2 * j + 1]) : __high2float(x[2 * j - 3]);
            o[j] = pack_bf16x2(value_of(even, lo, zero), value_of(odd, hi, zero));
          }
          if (token >= from && token < to)
            *reinterpret_cast<uint4 *>(rk + token * k.seq + (kGroup * n + 32 * a + 8 * t) * 2) = make_uint4(o[0], o[1], o[2], o[3]);
        }
      }
      const uint32_t pairs[2][2] = {{cv[u][n].x, cv[u][n].y}, {cv[u][n].z, cv[u][n].w}};  // [h][y], the halves are the tokens
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        __half2 x[2][4];
        codes_to_half2(pairs[h][0], x[0]);
        codes_to_half2(pairs[h][1], x[1]);
#pragma unroll
        for (int f = 0; f < 2; ++f) {
          const int token = 8 * h + 2 * t + f;
          const float scale = __low2float(sv[u][f][h][n]), zero = __high2float(sv[u][f][h][n]), even = scale * kEven,
                      odd = scale * kOdd;
          uint32_t o[4];
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const __half2 p = x[j / 2][j % 2 * 2], q = x[j / 2][j % 2 * 2 + 1];
            o[j] = pack_bf16x2(value_of(even, f ? __high2float(p) : __low2float(p), zero),
                               value_of(odd, f ? __high2float(q) : __low2float(q), zero));
          }
          if (token >= from && token < to)
            *reinterpret_cast<uint4 *>(rv + token * v.seq + (kGroup * n + 8 * g) * 2) = make_uint4(o[0], o[1], o[2], o[3]);
        }
      }
    }
  }
}

template <int D>
__global__ void __launch_bounds__(kWarps * 32) read_few_kernel(CacheView c, const int32_t *slots, const int32_t *begins, int seq, Rows k,
                                                                Rows v) {
  constexpr int NG = D / kGroup;
  grid_dependency_wait();
  grid_launch_dependents();
  const int lane = threadIdx.x % 32, work = blockIdx.x * kWarps + threadIdx.x / 32;
  const int j = work / c.heads_kv, head = work % c.heads_kv, i = blockIdx.y;
  if (j >= seq) return;
  const int slot = slot_of(c, slots, i), begin = begins ? begins[i] : 0;
  const int len = c.lens[max(slot, 0)], page = page_of(c, max(slot, 0), int64_t(max(begin, 0)) + j);  // asked for together
  if (slot < 0 || begin < 0 || len < 0 || len > max_tokens(c)) {
    if (work == 0 && lane == 0) report(c.status, STEEL_ERR_INVALID_ARG);
    return;
  }
  if (begin >= len - j) return;
  const int pos = begin + j, token = pos % kUnitTokens, m = lane % (D / 4);
  const unsigned char *in = unit_in(c, page, pos, head, unit_bytes(D), lane);
  if (!in) return;
  constexpr int kPasses = D == 64 ? 1 : 2;
#pragma unroll
  for (int pass = 0; pass < kPasses; ++pass) {
    const bool value = D == 64 ? lane >= 16 : pass == 1;
    const uint32_t codes = *reinterpret_cast<const uint16_t *>(in + (value ? value_place<NG>(token, m) : key_place<NG>(token, m)));
    const __half2 pair = *reinterpret_cast<const __half2 *>(in + scale_place<NG>(token, m / 16) + (value ? NG * 64 : 0));
    const float scale = __low2float(pair), zero = __high2float(pair);
    uint32_t o[2];
#pragma unroll
    for (int n = 0; n < 2; ++n)
      o[n] = pack_bf16x2(value_of(scale, float(codes >> (8 * n) & 15u), zero), value_of(scale, float(codes >> (8 * n + 4) & 15u), zero));
    const Rows &to = value ? v : k;
    *reinterpret_cast<uint2 *>(to.data + i * to.batch + head * to.head + j * to.seq + m * 8) = make_uint2(o[0], o[1]);
  }
}

// Units that `seq` tokens can touch, wherever they begin.
int units_of(int seq) { return (seq + kUnitTokens - 2) / kUnitTokens + 1; }

// Whether a warp takes a token and not a unit: where tokens are few altogether, because units take longer from their first access to their
// last, or a sequence has few, because most of a unit would be idle.  By tokens and by units, 8 heads, in us:
//   writing  head_dim 128: 64 x 16 tokens 5.6 and 8.6, 256 x 12 12.8 and 10.1, 512 x 4 9.2 and 15.4, 512 x 8 16.4 and 15.9;
//            head_dim 64: 32 x 16 2.8 and 5.4, 256 x 12 10.1 and 6.5, 512 x 4 7.3 and 10.3, 512 x 8 12.9 and 9.9
//   reading  head_dim 128: 64 x 4 2.1 and 2.2, 64 x 8 2.7 and 2.3, 512 x 2 3.9 and 5.2, 512 x 4 5.9 and 5.1;
//            head_dim 64: 32 x 8 2.0 and 2.0, 64 x 8 2.4 and 2.0, 512 x 2 3.7 and 3.7, 512 x 4 5.8 and 3.7
bool writes_few(const CacheView &c, int head_dim, int batch, int seq) {
  return seq <= (head_dim == 64 ? 6 : 8) || int64_t(batch) * seq * c.heads_kv <= 64 * head_dim;
}
bool reads_few(const CacheView &c, int batch, int seq) { return seq <= 2 || int64_t(batch) * seq * c.heads_kv <= 2048; }

}  // namespace

cudaError_t launch_append(const CacheView &c, int head_dim, const CacheBatch &b, int seq, const Rows &k, const Rows &v,
                          cudaStream_t stream) {
  if (writes_few(c, head_dim, b.batch, seq)) {
    const dim3 grid((int64_t(seq) * c.heads_kv + kWarps - 1) / kWarps, b.batch);
    return launch_overlapping(head_dim == 64 ? append_few_kernel<64> : append_few_kernel<128>, grid, dim3(kWarps * 32), 0, stream, c,
                              b, seq, k, v);
  }
  const int units = units_of(min(seq, c.max_pages << c.page_shift));
  const dim3 grid((int64_t(units) * c.heads_kv + kWarps - 1) / kWarps, b.batch);
  return launch_overlapping(head_dim == 64 ? append_kernel<64> : append_kernel<128>, grid, dim3(kWarps * 32), 0, stream, c, b,
                            seq, units, k, v);
}

cudaError_t launch_read(const CacheView &c, int head_dim, const int32_t *slots, const int32_t *begin, int batch, int seq,
                        const Rows &k, const Rows &v, cudaStream_t stream) {
  if (reads_few(c, batch, seq)) {
    const dim3 grid((int64_t(seq) * c.heads_kv + kWarps - 1) / kWarps, batch);
    return launch_overlapping(head_dim == 64 ? read_few_kernel<64> : read_few_kernel<128>, grid, dim3(kWarps * 32), 0, stream, c,
                              slots, begin, seq, k, v);
  }
  const int warps = (units_of(min(seq, c.max_pages << c.page_shift)) + kReadUnits - 1) / kReadUnits;  // of a head
  const dim3 grid((int64_t(warps) * c.heads_kv + kWarps - 1) / kWarps, batch);
  return launch_overlapping(head_dim == 64 ? read_kernel<64> : read_kernel<128>, grid, dim3(kWarps * 32), 0, stream, c, slots,
                            begin, seq, warps, k, v);
}

}  // namespace steel
