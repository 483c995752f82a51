// Attention of many query rows over a whole cache (prefix and cross attention), none of its tokens masked but those behind a
// sequence's length.  tcgen05 products; a CTA takes 128 rows (tokens x sequences x heads of a kv head) and a range of 64-token
// tiles of one (sequence, kv head) of the cache.
//
// The codes become operands without a rounding: with c in 0 .. 3, c s + z = s (c - 1) + (z + s), and s (c - 1), one of -s, 0, s,
// 2 s, is a half-precision number when s is (1-bit codes: s c + z).  The rest does not depend on the token (keys: within a
// group of tokens) or on the channel (values: within a group of channels), so it is a few more rows of the same operand:
//
//   S = Q [s (c - 1) | z, s of the token groups]                    128 + 16 columns, fp32
//   O += P [s (c - o) | z, o s of the channel groups | 1]           head_dim + 16 columns, fp32; the last one sums P
//
// o is 1 for even tokens, 2 for odd ones (1-bit values: 0 and 1).  Every addition of the tensor core to O drops what lies below
// the sum's last digit, always in one direction, and a sum over P of terms with a mean is a multiple of the result where that
// averages many tokens: with one o for all the codes' part has one, and z and o s each do.  So half precision takes z + o s,
// which then has none, as two rows hi + lo.  16 tokens at 40000, half precision, error in the result's norm, whose own rounding is
// 2.07e-4: 2.61e-4 with o = 1, z and s; 2.45e-4 with hi + lo alone; 2.07e-4 with both.
//
// Where 2 s would pass half precision's largest number (s above 32752), the operand holds a quarter of all that, and its product is
// made four times (keys: of a batch, values: of a tile).  Exact but for s and z below 2^-12 beside such scales.
//
// Q: half precision, scaled by a power of two for each row (exact for bfloat16 down to 2^-16 of the row's largest element).
// P: the softmax numerators times 2^R_PEXP, in half precision, rounded for bfloat16 results (2e-4 of the result's norm, an eighth
// of the result's own rounding; divided by the sum of the rounded P), as pairs hi + lo, a product each, for half-precision ones.
// Q and P are A operands in tensor memory.  Against pairs of codes and numerators, as the chunk kernel has them, that is 576
// (half precision: 864) in place of 1280 cycles of the tensor pipe for 64 tokens, and half the expansion.
//
// Tokens go in batches of 128, two tiles each, with two S.  Four groups of four softmax warps (thread = row = lane of tensor
// memory) take the tiles in turn: a warp's steps are short and wait for one another, so it takes several to fill the SM.  The
// softmax reference of a row is passed from group to group in the order of the tiles, before the exponentials, and is raised
// only when a logit exceeds it by R_TAU (log2 units), which takes a pass over O.  P takes columns of its S.  Eight warps expand
// (four keys, four values), one issues products, one copies packed data.  Window tokens go into the same operands as they are,
// bfloat16 ones scaled by a power of two for each batch.
//
// Bound: not one pipe, but two chains of latencies that compete for issue slots (60 to 70 % of them, tensor pipe 41 %).  A batch of
// 128 tokens takes 1.23 to 1.33 us a CTA, 2400 cycles (head_dim 128, bfloat16; half precision 1.51 to 1.59; head_dim 64 1.05 to
// 1.13 and 1.26 to 1.36), whether 17 or 128 rows exist, and a launch 8 to 9 us more (half precision, head_dim 64: 5 to 7).  Cycles
// of a batch: the products 1152 (half precision 1728).  S from its issue to the softmax warps 870,
// the search 900, the turn 500, the numerators 1700, to the issuing warp 250, and two batches are in flight.  The expansion of a
// batch's keys 2000 and 600 until the next one, values the same.  In copies: half of the expansion left out 0.57 us a tile for
// 0.63.  Measured and not kept, us a tile against 0.62: three expanding groups of four warps that take keys and values in turn 0.64;
// products and barriers of S a tile at a time, so that the next S waits for one tile's numerators 0.66, with three groups 0.76;
// 32 columns of S kept in registers through the turn 0.64; numerators by single multiply-adds 0.65; runs of tiles over several
// streams for 148 resident CTAs 0.69 (prompts of 100 tokens behind 16k 2 % faster, 200 tokens behind 6404 11 % slower).
// Before: two softmax groups 0.69, one for all 128 tokens 0.83, an O and a reference for each of two groups 0.89.
//
// Every wait on an mbarrier is bounded, as in the chunk kernel: a thread that gives up sets a flag that ends the others' waits,
// and the CTA reports through the status word.
#pragma once
#include "xq_internal.h"
#include "xq_layout.cuh"
#include "xq_mma.cuh"

namespace xq {
namespace {

constexpr int RB = XQ_BATCH;     // tokens of a batch
constexpr int RT = 64;           // of a tile, half a batch
constexpr int R_BUFS = 2;        // expanded batches of keys, of values
constexpr int R_RAW = 4;         // packed batches in flight
constexpr float R_TAU = 8.f;
constexpr int R_PEXP = 7;        // numerators are at most 2^(R_PEXP + R_TAU) as fp16
constexpr int R_GROUPS = 4;      // softmax groups of four warps, 0 .. 15
constexpr int R_EXPAND = 4;      // expanding warps of a kind: keys 16 .. 19, values 20 .. 23
constexpr int R_MMA = 24, R_LOAD = 25, R_THREADS = 26 * 32;
constexpr int R_UNITS = 4;       // window batches whose exponents are kept
constexpr uint32_t MAX_DOUBLED = 0x77ff;  // the largest half-precision number whose double is finite
constexpr uint32_t QUARTERS = 0x34003400;  // two of 1 / 4

// shared-memory matrix descriptor, K-major, 128-byte swizzle: rows of 128 bytes, groups of eight 1024 bytes apart
__device__ __forceinline__ uint64_t rows_desc(uint32_t addr) {
  return (uint64_t)((addr >> 4) & 0x3fff) | (uint64_t)1 << 16 | (uint64_t)(1024 >> 4) << 32 | (uint64_t)1 << 46 | (uint64_t)2 << 61;
}
// kind::f16 instruction descriptor: fp16 A and B, both K-major, fp32 accumulate, M = 128
__host__ __device__ constexpr uint32_t rows_idesc(int n) { return (1u << 4) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(128 >> 4) << 24); }
// D[128 x N] (+)= A[128 x 16] (tensor memory) * B[N x 16]^T (shared memory); issued by one thread
__device__ __forceinline__ void rows_mma(uint32_t d_tmem, uint32_t a_tmem, uint64_t b_desc, uint32_t idesc, bool accumulate) {
  asm volatile(
      "{\n.reg .pred p;\nsetp.ne.b32 p, %4, 0;\n"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n}\n" ::"r"(d_tmem),
      "r"(a_tmem), "l"(b_desc), "r"(idesc), "r"((uint32_t)accumulate) : "memory");
}
__device__ __forceinline__ void rows_commit(uint32_t bar) {
  asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n" ::"r"(bar) : "memory");
}
__device__ __forceinline__ uint32_t hadd2(uint32_t a, uint32_t b) {
  uint32_t d;
  asm("add.rn.f16x2 %0, %1, %2;\n" : "=r"(d) : "r"(a), "r"(b));
  return d;
}

__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {  // two fp32 fused multiply-adds
  uint64_t d;
  asm("fma.rn.f32x2 %0, %1, %2, %3;\n" : "=l"(d) : "l"(a), "l"(b), "l"(c));
  return d;
}
__device__ __forceinline__ uint64_t pair_of(float lo, float hi) {
  uint64_t d;
  asm("mov.b64 %0, {%1, %2};\n" : "=l"(d) : "f"(lo), "f"(hi));
  return d;
}
__device__ __forceinline__ float2 halves_of(uint64_t a) {
  float2 d;
  asm("mov.b64 {%0, %1}, %2;\n" : "=f"(d.x), "=f"(d.y) : "l"(a));
  return d;
}
// one lane's arrival, without a branch
__device__ __forceinline__ void arrive_if(bool p, uint32_t bar) {
  asm volatile("{\n.reg .pred p;\nsetp.ne.u32 p, %1, 0;\n@p mbarrier.arrive.shared::cta.b64 _, [%0];\n}\n" ::"r"(bar), "r"((uint32_t)p) : "memory");
}
// barriers of the softmax warps; of the loading warp, which has initialised the mbarriers, with the expanding warps; and with
// the others
__device__ __forceinline__ void softmax_sync() { asm volatile("bar.sync 1, %0;\n" ::"n"(R_GROUPS * 128) : "memory"); }
__device__ __forceinline__ void expand_sync() { asm volatile("bar.sync 2, %0;\n" ::"n"((2 * R_EXPAND + 1) * 32) : "memory"); }
__device__ __forceinline__ void start_sync() { asm volatile("bar.sync 3, %0;\n" ::"n"(R_GROUPS * 128 + 64) : "memory"); }
// A warp's bounded wait.  What follows when the first look fails is out of line: most looks do not, and the kernel's roles
// share an instruction cache.
__device__ __noinline__ bool warp_wait_longer(uint32_t bar, uint32_t parity, volatile int* dead) {
  return __all_sync(0xffffffffu, mbar_wait(bar, parity, dead));
}
__device__ __forceinline__ bool warp_wait(uint32_t bar, uint32_t parity, volatile int* dead) {
  return __all_sync(0xffffffffu, mbar_try_wait(bar, parity) != 0u) || warp_wait_longer(bar, parity, dead);
}

// two of them, looked at together
__device__ __forceinline__ bool warp_wait_both(uint32_t bar0, uint32_t parity0, uint32_t bar1, uint32_t parity1, volatile int* dead) {
  const uint32_t there0 = mbar_try_wait(bar0, parity0), there1 = mbar_try_wait(bar1, parity1);
  return __all_sync(0xffffffffu, (there0 & there1) != 0u) || (warp_wait_longer(bar0, parity0, dead) && warp_wait_longer(bar1, parity1, dead));
}

template <int D, int BK, int BV, int GS>
struct RowsLayout {
  static constexpr int NG = D / GS;
  static constexpr int KROW = D * BK / 8;              // packed bytes of a token's keys
  static constexpr int KN = RB + 16, VN = D + 16;      // rows of the operands: tokens and 16 more, channels and 16 more
  // an operand: blocks of 128-byte rows (64 channels of the keys, 64 tokens of the values)
  static constexpr int KBLOCK = KN * 128, KBYTES = D / 64 * KBLOCK, VBLOCK = VN * 128, VBYTES = RB / 64 * VBLOCK;
  // rows of the value operand, and columns of O, behind the channels: z of the channel groups; s, which only the expanding
  // warps read; ones, which sum P; o s (half precision: the sum of z and o s, rounded, and what the rounding left off)
  static constexpr int ZERO = D, SCALE = D + NG, ONES = D + 8, REST = D + 9;
  // a raw stage: key codes, key parameters, value codes, value parameters of a batch
  static constexpr int RAW_KM = RB * KROW, RAW_VC = RAW_KM + RB / GS * 4 * D, RAW_VM = RAW_VC + 16 * D * BV;
  static constexpr int RAW = RAW_VM + RB * 4 * NG;
  static constexpr int OFF_V = R_BUFS * KBYTES, OFF_RAW = OFF_V + R_BUFS * VBYTES, TOTAL = OFF_RAW + R_RAW * RAW;
  static_assert(KBLOCK % 1024 == 0 && VBLOCK % 1024 == 0 && RAW % 16 == 0, "alignment");
  static_assert(TOTAL + 1024 <= 226 * 1024, "shared memory");
  // tensor memory columns
  static constexpr uint32_t COL_Q = 0, COL_O = D / 2, COL_S = COL_O + VN;
  static_assert(COL_S + 2 * KN <= 512, "tensor memory");
};

// First column of the numerators of tokens 16 ks .. of a tile: in the place of their S, 32 tokens in 16 columns, half precision
// rests 16 columns on
__host__ __device__ constexpr uint32_t p_col(int ks) { return 32 * (ks >> 1) + 8 * (ks & 1); }

// The byte of 16-byte piece `piece` of an operand row, from the operand's start
__device__ __forceinline__ uint32_t piece_at(int row, int piece) { return (uint32_t)(row * 128 + ((piece ^ (row & 7)) << 4)); }

// Sixteen codes, four fields (at bits 0, BITS, 2 BITS, 3 BITS of every byte of w) of four bytes each, less OFFSET (the second
// and the fourth of a field's bytes: less ODD), times the scales of their pairs.  A field becomes a half-precision number
// beside an exponent whose last places it takes: 2^(10 - BITS j) + c.
template <int BITS, int OFFSET>
__device__ __forceinline__ uint32_t code_times(uint32_t w, int j, uint32_t s, uint32_t field) {
  const uint32_t base = 0x64006400u - 0x04000400u * (BITS * j);                        // 2^(10 - BITS j)
  const uint32_t less = (base | 0x80008000u) + OFFSET * (0x00010001u << (BITS * j));   // and OFFSET more
  return hmul2(hadd2((w & field) | base, less), s);
}
template <int OFF>
__device__ __forceinline__ void sts128_at(uint32_t a, uint32_t x, uint32_t y, uint32_t z, uint32_t w) {
  asm volatile("st.shared.v4.u32 [%0 + %5], {%1,%2,%3,%4};\n" ::"r"(a), "r"(x), "r"(y), "r"(z), "r"(w), "n"(OFF) : "memory");
}
template <int OFF>
__device__ __forceinline__ uint32_t lds32_at(uint32_t a) {
  uint32_t v;
  asm volatile("ld.shared.u32 %0, [%1 + %2];\n" : "=r"(v) : "r"(a), "n"(OFF) : "memory");
  return v;
}
template <int BITS, int OFFSET, int ODD, int OFF>
__device__ __forceinline__ void expand16(uint32_t w, const uint4& s0, const uint4& s1, uint32_t dst0, uint32_t dst1, const uint32_t (&f)[4]) {
  const uint32_t y = w >> 8;
  sts128_at<OFF>(dst0, code_times<BITS, OFFSET>(w, 0, s0.x, f[0]), code_times<BITS, ODD>(y, 0, s0.y, f[0]), code_times<BITS, OFFSET>(w, 1, s0.z, f[1]), code_times<BITS, ODD>(y, 1, s0.w, f[1]));
  sts128_at<OFF>(dst1, code_times<BITS, OFFSET>(w, 2, s1.x, f[2]), code_times<BITS, ODD>(y, 2, s1.y, f[2]), code_times<BITS, OFFSET>(w, 3, s1.z, f[3]), code_times<BITS, ODD>(y, 3, s1.w, f[3]));
}
// N rows of them, eight rows apart (1024 bytes of the operand), packed words STRIDE bytes apart; shift: of 1-bit codes' words
template <int N, int STRIDE, int K = 0>
__device__ __forceinline__ void load_codes(uint32_t src, uint32_t (&w)[N]) {
  if constexpr (K < N) {
    w[K] = lds32_at<K * STRIDE>(src);
    load_codes<N, STRIDE, K + 1>(src, w);
  }
}
template <int BITS, int OFFSET, int ODD, int N, int K = 0>
__device__ __forceinline__ void expand_rows(const uint32_t (&w)[N], int shift, const uint4& s0, const uint4& s1, uint32_t dst0, uint32_t dst1, const uint32_t (&f)[4]) {
  if constexpr (K < N) {
    expand16<BITS, OFFSET, ODD, 1024 * K>(BITS == 2 ? w[K] : w[K] >> shift, s0, s1, dst0, dst1, f);
    expand_rows<BITS, OFFSET, ODD, N, K + 1>(w, shift, s0, s1, dst0, dst1, f);
  }
}
// eight 16-bit numbers times f, as half precision in the operands' order: elements (0, 2), (1, 3), (4, 6), (5, 7)
template <bool F16>
__device__ __forceinline__ uint4 reorder8(const uint4& v, float f) {
  if (F16) return make_uint4(__byte_perm(v.x, v.y, 0x5410), __byte_perm(v.x, v.y, 0x7632), __byte_perm(v.z, v.w, 0x5410), __byte_perm(v.z, v.w, 0x7632));
  auto lo = [&](uint32_t x) { return __uint_as_float(x << 16) * f; };
  auto hi = [&](uint32_t x) { return __uint_as_float(x & 0xffff0000u) * f; };
  return make_uint4(pack_io2<true>(lo(v.x), lo(v.y)), pack_io2<true>(hi(v.x), hi(v.y)), pack_io2<true>(lo(v.z), lo(v.w)), pack_io2<true>(hi(v.z), hi(v.w)));
}
// running maximum of magnitudes, two 16-bit patterns at once
__device__ __forceinline__ uint32_t top_of(uint32_t m, const uint4& v) {
  return __vmaxu2(__vmaxu2(__vmaxu2(m, v.x & 0x7fff7fffu), __vmaxu2(v.y & 0x7fff7fffu, v.z & 0x7fff7fffu)), v.w & 0x7fff7fffu);
}
__device__ __forceinline__ float bf16_top(uint32_t m) { return __uint_as_float(max(m & 0xffffu, m >> 16) << 16); }

// whether one of the scales in two halves, in any lane's, is too large to be doubled
__device__ __forceinline__ bool any_large(uint32_t scales) {
  return __any_sync(0xffffffffu, max(scales & 0xffffu, scales >> 16) > MAX_DOUBLED);
}

// exponent that puts a window batch's largest magnitude into the range of half precision, 0 where it is there; at most `most`
// (126: its power of two and the inverse are normal numbers)
__device__ __forceinline__ int window_exponent(float mx, int most) {
  return min((mx >= 0.0625f && mx < 32768.f) || !(mx > 0.f) ? 0 : 14 - exponent_of(mx), most);
}
// 2^e for e from -256 to 127, 0 below the normal numbers
__device__ __forceinline__ float pow2_or_zero(int e) { return e < -126 ? 0.f : pow2i(e); }
// What the exponent of a window batch's values may exceed that of any batch before it by, packed ones (0) among them.  O is
// brought to it: without a batch's own scale its sums are below 2^64 (numerators 2^15, values 2^18, 2^31 tokens), and so stay
// below 2^124.  Smaller values have an error of up to 2^-85 of the largest ones before them.
constexpr int R_RISE = 60;

// Eight rows of 16 LANES bytes from shared memory, 16 bytes apart more than that: a warp's, the first one `first`.  to_row: of
// lane k, where row `first` + k goes, in strides.
template <int LANES>
__device__ __forceinline__ void store_rows(uint32_t from, uint8_t* to, size_t stride, uint32_t to_row, int first, int n_rows, int lane) {
  constexpr int AT_ONCE = 32 / LANES;
#pragma unroll
  for (int k = 0; k < 8 / AT_ONCE; ++k) {
    const int y = k * AT_ONCE + lane / LANES;
    const uint32_t row = __shfl_sync(0xffffffffu, to_row, y);
    const uint4 v = lds128(from + (first + y) * (16 * LANES + 16) + lane % LANES * 16);
    if (first + y < n_rows) *reinterpret_cast<uint4*>(to + row * stride + lane % LANES * 16) = v;
  }
}

// The sequence with the k-th longest length (of n <= 32; among equals the first).  All lanes of a warp.
__device__ __forceinline__ int by_length(const int* lengths, int n, int S, int k, int lane) {
  const int mine = lane < n ? max(0, min(S, lengths[lane])) : -1;
  int rank = 0;
  for (int j = 0; j < n; ++j) {
    const int other = __shfl_sync(0xffffffffu, mine, j);
    rank += other > mine || (other == mine && j < lane);
  }
  return __ffs(__ballot_sync(0xffffffffu, lane < n && rank == k)) - 1;
}

template <int D, int BK, int BV, int GS, bool F16>
__global__ void __launch_bounds__(R_THREADS, 1) rows_kernel(const __grid_constant__ RowsParams p) {
  using Ly = RowsLayout<D, BK, BV, GS>;
  constexpr int NG = Ly::NG;
  extern __shared__ uint8_t smem_raw[];
  __shared__ __align__(8) unsigned long long bar_mem[2 * R_RAW + 4 * R_BUFS + 2 + 2 * 4 + 4 * R_GROUPS + 3 * R_UNITS + 2];
  __shared__ float top_sm[R_GROUPS][ROWS_TILE], m_sm[ROWS_TILE];  // largest element of a quarter of a row of q; softmax reference
  __shared__ uint32_t unit_sm[R_UNITS][2][R_EXPAND];        // window batch, keys / values: largest magnitude of each expanding warp
  __shared__ volatile uint32_t quarter_sm[2][R_BUFS];       // keys, values: an expanded batch's parts (values: bits of its tiles) that are quarters
  __shared__ int value_e_sm[R_UNITS];                       // window batch: exponent of its values
  __shared__ uint32_t tmem_base_sm;
  __shared__ volatile int dead_sm;

  const Dims& dm = p.dm;
  const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), lane = tid & 31;
  const uint32_t sm = ((uint32_t)__cvta_generic_to_shared(smem_raw) + 1023u) & ~1023u;
  const uint32_t bars = (uint32_t)__cvta_generic_to_shared(&bar_mem[0]);
  const uint32_t bar_rfull = bars;                       // [R_RAW] a batch's packed data is there
  const uint32_t bar_rfree = bar_rfull + 8 * R_RAW;      // [R_RAW] all expanding warps are done with it
  const uint32_t bar_kfull = bar_rfree + 8 * R_RAW;      // [R_BUFS] a batch's keys are expanded
  const uint32_t bar_kfree = bar_kfull + 8 * R_BUFS;     // [R_BUFS] their products are complete
  const uint32_t bar_vfull = bar_kfree + 8 * R_BUFS;     // [R_BUFS] the same of the values
  const uint32_t bar_vfree = bar_vfull + 8 * R_BUFS;     // [R_BUFS]
  const uint32_t bar_s = bar_vfree + 8 * R_BUFS;         // [2] S of a batch is complete
  const uint32_t bar_p = bar_s + 16;                     // [2][2] the numerators of a batch's first / second tile are written
  const uint32_t bar_o = bar_p + 32;                     // [2][2] its value products are complete
  const uint32_t bar_turn = bar_o + 32;                  // [4 warps][R_GROUPS] the reference for a group's next tile is there
  const uint32_t bar_kunit = bar_turn + 32 * R_GROUPS;              // [R_UNITS] the magnitudes of a window batch's keys are known
  const uint32_t bar_vunit = bar_kunit + 8 * R_UNITS;    // [R_UNITS] the same of its values
  const uint32_t bar_ve = bar_vunit + 8 * R_UNITS;       // [R_UNITS] the exponent of its values is there
  const uint32_t bar_q = bar_ve + 8 * R_UNITS;           // Q is written
  const uint32_t bar_end = bar_q + 8;                    // every product is complete

  if (tid == 32 * R_LOAD) {
#pragma unroll
    for (int i = 0; i < R_RAW; ++i) {
      mbar_init(bar_rfull + 8 * i, 1);
      mbar_init(bar_rfree + 8 * i, 2 * R_EXPAND);
    }
#pragma unroll
    for (int i = 0; i < R_BUFS; ++i) {
      mbar_init(bar_kfull + 8 * i, R_EXPAND);
      mbar_init(bar_kfree + 8 * i, 1);
      mbar_init(bar_vfull + 8 * i, R_EXPAND);
      mbar_init(bar_vfree + 8 * i, 1);
    }
    mbar_init(bar_s, 1);
    mbar_init(bar_s + 8, 1);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      mbar_init(bar_p + 8 * i, 4);
      mbar_init(bar_o + 8 * i, 1);
#pragma unroll
      for (int k = 0; k < R_GROUPS; ++k) mbar_init(bar_turn + 8 * (R_GROUPS * i + k), 1);
    }
#pragma unroll
    for (int i = 0; i < R_UNITS; ++i) {
      mbar_init(bar_kunit + 8 * i, R_EXPAND);
      mbar_init(bar_vunit + 8 * i, R_EXPAND);
      mbar_init(bar_ve + 8 * i, 1);
    }
    mbar_init(bar_q, 4 * R_GROUPS);
    mbar_init(bar_end, 1);
    dead_sm = 0;
    asm volatile("fence.mbarrier_init.release.cluster;\n" ::: "memory");
  }
  const bool expands = warp >= 4 * R_GROUPS && warp < R_MMA;
  if (expands || warp == R_LOAD) expand_sync();
  // ---- the CTA's rows and batches ----
  const int G = dm.G;
  const int split = blockIdx.x % p.ns, rest = blockIdx.x / p.ns, rt = rest % p.row_tiles;
  int bh = rest / p.row_tiles, u = bh / dm.Hkv;
  const int hk = bh - u * dm.Hkv;
  const int row0 = rt * ROWS_TILE, n_rows = min(ROWS_TILE, p.T * p.each * G - row0);
  auto call_row = [&](int k) {  // of the stream's row row0 + k
    const int x = row0 + k, h = x % G, ji = x / G, i = ji % p.each, j = ji / p.each;
    return ((size_t)j * (dm.B * p.each) + (size_t)u * p.each + i) * dm.Hq + hk * G + h;
  };
  const int my_row = 8 * warp + (lane & 7);  // of q, for the warps that fetch it
  uint32_t my_call_row = warp < 4 * R_GROUPS && my_row < n_rows ? (uint32_t)call_row(my_row) : 0u;

  // (tensor memory is asked for after the wait: a CTA of the preceding kernel that shares the SM may still have to get its own;
  // late_wait: a decode kernel, whose CTAs have theirs when this one starts)
  if (!p.late_wait) grid_dependency_wait();
  grid_dependents_go();
  if (warp == R_MMA) tmem_alloc((uint32_t)__cvta_generic_to_shared(&tmem_base_sm), 512u);
  int n_q = p.n_q, r = p.r;
  if (p.longest_first) {
    u = by_length(p.lengths, dm.B, n_q + r, u, lane);
    bh = u * dm.Hkv + hk;
    if (warp < 4 * R_GROUPS && my_row < n_rows) my_call_row = (uint32_t)call_row(my_row);
  }
  if (p.lengths != nullptr) {
    const int S = max(0, min(n_q + r, p.lengths[u]));
    n_q = min(n_q, S);
    r = S - n_q;
  }
  const int pk_batches = (n_q + RB - 1) / RB, all_batches = pk_batches + (r + RB - 1) / RB;
  int t_lo, t_hi;
  share_of(all_batches, p.ns, split, t_lo, t_hi);
  const int N = t_hi - t_lo;
  const int n_pk = max(0, min(t_hi, pk_batches) - t_lo);  // packed batches of the range; batch i is window batch i - n_pk
  // exponent of a window batch's keys (which = 0), of its values (1)
  auto batch_exponent = [&](int i, int which, int most) {
    const uint32_t* m = unit_sm[(i - n_pk) % R_UNITS][which];
    uint32_t x = 0u;
#pragma unroll
    for (int k = 0; k < R_EXPAND; ++k) x = max(x, m[k]);
    return F16 ? 0 : window_exponent(bf16_top(x), most);
  };
  auto value_exponent = [&](int i) { return F16 ? 0 : value_e_sm[(i - n_pk) % R_UNITS]; };

  // a batch's packed data into its raw stage
  auto load = [&](int i) {
    const uint32_t dst = sm + Ly::OFF_RAW + (i % R_RAW) * Ly::RAW, bar = bar_rfull + 8 * (i % R_RAW);
    const size_t t = (size_t)t_lo + i;
    mbar_expect_tx(bar, Ly::RAW);
    bulk_load(dst, reinterpret_cast<const uint8_t*>(p.L.k_codes) + (size_t)bh * ((size_t)dm.nq_cap * Ly::KROW) + t * (RB * Ly::KROW), RB * Ly::KROW, bar);
    bulk_load(dst + Ly::RAW_KM, reinterpret_cast<const uint8_t*>(p.L.k_meta) + (size_t)bh * ((size_t)(dm.nq_cap / GS) * (4 * D)) + t * (RB / GS * 4 * D), RB / GS * 4 * D, bar);
    bulk_load(dst + Ly::RAW_VC, reinterpret_cast<const uint8_t*>(p.L.v_codes) + (size_t)bh * ((size_t)dm.nq_cap * (D * BV / 8)) + t * (16 * D * BV), 16 * D * BV, bar);
    bulk_load(dst + Ly::RAW_VM, reinterpret_cast<const uint8_t*>(p.L.v_meta) + (size_t)bh * ((size_t)dm.nq_cap * 4 * NG) + t * (RB * 4 * NG), RB * 4 * NG, bar);
  };
  // Before the barrier: the first packed batches, and q's rows into the second key operand's place, eight rows a
  // warp, lanes along a row.
  constexpr int QROW = 2 * D + 16;
  static_assert(ROWS_TILE * QROW <= Ly::KBYTES, "q fits");
  const uint32_t q_sm = sm + Ly::KBYTES;
  if (warp == R_LOAD) {
    if (lane == 0)
      for (int i = 0; i < min(R_RAW, n_pk); ++i) load(i);
    __syncwarp();
  } else if (warp < 4 * R_GROUPS) {
    constexpr int PIECES = D / 8, AT_ONCE = 32 / PIECES, ROWS = ROWS_TILE / (4 * R_GROUPS);
    const int first = ROWS * warp;
    uint4 x[ROWS / AT_ONCE];
#pragma unroll
    for (int k = 0; k < ROWS / AT_ONCE; ++k) {
      const int y = k * AT_ONCE + lane / PIECES;
      const uint32_t at = __shfl_sync(0xffffffffu, my_call_row, y);
      x[k] = first + y < n_rows ? reinterpret_cast<const uint4*>(p.q)[(size_t)at * PIECES + lane % PIECES] : make_uint4(0u, 0u, 0u, 0u);
    }
#pragma unroll
    for (int k = 0; k < ROWS / AT_ONCE; ++k)
      sts128(q_sm + (first + k * AT_ONCE + lane / PIECES) * QROW + lane % PIECES * 16, x[k].x, x[k].y, x[k].z, x[k].w);
  }

  // (the expanding warps need nothing of this, the first batch is expanded meanwhile: with the stores below 70.7 -> 68.0 us for
  // eight samples of each of four prompts of 5000, two layers)
  uint32_t tbase = 0u;
  if (!expands) {
    tc_fence_before();
    start_sync();
    tc_fence_after();
    tbase = tmem_base_sm;
  }

  if (warp == R_MMA) {
    // ================= products: the loop is warp-uniform, one elected lane issues =================
    constexpr uint32_t IDK = rows_idesc(Ly::KN), IDV = rows_idesc(Ly::VN);
    const uint32_t tb = __shfl_sync(0xffffffffu, tbase, 0), smu = __shfl_sync(0xffffffffu, sm, 0);
    bool ok = warp_wait(bar_q, 0, &dead_sm);
    // values of batch i - 2, a tile at a time, then keys of batch i, whose S takes the place of those numerators
#pragma unroll 1
    for (int i = 0; ok && i < N + 2; ++i) {
      const int b = i & 1;
      const uint32_t turn = ((i >> 1) & 1) ^ 1;  // of what belongs to batch i - 2
      const uint32_t dS = tb + Ly::COL_S + b * Ly::KN;
      if (i >= 2) {
        ok = warp_wait(bar_vfull + 8 * b, turn, &dead_sm);
#pragma unroll 1
        for (int g = 0; ok && g < 2; ++g) {
          ok = warp_wait(bar_p + 16 * b + 8 * g, turn, &dead_sm);
          if (!ok) break;
          tc_fence_after();
          if (elect_one()) {
            const uint64_t v = rows_desc(smu + Ly::OFF_V + b * Ly::VBYTES + g * Ly::VBLOCK);
            const uint32_t P = dS + g * RT;
            auto product = [&](bool sum) {
              if constexpr (F16) {  // the rests first: a sum drops what lies below its own last digit
#pragma unroll
                for (int ks = 0; ks < RT / 16; ++ks) rows_mma(tb + Ly::COL_O, P + p_col(ks) + 16, v + 2 * ks, IDV, sum || ks > 0);
                sum = true;
              }
#pragma unroll
              for (int ks = 0; ks < RT / 16; ++ks) rows_mma(tb + Ly::COL_O, P + p_col(ks), v + 2 * ks, IDV, sum || ks > 0);
            };
            product(i > 2 || g > 0);
            if (BV == 2 && (quarter_sm[1][b] >> g & 1u)) {
#pragma unroll 1
              for (int k = 0; k < 3; ++k) product(true);
            }
            rows_commit(bar_o + 16 * b + 8 * g);
            if (g == 1) rows_commit(bar_vfree + 8 * b);
          }
          __syncwarp();
        }
        if (!ok) break;
      }
      if (i < N) {
        ok = warp_wait(bar_kfull + 8 * b, (i >> 1) & 1, &dead_sm);
        if (!ok) break;
        tc_fence_after();
        if (elect_one()) {
          const uint64_t k = rows_desc(smu + b * Ly::KBYTES);
          auto product = [&](bool sum) {
#pragma unroll
            for (int ks = 0; ks < D / 16; ++ks) rows_mma(dS, tb + Ly::COL_Q + 8 * ks, k + (ks / 4) * (Ly::KBLOCK / 16) + 2 * (ks % 4), IDK, sum || ks > 0);
          };
          product(false);
          if (BK == 2 && quarter_sm[0][b] != 0u) {
#pragma unroll 1
            for (int x = 0; x < 3; ++x) product(true);
          }
          rows_commit(bar_s + 8 * b);
          rows_commit(bar_kfree + 8 * b);
        }
        __syncwarp();
      }
    }
    if (elect_one()) {  // also after a wait gave up: no product is in flight when the memory it uses is given up
      rows_commit(bar_end);
      for (int k = 0; k < WAIT_LIMIT && !mbar_try_wait(bar_end, 0); ++k) {}
    }
    __syncwarp();
  } else if (warp == R_LOAD) {
    // ================= packed data, a batch at a time (the first ones are on their way) =================
    if (lane == 0) {
      int i = min(R_RAW, n_pk);
      for (; i < n_pk; ++i) {
        if (!mbar_wait(bar_rfree + 8 * (i % R_RAW), (i / R_RAW - 1) & 1, &dead_sm)) break;
        load(i);
      }
      // no copy may be in flight when the shared memory is released (nobody may have waited for them if a wait gave up)
      for (int k = max(0, i - R_RAW); k < i; ++k)
        for (int n = 0; n < WAIT_LIMIT && !mbar_try_wait(bar_rfull + 8 * (k % R_RAW), (k / R_RAW) & 1); ++n) {}
    } else if (N > n_pk) {
      // window rows of the range: into L2 before the expanding warps come to them
      const int w_lo = (t_lo + n_pk - pk_batches) * RB, w_hi = min(r, (t_hi - pk_batches) * RB);
      const char* wk = reinterpret_cast<const char*>(p.L.win_k + ((size_t)bh * dm.R + w_lo) * D);
      const char* wv = reinterpret_cast<const char*>(p.L.win_v + ((size_t)bh * dm.R + w_lo) * D);
      for (int x = (lane - 1) * 128; x < (w_hi - w_lo) * 2 * D; x += 31 * 128) {
        asm volatile("prefetch.global.L2 [%0];\n" ::"l"(wk + x));
        asm volatile("prefetch.global.L2 [%0];\n" ::"l"(wv + x));
      }
    }
    __syncwarp();
  } else if (warp >= 4 * R_GROUPS) {
    // ================= expansion: keys (warps 16 .. 19), values (20 .. 23) =================
    const int ew = warp & 3, o = lane & 3, sub = lane >> 2;  // a lane's sixteen elements of 64, and its row of eight
    const bool keys = warp < 4 * R_GROUPS + R_EXPAND;
    // Keys: 64 channels from 64 kb on of the 32 tokens of each of the slots slot0 .. slot0 + PARTS - 1.  Values: D / 4 channels
    // from v_c0 on, all of one channel group, of the tokens of either half of the batch.
    constexpr int PARTS = D / 64, STEPS = D / 32;
    const int kb = D == 128 ? ew & 1 : 0, slot0 = D == 128 ? ew & 2 : ew;
    const int v_c0 = ew * (D / 4), vg = v_c0 / GS;
    const int rz = keys ? RB + 2 * slot0 : Ly::ZERO + vg, rs = keys ? rz + 1 : Ly::SCALE + vg;  // operand rows of the zero-points and of the scales
    const int row = keys ? 32 * slot0 + sub : v_c0 + sub;
    const int shift = ((keys ? BK : BV) == 2 ? 0 : 4) * (o & 1);
    constexpr int PERK = 32 / BK, CB = Ly::KROW < 16 ? Ly::KROW : 16;
    const int word = (64 * kb + 16 * o) / PERK;
    // what a lane reads, from the raw stage's start, and writes, from the operand's
    const uint32_t code_off = keys ? slot0 * (32 * Ly::KROW) + word * 4 / CB * (32 * CB) + word * 4 % CB + sub * CB
                                   : Ly::RAW_VC + (BV == 2 ? o * 4 : o / 2 * 4) + (v_c0 + sub) * 16;
    const uint32_t meta_off = keys ? Ly::RAW_KM + 2 * (lane * (D / 32) + 2 * kb) : Ly::RAW_VM + lane * (4 * NG);
    const uint32_t op_off = keys ? kb * Ly::KBLOCK : Ly::OFF_V;
    const int at = (lane & ~3) | ((lane & 1) << 1) | ((lane >> 1) & 1);  // place of channel `lane`: elements of four 0, 2, 1, 3
    const uint32_t params_off = keys ? piece_at(rz, at >> 3) + 2 * (at & 7) : piece_at(lane & 2 ? rz : rs, lane >> 3) + ((lane >> 2) & 1) * 8 + (lane & 1) * 4;
    const uint32_t rest_off = piece_at(Ly::REST + vg, lane >> 3) + ((lane >> 2) & 1) * 8 + (lane & 1) * 4;  // values
    const uint32_t row_off = piece_at(row, 2 * o), scales_off = piece_at(rs, 2 * o);
    static_assert(PARTS <= 2 && RB % 8 == 0, "rows rz + 2 x: bit 1 of rz is clear where x can be 1");
    // the row that sums the numerators: of tile ew of a batch, ones, or quarters where the rest of the operand is
    auto write_ones = [&](int b, uint32_t ones) {
      if (lane < 8) sts128(sm + Ly::OFF_V + b * Ly::VBYTES + ew * Ly::VBLOCK + piece_at(Ly::ONES, lane), ones, ones, ones, ones);
    };
    if (!keys && ew < 2) {
      for (int b = 0; b < R_BUFS; ++b) write_ones(b, 0x3c003c00u);
      proxy_fence();
    }
    uint32_t quarter_ones = 0u;  // bit b: of buffer b they are quarters
    __syncwarp();
    // The codes' fields: an instruction has room for one constant and the expansion needs two, so these are kept in registers.
    // Where keys and values have one width the compiler does that (2-bit keys, 1-bit values, 128 rows: 0.644 -> 0.623 us a tile;
    // both 2-bit: 0.647 -> 0.661).
    uint32_t fields[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int bits = keys ? BK : BV;
      fields[j] = (bits == 2 ? 0x00030003u : 0x00010001u) << (bits * j);
      if (BK != BV) asm volatile("" : "+r"(fields[j]));
    }
    int most = n_pk > 0 ? R_RISE : 126;  // for the next window batch's exponent of the values
#pragma unroll 1
    for (int i = 0; i < N; ++i) {
      const int b = i & 1;
      const bool packed = i < n_pk;
      {
        // the batch's packed data, and the operand's place: free, and for the second keys not q's any more
        const uint32_t bar_raw = bar_rfull + 8 * (i % R_RAW), raw_turn = (i / R_RAW) & 1;
        const uint32_t bar_free = i >= R_BUFS ? (keys ? bar_kfree : bar_vfree) + 8 * b : bar_q;
        const uint32_t free_turn = i >= R_BUFS ? ((i >> 1) & 1) ^ 1 : 0u;
        const bool waits = i >= R_BUFS || (keys && i == 1);
        if (packed && waits) {
          if (!warp_wait_both(bar_raw, raw_turn, bar_free, free_turn, &dead_sm)) break;
        } else {
          if (packed && !warp_wait(bar_raw, raw_turn, &dead_sm)) break;
          if (waits && !warp_wait(bar_free, free_turn, &dead_sm)) break;
        }
      }
      const uint32_t raw = sm + Ly::OFF_RAW + (i % R_RAW) * Ly::RAW;
      const uint32_t dst = sm + op_off + b * (keys ? Ly::KBYTES : Ly::VBYTES);
      const int valid = n_q - (t_lo + i) * RB;  // tokens of a packed batch that exist
      uint32_t quarter = 0u;                    // keys: the batch is in quarters; values: bit x, tile x is
      if (packed && keys) {
        // parameters of channels 64 kb + lane and 32 more, side by side in the group's order, to the operand's rows
        uint32_t sw[PARTS], zw[PARTS];
#pragma unroll
        for (int x = 0; x < PARTS; ++x) {
          const uint32_t meta = raw + meta_off + (slot0 + x) * 32 / GS * (4 * D);
          sw[x] = lds32(meta);
          zw[x] = lds32_at<2 * D>(meta);
        }
        if constexpr (BK == 2) {
          // the largest of all the batch's scales (each of the four warps looks at all of them: they have to agree)
          uint32_t top = 0u;
#pragma unroll
          for (int x = 0; x < RB / GS; ++x) {
            if (x * GS < valid) {
              const uint32_t scales = raw + Ly::RAW_KM + x * (4 * D) + lane * (D / 16);
              if constexpr (D == 128) {
                const uint2 v = lds64(scales);
                top = __vmaxu2(top, __vmaxu2(v.x, v.y));
              } else {
                top = __vmaxu2(top, lds32(scales));
              }
            }
          }
          if (any_large(top)) {
            quarter = 1u;
#pragma unroll
            for (int x = 0; x < PARTS; ++x) {
              sw[x] = hmul2(sw[x], QUARTERS);
              zw[x] = hmul2(zw[x], QUARTERS);
            }
          }
        }
#pragma unroll
        for (int x = 0; x < PARTS; ++x) {
          // (rows rz + 2 x and the one after it: bits of a row's number are exclusive-ored into the place of its pieces)
          const uint32_t to_z = ((dst + params_off) ^ (32u * x)) + 256u * x, to_s = (to_z ^ 16u) + 128u;
          sts16(to_z, zw[x] & 0xffffu);
          sts16(to_z ^ 64u, zw[x] >> 16);  // four pieces on
          sts16(to_s, sw[x] & 0xffffu);
          sts16(to_s ^ 64u, sw[x] >> 16);
        }
        __syncwarp();
#pragma unroll 1
        for (int x = 0; x < PARTS; ++x) {
          const uint32_t src = raw + code_off + x * (32 * Ly::KROW);
          const uint32_t d0 = dst + row_off + 4096u * x, d1 = d0 ^ 16u, s_row = ((dst + scales_off) ^ (32u * x)) + 256u * x;
          uint32_t codes[4];  // of eight tokens each (loads first: an access to shared memory does not move past another)
          load_codes<4, 8 * CB>(src, codes);
          const uint4 s0 = lds128(s_row), s1 = lds128(s_row ^ 16u);
          expand_rows<BK, BK - 1, BK - 1, 4>(codes, shift, s0, s1, d0, d1, fields);
        }
      } else if (packed) {
        // Parameters of tokens lane, lane + 32, + 64, + 96, (scale, zero-point); none of tokens that do not exist.  A word of the
        // operand's rows has tokens (t, t + 2): one of the two lanes writes s and o s, the other z.
        // (the scales of a token's other channel groups: the warps have to agree on what is in quarters)
        uint32_t sz[4], top[2] = {0u, 0u};
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const uint32_t at = raw + meta_off + k * (128 * NG);
          if constexpr (BV == 2 && NG > 1) {
            uint32_t scales[NG / 2];
            if constexpr (NG == 4) {
              const uint2 v = lds64(at);
              scales[0] = v.x;
              scales[1] = v.y;
            } else {
              scales[0] = lds32(at);
            }
            sz[k] = __byte_perm(NG == 4 && vg >= 2 ? scales[NG / 2 - 1] : scales[0], lds16(at + 2 * NG + 2 * vg), vg & 1 ? 0x5432 : 0x5410);
            if (valid < RB && lane + 32 * k >= valid) sz[k] = scales[0] = scales[NG / 2 - 1] = 0u;
            top[k >> 1] = __vmaxu2(top[k >> 1], NG == 4 ? __vmaxu2(scales[0], scales[NG / 2 - 1]) : scales[0]);
          } else {
            sz[k] = lds16(at + 2 * vg) | lds16(at + 2 * NG + 2 * vg) << 16;
            if (valid < RB && lane + 32 * k >= valid) sz[k] = 0u;
            top[k >> 1] = max(top[k >> 1], sz[k] & 0xffffu);
          }
        }
        if constexpr (BV == 2) {
#pragma unroll
          for (int x = 0; x < 2; ++x) {
            if (any_large(top[x])) {
              quarter |= 1u << x;
              sz[2 * x] = hmul2(sz[2 * x], QUARTERS);
              sz[2 * x + 1] = hmul2(sz[2 * x + 1], QUARTERS);
            }
          }
        }
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const uint32_t other = __shfl_xor_sync(0xffffffffu, sz[k], 2), first = lane & 2 ? other : sz[k], second = lane & 2 ? sz[k] : other;
          uint32_t s2 = __byte_perm(first, second, 0x5410), z2 = __byte_perm(first, second, 0x7632);
          const uint32_t to = (dst + params_off + (k >> 1) * Ly::VBLOCK) ^ (64u * (k & 1));
          uint32_t os = BV == 2 ? (lane & 1 ? hadd2(s2, s2) : s2) : (lane & 1 ? s2 : 0u);
          if constexpr (F16) {  // z and o s as the rounding of their sum and what it left off (D. E. Knuth's two-sum: exact)
            constexpr uint32_t minus = 0x80008000u;
            const uint32_t sum = hadd2(z2, os), t = hadd2(sum, z2 ^ minus);
            os = hadd2(hadd2(z2, hadd2(t, sum ^ minus)), hadd2(os, t ^ minus));
            z2 = sum;
          }
          sts32(to, lane & 2 ? z2 : s2);
          if (!(lane & 2)) sts32((dst + rest_off + (k >> 1) * Ly::VBLOCK) ^ (64u * (k & 1)), os);
        }
        __syncwarp();
#pragma unroll 1
        for (int x = 0; x < 2; ++x) {
          const uint32_t src = raw + code_off + x * (BV == 2 ? D * 16 : 8), block = dst + x * Ly::VBLOCK;
          const uint32_t d0 = block + row_off, d1 = d0 ^ 16u, s_row = block + scales_off;
          uint32_t codes[STEPS];
          load_codes<STEPS, 128>(src, codes);
          const uint4 s0 = lds128(s_row), s1 = lds128(s_row ^ 16u);
          expand_rows<BV, BV - 1, BV, STEPS>(codes, shift, s0, s1, d0, d1, fields);
        }
      } else {
        // a window batch: the warps of a kind settle its exponent, then write it
        const int w0 = (t_lo + i - pk_batches) * RB, n_w = min(RB, r - w0), slot_w = (i - n_pk) % R_UNITS;
        const uint4* rows = reinterpret_cast<const uint4*>((keys ? p.L.win_k : p.L.win_v) + ((size_t)bh * dm.R + w0) * D);
        const uint32_t bar_unit = (keys ? bar_kunit : bar_vunit) + 8 * slot_w;
        float f = 1.f;
        if (!F16) {
          uint32_t m = 0u;
#pragma unroll 4
          for (int x = ew * 32 + lane; x < n_w * (D / 8); x += 128) m = top_of(m, rows[x]);
          m = redux_max_u32(max(m & 0xffffu, m >> 16));
          if (lane == 0) unit_sm[slot_w][keys ? 0 : 1][ew] = m;
        }
        if (lane == 0) mbar_arrive(bar_unit);
        if (!F16) {
          if (!warp_wait(bar_unit, ((i - n_pk) / R_UNITS) & 1, &dead_sm)) break;
          const int e = batch_exponent(i, keys ? 0 : 1, keys ? 126 : most);
          f = pow2i(e);
          most = min(most, e + R_RISE);
          if (!keys && ew == 0 && lane == 0) value_e_sm[slot_w] = e;
        }
        arrive_if(!keys && ew == 0 && lane == 0, bar_ve + 8 * slot_w);
        if (keys) {
          // (the extra rows of a window batch's keys are not looked at)
          const uint32_t to = sm + b * Ly::KBYTES;
#pragma unroll 4
          for (int x = ew * 32 + lane; x < RB * (D / 8); x += 128) {
            const int y = x / (D / 8), c = x % (D / 8);
            const uint4 v = reorder8<F16>(y < n_w ? rows[x] : make_uint4(0u, 0u, 0u, 0u), f);
            sts128(to + (c >> 3) * Ly::KBLOCK + piece_at(y, c & 7), v.x, v.y, v.z, v.w);
          }
        } else {
          const uint32_t to = sm + Ly::OFF_V + b * Ly::VBYTES;
          const uint32_t* words = reinterpret_cast<const uint32_t*>(rows);
          if (lane < 16) {
            sts128(to + piece_at(lane < 8 ? rz : Ly::REST + vg, lane & 7), 0u, 0u, 0u, 0u);
            sts128(to + Ly::VBLOCK + piece_at(lane < 8 ? rz : Ly::REST + vg, lane & 7), 0u, 0u, 0u, 0u);
          }
          // eight tokens of two channels: lanes take neighbouring channels of a token
#pragma unroll 1
          for (int x = ew * 32 + lane; x < RB / 8 * (D / 2); x += 128) {
            const int c = x % (D / 2), piece = x / (D / 2);
            uint32_t y[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) y[k] = 8 * piece + k < n_w ? words[(size_t)(8 * piece + k) * (D / 2) + c] : 0u;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              const uint4 v = reorder8<F16>(make_uint4(__byte_perm(y[0], y[1], h ? 0x7632 : 0x5410), __byte_perm(y[2], y[3], h ? 0x7632 : 0x5410),
                                                  __byte_perm(y[4], y[5], h ? 0x7632 : 0x5410), __byte_perm(y[6], y[7], h ? 0x7632 : 0x5410)), f);
              sts128(to + (piece >> 3) * Ly::VBLOCK + piece_at(2 * c + h, piece & 7), v.x, v.y, v.z, v.w);
            }
          }
        }
      }
      if constexpr (BV == 2) {
        if (!keys && ew < 2 && (quarter >> ew & 1u) != (quarter_ones >> b & 1u)) {
          quarter_ones ^= 1u << b;
          write_ones(b, quarter >> ew & 1u ? QUARTERS : 0x3c003c00u);
        }
      }
      if ((keys ? BK : BV) == 2 && ew == 0 && lane == 0) quarter_sm[keys ? 0 : 1][b] = quarter;
      proxy_fence();
      __syncwarp();
      arrive_if(lane == 0, (keys ? bar_kfull : bar_vfull) + 8 * b);
      arrive_if(lane == 0 && packed, bar_rfree + 8 * (i % R_RAW));
    }
  } else {
    // ================= softmax: a group takes every fourth tile, one of every other batch; thread = row =================
    const int group = warp >> 2, b = group >> 1, g = group & 1, quarter = warp & 3, k_row = tid & 127;
    const uint32_t row_t = tbase + ((uint32_t)(quarter * 32) << 16);
    const bool idle = 32 * quarter >= n_rows;  // none of this warp's rows exists
    float cq = p.scale * 1.4426950408889634f;
    {
      // q: a quarter of this thread's row as fp16 in the operands' order, bfloat16 scaled by a power of two into [1, 2), to
      // tensor memory
      uint4 x[D / 32];
#pragma unroll
      for (int i = 0; i < D / 32; ++i) x[i] = lds128(q_sm + k_row * QROW + group * (D / 2) + 16 * i);
      float f = 1.f;
      if (!F16) {
        uint32_t m = 0u;
#pragma unroll
        for (int i = 0; i < D / 32; ++i) m = top_of(m, x[i]);
        top_sm[group][k_row] = bf16_top(m);
        softmax_sync();
        const float am = fmaxf(fmaxf(top_sm[0][k_row], top_sm[1][k_row]), fmaxf(top_sm[2][k_row], top_sm[3][k_row]));
        const int e = am > 0.f ? max(-100, min(100, -exponent_of(am))) : 0;
        f = pow2i(e);
        cq *= pow2i(-e);
      }
      uint32_t y[D / 8];
#pragma unroll
      for (int i = 0; i < D / 32; ++i) {
        const uint4 v = reorder8<F16>(x[i], f);
        y[4 * i] = v.x; y[4 * i + 1] = v.y; y[4 * i + 2] = v.z; y[4 * i + 3] = v.w;
      }
      tmem_st<D / 8>(row_t + Ly::COL_Q + group * (D / 8), y);
      tc_wait_st();
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(bar_q);
    }
    const uint32_t s_t = row_t + Ly::COL_S + b * Ly::KN + g * RT;
    const uint32_t my_turn = bar_turn + 8 * (R_GROUPS * quarter + group), next_turn = bar_turn + 8 * (R_GROUPS * quarter + (group + 1) % R_GROUPS);
#pragma unroll 1
    for (int i = b; i < N; i += 2) {
      const bool packed = i < n_pk;
      const uint32_t turn = (i >> 1) & 1;
      if (!warp_wait(bar_s + 8 * b, turn, &dead_sm)) break;
      if (!packed) {
        const int slot = (i - n_pk) % R_UNITS, round = ((i - n_pk) / R_UNITS) & 1;
        if (!warp_wait(bar_kunit + 8 * slot, round, &dead_sm) || !warp_wait(bar_ve + 8 * slot, round, &dead_sm)) break;
      }
      tc_fence_after();
      const int n_valid = (packed ? n_q - (t_lo + i) * RB : r - (t_lo + i - pk_batches) * RB) - RT * g;  // of this tile
      // 32 columns of S at a time, twice: for the search and for the numerators
      auto columns = [&](int x, uint32_t (&s)[32]) {
        tmem_ld<32>(s_t + 32 * x, s);
        tc_wait_ld();
        if (n_valid < 32 * x + 32) {
#pragma unroll
          for (int k = 0; k < 32; ++k)
            if (32 * x + k >= n_valid) s[k] = 0xff800000u;
        }
      };
      float c = cq, bias[2] = {0.f, 0.f}, xm = -CUDART_INF_F;
      if (!idle) {
        // logits in log2 units: S c + bias of their 32 tokens
        if (packed) {
          uint32_t e[8];
          tmem_ld<8>(row_t + Ly::COL_S + b * Ly::KN + RB, e);
          tc_wait_ld();
#pragma unroll
          for (int x = 0; x < 2; ++x) {
            const uint32_t z = g ? e[4 + 2 * x] : e[2 * x], y = g ? e[5 + 2 * x] : e[2 * x + 1];
            if (32 * x < n_valid) bias[x] = (__uint_as_float(z) + (BK == 2 ? __uint_as_float(y) : 0.f)) * cq;
          }
        } else {
          c *= pow2i(-batch_exponent(i, 0, 126));
        }
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          uint32_t s[32];
          columns(x, s);
          float a = __uint_as_float(s[0]), d = __uint_as_float(s[1]);
#pragma unroll
          for (int k = 2; k < 30; k += 4) {
            a = fmaxf(fmaxf(a, __uint_as_float(s[k])), __uint_as_float(s[k + 1]));
            d = fmaxf(fmaxf(d, __uint_as_float(s[k + 2])), __uint_as_float(s[k + 3]));
          }
          a = fmaxf(fmaxf(a, __uint_as_float(s[30])), __uint_as_float(s[31]));
          xm = fmaxf(xm, fmaf(fmaxf(a, d), c, bias[x]));
        }
      }
      // the reference that the tile before left
      float m = -CUDART_INF_F;
      if (i > 0 || g > 0) {
        if (!warp_wait(my_turn, group > 0 ? turn : turn ^ 1u, &dead_sm)) break;
        m = m_sm[k_row];
      }
      const float m_old = m;
      if (xm > m + R_TAU || (m == -CUDART_INF_F && xm > m)) m = ceilf(xm);
      m_sm[k_row] = m;
      __syncwarp();
      arrive_if(lane == 0, next_turn);
      // the exponent of the values in O changes with a batch's first tile
      const int de = packed || g > 0 ? 0 : value_exponent(i) - (i > n_pk ? value_exponent(i - 1) : 0);
      if ((i > 0 || g > 0) && !idle && __any_sync(0xffffffffu, m != m_old || de != 0)) {
        // O has to follow a raised reference, and the scale of the window's values: after the products of the tile before
        const int j = g ? i : i - 1;
        if (!warp_wait(bar_o + 16 * (j & 1) + 8 * (1 - g), (j >> 1) & 1, &dead_sm)) break;
        tc_fence_after();
        const float f = m_old == -CUDART_INF_F ? 0.f : ex2(m_old - m), fv = f * pow2_or_zero(de);
#pragma unroll 1
        for (int k = 0; k < Ly::VN; k += 16) {
          uint32_t y[16];
          tmem_ld<16>(row_t + Ly::COL_O + k, y);
          tc_wait_ld();
#pragma unroll
          for (int j = 0; j < 16; ++j) y[j] = __float_as_uint(__uint_as_float(y[j]) * (k == D && j == Ly::ONES - D ? f : fv));
          tmem_st<16>(row_t + Ly::COL_O + k, y);
        }
      }
      if (!idle) {
        // numerators, tokens (0, 2), (1, 3) of four side by side
        const uint64_t cc = pair_of(c, c);
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          uint32_t s[32];
          columns(x, s);
          const float off = m == -CUDART_INF_F ? 0.f : bias[x] + ((float)R_PEXP - m);
          const uint64_t oo = pair_of(off, off);
          uint32_t y[16];
          auto numerators = [&](int k, float (&v)[4]) {
            const float2 a = halves_of(fma2(pair_of(__uint_as_float(s[4 * k]), __uint_as_float(s[4 * k + 1])), cc, oo));
            const float2 d = halves_of(fma2(pair_of(__uint_as_float(s[4 * k + 2]), __uint_as_float(s[4 * k + 3])), cc, oo));
            v[0] = ex2(a.x); v[1] = ex2(a.y); v[2] = ex2(d.x); v[3] = ex2(d.y);
            y[2 * k] = pack_io2<true>(v[0], v[2]);
            y[2 * k + 1] = pack_io2<true>(v[1], v[3]);
          };
          if constexpr (F16) {
            uint32_t z[16];  // what the rounding left off
#pragma unroll
            for (int k = 0; k < 8; ++k) {
              float v[4];
              numerators(k, v);
              z[2 * k] = pack_io2<true>(v[0] - io2_lo<true>(y[2 * k]), v[2] - io2_hi<true>(y[2 * k]));
              z[2 * k + 1] = pack_io2<true>(v[1] - io2_lo<true>(y[2 * k + 1]), v[3] - io2_hi<true>(y[2 * k + 1]));
            }
            tmem_st<16>(s_t + 32 * x + 16, z);
          } else {
#pragma unroll
            for (int k = 0; k < 8; ++k) {
              float v[4];
              numerators(k, v);
            }
          }
          tmem_st<16>(s_t + 32 * x, y);
        }
        tc_wait_st();
      }
      tc_fence_before();
      __syncwarp();
      arrive_if(lane == 0, bar_p + 16 * b + 8 * g);
    }

    // ---- the result, or the split's partial: each group takes a quarter of the channels ----
    if (N > 0) mbar_wait(bar_end, 0, &dead_sm);
    softmax_sync();  // (every warp comes here, whatever failed)
    tc_fence_after();
    float m = N > 0 ? m_sm[k_row] : -CUDART_INF_F;
    const int ev = N > n_pk ? value_exponent(N - 1) : 0;
    const float unit = pow2i(-R_PEXP), back = pow2i(-ev);
    float l = 0.f, extra[NG];
    {
      uint32_t y[16];
      tmem_ld<16>(row_t + Ly::COL_O + D, y);
      tc_wait_ld();
      l = N > 0 ? __uint_as_float(y[Ly::ONES - D]) * unit : 0.f;
#pragma unroll
      for (int x = 0; x < NG; ++x) extra[x] = __uint_as_float(y[x]) + __uint_as_float(y[Ly::REST - D + x]);
    }
    const bool empty = N == 0;  // no token: the sums are not defined
    if (!empty && m == -CUDART_INF_F) m = CUDART_NAN_F;  // (no logit is a number, nor is the result)
    const float inv = p.part_acc != nullptr ? unit : unit / l;  // (times `back` it may be below the normal numbers)
    const bool wide = p.part_acc != nullptr || p.out_f32;
    // through shared memory (the operands' place), so that a warp stores whole rows (a bulk copy a row was slower)
    const uint32_t row_bytes = wide ? 4 * D : 2 * D, mine = sm + k_row * (row_bytes + 16);
#pragma unroll 1
    for (int k = 0; k < D / 4; k += 16) {
      const int c0 = group * (D / 4) + k;
      uint32_t y[16];
      tmem_ld<16>(row_t + Ly::COL_O + c0, y);
      tc_wait_ld();
      float z = extra[0], v[16];
#pragma unroll
      for (int x = 1; x < NG; ++x) z = c0 / GS == x ? extra[x] : z;
#pragma unroll
      for (int j = 0; j < 16; ++j) v[j] = empty ? 0.f : (__uint_as_float(y[j]) + z) * inv * back;
      if (wide) {
#pragma unroll
        for (int j = 0; j < 4; ++j)
          sts128(mine + 4 * c0 + 16 * j, __float_as_uint(v[4 * j]), __float_as_uint(v[4 * j + 1]), __float_as_uint(v[4 * j + 2]), __float_as_uint(v[4 * j + 3]));
      } else {
        uint32_t w[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) w[j] = F16 ? pack_io2<true>(v[2 * j], v[2 * j + 1]) : pack_io2<false>(v[2 * j], v[2 * j + 1]);
        sts128(mine + 2 * c0, w[0], w[1], w[2], w[3]);
        sts128(mine + 2 * c0 + 16, w[4], w[5], w[6], w[7]);
      }
    }
    softmax_sync();
    if (dead_sm == 0) {
      const int ns = p.part_acc != nullptr ? p.ns : 1;
      uint8_t* const to = (p.part_acc != nullptr ? reinterpret_cast<uint8_t*>(p.part_acc) : reinterpret_cast<uint8_t*>(p.out)) + (size_t)(ns > 1 ? split : 0) * row_bytes;
      if (wide) store_rows<D / 4>(sm, to, (size_t)ns * row_bytes, my_call_row, 8 * warp, n_rows, lane);
      else store_rows<D / 8>(sm, to, (size_t)ns * row_bytes, my_call_row, 8 * warp, n_rows, lane);
      if (p.part_acc != nullptr && group == 0 && k_row < n_rows)
        reinterpret_cast<float2*>(p.part_ml)[(size_t)call_row(k_row) * p.ns + split] = make_float2(m, empty ? 0.f : l);
    }
  }
  if (p.late_wait) grid_dependency_wait();
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (warp == R_MMA) tmem_dealloc(tbase, 512u);
  if (dead_sm != 0 && tid == 0) atomicExch(p.status, 1);
}

template <int D, int BK, int BV, int GS, bool F16>
cudaError_t rows_launch_one(const RowsParams& p, cudaStream_t st) {
  using Ly = RowsLayout<D, BK, BV, GS>;
  auto kernel = rows_kernel<D, BK, BV, GS, F16>;
  constexpr size_t SMEM = Ly::TOTAL + 1024;
  const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)SMEM);
  if (e != cudaSuccess) return e;
  return launch_dependent(kernel, dim3((unsigned)p.row_tiles * p.dm.B * p.dm.Hkv * p.ns), dim3(R_THREADS), SMEM, st, p);
}

}  // namespace

template <int D, bool F16>
cudaError_t launch_rows_t(const RowsParams& p, cudaStream_t st) {
  switch (p.L.bk * 100 + p.L.bv * 10 + (p.dm.g == 64)) {
    case 220: return rows_launch_one<D, 2, 2, 32, F16>(p, st);
    case 221: return rows_launch_one<D, 2, 2, 64, F16>(p, st);
    case 210: return rows_launch_one<D, 2, 1, 32, F16>(p, st);
    case 211: return rows_launch_one<D, 2, 1, 64, F16>(p, st);
    case 120: return rows_launch_one<D, 1, 2, 32, F16>(p, st);
    case 121: return rows_launch_one<D, 1, 2, 64, F16>(p, st);
    case 110: return rows_launch_one<D, 1, 1, 32, F16>(p, st);
    case 111: return rows_launch_one<D, 1, 1, 64, F16>(p, st);
  }
  return cudaErrorInvalidValue;
}

}  // namespace xq
