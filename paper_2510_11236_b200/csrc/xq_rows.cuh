// Attention of many query rows over a whole cache (prefix and cross attention), none of its tokens masked but those behind a
// sequence's length.  tcgen05 products; a CTA takes 128 rows (tokens x sequences x heads of a kv head) and a range of 64-token
// tiles of one (sequence, kv head) of the cache.
//
// The codes become operands without a rounding: with c in 0 .. 3, c s + z = s (c - 1) + (z + s), and s (c - 1), one of -s, 0, s,
// 2 s, is a half-precision number when s is (1-bit codes: s c + z).  The rest does not depend on the token (keys: within a
// group of tokens) or on the channel (values: within a group of channels), so it is a few more rows of the same operand:
//
//   S = Q [s (c - 1) | z, s of the tile's token groups]           64 + 16 columns, fp32
//   O += P [s (c - 1) | z, s of the channel groups | 1]           head_dim + 16 columns, fp32; the last one sums P
//
// Q: half precision, scaled by a power of two for each row (exact for bfloat16 down to 2^-16 of the row's largest element);
// P: the softmax numerators times 2^R_PEXP, rounded to half precision (2^-12 of each on average; the result is divided by the
// sum of the rounded ones), the one rounding of operands here.  Both are A operands in tensor memory.  Against pairs hi + lo of
// codes and numerators, as the chunk kernel has them, that is 608 in place of 1280 cycles of the tensor pipe a tile, and half
// the expansion.
//
// Even tiles and odd tiles are two streams with a softmax reference and an O of their own (Q 64, S 2 x 80, O 2 x 144: all 512
// columns of tensor memory), joined at the end: neither group of four softmax warps (thread = row = lane) waits for the other,
// and one works while the products of the other run.  The reference is raised only when a logit exceeds it by R_TAU (log2
// units); P takes the columns of its S.  Eight warps expand (four keys, four values), one issues products, one copies the packed
// data of 128 tokens at a time.  Window tokens go into the same operands as they are, bfloat16 ones scaled by a power of two.
//
// Every wait on an mbarrier is bounded, as in the chunk kernel: a thread that gives up sets a flag that ends the others' waits,
// and the CTA reports through the status word.
#pragma once
#include "xq_internal.h"
#include "xq_layout.cuh"
#include "xq_mma.cuh"

namespace xq {
namespace {

constexpr int RT = 64;           // tokens of a tile
constexpr int R_BUFS = 3;        // expanded tiles of keys, of values
constexpr int R_RAW = 3;         // packed batches of 128 tokens in flight
constexpr float R_TAU = 8.f;
constexpr int R_PEXP = 7;        // numerators are at most 2^(R_PEXP + R_TAU) as fp16
constexpr int R_MMA = 16, R_LOAD = 17, R_THREADS = 18 * 32;
constexpr uint32_t MAX_DOUBLED = 0x77ff;  // the largest half-precision number whose double is finite

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

template <int D, int BK, int BV, int GS>
struct RowsLayout {
  static constexpr int NG = D / GS;
  static constexpr int KROW = D * BK / 8;              // packed bytes of a token's keys
  static constexpr int KN = RT + 16, VN = D + 16;      // rows of the operands (N of the products)
  static constexpr int KBLOCK = KN * 128, KBYTES = D / 64 * KBLOCK, VBYTES = VN * 128;
  static constexpr int ONES = D + 8;                   // the operand row, and column of O, that sums P
  // a raw stage: key codes, key parameters, value codes, value parameters of 128 tokens
  static constexpr int RAW_KM = XQ_BATCH * KROW, RAW_VC = RAW_KM + XQ_BATCH / GS * 4 * D, RAW_VM = RAW_VC + 16 * D * BV;
  static constexpr int RAW = RAW_VM + XQ_BATCH * 4 * NG;
  static constexpr int OFF_V = R_BUFS * KBYTES, OFF_RAW = OFF_V + R_BUFS * VBYTES, TOTAL = OFF_RAW + R_RAW * RAW;
  static constexpr int XROW = D / 2 + 4;               // floats of a row that one group leaves the other
  static_assert(2 * ROWS_TILE * XROW * 4 <= OFF_RAW, "the exchange fits the operands");
  static_assert(KBLOCK % 1024 == 0 && VBYTES % 1024 == 0 && RAW % 16 == 0, "alignment");
  // tensor memory columns
  static constexpr uint32_t COL_Q = 0, COL_S = D / 2, COL_O = COL_S + 2 * KN;
  static_assert(COL_O + 2 * VN <= 512, "tensor memory");
};

// The byte of 16-byte piece `piece` of an operand row, from the operand's start
__device__ __forceinline__ uint32_t piece_at(int row, int piece) { return (uint32_t)(row * 128 + ((piece ^ (row & 7)) << 4)); }

// Eight codes, two fields (at bits 0 and BITS of every byte of w) of four bytes each, times the scales s of their pairs.  A
// field becomes a half-precision number beside an exponent whose last places it takes: 1024 + c, 2^(10 - BITS) + c.
template <int BITS>
__device__ __forceinline__ void expand8(uint32_t w, const uint4& s, uint32_t dst) {
  constexpr uint32_t F = BITS == 2 ? 0x00030003u : 0x00010001u;
  constexpr uint32_t E0 = 0x64006400u, E1 = BITS == 2 ? 0x5c005c00u : 0x60006000u;  // 1024; 256 or 512
  constexpr uint32_t N0 = BITS == 2 ? 0xe401e401u : 0xe400e400u, N1 = BITS == 2 ? 0xdc04dc04u : 0xe000e000u;  // less 1 for 2 bits
  const uint32_t y = w >> 8;
  sts128(dst, hmul2(hadd2((w & F) | E0, N0), s.x), hmul2(hadd2((y & F) | E0, N0), s.y),
         hmul2(hadd2((w & (F << BITS)) | E1, N1), s.z), hmul2(hadd2((y & (F << BITS)) | E1, N1), s.w));
}
// The same where a scale is too large to be doubled: c s + z, rounded (the operand's extra rows are then zero).  s, z: the
// parameters of element j at s_at(j), z_at(j) in shared memory.
template <int BITS, typename S, typename Z>
__device__ __forceinline__ void restore8(uint32_t w, S s_at, Z z_at, uint32_t dst) {
  uint32_t o[4];
#pragma unroll
  for (int k = 0; k < 4; ++k) {  // word k: elements (0, 2), (1, 3), (4, 6), (5, 7)
    const int e = (k >> 1) * 4 + (k & 1);
    float v[2];
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      const uint32_t c = (w >> (8 * ((e & 3) + 2 * x) + BITS * (e >> 2))) & ((1u << BITS) - 1u);
      v[x] = fmaf((float)c, f16_to_f(lds16(s_at(e + 2 * x))), f16_to_f(lds16(z_at(e + 2 * x))));
    }
    o[k] = pack_io2<true>(v[0], v[1]);
  }
  sts128(dst, o[0], o[1], o[2], o[3]);
}

// exponent that puts a window's largest magnitude into the range of half precision, 0 where it is there
__device__ __forceinline__ int window_exponent(float mx) {
  return (mx >= 0.0625f && mx < 32768.f) || !(mx > 0.f) ? 0 : 14 - exponent_of(mx);
}

template <int D, int BK, int BV, int GS>
__global__ void __launch_bounds__(R_THREADS, 1) rows_kernel(const __grid_constant__ RowsParams p) {
  using Ly = RowsLayout<D, BK, BV, GS>;
  constexpr int NG = Ly::NG;
  extern __shared__ uint8_t smem_raw[];
  __shared__ __align__(8) unsigned long long bar_mem[6 * 3 + 2 * 2 + 3];
  __shared__ float cq_sm[ROWS_TILE];
  __shared__ uint32_t win_max[2];  // largest |key|, |value| of the CTA's window tokens, as bits
  __shared__ uint32_t tmem_base_sm;
  __shared__ volatile int dead_sm;

  const Dims& dm = p.dm;
  const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), lane = tid & 31;
  const uint32_t sm = ((uint32_t)__cvta_generic_to_shared(smem_raw) + 1023u) & ~1023u;
  float* const xch = reinterpret_cast<float*>(smem_raw + (sm - (uint32_t)__cvta_generic_to_shared(smem_raw)));
  const uint32_t bars = (uint32_t)__cvta_generic_to_shared(&bar_mem[0]);
  const uint32_t bar_rfull = bars;               // [3] a batch's packed data is there
  const uint32_t bar_rfree = bar_rfull + 24;     // [3] all expanding warps are done with it
  const uint32_t bar_kfull = bar_rfree + 24;     // [3] a tile's keys are expanded
  const uint32_t bar_kfree = bar_kfull + 24;     // [3] their products are complete
  const uint32_t bar_vfull = bar_kfree + 24;     // [3] the same of the values
  const uint32_t bar_vfree = bar_vfull + 24;     // [3]
  const uint32_t bar_s = bar_vfree + 24;         // [2] S of an even / odd tile is complete (and the value products before it)
  const uint32_t bar_p = bar_s + 16;             // [2] its numerators are written
  const uint32_t bar_q = bar_p + 16;             // Q is written
  const uint32_t bar_win = bar_q + 8;            // win_max is final
  const uint32_t bar_end = bar_win + 8;          // every product is complete

  if (tid == 0) {
#pragma unroll
    for (int i = 0; i < 3; ++i) {
      mbar_init(bar_rfull + 8 * i, 1);
      mbar_init(bar_rfree + 8 * i, 8);
      mbar_init(bar_kfull + 8 * i, 4);
      mbar_init(bar_kfree + 8 * i, 1);
      mbar_init(bar_vfull + 8 * i, 4);
      mbar_init(bar_vfree + 8 * i, 1);
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      mbar_init(bar_s + 8 * i, 1);
      mbar_init(bar_p + 8 * i, 4);
    }
    mbar_init(bar_q, 4);
    mbar_init(bar_win, 4);
    mbar_init(bar_end, 1);
    win_max[0] = win_max[1] = 0u;
    dead_sm = 0;
    asm volatile("fence.mbarrier_init.release.cluster;\n" ::: "memory");
  }
  // (tensor memory is asked for after the wait: a CTA of the preceding kernel that shares the SM may still have to get its own)
  grid_dependency_wait();
  grid_dependents_go();
  if (warp == R_MMA) tmem_alloc((uint32_t)__cvta_generic_to_shared(&tmem_base_sm), 512u);

  // ---- the CTA's rows and tiles ----
  const int G = dm.G;
  const int split = blockIdx.x % p.ns, rest = blockIdx.x / p.ns, rt = rest % p.row_tiles, bh = rest / p.row_tiles;
  const int u = bh / dm.Hkv, hk = bh - u * dm.Hkv;
  const int row0 = rt * ROWS_TILE, n_rows = min(ROWS_TILE, p.T * p.each * G - row0);
  int n_q = p.n_q, r = p.r;
  if (p.lengths != nullptr) {
    const int S = max(0, min(n_q + r, p.lengths[u]));
    n_q = min(n_q, S);
    r = S - n_q;
  }
  const int pk_tiles = (n_q + RT - 1) / RT, all_tiles = pk_tiles + (r + RT - 1) / RT;
  int t_lo, t_hi;
  share_of((all_tiles + 1) / 2, p.ns, split, t_lo, t_hi);
  t_lo *= 2;
  t_hi = min(2 * t_hi, all_tiles);
  const int N = max(0, t_hi - t_lo);
  const int n_pk = max(0, min(t_hi, pk_tiles) - t_lo);  // packed tiles of the range
  auto call_row = [&](int k) {                          // of the stream's row row0 + k
    const int x = row0 + k, h = x % G, ji = x / G, i = ji % p.each, j = ji / p.each;
    return ((size_t)j * (dm.B * p.each) + (size_t)u * p.each + i) * dm.Hq + hk * G + h;
  };

  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tbase = tmem_base_sm;

  if (warp == R_MMA) {
    // ================= products: the loop is warp-uniform, one elected lane issues =================
    constexpr uint32_t IDK = rows_idesc(Ly::KN), IDV = rows_idesc(Ly::VN);
    const uint32_t tb = __shfl_sync(0xffffffffu, tbase, 0), smu = __shfl_sync(0xffffffffu, sm, 0);
    bool ok = __all_sync(0xffffffffu, mbar_wait(bar_q, 0, &dead_sm));
    // values of tile i - 2, then keys of tile i, whose S takes the place of that tile's numerators
#pragma unroll 1
    for (int i = 0; ok && i < N + 2; ++i) {
      if (i >= 2) {
        const int j = i - 2;
        ok = __all_sync(0xffffffffu, mbar_wait(bar_vfull + 8 * (j % 3), (j / 3) & 1, &dead_sm) &&
                                         mbar_wait(bar_p + 8 * (j & 1), (j >> 1) & 1, &dead_sm));
        if (!ok) break;
        tc_fence_after();
        if (elect_one()) {
          const uint32_t pt = tb + Ly::COL_S + (j & 1) * Ly::KN, dO = tb + Ly::COL_O + (j & 1) * Ly::VN;
          const uint64_t v = rows_desc(smu + Ly::OFF_V + (j % 3) * Ly::VBYTES);
#pragma unroll
          for (int ks = 0; ks < RT / 16; ++ks) rows_mma(dO, pt + 8 * ks, v + 2 * ks, IDV, j >= 2 || ks > 0);
          rows_commit(bar_vfree + 8 * (j % 3));
        }
        __syncwarp();
      }
      if (i < N) {
        ok = __all_sync(0xffffffffu, mbar_wait(bar_kfull + 8 * (i % 3), (i / 3) & 1, &dead_sm));
        if (!ok) break;
        tc_fence_after();
        if (elect_one()) {
          const uint32_t dS = tb + Ly::COL_S + (i & 1) * Ly::KN;
          const uint64_t k = rows_desc(smu + (i % 3) * Ly::KBYTES);
#pragma unroll
          for (int ks = 0; ks < D / 16; ++ks)
            rows_mma(dS, tb + Ly::COL_Q + 8 * ks, k + (ks / 4) * (Ly::KBLOCK / 16) + 2 * (ks % 4), IDK, ks > 0);
          rows_commit(bar_kfree + 8 * (i % 3));
          rows_commit(bar_s + 8 * (i & 1));
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
    // ================= packed data, 128 tokens at a time =================
    if (lane == 0) {
      const int batches = (n_pk + 1) / 2;
      const size_t first = (size_t)(t_lo / 2);
      const uint8_t* const kc = reinterpret_cast<const uint8_t*>(p.L.k_codes) + (size_t)bh * ((size_t)dm.nq_cap * Ly::KROW) + first * (XQ_BATCH * Ly::KROW);
      const uint8_t* const vc = reinterpret_cast<const uint8_t*>(p.L.v_codes) + (size_t)bh * ((size_t)dm.nq_cap * (D * BV / 8)) + first * (16 * D * BV);
      const uint8_t* const km = reinterpret_cast<const uint8_t*>(p.L.k_meta) + (size_t)bh * ((size_t)(dm.nq_cap / GS) * (4 * D)) + first * (XQ_BATCH / GS * 4 * D);
      const uint8_t* const vm = reinterpret_cast<const uint8_t*>(p.L.v_meta) + (size_t)bh * ((size_t)dm.nq_cap * 4 * NG) + first * (XQ_BATCH * 4 * NG);
      int i = 0;
      for (; i < batches; ++i) {
        if (i >= R_RAW && !mbar_wait(bar_rfree + 8 * (i % R_RAW), (i / R_RAW - 1) & 1, &dead_sm)) break;
        const uint32_t dst = sm + Ly::OFF_RAW + (i % R_RAW) * Ly::RAW, bar = bar_rfull + 8 * (i % R_RAW);
        mbar_expect_tx(bar, Ly::RAW);
        bulk_load(dst, kc + (size_t)i * (XQ_BATCH * Ly::KROW), XQ_BATCH * Ly::KROW, bar);
        bulk_load(dst + Ly::RAW_KM, km + (size_t)i * (XQ_BATCH / GS * 4 * D), XQ_BATCH / GS * 4 * D, bar);
        bulk_load(dst + Ly::RAW_VC, vc + (size_t)i * (16 * D * BV), 16 * D * BV, bar);
        bulk_load(dst + Ly::RAW_VM, vm + (size_t)i * (XQ_BATCH * 4 * NG), XQ_BATCH * 4 * NG, bar);
      }
      // no copy may be in flight when the shared memory is released (nobody may have waited for them if a wait gave up)
      for (int k = max(0, i - R_RAW); k < i; ++k)
        for (int n = 0; n < WAIT_LIMIT && !mbar_try_wait(bar_rfull + 8 * (k % R_RAW), (k / R_RAW) & 1); ++n) {}
    }
    __syncwarp();
  } else if (warp >= 8) {
    // ================= expansion: keys (warps 8 .. 11), values (12 .. 15) =================
    const int ew = warp & 3, o = lane & 7, sub = lane >> 3;  // a lane's piece of eight elements, and its row of four
    const bool keys = warp < 12;
    // keys: 64 channels from 64 kb of the 32 tokens of slot `slot` (head_dim 64: of 16 of them)
    const int kb = D == 128 ? ew & 1 : 0, slot = ew >> 1, k_tok = D == 128 ? 0 : 16 * (ew & 1);
    constexpr int K_TOKENS = D == 128 ? 32 : 16;
    // values: D / 4 channels from v_c0 on, all of one channel group
    const int v_c0 = ew * (D / 4), vg = v_c0 / GS;
    if (!keys && ew == 0) {  // the row that sums the numerators
      if (lane < 8)
        for (int b = 0; b < R_BUFS; ++b)
          sts128(sm + Ly::OFF_V + b * Ly::VBYTES + piece_at(Ly::ONES, lane), 0x3c003c00u, 0x3c003c00u, 0x3c003c00u, 0x3c003c00u);
      proxy_fence();
    }
#pragma unroll 1
    for (int i = 0; i < N; ++i) {
      const int t = t_lo + i, b = i % 3;
      const bool packed = i < n_pk;
      bool ok = i < 3 || mbar_wait((keys ? bar_kfree : bar_vfree) + 8 * b, (i / 3 - 1) & 1, &dead_sm);
      if (packed) ok = ok && mbar_wait(bar_rfull + 8 * ((i >> 1) % R_RAW), ((i >> 1) / R_RAW) & 1, &dead_sm);
      else ok = ok && mbar_wait(bar_win, 0, &dead_sm);
      if (!__all_sync(0xffffffffu, ok)) break;
      const uint32_t raw = sm + Ly::OFF_RAW + ((i >> 1) % R_RAW) * Ly::RAW;
      const int half = t & 1;
      if (keys) {
        const uint32_t dst = sm + b * Ly::KBYTES + kb * Ly::KBLOCK;
        const int rz = RT + 2 * slot, rs = rz + 1;  // operand rows of the zero-points and of the scales
        if (packed) {
          // parameters of channels 64 kb + lane and 32 more, side by side in the group's order
          const uint32_t meta = raw + Ly::RAW_KM + (half * RT + slot * 32) / GS * (4 * D);
          const uint32_t sw = lds32(meta + 2 * (lane * (D / 32) + 2 * kb)), zw = lds32(meta + 2 * (D + lane * (D / 32) + 2 * kb));
          const bool large = BK == 2 && __any_sync(0xffffffffu, (sw & 0xffffu) > MAX_DOUBLED || (sw >> 16) > MAX_DOUBLED);
#pragma unroll
          for (int x = 0; x < 2; ++x) {
            const int c = lane + 32 * x, at = (c & ~3) | ((c & 1) << 1) | ((c >> 1) & 1);  // elements of four: 0, 2, 1, 3
            sts16(dst + piece_at(rz, at >> 3) + 2 * (at & 7), large ? 0u : (x ? zw >> 16 : zw & 0xffffu));
            sts16(dst + piece_at(rs, at >> 3) + 2 * (at & 7), large ? 0u : (x ? sw >> 16 : sw & 0xffffu));
          }
          __syncwarp();
          constexpr int PER = 32 / BK, CB = Ly::KROW < 16 ? Ly::KROW : 16;
          const int word = (64 * kb + 8 * o) / PER, shift = 2 * BK * (o % (PER / 8));
          const uint32_t src = raw + (half * 2 + slot) * (32 * Ly::KROW) + word * 4 / CB * (32 * CB) + word * 4 % CB + (k_tok + sub) * CB;
          const int row = 32 * slot + k_tok + sub;
          if (!large) {
            const uint4 s = lds128(dst + piece_at(rs, o));
#pragma unroll
            for (int x = 0; x < K_TOKENS / 4; ++x) expand8<BK>(lds32(src + 4 * x * CB) >> shift, s, dst + piece_at(row + 4 * x, o));
          } else {
            auto at = [&](int e) { const int d = 64 * kb + 8 * o + e; return meta + 2 * (d % 32 * (D / 32) + d / 32); };
#pragma unroll 1
            for (int x = 0; x < K_TOKENS / 4; ++x)
              restore8<BK>(lds32(src + 4 * x * CB) >> shift, at, [&](int e) { return at(e) + 2 * D; }, dst + piece_at(row + 4 * x, o));
          }
        } else {
          const int w0 = (t - pk_tiles) * RT + 32 * slot + k_tok + sub;
          const uint4* rows = reinterpret_cast<const uint4*>(p.L.win_k + ((size_t)bh * dm.R + w0) * D) + 8 * kb + o;
          const float f = pow2i(window_exponent(__uint_as_float(win_max[0])));
#pragma unroll
          for (int x = 0; x < K_TOKENS / 4; ++x) {
            const uint4 v = w0 + 4 * x < r ? rows[(size_t)(4 * x) * (D / 8)] : make_uint4(0u, 0u, 0u, 0u);
            const uint32_t y[4] = {v.x, v.y, v.z, v.w};
            uint32_t z[4];
#pragma unroll
            for (int k = 0; k < 2; ++k) {
              z[2 * k] = pack_io2<true>(io_to_f(y[2 * k] & 0xffffu, p.f16) * f, io_to_f(y[2 * k + 1] & 0xffffu, p.f16) * f);
              z[2 * k + 1] = pack_io2<true>(io_to_f(y[2 * k] >> 16, p.f16) * f, io_to_f(y[2 * k + 1] >> 16, p.f16) * f);
            }
            sts128(dst + piece_at(32 * slot + k_tok + sub + 4 * x, o), z[0], z[1], z[2], z[3]);
          }
        }
      } else {
        const uint32_t dst = sm + Ly::OFF_V + b * Ly::VBYTES;
        const int rz = D + vg, rs = D + NG + vg;
        if (packed) {
          // parameters of tokens (ta, ta + 2) of the tile, a word of the operand's rows
          const int ta = 4 * (lane >> 1) + (lane & 1), valid = n_q - t * RT;
          const uint32_t meta = raw + Ly::RAW_VM + (half * RT + ta) * (4 * NG) + 2 * vg;
          uint32_t sw = 0u, zw = 0u;
          if (ta < valid) { sw = lds16(meta); zw = lds16(meta + 2 * NG); }
          if (ta + 2 < valid) { sw |= lds16(meta + 8 * NG) << 16; zw |= lds16(meta + 10 * NG) << 16; }
          const bool large = BV == 2 && __any_sync(0xffffffffu, (sw & 0xffffu) > MAX_DOUBLED || (sw >> 16) > MAX_DOUBLED);
          const uint32_t at = ((lane >> 1) & 1) * 8 + (lane & 1) * 4;
          sts32(dst + piece_at(rz, lane >> 2) + at, large ? 0u : zw);
          sts32(dst + piece_at(rs, lane >> 2) + at, large ? 0u : sw);
          __syncwarp();
          constexpr int PER = 32 / BV;
          const int shift = 2 * BV * (o % (PER / 8));
          const uint32_t src = raw + Ly::RAW_VC + (BV == 2 ? half * (D * 16) + o / 2 * 4 : (2 * half + o / 4) * 4) + (v_c0 + sub) * 16;
          if (!large) {
            const uint4 s = lds128(dst + piece_at(rs, o));
#pragma unroll
            for (int x = 0; x < D / 16; ++x) expand8<BV>(lds32(src + 64 * x) >> shift, s, dst + piece_at(v_c0 + sub + 4 * x, o));
          } else {
            // (tokens that do not exist: zero for zero, their numerators are)
            auto at = [&](int e) { return raw + Ly::RAW_VM + (half * RT + min(8 * o + e, valid - 1)) * (4 * NG) + 2 * vg; };
#pragma unroll 1
            for (int x = 0; x < D / 16; ++x)
              restore8<BV>(lds32(src + 64 * x) >> shift, at, [&](int e) { return at(e) + 2 * NG; }, dst + piece_at(v_c0 + sub + 4 * x, o));
          }
        } else {
          const int w0 = (t - pk_tiles) * RT + 8 * o;
          const uint32_t* rows = reinterpret_cast<const uint32_t*>(p.L.win_v + ((size_t)bh * dm.R + w0) * D) + v_c0 / 2 + sub;
          const float f = pow2i(window_exponent(__uint_as_float(win_max[1])));
          if (lane < 16) sts128(dst + piece_at(lane < 8 ? rz : rs, o), 0u, 0u, 0u, 0u);
#pragma unroll 1
          for (int x = 0; x < D / 32; ++x) {  // channels v_c0 + 2 sub + 8 x and the next one
            uint32_t y[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) y[k] = w0 + k < r ? rows[(size_t)k * (D / 2) + 4 * x] : 0u;
#pragma unroll
            for (int c = 0; c < 2; ++c) {
              uint32_t z[4];
#pragma unroll
              for (int k = 0; k < 4; ++k) {
                const int e = (k >> 1) * 4 + (k & 1);
                z[k] = pack_io2<true>(io_to_f((y[e] >> (16 * c)) & 0xffffu, p.f16) * f, io_to_f((y[e + 2] >> (16 * c)) & 0xffffu, p.f16) * f);
              }
              sts128(dst + piece_at(v_c0 + 2 * sub + 8 * x + c, o), z[0], z[1], z[2], z[3]);
            }
          }
        }
      }
      proxy_fence();
      __syncwarp();
      if (lane == 0) {
        mbar_arrive((keys ? bar_kfull : bar_vfull) + 8 * b);
        if (packed && (half || i + 1 == n_pk)) mbar_arrive(bar_rfree + 8 * ((i >> 1) % R_RAW));
      }
    }
  } else {
    // ================= softmax: group w takes the tiles i = w, w + 2, ...; thread = row =================
    const int w = warp >> 2, k_row = tid & 127;
    const uint32_t row_t = tbase + ((uint32_t)((warp & 3) * 32) << 16);
    const bool idle = 32 * (warp & 3) >= n_rows;  // none of this warp's rows exists
    if (w == 0) {
      // q: this thread's row as fp16, scaled by a power of two into [1, 2), in the operands' order, to tensor memory
      const bool real = k_row < n_rows;
      const uint4* src = reinterpret_cast<const uint4*>(p.q + (real ? call_row(k_row) * D : 0));
      uint32_t x[D / 2];
      float am = 0.f;
#pragma unroll
      for (int i = 0; i < D / 8; ++i) {
        const uint4 v = real ? src[i] : make_uint4(0u, 0u, 0u, 0u);
        x[4 * i] = v.x; x[4 * i + 1] = v.y; x[4 * i + 2] = v.z; x[4 * i + 3] = v.w;
      }
#pragma unroll
      for (int i = 0; i < D / 2; ++i)
        am = fmaxf(am, fmaxf(fabsf(io_to_f(x[i] & 0xffffu, p.f16)), fabsf(io_to_f(x[i] >> 16, p.f16))));
      const int e = am > 0.f ? max(-100, min(100, -exponent_of(am))) : 0;
      const float f = pow2i(e);
#pragma unroll
      for (int c = 0; c < D / 64; ++c) {
        uint32_t y[32];
#pragma unroll
        for (int m = 0; m < 16; ++m) {
          const uint32_t a = x[32 * c + 2 * m], d = x[32 * c + 2 * m + 1];
          y[2 * m] = pack_io2<true>(io_to_f(a & 0xffffu, p.f16) * f, io_to_f(d & 0xffffu, p.f16) * f);
          y[2 * m + 1] = pack_io2<true>(io_to_f(a >> 16, p.f16) * f, io_to_f(d >> 16, p.f16) * f);
        }
        tmem_st<32>(row_t + Ly::COL_Q + 32 * c, y);
      }
      tc_wait_st();
      cq_sm[k_row] = p.scale * 1.4426950408889634f * pow2i(-e);
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(bar_q);
    } else {
      // the largest magnitudes of the window tokens (half precision: they fit as they are)
      const int w_lo = max(0, t_lo - pk_tiles) * RT, w_hi = min(r, (t_hi - pk_tiles) * RT);
      if (!p.f16 && N > n_pk) {
        const uint4* wk = reinterpret_cast<const uint4*>(p.L.win_k + (size_t)bh * dm.R * D);
        const uint4* wv = reinterpret_cast<const uint4*>(p.L.win_v + (size_t)bh * dm.R * D);
        uint32_t mk = 0u, mv = 0u;
        auto top = [](uint32_t m, const uint4& v) {
          return __vmaxu2(__vmaxu2(__vmaxu2(m, v.x & 0x7fff7fffu), __vmaxu2(v.y & 0x7fff7fffu, v.z & 0x7fff7fffu)), v.w & 0x7fff7fffu);
        };
#pragma unroll 4
        for (int i = w_lo * (D / 8) + k_row; i < w_hi * (D / 8); i += 128) {
          mk = top(mk, wk[i]);
          mv = top(mv, wv[i]);
        }
        mk = redux_max_u32(max(mk & 0xffffu, mk >> 16));
        mv = redux_max_u32(max(mv & 0xffffu, mv >> 16));
        if (lane == 0) {
          atomicMax(&win_max[0], mk << 16);  // bfloat16 as the upper half of a float
          atomicMax(&win_max[1], mv << 16);
        }
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(bar_win);
    }
    bool ok = __all_sync(0xffffffffu, mbar_wait(bar_q, 0, &dead_sm));
    const float cq = cq_sm[k_row];
    float m = -CUDART_INF_F;
    const uint32_t s_t = row_t + Ly::COL_S + w * Ly::KN, o_t = row_t + Ly::COL_O + w * Ly::VN;
#pragma unroll 1
    for (int i = w; ok && i < N; i += 2) {
      const bool packed = i < n_pk;
      bool here = mbar_wait(bar_s + 8 * w, (i >> 1) & 1, &dead_sm);
      if (!packed) here = here && mbar_wait(bar_win, 0, &dead_sm);
      ok = __all_sync(0xffffffffu, here);
      if (!ok) break;
      tc_fence_after();
      const int t = t_lo + i, n_valid = packed ? n_q - t * RT : r - (t - pk_tiles) * RT;
      if (!idle) {
        uint32_t s[2][32], e[8];
        tmem_ld<32>(s_t, s[0]);
        tmem_ld<32>(s_t + 32, s[1]);
        tmem_ld<8>(s_t + RT, e);
        tc_wait_ld();
        if (n_valid < RT) {
#pragma unroll
          for (int k = 0; k < 64; ++k)
            if (k >= n_valid) s[k >> 5][k & 31] = 0xff800000u;
        }
        // logits in log2 units: S c + bias of their 32 tokens
        float c = cq, bias[2] = {0.f, 0.f};
        if (packed) {
#pragma unroll
          for (int h = 0; h < 2; ++h)
            if (32 * h < n_valid) bias[h] = (__uint_as_float(e[2 * h]) + (BK == 2 ? __uint_as_float(e[2 * h + 1]) : 0.f)) * cq;
        } else {
          c *= pow2i(-window_exponent(__uint_as_float(win_max[0])));
        }
        float x[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          float a = __uint_as_float(s[h][0]), d = __uint_as_float(s[h][1]);
#pragma unroll
          for (int k = 2; k < 32; k += 2) {
            a = fmaxf(a, __uint_as_float(s[h][k]));
            d = fmaxf(d, __uint_as_float(s[h][k + 1]));
          }
          x[h] = fmaf(fmaxf(a, d), c, bias[h]);
        }
        const float xm = fmaxf(x[0], x[1]), m_old = m;
        if (xm > m + R_TAU || (m == -CUDART_INF_F && xm > m)) m = ceilf(xm);
        // O has to follow a raised reference, and the scale of the window's values
        const int ev = !packed && i - 2 < n_pk ? window_exponent(__uint_as_float(win_max[1])) : 0;
        if (i >= 2 && __any_sync(0xffffffffu, m != m_old || ev != 0)) {
          const float f = m_old == -CUDART_INF_F ? 0.f : ex2(m_old - m), fv = f * pow2i(ev);
#pragma unroll 1
          for (int k = 0; k < Ly::VN; k += 16) {
            uint32_t y[16];
            tmem_ld<16>(o_t + k, y);
            tc_wait_ld();
#pragma unroll
            for (int j = 0; j < 16; ++j) y[j] = __float_as_uint(__uint_as_float(y[j]) * (k == D && j == 8 ? f : fv));
            tmem_st<16>(o_t + k, y);
          }
        }
        // numerators, tokens (0, 2), (1, 3) of four side by side
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const float off = m == -CUDART_INF_F ? 0.f : bias[h] + ((float)R_PEXP - m);
          uint32_t y[16];
#pragma unroll
          for (int k = 0; k < 8; ++k) {
            float v[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) v[j] = ex2(fmaf(__uint_as_float(s[h][4 * k + j]), c, off));
            y[2 * k] = pack_io2<true>(v[0], v[2]);
            y[2 * k + 1] = pack_io2<true>(v[1], v[3]);
          }
          tmem_st<16>(s_t + 16 * h, y);
        }
        tc_wait_st();
      }
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(bar_p + 8 * w);
    }

    // ---- the two groups' states: each takes half of the channels, and leaves the other half to the other group ----
    const bool has = N > w;
    if (N > 0) mbar_wait(bar_end, 0, &dead_sm);
    __syncwarp();
    tc_fence_after();
    float l = 0.f, rest_of[NG];
    const int ev = N > n_pk ? window_exponent(__uint_as_float(win_max[1])) : 0;  // (the last tile of either group that has a window tile)
    const bool ends_in_window = has && ((N - 1 - w) & ~1) + w >= n_pk;
    const float unit = pow2i(-R_PEXP), uv = ends_in_window ? unit * pow2i(-ev) : unit;
    {
      uint32_t y[16];
      if (has) {
        tmem_ld<16>(o_t + D, y);
        tc_wait_ld();
      }
      l = has ? __uint_as_float(y[8]) * unit : 0.f;
#pragma unroll
      for (int g = 0; g < NG; ++g) rest_of[g] = has ? __uint_as_float(y[g]) + (BV == 2 ? __uint_as_float(y[NG + g]) : 0.f) : 0.f;
    }
    auto channels = [&](int c0, float (&v)[16]) {  // 16 channels from c0 on, of one group
      uint32_t y[16];
      tmem_ld<16>(o_t + c0, y);
      tc_wait_ld();
      float z = rest_of[0];
#pragma unroll
      for (int g = 1; g < NG; ++g) z = c0 / GS == g ? rest_of[g] : z;
#pragma unroll
      for (int k = 0; k < 16; ++k) v[k] = has ? (__uint_as_float(y[k]) + z) * uv : 0.f;
    };
    float* const mine = xch + (size_t)(w * ROWS_TILE + k_row) * Ly::XROW;
#pragma unroll 1
    for (int k = 0; k < D / 2; k += 16) {
      float v[16];
      channels((1 - w) * (D / 2) + k, v);
#pragma unroll
      for (int j = 0; j < 4; ++j) *reinterpret_cast<float4*>(mine + k + 4 * j) = make_float4(v[4 * j], v[4 * j + 1], v[4 * j + 2], v[4 * j + 3]);
    }
    mine[D / 2] = m;
    mine[D / 2 + 1] = l;
    asm volatile("bar.sync 1, 256;\n" ::: "memory");
    const float* const other = xch + (size_t)((1 - w) * ROWS_TILE + k_row) * Ly::XROW;
    const float mo = other[D / 2], M = fmaxf(m, mo);
    const float fm = m == -CUDART_INF_F ? 0.f : ex2(m - M), fo = mo == -CUDART_INF_F ? 0.f : ex2(mo - M);
    const float L = fmaf(l, fm, other[D / 2 + 1] * fo);
    const float inv = p.part_acc != nullptr ? 1.f : (M == -CUDART_INF_F ? 0.f : 1.f / L);
    const bool store = k_row < n_rows && dead_sm == 0;
    const size_t row = store ? call_row(k_row) : 0;
#pragma unroll 1
    for (int k = 0; k < D / 2; k += 16) {
      float v[16];
      const int c0 = w * (D / 2) + k;
      channels(c0, v);
#pragma unroll
      for (int j = 0; j < 16; ++j) v[j] = fmaf(v[j], fm, other[k + j] * fo) * inv;
      if (!store) continue;
      if (p.part_acc != nullptr || p.out_f32) {
        float* const to = (p.part_acc != nullptr ? p.part_acc + (row * p.ns + split) * D : reinterpret_cast<float*>(p.out) + row * D) + c0;
#pragma unroll
        for (int j = 0; j < 4; ++j) reinterpret_cast<float4*>(to)[j] = make_float4(v[4 * j], v[4 * j + 1], v[4 * j + 2], v[4 * j + 3]);
      } else {
        uint32_t y[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) y[j] = p.f16 ? pack_io2<true>(v[2 * j], v[2 * j + 1]) : pack_io2<false>(v[2 * j], v[2 * j + 1]);
        uint4* const to = reinterpret_cast<uint4*>(reinterpret_cast<uint16_t*>(p.out) + row * D + c0);
        to[0] = make_uint4(y[0], y[1], y[2], y[3]);
        to[1] = make_uint4(y[4], y[5], y[6], y[7]);
      }
    }
    if (store && w == 0 && p.part_acc != nullptr) reinterpret_cast<float2*>(p.part_ml)[row * p.ns + split] = make_float2(M, L);
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (warp == R_MMA) tmem_dealloc(tbase, 512u);
  if (dead_sm != 0 && tid == 0) atomicExch(p.status, 1);
}

template <int D, int BK, int BV, int GS>
cudaError_t rows_launch_one(const RowsParams& p, cudaStream_t st) {
  using Ly = RowsLayout<D, BK, BV, GS>;
  auto kernel = rows_kernel<D, BK, BV, GS>;
  constexpr size_t SMEM = Ly::TOTAL + 1024;
  const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)SMEM);
  if (e != cudaSuccess) return e;
  return launch_dependent(kernel, dim3((unsigned)p.row_tiles * p.dm.B * p.dm.Hkv * p.ns), dim3(R_THREADS), SMEM, st, p);
}

}  // namespace

template <int D>
cudaError_t launch_rows_t(const RowsParams& p, cudaStream_t st) {
  switch (p.L.bk * 100 + p.L.bv * 10 + (p.dm.g == 64)) {
    case 220: return rows_launch_one<D, 2, 2, 32>(p, st);
    case 221: return rows_launch_one<D, 2, 2, 64>(p, st);
    case 210: return rows_launch_one<D, 2, 1, 32>(p, st);
    case 211: return rows_launch_one<D, 2, 1, 64>(p, st);
    case 120: return rows_launch_one<D, 1, 2, 32>(p, st);
    case 121: return rows_launch_one<D, 1, 2, 64>(p, st);
    case 110: return rows_launch_one<D, 1, 1, 32>(p, st);
    case 111: return rows_launch_one<D, 1, 1, 64>(p, st);
  }
  return cudaErrorInvalidValue;
}

}  // namespace xq
