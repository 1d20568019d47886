// Multi-query paged attention over the 4-bit KV cache (format: kvq_format.h).
//   o_r = sum_p w_rp v_p,  w_r = softmax over p <= ctx_b + j(r) of q_r . k_p / sqrt(D)
// for the R = G * n rows (position j = r / G, query head h G + r % G) of sequence b and kv head h.
//
// Values and keys are exact in bf16, so the products' only roundings are those of the weights. f32: three bf16 parts
// (24 bits). bf16: f16 weights (11 bits, times 2^10) beside the values as f16, which are exact while V's scales are
// 2^-21 .. 2^10; from its first pair of blocks with another scale on a wavefront takes two bf16 parts (16 bits) beside
// bf16 values. The sum is that of the rounded weights, by an MFMA with a row of ones. The error is that of the output's
// rounding then, rms 1.66e-3 of the output's rms (weights in one bf16 part: 2.3e-3). Kernel times of 128 sequences x 5
// positions at context 8192, and of 2 x 257 at 8100: 108 and 106 us, with values outside f16 158 and 152, with one bf16
// part 107 and 101.
//
// A workgroup has one kv head of a sequence, or of a part of its keys, and a group of up to 48 rows. Each of its
// wavefronts walks a range of pairs of 16-token blocks by itself, with running maxima and sums, and they join at the
// end: no barrier in the loop, and each record byte is read once per row group. The records come by LDS-DMA three
// pairs ahead (into registers they spilled: the first call below took twice as long). K goes into a scaled MFMA as it
// lies there (decoded to bf16: a quarter more), V is decoded: its scale belongs to a token, the product's sum index. The
// next pair's scores are computed beside this pair's weights and values.
//
// 32 query / 4 kv heads x 128, bf16, what bounds the call and what it takes on new inputs:
//   128 sequences x 5 positions at 8192: the records' 571 MB, 127 us, 4.5 TB/s (a large copy: 4.96; read requests 1.03
//     times the records); VALU 58% and MFMA 41% of the cycles
//   256 x 9 at 2048: 72 rows in groups of 3 and 2 tiles, the keys read twice (once through the L2), VALU and MFMA, 130 us
//   2 x 257 at 8100: 68 GFLOP in 344 workgroups where 512 fit, VALU and MFMA, 96 us, 710 TFLOP/s
//   16 x 5 at 32768-65536, cut: 429 MB in 105 us with the join's 5, 4.1 TB/s
//   1 x 1 at 700: launch, four dependent loads and the join, 7.2 us
// A loop iteration is 39 MFMAs and 216 VALU instructions at 3 tiles (of them 24 exp2, 64 for the decoded values, 5 for
// their scales' range); two wavefronts a SIMD, by registers, leave its time near the sum of both pipes. Tried, and what
// the first line then took, in percent: 64 keys an iteration (+2), 3 slots (+5), MFMA and VALU interleaved by schedule
// groups (+1 to 14), exponentials, scores and values in other orders (within 3); the second line: 5 tiles and one
// wavefront a SIMD, so that 72 rows read keys once (+25), a persistent loop over workgroups (-1).
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "internal.h"
#include "kvq_format.h"

namespace molt {
namespace {

constexpr float kLog2e = 1.4426950408889634f;
// f16 weights are times 2^10 and may grow by 2^5 before O is rescaled: up to 2^15, near the top of their range, so that
// those under 2^-24 of the largest become subnormal only. (A slack of 8 took as long for every case below.)
constexpr float kRescaleSlack = 5.0f;
constexpr float kWeightShift = 10.0f;
constexpr int kWaves = 4;
// Pairs of blocks in a wavefront's ring. Workgroups of one wavefront are bound by how many fit in LDS: 201 sequences x
// 180 positions x 8 heads at 0-404 took a quarter more with 4 than with 3; the others wait for memory (the first call
// above: 5% more with 3 than with 4).
constexpr int slots_of(int wavefronts) { return wavefronts == 1 ? 3 : 4; }

struct KvqAttnParams {
  const void* q;           // [B * n, Hq, D]
  const uint8_t* kc;
  const uint8_t* vc;
  const int32_t* bt;       // [B, max_blocks]
  const int32_t* ctx;      // [B]
  void* out;               // [B * n, Hq * D], row-major or tiled
  float* part_o;           // [nrg, Hkv, slots, group, D] partial outputs of split ranges
  float* part_ml;          // [nrg, Hkv, slots, group, 2] their maxima and sums
  int32_t* split;          // [nrg, B, 2] first slot and slots of a sequence
  int B, n, Hq, Hkv, max_blocks, num_blocks;
  int G, R;                // query heads per kv head, rows of a (b, h)
  int nrg, group;          // row groups of a (b, h) and rows of one (16 NT)
  int slots;               // workgroups of a (row group, kv head); B: one per sequence, nothing is cut
  int resident;            // workgroups that the chip holds
  int spread;              // a slot's heads run on one XCD
  int waves;               // wavefronts of a workgroup
  float c;                 // log2(e) / sqrt(D)
  int out_tiled;
};

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef floatx4_t UnalignedF4 __attribute__((aligned(4)));
typedef u32x4 UnalignedU4 __attribute__((aligned(2)));
typedef u32x2 UnalignedU2 __attribute__((aligned(2)));

// Keys 0 .. end - 1 are those that rows [r0, r1) of sequence b may see (the last row the most).
MOLT_DEV int visible_end(const KvqAttnParams& p, int ctx, int r1) {
  const long e = long(ctx) + (r1 - 1) / p.G + 1;
  return int(e < 0 ? 0 : e > 16l * p.max_blocks ? 16l * p.max_blocks : e);
}

// LDS-DMA: 16 (4) bytes a lane from src to dst + 16 (4) * lane; dst is the wavefront's. ONCE: nontemporal, for keys
// that one workgroup reads
typedef const __attribute__((address_space(1))) void* GlobalPtr;
typedef __attribute__((address_space(3))) void* LdsPtr;
template <bool ONCE>
MOLT_DEV void copy_lds16(const uint8_t* src, uint32_t dst) {
  if constexpr (ONCE) __builtin_amdgcn_global_load_lds((GlobalPtr)src, (LdsPtr)uintptr_t(dst), 16, 0, 2);
  else __builtin_amdgcn_global_load_lds((GlobalPtr)src, (LdsPtr)uintptr_t(dst), 16, 0, 0);
}
template <bool ONCE>
MOLT_DEV void copy_lds4(const uint8_t* src, uint32_t dst) {
  if constexpr (ONCE) __builtin_amdgcn_global_load_lds((GlobalPtr)src, (LdsPtr)uintptr_t(dst), 4, 0, 2);
  else __builtin_amdgcn_global_load_lds((GlobalPtr)src, (LdsPtr)uintptr_t(dst), 4, 0, 0);
}

// a wave-uniform value in scalar registers, whatever the compiler would make of how it came about
MOLT_DEV uint32_t in_sgpr(uint32_t x) {
  x = __builtin_amdgcn_readfirstlane(int(x));
  asm("" : "+s"(x));
  return x;
}
MOLT_DEV const uint8_t* in_sgpr(const uint8_t* p) {
  const uint64_t x = reinterpret_cast<uint64_t>(p);
  const uint32_t lo = __builtin_amdgcn_readfirstlane(int(x)), hi = __builtin_amdgcn_readfirstlane(int(x >> 32));
  p = reinterpret_cast<const uint8_t*>(uint64_t(hi) << 32 | lo);
  asm("" : "+s"(p));
  return p;
}

// x, which the compiler is not to extend to 64 bits elsewhere: an offset beside a scalar base
MOLT_DEV uint32_t here(uint32_t x) {
  asm("" : "+v"(x));
  return x;
}

// x as P bf16 or f16 values whose sum is x to 8 P or 11 P bits
template <int P, typename E>
MOLT_DEV void split(float x, E (&part)[P]) {
#pragma unroll
  for (int i = 0; i < P; ++i) {
    part[i] = E(x);
    x -= float(part[i]);                 // exact
  }
}

typedef _Float16 f16x8_t __attribute__((ext_vector_type(8)));
MOLT_DEV floatx4_t mfma_16x16x32(bf16x8_t a, bf16x8_t b, floatx4_t c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}
MOLT_DEV floatx4_t mfma_16x16x32(f16x8_t a, f16x8_t b, floatx4_t c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
}

// Query row as B operands of 16x16x32 bf16 MFMAs: three bf16 parts of dims D / 4 * g4 + 8 s .. +7 for k-step s, the
// order in which a lane's K codes lie. The parts are cut off, not rounded: three times 8 bits are the element's 24, and
// the largest elements do not round up to infinity.
template <int D>
MOLT_DEV void load_query_f32(const float* q, bool valid, int g4, bf16x8_t (&qf)[3][D / 32]) {
#pragma unroll
  for (int s = 0; s < D / 32; ++s) {
    floatx4_t x[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
    if (valid) {
      x[0] = *reinterpret_cast<const UnalignedF4*>(q + D / 4 * g4 + 8 * s);
      x[1] = *reinterpret_cast<const UnalignedF4*>(q + D / 4 * g4 + 8 * s + 4);
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      float rest = x[e / 4][e % 4];
#pragma unroll
      for (int u = 0; u < 3; ++u) {
        const float top = __uint_as_float(__float_as_uint(rest) & 0xffff0000u);
        qf[u][s][e] = __bf16(top);         // exact
        rest -= top;
      }
    }
  }
}

// Query row as B operands of 16x16x128 scaled MFMAs, whose A operand takes K's e2m1 codes and scale bytes
// as they lie in the cache. A bf16 value has 8 significant bits, an e4m3 one 4: with the row scaled by
// 2^-e so that its largest magnitude is in [128, 256), hi = e4m3(x 2^-e) leaves a rest of at most half a
// step, and lo = e4m3(rest 2^5) holds the rest exactly while it is a normal number; what smaller elements
// lose is under 2^-22 of the row's largest. So x = 2^e hi + 2^(e - 5) lo, the e8m0 bytes being the B scales.
// Lane (row, g4) holds k = 16 g4 .. +15 in the first 4 registers and 64 + 16 g4 .. +15 in the others. For D =
// 128, qp[0] is hi and qp[1] lo, k the dim; for D = 64 k = 0 .. 63 is hi, 64 .. 127 lo, with K's codes
// twice in the A operand. qs: the scale byte of the lane's k block (and for D = 128 lo's in the second byte).
template <int D>
MOLT_DEV void split_query_bf16(const u32x4 (&raw)[D / 64][2], int g4, int32x8_t (&qp)[D / 64], int& qs) {
  float x[D / 64][16];
  uint32_t amax = 0;
#pragma unroll
  for (int c = 0; c < D / 64; ++c)
#pragma unroll
    for (int v = 0; v < 2; ++v) {
      const u32x4 w = raw[c][v];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        x[c][8 * v + 2 * e] = __uint_as_float(w[e] << 16);
        x[c][8 * v + 2 * e + 1] = __uint_as_float(w[e] & 0xffff0000u);
        amax = max(amax, max((w[e] << 16) & 0x7fffffffu, w[e] & 0x7fff0000u));
      }
    }
  const float am = rows_max4(__uint_as_float(amax > 0x7f800000u ? 0x7f800000u : amax));   // NaN as infinity
  const int byte = max(int(__float_as_uint(am) >> 23) - 7, 6);
  const bool bad = __float_as_uint(am) == 0x7f800000u;     // an infinity or NaN: a row of NaN scores
  const float inv = __uint_as_float(uint32_t(254 - byte) << 23);
#pragma unroll
  for (int c = 0; c < D / 64; ++c)
#pragma unroll
    for (int v = 0; v < 4; ++v) {
      uint32_t hi = 0, lo = 0;
      float y[4], t[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) y[e] = x[c][4 * v + e] * inv;
      hi = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], hi, false);
      hi = __builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], hi, true);
      const auto a = __builtin_amdgcn_cvt_pk_f32_fp8(hi, false), b = __builtin_amdgcn_cvt_pk_f32_fp8(hi, true);
      t[0] = (y[0] - a[0]) * 32.f;
      t[1] = (y[1] - a[1]) * 32.f;
      t[2] = (y[2] - b[0]) * 32.f;
      t[3] = (y[3] - b[1]) * 32.f;
      lo = __builtin_amdgcn_cvt_pk_fp8_f32(t[0], t[1], lo, false);
      lo = __builtin_amdgcn_cvt_pk_fp8_f32(t[2], t[3], lo, true);
      if constexpr (D == 128) {
        qp[0][4 * c + v] = int(hi);
        qp[1][4 * c + v] = int(lo);
      } else {
        qp[0][v] = int(hi);
        qp[0][4 + v] = int(lo);
      }
    }
  qs = bad ? 0xffff : D == 128 ? byte | (byte - 5) << 8 : g4 < 2 ? byte : byte - 5;
}

// 4 output dims from column c of output row t on
template <typename T>
MOLT_DEV void store4(const KvqAttnParams& p, long t, long c, int D, const floatx4_t& a) {
  const long cols = long(p.Hq) * D;
  T* out = static_cast<T*>(p.out) + (p.out_tiled ? tiled_index(t, c, cols, sizeof(T)) : t * cols + c);
  if constexpr (sizeof(T) == 4)
    *reinterpret_cast<UnalignedF4*>(out) = a;
  else
    *reinterpret_cast<UnalignedU2*>(out) = u32x2{f32x2_to_bf16(a[0], a[1]), f32x2_to_bf16(a[2], a[3])};
}

// 1 / L, 0 for a row that sees no key
MOLT_DEV float inverse(float L) { return L == 0.f ? 0.f : 1.f / L; }

// dims d0 .. + 3 of row r of (b, h)
template <typename T>
MOLT_DEV void store_out4(const KvqAttnParams& p, int b, int h, int r, int D, int d0, const floatx4_t& a, float L) {
  store4<T>(p, long(b) * p.n + r / p.G, long(h * p.G + r % p.G) * D + d0, D, a * inverse(L));
}

// The work of slot `slot` of a row group (whose rows end before r1): part `part` of `parts` of sequence b, whose
// slots start at `first`; b < 0: none.
struct Share { int b, part, parts, first; };

// Few sequences, or sequences of uneven lengths, are cut into parts of about c pairs of blocks: max(1, ceil(T / c))
// of a sequence of T pairs. The lengths are known on the device only, so every workgroup works out c and its own
// place (a microsecond). Lane j weighs one of 64 values of c, from no cut at all down, by the time it would take, in
// pairs of blocks: the longest part, or all parts and what each costs besides (its start and its join of
// wavefronts, kPartCost) over the workgroups that are resident, half a part more where they do not all fit at
// once, and the joining launch (kJoinCost) if anything is cut. Of equal ones the longest c wins. The choice is flat about
// these constants: with half and twice kPartCost, and with none or a whole part more for the second round, 11 cut calls
// (1 to 100 sequences at contexts of 0 to 65536, both types) took within 4% of the same.
constexpr int kMaxCut = 256, kMinPairs = 4;
constexpr float kJoinCost = 15.f;       // (73 x 9 positions x 16 heads at 824-1649: 30.0 us, 34.4 with 30; others alike)
MOLT_DEV float cut(float pairs, float inv_c) { return fmaxf(1.f, ceilf(pairs * inv_c)); }

template <int NT>
MOLT_DEV Share find_share(const KvqAttnParams& p, int r1, int slot, float* lds) {
  constexpr int kPer = kMaxCut / kWave;
  constexpr float kPartCost = 48.f / NT;
  const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  float pairs[kPer];                     // of sequences lane, lane + 64, .. (in every wavefront)
  float sum = 0.f, most = 0.f;
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    const int b = lane + kWave * i;
    pairs[i] = b < p.B ? float((visible_end(p, p.ctx[b], r1) + 31) / 32) : -1.f;
    sum += fmaxf(pairs[i], 0.f);
    most = fmaxf(most, pairs[i]);
  }
  sum = wave_sum_dpp(sum);
  most = fmaxf(wave_max_dpp(most), float(kMinPairs));
  const float least = fminf(fmaxf(sum / float(p.slots), float(kMinPairs)), most);
  // (hardware approximations: the same in every workgroup)
  const float c = lane == 0 ? most : most * __builtin_amdgcn_exp2f(__builtin_amdgcn_logf(least / most) * (float(lane) / 63.f));
  // (and a little less than 1 / c: T pairs with c = T are one part)
  const float inv = __builtin_amdgcn_rcpf(c) * (1.f - 0x1p-20f);
  float n = 0.f;                         // parts with the lane's c; each wavefront counts 16 of 64 sequences
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    if (kWave * i >= p.B) break;
#pragma unroll
    for (int j = 0; j < kWave / kWaves; ++j) {      // (past the last sequence: no part)
      const float t = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(pairs[i]), wave * (kWave / kWaves) + j));
      n += t < 0.f ? 0.f : cut(t, inv);
    }
  }
  lds[wave * kWave + lane] = n;
  __syncthreads();
  n = lds[lane] + lds[kWave + lane] + lds[2 * kWave + lane] + lds[3 * kWave + lane];
  __syncthreads();
  const float res = float(p.resident) / (float(p.Hkv) * float(p.nrg));
  float cost = fmaxf(c + kPartCost, (sum + n * kPartCost) / res + (n > res ? 0.5f * c : 0.f));
  if (n > float(p.B)) cost += kJoinCost;
  if (n > float(p.slots)) cost = INFINITY;
  const float best = -wave_max_dpp(-cost);
  const int pick = __ffsll((unsigned long long)__ballot(cost == best)) - 1;
  const float inv_c = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(inv), pick));
  // the sequence that has the slot
  int before = 0;
  Share w{-1, 0, 1, 0};
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    if (kWave * i >= p.B || w.b >= 0) break;
    const int parts = lane + kWave * i < p.B ? int(cut(pairs[i], inv_c)) : 0;
    const int upto = before + wave_scan_dpp(parts);
    const unsigned long long has = __ballot(slot < upto);
    if (has) {
      const int l = __ffsll(has) - 1;
      w.b = kWave * i + l;
      w.parts = __builtin_amdgcn_readlane(parts, l);
      w.first = __builtin_amdgcn_readlane(upto, l) - w.parts;
      w.part = slot - w.first;
    }
    before = __builtin_amdgcn_readlane(upto, 63);
  }
  return w;
}

// bytes of LDS: the wavefronts' rings, later their results; the query operands (bf16)
template <int D, typename T, int NT, int W>
struct Lds {
  static constexpr int kSlots = slots_of(W);
  static constexpr int kPair = 32 * D + 256;                  // bytes of a pair in the ring
  static constexpr int kJoin = (16 * (D + 4) + 32) * 4;       // a wavefront's results of one tile
  static constexpr int kWaveBytes = kSlots * kPair > kJoin ? kSlots * kPair : kJoin;
  static constexpr int kQuery = sizeof(T) == 4 ? 0 : D / 64 * 2048;   // a tile's query operands
  static constexpr int kBytes = W * kWaveBytes + NT * kQuery;
};

template <bool HALF, int I>
MOLT_DEV uint32_t decode2(uint32_t codes, uint32_t scale_bits) {
  if constexpr (HALF) return kvq_decode2_f16<I>(codes, scale_bits);
  else return kvq_decode2<I>(codes, scale_bits);
}

// Adds a pair's weights exp2(sv - ref) to the rows' sums ls and its values, times them, to O^T. Both are taken as type E,
// the weights in P parts. codes: the pair's V codes in LDS, vs: the lane's V scale bytes. (As a lambda within attend this
// took 15 registers more of the f32 kernels: 143 us in place of 138 for 201 x 180 positions x 8 heads of 64 at 0-404.)
template <int D, bool F32, int NT, int P, typename E>
MOLT_DEV void add_pair(const floatx4_t (&sv)[2][NT], const float (&ref)[NT], const uint32_t (&vs)[2], const uint8_t* codes,
                       int lane, floatx4_t (&ls)[NT], floatx4_t (&o)[NT][D / 16], E) {
  typedef E Frag __attribute__((ext_vector_type(8)));
  constexpr bool HALF = std::is_same<E, _Float16>::value;
  constexpr int DT = D / 16;
  const int l16 = lane % 16, g4 = lane / 16;
  Frag pf[NT][P];
#pragma unroll
  for (int i = 0; i < NT; ++i) {
    float ps = 0.f;
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float w = __builtin_amdgcn_exp2f(sv[u][i][e] - ref[i]);
        if constexpr (F32) ps += w;
        E part[P];
        split<P>(w, part);
#pragma unroll
        for (int q = 0; q < P; ++q) pf[i][q][4 * u + e] = part[q];
      }
    if constexpr (F32) {
      ls[i][0] += ps;
    } else {
      const uint32_t one = HALF ? 0x3c003c00u : 0x3f803f80u;
      const u32x4 ones = {one, one, one, one};
#pragma unroll
      for (int q = 0; q < P; ++q) ls[i] = mfma_16x16x32(__builtin_bit_cast(Frag, ones), pf[i][q], ls[i]);
    }
  }
  // O^T += V^T P^T: lane (l16, g4) holds dims D / 16 * l16 + t (tile t) of tokens 4 g4 .. +3 of both blocks
  const uint8_t* src = codes + (D == 128 ? lane : g4 * 8 + l16 / 2) * 16;
  uint32_t vd[2][4][DT / 2];           // token's dims in pairs
#pragma unroll
  for (int u = 0; u < 2; ++u) {
    const u32x4 vc = *reinterpret_cast<const u32x4*>(src + 8 * D * u);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const uint32_t sc = kvq_scale_bits(vs[u], e);
      const uint32_t w = D == 128 ? vc[e] : vc[e] >> (16 * (l16 % 2));
      vd[u][e][0] = decode2<HALF, 0>(w, sc);
      vd[u][e][1] = decode2<HALF, 1>(w, sc);
      if constexpr (D == 128) {
        vd[u][e][2] = decode2<HALF, 2>(w, sc);
        vd[u][e][3] = decode2<HALF, 3>(w, sc);
      }
    }
  }
#pragma unroll
  for (int t = 0; t < DT; ++t) {
    u32x4 w;
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int e = 0; e < 2; ++e)
        w[2 * u + e] = __builtin_amdgcn_perm(vd[u][2 * e + 1][t / 2], vd[u][2 * e][t / 2], t % 2 ? 0x07060302u : 0x05040100u);
    const Frag vf = __builtin_bit_cast(Frag, w);
#pragma unroll
    for (int i = 0; i < NT; ++i)
#pragma unroll
      for (int q = 0; q < P; ++q) o[i][t] = mfma_16x16x32(vf, pf[i][q], o[i][t]);
  }
}

// Rows [r0, r0 + 16 NT) of kv head h over the keys of share w, by W wavefronts.
template <int D, typename T, int NT, bool ONCE, int W>
MOLT_DEV void attend(const KvqAttnParams& p, uint8_t* lds, int rg, int r0, int h, int slot, const Share& w) {
  typedef KvqRecord<D> Rec;
  constexpr bool F32 = sizeof(T) == 4;
  constexpr int kSlots = slots_of(W);
  constexpr int QP = 3;                  // bf16 parts of an f32 query element
  constexpr int KS = D / 32;             // MFMA steps over the dims of a score
  constexpr int DT = D / 16;             // 16-dim tiles of O^T
  constexpr int SLOT = Lds<D, T, NT, W>::kPair, kLds = Lds<D, T, NT, W>::kWaveBytes, QF = Lds<D, T, NT, W>::kQuery;
  constexpr int kCopies = D == 128 ? 5 : 3;   // vector memory instructions of a pair
  const int r1 = min(r0 + 16 * NT, p.R);
  const int b = w.b;
  const int lane = threadIdx.x % kWave, l16 = lane % 16, g4 = lane / 16;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  // The query rows are loaded first: behind the copies of keys and values they would wait for those. Wavefront i
  // makes the operands of tiles i, i + W, ..
  constexpr int QT = F32 ? 1 : (NT + W - 1) / W;
  long qrow[QT];
  u32x4 raw[QT][D / 64][2];
#pragma unroll
  for (int x = 0; x < QT; ++x) {
    const int qr = min(r0 + (F32 ? 0 : 16 * min(wave + W * x, NT - 1)) + l16, p.R - 1);
    qrow[x] = ((long(b) * p.n + qr / p.G) * p.Hq + h * p.G + qr % p.G) * D;
    if constexpr (!F32) {
      const uint16_t* src = static_cast<const uint16_t*>(p.q) + qrow[x] + 16 * g4;
#pragma unroll
      for (int c = 0; c < D / 64; ++c)
#pragma unroll
        for (int v = 0; v < 2; ++v) raw[x][c][v] = *reinterpret_cast<const UnalignedU4*>(src + 64 * c + 8 * v);
    }
  }
  const int ctx = p.ctx[b];
  const int end = visible_end(p, ctx, r1);
  const int nblk = (end + 15) / 16, npairs = (nblk + 1) / 2;
  int lim[NT];                           // last key that a row sees (past the last row: as the last)
#pragma unroll
  for (int i = 0; i < NT; ++i) lim[i] = visible_end(p, ctx, min(r0 + 16 * i + l16, p.R - 1) + 1) - 1;
  // the share's pairs of blocks, then the wavefront's
  const int s0 = int(long(npairs) * w.part / w.parts), s1 = int(long(npairs) * (w.part + 1) / w.parts);
  const int each = (s1 - s0) / W, more = (s1 - s0) % W;
  const int p0 = s0 + each * wave + min(wave, more), p1 = p0 + each + (wave < more ? 1 : 0);
  const int full_end = min(visible_end(p, ctx, r0 + 1), end);    // keys before are seen by every row
  uint8_t* ring = lds + wave * kLds;
  const uint32_t ring_at = uint32_t(uintptr_t((LdsPtr)ring));     // its LDS address
  uint8_t* qlds = lds + W * kLds;

  // Copies of a pair into a slot of the wavefront's ring: [K codes of both blocks][V codes][scales of K, of
  // V], K's 16-byte chunks in the order in which the lanes read them (dims 32 c .. of token t at chunk 16 c + t)
  typedef const __attribute__((address_space(4))) int32_t* ConstInt;
  const ConstInt btab = (ConstInt)(p.bt + long(b) * p.max_blocks);
  constexpr uint32_t SR = D / 32 * 4;    // lanes (dwords) of a record's scales
  const uint32_t ksrc = D == 128 ? l16 * 64 + g4 * 16 : l16 * 32 + g4 % 2 * 16;
  const uint32_t vsrc = D == 128 ? lane * 16 : lane % 32 * 16;
  const uint32_t spart = lane / SR % 4;
  const uint8_t* sbase = (spart < 2 ? p.kc : p.vc) + Rec::kCodes + lane % SR * 4;
  asm("" : "+v"(sbase));                 // (or the constant is added at every copy)
  auto issue = [&](int pi, const int (&id)[2]) __attribute__((always_inline)) {
    const uint32_t dst = in_sgpr(ring_at + uint32_t(pi - p0) % kSlots * SLOT);
    long rec[2];
#pragma unroll
    for (int u = 0; u < 2; ++u) rec[u] = (long(unsigned(id[u]) < unsigned(p.num_blocks) ? id[u] : 0) * p.Hkv + h) * Rec::kBytes;
    if constexpr (D == 128) {            // a base in scalar registers and a lane offset per copy
#pragma unroll
      for (int u = 0; u < 2; ++u) copy_lds16<ONCE>(in_sgpr(p.kc + rec[u]) + here(ksrc), dst + 1024 * u);
#pragma unroll
      for (int u = 0; u < 2; ++u) copy_lds16<ONCE>(in_sgpr(p.vc + rec[u]) + here(vsrc), dst + 2048 + 1024 * u);
    } else {
      const long r = lane < 32 ? rec[0] : rec[1];
      copy_lds16<ONCE>(p.kc + r + ksrc, dst);
      copy_lds16<ONCE>(p.vc + r + vsrc, dst + 1024);
    }
    copy_lds4<ONCE>(sbase + (spart % 2 ? rec[1] : rec[0]), dst + 32 * D);
  };
  auto ids = [&](int pi, int (&id)[2]) __attribute__((always_inline)) {
    id[0] = btab[min(2 * pi, nblk - 1)];
    const int second = btab[min(2 * pi + 1, nblk - 1)];
    id[1] = 2 * pi + 1 < nblk ? second : -1;
  };
  auto present = [&](const int (&id)[2]) __attribute__((always_inline)) {
    return (unsigned(id[0]) < unsigned(p.num_blocks) ? 1u : 0u) | (unsigned(id[1]) < unsigned(p.num_blocks) ? 2u : 0u);
  };
  uint32_t have = 0;                     // presence bits of the pairs in flight, the newest lowest
  int nid[2] = {-1, -1};
  if (p0 < p1) {
    int first[kSlots][2];
#pragma unroll
    for (int u = 0; u < kSlots; ++u) ids(p0 + u, first[u]);
#pragma unroll
    for (int u = 0; u < kSlots - 1; ++u) {
      if (p0 + u < p1) issue(p0 + u, first[u]);
      have = have << 2 | present(first[u]);
    }
    nid[0] = first[kSlots - 1][0];
    nid[1] = first[kSlots - 1][1];
  }

  // the query operands: in f32 each wavefront's own, in bf16 in LDS for all
  bf16x8_t qf[QP][KS];
  int qs[NT];                            // scale bytes of both fp8 parts
  if constexpr (F32) {
    load_query_f32<D>(static_cast<const float*>(p.q) + qrow[0], r0 + l16 < p.R, g4, qf);
  } else {
#pragma unroll
    for (int x = 0; x < QT; ++x) {
      const int tile = wave + W * x;
      if (tile >= NT) break;
      int32x8_t qp[D / 64];
      int sc;
      split_query_bf16<D>(raw[x], g4, qp, sc);
#pragma unroll
      for (int u = 0; u < D / 64; ++u) {
        int32x4_t* dst = reinterpret_cast<int32x4_t*>(qlds + tile * QF + u * 2048 + lane * 16);
        dst[0] = int32x4_t{qp[u][0], qp[u][1], qp[u][2], qp[u][3]};
        dst[64] = int32x4_t{qp[u][4], qp[u][5], qp[u][6], qp[u][7]};
      }
      reinterpret_cast<int*>(ring + (kSlots - 1) * SLOT)[64 * x + lane] = sc;   // in a slot not yet in use
    }
    lds_barrier();
#pragma unroll
    for (int i = 0; i < NT; ++i)
      qs[i] = reinterpret_cast<const int*>(lds + i % W * kLds + (kSlots - 1) * SLOT)[64 * (i / W) + lane];
    lds_barrier();
  }
  floatx4_t o[NT][DT], ls[NT];           // O^T; the rows' sums (bf16: by MFMA, the same in every register and group)
  float m[NT];                           // reference maximum (of scores in log2 units)
  float shift = F32 ? 0.f : kWeightShift;   // weights are exp2(score - ref), ref = m - shift, or 0 for a row that has
  float ref[NT];                            // seen no key: its exp2(-inf) is 0
  float bound[NT];                       // scores above it raise m
#pragma unroll
  for (int i = 0; i < NT; ++i) {
    m[i] = bound[i] = -INFINITY;
    ref[i] = 0.f;
    ls[i] = floatx4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int t = 0; t < DT; ++t) o[i][t] = floatx4_t{0.f, 0.f, 0.f, 0.f};
  }

  // S^T of pair pi and its V scale bytes: lane (row l16 of the tile) holds tokens 4 g4 + e of both blocks.
  // Lane (l16, g4) reads the codes of K's token l16, dims 32 g4 .. (D = 64: 32 (g4 % 2) .., in f32 16 g4 ..),
  // and its scale byte
  auto scores = [&](int pi, floatx4_t (&sv)[2][NT], uint32_t (&vs)[2]) __attribute__((always_inline)) {
    const uint8_t* src = ring + (pi - p0) % kSlots * SLOT;
    u32x4 k[2];
    uint32_t ks[2];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const uint8_t *kr = src + 8 * D * u, *sr = src + 32 * D + D / 2 * u;
      if constexpr (F32 && D == 64) {
        const u32x2 w = *reinterpret_cast<const u32x2*>(kr + (g4 / 2 * 16 + l16) * 16 + g4 % 2 * 8);
        k[u][0] = w[0];
        k[u][1] = w[1];
        ks[u] = sr[l16 * 2 + g4 / 2];
      } else {
        k[u] = *reinterpret_cast<const u32x4*>(kr + (D == 128 ? lane : lane % 32) * 16);
        ks[u] = sr[l16 * (D / 32) + g4 % (D / 32)];
      }
      vs[u] = *reinterpret_cast<const uint32_t*>(sr + D + (g4 * (D / 32) + l16 * (D / 16) / 32) * 4);
#pragma unroll
      for (int i = 0; i < NT; ++i) sv[u][i] = floatx4_t{0.f, 0.f, 0.f, 0.f};
    }
    if constexpr (F32) {
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int s = 0; s < KS; ++s) {
          const uint32_t sc = ks[u] << 23;
          const u32x4 w = {kvq_decode2<0>(k[u][s], sc), kvq_decode2<1>(k[u][s], sc),
                           kvq_decode2<2>(k[u][s], sc), kvq_decode2<3>(k[u][s], sc)};
          const bf16x8_t kf = __builtin_bit_cast(bf16x8_t, w);
#pragma unroll
          for (int q = 0; q < QP; ++q) sv[u][0] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, qf[q][s], sv[u][0], 0, 0, 0);
        }
    } else {
#pragma unroll
      for (int i = 0; i < NT; ++i)
#pragma unroll
        for (int q = 0; q < D / 64; ++q) {
          const int32x4_t* f = reinterpret_cast<const int32x4_t*>(qlds + i * QF + q * 2048 + lane * 16);
          const int32x4_t f0 = f[0], f1 = f[64];
          const int32x8_t qp = {f0[0], f0[1], f0[2], f0[3], f1[0], f1[1], f1[2], f1[3]};
#pragma unroll
          for (int u = 0; u < 2; ++u) {  // formats: A 4 (e2m1), B 0 (e4m3)
            const int32x8_t kf = {int(k[u][0]), int(k[u][1]), int(k[u][2]), int(k[u][3]), 0, 0, 0, 0};
            if (q == 0) sv[u][i] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(kf, qp, sv[u][i], 4, 0, 0, int(ks[u]), 0, qs[i]);
            else sv[u][i] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(kf, qp, sv[u][i], 4, 0, 0, int(ks[u]), 1, qs[i]);
          }
        }
    }
  };

  // What follows a pair's scores: masks where a row may not see a key, and the reference maxima.
  auto settle = [&](int pi, bool ok0, bool ok1, const floatx4_t (&raw)[2][NT], floatx4_t (&sv)[2][NT],
                    uint32_t (&vs)[2], auto half) __attribute__((always_inline)) {
    float mx[NT];
    auto maxima = [&]() __attribute__((always_inline)) {
#pragma unroll
      for (int i = 0; i < NT; ++i)
        mx[i] = fmaxf(fmaxf(fmaxf(fmaxf(sv[0][i][0], sv[0][i][1]), sv[0][i][2]),
                            fmaxf(fmaxf(sv[0][i][3], sv[1][i][0]), sv[1][i][1])),
                      fmaxf(sv[1][i][2], sv[1][i][3]));
    };
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int i = 0; i < NT; ++i) sv[u][i] = raw[u][i] * p.c;
    maxima();                            // beside the products, which the compiler knows to need no quieting
    if (32 * pi + 32 > full_end || !ok0 || !ok1) {
      // Keys that some row may not see: their scores are -inf for it, and their values must not reach it.
      // A probability of 0 does that, unless the value is NaN (scale byte 255, also in slots that were
      // never written): such groups are taken as codes times 1, and the rows that do see one get NaN in the
      // group's dims at once (O stays NaN).
      uint32_t bad = 0;
      int first = 32 * pi + 4 * g4;
      asm volatile("" : "+v"(first));     // or the comparisons are hoisted out of the branch
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int pos = first + 16 * u + e;
          const bool seen = pos < end && (u == 0 ? ok0 : ok1);
#pragma unroll
          for (int i = 0; i < NT; ++i) sv[u][i][e] = seen && pos <= lim[i] ? sv[u][i][e] : -INFINITY;
          const uint32_t byte = (vs[u] >> (8 * e)) & 255u;
          if (!seen || byte == kKvqScaleNan) vs[u] = (vs[u] & ~(255u << (8 * e))) | (127u << (8 * e));
          if (seen && byte == kKvqScaleNan) bad |= 1u << (4 * u + e);
        }
      if (__ballot(bad != 0)) {
        // output lane (row l16, g4) holds dims D / 4 * g4 .. of its row: group g4 * D / 128, whose scales
        // lanes of dims in it (l16 * D / 16) hold
        bool poison[NT];
#pragma unroll
        for (int i = 0; i < NT; ++i) poison[i] = false;
#pragma unroll 1
        for (int t = 0; t < 32; ++t) {   // the pair's tokens
          const uint32_t w = uint32_t(__shfl(int(bad), t % 16 / 4 * 16 + (g4 * D / 128) * (512 / D)));
          const bool nan = w >> (t / 16 * 4 + t % 4) & 1u;
#pragma unroll
          for (int i = 0; i < NT; ++i) poison[i] |= nan && 32 * pi + t <= lim[i];
        }
#pragma unroll
        for (int i = 0; i < NT; ++i)
#pragma unroll
          for (int t = 0; t < DT; ++t) o[i][t] += poison[i] ? __builtin_nanf("") : 0.f;
      }
      maxima();
    }
    bool grow = false;
#pragma unroll
    for (int i = 0; i < NT; ++i) grow |= mx[i] > bound[i];
    bool wide = false;
    if constexpr (decltype(half)::value) wide = kvq_outside_f16(vs[0], vs[1]) != 0;
    if (__ballot(grow || wide)) {
      if (__ballot(wide)) shift = 0.f;   // from f16 weights and values to bf16 ones, before they meet
#pragma unroll
      for (int i = 0; i < NT; ++i) {
        const float mn = fmaxf(m[i], rows_max4(mx[i]));
        // (scores past 2^20 are 2^-3 and more apart: the shift would be rounded)
        const float next = mn == -INFINITY ? 0.f : fabsf(mn) < 0x1p20f ? mn - shift : mn;
        const float alpha = m[i] == -INFINITY ? 0.f : exp2f(ref[i] - next);
        m[i] = mn;
        bound[i] = mn + kRescaleSlack;
        ref[i] = next;
        ls[i] *= alpha;
#pragma unroll
        for (int t = 0; t < DT; ++t) o[i][t] *= alpha;
      }
    }
  };

  typedef std::conditional_t<F32, __bf16, _Float16> First;   // what weights and values are held in at first
  constexpr std::integral_constant<bool, !F32> first{};       // (and whether that may change)
  floatx4_t sv[2][NT];
  uint32_t vs[2];
  // Pair pi is in when at most the copies of the pairs after it are in flight. The reads of pair pi - 2 are
  // done, so its slot takes pair pi + kSlots - 2.
  auto arrive = [&](int pi) __attribute__((always_inline)) {
    if (pi + kSlots - 3 < p1) asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"((kSlots - 3) * kCopies) : "memory");
    else asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
  };
  if (p0 < p1) {
    if (p0 + kSlots - 2 < p1) asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"((kSlots - 2) * kCopies) : "memory");
    else asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
    floatx4_t raw[2][NT];
    scores(p0, raw, vs);
    settle(p0, have >> (2 * kSlots - 4) & 1u, have >> (2 * kSlots - 4) & 2u, raw, sv, vs, first);
  }
  auto advance = [&](int pi) __attribute__((always_inline)) {
    arrive(pi + 1);
    if (pi + kSlots - 1 < p1) issue(pi + kSlots - 1, nid);
    have = have << 2 | present(nid);
    ids(pi + kSlots, nid);
  };
  // In each loop the scores of the next pair (past the last: of whatever its slot holds, not used) go beside the weights
  // and values of this one. The stretch without MFMAs, settle, goes first, so that the other wavefront's run beside it
  // (2 x 257 positions at 8100 took 2% more with the priorities the other way round, 9% without).
  int pi = p0;
  for (; pi < p1 && (F32 || shift != 0.f); ++pi) {
    advance(pi);
    __builtin_amdgcn_s_setprio(0);
    floatx4_t nsv[2][NT];
    uint32_t nvs[2];
    scores(pi + 1, nsv, nvs);
    add_pair<D, F32, NT, F32 ? 3 : 1>(sv, ref, vs, ring + (pi - p0) % kSlots * SLOT + 16 * D, lane, ls, o, First());
    __builtin_amdgcn_s_setprio(1);
    if (pi + 1 < p1)
      settle(pi + 1, have >> (2 * kSlots - 4) & 1u, have >> (2 * kSlots - 4) & 2u, nsv, sv, nvs, first);
    vs[0] = nvs[0];
    vs[1] = nvs[1];
  }
  if constexpr (!F32) {
    for (; pi < p1; ++pi) {
      advance(pi);
      __builtin_amdgcn_s_setprio(0);
      floatx4_t nsv[2][NT];
      uint32_t nvs[2];
      scores(pi + 1, nsv, nvs);
      add_pair<D, F32, NT, 2>(sv, ref, vs, ring + (pi - p0) % kSlots * SLOT + 16 * D, lane, ls, o, __bf16());
      __builtin_amdgcn_s_setprio(1);
      if (pi + 1 < p1)
        settle(pi + 1, have >> (2 * kSlots - 4) & 1u, have >> (2 * kSlots - 4) & 2u, nsv, sv, nvs, std::false_type());
      vs[0] = nvs[0];
      vs[1] = nvs[1];
    }
  }
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // no copy may outlive the ring

  if constexpr (W == 1) {                // nothing to join
#pragma unroll
    for (int i = 0; i < NT; ++i) {
      const float L = F32 ? rows_sum4(ls[i][0]) : ls[i][0];
      const int r = r0 + 16 * i + l16;
      if (r >= p.R) continue;
#pragma unroll
      for (int e = 0; e < 4; ++e)
#pragma unroll
        for (int t = 0; t < DT; t += 4)
          store_out4<T>(p, b, h, r, D, D / 4 * g4 + DT * e + t,
                        floatx4_t{o[i][t][e], o[i][t + 1][e], o[i][t + 2][e], o[i][t + 3][e]}, L);
    }
    return;
  }
  // the wavefronts' shares joined through LDS, one 16-row tile at a time
  constexpr int RS = D + 4;              // floats of a row, then 16 maxima and 16 sums
  float* own = reinterpret_cast<float*>(ring);
#pragma unroll
  for (int i = 0; i < NT; ++i) {
    const float lt = F32 ? rows_sum4(ls[i][0]) : ls[i][0];
    if (i > 0) __syncthreads();
#pragma unroll
    for (int e = 0; e < 4; ++e)
#pragma unroll
      for (int t = 0; t < DT; t += 4)   // dims D / 16 * (4 g4 + e) + t .. + 3
        *reinterpret_cast<floatx4_t*>(own + l16 * RS + D / 16 * (4 * g4 + e) + t) =
            floatx4_t{o[i][t][e], o[i][t + 1][e], o[i][t + 2][e], o[i][t + 3][e]};
    if (g4 == 0) {
      own[16 * RS + l16] = m[i] == -INFINITY ? m[i] : ref[i];
      own[16 * RS + 16 + l16] = lt;
    }
    __syncthreads();
    // thread = 8 dims of one row
    if (threadIdx.x >= 16 * (D / 8)) continue;
    const int row = threadIdx.x / (D / 8), d0 = threadIdx.x % (D / 8) * 8;
    const int r = r0 + 16 * i + row;
    if (r >= p.R) continue;
    const float* part = reinterpret_cast<const float*>(lds);
    float M = -INFINITY;
#pragma unroll
    for (int w = 0; w < W; ++w) M = fmaxf(M, part[w * (kLds / 4) + 16 * RS + row]);
    float L = 0.f;
    floatx4_t a[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
#pragma unroll
    for (int w = 0; w < W; ++w) {
      const float* pw = part + w * (kLds / 4);
      const float mw = pw[16 * RS + row];
      const float f = mw == -INFINITY ? 0.f : exp2f(mw - M);
      L += pw[16 * RS + 16 + row] * f;
      a[0] += *reinterpret_cast<const floatx4_t*>(pw + row * RS + d0) * f;
      a[1] += *reinterpret_cast<const floatx4_t*>(pw + row * RS + d0 + 4) * f;
    }
    if (w.parts == 1) {
      store_out4<T>(p, b, h, r, D, d0, a[0], L);
      store_out4<T>(p, b, h, r, D, d0 + 4, a[1], L);
    } else {
      const long pr = ((long(rg) * p.Hkv + h) * p.slots + slot) * p.group + 16 * i + row;
      *reinterpret_cast<floatx4_t*>(p.part_o + pr * D + d0) = a[0];
      *reinterpret_cast<floatx4_t*>(p.part_o + pr * D + d0 + 4) = a[1];
      if (d0 == 0) {
        p.part_ml[2 * pr] = M;
        p.part_ml[2 * pr + 1] = L;
      }
    }
  }
}

template <int D, typename T, int NT, bool ONCE, int W>
__global__ __launch_bounds__(W * kWave, 2) void kvq_attn_kernel(KvqAttnParams p) {
  __shared__ __attribute__((aligned(16))) uint8_t lds[Lds<D, T, NT, W>::kBytes];   // the only LDS object
  // Work item. Consecutive workgroups run on consecutive XCDs: the row groups of a slot and head, which read the same
  // keys, are 8 apart, and with many slots (spread) a slot's heads too, whose records share lines (read requests of 128
  // sequences x 4 heads at context 8192: 1.02 times the records' bytes, 1.07 with heads on neighbouring XCDs).
  const int bi = int(blockIdx.x), rg = bi / 8 % p.nrg, hi = bi / (8 * p.nrg), lo = bi % 8;
  const int h = p.spread ? hi % p.Hkv : (hi * 8 + lo) % p.Hkv;
  const int slot = p.spread ? hi / p.Hkv * 8 + lo : (hi * 8 + lo) / p.Hkv;
  if (slot >= p.slots) return;
  const int r0 = rg * 16 * NT, r1 = min(r0 + 16 * NT, p.R);
  Share w{slot, 0, 1, slot};
  if (W == kWaves && p.slots > p.B) {
    w = find_share<NT>(p, r1, slot, reinterpret_cast<float*>(lds));
    if (w.b < 0) return;
    if (h == 0 && w.part == 0 && threadIdx.x == 0) {
      p.split[2 * (long(rg) * p.B + w.b)] = w.first;
      p.split[2 * (long(rg) * p.B + w.b) + 1] = w.parts;
    }
  }
  // the last of several row groups may have a tile less
  if (NT == 3 && !ONCE && r1 - r0 <= 32) attend<D, T, 2, ONCE, W>(p, lds, rg, r0, h, slot, w);
  else attend<D, T, NT, ONCE, W>(p, lds, rg, r0, h, slot, w);
}

// log-sum-exp join of a sequence's slots, thread = 4 dims of one row. P = 1: a thread takes all slots; else P groups of
// threads every P-th, a row a workgroup, and then their sums through LDS.
template <int D, typename T, int P>
__global__ __launch_bounds__(256) void kvq_merge_kernel(KvqAttnParams p) {
  constexpr int O = D / 4, kU = 4;
  static_assert(P == 1 || P * O == 256, "a row or 256 / O rows a workgroup");
  const int d = threadIdx.x % O, g = P == 1 ? 0 : threadIdx.x / O;
  const int row = P == 1 ? int(blockIdx.x) * (256 / O) + int(threadIdx.x) / O : int(blockIdx.x);
  const int bh = row / p.R, r = row % p.R;
  const int b = bh / p.Hkv, h = bh % p.Hkv, rg = r / p.group;
  if (b >= p.B) return;
  const int2 sp = *reinterpret_cast<const int2*>(p.split + 2 * (long(rg) * p.B + b));
  if (sp.y == 1) return;
  const long pr0 = ((long(rg) * p.Hkv + h) * p.slots + sp.x) * p.group + r % p.group;
  float M = -INFINITY, L = 0.f;
  floatx4_t a = {0.f, 0.f, 0.f, 0.f};
  for (int s0 = g; s0 < sp.y; s0 += kU * P) {
    float2 ml[kU];
    floatx4_t o[kU];
#pragma unroll
    for (int u = 0; u < kU; ++u) {       // past the last: its own again, not added
      const long pr = pr0 + long(min(s0 + u * P, sp.y - 1)) * p.group;
      ml[u] = *reinterpret_cast<const float2*>(p.part_ml + 2 * pr);
      o[u] = *reinterpret_cast<const floatx4_t*>(p.part_o + pr * D + 4 * d);
    }
    float mn = M;
#pragma unroll
    for (int u = 0; u < kU; ++u) mn = fmaxf(mn, ml[u].x);
    // what has no maximum has seen no key, or NaN only: its factor is 0, its sum 0 or NaN
    const float ref = mn == -INFINITY ? 0.f : mn;
    const float f0 = exp2f(M - ref);
    M = mn;
    L *= f0;
    a *= f0;
#pragma unroll
    for (int u = 0; u < kU; ++u) {
      const bool live = s0 + u * P < sp.y;
      const float f = exp2f(ml[u].x - ref);
      L += live ? ml[u].y * f : 0.f;
#pragma unroll
      for (int e = 0; e < 4; ++e) a[e] += live ? o[u][e] * f : 0.f;
    }
  }
  if constexpr (P > 1) {
    __shared__ floatx4_t sum[256];
    __shared__ float2 stat[P];           // maximum and sum of the weights
    sum[threadIdx.x] = a;
    if (d == 0) stat[g] = make_float2(M, L);
    __syncthreads();
    if (g != 0) return;
#pragma unroll
    for (int u = 1; u < P; ++u) M = fmaxf(M, stat[u].x);
    const float ref = M == -INFINITY ? 0.f : M;
    L = 0.f;
    a = floatx4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int u = 0; u < P; ++u) {
      const float f = exp2f(stat[u].x - ref);
      L += stat[u].y * f;
      a += sum[u * O + d] * f;
    }
  }
  store_out4<T>(p, b, h, r, D, 4 * d, a, L);
}

constexpr int kMaxTiles = 3;             // 16-row tiles of a wavefront (bf16; one in f32)

// Row groups of as few 16-row tiles as cover the R rows. Slots: one per sequence where that gives as many workgroups
// as are resident (a cut for uneven lengths would cost 8% of even ones: the work of finding it, workgroups without a
// part, the joining launch), or the tables are short, else room for as many parts as are resident. Short: under
// kMinCut pairs, and where each workgroup has a compute unit and 8 wavefronts (kFew) those beat a cut for longer: us
// uncut and cut, with U workgroups at context 1000, 1400, 2000 and 3000, 1 sequence U = 4: 9.6, 10.7, 13.0, 16.9 and
// 10.9, 11.2, 11.5, 11.4; 8 sequences U = 32: 13.1, 14.6, 17.5, 22.0 and 15.4, 17.0, 19.1, 20.0; 30 sequences U = 240 of
// D = 64: 9.4, 10.6, 12.3, 15.3 and 16.6, 18.8, 19.5, 22.6.
constexpr int kMinCut = 24, kFew = 256;
// Wavefronts of an uncut workgroup, 1, 4 or 8: the fewer, the more workgroups run at a time and the less there is to
// join, the more, the sooner a long key range is done. The rule weighs rounds of workgroups by what one takes, a start and
// join and its pairs, with constants that fit what calls took, in us with 1, 4 and 8 wavefronts: 8 workgroups (3 tiles) of
// 1 pair 9.0, 9.0 and 9.5, of 4 pairs 12.2, 8.9 and 9.6, of 32 pairs 42, 17.4 and 15.4; 8 (f32, 64 dims) of 1 pair 5.2, 6.0
// and 5.7, of 32 pairs 31, 12.3 and 10.4; 1600 (3 tiles) of 1 pair 25, 33 and 58, of 4 to 8 pairs 33, 39 and 66; 2016 of 1
// pair (2.5 tiles) 26, 36 and 75; 1584 of 49 pairs (3 tiles) 167, 120 and 145; 19844 of up to 9 pairs (f32) 108, 256, 544.
constexpr int kMoreWaves = 8;
constexpr double kPairTime = 1.7;        // us of a wavefront for a pair of blocks
void set_plan(KvqAttnParams& p, int D, bool f32) {
  p.G = p.Hq / p.Hkv;
  p.R = p.G * p.n;
  const int tiles = (p.R + 15) / 16, most = f32 ? 1 : kMaxTiles;
  p.nrg = (tiles + most - 1) / most;
  const int nt = (tiles + p.nrg - 1) / p.nrg;
  p.group = 16 * nt;
  p.resident = 256 * (D == 128 || nt == 3 ? 2 : f32 || nt == 2 ? 3 : 4);   // by LDS and registers
  const long per = long(p.Hkv) * p.nrg, pairs = (p.max_blocks + 1) / 2;
  const long slots = std::min(p.resident / per, p.B * ((pairs + kMinPairs - 1) / kMinPairs));
  const bool longer = p.B * per <= kFew ? pairs > 2 * kMinCut + p.B * per / 2 : pairs >= kMinCut;
  p.slots = slots > p.B && p.B <= kMaxCut && longer ? int(slots) : p.B;
  p.spread = p.slots >= 64;
  p.waves = kWaves;
  if (p.slots == p.B) {
    // how many workgroups run at a time, and the us of one
    const int mem = slots_of(1) * (32 * D + 256) + (f32 ? 0 : D / 64 * 2048 * nt);   // Lds of one wavefront
    const double at_once[3] = {256.0 * std::min(8, 163840 / mem), double(p.resident), 256.0};
    const double each[3] = {4.0 + kPairTime * pairs, 7.0 + kPairTime * pairs / 4, 8.2 + kPairTime * pairs / 8};
    double best = 1e30;
    for (int i = 0; i < 3; ++i) {
      const double time = std::ceil(double(p.B) * per / at_once[i]) * each[i];
      if (time < best) { best = time; p.waves = i == 0 ? 1 : i == 1 ? kWaves : kMoreWaves; }
    }
  }
}

template <int D, typename T, int NT, bool ONCE>
void launch_w(const KvqAttnParams& p, unsigned grid, hipStream_t s) {
  if (p.waves == 1) kvq_attn_kernel<D, T, NT, ONCE, 1><<<grid, kWave, 0, s>>>(p);
  else if (p.waves == kWaves) kvq_attn_kernel<D, T, NT, ONCE, kWaves><<<grid, kWaves * kWave, 0, s>>>(p);
  else kvq_attn_kernel<D, T, NT, ONCE, kMoreWaves><<<grid, kMoreWaves * kWave, 0, s>>>(p);
}

template <int D, typename T, int NT>
void launch_nt(const KvqAttnParams& p, hipStream_t s) {
  const long units = p.spread ? (long(p.slots) + 7) / 8 * 8 * p.Hkv : (long(p.slots) * p.Hkv + 7) / 8 * 8;
  if constexpr (NT > 1 || sizeof(T) == 4) {      // (one tile of a bf16 row group is all there is)
    if (p.nrg > 1) return launch_w<D, T, NT, false>(p, unsigned(units * p.nrg), s);
  }
  launch_w<D, T, NT, true>(p, unsigned(units), s);
}

template <int D, typename T>
void launch_dt(const KvqAttnParams& p, hipStream_t s) {
  if constexpr (sizeof(T) == 4) {
    launch_nt<D, T, 1>(p, s);
  } else {
    if (p.group == 16) launch_nt<D, T, 1>(p, s);
    else if (p.group == 32) launch_nt<D, T, 2>(p, s);
    else launch_nt<D, T, 3>(p, s);
  }
  // (room for more than 8 slots a sequence: a row a workgroup; 1 sequence of 65536 keys x 4 kv heads: 4.7 us, by one
  // thread for all slots 16; 16 sequences with 8 slots each, 640 rows a head: 6.4 us, by one thread 4.7)
  const unsigned rows = unsigned(p.B * p.Hkv * p.R);
  constexpr int kRows = 1024 / D;        // of a workgroup
  if (p.slots > 8l * p.B) kvq_merge_kernel<D, T, kRows><<<rows, 256, 0, s>>>(p);
  else if (p.slots > p.B) kvq_merge_kernel<D, T, 1><<<(rows + kRows - 1) / kRows, 256, 0, s>>>(p);
}

void carve_parts(Carver& c, KvqAttnParams& p, int D) {
  if (p.slots <= p.B) return;
  const long rows = long(p.nrg) * p.Hkv * p.slots * p.group;
  p.part_o = c.take<float>(rows * D);
  p.part_ml = c.take<float>(rows * 2);
  p.split = c.take<int32_t>(2l * p.nrg * p.B);
}

}  // namespace

KvqPlan kvq_plan(int B, int n, int Hq, int Hkv, int D, int max_blocks, bool f32) {
  KvqAttnParams p{};
  p.B = B; p.n = n; p.Hq = Hq; p.Hkv = Hkv; p.max_blocks = max_blocks;
  set_plan(p, D, f32);
  return {p.nrg, p.group, p.slots, p.waves};
}

// (of the type that needs more)
size_t kvq_attention_ws_bytes(int B, int n, int Hq, int Hkv, int D, int max_blocks) {
  size_t most = 0;
  for (int f32 = 0; f32 < 2; ++f32) {
    KvqAttnParams p{};
    p.B = B; p.n = n; p.Hq = Hq; p.Hkv = Hkv; p.max_blocks = max_blocks;
    set_plan(p, D, f32 != 0);
    Carver c(nullptr, 0);
    carve_parts(c, p, D);
    if (c.used && c.used + 256 > most) most = c.used + 256;
  }
  return most;
}

hipError_t launch_kvq_attention(const void* q, const void* kc, const void* vc, const int32_t* bt,
                                const int32_t* ctx, int B, int n, int Hq, int Hkv, int D, int max_blocks,
                                int num_blocks, molt_dtype dt, void* out, bool out_tiled, void* ws,
                                hipStream_t s) {
  KvqAttnParams p{};
  p.q = q;
  p.kc = static_cast<const uint8_t*>(kc);
  p.vc = static_cast<const uint8_t*>(vc);
  p.bt = bt; p.ctx = ctx; p.out = out;
  p.B = B; p.n = n; p.Hq = Hq; p.Hkv = Hkv; p.max_blocks = max_blocks; p.num_blocks = num_blocks;
  p.c = kLog2e / sqrtf(float(D));
  p.out_tiled = out_tiled;
  set_plan(p, D, dt == MOLT_F32);
  Carver c(ws, 0);
  carve_parts(c, p, D);
  if (dt == MOLT_F32) {
    if (D == 128) launch_dt<128, float>(p, s); else launch_dt<64, float>(p, s);
  } else {
    if (D == 128) launch_dt<128, uint16_t>(p, s); else launch_dt<64, uint16_t>(p, s);
  }
  return hipGetLastError();
}

}  // namespace molt
