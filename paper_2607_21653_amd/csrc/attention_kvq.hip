// Multi-query paged attention over the 4-bit KV cache (format: kvq_format.h).
//   o_r = sum_p w_rp v_p,  w_r = softmax over p <= ctx_b + j(r) of q_r . k_p / sqrt(D)
// for the R = G * n rows (position j = r / G, query head h G + r % G) of sequence b and kv head h.
//
// Values and keys are exact in bf16, so the products' only roundings are those of the weights: in f32 three
// bf16 parts (24 bits); in bf16 one, with the sum taken of the rounded weights, by an MFMA with a row of ones.
// That adds a rounding like the output's own: rms error 2.07e-3 of the output's rms against 1.66e-3 with two
// parts, for which 128 sequences x 5 positions at context 8192 took 178 us, with one 135.
#include "internal.h"
#include "kvq_format.h"

namespace molt {
namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kRescaleSlack = 8.0f;   // probabilities may grow to 2^8 before O is rescaled
constexpr int kWaves = 4;
constexpr int kSlots = 4;               // pairs of blocks in a wavefront's ring

struct KvqAttnParams {
  const void* q;           // [B * n, Hq, D]
  const uint8_t* kc;
  const uint8_t* vc;
  const int32_t* bt;       // [B, max_blocks]
  const int32_t* ctx;      // [B]
  void* out;               // [B * n, Hq * D], row-major or tiled
  float* part_o;           // [B, Hkv, S, R, D]
  float* part_ml;          // [B, Hkv, S, R, 2]
  int B, n, Hq, Hkv, max_blocks, num_blocks;
  int G, R;                // query heads per kv head, rows of a (b, h)
  int nrg, group;          // row groups of a (b, h) and rows of one (16 NT)
  int splits, bps;         // splits of the longest table, blocks of one
  float c;                 // log2(e) / sqrt(D)
  int out_tiled;
};

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef bf16x8_t UnalignedBf16x8 __attribute__((aligned(2)));
typedef floatx4_t UnalignedF4 __attribute__((aligned(4)));
typedef u32x4 UnalignedU4 __attribute__((aligned(2)));

// Keys 0 .. end - 1 are those that rows [r0, r1) of sequence b may see (the last row the most).
MOLT_DEV int visible_end(const KvqAttnParams& p, int ctx, int r1) {
  const long e = long(ctx) + (r1 - 1) / p.G + 1;
  return int(e < 0 ? 0 : e > 16l * p.max_blocks ? 16l * p.max_blocks : e);
}

// LDS-DMA: 16 (4) bytes a lane from src to dst + 16 (4) * lane; dst is the wavefront's
typedef const __attribute__((address_space(1))) void* GlobalPtr;
typedef __attribute__((address_space(3))) void* LdsPtr;
MOLT_DEV void copy_lds16(const uint8_t* src, uint8_t* dst) { __builtin_amdgcn_global_load_lds((GlobalPtr)src, (LdsPtr)dst, 16, 0, 0); }
MOLT_DEV void copy_lds4(const uint8_t* src, uint8_t* dst) { __builtin_amdgcn_global_load_lds((GlobalPtr)src, (LdsPtr)dst, 4, 0, 0); }

// a wave-uniform value the compiler is to hold in scalar registers
MOLT_DEV long uniform(long x) {
  const uint32_t lo = __builtin_amdgcn_readfirstlane(int(x)), hi = __builtin_amdgcn_readfirstlane(int(x >> 32));
  return long(uint64_t(hi) << 32 | lo);
}

// x as P bf16 values whose sum is x to 8 P bits
template <int P>
MOLT_DEV void split_bf16(float x, __bf16 (&part)[P]) {
#pragma unroll
  for (int i = 0; i < P; ++i) {
    part[i] = __bf16(x);
    x -= float(part[i]);                 // exact
  }
}

// Query row as B operands of 16x16x32 bf16 MFMAs: three bf16 parts (24 bits) of dims D / 4 * g4 + 8 s .. +7
// for k-step s, the order in which a lane's K codes lie.
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
      __bf16 part[3];
      split_bf16<3>(x[e / 4][e % 4], part);
#pragma unroll
      for (int u = 0; u < 3; ++u) qf[u][s][e] = part[u];
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
MOLT_DEV void load_query_bf16(const uint16_t* q, bool valid, int g4, int32x8_t (&qp)[D / 64], int& qs) {
  float x[D / 64][16];
  uint32_t amax = 0;
#pragma unroll
  for (int c = 0; c < D / 64; ++c)
#pragma unroll
    for (int v = 0; v < 2; ++v) {
      u32x4 w = {0u, 0u, 0u, 0u};
      if (valid) w = *reinterpret_cast<const UnalignedU4*>(q + 64 * c + 16 * g4 + 8 * v);
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

// Output dims d0 .. + 7 of row r: a / L, zeros for a row that sees no key
template <typename T>
MOLT_DEV void store_out(const KvqAttnParams& p, int b, int h, int r, int D, int d0, const floatx4_t (&a)[2], float L) {
  const float inv = L == 0.f ? 0.f : 1.f / L;
  const long t = long(b) * p.n + r / p.G, c = (h * p.G + r % p.G) * D + d0, cols = long(p.Hq) * D;
  T* out = static_cast<T*>(p.out);
  if constexpr (sizeof(T) == 4) {
#pragma unroll
    for (int i = 0; i < 2; ++i)
      *reinterpret_cast<UnalignedF4*>(out + (p.out_tiled ? tiled_index(t, c + 4 * i, cols, 4) : t * cols + c + 4 * i)) = a[i] * inv;
  } else {
    *reinterpret_cast<UnalignedU4*>(out + (p.out_tiled ? tiled_index(t, c, cols, 2) : t * cols + c)) =
        u32x4{f32x2_to_bf16(a[0][0] * inv, a[0][1] * inv), f32x2_to_bf16(a[0][2] * inv, a[0][3] * inv),
              f32x2_to_bf16(a[1][0] * inv, a[1][1] * inv), f32x2_to_bf16(a[1][2] * inv, a[1][3] * inv)};
  }
}

template <int D, typename T, int NT>
__global__ __launch_bounds__(kWaves * kWave, 2) void kvq_attn_kernel(KvqAttnParams p) {
  typedef KvqRecord<D> Rec;
  constexpr bool F32 = sizeof(T) == 4;
  constexpr int QP = 3;                  // bf16 parts of an f32 query element
  constexpr int PP = F32 ? 3 : 1;        // bf16 parts of a probability (see the top)
  constexpr int KS = D / 32;             // MFMA steps over the dims of a score
  constexpr int DT = D / 16;             // 16-dim tiles of O^T
  constexpr int SLOT = 32 * D + 256;     // bytes of a pair in the ring
  constexpr int kCopies = D == 128 ? 5 : 3;   // vector memory instructions of a pair
  // the wavefronts' rings, then (kJoin floats each) their results; the query operands; the only LDS object
  constexpr int kJoin = 16 * (D + 4) + 32;
  constexpr int kLds = kSlots * SLOT > kJoin * 4 ? kSlots * SLOT : kJoin * 4;
  constexpr int QF = D / 64 * 2048;      // bytes of a tile's query operands
  __shared__ __attribute__((aligned(16))) uint8_t lds[kWaves * kLds + (F32 ? 0 : NT * QF)];

  // work item
  const int rg = int(blockIdx.x) % p.nrg;
  const int unit = int(blockIdx.x) / p.nrg;
  const int split = unit % p.splits;
  const int bh = unit / p.splits;
  const int b = bh / p.Hkv, h = bh % p.Hkv;
  const int r0 = rg * 16 * NT, r1 = min(r0 + 16 * NT, p.R);
  const int ctx = p.ctx[b];
  const int end = visible_end(p, ctx, r1);
  const int nblk = (end + 15) / 16, npairs = (nblk + 1) / 2;
  const int ns = (nblk + p.bps - 1) / p.bps;
  if (split >= max(ns, 1)) return;
  const int lane = threadIdx.x % kWave, l16 = lane % 16, g4 = lane / 16;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  // the split's pairs of blocks, then the wavefront's share
  const int s0 = ns > 0 ? int(long(npairs) * split / ns) : 0, s1 = ns > 0 ? int(long(npairs) * (split + 1) / ns) : 0;
  const int p0 = s0 + (s1 - s0) * wave / kWaves, p1 = s0 + (s1 - s0) * (wave + 1) / kWaves;
  const int full_end = min(visible_end(p, ctx, r0 + 1), end);    // keys before are seen by every row
  uint8_t* ring = lds + wave * kLds;
  uint8_t* qlds = lds + kWaves * kLds;

  // Copies of a pair into a slot of the wavefront's ring: [K codes of both blocks][V codes][scales of K, of
  // V], K's 16-byte chunks in the order in which the lanes read them (dims 32 c .. of token t at chunk 16 c + t)
  typedef const __attribute__((address_space(4))) int32_t* ConstInt;
  const ConstInt btab = (ConstInt)(p.bt + long(b) * p.max_blocks);
  constexpr uint32_t SR = D / 32 * 4;    // lanes (dwords) of a record's scales
  const uint32_t ksrc = D == 128 ? l16 * 64 + g4 * 16 : l16 * 32 + g4 % 2 * 16;
  const uint32_t vsrc = D == 128 ? lane * 16 : lane % 32 * 16;
  const uint32_t spart = lane / SR % 4;
  const uint8_t* sbase = (spart < 2 ? p.kc : p.vc) + Rec::kCodes + lane % SR * 4;
  auto issue = [&](int pi, const int (&id)[2]) __attribute__((always_inline)) {
    uint8_t* dst = ring + (pi - p0) % kSlots * SLOT;
    long rec[2];                         // kept in scalar registers: a uniform base and a lane offset per copy
#pragma unroll
    for (int u = 0; u < 2; ++u) rec[u] = uniform((long(unsigned(id[u]) < unsigned(p.num_blocks) ? id[u] : 0) * p.Hkv + h) * Rec::kBytes);
    if constexpr (D == 128) {
#pragma unroll
      for (int u = 0; u < 2; ++u) copy_lds16(p.kc + rec[u] + ksrc, dst + 1024 * u);
#pragma unroll
      for (int u = 0; u < 2; ++u) copy_lds16(p.vc + rec[u] + vsrc, dst + 2048 + 1024 * u);
    } else {
      const long r = lane < 32 ? rec[0] : rec[1];
      copy_lds16(p.kc + r + ksrc, dst);
      copy_lds16(p.vc + r + vsrc, dst + 1024);
    }
    copy_lds4(sbase + (spart % 2 ? rec[1] : rec[0]), dst + 32 * D);
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

  // Q^T operands: in f32 each wavefront's own, in bf16 in LDS for all, tile i made by wavefront i
  int lim[NT];                           // last key that the row sees
  bf16x8_t qf[QP][KS];
  int qs[NT];                            // scale bytes of both fp8 parts
#pragma unroll
  for (int i = 0; i < NT; ++i) {
    const int r = r0 + 16 * i + l16, j = r / p.G, gi = r % p.G;
    lim[i] = r < p.R ? ctx + j : -1;
    const long at = ((long(b) * p.n + j) * p.Hq + h * p.G + gi) * D;
    if constexpr (F32) {
      load_query_f32<D>(static_cast<const float*>(p.q) + at, r < p.R, g4, qf);
    } else if (wave == i) {
      int32x8_t qp[D / 64];
      int sc;
      load_query_bf16<D>(static_cast<const uint16_t*>(p.q) + at, r < p.R, g4, qp, sc);
#pragma unroll
      for (int u = 0; u < D / 64; ++u) {
        int32x4_t* dst = reinterpret_cast<int32x4_t*>(qlds + i * QF + u * 2048 + lane * 16);
        dst[0] = int32x4_t{qp[u][0], qp[u][1], qp[u][2], qp[u][3]};
        dst[64] = int32x4_t{qp[u][4], qp[u][5], qp[u][6], qp[u][7]};
      }
      *reinterpret_cast<int*>(lds + i * kLds + (kSlots - 1) * SLOT + lane * 4) = sc;   // in a slot not yet in use
    }
  }
  if constexpr (!F32) {
    lds_barrier();
#pragma unroll
    for (int i = 0; i < NT; ++i) qs[i] = *reinterpret_cast<const int*>(lds + i * kLds + (kSlots - 1) * SLOT + lane * 4);
    lds_barrier();
  }
  floatx4_t o[NT][DT], ls[NT];           // O^T; the rows' sums (bf16: by MFMA, the same in every register and group)
  float m[NT];                           // reference maximum (of raw scores)
  float ref[NT];                         // m, or 0 for a row that has seen no key: its exp2(-inf) is 0
  float bound[NT];                       // scores above it raise m
  const float slack = kRescaleSlack / p.c;
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
  auto settle = [&](int pi, bool ok0, bool ok1, floatx4_t (&sv)[2][NT], uint32_t (&vs)[2]) __attribute__((always_inline)) {
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
        // lanes of dims in it (l16 * D / 16) hold, their tokens 4 a .. 4 a + 3
        bool poison[NT];
#pragma unroll
        for (int i = 0; i < NT; ++i) poison[i] = false;
#pragma unroll
        for (int a = 0; a < 4; ++a) {
          const uint32_t w = uint32_t(__shfl(int(bad), a * 16 + (g4 * D / 128) * (512 / D)));
#pragma unroll
          for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int e = 0; e < 4; ++e)
#pragma unroll
              for (int i = 0; i < NT; ++i)
                if ((w >> (4 * u + e)) & 1u) poison[i] |= 32 * pi + 16 * u + 4 * a + e <= lim[i];
        }
#pragma unroll
        for (int i = 0; i < NT; ++i)
#pragma unroll
          for (int t = 0; t < DT; ++t) o[i][t] += poison[i] ? __builtin_nanf("") : 0.f;
      }
    }
    float mx[NT];
    bool grow = false;
#pragma unroll
    for (int i = 0; i < NT; ++i) {
      mx[i] = fmaxf(fmaxf(fmaxf(sv[0][i][0], sv[0][i][1]), fmaxf(sv[0][i][2], sv[0][i][3])),
                    fmaxf(fmaxf(sv[1][i][0], sv[1][i][1]), fmaxf(sv[1][i][2], sv[1][i][3])));
      grow |= mx[i] > bound[i];
    }
    if (__ballot(grow)) {
#pragma unroll
      for (int i = 0; i < NT; ++i) {
        const float mn = fmaxf(m[i], rows_max4(mx[i]));
        const float alpha = m[i] == -INFINITY ? 0.f : exp2f((m[i] - mn) * p.c);
        m[i] = mn;
        bound[i] = mn + slack;
        ref[i] = mn == -INFINITY ? 0.f : mn;
        ls[i] *= alpha;
#pragma unroll
        for (int t = 0; t < DT; ++t) o[i][t] *= alpha;
      }
    }
  };

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
    scores(p0, sv, vs);
    settle(p0, have >> (2 * kSlots - 4) & 1u, have >> (2 * kSlots - 4) & 2u, sv, vs);
  }
  for (int pi = p0; pi < p1; ++pi) {
    arrive(pi + 1);
    if (pi + kSlots - 1 < p1) issue(pi + kSlots - 1, nid);
    have = have << 2 | present(nid);
    ids(pi + kSlots, nid);
    // scores of the next pair (past the last: of whatever its slot holds, not used), beside the
    // probabilities and values of this one
    __builtin_amdgcn_s_setprio(1);
    floatx4_t nsv[2][NT];
    uint32_t nvs[2];
    scores(pi + 1, nsv, nvs);
    bf16x8_t pf[NT][PP];
#pragma unroll
    for (int i = 0; i < NT; ++i) {
      float ps = 0.f;
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float w = __builtin_amdgcn_exp2f((sv[u][i][e] - ref[i]) * p.c);
          if constexpr (F32) ps += w;
          __bf16 part[PP];
          split_bf16<PP>(w, part);
#pragma unroll
          for (int q = 0; q < PP; ++q) pf[i][q][4 * u + e] = part[q];
        }
      if constexpr (F32) {
        ls[i][0] += ps;
      } else {
        const uint32_t one = 0x3f803f80u;
        const u32x4 ones = {one, one, one, one};
#pragma unroll
        for (int q = 0; q < PP; ++q)
          ls[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, ones), pf[i][q], ls[i], 0, 0, 0);
      }
    }
    // O^T += V^T P^T: lane (l16, g4) holds dims D / 16 * l16 + t (tile t) of tokens 4 g4 .. +3 of both blocks
    const uint8_t* vsrc_lds = ring + (pi - p0) % kSlots * SLOT + 16 * D + (D == 128 ? lane : g4 * 8 + l16 / 2) * 16;
    uint32_t vd[2][4][DT / 2];           // token's dims as bf16 pairs
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const u32x4 vc = *reinterpret_cast<const u32x4*>(vsrc_lds + 8 * D * u);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const uint32_t sc = kvq_scale_bits(vs[u], e);
        if constexpr (D == 128) {
          vd[u][e][0] = kvq_decode2<0>(vc[e], sc);
          vd[u][e][1] = kvq_decode2<1>(vc[e], sc);
          vd[u][e][2] = kvq_decode2<2>(vc[e], sc);
          vd[u][e][3] = kvq_decode2<3>(vc[e], sc);
        } else {
          const uint32_t w = vc[e] >> (16 * (l16 % 2));
          vd[u][e][0] = kvq_decode2<0>(w, sc);
          vd[u][e][1] = kvq_decode2<1>(w, sc);
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
      const bf16x8_t vf = __builtin_bit_cast(bf16x8_t, w);
#pragma unroll
      for (int i = 0; i < NT; ++i)
#pragma unroll
        for (int q = 0; q < PP; ++q) o[i][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, pf[i][q], o[i][t], 0, 0, 0);
    }
    __builtin_amdgcn_s_setprio(0);
    if (pi + 1 < p1) settle(pi + 1, have >> (2 * kSlots - 4) & 1u, have >> (2 * kSlots - 4) & 2u, nsv, nvs);
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      vs[u] = nvs[u];
#pragma unroll
      for (int i = 0; i < NT; ++i) sv[u][i] = nsv[u][i];
    }
  }
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // no copy may outlive the ring

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
      own[16 * RS + l16] = m[i];
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
    for (int w = 0; w < kWaves; ++w) M = fmaxf(M, part[w * (kLds / 4) + 16 * RS + row]);
    float L = 0.f;
    floatx4_t a[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      const float* pw = part + w * (kLds / 4);
      const float mw = pw[16 * RS + row];
      const float f = mw == -INFINITY ? 0.f : exp2f((mw - M) * p.c);
      L += pw[16 * RS + 16 + row] * f;
      a[0] += *reinterpret_cast<const floatx4_t*>(pw + row * RS + d0) * f;
      a[1] += *reinterpret_cast<const floatx4_t*>(pw + row * RS + d0 + 4) * f;
    }
    if (p.splits == 1) {
      store_out<T>(p, b, h, r, D, d0, a, L);
    } else {
      const long pr = (long(bh) * p.splits + split) * p.R + r;
      *reinterpret_cast<floatx4_t*>(p.part_o + pr * D + d0) = a[0];
      *reinterpret_cast<floatx4_t*>(p.part_o + pr * D + d0 + 4) = a[1];
      if (d0 == 0) {
        p.part_ml[2 * pr] = M;
        p.part_ml[2 * pr + 1] = L;
      }
    }
  }
}

// log-sum-exp join of the splits: thread = 8 dims of one row
template <int D, typename T>
__global__ __launch_bounds__(256) void kvq_merge_kernel(KvqAttnParams p) {
  const long i = long(blockIdx.x) * 256 + threadIdx.x;
  const int d0 = int(i % (D / 8)) * 8;
  const long row = i / (D / 8);
  const int bh = int(row / p.R), r = int(row % p.R);
  const int b = bh / p.Hkv, h = bh % p.Hkv;
  if (b >= p.B) return;
  const int end = visible_end(p, p.ctx[b], min((r / p.group + 1) * p.group, p.R));
  const int ns = max(((end + 15) / 16 + p.bps - 1) / p.bps, 1);
  const long pr0 = long(bh) * p.splits * p.R + r;
  float M = -INFINITY;
  for (int s = 0; s < ns; ++s) M = fmaxf(M, p.part_ml[2 * (pr0 + long(s) * p.R)]);
  float L = 0.f;
  floatx4_t a[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
  for (int s = 0; s < ns; ++s) {
    const long pr = pr0 + long(s) * p.R;
    const float ms = p.part_ml[2 * pr];
    const float f = ms == -INFINITY ? 0.f : exp2f((ms - M) * p.c);
    L += p.part_ml[2 * pr + 1] * f;
    a[0] += *reinterpret_cast<const floatx4_t*>(p.part_o + pr * D + d0) * f;
    a[1] += *reinterpret_cast<const floatx4_t*>(p.part_o + pr * D + d0 + 4) * f;
  }
  store_out<T>(p, b, h, r, D, d0, a, L);
}

constexpr int kMaxTiles = 3;             // 16-row tiles of a wavefront (bf16; one in f32)

// Row groups of as few 16-row tiles as cover the R rows, and the splits of the key range: enough that
// the workgroups fill the chip (512 are resident), at least 8 blocks each.
void kvq_plan(KvqAttnParams& p, bool f32) {
  p.G = p.Hq / p.Hkv;
  p.R = p.G * p.n;
  const int tiles = (p.R + 15) / 16, most = f32 ? 1 : kMaxTiles;
  p.nrg = (tiles + most - 1) / most;
  p.group = 16 * ((tiles + p.nrg - 1) / p.nrg);
  const long units = long(p.B) * p.Hkv * p.nrg;
  long s = units >= 512 ? 1 : (1024 + units - 1) / units;
  const long cap = (p.max_blocks + 7) / 8;
  if (s > cap) s = cap;
  p.bps = int((p.max_blocks + s - 1) / s + 1) / 2 * 2;
  p.splits = (p.max_blocks + p.bps - 1) / p.bps;
}

template <int D, typename T, int NT>
void launch_nt(const KvqAttnParams& p, hipStream_t s) {
  kvq_attn_kernel<D, T, NT><<<unsigned(long(p.B) * p.Hkv * p.splits * p.nrg), kWaves * kWave, 0, s>>>(p);
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
  if (p.splits > 1) {
    const long threads = long(p.B) * p.Hkv * p.R * (D / 8);
    kvq_merge_kernel<D, T><<<unsigned((threads + 255) / 256), 256, 0, s>>>(p);
  }
}

void carve_parts(Carver& c, KvqAttnParams& p, int D) {
  if (p.splits <= 1) return;
  const long rows = long(p.B) * p.Hkv * p.splits * p.R;
  p.part_o = c.take<float>(rows * D);
  p.part_ml = c.take<float>(rows * 2);
}

}  // namespace

// f32 calls have more row groups, so never more splits: one size serves both types
size_t kvq_attention_ws_bytes(int B, int n, int Hq, int Hkv, int D, int max_blocks) {
  KvqAttnParams p{};
  p.B = B; p.n = n; p.Hq = Hq; p.Hkv = Hkv; p.max_blocks = max_blocks;
  kvq_plan(p, false);
  Carver c(nullptr, 0);
  carve_parts(c, p, D);
  return c.used ? c.used + 256 : 0;
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
  kvq_plan(p, dt == MOLT_F32);
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
