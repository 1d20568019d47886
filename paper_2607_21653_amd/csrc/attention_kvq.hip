// Multi-query paged attention over the 4-bit KV cache (format: kvq_format.h).
//   o_r = sum_p w_rp v_p,  w_r = softmax over p <= ctx_b + j(r) of q_r . k_p / sqrt(D)
// for the R = G * n rows (position j = r / G, query head h G + r % G) of sequence b and kv head h.
#include "internal.h"
#include "kvq_format.h"

namespace molt {
namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kRescaleSlack = 8.0f;   // probabilities may grow to 2^8 before O is rescaled
constexpr int kWaves = 4;

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
  constexpr int PP = F32 ? 3 : 2;        // bf16 parts of a probability
  constexpr int KS = D / 32;             // MFMA steps over the dims of a score
  constexpr int DT = D / 16;             // 16-dim tiles of O^T
  __shared__ __attribute__((aligned(16))) float s_o[kWaves][16][D + 4];
  __shared__ float s_m[kWaves][16], s_l[kWaves][16];

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

  // Q^T operands
  int lim[NT];                           // last key that the row sees
  bf16x8_t qf[F32 ? NT : 1][QP][KS];     // f32
  int32x8_t qp[F32 ? 1 : NT][D / 64];    // bf16
  int qs[F32 ? 1 : NT];                  // scale bytes of both fp8 parts
#pragma unroll
  for (int i = 0; i < NT; ++i) {
    const int r = r0 + 16 * i + l16, j = r / p.G, gi = r % p.G;
    lim[i] = r < p.R ? ctx + j : -1;
    const long at = ((long(b) * p.n + j) * p.Hq + h * p.G + gi) * D;
    if constexpr (F32) load_query_f32<D>(static_cast<const float*>(p.q) + at, r < p.R, g4, qf[i]);
    else load_query_bf16<D>(static_cast<const uint16_t*>(p.q) + at, r < p.R, g4, qp[i], qs[i]);
  }
  floatx4_t o[NT][DT];
  float m[NT], l[NT];
#pragma unroll
  for (int i = 0; i < NT; ++i) {
    m[i] = -INFINITY;
    l[i] = 0.f;
#pragma unroll
    for (int t = 0; t < DT; ++t) o[i][t] = floatx4_t{0.f, 0.f, 0.f, 0.f};
  }
  const int full_end = min(visible_end(p, ctx, r0 + 1), end);    // keys before are seen by every row

  typedef const __attribute__((address_space(4))) int32_t* ConstInt;
  const ConstInt btab = (ConstInt)(p.bt + long(b) * p.max_blocks);
  // Lane (l16, g4): codes of K's token l16, dims 32 g4 .. (D = 64: 32 (g4 % 2) .., in f32 16 g4 ..) and their
  // scale byte; V's tokens 4 g4 .. +3 of the octet that has dims D / 16 * l16 .., and their scale bytes
  struct Block { u32x4 k; u32x4 v; uint32_t ks, vs; };
  auto load = [&](Block& x, int id) __attribute__((always_inline)) {
    const long rec = (long(unsigned(id) < unsigned(p.num_blocks) ? id : 0) * p.Hkv + h) * Rec::kBytes;
    const uint8_t *kr = p.kc + rec, *vr = p.vc + rec;
    if constexpr (D == 128) {
      x.k = *reinterpret_cast<const u32x4*>(kr + l16 * 64 + g4 * 16);
      x.v = *reinterpret_cast<const u32x4*>(vr + lane * 16);
      x.ks = kr[Rec::k_scale(l16, g4)];
    } else {
      if constexpr (F32) {
        const u32x2 w = *reinterpret_cast<const u32x2*>(kr + l16 * 32 + g4 * 8);
        x.k[0] = w[0];
        x.k[1] = w[1];
        x.ks = kr[Rec::k_scale(l16, g4 / 2)];
      } else {
        x.k = *reinterpret_cast<const u32x4*>(kr + l16 * 32 + g4 % 2 * 16);
        x.ks = kr[Rec::k_scale(l16, g4 % 2)];
      }
      x.v = *reinterpret_cast<const u32x4*>(vr + (g4 * 8 + l16 / 2) * 16);
    }
    x.vs = *reinterpret_cast<const uint32_t*>(vr + Rec::v_scale(4 * g4, l16 * (D / 16) / 32));
  };

  for (int pi = p0; pi < p1; ++pi) {
    const bool two = 2 * pi + 1 < nblk;
    const int id[2] = {btab[2 * pi], two ? btab[2 * pi + 1] : -1};
    Block x[2];
    load(x[0], id[0]);
    load(x[1], id[1]);
    // S^T: lane (row l16 of the tile) holds tokens 4 g4 + e of both blocks
    floatx4_t sv[2][NT];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
#pragma unroll
      for (int i = 0; i < NT; ++i) sv[u][i] = floatx4_t{0.f, 0.f, 0.f, 0.f};
      if constexpr (F32) {
#pragma unroll
        for (int s = 0; s < KS; ++s) {
          const uint32_t sc = x[u].ks << 23;
          const u32x4 w = {kvq_decode2<0>(x[u].k[s], sc), kvq_decode2<1>(x[u].k[s], sc),
                           kvq_decode2<2>(x[u].k[s], sc), kvq_decode2<3>(x[u].k[s], sc)};
          const bf16x8_t kf = __builtin_bit_cast(bf16x8_t, w);
#pragma unroll
          for (int i = 0; i < NT; ++i)
#pragma unroll
            for (int q = 0; q < QP; ++q)
              sv[u][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, qf[i][q][s], sv[u][i], 0, 0, 0);
        }
      } else {
        const int32x8_t kf = {int(x[u].k[0]), int(x[u].k[1]), int(x[u].k[2]), int(x[u].k[3]), 0, 0, 0, 0};
#pragma unroll
        for (int i = 0; i < NT; ++i) {   // formats: A 4 (e2m1), B 0 (e4m3)
          sv[u][i] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(kf, qp[i][0], sv[u][i], 4, 0, 0, int(x[u].ks), 0, qs[i]);
          if constexpr (D == 128)
            sv[u][i] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(kf, qp[i][1], sv[u][i], 4, 0, 0, int(x[u].ks), 1, qs[i]);
        }
      }
    }
    bool poison[NT];
#pragma unroll
    for (int i = 0; i < NT; ++i) poison[i] = false;
    const bool ok0 = unsigned(id[0]) < unsigned(p.num_blocks), ok1 = unsigned(id[1]) < unsigned(p.num_blocks);
    if (32 * pi + 32 > full_end || !ok0 || !ok1) {
      // Keys that some row may not see: their scores are -inf for it, and their values must not reach it.
      // A probability of 0 does that, unless the value is NaN (scale byte 255, also in slots that were
      // never written): such groups are taken as codes times 1, and the rows that do see one get their
      // NaN in the group's dims afterwards.
      uint32_t bad = 0;
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int pos = 32 * pi + 16 * u + 4 * g4 + e;
          const bool seen = pos < end && (u == 0 ? ok0 : ok1);
#pragma unroll
          for (int i = 0; i < NT; ++i)
            if (!(seen && pos <= lim[i])) sv[u][i][e] = -INFINITY;
          const uint32_t byte = (x[u].vs >> (8 * e)) & 255u;
          if (!seen || byte == kKvqScaleNan) x[u].vs = (x[u].vs & ~(255u << (8 * e))) | (127u << (8 * e));
          if (seen && byte == kKvqScaleNan) bad |= 1u << (4 * u + e);
        }
      if (__ballot(bad != 0)) {
        // output lane (row l16, g4) holds dims D / 4 * g4 .. of its row: group g4 * D / 128, whose scales
        // lanes of dims in it (l16 * D / 16) hold, their tokens 4 a .. 4 a + 3
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
      }
    }
    // running maximum, O rescaled only when a row's grows by more than the slack
    float mx[NT];
    bool grow = false;
#pragma unroll
    for (int i = 0; i < NT; ++i) {
      const float v = fmaxf(fmaxf(fmaxf(sv[0][i][0], sv[0][i][1]), fmaxf(sv[0][i][2], sv[0][i][3])),
                            fmaxf(fmaxf(sv[1][i][0], sv[1][i][1]), fmaxf(sv[1][i][2], sv[1][i][3])));
      mx[i] = v;
      grow |= (v - m[i]) * p.c > kRescaleSlack || (v > m[i] && m[i] == -INFINITY);
    }
    if (__ballot(grow)) {
#pragma unroll
      for (int i = 0; i < NT; ++i) {
        const float mn = fmaxf(m[i], rows_max4(mx[i]));
        const float alpha = m[i] == -INFINITY ? 0.f : exp2f((m[i] - mn) * p.c);
        m[i] = mn;
        l[i] *= alpha;
#pragma unroll
        for (int t = 0; t < DT; ++t) o[i][t] *= alpha;
      }
    }
    bf16x8_t pf[NT][PP];
#pragma unroll
    for (int i = 0; i < NT; ++i) {
      const float ref = m[i] == -INFINITY ? 0.f : m[i];      // a row that has seen no key: exp2(-inf)
      float ps = 0.f;
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float w = __builtin_amdgcn_exp2f((sv[u][i][e] - ref) * p.c);
          ps += w;
          __bf16 part[PP];
          split_bf16<PP>(w, part);
#pragma unroll
          for (int q = 0; q < PP; ++q) pf[i][q][4 * u + e] = part[q];
        }
      l[i] += ps;
    }
    // O^T += V^T P^T: lane (l16, g4) holds dims D / 16 * l16 + t (tile t) of tokens 4 g4 .. +3 of both blocks
    uint32_t vd[2][4][DT / 2];           // token's dims as bf16 pairs
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const uint32_t sc = kvq_scale_bits(x[u].vs, e);
        if constexpr (D == 128) {
          vd[u][e][0] = kvq_decode2<0>(x[u].v[e], sc);
          vd[u][e][1] = kvq_decode2<1>(x[u].v[e], sc);
          vd[u][e][2] = kvq_decode2<2>(x[u].v[e], sc);
          vd[u][e][3] = kvq_decode2<3>(x[u].v[e], sc);
        } else {
          const uint32_t w = x[u].v[e] >> (16 * (l16 % 2));
          vd[u][e][0] = kvq_decode2<0>(w, sc);
          vd[u][e][1] = kvq_decode2<1>(w, sc);
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
#pragma unroll
    for (int i = 0; i < NT; ++i)
      if (poison[i])
#pragma unroll
        for (int t = 0; t < DT; ++t) o[i][t] += __builtin_nanf("");
  }

  // the wavefronts' shares joined through LDS, one 16-row tile at a time
#pragma unroll
  for (int i = 0; i < NT; ++i) {
    const float lt = rows_sum4(l[i]);
    if (i > 0) __syncthreads();
#pragma unroll
    for (int e = 0; e < 4; ++e)
#pragma unroll
      for (int t = 0; t < DT; t += 4)   // dims D / 16 * (4 g4 + e) + t .. + 3
        *reinterpret_cast<floatx4_t*>(&s_o[wave][l16][D / 16 * (4 * g4 + e) + t]) =
            floatx4_t{o[i][t][e], o[i][t + 1][e], o[i][t + 2][e], o[i][t + 3][e]};
    if (g4 == 0) {
      s_m[wave][l16] = m[i];
      s_l[wave][l16] = lt;
    }
    __syncthreads();
    // thread = 8 dims of one row
    if (threadIdx.x >= 16 * (D / 8)) continue;
    const int row = threadIdx.x / (D / 8), d0 = threadIdx.x % (D / 8) * 8;
    const int r = r0 + 16 * i + row;
    if (r >= p.R) continue;
    float M = s_m[0][row];
#pragma unroll
    for (int w = 1; w < kWaves; ++w) M = fmaxf(M, s_m[w][row]);
    float L = 0.f;
    floatx4_t a[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      const float f = s_m[w][row] == -INFINITY ? 0.f : exp2f((s_m[w][row] - M) * p.c);
      L += s_l[w][row] * f;
      a[0] += *reinterpret_cast<const floatx4_t*>(&s_o[w][row][d0]) * f;
      a[1] += *reinterpret_cast<const floatx4_t*>(&s_o[w][row][d0 + 4]) * f;
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
