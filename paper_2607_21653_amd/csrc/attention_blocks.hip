// Attention over listed blocks of the paged cache.
//   o_r = sum_p w_rp v_p,  w_r = softmax over the keys p <= ctx_b + j of the blocks that list (t, h) names
// for the G query rows r of position j of sequence b (t = b n + j) and kv head h, scores q . k / sqrt(D).
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "device_common.h"
#include "internal.h"

namespace molt {
namespace {

constexpr float kLog2e = 1.4426950408889634f;

struct BlocksArgs {
  const void* q; const void* kc; const void* vc; const int32_t* bt; const int32_t* ctx; const int32_t* blocks;
  void* out;
  float* part_o;                                 // [units, splits, 16, D] partial outputs of split lists
  float* part_ml;                                // [units, splits, 16, 2] their maxima and sums
  int B, n, Hq, Hkv, G, N, max_blocks, num_blocks;
  int row_groups, splits, per_split;             // groups of 16 query rows of a kv head; parts of a list, units of one
  int by_xcd;
  float c;                                       // log2(e) / sqrt(D)
};

typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));

// Entry e of a list, e in [e0, e0 + 64): lane e - e0 holds its block's place in the cache (-1: none) and how many of
// its 16 tokens the position sees.
struct Entries { int id, seen; };
MOLT_DEV Entries entries_of(const BlocksArgs& p, const int32_t* list, int e, bool there, int b, long pos) {
  Entries r{-1, 0};
  if (!there) return r;
  const int blk = list[e];
  if (blk < 0 || blk >= p.max_blocks || 16l * blk > pos) return r;
  const int id = p.bt[long(b) * p.max_blocks + blk];
  if (id < 0 || id >= p.num_blocks) return r;
  r.id = id;
  r.seen = int(min(16l, pos - 16l * blk + 1));
  return r;
}

// Running softmax of a lane's query row (lane % 16): maximum of the scores q . k, this lane's share of the sum, and O^T:
// dims 16 d + 4 (lane / 16) + i. A weight is exp2((s - m) c), of a difference of scores, so that the largest is 1 whatever
// the scores' size: s c less a rounded m c would be off by half a step of m c, 2^7 where that is past 2^31. (No slower:
// 16 sequences x 5 positions, 128 of 3000 blocks 39.5 us both ways, 2 x 257, 64 of 512 blocks 57.7 and 57.6.)
template <int D>
struct Running {
  float m = -__builtin_inff(), l = 0.f;
  floatx4_t o[D / 16];
};

// 2^((s - m) c), 0 for s = -inf and any m but that
MOLT_DEV float weight(float s, float m, float c) { return __builtin_amdgcn_exp2f((s - m) * c); }

// Scores s of a lane's M keys of one row (-inf: not seen) -> weights, with O and the sum rescaled
template <int D, int M>
MOLT_DEV void weigh(Running<D>& r, float (&s)[M], float c) {
  float top = s[0];
#pragma unroll
  for (int i = 1; i < M; ++i) top = fmaxf(top, s[i]);
  top = rows_max4(top);
  if (__any(top > r.m)) {
    const float m = fmaxf(r.m, top), f = r.m == m ? 1.f : weight(r.m, m, c);
    r.m = m;
    r.l *= f;
#pragma unroll
    for (int d = 0; d < D / 16; ++d) r.o[d] *= f;
  }
  const float base = r.m == -__builtin_inff() ? 0.f : r.m;
#pragma unroll
  for (int i = 0; i < M; ++i) {
    s[i] = weight(s[i], base, c);
    r.l += s[i];
  }
}

// A block's keys or values of one kv head on their way to LDS: 16 bytes a lane, in the cache's order, so that lanes side
// by side ask for bytes side by side. (As the MFMAs take them, 16 bytes of 16 tokens or dims by 16 lanes, each lane's are
// a request of its own: the loads are then bound by requests, at 20 bytes a cycle and CU.)
template <int D, typename T>
struct Raw {
  static constexpr int kBytes = 16 * D * int(sizeof(T)), kLoads = kBytes / 1024;
  u32x4_t w[kLoads];
  template <bool ONCE>                           // nontemporal, where one workgroup reads the block
  MOLT_DEV void load(const void* cache, long block_head, int lane) {
    const u32x4_t* from = reinterpret_cast<const u32x4_t*>(static_cast<const uint8_t*>(cache) + block_head * kBytes) + lane;
#pragma unroll
    for (int c = 0; c < kLoads; ++c) w[c] = ONCE ? __builtin_nontemporal_load(from + c * 64) : from[c * 64];
  }
};

// bf16: two blocks at a time. Scores S^T = K Q^T by 16x16x32 MFMAs whose A rows are tokens in such an order that a
// lane's 8 scores of the two tiles are those of 8 consecutive tokens of one block: rows 4 g + i of tile x are tokens
// 8 (g % 2) + 4 x + i of block g / 2. They are then the B operand of O^T = V^T P^T as they lie, and V's A operand is
// 16 contiguous bytes. Weights go in as two bf16 parts, 16 bits. In LDS a token's 16-byte chunks of K lie at chunk ^ f
// and a dim's two of V at half ^ f, with f of the token or dim, so that reads are free of bank conflicts.
template <int D>
struct PairBf16 {
  static constexpr int kBlocks = 2;
  static constexpr int kLds = 2 * Raw<D, uint16_t>::kBytes;              // the keys, then the values
  static constexpr int KC = D / 8;               // chunks of a token
  struct Query { bf16x8_t q[D / 32]; };
  MOLT_DEV static void load_q(Query& r, const void* qq, long row, bool there, int g) {
#pragma unroll
    for (int s = 0; s < D / 32; ++s) {
      u32x4_t w{0, 0, 0, 0};
      if (there) w = *reinterpret_cast<const u32x4_t*>(static_cast<const uint16_t*>(qq) + row * D + 32 * s + 8 * g);
      r.q[s] = __builtin_bit_cast(bf16x8_t, w);
    }
  }
  MOLT_DEV static int key_at(int block, int token, int chunk) {
    const int f = (token & 3) | (token >> 3 & 1) << 2;                    // (8 lanes read tokens 0 .. 3, 8 .. 11 or 4 more)
    return (block * 16 + token) * KC * 16 + (chunk ^ f) * 16;
  }
  MOLT_DEV static int value_at(int block, int dim, int half) {
    return (block * D + dim) * 32 + (half ^ (dim >> 2 & 1)) * 16;
  }
  Raw<D, uint16_t> k[2], v[2];
  template <bool ONCE>
  MOLT_DEV void load_keys(const BlocksArgs& p, const int (&id)[2], int h, int lane) {
#pragma unroll
    for (int y = 0; y < 2; ++y) k[y].template load<ONCE>(p.kc, long(id[y]) * p.Hkv + h, lane);
  }
  template <bool ONCE>
  MOLT_DEV void load_values(const BlocksArgs& p, const int (&id)[2], int h, int lane) {
#pragma unroll
    for (int y = 0; y < 2; ++y) v[y].template load<ONCE>(p.vc, long(id[y]) * p.Hkv + h, lane);
  }
  MOLT_DEV void store_keys(uint8_t* lds, int lane) const {
#pragma unroll
    for (int y = 0; y < 2; ++y)
#pragma unroll
      for (int c = 0; c < Raw<D, uint16_t>::kLoads; ++c) {
        const int at = c * 64 + lane;
        *reinterpret_cast<u32x4_t*>(lds + key_at(y, at / KC, at % KC)) = k[y].w[c];
      }
  }
  MOLT_DEV void store_values(uint8_t* lds, int lane) const {
#pragma unroll
    for (int y = 0; y < 2; ++y)
#pragma unroll
      for (int c = 0; c < Raw<D, uint16_t>::kLoads; ++c) {
        const int at = c * 64 + lane;
        *reinterpret_cast<u32x4_t*>(lds + value_at(y, at / 2, at % 2)) = v[y].w[c];
      }
  }
  typedef float Scores[8];
  MOLT_DEV static void scores(const uint8_t* lds, const Query& q, Scores& w, int g, int col) {
    floatx4_t s[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
#pragma unroll
    for (int x = 0; x < 2; ++x)
#pragma unroll
      for (int i = 0; i < D / 32; ++i) {
        const bf16x8_t k = *reinterpret_cast<const bf16x8_t*>(lds + key_at(col / 8, col / 4 % 2 * 8 + 4 * x + col % 4, 4 * i + g));
        s[x] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k, q.q[i], s[x], 0, 0, 0);
      }
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i] = s[i / 4][i % 4];
  }
  // seen: tokens of the blocks that the row sees
  MOLT_DEV static void use(const uint8_t* lds, Scores& w, const int (&seen)[2], Running<D>& r, int g, int col, float c) {
    const bool cut = seen[0] < 16 || seen[1] < 16;                       // wavefront-uniform
    const int mine = (g / 2 ? seen[1] : seen[0]) - g % 2 * 8;            // of the lane's 8 tokens
    if (cut) {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (i >= mine) w[i] = -__builtin_inff();
    }
    weigh<D, 8>(r, w, c);
    bf16x8_t hi, lo;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      hi[i] = __bf16(w[i]);
      lo[i] = __bf16(w[i] - float(hi[i]));
    }
#pragma unroll
    for (int d = 0; d < D / 16; ++d) {
      u32x4_t v = *reinterpret_cast<const u32x4_t*>(lds + value_at(g / 2, 16 * d + col, g % 2));
      if (cut) {                                 // what is not seen may be anything: 0 times it would be NaN
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = 2 * i >= mine ? 0 : 2 * i + 1 >= mine ? v[i] & 0xffffu : v[i];
      }
      const bf16x8_t a = __builtin_bit_cast(bf16x8_t, v);
      r.o[d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, hi, r.o[d], 0, 0, 0);
      r.o[d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, lo, r.o[d], 0, 0, 0);
    }
  }
};

// f32: one block at a time on 16x16x4 f32 MFMAs; step s of the scores takes dims D / 4 g + s, so that a lane's share of
// a token is contiguous; step i of O^T takes tokens 4 g + i, those of the lane's i-th score.
template <int D>
struct BlockF32 {
  static constexpr int kBlocks = 1;
  static constexpr int kLds = Raw<D, float>::kBytes;
  static constexpr int KC = D / 4;
  struct Query { floatx4_t q[D / 16]; };
  MOLT_DEV static void load_q(Query& r, const void* qq, long row, bool there, int g) {
#pragma unroll
    for (int s = 0; s < D / 16; ++s) {
      r.q[s] = floatx4_t{0.f, 0.f, 0.f, 0.f};
      if (there) r.q[s] = *reinterpret_cast<const floatx4_t*>(static_cast<const float*>(qq) + row * D + D / 4 * g + 4 * s);
    }
  }
  MOLT_DEV static int key_at(int token, int chunk) { return token * KC * 16 + (chunk ^ (token & 7)) * 16; }
  MOLT_DEV static int value_at(int dim, int chunk) { return dim * 64 + (chunk ^ (dim >> 1 & 3)) * 16; }
  Raw<D, float> k, v;
  template <bool ONCE>
  MOLT_DEV void load_keys(const BlocksArgs& p, const int (&id)[1], int h, int lane) {
    k.template load<ONCE>(p.kc, long(id[0]) * p.Hkv + h, lane);
  }
  template <bool ONCE>
  MOLT_DEV void load_values(const BlocksArgs& p, const int (&id)[1], int h, int lane) {
    v.template load<ONCE>(p.vc, long(id[0]) * p.Hkv + h, lane);
  }
  MOLT_DEV void store_keys(uint8_t* lds, int lane) const {
#pragma unroll
    for (int c = 0; c < Raw<D, float>::kLoads; ++c) {
      const int at = c * 64 + lane;
      *reinterpret_cast<u32x4_t*>(lds + key_at(at / KC, at % KC)) = k.w[c];
    }
  }
  MOLT_DEV void store_values(uint8_t* lds, int lane) const {
#pragma unroll
    for (int c = 0; c < Raw<D, float>::kLoads; ++c) {
      const int at = c * 64 + lane;
      *reinterpret_cast<u32x4_t*>(lds + value_at(at / 4, at % 4)) = v.w[c];
    }
  }
  typedef float Scores[4];
  MOLT_DEV static void scores(const uint8_t* lds, const Query& q, Scores& w, int g, int col) {
    floatx4_t s{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < D / 16; ++i) {
      const floatx4_t k = *reinterpret_cast<const floatx4_t*>(lds + key_at(col, D / 16 * g + i));
#pragma unroll
      for (int e = 0; e < 4; ++e) s = __builtin_amdgcn_mfma_f32_16x16x4f32(k[e], q.q[i][e], s, 0, 0, 0);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = s[i];
  }
  MOLT_DEV static void use(const uint8_t* lds, Scores& w, const int (&seen)[1], Running<D>& r, int g, int col, float c) {
    const int mine = seen[0] - 4 * g;
    if (seen[0] < 16) {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (i >= mine) w[i] = -__builtin_inff();
    }
    weigh<D, 4>(r, w, c);
#pragma unroll
    for (int d = 0; d < D / 16; ++d) {
      floatx4_t v = *reinterpret_cast<const floatx4_t*>(lds + value_at(16 * d + col, g));
      if (seen[0] < 16) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (i >= mine) v[i] = 0.f;
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) r.o[d] = __builtin_amdgcn_mfma_f32_16x16x4f32(v[i], w[i], r.o[d], 0, 0, 0);
    }
  }
};

MOLT_DEV void store4(uint16_t* p, floatx4_t x) {
  *reinterpret_cast<uint2*>(p) = make_uint2(f32x2_to_bf16(x[0], x[1]), f32x2_to_bf16(x[2], x[3]));
}
MOLT_DEV void store4(float* p, floatx4_t x) { *reinterpret_cast<floatx4_t*>(p) = x; }

// Workgroup = one list (or a part of it) and 16 query rows; wavefronts take its units (pairs of blocks, or blocks) in
// turn, a unit ahead in registers, with running softmaxes of their own, and join them in LDS.
// What bounds it goes by how much the lists share. 128 sequences x 1 position, 64 blocks of 4 kv heads x 128 (268 MB, none
// shared): 47 us, memory at 5.8 TB/s. 16 x 5 at 32768-65536, lists of 128 blocks that selections of similar rows share, 1.46
// lists' blocks in all: 38 us, 335 MB through the L2 caches of which 176 come from memory
// (4.6 TB/s). 2 x 257, 64 blocks: 58 us, 1.08 GB from L2 at 18 TB/s, its compute (VALU 35%, MFMA 16%, LDS 39% of the time
// busy) partly beside it. Positions in pairs over the union of their lists, 1.4 times a list's length, took 55 us there, but
// 7.5 in place of 5.2 for 4 x 3 positions and 130 or more in place of 122 for 128 x 5 whose lists share less.
template <int D, typename T, int W, bool ONCE>
__global__ __launch_bounds__(W* kWave, W == 8 || sizeof(T) == 4 ? 2 : 3) void blocks_attention_kernel(BlocksArgs p) {
  typedef std::conditional_t<sizeof(T) == 2, PairBf16<D>, BlockF32<D>> Unit;
  constexpr int KB = Unit::kBlocks, PER = kWave / KB;                    // blocks of a unit; units that lanes hold
  constexpr int kAcc = D / 16 * kWave * 16;                              // a wavefront's O for the join
  __shared__ __attribute__((aligned(16))) uint8_t lds[W][Unit::kLds > kAcc ? Unit::kLds : kAcc];
  __shared__ float ml[W][2][16];
  const int lane = threadIdx.x % kWave, g = lane / 16, col = lane % 16;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  // by XCD: a part of all lists of a sequence and kv head on one of them, since neighbouring positions list much the same
  // blocks. They read them at about the same time: lists begun at different places found less in the L2 cache (16
  // sequences x 5 positions, 128 of 1000 blocks: 43 us in place of 31)
  uint32_t item = blockIdx.x, group;
  const uint32_t inner = uint32_t(p.n) * p.row_groups;
  if (p.by_xcd) {
    group = item / 8 / inner * 8 + item % 8;
    item = item / 8 % inner;
    if (group >= uint32_t(p.B) * p.Hkv * p.splits) return;
  } else {
    group = item / inner;
    item %= inner;
  }
  const uint32_t bh = group / p.splits;
  const int split = int(group % p.splits), rg = int(item % p.row_groups);
  const int j = int(item / p.row_groups), h = int(bh % p.Hkv), b = int(bh / p.Hkv), t = b * p.n + j;
  const long pos = long(p.ctx[b]) + j;
  const int32_t* list = p.blocks + (long(t) * p.Hkv + h) * p.N;
  const int head = h * p.G + rg * 16 + col;
  const bool there = rg * 16 + col < p.G;

  typename Unit::Query q;
  Unit::load_q(q, p.q, long(t) * p.Hq + head, there, g);
  Running<D> r;
#pragma unroll
  for (int d = 0; d < D / 16; ++d) r.o[d] = floatx4_t{0.f, 0.f, 0.f, 0.f};
  const int units = (p.N + KB - 1) / KB, u0 = split * p.per_split, u1 = min(units, u0 + p.per_split);
  for (int base = u0; base < u1; base += W * PER) {
    const int mine = base + wave + lane / KB * W, e = mine * KB + lane % KB;
    const Entries en = entries_of(p, list, e, mine < u1 && e < p.N, b, pos);
    unsigned long long left = __ballot(en.seen > 0);                     // units with a key, by the lane of their first
    if (KB == 2) left = (left | left >> 1) & 0x5555555555555555ull;      // block
    if (!left) continue;
    Unit u;
    int id[KB], seen[KB];
    auto next = [&]() __attribute__((always_inline)) {
      const int i = __builtin_ctzll(left);
      left &= left - 1;
      int some = 0;
#pragma unroll
      for (int y = 0; y < KB; ++y) {
        id[y] = __builtin_amdgcn_readlane(en.id, i + y);
        seen[y] = __builtin_amdgcn_readlane(en.seen, i + y);
        if (id[y] >= 0) some = id[y];
      }
#pragma unroll
      for (int y = 0; y < KB; ++y)
        if (id[y] < 0) id[y] = some;             // the other block's, unseen
    };
    next();
    u.template load_keys<ONCE>(p, id, h, lane);
    u.template load_values<ONCE>(p, id, h, lane);
    for (;;) {
      int now[KB];
#pragma unroll
      for (int y = 0; y < KB; ++y) now[y] = seen[y];
      const bool more = left != 0;
      typename Unit::Scores w;
      u.store_keys(lds[wave], lane);
      if (more) {
        next();
        u.template load_keys<ONCE>(p, id, h, lane);
      }
      Unit::scores(lds[wave], q, w, g, col);
      u.store_values(lds[wave], lane);
      if (more) u.template load_values<ONCE>(p, id, h, lane);
      Unit::use(lds[wave], w, now, r, g, col, p.c);
      if (!more) break;
    }
  }

  r.l = rows_sum4(r.l);
  if (g == 0) { ml[wave][0][col] = r.m; ml[wave][1][col] = r.l; }
  __syncthreads();
  float m = ml[0][0][col];
#pragma unroll
  for (int w = 1; w < W; ++w) m = fmaxf(m, ml[w][0][col]);
  const float base = m == -__builtin_inff() ? 0.f : m, f = weight(r.m, base, p.c);
  float l = 0.f;
#pragma unroll
  for (int w = 0; w < W; ++w) l += weight(ml[w][0][col], base, p.c) * ml[w][1][col];
#pragma unroll
  for (int d = 0; d < D / 16; ++d) reinterpret_cast<floatx4_t*>(lds[wave])[d * kWave + lane] = r.o[d] * f;
  __syncthreads();
  r.m = m;
  r.l = l;
  // wavefront w stores dims 16 d .. + 15 for d = w, w + W, ..
#pragma unroll
  for (int d0 = 0; d0 < D / 16; d0 += W) {
    const int d = d0 + wave;
    if (d >= D / 16) break;
    floatx4_t o = reinterpret_cast<const floatx4_t*>(lds[0])[d * kWave + lane];
#pragma unroll
    for (int w = 1; w < W; ++w) o += reinterpret_cast<const floatx4_t*>(lds[w])[d * kWave + lane];
    if (p.splits > 1) {
      const long at = (((long(t) * p.Hkv + h) * p.row_groups + rg) * p.splits + split) * 16 + col;
      if (there) *reinterpret_cast<floatx4_t*>(p.part_o + at * D + 16 * d + 4 * g) = o;
      if (there && d == 0 && g == 0) { p.part_ml[at * 2] = r.m; p.part_ml[at * 2 + 1] = r.l; }
    } else if (there) {
      // l is 0 only where no key has weight; NaN scores leave NaN
      const float inv = r.l == 0.f ? 0.f : 1.f / r.l;
      store4(static_cast<T*>(p.out) + (long(t) * p.Hq + head) * D + 16 * d + 4 * g, o * inv);
    }
  }
}

// Joins the parts of split lists: thread = 4 dims of a query row (16 x 5 positions, 32 heads x 128, two parts: 4.8 us)
template <int D, typename T>
__global__ __launch_bounds__(256) void blocks_join_kernel(BlocksArgs p) {
  const long at = (long(blockIdx.x) * 256 + threadIdx.x) / (D / 4);
  const int d = threadIdx.x % (D / 4) * 4;
  if (at >= long(p.B) * p.n * p.Hq) return;
  const long th = at / p.G;                      // list
  const int row = int(at % p.G);
  const long first = ((th * p.row_groups + row / 16) * p.splits) * 16 + row % 16;
  float m = -__builtin_inff();
  for (int s = 0; s < p.splits; ++s) m = fmaxf(m, p.part_ml[(first + 16 * s) * 2]);
  const float base = m == -__builtin_inff() ? 0.f : m;
  float l = 0.f;
  floatx4_t o{0.f, 0.f, 0.f, 0.f};
  for (int s = 0; s < p.splits; ++s) {
    const float f = weight(p.part_ml[(first + 16 * s) * 2], base, p.c);
    l += f * p.part_ml[(first + 16 * s) * 2 + 1];
    o += f * *reinterpret_cast<const floatx4_t*>(p.part_o + (first + 16 * s) * D + d);
  }
  const float inv = l == 0.f ? 0.f : 1.f / l;
  store4(static_cast<T*>(p.out) + at * D + d, o * inv);
}

// How a call is launched. A list's time is that of its wavefronts' units one after the other (1.3 us each): few lists get 8
// wavefronts each, and parts, joined by a second launch, up to one workgroup a CU (1 x 1 position, 4 kv heads: 128 blocks
// 12.2 us, uncut 18.1; with 4 wavefronts and up to 3 parts a CU 12.5). More lists get 4 wavefronts, three workgroups to a
// CU, and parts where these leave 8 units to a wavefront (16 x 5: 256 blocks 46.8 us, uncut 55.4; 64 blocks 22.5 and
// 19.4). 64 x 1, 64 blocks: 8 wavefronts 24.7 us, 4 and parts 29.4. With 2 and 1 wavefronts: 2 x 257 61 and 64 us in place
// of 58, 16 x 5, 256 blocks 55 and 82 in place of 47. ONCE, loads that leave the caches alone, where no other
// workgroup reads a list's blocks: 256 x 1, 64 blocks 87 us, with ordinary loads 99; but 2 x 257 77 and 68.
// Of several positions there are no more parts than let each XCD hold all workgroups of its own, by XCD below (17 x 5 x 1
// head: 64 blocks 12.0 us, with one part more 15.0, 128 blocks 15.6 and 21.9; 10 x 5 x 1 in f32, 228 blocks 29.6 and 38.1).
struct BlocksPlan { int row_groups, splits, per_split, waves; };
// Workgroups on the fullest XCD, where `inner` of each group are on one
long fullest_xcd(long groups, long inner) { return (groups + 7) / 8 * inner; }
BlocksPlan blocks_plan(int B, int n, int Hq, int Hkv, int N) {
  BlocksPlan pl{};
  const int units = (N + 1) / 2;
  pl.row_groups = (Hq / Hkv + 15) / 16;
  const long inner = long(n) * pl.row_groups, lists = long(B) * Hkv * inner;
  pl.waves = lists <= 256 ? 8 : 4;
  const long most = std::max(1l, pl.waves == 8 ? std::min(256 / lists, long(units) / 8) : std::min(768 / lists, long(units) / 32));
  long parts = most;
  if (pl.waves == 8 && inner > 1) {
    while (parts > 1 && fullest_xcd(B * long(Hkv) * parts, inner) > 32) --parts;
    if (fullest_xcd(B * long(Hkv) * parts, inner) > 32) parts = most;
  }
  pl.per_split = int((units + parts - 1) / parts);
  pl.splits = (units + pl.per_split - 1) / pl.per_split;
  return pl;
}

// Whether workgroups by XCD, `inner` of each group on one, take about as many rounds of the CUs as in the grid's order: then
// what they share in L2 pays (x 5 positions x 4 kv heads, lists out of tables of 1000 blocks: 16 sequences, 128 blocks, 1.65
// lists' blocks in all, 33.7 us, in the grid's order 56.1; 128, 64 blocks, 2.15 lists', 124 and 196; 3, 256 blocks 17.1 and
// 19.1), else the fullest XCD's further round costs more (1 x 257 x 4 heads 56 and 35)
bool fits_by_xcd(long groups, long inner, int waves, molt_dtype dt) {
  const long places = 32 * (waves == 8 ? 1 : dt == MOLT_F32 ? 2 : 3);    // of an XCD
  const long fullest = (fullest_xcd(groups, inner) + places - 1) / places;
  const long even = (groups * inner + 8 * places - 1) / (8 * places);
  return 4 * fullest <= 5 * even;
}

}  // namespace

double blocks_attention_groups(int B, int n, int Hq, int Hkv, int N) {
  const BlocksPlan pl = blocks_plan(B, n, Hq, Hkv, N);
  return 2 * std::max((double(B) * Hkv + 7) * n * pl.row_groups * pl.splits, double(B) * n * Hq / 8);
}

size_t blocks_attention_ws_bytes(int B, int n, int Hq, int Hkv, int D, int N) {
  const BlocksPlan pl = blocks_plan(B, n, Hq, Hkv, N);
  if (pl.splits == 1) return 0;
  const size_t rows = size_t(B) * n * Hkv * pl.row_groups * pl.splits * 16;
  return rows * (D + 2) * sizeof(float) + 512;
}

hipError_t launch_blocks_attention(const void* q, const void* kc, const void* vc, const int32_t* bt, const int32_t* ctx,
                                   const int32_t* blocks, int B, int n, int Hq, int Hkv, int D, int max_blocks,
                                   int num_blocks, int N, molt_dtype dt, void* out, void* ws, size_t ws_bytes,
                                   hipStream_t s) {
  const BlocksPlan pl = blocks_plan(B, n, Hq, Hkv, N);
  const long groups = long(B) * Hkv * pl.splits;
  const long inner = long(n) * pl.row_groups;
  const int by_xcd = inner > 1 && fits_by_xcd(groups, inner, pl.waves, dt);
  const bool once = n == 1 && pl.row_groups == 1;
  BlocksArgs p{q, kc, vc, bt, ctx, blocks, out, nullptr, nullptr, B, n, Hq, Hkv, Hq / Hkv, N, max_blocks, num_blocks,
               pl.row_groups, pl.splits, dt == MOLT_F32 ? 2 * pl.per_split : pl.per_split, by_xcd,
               kLog2e / std::sqrt(float(D))};
  const size_t rows = size_t(B) * n * Hkv * pl.row_groups * pl.splits;
  if (pl.splits > 1) {
    Carver c(ws, ws_bytes);
    p.part_o = c.take<float>(rows * 16 * D);
    p.part_ml = c.take<float>(rows * 16 * 2);
  }
  const unsigned grid = unsigned((by_xcd ? (groups + 7) / 8 * 8 : groups) * inner);
  const unsigned joins = unsigned((long(B) * n * Hq * (D / 4) + 255) / 256);
  auto go = [&](auto d, auto* t) {
    constexpr int DD = decltype(d)::value;
    typedef std::remove_pointer_t<decltype(t)> T;
    auto run = [&](auto w, auto o) {
      constexpr int W = decltype(w)::value;
      blocks_attention_kernel<DD, T, W, decltype(o)::value><<<grid, W * kWave, 0, s>>>(p);
    };
    typedef std::integral_constant<int, 4> Four;
    typedef std::integral_constant<int, 8> Eight;
    if (pl.waves == 4) once ? run(Four{}, std::true_type{}) : run(Four{}, std::false_type{});
    else once ? run(Eight{}, std::true_type{}) : run(Eight{}, std::false_type{});
    if (p.splits > 1) blocks_join_kernel<DD, T><<<joins, 256, 0, s>>>(p);
  };
  auto by_dim = [&](auto* t) {
    if (D == 128) go(std::integral_constant<int, 128>{}, t);
    else go(std::integral_constant<int, 64>{}, t);
  };
  if (dt == MOLT_F32) by_dim(static_cast<float*>(nullptr));
  else by_dim(static_cast<uint16_t*>(nullptr));
  return hipGetLastError();
}

}  // namespace molt
