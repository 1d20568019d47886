// Selection of cache blocks for sparse attention: for every query position and kv head the blocks of largest score.
//   s(block) = max over the kv head's query rows of 2^(e_q + e) sum_d max(c_d hi_d, c_d lo_d)
// with the row's codes c (8 bits) and the block's bounds hi, lo (bounds_format.h). With c+ = max(c, 0) and c- = min(c, 0)
// the sum is c+ . hi + c- . lo, one product over 2 D whole numbers: 8-bit MFMAs, exact, and so is its scaling. Which
// blocks are the largest then depends on no order of summation.
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "bounds_format.h"
#include "internal.h"

namespace molt {
namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / kWave;
constexpr int kTiles = 4;                        // row tiles of a workgroup: 64 query rows

typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));
typedef uint32_t UnalignedU4 __attribute__((ext_vector_type(4), aligned(2)));
typedef float UnalignedF4 __attribute__((ext_vector_type(4), aligned(4)));

struct SelectArgs {
  const void* q; const uint8_t* bounds; const int32_t* bt; const int32_t* ctx; const int32_t* lens;
  int B, n, Hq, Hkv, G, N, n_first, n_last, max_blocks, num_blocks;
  uint32_t* keys;                                // [B n, Hkv, max_blocks]
  int32_t* out;                                  // [B n, Hkv, N]
};

// Keys order as scores do, as unsigned numbers: 0 for a block that the position does not see, above every score those
// of infinite score and those that a list holds anyway.
constexpr uint32_t kKeyHeld = 0xffffffffu, kKeyInfinite = 0xff800000u;
MOLT_DEV uint32_t order_key(float s) {
  const uint32_t u = __float_as_uint(s);
  return u ^ (uint32_t(int32_t(u) >> 31) | 0x80000000u);
}

// Blocks that position ctx[b] + j sees, 0 where the row does not count
MOLT_DEV int visible_blocks(const SelectArgs& p, int b, int j) {
  if (p.lens && j >= p.lens[b]) return 0;
  const long pos = long(p.ctx[b]) + j;
  return pos < 0 ? 0 : int(min(pos / 16 + 1, long(p.max_blocks)));
}

MOLT_DEV void load16(const uint16_t* p, float (&x)[16]) {
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const UnalignedU4 w = *reinterpret_cast<const UnalignedU4*>(p + 8 * i);
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      x[8 * i + 2 * c] = __uint_as_float(w[c] << 16);
      x[8 * i + 2 * c + 1] = __uint_as_float(w[c] & 0xffff0000u);
    }
  }
}
MOLT_DEV void load16(const float* p, float (&x)[16]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const UnalignedF4 w = *reinterpret_cast<const UnalignedF4*>(p + 4 * i);
#pragma unroll
    for (int c = 0; c < 4; ++c) x[4 * i + c] = w[c];
  }
}

// A query row as the A operands of 16x16x64 8-bit MFMAs: lane's row r = lane % 16; dims 16 g .. + 15 of each 64, for
// k-steps over the codes of hi (c+), then over those of lo (c-). Returns the row's exponent.
template <int D, typename T>
MOLT_DEV int query_codes(const T* q, bool there, int g, int32x4_t (&a)[D / 32]) {
  constexpr int S = D / 64;
  float x[S][16];
  uint32_t top = 0;
#pragma unroll
  for (int s = 0; s < S; ++s) {
    if (there) load16(q + 64 * s + 16 * g, x[s]);
    else for (int i = 0; i < 16; ++i) x[s][i] = 0.f;
#pragma unroll
    for (int i = 0; i < 16; ++i) top = max(top, __float_as_uint(x[s][i]) & 0x7fffffffu);
  }
  top = max(top, uint32_t(__shfl_xor(int(top), 16)));
  top = max(top, uint32_t(__shfl_xor(int(top), 32)));
  const bool bad = top >= 0x7f800000u;
  const int e = bad ? kBoundsMinExponent : bounds_exponent(top);
  const float r = pow2(-e);
#pragma unroll
  for (int s = 0; s < S; ++s)
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      int c[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) c[i] = bad ? 0 : int(__builtin_rintf(x[s][4 * w + i] * r));
      a[s][w] = int(pack_codes(max(c[0], 0), max(c[1], 0), max(c[2], 0), max(c[3], 0)));
      a[S + s][w] = int(pack_codes(min(c[0], 0), min(c[1], 0), min(c[2], 0), min(c[3], 0)));
    }
  return e;
}

// Scores of a workgroup's positions (GP rows of a tile each, the kv head's G query rows and rows that do not count)
// against a chunk of a sequence's blocks; wavefront = 16 blocks in turn. G > 16: TPP tiles a position.
template <int D, int GP, typename T>
__global__ __launch_bounds__(kThreads) void score_kernel(SelectArgs p, int pos_groups, int chunks, int chunk) {
  typedef BoundsRecord<D> Rec;
  constexpr int S = D / 32, PPT = 16 / GP;       // MFMA steps, positions of a tile
  const int lane = threadIdx.x % kWave, g = lane / 16, col = lane % 16;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  uint32_t item = blockIdx.x;
  const int c0 = int(item % chunks) * chunk;
  item /= chunks;
  const int h = int(item % p.Hkv);
  item /= p.Hkv;
  const int group = int(item % pos_groups), b = int(item / pos_groups);
  const int tpp = (p.G + 15) / 16;               // 1 where GP < 16
  const int j0 = group * (tpp > 1 ? 1 : kTiles * PPT);
  const int n_here = min(p.n - j0, tpp > 1 ? 1 : kTiles * PPT);
  const int count = p.lens ? min(n_here, p.lens[b] - j0) : n_here;       // rows that count
  const int end = count <= 0 ? 0 : min(visible_blocks(p, b, j0 + count - 1), c0 + chunk);
  if (c0 >= end) return;

  const T* q = static_cast<const T*>(p.q);
  for (int t0 = 0; t0 < tpp; t0 += kTiles) {     // one round but for G > 64
    int32x4_t a[kTiles][S];
    int eq[kTiles][4];
#pragma unroll
    for (int t = 0; t < kTiles; ++t) {
      const int j = tpp > 1 ? j0 : j0 + t * PPT + col / GP, head = tpp > 1 ? (t0 + t) * 16 + col : col % GP;
      const bool there = j < p.n && head < p.G;
      const int e = query_codes<D, T>(q + ((long(b) * p.n + j) * p.Hq + h * p.G + head) * D, there, g, a[t]);
#pragma unroll
      for (int i = 0; i < 4; ++i) eq[t][i] = __shfl(there ? e : 1000, 4 * g + i);   // of the accumulator's rows
    }
    for (int k0 = c0 + 16 * wave; k0 < end; k0 += 16 * kWaves) {
      const int blk = k0 + col;
      const int id = blk < end ? p.bt[long(b) * p.max_blocks + blk] : -1;
      const bool good = id >= 0 && id < p.num_blocks;
      const uint8_t* rec = p.bounds + (long(good ? id : 0) * p.Hkv + h) * Rec::kBytes;
      int32x4_t w[S];
#pragma unroll
      for (int s = 0; s < S; ++s) w[s] = *reinterpret_cast<const int32x4_t*>(rec + 64 * s + 16 * g);
      const int ek = int(int8_t(rec[Rec::kExponent]));
#pragma unroll
      for (int t = 0; t < kTiles; ++t) {
        const int first_j = tpp > 1 ? j0 : j0 + t * PPT;
        if (first_j >= p.n || (tpp > 1 && t0 + t >= tpp)) continue;
        int32x4_t acc{0, 0, 0, 0};
#pragma unroll
        for (int s = 0; s < S; ++s) acc = __builtin_amdgcn_mfma_i32_16x16x64_i8(a[t][s], w[s], acc, 0, 0, 0);
        float f[4];
#pragma unroll
        for (int i = 0; i < 4; ++i)
          f[i] = eq[t][i] == 1000 ? -__builtin_inff() : float(acc[i]) * pow2(min(max(eq[t][i] + ek, -100), 100));
        // rows 4 g + i of the tile: the positions' maxima
        constexpr int OUT = GP >= 4 ? 1 : 4 / GP;
        float best[OUT];
#pragma unroll
        for (int o = 0; o < OUT; ++o) {
          best[o] = f[o * (4 / OUT)];
#pragma unroll
          for (int i = 1; i < 4 / OUT; ++i) best[o] = fmaxf(best[o], f[o * (4 / OUT) + i]);
          if (GP >= 8) best[o] = fmaxf(best[o], __shfl_xor(best[o], 16));
          if (GP >= 16) best[o] = fmaxf(best[o], __shfl_xor(best[o], 32));
        }
        const bool writes = GP <= 4 || (GP == 8 ? g % 2 == 0 : g == 0);
#pragma unroll
        for (int o = 0; o < OUT; ++o) {
          const int j = first_j + (GP >= 4 ? 4 * g / GP : 4 * g / GP + o);
          if (!writes || j >= p.n || blk >= end) continue;
          const int last = visible_blocks(p, b, j) - 1;
          uint32_t key = 0;
          if (good && blk <= last) {
            key = ek == kBoundsNotFinite ? kKeyInfinite : order_key(best[o]);
            if (blk < p.n_first || blk > last - p.n_last) key = kKeyHeld;
          }
          uint32_t* to = p.keys + ((long(b) * p.n + j) * p.Hkv + h) * p.max_blocks + blk;
          if (tpp > 1 && (t0 || t)) key = max(key, *to);
          *to = key;
        }
      }
    }
  }
}

// Workgroup = one list. The N-th largest key by 8 bits at a time, from histograms in LDS; then the blocks above it and
// the first of those equal to it, in their order.
__global__ __launch_bounds__(kThreads) void pick_kernel(SelectArgs p) {
  __shared__ int hist[256];
  __shared__ int sums[2][kWaves];
  __shared__ int digit, above;
  const long list = blockIdx.x;
  const int t = int(list / p.Hkv), b = t / p.n, j = t % p.n;
  const int seen = visible_blocks(p, b, j);
  const uint32_t* keys = p.keys + list * p.max_blocks;
  int32_t* out = p.out + list * p.N;
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  uint32_t floor_key = 0;                        // keys under it are out, those above it in
  int equal = 0;                                 // of those equal to it, the first so many are in
  if (seen > p.N) {
    uint32_t prefix = 0;
    int need = p.N;
    for (int shift = 24; shift >= 0; shift -= 8) {
      hist[threadIdx.x] = 0;
      __syncthreads();
      for (int i = threadIdx.x; i < seen; i += kThreads) {
        const uint32_t key = keys[i];
        if (shift == 24 || key >> (shift + 8) == prefix >> (shift + 8)) atomicAdd(&hist[key >> shift & 255], 1);
      }
      __syncthreads();
      // keys of larger digits than 255 - thread
      const int mine = hist[255 - threadIdx.x];
      int s = wave_scan_dpp(mine);
      if (lane == kWave - 1) sums[0][wave] = s;
      __syncthreads();
      for (int w = 0; w < wave; ++w) s += sums[0][w];
      if (s >= need && s - mine < need) {
        digit = 255 - int(threadIdx.x);
        above = s - mine;
      }
      __syncthreads();
      prefix |= uint32_t(digit) << shift;
      need -= above;
    }
    floor_key = prefix;
    equal = need;
  }
  if (floor_key == 0) equal = 0;                 // what a position does not see is never taken
  int base_above = 0, base_equal = 0;
  for (int i0 = 0; i0 < seen; i0 += kThreads) {
    const int i = i0 + int(threadIdx.x);
    const uint32_t key = i < seen ? keys[i] : 0u;
    const bool in = key > floor_key, eq = key == floor_key && key != 0;
    const unsigned long long mi = __ballot(in), me = __ballot(eq), below = (1ull << lane) - 1;
    __syncthreads();
    if (lane == 0) { sums[0][wave] = __popcll(mi); sums[1][wave] = __popcll(me); }
    __syncthreads();
    int ai = base_above + __popcll(mi & below), ae = base_equal + __popcll(me & below);
    for (int w = 0; w < kWaves; ++w) {
      if (w < wave) { ai += sums[0][w]; ae += sums[1][w]; }
      base_above += sums[0][w];
      base_equal += sums[1][w];
    }
    if (in || (eq && ae < equal)) out[ai + min(ae, equal)] = i;
  }
  for (int i = base_above + min(base_equal, equal) + int(threadIdx.x); i < p.N; i += kThreads) out[i] = -1;
}

int pow2_rows(int G) { return G <= 1 ? 1 : G <= 2 ? 2 : G <= 4 ? 4 : G <= 8 ? 8 : 16; }

// Positions of a workgroup of score_kernel, and blocks
int score_positions(int G) { return G > 16 ? 1 : kTiles * 16 / pow2_rows(G); }
constexpr int kScoreChunk = 16 * kWaves * 2;

}  // namespace

double select_groups(int B, int n, int Hq, int Hkv, int max_blocks) {
  const double at = score_positions(Hq / Hkv);
  return std::max(double(B) * std::ceil(n / at) * Hkv * std::ceil(max_blocks / double(kScoreChunk)), double(B) * n * Hkv);
}

size_t select_ws_bytes(int B, int n, int Hkv, int max_blocks) {
  return size_t(B) * n * Hkv * max_blocks * sizeof(uint32_t) + 256;
}

hipError_t launch_select_blocks(const void* q, const void* bounds, const int32_t* bt, const int32_t* ctx,
                                const int32_t* lens, int B, int n, int Hq, int Hkv, int D, int max_blocks,
                                int num_blocks, int N, int n_first, int n_last, molt_dtype dt, int32_t* out, void* ws,
                                size_t ws_bytes, hipStream_t s) {
  Carver c(ws, ws_bytes);
  SelectArgs p{q, static_cast<const uint8_t*>(bounds), bt, ctx, lens, B, n, Hq, Hkv, Hq / Hkv, N, n_first, n_last,
               max_blocks, num_blocks, c.take<uint32_t>(size_t(B) * n * Hkv * max_blocks), out};
  const int gp = pow2_rows(p.G), per_group = score_positions(p.G), pos_groups = int((long(n) + per_group - 1) / per_group);
  const int chunk = kScoreChunk, chunks = (max_blocks + chunk - 1) / chunk;
  const unsigned grid = unsigned(long(B) * pos_groups * Hkv * chunks);
  auto go = [&](auto kernel) { kernel<<<grid, kThreads, 0, s>>>(p, pos_groups, chunks, chunk); };
  auto by_rows = [&](auto d, auto* t) {
    constexpr int DD = decltype(d)::value;
    typedef std::remove_pointer_t<decltype(t)> T;
    switch (gp) {
      case 1: go(score_kernel<DD, 1, T>); break;
      case 2: go(score_kernel<DD, 2, T>); break;
      case 4: go(score_kernel<DD, 4, T>); break;
      case 8: go(score_kernel<DD, 8, T>); break;
      default: go(score_kernel<DD, 16, T>);
    }
  };
  auto by_dim = [&](auto* t) {
    if (D == 128) by_rows(std::integral_constant<int, 128>{}, t);
    else by_rows(std::integral_constant<int, 64>{}, t);
  };
  if (dt == MOLT_F32) by_dim(static_cast<float*>(nullptr));
  else by_dim(static_cast<uint16_t*>(nullptr));
  if (hipError_t e = hipGetLastError()) return e;
  pick_kernel<<<unsigned(long(B) * n * Hkv), kThreads, 0, s>>>(p);
  return hipGetLastError();
}

}  // namespace molt
