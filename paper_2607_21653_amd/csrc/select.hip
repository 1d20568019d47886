// Selection of cache blocks for sparse attention: for every query position and kv head the blocks of largest score.
//   s(block) = max over the kv head's query rows of 2^(e_q + e) sum_d max(c_d hi_d, c_d lo_d)
// with the row's codes c (8 bits) and the block's bounds hi, lo (bounds_format.h). With c+ = max(c, 0) and c- = min(c, 0)
// the sum is c+ . hi + c- . lo, one product over 2 D whole numbers: 8-bit MFMAs, exact, and so is its scaling. Which
// blocks are the largest then depends on no order of summation.
//
// Bound by the records' bytes (2 D + 1 a block and kv head, read once for all of a position group's rows) and by the chain of
// id, record, product, search: 128 sequences x 5 positions at 8192, 4 kv heads x 128 (74 MB) 23.4 us, 3.1 TB/s; 16 x 5 at
// 32768-65536 (51 MB) 16.4 us for the scores and 8.6 for the lists; one position 7.1 us.
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "bounds_format.h"
#include "internal.h"

namespace molt {
namespace {

constexpr int kWaves = 8;
constexpr int kThreads = kWaves * kWave;
constexpr size_t kFusedLds = 112 << 10;          // 128 x 5 positions, 2000 blocks: 76.5 us, in two launches 81.6

typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));
typedef uint32_t UnalignedU4 __attribute__((ext_vector_type(4), aligned(2)));
typedef float UnalignedF4 __attribute__((ext_vector_type(4), aligned(4)));

struct SelectArgs {
  const void* q; const uint8_t* bounds; const int32_t* bt; const int32_t* ctx; const int32_t* lens;
  int B, n, Hq, Hkv, G, N, n_first, n_last, max_blocks, num_blocks;
  uint32_t* keys;                                // [B n, Hkv, max_blocks]
  int32_t* out;                                  // [B n, Hkv, N]
  int f32;                                       // q's type
  uint32_t block_bytes;                          // of a block's records
  int pos_groups, chunks, chunk, by_xcd;         // launch: groups of positions, chunks of blocks and their size,
                                                 // sequences by XCD
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
MOLT_DEV int query_codes(const T* q, int g, int32x4_t (&a)[D / 32]) {
  constexpr int S = D / 64;
  float x[S][16];
  uint32_t top = 0;
#pragma unroll
  for (int s = 0; s < S; ++s) {
    load16(q + 64 * s + 16 * g, x[s]);
#pragma unroll
    for (int i = 0; i < 16; ++i) top = max(top, __float_as_uint(x[s][i]) & 0x7fffffffu);
  }
  top = max(top, uint32_t(__shfl_xor(int(top), 16)));
  top = max(top, uint32_t(__shfl_xor(int(top), 32)));
  const bool bad = top >= 0x7f800000u;
  const int e = bad ? kBoundsMinExponent : bounds_exponent(top);
  const float r = pow2(-e), magic = 12582912.0f;   // 1.5 * 2^23: x r + magic rounds x r to a whole number, ties to
#pragma unroll                                     // even, whose two's complement is in the sum's low bits
  for (int s = 0; s < S; ++s)
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      uint32_t c[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) c[i] = __float_as_uint(__builtin_fmaf(x[s][4 * w + i], r, magic));
      uint32_t codes = (c[0] & 0xffu) | (c[1] & 0xffu) << 8 | (c[2] & 0xffu) << 16 | c[3] << 24;
      if (bad) codes = 0;
      const uint32_t sign = codes >> 7 & 0x01010101u, negative = (sign << 8) - sign;
      a[s][w] = int(codes & ~negative);
      a[S + s][w] = int(codes & negative);
    }
  return e;
}

// Query rows in tiles of 16: a position's rows are padded to GP = 4, 8 or 16 of them, and where G > 16 take several
// tiles; padding repeats the last row, which leaves the maximum as it is. A workgroup has the rows of 64 / GP positions,
// or of one.
struct Tiling { int tpp, positions; };           // tiles of a position, positions of a workgroup
template <int GP>
MOLT_DEV Tiling tiling_of(int G) {
  const int tpp = (G + 15) / 16;
  return {tpp, tpp > 1 ? 1 : 64 / GP};
}

// LDS of a workgroup: codes and exponents of its tiles of query rows, as MFMA operands; 16 records for each wavefront,
// which go through it into the MFMA's order
constexpr int kMaxTiles = 4;
template <int D>
struct ScoreLds {
  uint8_t records[kWaves][16 * 2 * D];
  int32x4_t a[kMaxTiles][D / 32][kWave];
  int32x4_t e[kMaxTiles][4];
};

// Codes of tiles t0 .. t0 + 3 of the workgroup's rows into LDS, a wavefront a tile
template <int D, int GP>
MOLT_DEV void stage_codes(const SelectArgs& p, const Tiling& ti, int b, int h, int j0, int t0, int wave, int lane,
                          ScoreLds<D>& lds) {
  const int g = lane / 16, col = lane % 16;
  if (wave < kMaxTiles) {
    const int j = ti.tpp > 1 ? j0 : min(j0 + (wave * 16 + col) / GP, p.n - 1);
    const int head = min(ti.tpp > 1 ? (t0 + wave) * 16 + col : col % GP, p.G - 1);
    const long at = ((long(b) * p.n + j) * p.Hq + h * p.G + head) * D;
    int32x4_t a[D / 32];
    const int e = p.f32 ? query_codes<D>(static_cast<const float*>(p.q) + at, g, a)
                        : query_codes<D>(static_cast<const uint16_t*>(p.q) + at, g, a);
#pragma unroll
    for (int s = 0; s < D / 32; ++s) lds.a[wave][s][lane] = a[s];
    if (g == 0) reinterpret_cast<int*>(lds.e[wave])[col] = e;
  }
}

// v_max_f32, which the compiler surrounds with instructions that quiet NaN: there is none here
MOLT_DEV float max_of(float a, float b) {
  float r;
  asm("v_max_f32 %0, %1, %2" : "=v"(r) : "v"(a), "v"(b));
  return r;
}

// 16 records on their way: 16 bytes a lane, a record's bytes by lanes side by side (as the MFMA takes them, 16 bytes
// of 16 records by 16 lanes, each lane's would be a request of its own); lanes 0 .. 15 have a record's exponent.
template <int D>
struct Records {
  static constexpr int L = 2 * D / 16, PB = kWave / L, S = D / 32;       // lanes a record, records a load, loads
  int32x4_t w[S];
  int e, block;                                  // of record lane % 16; block < 0: none
  MOLT_DEV void load(const SelectArgs& p, const uint8_t* head, int id, int lane) {
    block = id >= 0 && id < p.num_blocks ? id : -1;
    const int use = max(block, 0);               // (block 0's in the place of one that is not there)
#pragma unroll
    for (int c = 0; c < S; ++c) {
      const uint32_t r = uint32_t(__shfl(use, c * PB + lane / L));
      w[c] = *reinterpret_cast<const int32x4_t*>(head + uint64_t(r) * p.block_bytes + lane % L * 16);
    }
    if (lane < 16) e = int(int8_t(head[uint64_t(uint32_t(use)) * p.block_bytes + BoundsRecord<D>::kExponent]));
  }
  // to LDS, the 16-byte chunks of record r at places chunk ^ r, so that both ways are free of conflicts
  MOLT_DEV void store(uint8_t* to, int lane) const {
#pragma unroll
    for (int c = 0; c < S; ++c) {
      const int r = c * PB + lane / L;
      *reinterpret_cast<int32x4_t*>(to + r * 2 * D + ((lane % L) ^ (r % L)) * 16) = w[c];
    }
  }
  MOLT_DEV static void operand(const uint8_t* from, int lane, int32x4_t (&f)[S]) {
    const int g = lane / 16, col = lane % 16;
#pragma unroll
    for (int s = 0; s < S; ++s)
      f[s] = *reinterpret_cast<const int32x4_t*>(from + col * 2 * D + ((4 * s + g) ^ (col % L)) * 16);
  }
};

// Keys of the workgroup's positions for blocks c0 .. end - 1 of the sequence, of position i at keys + i * stride, block
// c0 + x at [x]. (Which of them the position sees, the pick knows.) Wavefront = 32 blocks in turn, the next 32 records in
// registers, the places of the 32 after them.
template <int D, int GP, typename Keys>
MOLT_DEV void score_blocks(const SelectArgs& p, int b, int h, int j0, int c0, int end, int wave, int lane,
                           ScoreLds<D>& lds, Keys keys, long stride) {
  constexpr int S = D / 32, STEP = 32 * kWaves;
  const int g = lane / 16, col = lane % 16;
  const Tiling ti = tiling_of<GP>(p.G);
  const int32_t* row = p.bt + long(b) * p.max_blocks;
  const uint8_t* head = p.bounds + long(h) * BoundsRecord<D>::kBytes;
  auto place = [&](int at) { return at < end ? row[at] : -1; };
  for (int t0 = 0; t0 < ti.tpp; t0 += kMaxTiles) {   // one round but for G > 64
    const int k1 = c0 + 32 * wave + col;
    const int id0 = place(k1), id1 = place(k1 + 16);
    int next0 = place(k1 + STEP), next1 = place(k1 + STEP + 16);
    if (t0) __syncthreads();
    stage_codes<D, GP>(p, ti, b, h, j0, t0, wave, lane, lds);
    Records<D> r0, r1;
    r0.load(p, head, id0, lane);
    r1.load(p, head, id1, lane);
    __syncthreads();
    const int tiles = ti.tpp > 1 ? min(ti.tpp - t0, kMaxTiles) : min((p.n - j0 + 16 / GP - 1) / (16 / GP), kMaxTiles);
    uint8_t* mine = lds.records[wave];
    for (int k0 = k1; k0 - col < end; k0 += STEP) {
      int32x4_t f0[S], f1[S];
      r0.store(mine, lane);
      Records<D>::operand(mine, lane, f0);
      r1.store(mine, lane);
      Records<D>::operand(mine, lane, f1);
      const int ek0 = __shfl(r0.e, col), ek1 = __shfl(r1.e, col);
      const bool no0 = r0.block < 0, no1 = r1.block < 0;
      r0.load(p, head, next0, lane);
      r1.load(p, head, next1, lane);
      next0 = place(k0 + 2 * STEP);
      next1 = place(k0 + 2 * STEP + 16);
      float best0 = -__builtin_inff(), best1 = best0;
      for (int t = 0; t < tiles; ++t) {
        int32x4_t acc0{0, 0, 0, 0}, acc1{0, 0, 0, 0};
#pragma unroll
        for (int s = 0; s < S; ++s) {
          const int32x4_t a = lds.a[t][s][lane];
          acc0 = __builtin_amdgcn_mfma_i32_16x16x64_i8(a, f0[s], acc0, 0, 0, 0);
          acc1 = __builtin_amdgcn_mfma_i32_16x16x64_i8(a, f1[s], acc1, 0, 0, 0);
        }
        const int32x4_t eq = lds.e[t][g];        // of rows 4 g + i
        float x0[4], x1[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          x0[i] = __builtin_ldexpf(float(acc0[i]), min(max(eq[i] + ek0, -100), 100));
          x1[i] = __builtin_ldexpf(float(acc1[i]), min(max(eq[i] + ek1, -100), 100));
        }
        float m0 = max_of(max_of(x0[0], x0[1]), max_of(x0[2], x0[3]));
        float m1 = max_of(max_of(x1[0], x1[1]), max_of(x1[2], x1[3]));
        if (GP >= 8) {                           // a position's rows are in 2 or 4 of the g
          const auto y0 = __builtin_amdgcn_permlane16_swap(__float_as_uint(m0), __float_as_uint(m0), false, false);
          const auto y1 = __builtin_amdgcn_permlane16_swap(__float_as_uint(m1), __float_as_uint(m1), false, false);
          m0 = max_of(__uint_as_float(y0[0]), __uint_as_float(y0[1]));
          m1 = max_of(__uint_as_float(y1[0]), __uint_as_float(y1[1]));
        }
        if (GP >= 16) {
          const auto y0 = __builtin_amdgcn_permlane32_swap(__float_as_uint(m0), __float_as_uint(m0), false, false);
          const auto y1 = __builtin_amdgcn_permlane32_swap(__float_as_uint(m1), __float_as_uint(m1), false, false);
          m0 = max_of(__uint_as_float(y0[0]), __uint_as_float(y0[1]));
          m1 = max_of(__uint_as_float(y1[0]), __uint_as_float(y1[1]));
          if (ti.tpp > 1) {
            best0 = m0 = max_of(best0, m0);
            best1 = m1 = max_of(best1, m1);
            if (t < tiles - 1) continue;
          }
        }
        const int i = ti.tpp > 1 ? 0 : (t * 16 + 4 * g) / GP;
        if (4 * g % GP != 0 || j0 + i >= p.n) continue;
        uint32_t key0 = ek0 == kBoundsNotFinite ? kKeyInfinite : order_key(m0);
        uint32_t key1 = ek1 == kBoundsNotFinite ? kKeyInfinite : order_key(m1);
        if (no0) key0 = 0;
        if (no1) key1 = 0;
        auto to = keys + i * stride + (k0 - c0);
        if (GP == 16 && t0) {                    // over the rounds
          if (k0 < end) key0 = max(key0, to[0]);
          if (k0 + 16 < end) key1 = max(key1, to[16]);
        }
        if (k0 < end) to[0] = key0;
        if (k0 + 16 < end) to[16] = key1;
      }
    }
  }
}

// What a list holds beside the scores: the first blocks and the last that the position sees, before all others
MOLT_DEV uint32_t list_key(const SelectArgs& p, uint32_t key, int blk, int seen) {
  return key != 0 && (blk < p.n_first || blk >= seen - p.n_last) ? kKeyHeld : key;
}

// Sum over the wavefront of four numbers at once; PACKED: of numbers that sum to less than 2^16
struct Four { uint32_t x[4]; };
template <bool PACKED>
MOLT_DEV Four wave_sum4(const Four& c) {
  auto total = [](uint32_t v) { return uint32_t(__builtin_amdgcn_readlane(wave_scan_dpp(int(v)), 63)); };
  if (PACKED) {
    const uint32_t a = total(c.x[0] | c.x[1] << 16), b = total(c.x[2] | c.x[3] << 16);
    return Four{{a & 0xffffu, a >> 16, b & 0xffffu, b >> 16}};
  }
  return Four{{total(c.x[0]), total(c.x[1]), total(c.x[2]), total(c.x[3])}};
}
MOLT_DEV uint32_t wave_max_u32(uint32_t v) {
  v = max(v, dpp_u32<0x111, 0xF>(v, 0u));
  v = max(v, dpp_u32<0x112, 0xF>(v, 0u));
  v = max(v, dpp_u32<0x114, 0xF>(v, 0u));
  v = max(v, dpp_u32<0x118, 0xF>(v, 0u));
  v = max(v, dpp_u32<0x142, 0xA>(v, 0u));
  v = max(v, dpp_u32<0x143, 0xC>(v, 0u));
  return lane63(v);
}

// The border of the N largest keys: keys >= lo are in, and of those equal to `equal_key` (if `equal` > 0) the first
// `equal`. It is searched between the smallest and the largest key, by the counts of 256 parts of what is left, which ends as
// soon as just N keys are not below a part's start; only where equal keys straddle the border does it run down to that key.
struct Border { uint32_t lo, equal_key; int equal; };
constexpr int kBins = 4 * kWave;

// More than N keys are >= lo (c_lo of them), fewer than N are >= hi (c_hi); or N are >= lo
struct Search {
  uint32_t lo, hi;
  int c_lo, c_hi;
  bool exact;
  MOLT_DEV bool done() const { return exact || hi - lo <= 1; }
  MOLT_DEV int shift() const { return max(24 - __builtin_clz(hi - lo - 1), 0); }     // a part's size
  MOLT_DEV void add(uint32_t* bins, int shift, uint32_t key) const {
    if (key >= lo && key < hi) atomicAdd(&bins[(key - lo) >> shift], 1u);
  }
  // to the part that the border is in (16-byte aligned bins)
  MOLT_DEV void narrow(const uint32_t* bins, int shift, int N, int lane) {
    const u32x4_t b = reinterpret_cast<const u32x4_t*>(bins)[lane];
    const int upto = wave_scan_dpp(int(b[0] + b[1] + b[2] + b[3]));
    // keys from the start of each of the lane's parts on
    const int c3 = c_lo - upto + int(b[3]), c2 = c3 + int(b[2]), c1 = c2 + int(b[1]), c0 = c1 + int(b[0]);
    const int l = 63 - __builtin_clzll(__ballot(c0 >= N));                           // (lane 0's are c_lo)
    const int u = c3 >= N ? 3 : c2 >= N ? 2 : c1 >= N ? 1 : 0;
    const int from = c3 >= N ? c3 : c2 >= N ? c2 : c1 >= N ? c1 : c0;
    const int here = int(c3 >= N ? b[3] : c2 >= N ? b[2] : c1 >= N ? b[1] : b[0]);
    lo += uint32_t(__builtin_amdgcn_readlane(4 * lane + u, l)) << shift;
    if (hi - lo > 1u << shift) hi = lo + (1u << shift);
    c_lo = __builtin_amdgcn_readlane(from, l);
    c_hi = c_lo - __builtin_amdgcn_readlane(here, l);
    exact = c_lo == N;
  }
  MOLT_DEV Border border(int N) const {
    if (exact) return {lo, 0u, 0};
    return {lo + 1, lo, N - c_hi};
  }
};
// The end of a search, once no more than 32 keys are between the borders: few keys lie close together now and then, and
// parting them would take many more steps. They go to a lane each (room: these keys, then 0; 16-byte aligned), which
// counts those above its own.
constexpr int kRoom = 32;
MOLT_DEV Border rank_room(const Search& s, const uint32_t* room, int N, int lane) {
  const uint32_t own = lane < kRoom ? room[lane] : 0u, mine = own ? own : ~0u;
  int above = s.c_hi, with = s.c_hi;             // keys above the lane's, and those with the equal ones
#pragma unroll
  for (int i = 0; i < kRoom / 4; ++i) {
    const u32x4_t k = reinterpret_cast<const u32x4_t*>(room)[i];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      above += k[u] > mine;
      with += k[u] >= mine;
    }
  }
  const int l = __builtin_ctzll(__ballot(own != 0 && above < N && with >= N));       // one there is, and equal ones
  const uint32_t k = uint32_t(__builtin_amdgcn_readlane(int(mine), l));
  above = __builtin_amdgcn_readlane(above, l);
  if (__builtin_amdgcn_readlane(with, l) == N) return {k, 0u, 0};
  return {k + 1, k, N - above};
}
// A search by one wavefront that has all keys, M a lane
struct SearchLds { uint32_t bins[kBins], room[kRoom]; };
template <int M>
MOLT_DEV Border wave_search(Search s, const uint32_t (&key)[M], int N, SearchLds& lds, int lane) {
  while (!s.done() && s.c_lo - s.c_hi > kRoom) {
    const int shift = s.shift();
    reinterpret_cast<u32x4_t*>(lds.bins)[lane] = u32x4_t{0, 0, 0, 0};
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int i = 0; i < M; ++i) s.add(lds.bins, shift, key[i]);
    __builtin_amdgcn_wave_barrier();
    s.narrow(lds.bins, shift, N, lane);
    __builtin_amdgcn_wave_barrier();
  }
  if (s.done()) return s.border(N);
  const unsigned long long below = (1ull << lane) - 1;
  int at = 0;
  if (lane < kRoom) lds.room[lane] = 0;
  __builtin_amdgcn_wave_barrier();
#pragma unroll
  for (int i = 0; i < M; ++i) {
    const bool in = key[i] >= s.lo && key[i] < s.hi;
    const unsigned long long mask = __ballot(in);
    if (in) lds.room[at + __popcll(mask & below)] = key[i];
    at += __popcll(mask);
  }
  __builtin_amdgcn_wave_barrier();
  return rank_room(s, lds.room, N, lane);
}

// What the keys of m per lane are: how many, how many that a list holds anyway, the largest of the others and of their
// complements
struct Range { uint32_t some, held, top, low; };
template <typename Key>
MOLT_DEV Range range_of(int m, Key key) {
  Range r{0, 0, 0, 0};
#pragma unroll
  for (int i = 0; i < m; ++i) {
    const uint32_t k = key(i);
    r.some += k != 0;
    r.held += k == kKeyHeld;
    if (k != 0 && k != kKeyHeld) {
      r.top = max(r.top, k);
      r.low = max(r.low, ~k);
    }
  }
  return r;
}
MOLT_DEV Search search_of(const Range& r, int N) {
  return {~r.low, r.top + 1, int(r.some), int(r.held), false};
}

// The blocks of keys within the border, in ascending order: a wavefront has those of blocks first + 64 i + lane. `at` of
// them, and `match` equal ones, are in front of it.
template <typename Key>
MOLT_DEV void emit(int m, Key key, const Border& b, int32_t* out, int first, int lane, int at, int match) {
  const unsigned long long below = (1ull << lane) - 1;
#pragma unroll
  for (int i = 0; i < m; ++i) {
    const uint32_t k = key(i);
    bool in = k >= b.lo;
    const unsigned long long mi = __ballot(in);
    int to = at + __popcll(mi & below);
    at += __popcll(mi);
    if (b.equal) {
      const unsigned long long me = __ballot(k == b.equal_key);
      const int rank = match + __popcll(me & below);
      to += min(rank, b.equal);
      in = in || (k == b.equal_key && rank < b.equal);
      match += __popcll(me);
    }
    if (in) out[to] = first + 64 * i + lane;
  }
}

// A workgroup's place: sequence, kv head, position group and chunk of blocks. A sequence's heads, whose records lie side
// by side, run on one XCD where that leaves none idle for long (x 5 positions: 12 sequences, 2000 blocks 14.8 us, in the
// grid's order 15.5; 47, 600 blocks 21.2 and 25.9; but 4, 2000 blocks 11.7 and 11.2; x 1: 9, 1500 blocks 12.4 and 10.8).
struct Item { int b, h, group, chunk; };
MOLT_DEV Item item_of(const SelectArgs& p) {
  uint32_t at = blockIdx.x;
  const uint32_t inner = uint32_t(p.pos_groups) * p.Hkv * p.chunks;
  Item it;
  if (p.by_xcd) {
    const uint32_t slot = at / 8;
    it.b = int(slot / inner * 8 + at % 8);
    at = slot % inner;
  } else {
    it.b = int(at / inner);
    at %= inner;
  }
  it.h = int(at % p.Hkv);
  at /= p.Hkv;
  it.chunk = int(at % p.chunks);
  it.group = int(at / p.chunks);
  return it;
}

// Short tables whose keys fit in LDS: scores and lists in one launch; a wavefront a list
constexpr int kFusedBlocks = 2048;
template <int D, int GP>
__global__ __launch_bounds__(kThreads, 4) void select_kernel(SelectArgs p) {
  extern __shared__ __align__(16) char dyn[];
  ScoreLds<D>& lds = *reinterpret_cast<ScoreLds<D>*>(dyn);
  uint32_t* keys = reinterpret_cast<uint32_t*>(dyn + sizeof(ScoreLds<D>));
  const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const Item it = item_of(p);
  if (it.b >= p.B) return;
  const int positions = tiling_of<GP>(p.G).positions, j0 = it.group * positions, here = min(p.n - j0, positions);
  const int counted = p.lens ? min(here, p.lens[it.b] - j0) : here;
  const int end = counted > 0 ? visible_blocks(p, it.b, j0 + counted - 1) : 0;
  score_blocks<D, GP>(p, it.b, it.h, j0, 0, end, wave, lane, lds, keys, p.max_blocks);
  __syncthreads();
  SearchLds* of_wave = reinterpret_cast<SearchLds*>(dyn);                // the records' place
  static_assert(sizeof(ScoreLds<D>) >= kWaves * sizeof(SearchLds));
  for (int i = wave; i < here; i += kWaves) {
    const int seen = visible_blocks(p, it.b, j0 + i);
    int32_t* out = p.out + ((long(it.b) * p.n + j0 + i) * p.Hkv + it.h) * p.N;
    const uint32_t* mine = keys + i * p.max_blocks;
    auto go = [&](auto m) {
      constexpr int M = decltype(m)::value;
      uint32_t key[M];
#pragma unroll
      for (int x = 0; x < M; ++x) {
        const int blk = x * kWave + lane;
        key[x] = blk < seen ? list_key(p, mine[blk], blk, seen) : 0u;
      }
      auto at = [&](int x) { return key[x]; };
      Range r = range_of(M, at);
      const Four n = wave_sum4<true>(Four{{r.some, r.held, 0, 0}});
      Border border{1, 0, 0};
      if (int(n.x[0]) > p.N) {
        r = Range{n.x[0], n.x[1], wave_max_u32(r.top), wave_max_u32(r.low)};
        if (int(r.held) == p.N) border.lo = kKeyHeld;
        else border = wave_search<M>(search_of(r, p.N), key, p.N, of_wave[wave], lane);
      }
      emit(M, at, border, out, 0, lane, 0, 0);
      for (int x = min(int(n.x[0]), p.N) + lane; x < p.N; x += kWave) out[x] = -1;
    };
    if (seen <= 4 * kWave) go(std::integral_constant<int, 4>{});
    else if (seen <= 9 * kWave) go(std::integral_constant<int, 9>{});
    else if (seen <= 16 * kWave) go(std::integral_constant<int, 16>{});
    else go(std::integral_constant<int, kFusedBlocks / kWave>{});
  }
}

// Longer tables: keys of chunks of blocks into the workspace ..
template <int D, int GP>
__global__ __launch_bounds__(kThreads, 4) void score_kernel(SelectArgs p) {
  __shared__ ScoreLds<D> lds;
  const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const Item it = item_of(p);
  if (it.b >= p.B) return;
  const int positions = tiling_of<GP>(p.G).positions, j0 = it.group * positions, here = min(p.n - j0, positions);
  const int counted = p.lens ? min(here, p.lens[it.b] - j0) : here, c0 = it.chunk * p.chunk;
  const int end = counted > 0 ? min(visible_blocks(p, it.b, j0 + counted - 1), c0 + p.chunk) : 0;
  if (c0 >= end) return;
  score_blocks<D, GP>(p, it.b, it.h, j0, c0, end, wave, lane, lds,
                      p.keys + ((long(it.b) * p.n + j0) * p.Hkv + it.h) * p.max_blocks + c0, long(p.Hkv) * p.max_blocks);
}

// .. and a workgroup a list, M keys to a thread (0: of tables of any size, the keys read again for each count)
template <int M, int kPickWaves>
__global__ __launch_bounds__(kPickWaves* kWave) void pick_kernel(SelectArgs p) {
  constexpr int kPickThreads = kPickWaves * kWave;
  __shared__ Four part[2][kPickWaves];
  __shared__ __attribute__((aligned(16))) uint32_t bins[3][kBins], room[kRoom];
  __shared__ int n_room;
  const long list = blockIdx.x;
  const int t = int(list / p.Hkv), b = t / p.n, j = t % p.n, lane = threadIdx.x % kWave;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const uint32_t* keys = p.keys + list * p.max_blocks;
  int m = M, first = wave * M * kWave;
  uint32_t key[M ? M : 1];
#pragma unroll
  for (int x = 0; x < M; ++x) {                  // (before it is known how many of them count)
    const int i = first + x * kWave + lane;
    key[x] = i < p.max_blocks ? keys[i] : 0u;
  }
  if (threadIdx.x == 0) n_room = 0;
  if (threadIdx.x < kRoom) room[threadIdx.x] = 0;
  for (int x = threadIdx.x; x < kBins; x += kPickThreads) bins[0][x] = 0;
  const int seen = visible_blocks(p, b, j);
#pragma unroll
  for (int x = 0; x < M; ++x) {
    const int i = first + x * kWave + lane;
    key[x] = i < seen ? list_key(p, key[x], i, seen) : 0u;
  }
  if (M == 0) {
    m = (seen + kPickThreads - 1) / kPickThreads;
    first = wave * m * kWave;
  }
  auto at = [&](int x) __attribute__((always_inline)) {
    if (M) return key[M ? x : 0];
    const int i = first + x * kWave + lane;
    return i < seen ? list_key(p, keys[i], i, seen) : 0u;
  };
  int turn = 0;                                  // two sets of numbers in turn: one barrier an exchange
  auto exchange = [&](const Four& c) {
    turn ^= 1;
    if (lane == 0) part[turn][wave] = c;
    __syncthreads();
  };
  Range r = range_of(m, at);
  const Four n = wave_sum4<M != 0>(Four{{r.some, r.held, 0, 0}});
  exchange(Four{{n.x[0], n.x[1], wave_max_u32(r.top), wave_max_u32(r.low)}});
  r = Range{0, 0, 0, 0};
#pragma unroll
  for (int w = 0; w < kPickWaves; ++w) {
    const Four x = part[turn][w];
    r = Range{r.some + x.x[0], r.held + x.x[1], max(r.top, x.x[2]), max(r.low, x.x[3])};
  }
  Border border{1, 0, 0};
  if (int(r.some) > p.N) {
    Search s = search_of(r, p.N);
    if (int(r.held) == p.N) {
      border.lo = kKeyHeld;
    } else {
      for (int now = 0; !s.done() && s.c_lo - s.c_hi > kRoom;) {         // three sets of bins in turn: one barrier a step
        const int next = now == 2 ? 0 : now + 1, shift = s.shift();
        for (int x = threadIdx.x; x < kBins; x += kPickThreads) bins[next][x] = 0;
#pragma unroll
        for (int x = 0; x < m; ++x) s.add(bins[now], shift, at(x));
        __syncthreads();
        s.narrow(bins[now], shift, p.N, lane);
        now = next;
      }
      if (!s.done()) {
        int mine = 0;
#pragma unroll
        for (int x = 0; x < m; ++x) {
          const uint32_t k = at(x);
          mine += k >= s.lo && k < s.hi;
        }
        const int upto = wave_scan_dpp(mine);
        int to = 0;                              // (the wavefronts in any order: the keys are counted only)
        if (lane == kWave - 1 && upto) to = atomicAdd(&n_room, upto);
        to = __builtin_amdgcn_readlane(to, kWave - 1) + upto - mine;
#pragma unroll
        for (int x = 0; x < m; ++x) {
          const uint32_t k = at(x);
          if (k >= s.lo && k < s.hi) room[to++] = k;
        }
        __syncthreads();
        border = rank_room(s, room, p.N, lane);
      } else {
        border = s.border(p.N);
      }
    }
  }
  Four c{{0, 0, 0, 0}};
#pragma unroll
  for (int x = 0; x < m; ++x) {
    const uint32_t k = at(x);
    c.x[0] += k >= border.lo;
    c.x[1] += k == border.equal_key;
  }
  c = wave_sum4<M != 0>(c);
  exchange(c);
  int in = 0, equal = 0;                         // in front of the wavefront
#pragma unroll
  for (int w = 0; w < kPickWaves; ++w)
    if (w < wave) { in += int(part[turn][w].x[0]); equal += int(part[turn][w].x[1]); }
  int32_t* out = p.out + list * p.N;
  emit(m, at, border, out, first, lane, in, equal);
  for (int x = min(int(r.some), p.N) + int(threadIdx.x); x < p.N; x += kPickThreads) out[x] = -1;
}

constexpr unsigned kManyLists = 256;
int padded_rows(int G) { return G <= 4 ? 4 : G <= 8 ? 8 : 16; }
int score_positions(int G) { return G > 16 ? 1 : 64 / padded_rows(G); }

// LDS of a call in one launch; 0 where it takes two. One launch is the faster one where it makes a workgroup for every CU
// (64 sequences x 1 position, 4 kv heads x 128: 600 blocks 15.2 us, two launches 19.2; 1300 blocks 26.0 and 28.5; 128 x 5:
// 25.9 and 37.2, 44.9 and 56.0), and else for tables so short that one workgroup is done with them before a second launch
// would begin (1 x 1: 300 blocks 8.1 and 9.3, 600 blocks 10.9 and 9.7; 16 x 5: 400 blocks 11.3 and 13.2, 600 blocks 14.1
// and 13.6).
size_t fused_lds(int B, int n, int G, int Hkv, int D, int max_blocks) {
  const long groups = long(B) * Hkv * ((long(n) + score_positions(G) - 1) / score_positions(G));
  if (max_blocks > (groups >= 256 ? kFusedBlocks : 448)) return 0;
  const size_t fixed = D == 128 ? sizeof(ScoreLds<128>) : sizeof(ScoreLds<64>);
  const size_t bytes = fixed + size_t(std::min(n, score_positions(G))) * max_blocks * sizeof(uint32_t);
  return bytes <= kFusedLds ? bytes : 0;
}

// Blocks of a workgroup of a call in two launches: as many rounds of 256 as leave workgroups enough (x 5 positions, 4 kv
// heads; 1, 2, 3, 4 rounds: 16 sequences at 32768-65536 26.5 us, 24.9, 26.9, 29.7; 2, 4, 8: 32, 4000 blocks 41.5, 38.9, 39.7;
// 128, 4000 blocks 164, 157, 157; 32, 2200 blocks 31.9, 32.4, 35.4)
int score_chunk(int B, int n, int G, int Hkv, int max_blocks) {
  const long groups = long(B) * Hkv * ((long(n) + score_positions(G) - 1) / score_positions(G));
  constexpr int round = 32 * kWaves;
  auto made = [&](int rounds) { return groups * ((long(max_blocks) + rounds * round - 1) / (rounds * round)); };
  return made(4) >= 512 ? 4 * round : made(2) >= 256 ? 2 * round : round;
}

}  // namespace

double select_groups(int B, int n, int Hq, int Hkv, int D, int max_blocks) {
  const int G = Hq / Hkv;
  const double chunks = fused_lds(B, n, G, Hkv, D, max_blocks) ? 1 : std::ceil(max_blocks / double(score_chunk(B, n, G, Hkv, max_blocks)));
  return 2 * std::max((double(B) + 7) * std::ceil(n / double(score_positions(G))) * Hkv * chunks, double(B) * n * Hkv);
}

size_t select_ws_bytes(int B, int n, int Hq, int Hkv, int D, int max_blocks) {
  if (fused_lds(B, n, Hq / Hkv, Hkv, D, max_blocks)) return 0;
  return size_t(B) * n * Hkv * max_blocks * sizeof(uint32_t) + 256;
}

hipError_t launch_select_blocks(const void* q, const void* bounds, const int32_t* bt, const int32_t* ctx,
                                const int32_t* lens, int B, int n, int Hq, int Hkv, int D, int max_blocks,
                                int num_blocks, int N, int n_first, int n_last, molt_dtype dt, int32_t* out, void* ws,
                                size_t ws_bytes, hipStream_t s) {
  SelectArgs p{};
  p.q = q; p.bounds = static_cast<const uint8_t*>(bounds); p.bt = bt; p.ctx = ctx; p.lens = lens;
  p.B = B; p.n = n; p.Hq = Hq; p.Hkv = Hkv; p.G = Hq / Hkv; p.N = N; p.n_first = n_first; p.n_last = n_last;
  p.max_blocks = max_blocks; p.num_blocks = num_blocks; p.out = out;
  p.f32 = dt == MOLT_F32;
  const size_t lds = fused_lds(B, n, p.G, Hkv, D, max_blocks);
  const bool fused = lds != 0;
  const int positions = score_positions(p.G);
  p.pos_groups = int((long(n) + positions - 1) / positions);
  p.chunks = 1;
  p.block_bytes = uint32_t(Hkv) * (2 * D + 16);
  p.by_xcd = B % 8 == 0 || B >= 12;
  if (!fused) {
    p.chunk = score_chunk(B, n, p.G, Hkv, max_blocks);
    p.chunks = (max_blocks + p.chunk - 1) / p.chunk;
    Carver c(ws, ws_bytes);
    p.keys = c.take<uint32_t>(size_t(B) * n * Hkv * max_blocks);
  }
  const long inner = long(p.pos_groups) * Hkv * p.chunks;
  const unsigned grid = unsigned((p.by_xcd ? (long(B) + 7) / 8 * 8 : long(B)) * inner);
  auto go = [&](auto d, auto gp) {
    constexpr int DD = decltype(d)::value, GP = decltype(gp)::value;
    if (fused) select_kernel<DD, GP><<<grid, kThreads, lds, s>>>(p);
    else score_kernel<DD, GP><<<grid, kThreads, 0, s>>>(p);
  };
  auto by_rows = [&](auto d) {
    const int gp = padded_rows(p.G);
    if (gp == 4) go(d, std::integral_constant<int, 4>{});
    else if (gp == 8) go(d, std::integral_constant<int, 8>{});
    else go(d, std::integral_constant<int, 16>{});
  };
  if (D == 128) by_rows(std::integral_constant<int, 128>{});
  else by_rows(std::integral_constant<int, 64>{});
  if (hipError_t e = hipGetLastError()) return e;
  if (fused) return hipSuccess;
  const unsigned lists = unsigned(long(B) * n * Hkv);
  auto pick = [&](auto m, auto waves) {
    constexpr int M = decltype(m)::value, W = decltype(waves)::value;
    pick_kernel<M, W><<<lists, W * kWave, 0, s>>>(p);
  };
  // many lists: few wavefronts each, which wait less for each other; few: as many as shorten the list's own time
  // (x 5 positions x 4 kv heads, 2200 blocks: 128 sequences 99.9 us, with 8 wavefronts 105, 16 sequences 23.1 and 22.8,
  // 8 sequences 15.6 and 14.3)
  if (lists >= kManyLists && max_blocks <= 16 * 2 * kWave) pick(std::integral_constant<int, 16>{}, std::integral_constant<int, 2>{});
  else if (lists >= kManyLists && max_blocks <= 16 * 4 * kWave) pick(std::integral_constant<int, 16>{}, std::integral_constant<int, 4>{});
  else if (max_blocks <= 4 * 8 * kWave) pick(std::integral_constant<int, 4>{}, std::integral_constant<int, 8>{});
  else if (max_blocks <= 9 * 8 * kWave) pick(std::integral_constant<int, 9>{}, std::integral_constant<int, 8>{});
  else if (max_blocks <= 16 * 8 * kWave) pick(std::integral_constant<int, 16>{}, std::integral_constant<int, 8>{});
  else pick(std::integral_constant<int, 0>{}, std::integral_constant<int, 8>{});
  return hipGetLastError();
}

}  // namespace molt
