// The paged cache's upkeep on the GPU: block tables that follow the lengths, rows written by slot, the bounds of
// each block's keys.
#include <type_traits>

#include "bounds_format.h"
#include "internal.h"

namespace molt {
namespace {

constexpr int kThreads = 256;

// ---------------------------------------------------------------- tables and slots

constexpr int kPlanThreads = 1024;
constexpr int kPlanWaves = kPlanThreads / kWave;

// What a call does with sequence b's row of the table: entries have .. have + take - 1 come from the ring's places
// first .. behind its head, entries keep .. have - 1 go to places back .. of it (-1: none do), rows 0 .. placed - 1 get
// slots.
struct PlanRow { int have, take, first, keep, back, placed, ctx; };

struct PlanArgs {
  int32_t* bt; int32_t* n_blocks; const int32_t* ctx; const int32_t* n_new; int32_t* pool; const int32_t* shared;
  int B, n, max_blocks, num_blocks;
  int32_t* slots; int32_t* placed;
  PlanRow* rows;                                 // [B + 1]; the last one's `first` is the ring's head before the call
};

MOLT_DEV int ring_wrap(long at, int cap) { return int(at >= cap ? at - cap : at); }   // at < 2 cap

// Row j of sequence b: its slot, and the table entry that it is the first to use. Entries of the pool are read from the
// ring itself: nothing waits for the table.
MOLT_DEV void plan_slot(const PlanArgs& p, const PlanRow& r, int b, int j, int head) {
  const int cap = p.num_blocks;
  const int32_t* ring = p.pool + 2;
  int32_t* row = p.bt + long(b) * p.max_blocks;
  int slot = -1;
  if (j < r.placed) {
    const int pos = r.ctx + j, i = pos / 16;       // i < have + take
    int id;
    if (i >= r.have) {
      id = ring[ring_wrap(long(head) + r.first + (i - r.have), cap)];
      if (j == 0 || pos % 16 == 0) row[i] = id;
    } else {
      id = row[i];
    }
    if (id >= 0 && id < cap) slot = id * 16 + pos % 16;
    if (j == 0)                                  // a table that lacks blocks of the cached tokens
      for (int k = r.have; k < i; ++k) row[k] = ring[ring_wrap(long(head) + r.first + (k - r.have), cap)];
  }
  p.slots[long(b) * p.n + j] = slot;
}

// a finished sequence's entries into the ring, `threads` at a time
MOLT_DEV void plan_return(const PlanArgs& p, const PlanRow& r, int b, int thread, int threads) {
  const int32_t* row = p.bt + long(b) * p.max_blocks;
  const int m = r.have - r.keep;
  int i = thread;
  for (; i + 3l * threads < m; i += 4 * threads) {
    int id[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) id[u] = row[r.keep + i + u * threads];
#pragma unroll
    for (int u = 0; u < 4; ++u) p.pool[2 + ring_wrap(long(r.back) + i + u * threads, p.num_blocks)] = id[u];
  }
  for (; i < m; i += threads) p.pool[2 + ring_wrap(long(r.back) + i, p.num_blocks)] = row[r.keep + i];
}

// Inclusive sums over the workgroup's threads of v and w in [0, 2^31), in 64 bits: their halves of 16 bits apart on DPP
struct Pair { long a, b; };
MOLT_DEV Pair plan_scan(int v, int w, Pair* red, Pair& total) {
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  const Pair s{(long(wave_scan_dpp(v >> 16)) << 16) + wave_scan_dpp(v & 0xffff),
               (long(wave_scan_dpp(w >> 16)) << 16) + wave_scan_dpp(w & 0xffff)};
  __syncthreads();
  if (lane == kWave - 1) red[wave] = s;
  __syncthreads();
  Pair before{0, 0}, all{0, 0};
#pragma unroll
  for (int i = 0; i < kPlanWaves; ++i) {
    const Pair x = red[i];
    if (i < wave) { before.a += x.a; before.b += x.b; }
    all.a += x.a;
    all.b += x.b;
  }
  total = all;
  return Pair{s.a + before.a, s.b + before.b};
}

// One workgroup. Who gets what is a matter of prefix sums of the rows' demands, in the rows' order: nothing depends on
// timing. Taken places [head, head + taken) and returned ones behind head + count are apart, so both go on at once.
// WHOLE: the slots and the entries too (up to kPlanThreads sequences), else plan_rows_kernel does them.
// Its time is that of a chain of loads, two scans and stores on one CU: 128 sequences x 5 rows 5.6 us; 300 x 4001 rows
// (5 MB) 5.3 us and 4.7 us for plan_rows_kernel.
template <bool WHOLE>
__global__ __launch_bounds__(kPlanThreads) void plan_kernel(PlanArgs p) {
  __shared__ Pair red[kPlanWaves];
  __shared__ unsigned long long ends[2];         // places taken and returned, as far as the pool goes
  __shared__ PlanRow held[WHOLE ? kPlanThreads : 1];
  const int cap = p.num_blocks;
  const int head = int(uint32_t(p.pool[0]) % uint32_t(cap)), count = min(max(p.pool[1], 0), cap);
  if (threadIdx.x < 2) ends[threadIdx.x] = 0;
  long demanded = 0, given = 0;                  // of the rows before
  for (int b0 = 0; b0 < p.B; b0 += kPlanThreads) {
    const int b = b0 + int(threadIdx.x);
    PlanRow r{0, 0, 0, 0, -1, 0, 0};
    int want = 0, give = 0;
    bool fits = false, done = false;
    if (b < p.B) {
      const int ctx = p.ctx[b], m = p.n_new[b];
      r.have = p.n_blocks[b];
      r.ctx = ctx;
      const bool sound = r.have >= 0 && r.have <= p.max_blocks;
      const long end = long(ctx) + m;
      done = sound && m < 0;
      fits = sound && m >= 0 && m <= p.n && ctx >= 0 && end <= 16l * p.max_blocks;
      if (fits && m > 0) want = max(0, int((end + 15) / 16) - r.have);
      if (done) {
        r.keep = p.shared ? max(p.shared[b], 0) : 0;
        give = max(0, r.have - r.keep);
      }
      if (fits) r.placed = m;
    }
    Pair all;
    const Pair sums = plan_scan(want, give, red, all);
    const long upto = demanded + sums.a, gave = given + sums.b;
    if (want && upto <= count) {
      r.take = want;
      r.first = int(upto - want);
      atomicMax(&ends[0], (unsigned long long)upto);
    } else if (want) {
      r.placed = 0;                              // the pool does not reach so far
    }
    if (give && gave <= cap - count) {           // (a ring that would run over holds ids twice: they are dropped)
      r.back = int((long(head) + count + gave - give) % cap);
      atomicMax(&ends[1], (unsigned long long)gave);
    }
    if (b < p.B) {
      p.placed[b] = r.placed;
      if (done) p.n_blocks[b] = 0;
      else if (r.take) p.n_blocks[b] = r.have + r.take;
      if (WHOLE) held[threadIdx.x] = r;
      else p.rows[b] = r;
    }
    demanded += all.a;
    given += all.b;
  }
  __syncthreads();
  if (threadIdx.x == 0) {
    p.pool[0] = int((head + long(ends[0])) % cap);
    p.pool[1] = count - int(ends[0]) + int(ends[1]);
    if (!WHOLE) p.rows[p.B].first = head;
  }
  if (!WHOLE) return;
  for (int at = threadIdx.x; at < p.B * p.n; at += kPlanThreads) plan_slot(p, held[at / p.n], at / p.n, at % p.n, head);
  for (int b = threadIdx.x / kWave; b < p.B; b += kPlanWaves)
    if (held[b].back >= 0) plan_return(p, held[b], b, threadIdx.x % kWave, kWave);
}

// after plan_kernel<false>: a thread per slot, then a workgroup per sequence for what it gives back
__global__ __launch_bounds__(kThreads) void plan_rows_kernel(PlanArgs p, uint32_t slot_groups) {
  if (blockIdx.x < slot_groups) {
    const uint32_t at = blockIdx.x * kThreads + threadIdx.x;
    const uint32_t b = at / uint32_t(p.n);
    if (b < uint32_t(p.B)) plan_slot(p, p.rows[b], int(b), int(at - b * uint32_t(p.n)), p.rows[p.B].first);
    return;
  }
  const int b = int(blockIdx.x - slot_groups);
  const PlanRow r = p.rows[b];
  if (r.back >= 0) plan_return(p, r, b, threadIdx.x, kThreads);
}

// One launch where its threads have few slots each: 512 sequences x 5 rows 6.7 us, two launches 8.8; 1024 x 1 8.8 and 8.6;
// 1024 x 5 10.3 and 8.7; 64 x 257 9.6 and 8.7
bool plan_whole(int B, int n) { return B <= kPlanThreads && long(B) * n <= 4 * kPlanThreads; }

// ---------------------------------------------------------------- rows by slot

constexpr int kWriteRows = 16, kFewRows = 4;
// Runs of a tile from which its rows go one by one (8000 rows in runs of 1 33.8 us, run by run 54.7)
constexpr int kManyRuns = 5;
// Rows x 128 dims up to which rows count as few: 1024 rows of 4 kv heads x 128. Calls back to back, bf16: 640 rows in
// runs of 5 4.7 us, by runs 9.7; 2048 rows in runs of 5 8.9 and 11.4, of 1000 8.4 and 6.0; 4000 rows 14.4 and 13.6, 13.9
// and 6.9. The host does not know the runs. From 2048 rows on, one kernel for all would cost prompts as much as it saves
// runs of 5, or more, and calls of so many rows are prompts': a verify step of 5 positions would be of 400 sequences.
constexpr long kFewUnits = 4096;

// two elements of a row at any element alignment, as the bits that the cache holds
typedef uint32_t UnalignedU1 __attribute__((aligned(2)));
typedef uint32_t u32x2_t __attribute__((ext_vector_type(2)));
typedef u32x2_t UnalignedU2 __attribute__((aligned(4)));
typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));

// Dims d and d + 1 of a row of k and v at a slot of the cache
template <int D, typename T, typename Two>
MOLT_DEV void store_row(T* kc, T* vc, int slot, int Hkv, int h, int d, Two x, Two y) {
  const long rec = (long(slot / 16) * Hkv + h) * 16 * D;
  *reinterpret_cast<Two*>(kc + rec + slot % 16 * D + d) = x;
  T* out = vc + rec + d * 16 + slot % 16;
  if constexpr (sizeof(T) == 2) {
    out[0] = T(y);
    out[16] = T(y >> 16);
  } else {
    out[0] = __uint_as_float(y[0]);
    out[16] = __uint_as_float(y[1]);
  }
}

// Wavefront = R rows of k and v and 128 dims: a head of 128 dims or two of 64; lane = two dims. The rows fall into
// runs of consecutive slots of one block; a wavefront writes the runs that begin among its rows, up to their ends, one
// after the other. A run that fills its block's 16 slots leaves V, whose tokens are contiguous, in whole 16-byte stores;
// other runs leave it in stores of 4 bytes where both tokens of a pair are there. Bound by memory where runs are long: 24000
// rows of 4 heads x 128 in bf16 (98 MB in and out) 24 us, 4.1 TB/s. Single rows are bound by V's stores of one element, each
// in a sector of its own (16000 rows 97 us).
template <int D, typename T>
__global__ __launch_bounds__(kThreads) void kv_write_kernel(const T* __restrict__ k, long k_stride,
                                                            const T* __restrict__ v, long v_stride,
                                                            const int32_t* __restrict__ slots, int rows, int Hkv,
                                                            int num_blocks, T* __restrict__ kc, T* __restrict__ vc) {
  constexpr int HPW = 128 / D, R = kWriteRows;
  const int heads = (Hkv + HPW - 1) / HPW;
  const uint32_t item = blockIdx.x * (kThreads / kWave) + __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const uint32_t tile = item / uint32_t(heads);
  const int r0 = int(tile) * R, lane = threadIdx.x % kWave;
  if (r0 >= rows) return;
  const int h = int(item - tile * heads) * HPW + lane / (D / 2), d = lane % (D / 2) * 2;
  // lane l: the slot of row r0 - 1 + l, up to the last row of a run that begins at r0 + R - 1
  const int row = r0 - 1 + lane;
  const int slot = row >= 0 && row < rows && lane <= R + 16 ? slots[row] : -1;
  const bool good = slot >= 0 && slot / 16 < num_blocks;
  // (where it follows on from row r0 - 1 within a block, row r0 belongs to a run of the tile before)
  const int before = __shfl_up(slot, 1);
  const bool starts = good && lane > 0 && (slot % 16 == 0 || before != slot - 1);
  const uint32_t begin = uint32_t(__ballot(starts) >> 1), live = uint32_t(__ballot(good) >> 1);   // bit i: row r0 + i
  const bool there = h < Hkv;
  uint32_t left = begin & ((1u << R) - 1);
  if (__builtin_popcount(left) >= kManyRuns) {   // all rows between the first run's and the last run's beginning
    const int i0 = __builtin_ctz(left), i1 = 31 - __builtin_clz(left);
    if (there) {
      typedef std::conditional_t<sizeof(T) == 2, uint32_t, u32x2_t> Two;
      typedef std::conditional_t<sizeof(T) == 2, UnalignedU1, UnalignedU2> UnalignedTwo;
      Two x[R], y[R];
#pragma unroll
      for (int i = 0; i < R; ++i) {
        const long r = r0 + min(max(i, i0), i1);
        x[i] = *reinterpret_cast<const UnalignedTwo*>(k + r * k_stride + h * D + d);
        y[i] = *reinterpret_cast<const UnalignedTwo*>(v + r * v_stride + h * D + d);
      }
#pragma unroll
      for (int i = 0; i < R; ++i)
        if (i >= i0 && i < i1 && live >> i & 1)
          store_row<D, T>(kc, vc, __builtin_amdgcn_readlane(slot, i + 1), Hkv, h, d, x[i], y[i]);
    }
    left = 1u << i1;
  }
  for (; left; left &= left - 1) {
    const int i = __builtin_ctz(left);
    const uint32_t stop = (begin | ~live) >> i >> 1;                     // what ends the run
    const int len = min(stop ? __builtin_ctz(stop) + 1 : 32, 16);
    const int s = __builtin_amdgcn_readlane(slot, i + 1), first = s % 16;
    const long rec = (long(s / 16) * Hkv + h) * 16 * D;
    if (!there) continue;
    if constexpr (sizeof(T) == 2) {
      uint32_t x[16], y[16];
#pragma unroll
      for (int t = 0; t < 16; ++t) {
        const long r = r0 + i + min(max(t - first, 0), len - 1);         // (some row of the run where t has none)
        x[t] = *reinterpret_cast<const UnalignedU1*>(k + r * k_stride + h * D + d);
        y[t] = *reinterpret_cast<const UnalignedU1*>(v + r * v_stride + h * D + d);
      }
#pragma unroll
      for (int t = 0; t < 16; ++t)
        if (t >= first && t < first + len) *reinterpret_cast<uint32_t*>(kc + rec + t * D + d) = x[t];
      T* out = vc + rec + d * 16;                                        // dims d and d + 1: 32 elements
      uint32_t lo[8], hi[8];
#pragma unroll
      for (int t = 0; t < 8; ++t) {
        lo[t] = (y[2 * t] & 0xffffu) | y[2 * t + 1] << 16;
        hi[t] = y[2 * t] >> 16 | (y[2 * t + 1] & 0xffff0000u);
      }
      if (len == 16) {
        u32x4_t* o = reinterpret_cast<u32x4_t*>(out);
        o[0] = u32x4_t{lo[0], lo[1], lo[2], lo[3]};
        o[1] = u32x4_t{lo[4], lo[5], lo[6], lo[7]};
        o[2] = u32x4_t{hi[0], hi[1], hi[2], hi[3]};
        o[3] = u32x4_t{hi[4], hi[5], hi[6], hi[7]};
      } else {
#pragma unroll
        for (int t = 0; t < 8; ++t) {
          const bool a = 2 * t >= first && 2 * t < first + len, b = 2 * t + 1 >= first && 2 * t + 1 < first + len;
          if (a && b) {
            *reinterpret_cast<uint32_t*>(out + 2 * t) = lo[t];
            *reinterpret_cast<uint32_t*>(out + 16 + 2 * t) = hi[t];
          } else if (a) {
            out[2 * t] = T(lo[t]);
            out[16 + 2 * t] = T(hi[t]);
          } else if (b) {
            out[2 * t + 1] = T(lo[t] >> 16);
            out[16 + 2 * t + 1] = T(hi[t] >> 16);
          }
        }
      }
    } else {
      u32x2_t x[16], y[16];
#pragma unroll
      for (int t = 0; t < 16; ++t) {
        const long r = r0 + i + min(max(t - first, 0), len - 1);         // (some row of the run where t has none)
        x[t] = *reinterpret_cast<const UnalignedU2*>(k + r * k_stride + h * D + d);
        y[t] = *reinterpret_cast<const UnalignedU2*>(v + r * v_stride + h * D + d);
      }
#pragma unroll
      for (int t = 0; t < 16; ++t)
        if (t >= first && t < first + len) *reinterpret_cast<u32x2_t*>(kc + rec + t * D + d) = x[t];
      uint32_t* out = reinterpret_cast<uint32_t*>(vc) + rec + d * 16;
      if (len == 16) {
        u32x4_t* o = reinterpret_cast<u32x4_t*>(out);
#pragma unroll
        for (int c = 0; c < 2; ++c)
#pragma unroll
          for (int t = 0; t < 4; ++t)
            o[4 * c + t] = u32x4_t{y[4 * t][c], y[4 * t + 1][c], y[4 * t + 2][c], y[4 * t + 3][c]};
      } else {
#pragma unroll
        for (int t = 0; t < 16; ++t)
          if (t >= first && t < first + len) { out[t] = y[t][0]; out[16 + t] = y[t][1]; }
      }
    }
  }
}

// The same for few rows, where the time is that of the loads in a row: wavefront = 4 rows, read before it is known where
// they go; V's tokens are stored one by one. 640 rows of 4 heads x 128 in bf16, runs of 5: 5.2 us in a kernel trace, 4.7 a call
// back to back, the loads' and the launch's latency.
template <int D, typename T>
__global__ __launch_bounds__(kThreads) void kv_write_few_kernel(const T* __restrict__ k, long k_stride,
                                                                const T* __restrict__ v, long v_stride,
                                                                const int32_t* __restrict__ slots, int rows, int Hkv,
                                                                int num_blocks, T* __restrict__ kc, T* __restrict__ vc) {
  constexpr int HPW = 128 / D, R = kFewRows;
  typedef std::conditional_t<sizeof(T) == 2, uint32_t, u32x2_t> Two;
  typedef std::conditional_t<sizeof(T) == 2, UnalignedU1, UnalignedU2> UnalignedTwo;
  const int heads = (Hkv + HPW - 1) / HPW;
  const uint32_t item = blockIdx.x * (kThreads / kWave) + __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const uint32_t tile = item / uint32_t(heads);
  const int r0 = int(tile) * R, lane = threadIdx.x % kWave;
  const int h = int(item - tile * heads) * HPW + lane / (D / 2), d = lane % (D / 2) * 2;
  if (r0 >= rows || h >= Hkv) return;
  int slot[R];
  Two x[R], y[R];
#pragma unroll
  for (int i = 0; i < R; ++i) {
    const long r = min(r0 + i, rows - 1);
    slot[i] = r0 + i < rows ? slots[r] : -1;
    x[i] = *reinterpret_cast<const UnalignedTwo*>(k + r * k_stride + h * D + d);
    y[i] = *reinterpret_cast<const UnalignedTwo*>(v + r * v_stride + h * D + d);
  }
#pragma unroll
  for (int i = 0; i < R; ++i) {
    if (slot[i] >= 0 && slot[i] / 16 < num_blocks) store_row<D, T>(kc, vc, slot[i], Hkv, h, d, x[i], y[i]);
  }
}

// ---------------------------------------------------------------- bounds of the keys

MOLT_DEV void load_octet(const uint16_t* p, float (&x)[8]) {
  const u32x4_t w = *reinterpret_cast<const u32x4_t*>(p);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[2 * i] = __uint_as_float(w[i] << 16);
    x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
  }
}
MOLT_DEV void load_octet(const float* p, float (&x)[8]) {
  const floatx4_t a = *reinterpret_cast<const floatx4_t*>(p), b = *reinterpret_cast<const floatx4_t*>(p + 4);
#pragma unroll
  for (int i = 0; i < 4; ++i) { x[i] = a[i]; x[4 + i] = b[i]; }
}

// Wavefront = one block of a sequence and one kv head: lane = an octet of dims of every (512 / D)-th token. The
// block is read whole, cached tokens with it, so that what a record holds never depends on how it came about.
// Bound by latency, a block's id before the block, and then by memory: 128 x 5 rows 3.6 us, 24000 rows (27 MB) 8.8 us, 3.0
// TB/s; two blocks a wavefront, in registers at once, took 14.4 in place of 10.6.
template <int D, typename T>
__global__ __launch_bounds__(kThreads) void bounds_update_kernel(const T* __restrict__ kc, uint8_t* __restrict__ bounds,
                                                                 const int32_t* __restrict__ bt,
                                                                 const int32_t* __restrict__ starts,
                                                                 const int32_t* __restrict__ lens, int B, int n, int nblk,
                                                                 int Hkv, int max_blocks, int num_blocks) {
  typedef BoundsRecord<D> Rec;
  constexpr int O = D / 8, TPI = kWave / O, NI = 16 / TPI;              // octets, tokens of a load, loads
  const uint32_t item = blockIdx.x * (kThreads / kWave) + __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const uint32_t rest = item / uint32_t(Hkv), b = rest / uint32_t(nblk);
  const int h = int(item - rest * Hkv);
  if (b >= uint32_t(B)) return;
  const int start = starts[b], m = lens ? min(max(lens[b], 0), n) : n;
  const long blk = (long(start) >> 4) + long(rest - b * nblk), end = long(start) + m;
  if (m == 0 || blk < 0 || blk >= max_blocks || 16 * blk >= end) return;
  const int id = bt[long(b) * max_blocks + blk];
  if (id < 0 || id >= num_blocks) return;
  const int seen = int(min(16l, end - 16 * blk));                        // tokens 0 .. seen - 1 of the block
  const int lane = threadIdx.x % kWave, oct = lane % O;
  const T* src = kc + (long(id) * Hkv + h) * 16 * D;
  float x[NI][8];
#pragma unroll
  for (int i = 0; i < NI; ++i) load_octet(src + (i * TPI + lane / O) * D + oct * 8, x[i]);
  float hi[8], lo[8], finite = 0.f;              // lo: of the negated keys; finite: 0 as long as all keys are
#pragma unroll
  for (int e = 0; e < 8; ++e) hi[e] = lo[e] = -__builtin_inff();
#pragma unroll
  for (int i = 0; i < NI; ++i)
    if (i * TPI + lane / O < seen) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        hi[e] = fmaxf(hi[e], x[i][e]);
        lo[e] = fmaxf(lo[e], -x[i][e]);
        finite = __builtin_fmaf(x[i][e], 0.f, finite);
      }
    }
  if (O == 8) {                                  // lanes l, l ^ 8: a rotation of the 16-lane row
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      hi[e] = fmaxf(hi[e], __uint_as_float(dpp_u32<0x128, 0xF>(__float_as_uint(hi[e]), 0u)));
      lo[e] = fmaxf(lo[e], __uint_as_float(dpp_u32<0x128, 0xF>(__float_as_uint(lo[e]), 0u)));
    }
  }
  // Over the 16-lane rows, each of which ends with its share: rows 0 and 1 the octet's first and second 4 of hi, rows 2
  // and 3 those of lo. A row swap brings two values' partners together, so that one maximum serves both.
  float w[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const auto u = __builtin_amdgcn_permlane16_swap(__float_as_uint(hi[e]), __float_as_uint(hi[e + 4]), false, false);
    const auto v = __builtin_amdgcn_permlane16_swap(__float_as_uint(lo[e]), __float_as_uint(lo[e + 4]), false, false);
    const float hh = fmaxf(__uint_as_float(u[0]), __uint_as_float(u[1]));
    const float ll = fmaxf(__uint_as_float(v[0]), __uint_as_float(v[1]));
    const auto y = __builtin_amdgcn_permlane32_swap(__float_as_uint(hh), __float_as_uint(ll), false, false);
    w[e] = fmaxf(__uint_as_float(y[0]), __uint_as_float(y[1]));
  }
  const bool bad = __any(finite != 0.f);         // (NaN is)
  const float a = wave_max_dpp(fmaxf(fmaxf(fabsf(w[0]), fabsf(w[1])), fmaxf(fabsf(w[2]), fabsf(w[3]))));
  const int e = bad ? kBoundsNotFinite : bounds_exponent(__float_as_uint(a));
  const float r = bad ? 0.f : pow2(-e);
  const bool low = lane >= 32;
  int c[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int up = bad ? 0 : int(__builtin_ceilf(w[i] * r));
    c[i] = low ? -up : up;                       // floor(x) = -ceil(-x)
  }
  uint8_t* rec = bounds + (long(id) * Hkv + h) * Rec::kBytes;
  if (O == 16 || lane % 16 < O)
    *reinterpret_cast<uint32_t*>(rec + (low ? D : 0) + oct * 8 + lane / 16 % 2 * 4) = pack_codes(c[0], c[1], c[2], c[3]);
  if (lane == kWave - 1) *reinterpret_cast<u32x4_t*>(rec + Rec::kExponent) = u32x4_t{uint32_t(e) & 0xffu, 0, 0, 0};
}

// thread = four dims of a record; 512 records of 128 dims 2.7 us, 6040 4.6: a launch's time
template <int D>
__global__ __launch_bounds__(kThreads) void bounds_read_kernel(const uint8_t* __restrict__ bounds,
                                                               const int32_t* __restrict__ ids, long records, int Hkv,
                                                               int num_blocks, float* __restrict__ hi,
                                                               float* __restrict__ lo) {
  typedef BoundsRecord<D> Rec;
  const long at = (long(blockIdx.x) * kThreads + threadIdx.x) / (D / 4);
  const int d = threadIdx.x % (D / 4) * 4;
  if (at >= records) return;
  const int id = ids[at / Hkv];
  const float nan = __uint_as_float(0x7fc00000u), inf = __builtin_inff();
  floatx4_t a{nan, nan, nan, nan}, b = a;
  if (id >= 0 && id < num_blocks) {
    const uint8_t* rec = bounds + (long(id) * Hkv + at % Hkv) * Rec::kBytes;
    const int e = int(int8_t(rec[Rec::kExponent]));
    const uint32_t x = *reinterpret_cast<const uint32_t*>(rec + d), y = *reinterpret_cast<const uint32_t*>(rec + D + d);
    const float unit = pow2(min(max(e, kBoundsMinExponent), kBoundsMaxExponent));   // (codes from 64 on pass f32 at 2^122)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      a[i] = e == kBoundsNotFinite ? inf : float(int8_t(x >> 8 * i)) * unit;
      b[i] = e == kBoundsNotFinite ? -inf : float(int8_t(y >> 8 * i)) * unit;
    }
  }
  *reinterpret_cast<floatx4_t*>(hi + at * D + d) = a;
  *reinterpret_cast<floatx4_t*>(lo + at * D + d) = b;
}

}  // namespace

size_t plan_ws_bytes(int B, int n) { return plan_whole(B, n) ? 0 : (size_t(B) + 1) * sizeof(PlanRow) + 256; }

hipError_t launch_plan_blocks(int32_t* bt, int32_t* n_blocks, const int32_t* ctx, const int32_t* n_new, int32_t* pool,
                              const int32_t* shared, int B, int n, int max_blocks, int num_blocks, int32_t* slots,
                              int32_t* placed, void* ws, size_t ws_bytes, hipStream_t s) {
  PlanArgs p{bt, n_blocks, ctx, n_new, pool, shared, B, n, max_blocks, num_blocks, slots, placed, nullptr};
  if (plan_whole(B, n)) {
    plan_kernel<true><<<1, kPlanThreads, 0, s>>>(p);
    return hipGetLastError();
  }
  Carver c(ws, ws_bytes);
  p.rows = c.take<PlanRow>(size_t(B) + 1);
  plan_kernel<false><<<1, kPlanThreads, 0, s>>>(p);
  const uint32_t slot_groups = uint32_t((long(B) * n + kThreads - 1) / kThreads);
  plan_rows_kernel<<<slot_groups + uint32_t(B), kThreads, 0, s>>>(p, slot_groups);
  return hipGetLastError();
}

hipError_t launch_kv_write(const void* k, long k_stride, const void* v, long v_stride, const int32_t* slots, int rows,
                           int Hkv, int D, int num_blocks, molt_dtype dt, void* kc, void* vc, hipStream_t s) {
  const long units = (Hkv * long(D) + 127) / 128;
  const bool few = rows * units <= kFewUnits;
  const int R = few ? kFewRows : kWriteRows;
  const long waves = (long(rows) + R - 1) / R * units;
  const unsigned grid = unsigned((waves + kThreads / kWave - 1) / (kThreads / kWave));
  auto go = [&](auto kernel, auto* t) {
    typedef decltype(t) P;
    kernel<<<grid, kThreads, 0, s>>>(static_cast<P>(const_cast<void*>(k)), k_stride, static_cast<P>(const_cast<void*>(v)),
                                     v_stride, slots, rows, Hkv, num_blocks, static_cast<P>(kc), static_cast<P>(vc));
  };
  auto by_dim = [&](auto* t) {
    typedef std::remove_pointer_t<decltype(t)> T;
    if (few) {
      if (D == 128) go(kv_write_few_kernel<128, T>, t); else go(kv_write_few_kernel<64, T>, t);
    } else {
      if (D == 128) go(kv_write_kernel<128, T>, t); else go(kv_write_kernel<64, T>, t);
    }
  };
  if (dt == MOLT_F32) by_dim(static_cast<float*>(nullptr));
  else by_dim(static_cast<uint16_t*>(nullptr));
  return hipGetLastError();
}

hipError_t launch_bounds_update(const void* kc, void* bounds, const int32_t* bt, const int32_t* starts,
                                const int32_t* lens, int B, int n, int Hkv, int D, int max_blocks, int num_blocks,
                                molt_dtype dt, hipStream_t s) {
  const int nblk = int((long(n) + 30) / 16);                             // blocks that n positions may touch
  const long waves = long(B) * nblk * Hkv;
  const unsigned grid = unsigned((waves + kThreads / kWave - 1) / (kThreads / kWave));
  auto go = [&](auto kernel, auto* c) {
    kernel<<<grid, kThreads, 0, s>>>(c, static_cast<uint8_t*>(bounds), bt, starts, lens, B, n, nblk, Hkv, max_blocks,
                                     num_blocks);
  };
  if (dt == MOLT_F32) {
    auto* c = static_cast<const float*>(kc);
    if (D == 128) go(bounds_update_kernel<128, float>, c); else go(bounds_update_kernel<64, float>, c);
  } else {
    auto* c = static_cast<const uint16_t*>(kc);
    if (D == 128) go(bounds_update_kernel<128, uint16_t>, c); else go(bounds_update_kernel<64, uint16_t>, c);
  }
  return hipGetLastError();
}

hipError_t launch_bounds_read(const void* bounds, const int32_t* ids, int M, int Hkv, int D, int num_blocks, float* hi,
                              float* lo, hipStream_t s) {
  const long records = long(M) * Hkv;
  const unsigned grid = unsigned((records * (D / 4) + kThreads - 1) / kThreads);
  auto* b = static_cast<const uint8_t*>(bounds);
  if (D == 128) bounds_read_kernel<128><<<grid, kThreads, 0, s>>>(b, ids, records, Hkv, num_blocks, hi, lo);
  else bounds_read_kernel<64><<<grid, kThreads, 0, s>>>(b, ids, records, Hkv, num_blocks, hi, lo);
  return hipGetLastError();
}

}  // namespace molt
