// Rows into and out of the 4-bit KV cache (format: kvq_format.h).
#include "internal.h"
#include "kvq_format.h"

namespace molt {
namespace {

constexpr int kThreads = 256;

// 8 consecutive row elements at any element alignment
typedef uint32_t U4 __attribute__((ext_vector_type(4), aligned(2)));
typedef float F4 __attribute__((ext_vector_type(4), aligned(4)));

MOLT_DEV void load8(const uint16_t* p, float (&x)[8]) {
  const U4 w = *reinterpret_cast<const U4*>(p);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[2 * i] = __uint_as_float(w[i] << 16);
    x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
  }
}
MOLT_DEV void load8(const float* p, float (&x)[8]) {
  const F4 a = *reinterpret_cast<const F4*>(p), b = *reinterpret_cast<const F4*>(p + 4);
#pragma unroll
  for (int i = 0; i < 4; ++i) { x[i] = a[i]; x[4 + i] = b[i]; }
}
MOLT_DEV void store8(uint16_t* p, const uint32_t (&v)[4]) { *reinterpret_cast<U4*>(p) = U4{v[0], v[1], v[2], v[3]}; }
MOLT_DEV void store8(float* p, const uint32_t (&v)[4]) {
  F4 a, b;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    a[2 * i] = __uint_as_float(v[i] << 16);
    a[2 * i + 1] = __uint_as_float(v[i] & 0xffff0000u);
    b[2 * i] = __uint_as_float(v[2 + i] << 16);
    b[2 * i + 1] = __uint_as_float(v[2 + i] & 0xffff0000u);
  }
  *reinterpret_cast<F4*>(p) = a;
  *reinterpret_cast<F4*>(p + 4) = b;
}

// Both kernels: wavefront = one block of one sequence, and one kv head of 128 dims or two of 64, its keys and its
// values. The block's place is found once, on the scalar unit, and all of a wavefront's loads are in flight together.
// Bound by HBM, or by the launch and three dependent loads where there is little: 4 kv heads x 128, bf16, 128 sequences
// x 5 rows written in 4.6 us and read in 3.7; f32, 4000 rows written in 5.8 us (18.6 MB, 3.2 TB/s) and 6000 read, a third
// of them zeros, in 8.6; 144000 bf16 rows read, of 262144 with the zeros behind, in 123 us (5.0 TB/s; a large copy: 4.96).
// Keys: instruction i, lane: an octet of dims of one token, 16 contiguous bytes of a bf16 row and 4 of the cache;
// values: the lane has an octet of dims of the 4 tokens that share its 16 bytes of the cache.
template <int D>
struct Tile {
  static constexpr int O = D / 8;                // octets of a head
  static constexpr int HPW = 128 / D;            // heads of a wavefront
  int lane;
  MOLT_DEV int k_head(int i) const { return HPW == 2 ? i / 2 : 0; }
  MOLT_DEV int k_token(int i) const { return HPW == 2 ? i % 2 * 8 + lane / O : i * 4 + lane / O; }
  MOLT_DEV int v_head() const { return HPW == 2 ? lane / 32 : 0; }
  MOLT_DEV int v_quad() const { return lane % (4 * O) / O; }
  MOLT_DEV int oct() const { return lane % O; }
};

// Where a wavefront's tokens are: token t of its block is row first + t of sequence b's rows (valid in [lo, hi)),
// records of head h0 on in block id of the caches (id < 0: no place)
struct Place { int b, h0, first, lo, hi, id; bool any; };
template <int D>
MOLT_DEV Place find_place(const KvqRows& p, int nblk) {
  constexpr int HPW = Tile<D>::HPW;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const uint32_t item = blockIdx.x * (kThreads / kWave) + wave;     // < 2^31 (the sizes that the C entries take)
  const uint32_t heads = uint32_t(p.Hkv + HPW - 1) / HPW, rest = item / heads;
  Place w;
  w.h0 = int(item - rest * heads) * HPW;
  const uint32_t bb = rest / uint32_t(nblk);
  const int k = int(rest - bb * uint32_t(nblk));
  w.any = bb < uint32_t(p.B);
  w.b = int(w.any ? bb : 0);
  const int start = p.start[w.b];
  const long blk = (long(start) >> 4) + k;       // block of the sequence, may be negative
  w.first = int(16 * blk - start);
  w.lo = -min(w.first, 0);                       // tokens of the block that are rows 0 .. n - 1
  w.hi = min(16, p.n - w.first);
  w.any = w.any && w.hi > w.lo;
  w.id = -1;
  if (w.any && blk >= 0 && blk < p.max_blocks) {
    const int id = p.bt[long(w.b) * p.max_blocks + blk];
    if (id >= 0 && id < p.num_blocks) w.id = id;
  }
  return w;
}

MOLT_DEV uint32_t magnitude(const float (&x)[8]) {
  uint32_t a = 0;
#pragma unroll
  for (int e = 0; e < 8; ++e) a = max(a, __float_as_uint(x[e]) & 0x7fffffffu);
  return a;
}
// largest over the 4 lanes of a group (lanes l, l ^ 1, l ^ 2, l ^ 3: DPP quad permutations)
MOLT_DEV uint32_t group_max(uint32_t a) {
  a = max(a, dpp_u32<0xB1, 0xF>(a, 0u));
  return max(a, dpp_u32<0x4E, 0xF>(a, 0u));
}

template <int D, typename T>
__global__ __launch_bounds__(kThreads) void kvq_write_kernel(KvqRows p, int nblk, const T* __restrict__ k, long k_stride,
                                                             const T* __restrict__ v, long v_stride) {
  typedef KvqRecord<D> Rec;
  const Place w = find_place<D>(p, nblk);
  if (!w.any || w.id < 0) return;
  const Tile<D> t{int(threadIdx.x % kWave)};
  const int hi = p.lens ? min(w.hi, min(max(p.lens[w.b], 0), p.n) - w.first) : w.hi;
  const long row0 = long(w.b) * p.n + w.first;
  const long rec = (long(w.id) * p.Hkv + w.h0) * Rec::kBytes;
  const int oct = t.oct();
  float x[4][8], y[4][8];
  bool kok[4], vok[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int tok = t.k_token(i), h = w.h0 + t.k_head(i);
    kok[i] = tok >= w.lo && tok < hi && h < p.Hkv;
    if (kok[i]) load8(k + (row0 + tok) * k_stride + h * D + oct * 8, x[i]);
    else for (int e = 0; e < 8; ++e) x[i][e] = 0.f;
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int tok = 4 * t.v_quad() + i, h = w.h0 + t.v_head();
    vok[i] = tok >= w.lo && tok < hi && h < p.Hkv;
    if (vok[i]) load8(v + (row0 + tok) * v_stride + h * D + oct * 8, y[i]);
    else for (int e = 0; e < 8; ++e) y[i][e] = 0.f;
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t s = kvq_scale(group_max(magnitude(x[i])));
    const uint32_t code = kvq_encode8(x[i], s);
    uint8_t* r = p.kc + rec + t.k_head(i) * Rec::kBytes;
    if (kok[i]) {
      *reinterpret_cast<uint32_t*>(r + Rec::k_code(t.k_token(i), oct)) = code;
      if (oct % 4 == 0) r[Rec::k_scale(t.k_token(i), oct / 4)] = uint8_t(s);
    }
  }
  uint32_t code[4], s[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    s[i] = kvq_scale(group_max(magnitude(y[i])));
    code[i] = kvq_encode8(y[i], s[i]);
  }
  uint8_t* r = p.vc + rec + t.v_head() * Rec::kBytes;
  if (vok[0] && vok[3]) {                        // rows are consecutive
    *reinterpret_cast<uint4*>(r + Rec::v_code(4 * t.v_quad(), oct)) = make_uint4(code[0], code[1], code[2], code[3]);
    if (oct % 4 == 0)
      *reinterpret_cast<uint32_t*>(r + Rec::v_scale(4 * t.v_quad(), oct / 4)) = s[0] | s[1] << 8 | s[2] << 16 | s[3] << 24;
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (!vok[i]) continue;
      *reinterpret_cast<uint32_t*>(r + Rec::v_code(4 * t.v_quad() + i, oct)) = code[i];
      if (oct % 4 == 0) r[Rec::v_scale(4 * t.v_quad() + i, oct / 4)] = uint8_t(s[i]);
    }
  }
}

MOLT_DEV void decode8(uint32_t code, uint32_t scale_bits, uint32_t (&w)[4]) {
  w[0] = kvq_decode2<0>(code, scale_bits);
  w[1] = kvq_decode2<1>(code, scale_bits);
  w[2] = kvq_decode2<2>(code, scale_bits);
  w[3] = kvq_decode2<3>(code, scale_bits);
}

template <int D, typename T>
__global__ __launch_bounds__(kThreads) void kvq_read_kernel(KvqRows p, int nblk, T* __restrict__ k, T* __restrict__ v) {
  typedef KvqRecord<D> Rec;
  const Place w = find_place<D>(p, nblk);
  if (!w.any) return;
  const Tile<D> t{int(threadIdx.x % kWave)};
  // rows from `hi` on and rows of a block without a place are zeros: nothing is read for them
  const int hi = w.id < 0 ? 0 : p.lens ? min(w.hi, min(max(p.lens[w.b], 0), p.n) - w.first) : w.hi;
  const long row0 = long(w.b) * p.n + w.first;
  const long rec = (long(max(w.id, 0)) * p.Hkv + w.h0) * Rec::kBytes;
  const int oct = t.oct();
  uint32_t kcode[4], ks[4], vs = 0;
  uint4 vcode = make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    kcode[i] = ks[i] = 0;
    if (t.k_token(i) < hi && w.h0 + t.k_head(i) < p.Hkv) {
      const uint8_t* r = p.kc + rec + t.k_head(i) * Rec::kBytes;
      kcode[i] = *reinterpret_cast<const uint32_t*>(r + Rec::k_code(t.k_token(i), oct));
      ks[i] = r[Rec::k_scale(t.k_token(i), oct / 4)];
    }
  }
  if (4 * t.v_quad() < hi && w.h0 + t.v_head() < p.Hkv) {
    const uint8_t* r = p.vc + rec + t.v_head() * Rec::kBytes;
    vcode = *reinterpret_cast<const uint4*>(r + Rec::v_code(4 * t.v_quad(), oct));
    vs = *reinterpret_cast<const uint32_t*>(r + Rec::v_scale(4 * t.v_quad(), oct / 4));
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int tok = t.k_token(i), h = w.h0 + t.k_head(i);
    if (tok < w.lo || tok >= w.hi || h >= p.Hkv) continue;
    uint32_t o[4];
    decode8(kcode[i], ks[i] << 23, o);           // zero codes where nothing was read
    store8(k + ((row0 + tok) * p.Hkv + h) * D + oct * 8, o);
  }
  const uint32_t c[4] = {vcode.x, vcode.y, vcode.z, vcode.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int tok = 4 * t.v_quad() + i, h = w.h0 + t.v_head();
    if (tok < w.lo || tok >= w.hi || h >= p.Hkv) continue;
    uint32_t o[4] = {0u, 0u, 0u, 0u};
    if (tok < hi) decode8(c[i], kvq_scale_bits(vs, i), o);
    store8(v + ((row0 + tok) * p.Hkv + h) * D + oct * 8, o);
  }
}

// The decoder's rows: workgroup = token t of the QKV projection's f32 rows, rotated in f64 with the step's table as for
// the other caches. q -> q_out; thread = octet of a key (both halves of its pairs read, its own rotated) or value
// head, rounded to the model's type, then quantised: the bytes that kvq_write makes of those rows. 640 tokens of 32 query
// and 2 x 4 kv heads x 128, bf16: 10.9 us, 19 MB (the f32 rows in, q and the records out); the QKV product before it takes
// 24.1, together 35 where the product that rotates and stores in its epilogue takes 32 for the bf16 cache.
MOLT_DEV void store_q(uint16_t* p, float x) { *p = f32_to_bf16(x); }
MOLT_DEV void store_q(float* p, float x) { *p = x; }
template <int D, typename T>
__global__ __launch_bounds__(kThreads) void rope_kvq_kernel(const float* __restrict__ qkv, int k, int Hq, int Hkv,
                                                            const double2* __restrict__ table,
                                                            const int32_t* __restrict__ ctx,
                                                            const int32_t* __restrict__ bt, int max_blocks,
                                                            int num_blocks, T* __restrict__ q_out,
                                                            uint8_t* __restrict__ kc, uint8_t* __restrict__ vc) {
  typedef KvqRecord<D> Rec;
  constexpr int half = D / 2, O = D / 8;
  const int t = blockIdx.x, b = t / (k + 1);
  const double2* cs = table + long(t) * half;
  const float* row = qkv + long(t) * (Hq + 2 * Hkv) * D;
  for (int w = threadIdx.x; w < Hq * half; w += kThreads) {
    const int h = w / half, i = w % half;
    const double a = row[h * D + i], c = row[h * D + i + half];
    const double2 r = cs[i];
    store_q(q_out + (long(t) * Hq + h) * D + i, float(a * r.x - c * r.y));
    store_q(q_out + (long(t) * Hq + h) * D + i + half, float(c * r.x + a * r.y));
  }
  const long pos = long(ctx[b]) + t % (k + 1);
  if (pos < 0 || pos >= 16l * max_blocks) return;
  const int blk = bt[long(b) * max_blocks + pos / 16], slot = int(pos % 16);
  if (blk < 0 || blk >= num_blocks) return;
  for (int w = threadIdx.x; w < 2 * Hkv * O; w += kThreads) {
    const bool value = w >= Hkv * O;
    const int h = w / O % Hkv, oct = w % O;
    const float* src = row + long(Hq + (value ? Hkv : 0) + h) * D;
    float x[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int d = oct * 8 + e;
      float v = src[d];
      if (!value) {
        const double other = src[d < half ? d + half : d - half];
        const double2 r = cs[d % half];
        v = float(d < half ? v * r.x - other * r.y : v * r.x + other * r.y);
      }
      x[e] = sizeof(T) == 2 ? round_to_bf16(v) : v;
    }
    const uint32_t s = kvq_scale(group_max(magnitude(x)));
    uint8_t* rec = (value ? vc : kc) + (long(blk) * Hkv + h) * Rec::kBytes;
    *reinterpret_cast<uint32_t*>(rec + (value ? Rec::v_code(slot, oct) : Rec::k_code(slot, oct))) = kvq_encode8(x, s);
    if (oct % 4 == 0) rec[value ? Rec::v_scale(slot, oct / 4) : Rec::k_scale(slot, oct / 4)] = uint8_t(s);
  }
}

// blocks that n consecutive positions may touch, and workgroups of a call
int blocks_of(int n) { return int((long(n) + 30) / 16); }
unsigned grid_of(const KvqRows& p, int D) {
  const long waves = long(p.B) * blocks_of(p.n) * ((p.Hkv * D + 127) / 128);
  return unsigned((waves + kThreads / kWave - 1) / (kThreads / kWave));
}

}  // namespace

hipError_t launch_kvq_write(const KvqRows& p, const void* k, long k_stride, const void* v, long v_stride, int D,
                            molt_dtype dt, hipStream_t s) {
  const unsigned grid = grid_of(p, D);
  auto go = [&](auto kernel, auto* kk, auto* vv) { kernel<<<grid, kThreads, 0, s>>>(p, blocks_of(p.n), kk, k_stride, vv, v_stride); };
  if (dt == MOLT_F32) {
    auto *a = static_cast<const float*>(k), *b = static_cast<const float*>(v);
    if (D == 128) go(kvq_write_kernel<128, float>, a, b); else go(kvq_write_kernel<64, float>, a, b);
  } else {
    auto *a = static_cast<const uint16_t*>(k), *b = static_cast<const uint16_t*>(v);
    if (D == 128) go(kvq_write_kernel<128, uint16_t>, a, b); else go(kvq_write_kernel<64, uint16_t>, a, b);
  }
  return hipGetLastError();
}

hipError_t launch_kvq_read(const KvqRows& p, void* k, void* v, int D, molt_dtype dt, hipStream_t s) {
  const unsigned grid = grid_of(p, D);
  auto go = [&](auto kernel, auto* kk, auto* vv) { kernel<<<grid, kThreads, 0, s>>>(p, blocks_of(p.n), kk, vv); };
  if (dt == MOLT_F32) {
    auto *a = static_cast<float*>(k), *b = static_cast<float*>(v);
    if (D == 128) go(kvq_read_kernel<128, float>, a, b); else go(kvq_read_kernel<64, float>, a, b);
  } else {
    auto *a = static_cast<uint16_t*>(k), *b = static_cast<uint16_t*>(v);
    if (D == 128) go(kvq_read_kernel<128, uint16_t>, a, b); else go(kvq_read_kernel<64, uint16_t>, a, b);
  }
  return hipGetLastError();
}

hipError_t launch_rope_kvq_write(const float* qkv, int B, int k, int Hq, int Hkv, int D, const void* table,
                                 const int32_t* ctx, const int32_t* bt, int max_blocks, int num_blocks,
                                 molt_dtype dt, void* q_out, void* k_cache, void* v_cache, hipStream_t s) {
  auto go = [&](auto kernel, auto* q) {
    kernel<<<B * (k + 1), kThreads, 0, s>>>(qkv, k, Hq, Hkv, static_cast<const double2*>(table), ctx, bt, max_blocks,
                                            num_blocks, q, static_cast<uint8_t*>(k_cache),
                                            static_cast<uint8_t*>(v_cache));
  };
  if (dt == MOLT_F32) {
    auto* q = static_cast<float*>(q_out);
    if (D == 128) go(rope_kvq_kernel<128, float>, q); else go(rope_kvq_kernel<64, float>, q);
  } else {
    auto* q = static_cast<uint16_t*>(q_out);
    if (D == 128) go(rope_kvq_kernel<128, uint16_t>, q); else go(rope_kvq_kernel<64, uint16_t>, q);
  }
  return hipGetLastError();
}

}  // namespace molt
