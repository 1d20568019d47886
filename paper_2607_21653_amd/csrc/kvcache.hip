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

// Block and slot of position start[b] + j; block < 0 where the row has none
MOLT_DEV void place(const KvqRows& p, int b, int j, int& blk, int& slot) {
  const long pos = long(p.start[b]) + j;
  blk = -1;
  slot = int(pos & 15);
  if ((p.lens && j >= p.lens[b]) || pos < 0 || pos >= 16l * p.max_blocks) return;
  const int id = p.bt[long(b) * p.max_blocks + pos / 16];
  if (id >= 0 && id < p.num_blocks) blk = id;
}

// Thread = octet of 8 dims of (row, head) of K or V: the group's largest magnitude over its 4
// lanes, then 4 code bytes.
template <int D, typename T>
__global__ __launch_bounds__(kThreads) void kvq_write_kernel(KvqRows p, const T* __restrict__ k, long k_stride,
                                                             const T* __restrict__ v, long v_stride) {
  typedef KvqRecord<D> Rec;
  const long i = long(blockIdx.x) * kThreads + threadIdx.x;
  const int oct = int(i % (D / 8));
  const long rh = i / (D / 8);
  const int h = int(rh % p.Hkv);
  const long row = rh / p.Hkv % (long(p.B) * p.n);
  const bool value = rh / p.Hkv / (long(p.B) * p.n) != 0;
  if (rh >= 2l * p.B * p.n * p.Hkv) return;      // whole groups: D / 8 lanes of a head stay together
  int blk, slot;
  place(p, int(row / p.n), int(row % p.n), blk, slot);
  if (blk < 0) return;
  float x[8];
  load8((value ? v + row * v_stride : k + row * k_stride) + h * D + oct * 8, x);
  uint32_t a = 0;
#pragma unroll
  for (int e = 0; e < 8; ++e) a = max(a, __float_as_uint(x[e]) & 0x7fffffffu);
  a = max(a, uint32_t(__shfl_xor(int(a), 1)));
  a = max(a, uint32_t(__shfl_xor(int(a), 2)));
  const uint32_t s = kvq_scale(a);
  const uint32_t code = kvq_encode8(x, s);
  uint8_t* rec = (value ? p.vc : p.kc) + (long(blk) * p.Hkv + h) * Rec::kBytes;
  *reinterpret_cast<uint32_t*>(rec + (value ? Rec::v_code(slot, oct) : Rec::k_code(slot, oct))) = code;
  if (oct % 4 == 0) rec[value ? Rec::v_scale(slot, oct / 4) : Rec::k_scale(slot, oct / 4)] = uint8_t(s);
}

template <int D, typename T>
__global__ __launch_bounds__(kThreads) void kvq_read_kernel(KvqRows p, T* __restrict__ k, T* __restrict__ v) {
  typedef KvqRecord<D> Rec;
  const long i = long(blockIdx.x) * kThreads + threadIdx.x;
  const int oct = int(i % (D / 8));
  const long rh = i / (D / 8);
  const int h = int(rh % p.Hkv);
  const long row = rh / p.Hkv % (long(p.B) * p.n);
  const bool value = rh / p.Hkv / (long(p.B) * p.n) != 0;
  if (rh >= 2l * p.B * p.n * p.Hkv) return;
  int blk, slot;
  place(p, int(row / p.n), int(row % p.n), blk, slot);
  uint32_t w[4] = {0, 0, 0, 0};
  if (blk >= 0) {
    const uint8_t* rec = (value ? p.vc : p.kc) + (long(blk) * p.Hkv + h) * Rec::kBytes;
    const uint32_t code = *reinterpret_cast<const uint32_t*>(rec + (value ? Rec::v_code(slot, oct) : Rec::k_code(slot, oct)));
    const uint32_t s = uint32_t(rec[value ? Rec::v_scale(slot, oct / 4) : Rec::k_scale(slot, oct / 4)]) << 23;
    w[0] = kvq_decode2<0>(code, s);
    w[1] = kvq_decode2<1>(code, s);
    w[2] = kvq_decode2<2>(code, s);
    w[3] = kvq_decode2<3>(code, s);
  }
  store8((value ? v : k) + (row * p.Hkv + h) * D + oct * 8, w);
}

}  // namespace

hipError_t launch_kvq_write(const KvqRows& p, const void* k, long k_stride, const void* v, long v_stride, int D,
                            molt_dtype dt, hipStream_t s) {
  const long threads = 2l * p.B * p.n * p.Hkv * (D / 8);
  const unsigned grid = unsigned((threads + kThreads - 1) / kThreads);
  auto go = [&](auto kernel, auto* kk, auto* vv) { kernel<<<grid, kThreads, 0, s>>>(p, kk, k_stride, vv, v_stride); };
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
  const long threads = 2l * p.B * p.n * p.Hkv * (D / 8);
  const unsigned grid = unsigned((threads + kThreads - 1) / kThreads);
  auto go = [&](auto kernel, auto* kk, auto* vv) { kernel<<<grid, kThreads, 0, s>>>(p, kk, vv); };
  if (dt == MOLT_F32) {
    auto *a = static_cast<float*>(k), *b = static_cast<float*>(v);
    if (D == 128) go(kvq_read_kernel<128, float>, a, b); else go(kvq_read_kernel<64, float>, a, b);
  } else {
    auto *a = static_cast<uint16_t*>(k), *b = static_cast<uint16_t*>(v);
    if (D == 128) go(kvq_read_kernel<128, uint16_t>, a, b); else go(kvq_read_kernel<64, uint16_t>, a, b);
  }
  return hipGetLastError();
}

}  // namespace molt
