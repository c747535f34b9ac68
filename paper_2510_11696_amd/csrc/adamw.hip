// lora_adamw_*: the optimizer step on the LoRA matrices, all tensors in one launch, with the moments in 32 bits or in 8, and the
// gradients' norm for clipping.  With g the gradient (times *grad_scale), t the step:
//   m' = b1 m + (1 - b1) g                      v' = b2 v + (1 - b2) g^2
//   p' = p (1 - lr wd) - lr / (1 - b1^t) m' / ( sqrt(v') / sqrt(1 - b2^t) + eps )
// every operation one IEEE fp32 rounding (this file is compiled without contraction), the factors formed in fp64 and rounded once.
// The parameters are fp32; their bf16 copies, which the linears read, are written on the way.
//
// Moments in 8 bits.  Blocks of 32 elements share a byte f, the exponent field of the block's largest magnitude as fp32 (at least 1;
// 255 for a block with an infinity or a NaN, which reads as NaN throughout).  Powers of two scale exactly, so nothing is lost but the
// 8-bit rounding itself.
//   m: sign, 4 exponent bits, 3 mantissa bits (value: the bits at fp32's bit 20, times 2^(f - 14)).  The largest magnitude of a block has
//      exponent 14 of 15, so rounding up never overflows the code; where the value would be 2^128 (f = 254), 1.875 2^127 stands in its place.
//   v: 5 exponent bits, 3 mantissa bits, times 2^(f - 30), 30 of 31 as above.  A v above zero never becomes zero (smallest code 1): m reaches down to 2^-16 of
//      its block's largest, sqrt(v) to 2^-16 too, and m / sqrt(v) stays bounded.
// Both are rounded up in magnitude with the probability of what is cut off.  To nearest, they would stop moving: under a steady gradient
// g the first moment changes by 0.1 (g - m) and stays where that is under half a step, up to a quarter below g; the second by
// 0.001 (g^2 - v), so that after some sixteen steps v would freeze at a sixtieth of where it belongs while 1 - b2^t goes on to 1.
// m and v of an element share its 16 random bits: each is unbiased, and that both go up on the same fraction does no harm.
// The random bits are a pure function of (seed, t, index): group b of eight elements of the state takes the four words of Philox4x32
// with 10 rounds, counter (b lo, b hi, t lo, t hi), key (seed lo, seed hi); element j the low (even j) or high half of word j / 2.
//
// What bounds the step: memory, 30 bytes per element with 32-bit moments, 18.1 with 8-bit ones: 68.8 M elements in 349 us (5.9 TB/s), 80.7 M in
// 245 us (6.0 TB/s); a plain copy of 2 GiB reaches 4.9.  Eight elements per lane, so that 8-bit moments are 8-byte accesses and a block
// of 32 is four lanes; one workgroup per 2048 elements of one tensor, so that its addresses are uniform.
#include <math.h>
#include <stdlib.h>
#include "common.hpp"
#include "philox.hpp"

namespace qerl {

constexpr int kStateBlock = 32;       // elements that share a scale byte; tensors start at multiples of it in the state
constexpr int kChunk = 2048;          // elements of one tensor that a workgroup takes at a time
constexpr int kAdamThreads = 256;
constexpr int64_t kMaxChunks = ((int64_t)1 << 24) - 1;   // a launch has fewer than 2^32 threads

struct AdamTensor { float* p; uint16_t* copy; const float* g; int64_t n, state0, chunk0; };   // state0: first element in the state
constexpr int kTableBatch = 64;
struct TableBatch { AdamTensor t[kTableBatch]; };
static_assert(sizeof(TableBatch) <= 3584, "kernel arguments");

struct AdamArgs {
  const AdamTensor* table; const uint32_t* owner;        // tensor of each chunk
  void* m; void* v; uint8_t* ms; uint8_t* vs;
  float b1, omb1, b2, omb2, eps;
  float decay, step_size, isb2;                          // from the host, or (device_hyper) formed from the doubles below
  double lr, beta1, beta2, wd; int64_t step;
  const float* lr_dev; const int64_t* step_dev; const float* grad_scale;
  uint32_t k0, k1;
};

// b^t by squaring
__host__ __device__ inline double int_power(double b, int64_t t) {
  double r = 1.0;
  for (; t > 0; t >>= 1, b *= b)
    if (t & 1) r *= b;
  return r;
}
struct AdamFactors { float decay, step_size, isb2; };
__host__ __device__ inline AdamFactors adam_factors(double lr, double beta1, double beta2, double wd, int64_t t) {
  return AdamFactors{(float)(1.0 - lr * wd), (float)(lr / (1.0 - int_power(beta1, t))), (float)(1.0 / sqrt(1.0 - int_power(beta2, t)))};
}

// largest of the block of 32, which four neighbouring lanes hold eight of each
__device__ __forceinline__ uint32_t quad_max(uint32_t v) {
  const uint32_t a = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0xB1, 0xf, 0xf, false);   // quad_perm [1,0,3,2]
  v = v > a ? v : a;
  const uint32_t b = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x4E, 0xf, 0xf, false);   // quad_perm [2,3,0,1]
  return v > b ? v : b;
}
__device__ __forceinline__ uint32_t block_field(const float (&x)[8]) {
  uint32_t top = 0;
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const uint32_t b = __float_as_uint(x[j]) & 0x7fffffffu;
    top = top > b ? top : b;
  }
  top = quad_max(top) >> 23;
  return top > 1u ? top : 1u;
}
__device__ __forceinline__ float decode_m(uint32_t c, uint32_t field) {
  const float mag = ldexpf(__uint_as_float((c & 127u) << 20), (int)field - 14);
  return field == 255u ? __uint_as_float(0x7fc00000u) : (c & 128u) ? -mag : mag;
}
__device__ __forceinline__ float decode_v(uint32_t c, uint32_t field) {
  return field == 255u ? __uint_as_float(0x7fc00000u) : ldexpf(__uint_as_float(c << 20), (int)field - 30);
}
// largest code: the next one's value is not finite where the block reaches fp32's last power of two
__device__ __forceinline__ uint32_t last_code(int top, uint32_t field) { return field == 254u ? 8u * top + 7u : 8u * top + 8u; }
__device__ __forceinline__ uint32_t encode_m(float x, uint32_t field, uint32_t random16) {
  const uint32_t b = __float_as_uint(ldexpf(fabsf(x), 14 - (int)field));
  const uint32_t up = (b + (random16 << 4)) >> 20, last = last_code(14, field), c = up < last ? up : last;
  return field == 255u ? 0u : c | (x < 0.f ? 128u : 0u);
}
__device__ __forceinline__ uint32_t encode_v(float x, uint32_t field, uint32_t random16) {
  const uint32_t b = __float_as_uint(ldexpf(x, 30 - (int)field));
  const uint32_t up = (b + (random16 << 4)) >> 20, last = last_code(30, field), c = up < last ? up : last;
  return field == 255u || !(x > 0.f) ? 0u : c > 1u ? c : 1u;
}

__global__ __launch_bounds__(64) void adamw_table_kernel(const TableBatch batch, int count, AdamTensor* out, uint32_t* arrived) {
  const int i = threadIdx.x;
  if (i == 0) *arrived = 0u;
  if (i < count) out[i] = batch.t[i];
}
__global__ __launch_bounds__(256) void adamw_owner_kernel(const AdamTensor* table, uint32_t* owner) {
  const AdamTensor t = table[blockIdx.x];
  const int64_t n = (t.n + kChunk - 1) / kChunk;
  for (int64_t i = threadIdx.x; i < n; i += 256) owner[t.chunk0 + i] = blockIdx.x;
}

template <int BITS, bool DEVICE_HYPER>
__global__ __launch_bounds__(kAdamThreads) void adamw_kernel(const AdamArgs a) {
  float scale = 1.f;
  if (a.grad_scale) {
    scale = *a.grad_scale;
    if (!isfinite(scale)) return;                        // an overflowed gradient: the step leaves everything as it is
  }
  float decay = a.decay, step_size = a.step_size, isb2 = a.isb2;
  int64_t step = a.step;
  if constexpr (DEVICE_HYPER) {
    if (a.step_dev) step = *a.step_dev;
    const double lr = a.lr_dev ? (double)*a.lr_dev : a.lr;
    if (step < 1 || !(lr >= 0.0) || !isfinite(lr)) return;   // what the host refuses
    const AdamFactors f = adam_factors(lr, a.beta1, a.beta2, a.wd, step);
    if (!isfinite(f.decay) || !isfinite(f.step_size)) return;
    decay = f.decay; step_size = f.step_size; isb2 = f.isb2;
  }
  const uint32_t chunk = blockIdx.x;
  const AdamTensor t = a.table[a.owner[chunk]];
  const int64_t i0 = ((int64_t)chunk - t.chunk0) * kChunk + (int64_t)threadIdx.x * 8;
  if (i0 >= (t.n + kStateBlock - 1) / kStateBlock * kStateBlock) return;   // the four lanes of a block of 32 stay together
  const int64_t s0 = t.state0 + i0;
  const int inside = t.n - i0 >= 8 ? 8 : t.n > i0 ? (int)(t.n - i0) : 0;   // elements of the tensor; what follows in the state is kept zero
  float g[8], p[8], m[8], v[8];
  if (inside == 8) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const f32x4 gv = *reinterpret_cast<const f32x4*>(t.g + i0 + 4 * h), pv = *reinterpret_cast<const f32x4*>(t.p + i0 + 4 * h);
#pragma unroll
      for (int j = 0; j < 4; ++j) { g[4 * h + j] = gv[j]; p[4 * h + j] = pv[j]; }
    }
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) { g[j] = j < inside ? t.g[i0 + j] : 0.f; p[j] = j < inside ? t.p[i0 + j] : 0.f; }
  }
  if constexpr (BITS == 32) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const f32x4 mv = *reinterpret_cast<const f32x4*>(static_cast<const float*>(a.m) + s0 + 4 * h);
      const f32x4 vv = *reinterpret_cast<const f32x4*>(static_cast<const float*>(a.v) + s0 + 4 * h);
#pragma unroll
      for (int j = 0; j < 4; ++j) { m[4 * h + j] = mv[j]; v[4 * h + j] = vv[j]; }
    }
  } else {
    const u32x2 mc = *reinterpret_cast<const u32x2*>(static_cast<const uint8_t*>(a.m) + s0), vc = *reinterpret_cast<const u32x2*>(static_cast<const uint8_t*>(a.v) + s0);
    const uint32_t mf = a.ms[s0 / kStateBlock], vf = a.vs[s0 / kStateBlock];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      m[j] = decode_m((mc[j >> 2] >> (8 * (j & 3))) & 255u, mf);
      v[j] = decode_v((vc[j >> 2] >> (8 * (j & 3))) & 255u, vf);
    }
  }
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const float gs = a.grad_scale ? g[j] * scale : g[j];
    m[j] = a.b1 * m[j] + a.omb1 * gs;
    v[j] = a.b2 * v[j] + a.omb2 * (gs * gs);
    const float root = sqrtf(v[j]) * isb2 + a.eps;
    p[j] = p[j] * decay - step_size * m[j] / root;
  }
  if (inside < 8) {
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (j >= inside) m[j] = v[j] = 0.f;
  }
  if (inside == 8) {
#pragma unroll
    for (int h = 0; h < 2; ++h) *reinterpret_cast<f32x4*>(t.p + i0 + 4 * h) = f32x4{p[4 * h], p[4 * h + 1], p[4 * h + 2], p[4 * h + 3]};
    if (t.copy)
      *reinterpret_cast<u32x4*>(t.copy + i0) = u32x4{pack_bf16x2(p[0], p[1]), pack_bf16x2(p[2], p[3]), pack_bf16x2(p[4], p[5]), pack_bf16x2(p[6], p[7])};
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (j < inside) {
        t.p[i0 + j] = p[j];
        if (t.copy) t.copy[i0 + j] = (uint16_t)f32_to_bf16_bits(p[j]);
      }
  }
  if constexpr (BITS == 32) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      *reinterpret_cast<f32x4*>(static_cast<float*>(a.m) + s0 + 4 * h) = f32x4{m[4 * h], m[4 * h + 1], m[4 * h + 2], m[4 * h + 3]};
      *reinterpret_cast<f32x4*>(static_cast<float*>(a.v) + s0 + 4 * h) = f32x4{v[4 * h], v[4 * h + 1], v[4 * h + 2], v[4 * h + 3]};
    }
  } else {
    const uint32_t mf = block_field(m), vf = block_field(v);
    const uint64_t b = (uint64_t)s0 / 8;
    const Philox4 r = philox4x32_10((uint32_t)b, (uint32_t)(b >> 32), (uint32_t)step, (uint32_t)((uint64_t)step >> 32), a.k0, a.k1);
    u32x2 mc = {0u, 0u}, vc = {0u, 0u};
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const uint32_t random16 = (r.v[j >> 1] >> (16 * (j & 1))) & 0xffffu;
      mc[j >> 2] |= encode_m(m[j], mf, random16) << (8 * (j & 3));
      vc[j >> 2] |= encode_v(v[j], vf, random16) << (8 * (j & 3));
    }
    *reinterpret_cast<u32x2*>(static_cast<uint8_t*>(a.m) + s0) = mc;
    *reinterpret_cast<u32x2*>(static_cast<uint8_t*>(a.v) + s0) = vc;
    if ((threadIdx.x & 3) == 0) {
      a.ms[s0 / kStateBlock] = (uint8_t)mf;
      a.vs[s0 / kStateBlock] = (uint8_t)vf;
    }
  }
}

// Moments in 8 bits -> fp32
__global__ __launch_bounds__(256) void adamw_moments_kernel(const uint8_t* mc, const uint8_t* vc, const uint8_t* ms, const uint8_t* vs,
                                                            int64_t groups, float* m, float* v) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= groups) return;
  const u32x2 cm = reinterpret_cast<const u32x2*>(mc)[i], cv = reinterpret_cast<const u32x2*>(vc)[i];
  const uint32_t fm = ms[i / 4], fv = vs[i / 4];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    f32x4 a, b;
#pragma unroll
    for (int j = 0; j < 4; ++j) { a[j] = decode_m((cm[h] >> (8 * j)) & 255u, fm); b[j] = decode_v((cv[h] >> (8 * j)) & 255u, fv); }
    reinterpret_cast<f32x4*>(m)[2 * i + h] = a;
    reinterpret_cast<f32x4*>(v)[2 * i + h] = b;
  }
}

// Sum of squares of all gradients: a workgroup sums a contiguous range of chunks in fp64 (a square of an fp32 value is exact there); the
// last one to finish adds the workgroups' sums in their order, so that nothing depends on which one it was, and sets the counter back.
// Sums and counter pass between the XCDs' caches by accesses at device scope.  323 MB in 100 us (3.2 TB/s): a group of chunks waits for its tensors'
// numbers, then for their table entries, then for its gradients, before the next one begins.
constexpr int kNormGroups = 2048, kNormAhead = 4;
struct NormArea { double partial[kNormGroups]; uint32_t arrived; };
__device__ __forceinline__ double block_sum64(double v, double* smem) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
  if ((threadIdx.x & 63) == 0) smem[threadIdx.x >> 6] = v;
  __syncthreads();
  return (smem[0] + smem[1]) + (smem[2] + smem[3]);
}
__global__ __launch_bounds__(256) void adamw_norm_kernel(const AdamTensor* table, const uint32_t* owner, int64_t chunks, NormArea* area, double max_norm,
                                                         float* norm, float* scale) {
  __shared__ double smem[2][4];
  __shared__ uint32_t order;
  const int64_t c0 = chunks * blockIdx.x / gridDim.x, c1 = chunks * (blockIdx.x + 1) / gridDim.x;
  double sum = 0.0;
  for (int64_t c = c0; c < c1; c += kNormAhead) {       // some chunks at a time: their places, then their values, are all on their way together
    const float* g[kNormAhead];
    int left[kNormAhead];
#pragma unroll
    for (int u = 0; u < kNormAhead; ++u) {
      const int64_t at = c + u < c1 ? c + u : c1 - 1;
      const AdamTensor t = table[owner[at]];
      const int64_t i0 = (at - t.chunk0) * kChunk + (int64_t)threadIdx.x * 8, rest = c + u < c1 ? t.n - i0 : 0;
      g[u] = t.g + i0;
      left[u] = rest >= 8 ? 8 : rest > 0 ? (int)rest : 0;
    }
    f32x4 v[kNormAhead][2] = {};
#pragma unroll
    for (int u = 0; u < kNormAhead; ++u)
      if (left[u] == 8) {
        v[u][0] = *reinterpret_cast<const f32x4*>(g[u]);
        v[u][1] = *reinterpret_cast<const f32x4*>(g[u] + 4);
      }
#pragma unroll
    for (int u = 0; u < kNormAhead; ++u) {
#pragma unroll
      for (int j = 0; j < 8; ++j) sum += (double)v[u][j >> 2][j & 3] * (double)v[u][j >> 2][j & 3];
      if (left[u] < 8)
        for (int j = 0; j < left[u]; ++j) sum += (double)g[u][j] * (double)g[u][j];
    }
  }
  sum = block_sum64(sum, smem[0]);
  uint64_t* partial = reinterpret_cast<uint64_t*>(area->partial);
  if (threadIdx.x == 0) {
    __hip_atomic_store(partial + blockIdx.x, __builtin_bit_cast(uint64_t, sum), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");     // the sum is where all see it before the count is; a release would write the L2 back
    order = __hip_atomic_fetch_add(&area->arrived, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  }
  __syncthreads();
  if (order != gridDim.x - 1) return;
  sum = 0.0;
  for (int i = threadIdx.x; i < (int)gridDim.x; i += 256)
    sum += __builtin_bit_cast(double, __hip_atomic_load(partial + i, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT));
  sum = block_sum64(sum, smem[1]);
  if (threadIdx.x == 0) {
    const double r = sqrt(sum), s = max_norm / (r + 1e-6);
    if (norm) *norm = (float)r;
    *scale = isfinite(r) ? (float)(s < 1.0 ? s : 1.0) : __uint_as_float(0x7fc00000u);
    __hip_atomic_store(&area->arrived, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  }
}

struct Span { uintptr_t begin, end; int write; };
static int by_begin(const void* a, const void* b) {
  const uintptr_t x = static_cast<const Span*>(a)->begin, y = static_cast<const Span*>(b)->begin;
  return x < y ? -1 : x > y;
}
// 0, 1 if memory that a step writes is named twice among the tensors and what else is written, -1 if the list of spans could not be held
static int overlaps(const qerl_adamw_tensor* t, int n, const Span* others, int n_others) {
  Span* s = static_cast<Span*>(malloc(sizeof(Span) * (3 * (size_t)n + n_others)));
  if (!s) return -1;
  size_t k = 0;
  for (int i = 0; i < n_others; ++i)
    if (others[i].end > others[i].begin) s[k++] = others[i];
  for (int i = 0; i < n; ++i) {
    if (t[i].n == 0) continue;
    const uintptr_t p = (uintptr_t)t[i].param_f32, c = (uintptr_t)t[i].copy_bf16, g = (uintptr_t)t[i].grad_f32;
    s[k++] = Span{p, p + 4 * (uintptr_t)t[i].n, 1};
    if (c) s[k++] = Span{c, c + 2 * (uintptr_t)t[i].n, 1};
    s[k++] = Span{g, g + 4 * (uintptr_t)t[i].n, 0};
  }
  qsort(s, k, sizeof(Span), by_begin);
  uintptr_t end[2] = {0, 0};                             // of what was read, written so far
  int bad = 0;
  for (size_t i = 0; i < k && !bad; ++i) {
    bad = s[i].begin < end[1] || (s[i].write && s[i].begin < end[0]);
    if (s[i].end > end[s[i].write]) end[s[i].write] = s[i].end;
  }
  free(s);
  return bad;
}

// The table: what the norm's workgroups hand over, the tensors, the tensor of each chunk
constexpr size_t kNormBytes = (sizeof(NormArea) + 255) & ~(size_t)255;
static size_t owner_offset(int n) { return kNormBytes + (((size_t)n * sizeof(AdamTensor) + 255) & ~(size_t)255); }
struct AdamLayout { int64_t elements, chunks; size_t bytes; };
static bool adam_layout(const qerl_adamw_tensor* t, int n, AdamLayout& l) {
  if (!t || n < 1 || n > (1 << 20)) return false;
  l.elements = l.chunks = 0;
  for (int i = 0; i < n; ++i) {
    if (t[i].n < 0 || t[i].n > ((int64_t)1 << 40)) return false;
    l.elements += ceil_div(t[i].n, kStateBlock) * kStateBlock;
    l.chunks += ceil_div(t[i].n, kChunk);
    if (l.chunks > kMaxChunks) return false;
  }
  l.bytes = (owner_offset(n) + (size_t)l.chunks * 4 + 255) & ~(size_t)255;
  return true;
}
static const AdamTensor* tensors_of(const qerl_adamw_plan* p) { return reinterpret_cast<const AdamTensor*>(static_cast<const uint8_t*>(p->table) + kNormBytes); }
static const uint32_t* owner_of(const qerl_adamw_plan* p) {
  return reinterpret_cast<const uint32_t*>(static_cast<const uint8_t*>(p->table) + owner_offset(p->n_tensors));
}
static int plan_status(const qerl_adamw_plan* p) {
  if (!p) return QERL_ERR_NULL;
  if (p->chunks < 0 || p->chunks > kMaxChunks || p->n_tensors < 1 || p->elements < 0) return QERL_ERR_SHAPE;
  return p->table ? QERL_OK : QERL_ERR_NULL;
}

}  // namespace qerl

using namespace qerl;

extern "C" size_t lora_adamw_plan_bytes(const qerl_adamw_tensor* tensors, int n_tensors) {
  AdamLayout l;
  return adam_layout(tensors, n_tensors, l) ? l.bytes : 0;
}
extern "C" int64_t lora_adamw_state_elements(const qerl_adamw_tensor* tensors, int n_tensors) {
  AdamLayout l;
  return adam_layout(tensors, n_tensors, l) ? l.elements : -1;
}

extern "C" int lora_adamw_make_plan(const qerl_adamw_tensor* tensors, int n_tensors, void* table, size_t table_bytes,
                                    qerl_adamw_plan* plan, void* stream) {
  if (!tensors || !plan) return QERL_ERR_NULL;
  AdamLayout l;
  if (!adam_layout(tensors, n_tensors, l)) return QERL_ERR_SHAPE;
  for (int i = 0; i < n_tensors; ++i) {
    const qerl_adamw_tensor& t = tensors[i];
    if (t.n == 0) continue;
    if (!t.param_f32 || !t.grad_f32) return QERL_ERR_NULL;
    if (!aligned(t.param_f32, 16) || !aligned(t.grad_f32, 16) || !aligned(t.copy_bf16, 16)) return QERL_ERR_ALIGN;
  }
  if (const int o = overlaps(tensors, n_tensors, nullptr, 0)) return o > 0 ? QERL_ERR_SHAPE : QERL_ERR_WORKSPACE;
  if (!table || table_bytes < l.bytes) return QERL_ERR_WORKSPACE;
  if (!aligned(table, 256)) return QERL_ERR_WORKSPACE;
  const Span own = {(uintptr_t)table, (uintptr_t)table + l.bytes, 1};
  if (const int o = overlaps(tensors, n_tensors, &own, 1)) return o > 0 ? QERL_ERR_SHAPE : QERL_ERR_WORKSPACE;
  AdamTensor* out = reinterpret_cast<AdamTensor*>(static_cast<uint8_t*>(table) + kNormBytes);
  TableBatch batch = {};
  int64_t state0 = 0, chunk0 = 0;
  for (int i = 0; i < n_tensors; ++i) {
    const qerl_adamw_tensor& t = tensors[i];
    batch.t[i % kTableBatch] = AdamTensor{t.param_f32, static_cast<uint16_t*>(t.copy_bf16), t.grad_f32, t.n, state0, chunk0};
    state0 += ceil_div(t.n, kStateBlock) * kStateBlock;
    chunk0 += ceil_div(t.n, kChunk);
    if (i % kTableBatch == kTableBatch - 1 || i == n_tensors - 1)
      adamw_table_kernel<<<dim3(1), dim3(64), 0, (hipStream_t)stream>>>(batch, i % kTableBatch + 1, out + i / kTableBatch * kTableBatch, &static_cast<NormArea*>(table)->arrived);
  }
  *plan = qerl_adamw_plan{table, l.elements, l.chunks, n_tensors};
  if (l.chunks > 0)
    adamw_owner_kernel<<<dim3((unsigned)n_tensors), dim3(256), 0, (hipStream_t)stream>>>(out, const_cast<uint32_t*>(owner_of(plan)));
  return launch_status();
}

static bool apart(const void* a, size_t na, const void* b, size_t nb) {
  const uintptr_t x = (uintptr_t)a, y = (uintptr_t)b;
  return x + na <= y || y + nb <= x;
}
static int state_status(const qerl_adamw_state* s, int64_t elements) {
  if (!s) return QERL_ERR_NULL;
  if (s->bits != 8 && s->bits != 32) return QERL_ERR_SHAPE;
  if (elements == 0) return QERL_OK;
  if (!s->m || !s->v || (s->bits == 8 && (!s->m_scale || !s->v_scale))) return QERL_ERR_NULL;
  if (!aligned(s->m, 16) || !aligned(s->v, 16)) return QERL_ERR_ALIGN;
  const size_t n = (size_t)elements * (s->bits / 8), b = (size_t)elements / kStateBlock;
  if (!apart(s->m, n, s->v, n)) return QERL_ERR_SHAPE;
  if (s->bits == 8 && !(apart(s->m_scale, b, s->v_scale, b) && apart(s->m, n, s->m_scale, b) && apart(s->m, n, s->v_scale, b) &&
                        apart(s->v, n, s->m_scale, b) && apart(s->v, n, s->v_scale, b)))
    return QERL_ERR_SHAPE;
  return QERL_OK;
}

extern "C" int lora_adamw_check_state(const qerl_adamw_tensor* tensors, int n_tensors, const void* table, const qerl_adamw_state* state) {
  if (!tensors || !state) return QERL_ERR_NULL;
  AdamLayout l;
  if (!adam_layout(tensors, n_tensors, l)) return QERL_ERR_SHAPE;
  if (const int e = state_status(state, l.elements)) return e;
  if (l.elements == 0) return QERL_OK;
  const uintptr_t n = (uintptr_t)l.elements * (state->bits / 8), b = state->bits == 8 ? (uintptr_t)l.elements / kStateBlock : 0;
  const auto span = [](const void* p, uintptr_t bytes) { return Span{(uintptr_t)p, (uintptr_t)p + bytes, 1}; };
  const Span others[5] = {span(state->m, n), span(state->v, n), span(state->m_scale, b), span(state->v_scale, b), span(table, table ? l.bytes : 0)};
  const int o = overlaps(tensors, n_tensors, others, 5);
  return o == 0 ? QERL_OK : o > 0 ? QERL_ERR_SHAPE : QERL_ERR_WORKSPACE;
}

extern "C" int lora_adamw_step(const qerl_adamw_plan* plan, const qerl_adamw_state* state, const qerl_adamw_hyper* h, void* stream) {
  if (const int e = plan_status(plan)) return e;
  if (const int e = state_status(state, plan->elements)) return e;
  if (!h) return QERL_ERR_NULL;
  const bool lr_ok = h->lr_device || (isfinite(h->lr) && h->lr >= 0), step_ok = h->step_device || h->step >= 1;
  const float eps = (float)h->eps;                       // as the kernel adds it: 0 would make 0 / 0 of every element without a gradient
  if (!lr_ok || !step_ok || !(h->beta1 >= 0 && h->beta1 < 1) || !(h->beta2 >= 0 && h->beta2 < 1) || !(eps > 0 && isfinite(eps)) ||
      !(h->weight_decay >= 0 && isfinite(h->weight_decay)))
    return QERL_ERR_SHAPE;
  const bool dev = h->lr_device || h->step_device;
  const AdamFactors f = dev ? AdamFactors{} : adam_factors(h->lr, h->beta1, h->beta2, h->weight_decay, h->step);
  if (!isfinite(f.decay) || !isfinite(f.step_size)) return QERL_ERR_SHAPE;
  if (!aligned(h->lr_device, 4) || !aligned(h->step_device, 8) || !aligned(h->grad_scale, 4)) return QERL_ERR_ALIGN;
  if (plan->chunks == 0) return QERL_OK;
  AdamArgs a = {};
  a.table = tensors_of(plan);
  a.owner = owner_of(plan);
  a.m = state->m; a.v = state->v; a.ms = state->m_scale; a.vs = state->v_scale;
  a.b1 = (float)h->beta1; a.omb1 = (float)(1.0 - h->beta1); a.b2 = (float)h->beta2; a.omb2 = (float)(1.0 - h->beta2); a.eps = eps;
  a.lr = h->lr; a.beta1 = h->beta1; a.beta2 = h->beta2; a.wd = h->weight_decay; a.step = h->step;
  a.lr_dev = h->lr_device; a.step_dev = h->step_device; a.grad_scale = h->grad_scale;
  a.k0 = (uint32_t)h->seed; a.k1 = (uint32_t)(h->seed >> 32);
  a.decay = f.decay; a.step_size = f.step_size; a.isb2 = f.isb2;
  const dim3 grid((unsigned)plan->chunks), block(kAdamThreads);
  hipStream_t st = (hipStream_t)stream;
  if (state->bits == 8) {
    if (dev) adamw_kernel<8, true><<<grid, block, 0, st>>>(a);
    else adamw_kernel<8, false><<<grid, block, 0, st>>>(a);
  } else {
    if (dev) adamw_kernel<32, true><<<grid, block, 0, st>>>(a);
    else adamw_kernel<32, false><<<grid, block, 0, st>>>(a);
  }
  return launch_status();
}

extern "C" int lora_adamw_moments(const qerl_adamw_plan* plan, const qerl_adamw_state* state, float* m, float* v, void* stream) {
  if (const int e = plan_status(plan)) return e;
  if (const int e = state_status(state, plan->elements)) return e;
  if (state->bits != 8) return QERL_ERR_SHAPE;
  const int64_t groups = plan->elements / 8;
  if (groups == 0) return QERL_OK;
  if (!m || !v) return QERL_ERR_NULL;
  if (!aligned(m, 16) || !aligned(v, 16)) return QERL_ERR_ALIGN;
  adamw_moments_kernel<<<dim3((unsigned)ceil_div(groups, 256)), dim3(256), 0, (hipStream_t)stream>>>(
      static_cast<const uint8_t*>(state->m), static_cast<const uint8_t*>(state->v), state->m_scale, state->v_scale, groups, m, v);
  return launch_status();
}

extern "C" int lora_adamw_grad_norm(const qerl_adamw_plan* plan, double max_norm, float* norm, float* scale, void* stream) {
  if (const int e = plan_status(plan)) return e;
  if (!scale) return QERL_ERR_NULL;
  if (!(max_norm > 0)) return QERL_ERR_SHAPE;
  if (!aligned(scale, 4) || !aligned(norm, 4)) return QERL_ERR_ALIGN;
  const int n = plan->chunks < 1 ? 1 : (int)(plan->chunks < kNormGroups ? plan->chunks : kNormGroups);
  adamw_norm_kernel<<<dim3((unsigned)n), dim3(256), 0, (hipStream_t)stream>>>(tensors_of(plan), owner_of(plan), plan->chunks, static_cast<NormArea*>(const_cast<void*>(plan->table)),
                                                                           max_norm, norm, scale);
  return launch_status();
}
