// One AdamW step over many tensors.  Per element, in fp32:
//   g = grad_scale * sum of the gradient's parts;  m = b1 m + (1 - b1) g;  v = b2 v + (1 - b2) g^2;
//   w = w - (lr / (1 - b1^t) * m / (sqrt(v / (1 - b2^t)) + eps) + lr * decay * w)
// every product and sum rounded by itself (no contraction), so that a step has the same bits however it is compiled.  The decay is
// subtracted together with the update instead of scaling w by 1 - lr * decay, which fp32 cannot tell from 1 closely enough.
//
// Moments of 8 bits: e4m3 numbers, 128 consecutive ones sharing a power of two (a byte e: 2^(e - 127)) that brings the largest to at
// most 448.  They are rounded up or down at random, in proportion to their place between the two neighbours: v changes by one part
// in a thousand a step and its numbers are an eighth apart, so rounded to nearest it would never move.  A v above zero stays
// above zero, or the next step divided by eps alone.  bf16 weights without an fp32 copy are rounded the same way, for the same
// reason.  The random bits are a hash of (seed, step, tensor, element): no state, and the same call gives the same bits.
#include <math.h>
#include <stdlib.h>

#include "common.hpp"

namespace optimus {
namespace {

constexpr int kGroup = 128;                    // elements that share a scale
constexpr int kPerLane = 8, kThreads = 256;
constexpr int kChunk = kPerLane * kThreads;    // elements of a workgroup
constexpr long long kMostGroups = (1ll << 32) / kThreads - 1;   // of a launch: 2^32 threads
constexpr int kTensors = 40;                   // of one launch: its table travels in the kernel's arguments (4 KiB at most)

struct AdamwJob {
  void* param;
  float* master;
  const void* grad;
  void* m;
  void* v;
  unsigned char* m_scale;   // 8-bit moments
  unsigned char* v_scale;
  long long n;
  unsigned key;             // hash of (seed, tensor)
  float decay, shrink;      // shrink: lr * decay of the host's rate
  int parts;
  unsigned char param_bf16, grad_bf16;
};
struct AdamwArgs {
  float b1, b2, c1, c2, eps;      // c = 1 - b
  float lr, step_size, root;      // lr / (1 - b1^t), 1 / sqrt(1 - b2^t): of the host's step and rate
  double log_b1, log_b2;
  long long step;
  const float* grad_scale;
  const float* lr_dev;
  const long long* step_dev;
  int count;
  unsigned first[kTensors];       // first workgroup of each tensor
  AdamwJob job[kTensors];
};
static_assert(sizeof(AdamwArgs) <= 4000, "kernel arguments");

// 32-bit hash: two multiplications by odd constants (fractional bits of the golden ratio and of the root of 3) between shifts
__host__ __device__ inline unsigned mix(unsigned x) {
  x ^= x >> 16;
  x *= 0x9E3779B1u;
  x ^= x >> 15;
  x *= 0xBB67AE85u;
  return x ^ (x >> 16);
}

typedef __attribute__((ext_vector_type(4), aligned(4))) float f32x4u;     // as found: a slice of a larger buffer starts at any element
typedef __attribute__((ext_vector_type(8), aligned(2))) unsigned short u16x8u;
typedef __attribute__((ext_vector_type(2), aligned(1))) unsigned u32x2u;

// eight elements of a lane, `left` of them inside the tensor
__device__ __forceinline__ void load_f32(const float* p, int left, float x[8]) {
  if (left >= 8) {
    const f32x4u a = *(const f32x4u*)p, b = *(const f32x4u*)(p + 4);
#pragma unroll
    for (int k = 0; k < 4; ++k) { x[k] = a[k]; x[4 + k] = b[k]; }
  } else {
#pragma unroll
    for (int k = 0; k < 8; ++k) x[k] = k < left ? p[k] : 0.f;
  }
}
__device__ __forceinline__ void store_f32(float* p, int left, const float x[8]) {
  if (left >= 8) {
    *(f32x4u*)p = f32x4u{x[0], x[1], x[2], x[3]};
    *(f32x4u*)(p + 4) = f32x4u{x[4], x[5], x[6], x[7]};
  } else {
#pragma unroll
    for (int k = 0; k < 8; ++k)
      if (k < left) p[k] = x[k];
  }
}
__device__ __forceinline__ void load_bf16(const bf16_t* p, int left, float x[8]) {
  if (left >= 8) {
    const u16x8u a = *(const u16x8u*)p;
#pragma unroll
    for (int k = 0; k < 8; ++k) x[k] = bf16_to_f32(a[k]);
  } else {
#pragma unroll
    for (int k = 0; k < 8; ++k) x[k] = k < left ? bf16_to_f32(p[k]) : 0.f;
  }
}
__device__ __forceinline__ void store_bits16(bf16_t* p, int left, const bf16_t x[8]) {
  if (left >= 8) {
    u16x8u a;
#pragma unroll
    for (int k = 0; k < 8; ++k) a[k] = x[k];
    *(u16x8u*)p = a;
  } else {
#pragma unroll
    for (int k = 0; k < 8; ++k)
      if (k < left) p[k] = x[k];
  }
}
__device__ __forceinline__ u32x2u load_bytes(const unsigned char* p, int left) {
  if (left >= 8) return *(const u32x2u*)p;
  u32x2u w = {0, 0};
#pragma unroll
  for (int k = 0; k < 8; ++k)
    if (k < left) w[k >> 2] |= (unsigned)p[k] << (8 * (k & 3));
  return w;
}
__device__ __forceinline__ void store_bytes(unsigned char* p, int left, u32x2u w) {
  if (left >= 8) {
    *(u32x2u*)p = w;
  } else {
#pragma unroll
    for (int k = 0; k < 8; ++k)
      if (k < left) p[k] = (unsigned char)(w[k >> 2] >> (8 * (k & 3)));
  }
}

// 2^(byte - 127); 255 stands for NaN, 0 for a number below the normal ones
__device__ __forceinline__ float scale_of(unsigned byte) {
  return __uint_as_float(byte == 255 ? 0x7FC00000u : byte == 0 ? 0x00400000u : byte << 23);
}
__device__ __forceinline__ void unpack8(u32x2u w, float scale, float x[8]) {
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    x[4 * h + 0] = __builtin_amdgcn_cvt_f32_fp8((int)w[h], 0) * scale;
    x[4 * h + 1] = __builtin_amdgcn_cvt_f32_fp8((int)w[h], 1) * scale;
    x[4 * h + 2] = __builtin_amdgcn_cvt_f32_fp8((int)w[h], 2) * scale;
    x[4 * h + 3] = __builtin_amdgcn_cvt_f32_fp8((int)w[h], 3) * scale;
  }
}
// largest of the 16 lanes of a row, in all of them (a rotation by 8, 4, 2 and 1)
__device__ __forceinline__ unsigned row_max(unsigned x) {
  x = max(x, (unsigned)__builtin_amdgcn_update_dpp(0, (int)x, 0x128, 0xf, 0xf, false));
  x = max(x, (unsigned)__builtin_amdgcn_update_dpp(0, (int)x, 0x124, 0xf, 0xf, false));
  x = max(x, (unsigned)__builtin_amdgcn_update_dpp(0, (int)x, 0x122, 0xf, 0xf, false));
  return max(x, (unsigned)__builtin_amdgcn_update_dpp(0, (int)x, 0x121, 0xf, 0xf, false));
}
// The group's byte of scale and the lane's eight numbers.  dither: 16 random bits each.  A group whose largest magnitude is not finite
// gets 255, NaN for all of it.
template <bool POSITIVE>
__device__ __forceinline__ u32x2u pack8(const float x[8], const unsigned dither[8], unsigned* scale_byte) {
  unsigned most = 0;
#pragma unroll
  for (int k = 0; k < 8; ++k) most = max(most, __float_as_uint(x[k]) & 0x7FFFFFFFu);   // NaN above infinity above the rest
  most = row_max(most);
  // 448 = 1.75 * 2^8: a fraction above 0.75 takes the next power
  const bool bad = most >= 0x7F800000u;
  const int byte = max((int)((most + 0x1FFFFFu) >> 23) - 8, 0);
  *scale_byte = bad ? 255u : (unsigned)byte;
  const float inverse = bad ? 0.f : __uint_as_float((unsigned)(254 - byte) << 23);
  u32x2u w = {0, 0};
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    const float a = bad ? 0.f : fabsf(x[k]) * inverse;
    const unsigned normal = ((__float_as_uint(a) + (dither[k] << 4)) >> 20) - (120u << 3);
    const unsigned small = ((unsigned)(a * 33554432.0f) + dither[k]) >> 16;   // below 2^-6 the numbers are 2^-9 apart
    unsigned code = a >= 0.015625f ? normal : small;
    if (POSITIVE) code = x[k] > 0.f && code == 0 ? 1u : code;
    else code |= x[k] < 0.f && code != 0 ? 128u : 0u;
    w[k >> 2] |= code << (8 * (k & 3));
  }
  return w;
}

// EXACT: root and division are rounded exactly.  Otherwise root and reciprocal are of one unit in the last place, a 4e-7th of the update,
// which w's own rounding hides (25 operations less, and with 8-bit moments and two hashes an element the arithmetic is what counts).  They
// take numbers below 2^-126 for 0, so that a root below 2^-63 is lost, up to 2^-63 / sqrt(1 - beta2) of what eps is added to: as small a
// part of the update where eps is 2^-42 / sqrt(1 - beta2) or more (beta2 = 0.999: 7e-12), all of it beside a tiny eps.
template <bool EXACT>
__global__ __launch_bounds__(kThreads) void adamw_kernel(AdamwArgs a) {
#pragma clang fp contract(off)
  // the tensor of this workgroup: the last one that does not start behind it
  const int lane = threadIdx.x & 63;
  const bool behind = lane < a.count && a.first[min(lane, kTensors - 1)] <= blockIdx.x;
  const int which = __builtin_amdgcn_readfirstlane(__popcll(__builtin_amdgcn_ballot_w64(behind)) - 1);
  const AdamwJob& t = a.job[which];
  float step_size = a.step_size, root = a.root, lr = a.lr;
  long long step = a.step;
  if (a.lr_dev) lr = *a.lr_dev;
  if (a.step_dev) {
    step = *a.step_dev;
    root = (float)(1.0 / sqrt(-expm1((double)step * a.log_b2)));
  }
  if (a.lr_dev || a.step_dev) step_size = (float)((double)lr / -expm1((double)step * a.log_b1));
  const float shrink = a.lr_dev ? lr * t.decay : t.shrink, gs = a.grad_scale ? *a.grad_scale : 1.0f;
  const unsigned key = mix(mix(t.key + (unsigned)step) ^ (unsigned)(step >> 32));

  const long long e0 = (long long)(blockIdx.x - a.first[which]) * kChunk + (long long)threadIdx.x * kPerLane;
  const int left = (int)min(max(t.n - e0, 0ll), 8ll);
  if (__builtin_amdgcn_ballot_w64(left > 0) == 0) return;
  const long long at = left > 0 ? e0 : 0;

  float g[8], m[8], v[8], w[8];
  if (t.grad_bf16) load_bf16((const bf16_t*)t.grad + at, left, g);
  else load_f32((const float*)t.grad + at, left, g);
  for (int part = 1; part < t.parts; ++part) {
    float x[8];
    if (t.grad_bf16) load_bf16((const bf16_t*)t.grad + part * t.n + at, left, x);
    else load_f32((const float*)t.grad + part * t.n + at, left, x);
#pragma unroll
    for (int k = 0; k < 8; ++k) g[k] += x[k];
  }
  if (t.m_scale) {
    const u32x2u mw = load_bytes((const unsigned char*)t.m + at, left), vw = load_bytes((const unsigned char*)t.v + at, left);
    unpack8(mw, scale_of(t.m_scale[at / kGroup]), m);
    unpack8(vw, scale_of(t.v_scale[at / kGroup]), v);
  } else {
    load_f32((const float*)t.m + at, left, m);
    load_f32((const float*)t.v + at, left, v);
  }
  if (t.master) load_f32(t.master + at, left, w);
  else if (t.param_bf16) load_bf16((const bf16_t*)t.param + at, left, w);
  else load_f32((const float*)t.param + at, left, w);

#pragma unroll
  for (int k = 0; k < 8; ++k) {
    const float gk = a.grad_scale ? g[k] * gs : g[k];
    m[k] = a.b1 * m[k] + a.c1 * gk;
    v[k] = a.b2 * v[k] + a.c2 * (gk * gk);
    const float move = EXACT ? m[k] / (sqrtf(v[k]) * root + a.eps) : m[k] * __builtin_amdgcn_rcpf(__builtin_amdgcn_sqrtf(v[k]) * root + a.eps);
    w[k] = w[k] - (step_size * move + shrink * w[k]);
  }

  unsigned hash[8];
  const unsigned high = (unsigned)(e0 >> 32) * 0x9E3779B1u;
#pragma unroll
  for (int k = 0; k < 8; ++k) hash[k] = mix((((unsigned)e0 + k) + high) ^ key);
  if (t.m_scale) {
    if (left < 8) {   // what lies behind the tensor has no part in its last group's scale
#pragma unroll
      for (int k = 0; k < 8; ++k)
        if (k >= left) m[k] = v[k] = 0.f;
    }
    unsigned dm[8], dv[8], ms, vs;
#pragma unroll
    for (int k = 0; k < 8; ++k) { dm[k] = hash[k] >> 16; dv[k] = hash[k] & 0xFFFFu; }
    const u32x2u mw = pack8<false>(m, dm, &ms), vw = pack8<true>(v, dv, &vs);
    store_bytes((unsigned char*)t.m + at, left, mw);
    store_bytes((unsigned char*)t.v + at, left, vw);
    if ((lane & 15) == 0 && left > 0) {
      t.m_scale[at / kGroup] = (unsigned char)ms;
      t.v_scale[at / kGroup] = (unsigned char)vs;
    }
  } else {
    store_f32((float*)t.m + at, left, m);
    store_f32((float*)t.v + at, left, v);
  }
  if (!t.param_bf16) {
    store_f32((float*)t.param + at, left, w);
  } else {
    bf16_t p[8];
    if (t.master) {
      store_f32(t.master + at, left, w);
#pragma unroll
      for (int k = 0; k < 8; ++k) p[k] = f32_to_bf16(w[k]);
    } else {
#pragma unroll
      for (int k = 0; k < 8; ++k) {   // up where the 16 bits below bf16 and as many random ones carry; infinities and NaN as they are
        const unsigned b = __float_as_uint(w[k]);
        const bool finite = (b & 0x7F800000u) != 0x7F800000u;
        p[k] = finite ? (bf16_t)((b + (mix(hash[k] ^ 0x6A09E667u) & 0xFFFFu)) >> 16) : f32_to_bf16(w[k]);
      }
    }
    store_bits16((bf16_t*)t.param + at, left, p);
  }
}

// memory [p, p + bytes) of the parameters: no two tensors' may meet
struct Range { uintptr_t at, end; };
int compare_ranges(const void* x, const void* y) {
  const uintptr_t a = ((const Range*)x)->at, b = ((const Range*)y)->at;
  return a < b ? -1 : a > b;
}

int check_tensor(const optimus_adamw_tensor& t) {
  if (!t.param || !t.grad || !t.m || !t.v) return OPTIMUS_EINVAL;
  if ((t.m_scale == nullptr) != (t.v_scale == nullptr)) return OPTIMUS_EINVAL;
  if ((t.param_dtype != OPTIMUS_BF16 && t.param_dtype != OPTIMUS_FP32) || (t.grad_dtype != OPTIMUS_BF16 && t.grad_dtype != OPTIMUS_FP32))
    return OPTIMUS_EDTYPE;
  if (t.master && t.param_dtype != OPTIMUS_BF16) return OPTIMUS_EINVAL;
  if (t.n < 1 || t.n > (1ll << 34) || t.grad_parts < 1 || t.grad_parts > 65536) return OPTIMUS_ESHAPE;
  if (!isfinite(t.weight_decay)) return OPTIMUS_EINVAL;
  const uintptr_t pe = t.param_dtype == OPTIMUS_BF16 ? 1 : 3, ge = t.grad_dtype == OPTIMUS_BF16 ? 1 : 3, me = t.m_scale ? 0 : 3;
  if ((uintptr_t)t.param & pe || (uintptr_t)t.grad & ge || ((uintptr_t)t.m | (uintptr_t)t.v) & me || (uintptr_t)t.master & 3) return OPTIMUS_EINVAL;
  return OPTIMUS_OK;
}

}  // namespace

int adamw_check(const optimus_adamw_cfg* cfg, const optimus_adamw_tensor* tensors, int count) {
  if (!cfg || !tensors) return OPTIMUS_EINVAL;
  if (count < 1 || count > (1 << 20)) return OPTIMUS_ESHAPE;
  if (!isfinite(cfg->lr) || !(cfg->beta1 >= 0 && cfg->beta1 < 1) || !(cfg->beta2 >= 0 && cfg->beta2 < 1) || !((float)cfg->eps > 0) || !isfinite(cfg->eps) ||
      (cfg->step < 1 && !cfg->step_on_device))
    return OPTIMUS_EINVAL;
  for (int k = 0; k < count; ++k)
    if (const int rc = check_tensor(tensors[k])) return rc;
  Range few[64];
  Range* r = count <= 64 ? few : (Range*)malloc(sizeof(Range) * (size_t)count);
  if (!r) return OPTIMUS_EHIP;
  for (int k = 0; k < count; ++k) {
    r[k].at = (uintptr_t)tensors[k].param;
    r[k].end = r[k].at + (uintptr_t)tensors[k].n * (tensors[k].param_dtype == OPTIMUS_BF16 ? 2 : 4);
  }
  qsort(r, (size_t)count, sizeof(Range), compare_ranges);
  bool meet = false;
  for (int k = 1; k < count; ++k) meet = meet || r[k].at < r[k - 1].end;
  if (r != few) free(r);
  return meet ? OPTIMUS_EINVAL : OPTIMUS_OK;
}

int adamw_launch(const optimus_adamw_cfg* cfg, unsigned long long seed, const optimus_adamw_tensor* tensors, int count, hipStream_t st) {
  AdamwArgs a = {};
  a.b1 = (float)cfg->beta1; a.b2 = (float)cfg->beta2; a.c1 = (float)(1.0 - cfg->beta1); a.c2 = (float)(1.0 - cfg->beta2);
  a.eps = (float)cfg->eps; a.lr = (float)cfg->lr;
  a.log_b1 = log(cfg->beta1); a.log_b2 = log(cfg->beta2);
  a.step = cfg->step;
  if (!cfg->step_on_device) {
    a.step_size = (float)(cfg->lr / -expm1((double)cfg->step * a.log_b1));
    a.root = (float)(1.0 / sqrt(-expm1((double)cfg->step * a.log_b2)));
  }
  a.grad_scale = cfg->grad_scale; a.lr_dev = cfg->lr_on_device; a.step_dev = (const long long*)cfg->step_on_device;
  const bool exact = cfg->eps * sqrt(1.0 - cfg->beta2) < 0x1p-42;
  for (int k = 0; k < count;) {
    unsigned groups = 0;
    a.count = 0;
    while (k < count && a.count < kTensors) {
      const optimus_adamw_tensor& t = tensors[k];
      const long long own = (t.n + kChunk - 1) / kChunk;   // at most 2^23
      if (a.count > 0 && groups + own > kMostGroups) break;
      AdamwJob& j = a.job[a.count];
      j = {t.param, t.master, t.grad, t.m, t.v, t.m_scale, t.v_scale, (long long)t.n, 0, 0.f, 0.f, t.grad_parts, 0, 0};
      j.key = mix(mix((unsigned)seed + 0x9E3779B1u * (unsigned)(k + 1)) ^ (unsigned)(seed >> 32));
      j.decay = t.weight_decay;
      j.shrink = (float)(cfg->lr * t.weight_decay);
      j.param_bf16 = t.param_dtype == OPTIMUS_BF16;
      j.grad_bf16 = t.grad_dtype == OPTIMUS_BF16;
      a.first[a.count++] = groups;
      groups += (unsigned)own;
      ++k;
    }
    if (exact) adamw_kernel<true><<<groups, kThreads, 0, st>>>(a);   // (a kernel of its own: one that chose took 520 us for 486)
    else adamw_kernel<false><<<groups, kThreads, 0, st>>>(a);
    if (const int rc = hip_launch_status()) return rc;
  }
  return OPTIMUS_OK;
}

}  // namespace optimus

using namespace optimus;

extern "C" int optimus_adamw_step(const optimus_adamw_cfg* cfg, const optimus_adamw_tensor* tensors, int count, void* stream) {
  if (const int rc = adamw_check(cfg, tensors, count)) return rc;
  return adamw_launch(cfg, cfg->seed, tensors, count, (hipStream_t)stream);
}
