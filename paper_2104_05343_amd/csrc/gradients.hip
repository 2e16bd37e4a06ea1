// The norm of the gradients of many tensors, and their clipping.
//   norm = sqrt(sum over tensors and elements of g^2), g the fp32 sum of an element's parts;  scale = min(1, max_norm / norm)
// Squares and their sums are 64 bits: in fp32 a gradient below 1e-19 or above 1e19 would have no square, and a long sum loses digits.
// (An element costs a conversion and a fused multiply-add of full rate, a quarter of what memory takes to deliver it.)  A workgroup adds
// its piece of one tensor, a last one adds the pieces in their order: the same list gives the same bits.
//
// Bound: memory.  The clipping reads the gradients a second time, last ones first: those the norm has read last are in the
// Infinity Cache still.  50 * 10^6 fp32 numbers: 40 us (5.0 TB/s), 5 for the last workgroup, 67 for the clipping (6.0 TB/s of its own bytes),
// 126 for the two calls; 8 * 10^8 in bf16: 312 (5.2), 7, 546 (5.9), 867.
#include <math.h>
#include <stdlib.h>

#include "common.hpp"

namespace optimus {
namespace {

constexpr int kPerLane = 8, kThreads = 256, kStep = kPerLane * kThreads;
constexpr int kTensors = 96;                 // of one launch: its table travels in the kernel's arguments
constexpr int kPieces = 2048;                // aimed at over a whole list: all run at once, eight a compute unit (8192: 7 to 15 us more in the last workgroup)
constexpr long long kLeastPiece = 2 * kStep;
constexpr int kClipSteps = 4;                // of a workgroup of the clipping
constexpr int kFinish = 1024;

struct Job {
  const void* grad;
  void* clipped;
  long long n;
  int parts;
  unsigned char bf16;
};
struct NormArgs {
  long long piece;            // elements of a workgroup, a multiple of kStep
  double* sums;               // [pieces of the list]
  uint2* pieces;              // [tensors of the list]: first piece, how many
  unsigned first_piece;       // of this launch
  int first_tensor;
  int count;
  unsigned first[kTensors];   // first workgroup of each tensor
  Job job[kTensors];
};
struct ClipArgs {
  const float* scale;
  unsigned groups;
  int count;
  unsigned first[kTensors];
  Job job[kTensors];
};
static_assert(sizeof(NormArgs) <= 4000 && sizeof(ClipArgs) <= 4000, "kernel arguments");

typedef __attribute__((ext_vector_type(4), aligned(4))) float f32x4u;   // as found: a slice of a larger buffer starts at any element
typedef __attribute__((ext_vector_type(8), aligned(2))) unsigned short u16x8u;

__device__ __forceinline__ void load8(const float* p, float x[8]) {
  const f32x4u a = *(const f32x4u*)p, b = *(const f32x4u*)(p + 4);
#pragma unroll
  for (int k = 0; k < 4; ++k) { x[k] = a[k]; x[4 + k] = b[k]; }
}
__device__ __forceinline__ void load8(const bf16_t* p, float x[8]) {
  const u16x8u a = *(const u16x8u*)p;
#pragma unroll
  for (int k = 0; k < 8; ++k) x[k] = bf16_to_f32(a[k]);
}
__device__ __forceinline__ float load1(const float* p) { return *p; }
__device__ __forceinline__ float load1(const bf16_t* p) { return bf16_to_f32(*p); }
__device__ __forceinline__ void store8(float* p, const float x[8]) {
  *(f32x4u*)p = f32x4u{x[0], x[1], x[2], x[3]};
  *(f32x4u*)(p + 4) = f32x4u{x[4], x[5], x[6], x[7]};
}
__device__ __forceinline__ void store8(bf16_t* p, const float x[8]) {
  u16x8u a;
#pragma unroll
  for (int k = 0; k < 8; ++k) a[k] = f32_to_bf16(x[k]);
  *(u16x8u*)p = a;
}
__device__ __forceinline__ void store1(float* p, float x) { *p = x; }
__device__ __forceinline__ void store1(bf16_t* p, float x) { *p = f32_to_bf16(x); }

// eight elements from `at` on, `left` of them (from 1 on) inside the tensor, their parts added in order; zeros behind them
template <typename T>
__device__ __forceinline__ void gradient8(const T* g, long long n, int parts, long long at, long long left, float x[8]) {
  if (left >= 8) {
    load8(g + at, x);
    for (int p = 1; p < parts; ++p) {
      float y[8];
      load8(g + p * n + at, y);
#pragma unroll
      for (int k = 0; k < 8; ++k) x[k] += y[k];
    }
  } else {
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      x[k] = 0.f;
      if (k < left) {
        x[k] = load1(g + at + k);
        for (int p = 1; p < parts; ++p) x[k] += load1(g + p * n + at + k);
      }
    }
  }
}

__device__ __forceinline__ double wave_sum(double v) {
#pragma unroll
  for (int step = 1; step < 64; step <<= 1) v += __shfl_xor(v, step);
  return v;
}

template <typename T>
__device__ __forceinline__ double squares(const Job& t, long long from, long long to) {
  double sum[2] = {0.0, 0.0};
  const T* g = (const T*)t.grad;
  long long at = from + (long long)threadIdx.x * kPerLane;
  if (t.parts == 1) {   // four steps in flight
    for (; at + 3 * kStep + 8 <= to; at += 4 * kStep) {
      float x[4][8];
#pragma unroll
      for (int u = 0; u < 4; ++u) load8(g + at + u * kStep, x[u]);
#pragma unroll
      for (int u = 0; u < 4; ++u)
#pragma unroll
        for (int k = 0; k < 8; ++k) sum[k & 1] = fma((double)x[u][k], (double)x[u][k], sum[k & 1]);
    }
  }
  for (; at < to; at += kStep) {
    float x[8];
    gradient8(g, t.n, t.parts, at, to - at, x);
#pragma unroll
    for (int k = 0; k < 8; ++k) sum[k & 1] = fma((double)x[k], (double)x[k], sum[k & 1]);
  }
  return sum[0] + sum[1];
}

// the tensor of a workgroup: the last one that does not start behind it
__device__ __forceinline__ int tensor_of(const unsigned* first, int count, unsigned group) {
  const int lane = threadIdx.x & 63;
  int which = -1;
#pragma unroll
  for (int k = 0; k < kTensors; k += 64) {
    const bool behind = k + lane < count && first[min(k + lane, kTensors - 1)] <= group;
    which += __popcll(__builtin_amdgcn_ballot_w64(behind));
  }
  return __builtin_amdgcn_readfirstlane(which);
}

__global__ __launch_bounds__(kThreads) void norm_kernel(NormArgs a) {
  __shared__ double parts[kThreads / 64];
  const int which = tensor_of(a.first, a.count, blockIdx.x);
  const Job& t = a.job[which];
  const unsigned piece = blockIdx.x - a.first[which];
  const long long from = piece * a.piece, to = min(t.n, from + a.piece);
  const double sum = wave_sum(t.bf16 ? squares<bf16_t>(t, from, to) : squares<float>(t, from, to));
  if ((threadIdx.x & 63) == 0) parts[threadIdx.x >> 6] = sum;
  __syncthreads();
  if (threadIdx.x) return;
  a.sums[a.first_piece + blockIdx.x] = (parts[0] + parts[1]) + (parts[2] + parts[3]);
  if (piece == 0) a.pieces[a.first_tensor + which] = make_uint2(a.first_piece + blockIdx.x, (unsigned)((t.n + a.piece - 1) / a.piece));
}

// One workgroup: the pieces to norms, norm and scale.  A wavefront takes 64 tensors at a time: those of few pieces a lane each, the others
// one after the other with all lanes.
__global__ __launch_bounds__(kFinish) void norm_finish_kernel(const double* sums, const uint2* pieces, int count, float max_norm, float* norm,
                                                              float* scale, float* norms) {
  constexpr int kWaves = kFinish / 64;
  constexpr unsigned kFew = 4;
  __shared__ double parts[kWaves];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  double total = 0.0;
  const int each = min(64, (count + kWaves - 1) / kWaves);   // few tensors: a wavefront fewer of them
  for (int k0 = wave * each; k0 < count; k0 += kWaves * each) {
    const bool mine = lane < each && k0 + lane < count;
    const uint2 p = mine ? pieces[k0 + lane] : make_uint2(0, 0);
    double sum = 0.0;
    if (p.y <= kFew)
      for (unsigned k = 0; k < p.y; ++k) sum += sums[p.x + k];
    unsigned long long many = __builtin_amdgcn_ballot_w64(p.y > kFew);
    while (many) {
      const int k = __builtin_ctzll(many);
      many &= many - 1;
      const unsigned at = __builtin_amdgcn_readlane(p.x, k), number = __builtin_amdgcn_readlane(p.y, k);
      double s[4] = {0.0, 0.0, 0.0, 0.0};
      for (unsigned e = lane; e < number; e += 512) {   // eight loads in flight
        double x[8];
#pragma unroll
        for (int u = 0; u < 8; ++u) x[u] = e + 64 * u < number ? sums[at + e + 64 * u] : 0.0;
#pragma unroll
        for (int u = 0; u < 8; ++u) s[u & 3] += x[u];
      }
      const double all = wave_sum((s[0] + s[1]) + (s[2] + s[3]));
      if (lane == k) sum = all;
    }
    if (mine && norms) norms[k0 + lane] = (float)sqrt(sum);
    total += sum;
  }
  total = wave_sum(total);
  if (lane == 0) parts[wave] = total;
  __syncthreads();
  if (threadIdx.x) return;
  total = 0.0;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) total += parts[w];
  const double x = sqrt(total);
  *norm = (float)x;
  // a sum that is not finite (a gradient that is not) gives NaN, not 0: what it scales would be zeros beside NaN
  if (scale) *scale = !(x <= 1.7976931348623157e308) ? NAN : x > (double)max_norm ? (float)((double)max_norm / x) : 1.0f;
}

template <typename T>
__device__ __forceinline__ void clip(const Job& t, long long from, float scale) {
  const T* g = (const T*)t.grad;
  T* out = (T*)t.clipped;
  const long long at = from + (long long)threadIdx.x * kPerLane;
  float x[kClipSteps][8];
#pragma unroll
  for (int u = 0; u < kClipSteps; ++u) {
    const long long e = at + u * kStep;
    if (e < t.n) gradient8(g, t.n, t.parts, e, t.n - e, x[u]);
  }
#pragma unroll
  for (int u = 0; u < kClipSteps; ++u) {
    const long long e = at + u * kStep, left = t.n - e;
#pragma unroll
    for (int k = 0; k < 8; ++k) x[u][k] *= scale;
    if (left >= 8) {
      store8(out + e, x[u]);
    } else {
#pragma unroll
      for (int k = 0; k < 8; ++k)
        if (k < left) store1(out + e + k, x[u][k]);
    }
  }
}

__global__ __launch_bounds__(kThreads) void clip_kernel(ClipArgs a) {
  const unsigned group = a.groups - 1 - blockIdx.x;   // (the last gradients first)
  const int which = tensor_of(a.first, a.count, group);
  const Job& t = a.job[which];
  const float scale = *a.scale;
  if (scale == 1.0f && t.parts == 1 && t.grad == t.clipped) return;
  const long long from = (long long)(group - a.first[which]) * (kClipSteps * kStep);
  if (t.bf16) clip<bf16_t>(t, from, scale);
  else clip<float>(t, from, scale);
}

struct Range { uintptr_t at, end; bool written; };
int compare_ranges(const void* x, const void* y) {
  const uintptr_t a = ((const Range*)x)->at, b = ((const Range*)y)->at;
  return a < b ? -1 : a > b;
}

// clip: `clipped` is looked at too: every one is its own gradient or meets neither another one nor any gradient
int check(const optimus_gradient* g, int count, bool clip) {
  if (!g) return OPTIMUS_EINVAL;
  if (count < 1 || count > (1 << 16)) return OPTIMUS_ESHAPE;
  for (int k = 0; k < count; ++k) {
    if (!g[k].grad || (clip && !g[k].clipped)) return OPTIMUS_EINVAL;
    if (g[k].dtype != OPTIMUS_BF16 && g[k].dtype != OPTIMUS_FP32) return OPTIMUS_EDTYPE;
    if (g[k].n < 1 || g[k].n > (1ll << 34) || g[k].parts < 1 || g[k].parts > 65536) return OPTIMUS_ESHAPE;
    const uintptr_t e = g[k].dtype == OPTIMUS_BF16 ? 1 : 3;
    if ((uintptr_t)g[k].grad & e || (clip && (uintptr_t)g[k].clipped & e)) return OPTIMUS_EINVAL;
  }
  if (!clip) return OPTIMUS_OK;
  Range few[64];
  Range* r = count <= 32 ? few : (Range*)malloc(sizeof(Range) * 2 * (size_t)count);
  if (!r) return OPTIMUS_EHIP;
  int n = 0;
  for (int k = 0; k < count; ++k) {
    const uintptr_t size = g[k].dtype == OPTIMUS_BF16 ? 2 : 4, one = (uintptr_t)g[k].n * size, from = (uintptr_t)g[k].grad, to = (uintptr_t)g[k].clipped;
    r[n++] = {from, from + one * g[k].parts, from == to};
    if (from != to) r[n++] = {to, to + one, true};
  }
  qsort(r, (size_t)n, sizeof(Range), compare_ranges);
  bool meet = false;
  uintptr_t any = 0, written = 0;   // ends of the ranges so far
  for (int k = 0; k < n; ++k) {
    meet = meet || r[k].at < written || (r[k].written && r[k].at < any);
    if (r[k].end > any) any = r[k].end;
    if (r[k].written && r[k].end > written) written = r[k].end;
  }
  if (r != few) free(r);
  return meet ? OPTIMUS_EINVAL : OPTIMUS_OK;
}

// Elements of a workgroup: by the whole list, so that a long one has as many pieces as the last workgroup adds in a few microseconds
long long piece_of(const optimus_gradient* g, int count) {
  long long total = 0;
  for (int k = 0; k < count; ++k) total += g[k].n * g[k].parts / kPieces + 1;
  const long long piece = (total + kStep - 1) / kStep * kStep;
  return piece < kLeastPiece ? kLeastPiece : piece;
}
long long pieces_of(const optimus_gradient* g, int count, long long piece) {
  long long sum = 0;
  for (int k = 0; k < count; ++k) sum += (g[k].n + piece - 1) / piece;
  return sum;
}
Job job_of(const optimus_gradient& g) { return {g.grad, g.clipped, (long long)g.n, g.parts, (unsigned char)(g.dtype == OPTIMUS_BF16)}; }

}  // namespace
}  // namespace optimus

using namespace optimus;

extern "C" size_t optimus_gradient_norm_workspace_bytes(const optimus_gradient* gradients, int count) {
  if (check(gradients, count, false)) return 0;
  return (size_t)(pieces_of(gradients, count, piece_of(gradients, count)) + count) * 8;
}

extern "C" int optimus_gradient_norm(const optimus_gradient* gradients, int count, float max_norm, float* norm, float* scale, float* norms, void* ws,
                                     size_t ws_bytes, void* stream) {
  if (!norm || ((uintptr_t)norm | (uintptr_t)scale | (uintptr_t)norms) & 3) return OPTIMUS_EINVAL;
  if (const int rc = check(gradients, count, false)) return rc;
  if (!(max_norm > 0)) return OPTIMUS_EINVAL;
  const long long piece = piece_of(gradients, count), pieces = pieces_of(gradients, count, piece);
  if (!ws || ws_bytes < (size_t)(pieces + count) * 8 || (uintptr_t)ws & 7) return OPTIMUS_EWORKSPACE;
  const hipStream_t st = (hipStream_t)stream;
  NormArgs a = {};
  a.piece = piece;
  a.sums = (double*)ws;
  a.pieces = (uint2*)(a.sums + pieces);
  for (int k = 0; k < count;) {
    unsigned groups = 0;
    a.first_tensor = k;
    for (a.count = 0; k < count && a.count < kTensors; ++k, ++a.count) {
      a.job[a.count] = job_of(gradients[k]);
      a.first[a.count] = groups;
      groups += (unsigned)((gradients[k].n + piece - 1) / piece);
    }
    norm_kernel<<<groups, kThreads, 0, st>>>(a);
    if (const int rc = hip_launch_status()) return rc;
    a.first_piece += groups;
  }
  norm_finish_kernel<<<1, kFinish, 0, st>>>(a.sums, a.pieces, count, max_norm, norm, scale, norms);
  return hip_launch_status();
}

extern "C" int optimus_gradient_clip(const optimus_gradient* gradients, int count, const float* scale, void* stream) {
  if (!scale || (uintptr_t)scale & 3) return OPTIMUS_EINVAL;
  if (const int rc = check(gradients, count, true)) return rc;
  const hipStream_t st = (hipStream_t)stream;
  ClipArgs a = {};
  a.scale = scale;
  constexpr long long own = kClipSteps * kStep, most = (1ll << 32) / kThreads - 1;   // (2^32 threads of a launch)
  for (int k = count; k > 0;) {   // the last tensors first
    int from = k;
    long long groups = 0;
    while (from > 0 && k - from < kTensors) {
      const long long more = (gradients[from - 1].n + own - 1) / own;   // at most 2^21
      if (groups > 0 && groups + more > most) break;
      groups += more;
      --from;
    }
    a.count = k - from;
    unsigned first = 0;
    for (int e = 0; e < a.count; ++e) {
      a.job[e] = job_of(gradients[from + e]);
      a.first[e] = first;
      first += (unsigned)((gradients[from + e].n + own - 1) / own);
    }
    a.groups = first;
    clip_kernel<<<first, kThreads, 0, st>>>(a);
    if (const int rc = hip_launch_status()) return rc;
    k = from;
  }
  return OPTIMUS_OK;
}
