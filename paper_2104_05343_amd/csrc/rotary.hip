// Rotary positions on the queries and keys of qkv blocks.  Pair p of a head's leading 2P elements turns by the angle
//   a = position[axis(p)][token] * turn[p]      (in revolutions; turn = scale * frequency / (2 pi), 64 bits)
//   (x, y) -> (x cos a - y sin a, x sin a + y cos a);   the gradient is the same with -a.
// The angle is a product in 64 bits, less its whole revolutions, before it becomes fp32: a position of 10^6 times a frequency of 1 has
// six digits in front of the point, and fp32 would keep one behind it.  Cosine and sine are fp32, the rotation is fp32, one rounding.
//
// Bound: memory (two of three parts of qkv read and written in place, all of it into another matrix): 4 x 16384 x 3 * 1024 in bf16, three axes, 151 us,
// 5.3 TB/s; 2048 rows of 8 heads of 128 in place 5.3 us, of which a launch is most; one token of eight sequences 3.8.  A token's angles serve every
// head's query and key, so a workgroup computes them once for its tokens, into LDS, and then walks over (head, query or key, chunk of
// up to 16 bytes); a chunk's partners lie P elements further, or beside it.
#include <math.h>

#include "common.hpp"

namespace optimus {
namespace {

constexpr int kThreads = 256, kMaxPairs = 128, kMaxAxes = 4, kTable = 1024;   // kTable: angles of a workgroup

struct RotaryArgs {
  const void* x;
  void* y;
  const int* positions;      // [axes][sequences of the grid * s]
  long long rows;            // of a device
  long long all_rows;
  long long dev;             // elements of a device's block
  int q, dev0, ld, d, nh, pairs;
  int tokens;                // of a workgroup
  int chunks;                // of a head's pairs
  int copies;                // chunks of a head that only move (another matrix)
  unsigned by_token, by_chunks, by_copies, by_pairs, by_head_copies;   // ceil(2^32 / number): division by a product
  float sign;
  double turn[kMaxPairs];    // revolutions of one step of the position
  unsigned char axis[kMaxPairs];
};
static_assert(sizeof(RotaryArgs) <= 4000, "kernel arguments");

// u / n for m = ceil(2^32 / n): exact while u * n <= 2^32 (m is less than n / 2^32 of itself too large); n = 1 has m = 0, m = 1 gives 0
__device__ __forceinline__ unsigned divide(unsigned u, unsigned m) { return m ? __umulhi(u, m) : u; }

template <typename T, int E> struct Chunk;   // E elements as found in memory: a matrix may start at any element
template <int E> struct Chunk<bf16_t, E> {
  typedef __attribute__((ext_vector_type(E), aligned(2))) unsigned short V;
  __device__ static void move(const bf16_t* p, bf16_t* to) { *(V*)to = *(const V*)p; }
  __device__ static void load(const bf16_t* p, float f[E]) {
    const V v = *(const V*)p;
#pragma unroll
    for (int k = 0; k < E; ++k) f[k] = bf16_to_f32(v[k]);
  }
  __device__ static void store(bf16_t* p, const float f[E]) {
    V v;
#pragma unroll
    for (int k = 0; k < E; ++k) v[k] = f32_to_bf16(f[k]);
    *(V*)p = v;
  }
};
template <> struct Chunk<bf16_t, 1> {
  __device__ static void move(const bf16_t* p, bf16_t* to) { *to = *p; }
  __device__ static void load(const bf16_t* p, float f[1]) { f[0] = bf16_to_f32(*p); }
  __device__ static void store(bf16_t* p, const float f[1]) { *p = f32_to_bf16(f[0]); }
};
template <int E> struct Chunk<float, E> {
  typedef __attribute__((ext_vector_type(E), aligned(4))) float V;
  __device__ static void move(const float* p, float* to) { *(V*)to = *(const V*)p; }
  __device__ static void load(const float* p, float f[E]) {
    const V v = *(const V*)p;
#pragma unroll
    for (int k = 0; k < E; ++k) f[k] = v[k];
  }
  __device__ static void store(float* p, const float f[E]) {
    V v;
#pragma unroll
    for (int k = 0; k < E; ++k) v[k] = f[k];
    *(V*)p = v;
  }
};
template <> struct Chunk<float, 1> {
  __device__ static void move(const float* p, float* to) { *to = *p; }
  __device__ static void load(const float* p, float f[1]) { f[0] = *p; }
  __device__ static void store(float* p, const float f[1]) { *p = f[0]; }
};

// E: elements of a chunk.  BESIDE: a pair is two neighbours (E even, a chunk holds E / 2 pairs); otherwise P elements apart.
template <typename T, int E, bool BESIDE>
__global__ __launch_bounds__(kThreads) void rotary_kernel(RotaryArgs a) {
  __shared__ __attribute__((aligned(16))) float2 table[kTable];   // [token][pair]: cosine, sine
  const int tid = threadIdx.x, P = a.pairs;
  const long long row0 = (long long)blockIdx.x * a.tokens;
  const int tokens = (int)min((long long)a.tokens, a.rows - row0);
  const int dev = a.dev0 + blockIdx.y;
  const int* positions = a.positions + (dev / a.q) * a.rows + row0;
  for (int u = tid; u < tokens * P; u += kThreads) {
    const int token = (int)divide(u, a.by_pairs), p = u - token * P;
    double r = (double)positions[a.axis[p] * a.all_rows + token] * a.turn[p];
    r -= rint(r);
    float s, c;
    sincospif(2.0f * (float)r, &s, &c);
    table[u] = make_float2(c, a.sign * s);
  }
  __syncthreads();
  const long long base = blockIdx.y * a.dev + row0 * a.ld;
  const T* X = (const T*)a.x + base;
  T* Y = (T*)a.y + base;
  const int turned = 2 * a.nh * a.chunks;   // chunks (or pairs of them) of a token
  for (int u = tid; u < tokens * turned; u += kThreads) {
    const int token = (int)divide(u, a.by_token), v = u - token * turned;
    const int head2 = (int)divide(v, a.by_chunks), chunk = v - head2 * a.chunks;
    const int at = token * a.ld + ((head2 >> 1) * 3 + (head2 & 1)) * a.d + chunk * E;
    if (BESIDE) {
      const float2* t = table + token * P + chunk * (E / 2);
      float f[E];
      Chunk<T, E>::load(X + at, f);
#pragma unroll
      for (int k = 0; k < E / 2; ++k) {
        const float c = t[k].x, s = t[k].y, x = f[2 * k], y = f[2 * k + 1];
        f[2 * k] = fmaf(x, c, -(y * s));
        f[2 * k + 1] = fmaf(x, s, y * c);
      }
      Chunk<T, E>::store(Y + at, f);
    } else {
      const float2* t = table + token * P + chunk * E;
      float f[E], g[E];
      Chunk<T, E>::load(X + at, f);
      Chunk<T, E>::load(X + at + P, g);
#pragma unroll
      for (int k = 0; k < E; ++k) {
        const float c = t[k].x, s = t[k].y, x = f[k], y = g[k];
        f[k] = fmaf(x, c, -(y * s));
        g[k] = fmaf(x, s, y * c);
      }
      Chunk<T, E>::store(Y + at, f);
      Chunk<T, E>::store(Y + at + P, g);
    }
  }
  // what does not turn: the rest of a head's query and key, its value
  const int moved = a.nh * a.copies, rest = (a.d - 2 * P) / E;
  for (int u = tid; u < tokens * moved; u += kThreads) {
    const int token = (int)divide(u, a.by_copies), v = u - token * moved;
    const int head = (int)divide(v, a.by_head_copies), c = v - head * a.copies;
    const int in_head = c < 2 * rest ? (c >= rest ? a.d - rest * E : 0) + 2 * P + c * E : 2 * a.d + (c - 2 * rest) * E;
    const int at = token * a.ld + head * 3 * a.d + in_head;
    Chunk<T, E>::move(X + at, Y + at);
  }
}

// base^(-k / n) as a product of two powers, k = 8 a + r: a power is 28 ns of a call that takes 8 us, 64 of them were 1.8
struct Ladder {
  double fine[8], coarse[kMaxPairs / 8];
  void make(double base, int n) {
    fine[0] = coarse[0] = 1.0;
    for (int k = 1; k < 8 && k < n; ++k) fine[k] = pow(base, -(double)k / n);
    for (int k = 1; 8 * k < n; ++k) coarse[k] = pow(base, -(double)(8 * k) / n);
  }
  double at(int k) const { return fine[k & 7] * coarse[k >> 3]; }
};

unsigned reciprocal(int n) { return n <= 1 ? 0u : (unsigned)(((1ull << 32) + n - 1) / n); }

template <typename T, int E>
void launch(const RotaryArgs& a, bool beside, dim3 grid, hipStream_t st) {
  if constexpr (E > 1) {
    if (beside) {
      rotary_kernel<T, E, true><<<grid, kThreads, 0, st>>>(a);
      return;
    }
  }
  rotary_kernel<T, E, false><<<grid, kThreads, 0, st>>>(a);
}

int run(const void* x, void* y, int b, int s, int h, int n, int q, int i, int j, int dtype, const optimus_rotary_axes* r, bool back, void* stream) {
  if (!x || !y || !r || !r->positions) return OPTIMUS_EINVAL;
  if (dtype != OPTIMUS_BF16 && dtype != OPTIMUS_FP32) return OPTIMUS_EDTYPE;
  if (q <= 0 || !fits_int(h, q) || b <= 0 || s <= 0 || h <= 0 || n <= 0 || b % q || n % q || h % n) return OPTIMUS_ESHAPE;
  const bool all = i == OPTIMUS_ALL && j == OPTIMUS_ALL;
  if (!all && (i < 0 || j < 0 || i >= q || j >= q)) return OPTIMUS_ECOORD;
  if (r->axes < 1 || r->axes > kMaxAxes || !(r->base > 0) || !isfinite(r->base)) return OPTIMUS_EINVAL;
  RotaryArgs a = {};
  int left[kMaxAxes] = {}, done[kMaxAxes] = {};
  for (int k = 0; k < r->axes; ++k) {
    if (r->pairs[k] < 1 || r->pairs[k] > kMaxPairs) return OPTIMUS_ESHAPE;
    if (!isfinite(r->scale[k])) return OPTIMUS_EINVAL;
    left[k] = r->pairs[k];
    a.pairs += left[k];
  }
  a.d = h / n;
  a.nh = n / q;
  // (the divisions by products are exact up to here: at most 2^18 chunks of a token, 2^14 of a head)
  if (a.pairs > kMaxPairs || 2 * a.pairs > a.d || a.d > 4096 || 3ll * h / q > (1 << 18)) return OPTIMUS_ESHAPE;
  a.ld = 3 * h / q;
  a.rows = (long long)(b / q) * s;
  a.all_rows = (long long)b * s;
  a.dev = a.rows * a.ld;
  a.q = q;
  a.dev0 = all ? 0 : i * q + j;
  const int ndev = all ? q * q : 1;
  if (ndev > 65535) return OPTIMUS_ESHAPE;
  const size_t size = dtype == OPTIMUS_BF16 ? 2 : 4;
  if (((uintptr_t)x | (uintptr_t)y) & (size - 1) || (uintptr_t)r->positions & 3) return OPTIMUS_EINVAL;
  const char* from = (const char*)x + a.dev0 * a.dev * (long long)size;
  char* to = (char*)y + a.dev0 * a.dev * (long long)size;
  const long long bytes = ndev * a.dev * (long long)size;
  if (from != to && from < to + bytes && to < from + bytes) return OPTIMUS_EINVAL;
  a.x = from;
  a.y = to;
  a.positions = r->positions;
  a.sign = back ? -1.0f : 1.0f;
  Ladder ladder[kMaxAxes];
  for (int k = 0; k < (r->shared_ladder ? 1 : r->axes); ++k) ladder[k].make(r->base, r->shared_ladder ? a.pairs : r->pairs[k]);
  for (int p = 0, k = 0; p < a.pairs; ++p) {
    if (r->in_turn) {
      while (left[k] == 0) k = (k + 1) % r->axes;
    } else if (left[k] == 0) {
      ++k;
    }
    a.axis[p] = (unsigned char)k;
    a.turn[p] = r->scale[k] * (r->shared_ladder ? ladder[0].at(p) : ladder[k].at(done[k])) / 6.283185307179586476925;
    if (!(fabs(a.turn[p]) < 0x1p20)) return OPTIMUS_EINVAL;   // (past it 53 bits hold a large position's whole turns and nothing behind the point)
    --left[k];
    ++done[k];
    if (r->in_turn) k = (k + 1) % r->axes;
  }
  // the widest chunk that pairs and heads are whole numbers of
  int e = size == 2 ? 8 : 4;
  while (e > 1 && ((r->interleaved ? 2 * a.pairs : a.pairs) % e || a.d % e)) e >>= 1;
  if (e == 1 && r->interleaved) return OPTIMUS_ESHAPE;   // (a head of odd width)
  a.chunks = (r->interleaved ? 2 * a.pairs : a.pairs) / e;
  a.copies = from == to ? 0 : (2 * (a.d - 2 * a.pairs) + a.d) / e;
  // Tokens of a workgroup: as many as share the work of a few rounds of 256 lanes, fewer while workgroups are too few to fill the card.
  a.tokens = 1;
  while (a.tokens < 8 && 2 * a.tokens * a.pairs <= kTable && a.tokens * 2 * a.nh * a.chunks < 4 * kThreads &&
         2 * a.tokens * a.nh * a.copies <= (1 << 14) && (a.rows + 2 * a.tokens - 1) / (2 * a.tokens) * ndev >= 4 * num_cus())
    a.tokens *= 2;
  a.by_token = a.tokens == 1 ? 1u : reciprocal(2 * a.nh * a.chunks);
  a.by_chunks = reciprocal(a.chunks);
  a.by_pairs = reciprocal(a.pairs);
  a.by_copies = a.tokens == 1 ? 1u : reciprocal(a.nh * a.copies);
  a.by_head_copies = reciprocal(a.copies);
  const long long groups = (a.rows + a.tokens - 1) / a.tokens;
  if (groups * kThreads >= 1ll << 32) return OPTIMUS_ESHAPE;
  const dim3 grid((unsigned)groups, ndev);
  const hipStream_t st = (hipStream_t)stream;
  const bool beside = r->interleaved != 0;
  if (size == 2) {
    switch (e) {
      case 8: launch<bf16_t, 8>(a, beside, grid, st); break;
      case 4: launch<bf16_t, 4>(a, beside, grid, st); break;
      case 2: launch<bf16_t, 2>(a, beside, grid, st); break;
      default: launch<bf16_t, 1>(a, false, grid, st);
    }
  } else {
    switch (e) {
      case 4: launch<float, 4>(a, beside, grid, st); break;
      case 2: launch<float, 2>(a, beside, grid, st); break;
      default: launch<float, 1>(a, false, grid, st);
    }
  }
  return hip_launch_status();
}

}  // namespace
}  // namespace optimus

extern "C" int optimus_rotary(const void* qkv, void* out, int b, int s, int h, int n, int q, int i, int j, int dtype, const optimus_rotary_axes* axes,
                              void* stream) {
  return optimus::run(qkv, out, b, s, h, n, q, i, j, dtype, axes, false, stream);
}
extern "C" int optimus_rotary_bwd(const void* d_out, void* d_qkv, int b, int s, int h, int n, int q, int i, int j, int dtype,
                                  const optimus_rotary_axes* axes, void* stream) {
  return optimus::run(d_out, d_qkv, b, s, h, n, q, i, j, dtype, axes, true, stream);
}
