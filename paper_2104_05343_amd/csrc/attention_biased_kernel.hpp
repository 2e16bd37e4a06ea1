// Fused local attention whose scores are changed before the soft-max (attention_fused_kernel.hpp has the layout of the work, which is
// the same here):
//   S = Q K^T / sqrt(d);  S = cap tanh(S / cap);  S -= slope[head] |t - u|, or S += table[head][bucket(t - u)];
//   pair (t, u) is left out where the documents of t and u differ or t is padding (document < 0), where the mask is causal and u is
//   behind both t and the prefix, and where the table's number is -1e30 or less.
// A row that is left without a pair has output 0, log-sum-exp -infinity and no gradients.
//
// Backward: P = exp(S - lse), dS = P (dO V^T - rowsum(dO * O)); the table's gradient is the sum of dS over a bucket's pairs; from
// there on dS (1 - tanh^2).
//
// What the additions cost beside the 32 to 64 clk a matrix instruction takes: the tanh 7 operations a score (the largest of the tile
// among them) while a tile's scores stay below a quarter of the cap (odd polynomial), else an exponential and a reciprocal, beside a cap
// beyond 64 both; slopes 2;
// the table nothing but one fused multiply-add where a whole tile lies in the last bucket, one LDS read where it does not.  Blocks of
// keys that share no document with the workgroup's rows are not loaded: documents packed one after the other cost the sum of their
// squares.
#pragma once
#include "attention_fused_kernel.hpp"

namespace optimus {

constexpr int kMaxBuckets = 128, kMaxDistance = 1024;

typedef __attribute__((ext_vector_type(4))) int i32x4_t;
// read through the scalar cache: the same address in every lane, written by an earlier kernel
typedef const __attribute__((address_space(4))) i32x4_t* BlockList;

struct BiasedArgs {
  FusedArgs f;
  int nb, q, dev0;           // sequences of a device, grid, first device of the launch
  int causal, nblk;          // nblk: blocks of 64 tokens of a sequence
  float cap_log2;            // cap * log2(e)
  float weight_lo;           // what the rounding of the scores' weight (and of the tanh's first coefficient) loses
  float cap_pre;             // a power of two that Q K^T is scaled by beside a large cap: x; 1 otherwise
  float cap_exp;             // 2 u log2(e) / x
  float tanh_of[5];          // coefficients of tanh u at x, x^3, .. x^9
  float cap_small;           // x below which the polynomial is taken: u = 1/4
  int buckets, side, two_sided, far;   // side: buckets of one side; far: first distance of its last one
  int ntiles;                // row tiles of a matrix in the parts of the table's gradient
  const float* slopes;       // [heads]
  const float* table;        // [heads][buckets]
  const int* documents;      // [sequences][s]
  const int* prefix;         // [sequences]
  const i32x4_t* blocks;     // [sequences][nblk]: smallest and largest document of 64 tokens, 1 if there is padding
  float* table_parts;        // [device][matrix][tile][buckets], or nullptr
  unsigned short first[kMaxBuckets + 1];   // first distance of each bucket of a side; one more than any at the end
};

// csrc/attention_biased*.hip
void launch_attn_biased_prepare(const BiasedArgs& a, int d, bool delta, int nmat, int ndev, hipStream_t st);
int launch_attn_biased_bwd_kernels(const BiasedArgs& a, const AttnBiasedDesc& d, hipStream_t st);

namespace {

// The kernels' CAP: 0 none, 1 up to 64, 2 beyond (tanh16).
inline int cap_form(const AttnBiasedDesc& b) { return b.cap > 64 ? 2 : b.cap > 0 ? 1 : 0; }
// Calls run(width, cap, bias), constants of the kernels' D, CAP and BIAS.
template <class F>
void with_kind(const AttnBiasedDesc& b, F run) {
  using std::integral_constant;
  auto with_cap = [&](auto width, auto cap) {
    if (b.table) run(width, cap, integral_constant<int, 2>());
    else if (b.slopes) run(width, cap, integral_constant<int, 1>());
    else run(width, cap, integral_constant<int, 0>());
  };
  auto with_width = [&](auto width) {
    switch (cap_form(b)) {
      case 0: with_cap(width, integral_constant<int, 0>()); break;
      case 1: with_cap(width, integral_constant<int, 1>()); break;
      default: with_cap(width, integral_constant<int, 2>());
    }
  };
  if (b.base.d == 64) with_width(integral_constant<int, 64>());
  else with_width(integral_constant<int, 128>());
}

// What a wavefront knows about its matrix.
struct Matrix {
  int dev, mat, seq, head, prefix;
  int ghead;
  const int* docs;       // of the sequence, or nullptr
  BlockList blocks;
  long long qkv, attn, vec;   // element offsets of the matrix' first row (head's columns included)
};
template <int D>
__device__ __forceinline__ Matrix matrix_of(const BiasedArgs& a, int mat, int dev) {
  Matrix m;
  const FusedArgs& f = a.f;
  m.dev = dev; m.mat = mat;
  m.seq = mat / f.nh; m.head = mat % f.nh;
  const int at = a.dev0 + dev;
  const int gseq = at / a.q * a.nb + m.seq;
  m.ghead = at % a.q * f.nh + m.head;
  m.prefix = a.prefix ? min(max(a.prefix[gseq], 0), f.s) : 0;
  m.docs = a.documents ? a.documents + (long long)gseq * f.s : nullptr;
  m.blocks = (BlockList)(unsigned long long)(a.blocks + (long long)gseq * a.nblk);
  m.qkv = dev * f.dev_qkv + (long long)m.seq * f.s * f.ld + m.head * 3 * D;
  m.attn = dev * f.dev_attn + (long long)m.seq * f.s * f.ldo + m.head * D;
  m.vec = dev * f.dev_vec + (long long)mat * f.s;
  return m;
}

// ---- blocks of 64 tokens and their documents ----
__device__ __forceinline__ bool share_documents(i32x4_t x, i32x4_t y) { return x.x <= y.y && x.y >= y.x; }
// every pair of the two blocks, which share documents, is of one document
__device__ __forceinline__ bool one_document(i32x4_t x, i32x4_t y) { return x.x == x.y && y.x == y.y && !(x.z | y.z); }
// First and last + 1 of the blocks lo .. hi - 1 that share documents with the blocks own0 .. own1 (the workgroup's rows).  Every
// wavefront looks at all of them, 64 at a time: no barrier.
__device__ __forceinline__ void live_blocks(BlockList blocks, int own0, int own1, int& lo, int& hi) {
  const i32x4_t r0 = blocks[own0], r1 = blocks[own1];
  const i32x4_t* list = (const i32x4_t*)(unsigned long long)blocks;
  const int lane = threadIdx.x & 63;
  int first = 0, last = -1;
  for (int b = lo; b < hi; b += 64) {
    const i32x4_t x = list[min(b + lane, hi - 1)];
    const unsigned long long m = __builtin_amdgcn_ballot_w64(b + lane < hi && (share_documents(x, r0) || share_documents(x, r1)));
    if (m) {
      if (last < 0) first = b + __builtin_ctzll(m);
      last = b + 63 - __builtin_clzll(m);
    }
  }
  lo = first;
  hi = last + 1;
}

// A tile whose padded rows (and those past the end) become zeros in LDS: what a padded token's rows hold is not looked at, and zero
// times infinity would be NaN.
template <int D, int NW, int ROWS>
struct RowLoader : TileLoader<D, NW, ROWS, true> {
  using Base = TileLoader<D, NW, ROWS, true>;
  // docs: nullptr if no row of the tile is padding.  row0 < s.
  __device__ __forceinline__ void issue(const bf16_t* mat, int row0, int s, bf16_t* tile, const int* docs) const {
    if (!docs) {
      Base::issue(mat, row0, s, tile);
      return;
    }
    const unsigned lds_base = (unsigned)(size_t)(__attribute__((address_space(3))) bf16_t*)tile;
    const i32x4 rsrc = make_rsrc(mat + (long long)row0 * Base::ld);
    unsigned o[Base::PER];
#pragma unroll
    for (int it = 0; it < Base::PER; ++it) {
      const int src = row0 + (Base::wave * Base::PER + it) * Base::ROWS_PER_KIB + Base::lane / Base::CH;
      o[it] = src >= s || docs[min(src, s - 1)] < 0 ? 0x80000000u : Base::off[it];   // beyond the resource: zeros
    }
#pragma unroll
    for (int it = 0; it < Base::PER; ++it) {
      const unsigned m0v = __builtin_amdgcn_readfirstlane(lds_base + (unsigned)(Base::wave * Base::PER + it) * 1024u);
      asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tbuffer_load_dwordx4 %0, %1, 0 offen lds" ::"v"(o[it]), "s"(rsrc), "s"(m0v) : "memory", "m0");
    }
  }
};
__device__ __forceinline__ bf16x8 zero_if(bool z, bf16x8 v) {
  u32x4 w = __builtin_bit_cast(u32x4, v);
#pragma unroll
  for (int k = 0; k < 4; ++k) w[k] = z ? 0u : w[k];
  return __builtin_bit_cast(bf16x8, w);
}

// ---- fragments by byte addresses in LDS ----
// A lane's place in a tile is one number; the swizzle makes the step along a row (16 contraction elements, 32 columns) an exclusive or
// with a constant, since tiles are aligned to their rows, and whole groups of 16 rows an offset in the instruction.  One register a
// tile then: kept apart, the places of a block's fragments are 16 to 24 registers, and were spilled.
template <int D>
__device__ __forceinline__ unsigned lane_rows(int lane) {
  const int row = lane & 31;
  return (unsigned)(row * D * 2 + (((lane >> 5) ^ swz<D>(row)) << 4));
}
template <int D>
__device__ __forceinline__ unsigned lane_cols(int lane) {
  const int lg = lane & 15, col = (((lane >> 4) & 1) << 4) + ((lg & 3) << 2), row = ((lane >> 5) << 2) + (lg >> 2);
  return (unsigned)((row * D + (((col >> 3) ^ swz<D>(row)) << 3) + (col & 7)) * 2);
}
__device__ __forceinline__ unsigned lds_address(const void* p) { return (unsigned)(size_t)(__attribute__((address_space(3))) const void*)p; }
// at: address of the tile plus lane_rows; fragment frag_rows<D>(tile, row0, ks, lane)
template <int D>
__device__ __forceinline__ bf16x8 rows_at(unsigned at, int row0, int ks) {
  return *(__attribute__((address_space(3))) const bf16x8*)(size_t)((at ^ (unsigned)(ks * 32)) + (unsigned)(row0 * D * 2));
}
// at: address of the tile plus lane_cols; fragment frag_cols_acc_order<D>(tile, row0, 32 * dt, lane)
template <int D>
__device__ __forceinline__ bf16x8 cols_at(unsigned at, int row0, int dt) {
  typedef __attribute__((address_space(3))) s16x4* P;
  s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((P)(size_t)((at ^ (unsigned)(dt * 64)) + (unsigned)(row0 * D * 2)));
  s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((P)(size_t)((at ^ (unsigned)(dt * 64 + 32)) + (unsigned)((row0 + 8) * D * 2)));
  s16x8 v = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
  return __builtin_bit_cast(bf16x8, v);
}

// ---- the scores ----
// place of accumulator slot r in its 32 x 32 tile, without the lane's 4 * (lane / 32)
__device__ constexpr int slot(int r) { return 8 * (r >> 2) + (r & 3); }

// v = Q K^T -> tanh(u), u = v / (sqrt(d) cap).  Below a quarter the odd polynomial up to the ninth power, in v itself (relative error
// 1e-8); above, 1 - 2 / (exp(2u) + 1), whose absolute error of a unit or two in the last place of 1 is a relative one of 1e-6 of such a
// score.  A tile with a score beyond a quarter takes the second form for all of them where that error, of the cap whatever the score, is
// small beside the rounding of P to bf16: up to a cap of 64 1.8e-5 of a score at most, 6e-6 as a rule.
// CAP 2 (a larger cap) and FINE (where sums of dS are an fp32 result): the polynomial for each score below a quarter, and the reciprocal
// refined by a Newton step.  (16 matrices of 4096 of width 128, causal, every tile beyond a quarter: forward 110 us, with CAP 2 153;
// width 64 93 and 137.)
// CAP 2 scales v by a power of two first: its powers, and those of 1 / (sqrt(d) cap), leave fp32's range else.
template <int CAP, bool FINE = false>
__device__ __forceinline__ void tanh16(f32x16& v, const BiasedArgs& a) {
  if (CAP == 2) {
#pragma unroll
    for (int r = 0; r < 16; ++r) v[r] *= a.cap_pre;
  }
  auto polynomial = [&](float x) {
    const float y = x * x;
    return x * fmaf(y, fmaf(y, fmaf(y, fmaf(y, a.tanh_of[4], a.tanh_of[3]), a.tanh_of[2]), a.tanh_of[1]), a.tanh_of[0]);
  };
  float mx = 0.f;
#pragma unroll
  for (int r = 0; r < 16; ++r) mx = fmaxf(mx, fabsf(v[r]));
  if (__builtin_amdgcn_ballot_w64(mx < a.cap_small) == ~0ull) {
#pragma unroll
    for (int r = 0; r < 16; ++r) v[r] = polynomial(v[r]);
  } else {
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const float e1 = __builtin_amdgcn_exp2f(v[r] * a.cap_exp) + 1.0f;
      float q = __builtin_amdgcn_rcpf(e1);
      if (FINE || CAP == 2) {
        q = e1 < 1e30f ? fmaf(fmaf(-e1, q, 1.0f), q, q) : q;   // (infinity times zero)
        const float near = polynomial(v[r]);
        v[r] = fabsf(v[r]) < a.cap_small ? near : fmaf(-2.0f, q, 1.0f);
      } else {
        v[r] = fmaf(-2.0f, q, 1.0f);
      }
    }
  }
}

// The bias of a wavefront's head, in units of log2.  BIAS: 0 none, 1 slopes, 2 table.
template <int BIAS>
struct BiasLds {
  float numbers[BIAS == 2 ? 2 * kMaxDistance + 1 : 1];   // by distance, -far .. far
  int first[BIAS == 2 ? kMaxBuckets + 1 : 1];
};
struct Bias {
  float slope2;
  const float* at0;          // LDS: entry of distance 0
  float far_pos, far_neg;    // from `far` on, and down from `-back` on
  int far, back;
};
__device__ __forceinline__ int bucket_of(const BiasedArgs& a, const int* first, int dist) {
  if (dist < 0 && !a.two_sided) return 0;
  const int n = abs(dist);
  int k = 0;   // the last bucket that does not begin behind n
#pragma unroll
  for (int step = kMaxBuckets / 2; step; step >>= 1)
    if (k + step < a.side && first[k + step] <= n) k += step;
  return dist < 0 ? k + a.side : k;
}
// With a table two barriers: behind the first distances of the buckets, behind the numbers.
template <int BIAS>
__device__ __forceinline__ Bias make_bias(const BiasedArgs& a, int ghead, BiasLds<BIAS>& lds) {
  Bias b = {};
  // (the same in every lane: scalar registers)
  auto uniform = [](float x) { return __uint_as_float((unsigned)__builtin_amdgcn_readfirstlane((int)__float_as_uint(x))); };
  if (BIAS == 1) b.slope2 = uniform(a.slopes[ghead] * LOG2E);
  if (BIAS == 2) {
    for (int k = threadIdx.x; k <= a.side; k += blockDim.x) lds.first[k] = a.first[k];
    __syncthreads();
    for (int k = threadIdx.x; k <= 2 * a.far; k += blockDim.x) {
      const float x = a.table[(long long)ghead * a.buckets + bucket_of(a, lds.first, k - a.far)];
      lds.numbers[k] = x <= -1e30f ? -INFINITY : x * LOG2E;
    }
    __syncthreads();
    b.at0 = lds.numbers + a.far;
    b.far = a.far;
    b.back = a.two_sided ? a.far : 0;
    b.far_pos = uniform(b.at0[b.far]);
    b.far_neg = uniform(b.at0[-b.back]);
  }
  return b;
}

// Tiles of n columns or rows whose smallest distance t - u is lo and largest hi, scores (their tanh with CAP) in v.  SIGN: of the
// distance along a lane's slots; the lane's slot r lies at dist0 + SIGN * slot(r).
//
// plain: every pair of the tile has one sign (slopes) or one bucket (table), so that log2(e) times the score is v * w + c.
template <int BIAS>
__device__ __forceinline__ bool plain_tile(const Bias& b, int lo, int hi) {
  return BIAS == 1 ? lo >= 0 || hi <= 0 : BIAS == 2 ? lo >= b.far || hi <= -b.back : true;
}
template <int CAP, int BIAS>
__device__ __forceinline__ void plain_weights(const BiasedArgs& a, const Bias& b, int lo, float& w, float& c) {
  w = BIAS == 1 ? 1.0f : CAP ? a.cap_log2 : a.f.scale_log2;
  c = BIAS == 2 ? (lo >= b.far ? b.far_pos : b.far_neg) : 0.f;
}
template <int CAP, int BIAS, int SIGN>
__device__ __forceinline__ void plain16(f32x16& v, const BiasedArgs& a, const Bias& b, int dist0, int lo) {
  if (BIAS == 1) {
    const float sg = lo >= 0 ? -b.slope2 : b.slope2, base = sg * (float)dist0, w = CAP ? a.cap_log2 : a.f.scale_log2;
#pragma unroll
    for (int r = 0; r < 16; ++r) v[r] = fmaf(v[r], w, fmaf(sg, (float)(SIGN * slot(r)), base));
  }
}
// Any tile: log2(e) times the score, -infinity where the pair is left out: the other token's place (at + slot(r)) behind `bound`
// (SIGN < 0) or ahead of it, or of another document than `doc`.  docs: LDS, the other tokens' from the lane's slot 0 on.  FINE: hi + lo
// is taken off the score, hi before the bias: with a row's log-sum-exp what is rounded then is small where it counts.
template <int CAP, int BIAS, int SIGN, bool FINE = false>
__device__ __forceinline__ void any16(f32x16& v, const BiasedArgs& a, const Bias& b, int dist0, int at, int bound, const int* docs, int doc,
                                      float hi = 0.f, float lo = 0.f) {
  asm volatile("");   // a branch, not selects: taken by few tiles, and seven operations a score
  const float w = CAP ? a.cap_log2 : a.f.scale_log2;
  const int reach = bound - at;
#pragma unroll
  for (int c = 0; c < 4; ++c) {
    const int4 o = *(const int4*)(docs + 8 * c);
    const int other[4] = {o.x, o.y, o.z, o.w};
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int r = 4 * c + e, dist = dist0 + SIGN * slot(r);
      float x = FINE ? fmaf(v[r], w, -hi) : v[r] * w;
      if (BIAS == 1) x = fmaf(-b.slope2, fabsf((float)dist), x);
      if (BIAS == 2) {
        const float bias = b.at0[min(max(dist, -b.far), b.far)];
        x += FINE ? fmaf(v[r], a.weight_lo, bias - lo) : bias;
      }
      const bool out = (SIGN < 0 ? slot(r) > reach : slot(r) < reach) | (other[e] != doc) | (doc < 0);
      v[r] = out ? -INFINITY : x;
    }
  }
}

}  // namespace
}  // namespace optimus
