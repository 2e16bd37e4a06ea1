// Fused local attention whose scores are changed before the soft-max (attention_fused_kernel.hpp has the layout of the work, which is
// the same here):
//   S = Q K^T / sqrt(d);  S = cap tanh(S / cap);  S -= slope[head] |t - u|, or S += table[head][bucket(u - t)];
//   pair (t, u) is left out where the documents of t and u differ or t is padding (document < 0), where the mask is causal and u is
//   behind both t and the prefix, and where the table's number is -1e30 or less.
// A row that is left without a pair has output 0, log-sum-exp -infinity and no gradients.
//
// Backward: P = exp(S - lse), dS = P (dO V^T - rowsum(dO * O)); the table's gradient is the sum of dS over a bucket's pairs; from
// there on dS (1 - tanh^2).
//
// What the additions cost beside the 32 to 64 clk a matrix instruction takes: the tanh 7 operations a score while a tile's scores stay
// below a quarter of the cap (odd polynomial), else an exponential and a reciprocal; slopes 2; the table nothing but one fused
// multiply-add where a whole tile lies in the last bucket, one LDS read where it does not.  Blocks of keys that share no document with
// the workgroup's rows are not loaded: documents packed one after the other cost the sum of their squares.
#pragma once
#include "attention_fused_kernel.hpp"

namespace optimus {

constexpr int kMaxBuckets = 128, kMaxDistance = 1024, kTableMargin = 64;

typedef __attribute__((ext_vector_type(4))) int i32x4_t;
// read through the scalar cache: the same address in every lane, written by an earlier kernel
typedef const __attribute__((address_space(4))) i32x4_t* BlockList;

struct BiasedArgs {
  FusedArgs f;
  int nb, q, dev0;           // sequences of a device, grid, first device of the launch
  int causal, nblk;          // nblk: blocks of 64 tokens of a sequence
  float cap_log2;            // cap * log2(e)
  float cap_in, cap_exp;     // 1 / (sqrt(d) cap);  2 log2(e) / (sqrt(d) cap)
  float cap_small;           // Q K^T below which the polynomial is taken: cap sqrt(d) / 4
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
// First and last + 1 of the blocks lo .. hi - 1 that share documents with the blocks own0 .. own1 (the workgroup's rows).
__device__ __forceinline__ void live_blocks(BlockList blocks, int own0, int own1, int& lo, int& hi, int* lds2) {
  const int tid = threadIdx.x, n = blockDim.x;
  if (tid == 0) { lds2[0] = 0x7fffffff; lds2[1] = -1; }
  __syncthreads();
  const i32x4_t r0 = blocks[own0], r1 = blocks[own1];
  int first = 0x7fffffff, last = -1;
  for (int b = lo + tid; b < hi; b += n) {
    const i32x4_t x = ((const i32x4_t*)(unsigned long long)blocks)[b];
    if (share_documents(x, r0) || share_documents(x, r1)) { first = min(first, b); last = b; }
  }
  if (last >= 0) { atomicMin(&lds2[0], first); atomicMax(&lds2[1], last); }   // (of integers in LDS: the order does not matter)
  __syncthreads();
  const int x = __builtin_amdgcn_readfirstlane(lds2[0]), y = __builtin_amdgcn_readfirstlane(lds2[1]);
  lo = y < 0 ? 0 : x;
  hi = y + 1;
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

// ---- the scores ----
// place of accumulator slot r in its 32 x 32 tile, without the lane's 4 * (lane / 32)
__device__ constexpr int slot(int r) { return 8 * (r >> 2) + (r & 3); }

// v = Q K^T -> tanh(v / (sqrt(d) cap)).  Below a quarter the odd polynomial up to the ninth power (relative error 1e-8); above,
// 1 - 2 / (exp(2x) + 1), whose absolute error of a unit in the last place of 1 is a relative one of 5e-7 of such a score.
__device__ __forceinline__ void tanh16(f32x16& v, const BiasedArgs& a) {
  float mx = 0.f;
#pragma unroll
  for (int r = 0; r < 16; ++r) mx = fmaxf(mx, fabsf(v[r]));
  if (__builtin_amdgcn_ballot_w64(mx < a.cap_small) == ~0ull) {
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const float x = v[r] * a.cap_in, y = x * x;
      v[r] = fmaf(x * y, fmaf(y, fmaf(y, fmaf(y, 62.0f / 2835.0f, -17.0f / 315.0f), 2.0f / 15.0f), -1.0f / 3.0f), x);
    }
  } else {
#pragma unroll
    for (int r = 0; r < 16; ++r) v[r] = fmaf(-2.0f, __builtin_amdgcn_rcpf(__builtin_amdgcn_exp2f(v[r] * a.cap_exp) + 1.0f), 1.0f);
  }
}

// The bias of a wavefront's head, in units of log2.  BIAS: 0 none, 1 slopes, 2 table.
template <int BIAS>
struct Bias {
  float slope2;
  const float* at0;          // LDS: entry of distance 0
  float far_pos, far_neg;    // from `far` on, and down from `-back` on
  int far, back;
  // lds: [2 (far + kTableMargin) + 1] numbers and kMaxBuckets + 1 first distances; the caller's barrier follows
  __device__ __forceinline__ void init(const BiasedArgs& a, int ghead) {
    if (BIAS == 1) slope2 = a.slopes[ghead] * LOG2E;
    if (BIAS == 2) { far = a.far; back = a.two_sided ? a.far : 0; }
  }
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
// The head's table by distance.  Two barriers: behind the first distances, behind the numbers.
__device__ __forceinline__ void fill_table(const BiasedArgs& a, int ghead, float* numbers, int* first) {
  for (int k = threadIdx.x; k <= a.side; k += blockDim.x) first[k] = a.first[k];
  __syncthreads();
  const int reach = a.far + kTableMargin;
  for (int k = threadIdx.x; k <= 2 * reach; k += blockDim.x) {
    const float x = a.table[(long long)ghead * a.buckets + bucket_of(a, first, k - reach)];
    numbers[k] = x <= -1e30f ? -INFINITY : x * LOG2E;
  }
  __syncthreads();
}

// v: 32 x 32 scores (tanh of them with CAP) -> log2(e) times the score.  The lane's slot r lies at distance t - u =
// dist0 + SIGN * slot(r); lo, hi: smallest and largest distance of the tile.
template <bool CAP, int BIAS, int SIGN>
__device__ __forceinline__ float score2(float v, int r, const BiasedArgs& a, const Bias<BIAS>& b, float base, float dist0f, const float* near) {
  // base: a constant added to every score of the tile (BIAS 2, far), near: its entries in LDS
  const float w = CAP ? a.cap_log2 : a.f.scale_log2;
  if (BIAS == 1) return fmaf(-b.slope2, fabsf(dist0f + (float)(SIGN * slot(r))), v * w);
  if (BIAS == 2) return fmaf(v, w, near ? near[SIGN * slot(r)] : base);
  return v * w;
}
template <int BIAS>
struct TileBias {
  float base, dist0f;
  bool near;
  const float* entry;
};
template <int BIAS>
__device__ __forceinline__ TileBias<BIAS> tile_bias(const Bias<BIAS>& b, int dist0, int lo, int hi) {
  TileBias<BIAS> t = {};
  if (BIAS == 1) t.dist0f = (float)dist0;
  if (BIAS == 2) {
    t.near = lo < b.far && hi > -b.back;
    t.base = lo >= b.far ? b.far_pos : b.far_neg;
    t.entry = b.at0 + dist0;
  }
  return t;
}
// all sixteen, in place
template <bool CAP, int BIAS, int SIGN>
__device__ __forceinline__ void scores16(f32x16& v, const BiasedArgs& a, const Bias<BIAS>& b, const TileBias<BIAS>& t) {
  if (BIAS == 2 && t.near) {
#pragma unroll
    for (int r = 0; r < 16; ++r) v[r] = score2<CAP, BIAS, SIGN>(v[r], r, a, b, 0.f, 0.f, t.entry);
  } else {
#pragma unroll
    for (int r = 0; r < 16; ++r) v[r] = score2<CAP, BIAS, SIGN>(v[r], r, a, b, t.base, t.dist0f, nullptr);
  }
}

template <int BIAS>
struct BiasLds {
  static constexpr int kNumbers = BIAS == 2 ? 2 * (kMaxDistance + kTableMargin) + 1 : 1;
  float numbers[kNumbers];
  int first[BIAS == 2 ? kMaxBuckets + 1 : 1];
};
template <int BIAS>
__device__ __forceinline__ Bias<BIAS> make_bias(const BiasedArgs& a, int ghead, BiasLds<BIAS>& lds) {
  Bias<BIAS> b = {};
  b.init(a, ghead);
  if (BIAS == 2) {
    fill_table(a, ghead, lds.numbers, lds.first);
    b.at0 = lds.numbers + a.far + kTableMargin;
    b.far_pos = b.at0[a.far];
    b.far_neg = b.at0[-b.back];
  }
  return b;
}

}  // namespace
}  // namespace optimus
