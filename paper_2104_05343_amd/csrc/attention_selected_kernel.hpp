// Attention in which a query sees some blocks of keys only: its own and those that a cheap score ranks highest.
//   mean[v] = mean of block v's keys, rounded to bf16;  score(t, v) = q_t . mean[v]
//   a query attends to its own block and to the count - 1 others of highest score (causal: among those in front of its own)
// The choice is one step (attention_select.hip), the attention over any chosen blocks another (attention_selected.hip forward,
// attention_selected_bwd.hip backward); tiles, fragments and layouts are those of the fused attention (attention_fused_kernel.hpp).
//
// Where queries choose many of the blocks that they could, it is the fused attention with a mask (attention_selected_masked.hip).
//
// How the work is cut otherwise (lists).  Neighbouring queries choose different blocks, so a tile of queries has no common keys to load and a tile of
// the dense attention would be mostly masked.  The other way round a block of keys has a list of the queries that chose it.  A workgroup takes a
// block and a piece of its list: the block's K and V are loaded once, queries come 64 or 128 at a time, gathered by their numbers, and every
// product is dense.  What a query gets from one block is a partial result, its part of the output with a maximum and a sum (forward) or of dQ
// (backward): a row of fp16 numbers that goes to memory at the pair's place in the list, and a second kernel adds up each query's rows, at the
// places that the step which makes the lists has noted.  dK and dV stay in the workgroup; blocks of several pieces are added up behind it.
// The rows are count * s * d * 2 bytes a matrix, written and read: this, beside the products, bounds the form; they are made for 1 GiB at a time.
// Measured, 8 (sequence, head)s of 32768 x 128, 16 of 256 blocks of 128 keys: lists 61 us, products 470 (585 TFLOP/s of the chosen pairs), sums 258 (1.1 GB,
// 4.3 TB/s); without the rows' stores the products take 330.
#pragma once
#include "attention_biased_kernel.hpp"

namespace optimus {

constexpr int kListChunk = 256;        // queries of a workgroup that makes the lists
constexpr int kMaskedBlocks = 256;     // most blocks of a sequence in the masked form
constexpr int kQueries = 128;          // list rows of a tile

typedef _Float16 f16_t;

struct SelectedArgs {
  FusedArgs f;                         // f.attn, f.lse, f.d_attn, f.d_qkv, f.delta: first device of the launch
  const int* selected;                 // [matrix][s][count], first device of the launch
  int* chosen;                         // the same, written (attention_select)
  const int* lengths;                  // [sequences of the grid], or nullptr
  bf16_t* means;                       // [matrix][blocks][d]
  float* mean_sizes;                   // [matrix][blocks]: Euclidean norms, rounded up
  int nb, nmat, q, dev0, causal;       // sequences and matrices of a device
  int block, blocks, count;            // keys of a block, blocks of a sequence, blocks of a query
  // the masked form
  unsigned by_steps;                   // ceil(2^32 / (block / 64)), see divide
  int mask_words;                      // of a block's queries, 32 a word
  unsigned* mask;                      // [matrix][block][mask_words]: whether a query has chosen the block
  // lists
  int mats, mat0, portion;             // matrices of the call, first one of this launch, how many it has
  int chunks;                          // kListChunk pieces of a sequence
  int seg[2], most[2];                 // kind 0: forward and dQ, 1: dK and dV: list rows of an item, about; most items of a matrix
  int* counts;                         // [matrix][chunks + 1][block]: pairs, or (list_sums_kernel) those of earlier chunks
  int* first_item;                     // [kind][matrix][blocks + 1]
  i32x4_t* items[2];                   // [matrix][most]: block, place of the first pair, pairs, -
  int* list;                           // [matrix][s * count]: query of every pair
  int* places;                         // [matrix][s][count]: place of the pair in list, -1: none
  f16_t* rows;                         // [matrix - mat0][s * count][d]: partial results, see store_parts
  float* units;                        // [matrix - mat0][s * count]: what a row's numbers are to be multiplied by; joint: [d / 32] of 32 columns each
  float2* ml;                          // [matrix - mat0][s * count]: maximum of log2(e) Q K^T / sqrt(d), sum of exponentials
  float* key_rows;                     // [matrix - mat0][item][block / 64][dK, dV][64][d]
};

// What the host decides; bytes of the workspace, in this order
struct SelectedPlan {
  bool masked;
  bool joint;                          // lists, all gradients in one pass
  int mats, chunks, mask_words;
  int portion, key_portion;            // matrices whose partial results are in memory at a time: of queries, of keys
  int seg[2], most[2];
  size_t delta, mask, counts, first_item, items[2], list, places, rows, units, ml, keys, total;
};

// csrc/attention_selected*.hip
int launch_selected_bwd_kernels(const SelectedArgs& a, const SelectedPlan& p, int d, hipStream_t st);
void launch_selected_dq_combine(const SelectedArgs& a, int d, bool joint, hipStream_t st);
void launch_selected_masked(const SelectedArgs& a, int mats, int d, bool bwd, hipStream_t st);

namespace {

// u / n for m = ceil(2^32 / n): exact while u * n <= 2^32; n = 1 has m = 0
__device__ __forceinline__ unsigned divide(unsigned u, unsigned m) { return m ? __umulhi(u, m) : u; }

// What a wavefront knows about its matrix, mm counted over the devices of the launch.
struct SelMatrix {
  int len;
  long long qkv, attn, vec;   // element offsets of the matrix' first row
};
template <int D>
__device__ __forceinline__ SelMatrix selected_matrix(const SelectedArgs& a, int mm) {
  SelMatrix m;
  const FusedArgs& f = a.f;
  const int dev = mm / a.nmat, mat = mm % a.nmat, seq = mat / f.nh, head = mat % f.nh;
  // (the same in every lane: loads through buffer resources want it in a scalar register)
  m.len = __builtin_amdgcn_readfirstlane(a.lengths ? min(max(a.lengths[(a.dev0 + dev) / a.q * a.nb + seq], 0), f.s) : f.s);
  m.qkv = dev * f.dev_qkv + (long long)seq * f.s * f.ld + head * 3 * D;
  m.attn = dev * f.dev_attn + (long long)seq * f.s * f.ldo + head * D;
  m.vec = (long long)mm * f.s;
  return m;
}

// A tile's accumulators, products with the rows' operand in the A slot: lane n = lane % 32 holds column 32 dt + n of the rows
// slot(r) + 4 (lane / 32).  A row goes to memory as [n][dt], so that 32 lanes write it whole with 4 (or 2) numbers each; what reads it
// undoes the order.
template <int DT> struct RowPart;
template <> struct RowPart<4> { typedef __attribute__((ext_vector_type(4))) float V; };
template <> struct RowPart<2> { typedef __attribute__((ext_vector_type(2))) float V; };
template <int DT>
__device__ __forceinline__ void store_rows(float* to, const f32x16 (&acc)[DT], int left, int g, int lane) {
  typedef typename RowPart<DT>::V V;
#pragma unroll
  for (int r = 0; r < 16; ++r) {
    const int row = slot(r) + 4 * g;
    V v;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) v[dt] = acc[dt][r];
    if (row < left) *(V*)(to + row * (32 * DT) + (lane & 31) * DT) = v;
  }
}
// A pair's partial result, rounded to fp16: a block's part of a query's output, or of its dQ, off by 2^-12 of itself, where the rounding of P
// and dS to bf16 has left it off by some 2^-9; the sums over a block's keys and over the blocks stay fp32.  (8 (sequence, head)s of 32768 x 128,
// 16 of 256 blocks: 2.2 GB of fp32 rows cost 300 us to write beside the products' 417, and 389 to read.)  Each row is scaled by a power of
// two that brings its largest number to 2^14, so that nothing is lost to fp16's range but what is below 2^-28 of that.
// Lanes trade their numbers until a store has 128 whole bytes of a row: the forward products of the case above take 536 us with 32 bytes of a row in a
// store, 490 with 64, 474 with 128; 464 with 256, whose lanes have a column each, and 100 instructions more a tile for the scales (width 64: 2 to 5 % slower).

// The maximum that passes NaN on: two operands or three an instruction.  (fmaxf first clears signalling NaN out of every operand that might be one,
// such as a matrix instruction's result, by an instruction of its own.)
__device__ __forceinline__ float larger(float x, float y) { return __builtin_elementwise_maximum(x, y); }
__device__ __forceinline__ float largest(const f32x16& v, float m) {
#pragma unroll
  for (int r = 0; r < 16; r += 2) m = larger(larger(m, v[r]), v[r + 1]);
  return m;
}
// Whether a wavefront's scores have to be rounded before what is subtracted from them, a rounded score itself: that is off by up to 2^-24 of itself, and
// scores times the factor less it are not, so that from 2^31 on an exponent above zero overflows, and one below leaves a row nothing.  (Finite: a
// row that has seen nothing has -infinity.  Choice and forward of 128 (sequence, head)s of 4096 x 64 with a mask 438 us without this, 444 with it; lists as before.)
__device__ __forceinline__ bool large_scores(float subtracted) {
  const float size = fabsf(subtracted);
  return __builtin_amdgcn_ballot_w64(size > 0x1p28f && size < INFINITY) != 0;
}
template <int N>
__device__ __forceinline__ float score_weight(f32x16 (&scores)[N], float weight, bool large) {   // what the scores are to be multiplied by then
  if (!large) return weight;
#pragma unroll
  for (int t = 0; t < N; ++t)
#pragma unroll
    for (int r = 0; r < 16; ++r) scores[t][r] *= weight;
  return 1.0f;
}
// A lane has one row's numbers: products with the rows' operand in the B slot, slot r of a 32 x 32 tile is column slot(r) + 4 g.  What scales them, the
// reciprocal of what they are to be multiplied by later: 2^(141 - e) for a largest number of biased exponent e.
struct RowScale { float scale; unsigned unit; };
__device__ __forceinline__ RowScale row_scale(float most) {
  const auto both = __builtin_amdgcn_permlane32_swap(__float_as_uint(most), __float_as_uint(most), false, false);
  most = larger(__uint_as_float(both[0]), __uint_as_float(both[1]));
  const int e = min(max((int)(__float_as_uint(most) >> 23 & 255), 16), 254);
  return {__uint_as_float((unsigned)(268 - e) << 23), (unsigned)(e - 14) << 23};
}
__device__ __forceinline__ float largest_size(const f32x16& v, float m) {
#pragma unroll
  for (int r = 0; r < 16; r += 2) m = larger(larger(m, fabsf(v[r])), fabsf(v[r + 1]));
  return m;
}
// 32 columns of a wavefront's 32 rows as fp16: lane n % 16 of w[k] has row 16 k + n % 16, columns 16 (n / 16 % 2) + 8 (n / 32) .. + 7
__device__ __forceinline__ void pack_columns(const f32x16& acc, float scale, u32x4 (&w)[2]) {
  typedef __attribute__((ext_vector_type(4))) _Float16 Four;
  u32x2 h[4];
#pragma unroll
  for (int c = 0; c < 4; ++c) {
    Four x;
#pragma unroll
    for (int k = 0; k < 4; ++k) x[k] = (f16_t)(acc[4 * c + k] * scale);
    h[c] = __builtin_bit_cast(u32x2, x);
  }
#pragma unroll
  for (int c = 0; c < 2; ++c) {   // lanes 0 .. 31: columns 16 c .. + 7, the others the next eight
    const auto lo = __builtin_amdgcn_permlane32_swap(h[2 * c][0], h[2 * c + 1][0], false, false);
    const auto hi = __builtin_amdgcn_permlane32_swap(h[2 * c][1], h[2 * c + 1][1], false, false);
    w[c] = u32x4{lo[0], hi[0], lo[1], hi[1]};
  }
#pragma unroll
  for (int k = 0; k < 4; ++k) {   // lanes 16 .. 31 and 48 .. 63 of the first with the sixteen before them of the second: rows 0 .. 15, rows 16 .. 31
    const auto r = __builtin_amdgcn_permlane16_swap(w[0][k], w[1][k], false, false);
    w[0][k] = r[0];
    w[1][k] = r[1];
  }
}
template <int CTRL, int BANKS>
__device__ __forceinline__ unsigned moved_into(unsigned old, unsigned x) { return (unsigned)__builtin_amdgcn_update_dpp((int)old, (int)x, CTRL, 0xf, BANKS, false); }

// A wavefront's 32 rows, `rows` of them there, whole.
// Through buffer resources that end behind the last row: a store under a condition would have the wait for the next tile's queries, which are
// requested ahead of it, wait for the stores too.
template <int DT>
__device__ __forceinline__ void store_parts(f16_t* to, float* units, const f32x16 (&acc)[DT], int rows, int g, int lane) {
  const int left = __builtin_amdgcn_readfirstlane(rows), row = lane & 31;
  const auto to_units = __builtin_amdgcn_make_buffer_rsrc(units, 0, left * 4, 0x00020000);
  const auto to_rows = __builtin_amdgcn_make_buffer_rsrc(to, 0, left * (64 * DT), 0x00020000);
  float most = 0.f;
#pragma unroll
  for (int dt = 0; dt < DT; ++dt) most = largest_size(acc[dt], most);
  const RowScale s = row_scale(most);
  __builtin_amdgcn_raw_buffer_store_b32((int)s.unit, to_units, g == 0 ? row * 4 : 0x7fffffff, 0, 0);
#pragma unroll
  for (int dt = 0; dt < DT; dt += 2) {   // 64 columns: stores of eight rows' whole 128 bytes
    u32x4 w[2][2];
    pack_columns(acc[dt], s.scale, w[0]);
    pack_columns(acc[dt + 1], s.scale, w[1]);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      u32x4 first, second;
#pragma unroll
      for (int k = 0; k < 4; ++k) {   // eight lanes of sixteen trade: rows 0 .. 7 with both column halves, rows 8 .. 15
        first[k] = moved_into<0x128, 0xc>(w[0][h][k], w[1][h][k]);
        second[k] = moved_into<0x128, 0x3>(w[1][h][k], w[0][h][k]);
      }
      const int at = (16 * h + (lane & 7)) * (64 * DT) + dt * 64 + (lane >> 3 & 1) * 64 + (lane >> 4 & 1) * 32 + (lane >> 5) * 16;
      __builtin_amdgcn_raw_buffer_store_b128(first, to_rows, at, 0, 0);
      __builtin_amdgcn_raw_buffer_store_b128(second, to_rows, at + 8 * 64 * DT, 0, 0);
    }
  }
}
// A half-wavefront's row of D numbers in LDS, columns in order -> bf16 at `to`.
template <int DT>
__device__ __forceinline__ void write_ordered(bf16_t* to, const float* lds, int n, bool write) {
  if (DT == 4) {
    const float4 x = *(const float4*)(lds + 4 * n);
    if (write) *(u32x2*)(to + 4 * n) = u32x2{pack2_bf16(x.x, x.y), pack2_bf16(x.z, x.w)};
  } else {
    const float2 x = *(const float2*)(lds + 2 * n);
    if (write) *(unsigned*)(to + 2 * n) = pack2_bf16(x.x, x.y);
  }
}
// The same from [n][dt] in registers, through LDS of its own.
template <int DT>
__device__ __forceinline__ void write_row(bf16_t* to, const typename RowPart<DT>::V v, float* lds, int n, bool write) {
#pragma unroll
  for (int dt = 0; dt < DT; ++dt) lds[dt * 32 + n] = v[dt];
  __builtin_amdgcn_wave_barrier();
  write_ordered<DT>(to, lds, n, write);
  __builtin_amdgcn_wave_barrier();
}

// Work of a workgroup: a block and a piece of its list.  Workgroups count the matrices of a launch first: neighbours go to the eight dies in turn,
// so that (of a multiple of eight) each die's L2 has the queries of its own ones.
struct ListItem {
  int block, start, pairs;
};
__device__ __forceinline__ bool list_item(const SelectedArgs& a, int kind, int mm, int k, ListItem* it) {
  const int* first = a.first_item + ((long long)kind * a.mats + mm) * (a.blocks + 1);
  if (k >= first[a.blocks]) return false;
  const i32x4_t x = a.items[kind][(long long)mm * a.most[kind] + k];
  it->block = __builtin_amdgcn_readfirstlane(x.x);
  it->start = __builtin_amdgcn_readfirstlane(x.y);
  it->pairs = __builtin_amdgcn_readfirstlane(x.z);
  return true;
}

}  // namespace
}  // namespace optimus
