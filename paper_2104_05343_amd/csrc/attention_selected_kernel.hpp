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
// Measured, 8 (sequence, head)s of 32768 x 128, 16 of 256 blocks of 128 keys: lists 65 us, products 466 (590 TFLOP/s of the chosen pairs), sums 255 (1.1 GB,
// 4.3 TB/s); without the rows' stores the products take 330.
#pragma once
#include "attention_biased_kernel.hpp"

namespace optimus {

constexpr int kListChunk = 256;        // queries of a workgroup that makes the lists
constexpr int kMostBlocks = 1024, kMostCount = 64;
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
  int* counts;                         // [matrix][chunk][block]: pairs
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
template <int DT> struct RowHalves;
template <> struct RowHalves<4> { typedef __attribute__((ext_vector_type(4))) _Float16 V; };
template <> struct RowHalves<2> { typedef __attribute__((ext_vector_type(2))) _Float16 V; };

template <int CTRL>
__device__ __forceinline__ float lane_moved(float x) {
  return __uint_as_float((unsigned)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(x), CTRL, 0xf, 0xf, false));
}
// first: [a's row of 16 lanes 0, b's 0, a's 2, b's 2]; second: [a's 1, b's 1, a's 3, b's 3]
__device__ __forceinline__ void swap_rows(float& a, float& b) {
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(a), __float_as_uint(b), false, false);
  a = __uint_as_float(r[0]);
  b = __uint_as_float(r[1]);
}
// The maximum that passes NaN on: two operands or three an instruction.  (fmaxf first clears signalling NaN out of every operand that might be one,
// such as a matrix instruction's result, by an instruction of its own.)
__device__ __forceinline__ float larger(float x, float y) { return __builtin_elementwise_maximum(x, y); }
__device__ __forceinline__ float largest(const f32x16& v, float m) {
#pragma unroll
  for (int r = 0; r < 16; r += 2) m = larger(larger(m, v[r]), v[r + 1]);
  return m;
}
template <int DT>
__device__ __forceinline__ void store_parts(f16_t* to, float* units, const f32x16 (&acc)[DT], int rows, int g, int lane) {
  const int left = __builtin_amdgcn_readfirstlane(rows);
  typedef typename RowHalves<DT>::V V;
  // largest of row r over 32 lanes, 16 rows at once: with every step a lane keeps half as many of them
  float most[16];
#pragma unroll
  for (int r = 0; r < 16; ++r) {
    most[r] = larger(fabsf(acc[0][r]), fabsf(acc[1][r]));
    if constexpr (DT == 4) most[r] = larger(larger(most[r], fabsf(acc[2][r])), fabsf(acc[3][r]));
  }
#pragma unroll
  for (int r = 0; r < 8; ++r) {   // rows r and r + 8: lanes 0 .. 15 keep the first
    swap_rows(most[r], most[r + 8]);
    most[r] = larger(most[r], most[r + 8]);
  }
  const bool upper = lane & 8;
#pragma unroll
  for (int r = 0; r < 4; ++r) {   // rows r and r + 4: every other eight lanes
    const float keep = upper ? most[r + 4] : most[r], give = upper ? most[r] : most[r + 4];
    most[r] = larger(keep, lane_moved<0x128>(give));
    most[r] = larger(most[r], lane_moved<0xB1>(most[r]));
    most[r] = larger(most[r], lane_moved<0x4E>(most[r]));
    most[r] = larger(most[r], lane_moved<0x141>(most[r]));
  }
  // a lane's four rows are r + 4 (lane / 8 % 4).  2^(141 - e) for a largest number of biased exponent e
  float scale[16];
  float4 unit;
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    const int e = min(max((int)(__float_as_uint(most[r]) >> 23 & 255), 16), 254);
    scale[r] = __uint_as_float((unsigned)(268 - e) << 23);
    (&unit.x)[r] = __uint_as_float((unsigned)(e - 14) << 23);
  }
  const int first_row = 8 * (lane >> 3 & 3) + 4 * g;   // slot(r) + 4 g of them
  // Through buffer resources that end behind the last row: a store under a condition would have the wait for the next tile's queries, which are
  // requested ahead of it, wait for the stores too.
  const auto to_units = __builtin_amdgcn_make_buffer_rsrc(units, 0, left * 4, 0x00020000);
  const auto to_rows = __builtin_amdgcn_make_buffer_rsrc(to, 0, left * (64 * DT), 0x00020000);
#pragma unroll
  for (int r = 0; r < 4; ++r)
    __builtin_amdgcn_raw_buffer_store_b32((int)__float_as_uint((&unit.x)[r]), to_units, (lane & 7) == 0 ? (first_row + r) * 4 : 0x7fffffff, 0, 0);
  // and back to all lanes
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    const float other = lane_moved<0x128>(scale[r]);
    scale[r + 4] = upper ? scale[r] : other;
    scale[r] = upper ? other : scale[r];
  }
#pragma unroll
  for (int r = 0; r < 8; ++r) {
    scale[r + 8] = scale[r];
    swap_rows(scale[r], scale[r + 8]);
  }
#pragma unroll
  for (int r = 0; r < 16; ++r) {
    const int row = slot(r) + 4 * g;
    V v;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) v[dt] = (f16_t)(acc[dt][r] * scale[r]);
    const int at = row * (64 * DT) + (lane & 31) * (2 * DT);
    if constexpr (DT == 4) __builtin_amdgcn_raw_buffer_store_b64(__builtin_bit_cast(u32x2, v), to_rows, at, 0, 0);
    else __builtin_amdgcn_raw_buffer_store_b32(__builtin_bit_cast(int, v), to_rows, at, 0, 0);
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
