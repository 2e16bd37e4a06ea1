// Attention over chosen blocks as the fused attention with a mask (attention_selected_kernel.hpp): where queries choose many of the blocks that
// they could, all tiles of the matrix are computed and blocks that a row has not chosen get weight zero.  No lists, no
// partial results.  A row's choice is a bit a block; that a row has not chosen a block costs nothing a score: its maximum, or the
// log-sum-exp that is subtracted, is infinite for the time of the block.
// Bound: as the fused attention, over all pairs.  16 (sequence, head)s of 4096 x 128, causal: forward 91 us (780 TFLOP/s of all pairs), backward 290
// (the fused attention with no choice 84 and 312 then).
#include "attention_selected_kernel.hpp"

namespace optimus {
namespace {

constexpr int kMaskWords = kMaskedBlocks / 32;

__device__ __forceinline__ float weight_of(float x) { return __builtin_amdgcn_fmed3f(__builtin_amdgcn_exp2f(x), 0.f, 1.f); }
__device__ __forceinline__ float lse2_of(float lse) { return lse == -INFINITY ? INFINITY : lse * LOG2E; }

// Choices of the workgroup's rows as bits, [word][row], a thread a row.
template <int ROWS>
__device__ __forceinline__ void row_blocks(const SelectedArgs& a, int mm, int len, int t0, unsigned (*bits)[ROWS]) {
  const int row = threadIdx.x, t = t0 + row;
  if (row >= ROWS) return;
#pragma unroll
  for (int w = 0; w < kMaskWords; ++w) bits[w][row] = 0;
  if (t >= len) return;
  const int* own = a.selected + ((long long)mm * a.f.s + t) * a.count;
#pragma unroll 4
  for (int e = 0; e < a.count; ++e) {
    const int v = own[e];
    if (v >= 0 && v < a.blocks) bits[v >> 5][row] |= 1u << (v & 31);
  }
}
// block of 64 keys number kb -> block of the choice
__device__ __forceinline__ int block_of(const SelectedArgs& a, int kb) { return (int)divide((unsigned)kb, a.by_steps); }

// Forward: as the attention with changed scores and none of the changes (attention_biased.hip).
template <int D, int NRG>
__global__ __launch_bounds__(NRG * 128, D == 64 && NRG == 4 ? 4 : NRG == 4 || D == 64 ? 2 : 1) void masked_fwd_kernel(SelectedArgs a) {
  constexpr int KS = D / 16, DT = D / 32, BQ = NRG * 32, AHEAD = D == 64 ? 1 : 2;
  __shared__ __attribute__((aligned(1024))) bf16_t lds[2][2][PAIR * D];  // [stage][K, V][pair tile]
  __shared__ unsigned bits[kMaskWords][BQ];
  const FusedArgs& f = a.f;
  const int tid = threadIdx.x, lane = tid & 63, g = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int rg = wave % NRG, par = wave / NRG;
  const int mm = blockIdx.x, tile = gridDim.y - 1 - blockIdx.y;   // the longest causal loops first
  const SelMatrix m = selected_matrix<D>(a, mm);
  const bf16_t* Qp = f.qkv + m.qkv;
  const bf16_t* Kp = Qp + D;
  const bf16_t* Vp = Qp + 2 * D;
  const int s = m.len;
  const int q0 = tile * BQ + rg * 32;
  const int query = q0 + (lane & 31);
  const int qrow = min(query, max(s - 1, 0));
  bf16x8 qf[KS];
#pragma unroll
  for (int ks = 0; ks < KS; ++ks) qf[ks] = *(const bf16x8*)(Qp + (long long)qrow * f.ld + ks * 16 + g * 8);
  const int wg_hi = min(tile * BQ + BQ, s) - 1;   // last query row of the workgroup
  const int kb_hi = tile * BQ >= s ? 0 : (a.causal ? wg_hi : s - 1) / BLK + 1;
  const int n_it = (kb_hi + 1) / 2;
  const int wave_last = q0 >= s ? -1 : a.causal ? min(q0 + 31, s - 1) : s - 1;
  const int limit = a.causal ? qrow : s - 1;

  f32x16 oacc[DT];
#pragma unroll
  for (int dt = 0; dt < DT; ++dt) oacc[dt] = zero16();
  float m_run = -INFINITY, l_run = 0.f;
  bool large = false;
  const unsigned in_rows = lds_address(lds) + lane_rows<D>(lane), in_cols = lds_address(lds) + lane_cols<D>(lane);
  TileLoader<D, 2 * NRG, PAIR, true> ldr;
  ldr.init(f.ld, wave, lane);
  if (n_it > 0) {
    ldr.issue(Kp, 0, s, lds[0][0]);
    ldr.issue(Vp, 0, s, lds[0][1]);
  }
  row_blocks<BQ>(a, mm, s, tile * BQ, bits);
  wait_loads_and_barrier();
  for (int it = 0; it < n_it; ++it) {
    const int st = it & 1;
    if (it + 1 < n_it) {
      ldr.issue(Kp, (it + 1) * PAIR, s, lds[st ^ 1][0]);
      ldr.issue(Vp, (it + 1) * PAIR, s, lds[st ^ 1][1]);
    }
    const int kb = 2 * it + par, kbase = kb * BLK, v = block_of(a, kb);
    const bool chosen = kbase <= wave_last && (bits[v >> 5][rg * 32 + (lane & 31)] >> (v & 31) & 1);
    if (__builtin_amdgcn_ballot_w64(chosen) != 0) {
      const unsigned stage = (unsigned)((st * 2 * PAIR + par * BLK) * D * 2);
      const unsigned kt = in_rows + stage, vt = in_cols + stage;
      f32x16 sacc[2];
      sacc[0] = zero16();
      sacc[1] = zero16();
      pipelined<2 * KS, AHEAD>([&](int n) { return rows_at<D>(kt, n / KS * 32, n % KS); },
                               [&](int n, const bf16x8& x) {
                                 sacc[n / KS] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x, qf[n % KS], sacc[n / KS], 0, 0, 0);
                               });
      const bool masked = a.causal ? kbase + BLK - 1 > q0 : kbase + BLK > s;
      if (masked) {
        const int reach = limit - kbase - 4 * g;
#pragma unroll
        for (int t2 = 0; t2 < 2; ++t2)
#pragma unroll
          for (int r = 0; r < 16; ++r) sacc[t2][r] = 32 * t2 + slot(r) > reach ? -INFINITY : sacc[t2][r];
      }
      float mx = halfwave_max(largest(sacc[1], largest(sacc[0], -INFINITY))) * f.scale_log2;
      mx = chosen ? mx : -INFINITY;
      const bool move = __builtin_amdgcn_ballot_w64(mx > m_run + 8.0f) != 0;
      const float m_new = move ? fmaxf(m_run, mx) : m_run;
      if (move) large = large_scores(m_new);
      const float weight = score_weight(sacc, f.scale_log2, large);
      const float m_sub = m_new == -INFINITY ? 0.f : m_new;
      const float off = chosen ? -m_sub : -INFINITY;
      float sum = 0.f;
#pragma unroll
      for (int t2 = 0; t2 < 2; ++t2)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const float p = __builtin_amdgcn_exp2f(fmaf(sacc[t2][r], weight, off));
          sacc[t2][r] = p;
          sum += p;
        }
      sum = halfwave_sum(sum);
      if (move) {
        const float alpha = __builtin_amdgcn_exp2f(m_run - m_sub);
        l_run *= alpha;
#pragma unroll
        for (int dt = 0; dt < DT; ++dt)
#pragma unroll
          for (int r = 0; r < 16; ++r) oacc[dt][r] *= alpha;
        m_run = m_new;
      }
      l_run += sum;
      bf16x8 pf[2][2];
#pragma unroll
      for (int t2 = 0; t2 < 2; ++t2) {
        pf[t2][0] = pack_acc<0>(sacc[t2]);
        pf[t2][1] = pack_acc<1>(sacc[t2]);
      }
      pipelined<4 * DT, AHEAD>([&](int n) { return cols_at<D>(vt, PAIR + n / DT * 16, n % DT); },
                               [&](int n, const bf16x8& x) {
                                 oacc[n % DT] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x, pf[n / (2 * DT)][n / DT & 1], oacc[n % DT], 0, 0, 0);
                               });
    }
    wait_loads_and_barrier();
  }
  // merge the two parities: the odd one hands (m, l, O) over through LDS
  float* xch = (float*)&lds[0][0][0] + rg * (DT * 16 + 2) * 64;
  if (par == 1) {
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
      for (int r = 0; r < 16; ++r) xch[(dt * 16 + r) * 64 + lane] = oacc[dt][r];
    xch[(DT * 16) * 64 + lane] = m_run;
    xch[(DT * 16 + 1) * 64 + lane] = l_run;
  }
  __syncthreads();
  if (par == 0 && query < f.s) {
    const float m1 = xch[(DT * 16) * 64 + lane], l1 = xch[(DT * 16 + 1) * 64 + lane];
    const float top = fmaxf(m_run, m1), m_sub = top == -INFINITY ? 0.f : top;
    const float a0 = __builtin_amdgcn_exp2f(m_run - m_sub), a1 = __builtin_amdgcn_exp2f(m1 - m_sub);
    const float l = l_run * a0 + l1 * a1;
    const float inv = l == 0.f ? 0.f : 1.0f / l;   // (no pair: zeros; past the end of the sequence nothing is chosen)
    const float w0 = a0 * inv, w1 = a1 * inv;
    bf16_t* Op = f.attn + m.attn + (long long)query * f.ldo;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        float o[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] = oacc[dt][4 * c + e] * w0 + xch[(dt * 16 + 4 * c + e) * 64 + lane] * w1;
        u32x2 x = {pack2_bf16(o[0], o[1]), pack2_bf16(o[2], o[3])};
        *(u32x2*)(Op + dt * 32 + 8 * c + 4 * g) = x;
      }
    if (g == 0) f.lse[m.vec + query] = l == 0.f ? -INFINITY : (m_sub + __log2f(l)) * LN2;
  }
}

// ---------------------------------------------------------------- backward
// Ahead of the others, 128 queries a workgroup: rowsum(dO * O), 0 past the end of a sequence, and the choices by blocks, a bit a query.
constexpr int kPrepared = 128;
template <int D>
__global__ __launch_bounds__(256) void masked_prepare_kernel(SelectedArgs a) {
  __shared__ unsigned bits[kMaskedBlocks][kPrepared / 32];
  const FusedArgs& f = a.f;
  const int tid = threadIdx.x, lane = tid & 63, g = lane >> 5, wave = tid >> 6, mm = blockIdx.y, t0 = blockIdx.x * kPrepared;
  const SelMatrix m = selected_matrix<D>(a, mm);
  for (int k = tid; k < a.blocks * (kPrepared / 32); k += 256) (&bits[0][0])[k] = 0;
  __syncthreads();
  if (tid < kPrepared && t0 + tid < m.len) {
    const int* own = a.selected + (m.vec + t0 + tid) * a.count;
#pragma unroll 4
    for (int e = 0; e < a.count; ++e) {
      const int v = own[e];
      if (v >= 0 && v < a.blocks) atomicOr(&bits[v][tid >> 5], 1u << (tid & 31));
    }
  }
  {
    const int t = t0 + wave * 32 + (lane & 31), row = min(t, f.s - 1);
    float delta = 0.f;
    if (t < m.len) {
      const bf16_t* G = f.d_attn + m.attn + (long long)row * f.ldo + g * 8;
      const bf16_t* O = f.attn + m.attn + (long long)row * f.ldo + g * 8;
#pragma unroll
      for (int ks = 0; ks < D / 16; ++ks) delta += delta_piece(*(const bf16x8*)(G + ks * 16), *(const bf16x8*)(O + ks * 16));
    }
    delta = halfwave_sum(delta);
    if (g == 0 && t < f.s) f.delta[m.vec + t] = delta;
  }
  __syncthreads();
  for (int k = tid; k < a.blocks * (kPrepared / 32); k += 256) {
    const int v = k / (kPrepared / 32), w = k % (kPrepared / 32), at = blockIdx.x * (kPrepared / 32) + w;
    if (at < a.mask_words) a.mask[((long long)mm * a.blocks + v) * a.mask_words + at] = bits[v][w];
  }
}

template <int D, int NRG>
struct MaskedDqLds {
  bf16_t tile[2][2][PAIR * D];   // [stage][K, V]
  unsigned bits[kMaskWords][NRG * 32];
};
template <int D>
struct MaskedDkvLds {
  bf16_t tile[2][2][PAIR * D];   // [stage][Q, dO]
  alignas(16) float l[2][PAIR];
  alignas(16) float d[2][PAIR];
};
struct MaskedWideLds {
  bf16_t block[2][2][BLK * 128];   // [stage][Q, dO]
  bf16_t v[128 * 128], k[128 * 128];
  alignas(16) float l[2][2][BLK];  // [stage][which of the two blocks' choice]
  alignas(16) float d[2][BLK];
};

template <int D, int NRG>
__device__ __forceinline__ void masked_dq_body(const SelectedArgs& a, MaskedDqLds<D, NRG>& lds, int tile, int mm) {
  constexpr int KS = D / 16, DT = D / 32, BQ = NRG * 32;
  const FusedArgs& f = a.f;
  const int tid = threadIdx.x, lane = tid & 63, g = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int rg = wave % NRG, par = wave / NRG;
  const SelMatrix m = selected_matrix<D>(a, mm);
  const bf16_t* Qp = f.qkv + m.qkv;
  const bf16_t* Kp = Qp + D;
  const bf16_t* Vp = Qp + 2 * D;
  const int s = m.len;
  const int q0 = tile * BQ + rg * 32;
  const int query = q0 + (lane & 31);
  const int qrow = min(query, max(s - 1, 0));
  bf16x8 qf[KS], dof[KS];
#pragma unroll
  for (int ks = 0; ks < KS; ++ks) {
    qf[ks] = *(const bf16x8*)(Qp + (long long)qrow * f.ld + ks * 16 + g * 8);
    dof[ks] = *(const bf16x8*)(f.d_attn + m.attn + (long long)qrow * f.ldo + ks * 16 + g * 8);
  }
  const float delta = f.delta[m.vec + qrow], lse = f.lse[m.vec + qrow];
  const int wg_hi = min(tile * BQ + BQ, s) - 1;
  const int kb_hi = tile * BQ >= s ? 0 : (a.causal ? wg_hi : s - 1) / BLK + 1;
  const int n_it = (kb_hi + 1) / 2;
  const int wave_last = q0 >= s ? -1 : a.causal ? min(q0 + 31, s - 1) : s - 1;
  const int limit = a.causal ? qrow : s - 1;
  f32x16 dqacc[DT];
#pragma unroll
  for (int dt = 0; dt < DT; ++dt) dqacc[dt] = zero16();
  const unsigned in_rows = lds_address(lds.tile) + lane_rows<D>(lane), in_cols = lds_address(lds.tile) + lane_cols<D>(lane);
  TileLoader<D, 2 * NRG, PAIR, true> ldr;
  ldr.init(f.ld, wave, lane);
  if (n_it > 0) {
    ldr.issue(Kp, 0, s, lds.tile[0][0]);
    ldr.issue(Vp, 0, s, lds.tile[0][1]);
  }
  row_blocks<BQ>(a, mm, s, tile * BQ, lds.bits);
  const float lse2 = lse2_of(lse);
  wait_loads_and_barrier();
  for (int it = 0; it < n_it; ++it) {
    const int st = it & 1;
    if (it + 1 < n_it) {
      ldr.issue(Kp, (it + 1) * PAIR, s, lds.tile[st ^ 1][0]);
      ldr.issue(Vp, (it + 1) * PAIR, s, lds.tile[st ^ 1][1]);
    }
    const int kb = 2 * it + par, kbase = kb * BLK, v = block_of(a, kb);
    const bool chosen = kbase <= wave_last && (lds.bits[v >> 5][rg * 32 + (lane & 31)] >> (v & 31) & 1);
    if (__builtin_amdgcn_ballot_w64(chosen) != 0) {
      const unsigned stage = (unsigned)((st * 2 * PAIR + par * BLK) * D * 2);
      const unsigned kt = in_rows + stage, kc = in_cols + stage;
      const bool masked = a.causal ? kbase + BLK - 1 > q0 : kbase + BLK > s;
      const float off = chosen ? lse2 : INFINITY;
#pragma unroll
      for (int t2 = 0; t2 < 2; ++t2) {
        f32x16 sacc = zero16(), pacc = zero16();
        pipelined<2 * KS, 2>([&](int n) { return rows_at<D>(kt, (n & 1 ? PAIR : 0) + t2 * 32, n / 2); },
                             [&](int n, const bf16x8& x) {
                               f32x16& acc = n & 1 ? pacc : sacc;
                               acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x, n & 1 ? dof[n / 2] : qf[n / 2], acc, 0, 0, 0);
                             });
        const int reach = limit - kbase - 32 * t2 - 4 * g;
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          float p = weight_of(fmaf(sacc[r], f.scale_log2, -off));
          if (masked && slot(r) > reach) p = 0.f;
          sacc[r] = p * (pacc[r] - delta);   // dS^T
        }
        const bf16x8 dsf[2] = {pack_acc<0>(sacc), pack_acc<1>(sacc)};
        pipelined<2 * DT, 2>([&](int n) { return cols_at<D>(kc, t2 * 32 + n / DT * 16, n % DT); },
                             [&](int n, const bf16x8& x) {
                               const int dt = n % DT;
                               dqacc[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x, dsf[n / DT], dqacc[dt], 0, 0, 0);
                             });
      }
    }
    wait_loads_and_barrier();
  }
  float* xch = (float*)&lds.tile[0][0][0] + rg * (DT * 16) * 64;
  if (par == 1) {
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
      for (int r = 0; r < 16; ++r) xch[(dt * 16 + r) * 64 + lane] = dqacc[dt][r];
  }
  __syncthreads();
  if (par == 0 && query < f.s) {
    bf16_t* dQp = f.d_qkv + m.qkv + (long long)query * f.ld;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        float o[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] = (dqacc[dt][4 * c + e] + xch[(dt * 16 + 4 * c + e) * 64 + lane]) * f.scale;
        u32x2 w = {pack2_bf16(o[0], o[1]), pack2_bf16(o[2], o[3])};
        *(u32x2*)(dQp + dt * 32 + 8 * c + 4 * g) = w;
      }
  }
}

// 32 x 32 scores (rows: queries q0 .., columns: keys) and dP -> P and dS in their place.  l, d: of the 32 queries, l infinite for those that
// have not chosen the keys' block
__device__ __forceinline__ void masked_scores(f32x16& sacc, f32x16& pacc, const float* l, const float* d, float scale_log2, bool masked, int reach, int g) {
#pragma unroll
  for (int c = 0; c < 4; ++c) {
    const float4 l4 = *(const float4*)(l + 8 * c + 4 * g), d4 = *(const float4*)(d + 8 * c + 4 * g);
    const float lv[4] = {l4.x, l4.y, l4.z, l4.w}, dv[4] = {d4.x, d4.y, d4.z, d4.w};
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int r = 4 * c + e;
      float p = weight_of(fmaf(sacc[r], scale_log2, -lv[e]));
      if (masked && slot(r) < reach) p = 0.f;
      sacc[r] = p;
      pacc[r] = p * (pacc[r] - dv[e]);
    }
  }
}

template <int D, int NRG>
__device__ __forceinline__ void masked_dkv_body(const SelectedArgs& a, MaskedDkvLds<D>& lds, int tile, int mm) {
  constexpr int KS = D / 16, DT = D / 32, BKW = NRG * 32;
  static_assert(NRG == 2, "64 keys, which are of one block");
  const FusedArgs& f = a.f;
  const int tid = threadIdx.x, lane = tid & 63, g = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int rg = wave % NRG, par = wave / NRG;
  const SelMatrix m = selected_matrix<D>(a, mm);
  const int s = m.len;
  const bf16_t* Qp = f.qkv + m.qkv;
  const bf16_t* Gp = f.d_attn + m.attn;
  const float* Lp = f.lse + m.vec;
  const float* Dp = f.delta + m.vec;
  const int kt0 = tile * BKW, k0 = kt0 + rg * 32;
  const int key = k0 + (lane & 31);
  const int krow = min(key, max(s - 1, 0));
  const unsigned* mask = a.mask + ((long long)mm * a.blocks + block_of(a, tile)) * a.mask_words;
  bf16x8 kf[KS], vf[KS];
#pragma unroll
  for (int ks = 0; ks < KS; ++ks) {
    kf[ks] = *(const bf16x8*)(Qp + D + (long long)krow * f.ld + ks * 16 + g * 8);
    vf[ks] = *(const bf16x8*)(Qp + 2 * D + (long long)krow * f.ld + ks * 16 + g * 8);
  }
  const int qb_lo = a.causal ? kt0 / BLK : 0, qb_hi = kt0 >= s ? 0 : (s + BLK - 1) / BLK;
  const int it_lo = qb_lo / 2, n_it = (qb_hi + 1) / 2;
  f32x16 dkacc[DT], dvacc[DT];
#pragma unroll
  for (int dt = 0; dt < DT; ++dt) {
    dkacc[dt] = zero16();
    dvacc[dt] = zero16();
  }
  const unsigned in_rows = lds_address(lds.tile) + lane_rows<D>(lane), in_cols = lds_address(lds.tile) + lane_cols<D>(lane);
  TileLoader<D, 2 * NRG, PAIR, true> ldq, ldg;
  ldq.init(f.ld, wave, lane);
  ldg.init(f.ldo, wave, lane);
  float next_l = 0.f, next_d = 0.f;
  auto load_pair = [&](int it, int st) {
    if (tid < PAIR) {
      const int row = it * PAIR + tid, at = min(row, s - 1);
      next_l = row < s && (mask[row >> 5] >> (row & 31) & 1) ? lse2_of(Lp[at]) : INFINITY;
      next_d = Dp[at];
    }
    ldq.issue(Qp, it * PAIR, s, lds.tile[st][0]);
    ldg.issue(Gp, it * PAIR, s, lds.tile[st][1]);
  };
  auto store_rows = [&](int st) {
    if (tid < PAIR) {
      lds.l[st][tid] = next_l;
      lds.d[st][tid] = next_d;
    }
  };
  if (it_lo < n_it) load_pair(it_lo, 0);
  store_rows(0);
  wait_loads_and_barrier();
  for (int it = it_lo; it < n_it; ++it) {
    const int st = (it - it_lo) & 1;
    if (it + 1 < n_it) load_pair(it + 1, st ^ 1);
    const int qb = 2 * it + par, qbase = qb * BLK;
    const bool any = __builtin_amdgcn_ballot_w64(lds.l[st][par * BLK + lane] < INFINITY) != 0;   // of the 64 queries
    if (k0 < s && qb >= qb_lo && qb < qb_hi && (!a.causal || qbase + BLK - 1 >= k0) && any) {
      const unsigned stage = (unsigned)((st * 2 * PAIR + par * BLK) * D * 2);
      const unsigned qt = in_rows + stage, qc = in_cols + stage;
      const bool masked = a.causal && qbase < k0 + 31;
#pragma unroll
      for (int t2 = 0; t2 < 2; ++t2) {
        f32x16 sacc = zero16(), pacc = zero16();
        pipelined<2 * KS, 2>([&](int n) { return rows_at<D>(qt, (n & 1 ? PAIR : 0) + t2 * 32, n / 2); },
                             [&](int n, const bf16x8& x) {
                               f32x16& acc = n & 1 ? pacc : sacc;
                               acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x, n & 1 ? vf[n / 2] : kf[n / 2], acc, 0, 0, 0);
                             });
        const int at = par * BLK + t2 * 32;
        masked_scores(sacc, pacc, lds.l[st] + at, lds.d[st] + at, f.scale_log2, masked, key - qbase - t2 * 32 - 4 * g, g);
        const bf16x8 pf[2] = {pack_acc<0>(sacc), pack_acc<1>(sacc)}, dsf[2] = {pack_acc<0>(pacc), pack_acc<1>(pacc)};
        pipelined<4 * DT, 2>([&](int n) { return cols_at<D>(qc, (n & 1 ? 0 : PAIR) + t2 * 32 + n / (2 * DT) * 16, n / 2 % DT); },
                             [&](int n, const bf16x8& x) {
                               const int dt = n / 2 % DT, u = n / (2 * DT);
                               f32x16& acc = n & 1 ? dkacc[dt] : dvacc[dt];
                               acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x, n & 1 ? dsf[u] : pf[u], acc, 0, 0, 0);
                             });
      }
    }
    if (it + 1 < n_it) store_rows(st ^ 1);
    wait_loads_and_barrier();
  }
  float* xch = (float*)&lds.tile[0][0][0] + rg * (2 * DT * 16) * 64;
  if (par == 1) {
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        xch[(dt * 16 + r) * 64 + lane] = dkacc[dt][r];
        xch[((DT + dt) * 16 + r) * 64 + lane] = dvacc[dt][r];
      }
  }
  __syncthreads();
  if (par == 0 && key < f.s) {   // (past the end of the sequence: zeros, whatever the last key's row gave)
    const float w = key < s ? 1.0f : 0.f;
    bf16_t* dKp = f.d_qkv + m.qkv + (long long)key * f.ld + D;
    bf16_t* dVp = dKp + D;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        float k4[4], v4[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          k4[e] = w == 0.f ? 0.f : (dkacc[dt][4 * c + e] + xch[(dt * 16 + 4 * c + e) * 64 + lane]) * f.scale;
          v4[e] = w == 0.f ? 0.f : dvacc[dt][4 * c + e] + xch[((DT + dt) * 16 + 4 * c + e) * 64 + lane];
        }
        u32x2 wk = {pack2_bf16(k4[0], k4[1]), pack2_bf16(k4[2], k4[3])};
        u32x2 wv = {pack2_bf16(v4[0], v4[1]), pack2_bf16(v4[2], v4[3])};
        *(u32x2*)(dKp + dt * 32 + 8 * c + 4 * g) = wk;
        *(u32x2*)(dVp + dt * 32 + 8 * c + 4 * g) = wv;
      }
  }
}

// Head width 128, 128 keys, eight wavefronts (see the attention with changed scores): own V rows and half of the K fragments in LDS, 64 queries
// at a time, a wavefront half of them.  The keys are of one or two blocks.
__device__ __forceinline__ void masked_dkv_wide_body(const SelectedArgs& a, MaskedWideLds& lds, int tile, int mm) {
  constexpr int D = 128, KS = D / 16, DT = D / 32, BKW = 128, KREG = KS / 2;
  const FusedArgs& f = a.f;
  const int tid = threadIdx.x, lane = tid & 63, g = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int rg = wave & 3, par = wave >> 2;
  const SelMatrix m = selected_matrix<D>(a, mm);
  const int s = m.len;
  const bf16_t* Qp = f.qkv + m.qkv;
  const bf16_t* Gp = f.d_attn + m.attn;
  const float* Lp = f.lse + m.vec;
  const float* Dp = f.delta + m.vec;
  const int kt0 = tile * BKW, k0 = kt0 + rg * 32;
  const int key = k0 + (lane & 31);
  const int krow = min(key, max(s - 1, 0));
  const unsigned* mask0 = a.mask + ((long long)mm * a.blocks + block_of(a, 2 * tile)) * a.mask_words;
  const unsigned* mask1 = a.mask + ((long long)mm * a.blocks + min(block_of(a, 2 * tile + 1), a.blocks - 1)) * a.mask_words;
  bf16x8 kf[KREG];
#pragma unroll
  for (int ks = 0; ks < KREG; ++ks) kf[ks] = *(const bf16x8*)(Qp + D + (long long)krow * f.ld + ks * 16 + g * 8);
  if (kt0 < s) {
    TileLoader<D, 8, BKW, true> own;
    own.init(f.ld, wave, lane);
    own.issue(Qp + 2 * D, kt0, s, lds.v);
    own.issue(Qp + D, kt0, s, lds.k);
  }
  const int qb_lo = a.causal ? kt0 / BLK : 0, qb_hi = kt0 >= s ? 0 : (s + BLK - 1) / BLK;
  f32x16 dkacc[DT], dvacc[DT];
#pragma unroll
  for (int dt = 0; dt < DT; ++dt) {
    dkacc[dt] = zero16();
    dvacc[dt] = zero16();
  }
  const unsigned in_rows = lds_address(lds.block) + lane_rows<D>(lane) + par * 32 * D * 2, in_cols = lds_address(lds.block) + lane_cols<D>(lane) + par * 32 * D * 2;
  const unsigned own_rows = lds_address(lds.v) + lane_rows<D>(lane) + rg * 32 * D * 2;
  TileLoader<D, 8, BLK, true> ldq, ldg;
  ldq.init(f.ld, wave, lane);
  ldg.init(f.ldo, wave, lane);
  float next_l[2] = {0.f, 0.f}, next_d = 0.f;
  auto load_block = [&](int qb, int st) {
    if (tid < BLK) {
      const int row = qb * BLK + tid, at = min(row, s - 1);
      const float l = row < s ? lse2_of(Lp[at]) : INFINITY;
      next_l[0] = row < s && (mask0[row >> 5] >> (row & 31) & 1) ? l : INFINITY;
      next_l[1] = row < s && (mask1[row >> 5] >> (row & 31) & 1) ? l : INFINITY;
      next_d = Dp[at];
    }
    ldq.issue(Qp, qb * BLK, s, lds.block[st][0]);
    ldg.issue(Gp, qb * BLK, s, lds.block[st][1]);
  };
  auto store_rows = [&](int st) {
    if (tid < BLK) {
      lds.l[st][0][tid] = next_l[0];
      lds.l[st][1][tid] = next_l[1];
      lds.d[st][tid] = next_d;
    }
  };
  if (qb_lo < qb_hi) load_block(qb_lo, 0);
  store_rows(0);
  wait_loads_and_barrier();
  for (int qb = qb_lo; qb < qb_hi; ++qb) {
    const int st = (qb - qb_lo) & 1;
    if (qb + 1 < qb_hi) load_block(qb + 1, st ^ 1);
    const int q0 = qb * BLK + par * 32;   // this wavefront's queries
    const float* l = lds.l[st][rg >> 1] + par * 32;
    const bool any = __builtin_amdgcn_ballot_w64(l[lane & 31] < INFINITY) != 0;
    if (k0 < s && q0 < s && (!a.causal || q0 + 31 >= k0) && any) {
      const unsigned stage = (unsigned)(st * 2 * BLK * D * 2);
      const unsigned qt = in_rows + stage, qc = in_cols + stage;
      f32x16 sacc = zero16(), pacc = zero16();
      struct Two { bf16x8 q, own; };
      pipelined<2 * KS, 2>([&](int n) {
                             const int ks = n / 2;
                             Two x;
                             x.q = rows_at<D>(qt, n & 1 ? BLK : 0, ks);
                             if (n & 1) x.own = rows_at<D>(own_rows, 0, ks);
                             else x.own = ks < KREG ? kf[ks < KREG ? ks : 0] : rows_at<D>(own_rows, BKW, ks);
                             return x;
                           },
                           [&](int n, const Two& x) {
                             f32x16& acc = n & 1 ? pacc : sacc;
                             acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x.q, x.own, acc, 0, 0, 0);
                           });
      masked_scores(sacc, pacc, l, lds.d[st] + par * 32, f.scale_log2, a.causal && q0 < k0 + 31, key - q0 - 4 * g, g);
      const bf16x8 pf[2] = {pack_acc<0>(sacc), pack_acc<1>(sacc)}, dsf[2] = {pack_acc<0>(pacc), pack_acc<1>(pacc)};
      pipelined<4 * DT, 2>([&](int n) { return cols_at<D>(qc, (n & 1 ? 0 : BLK) + n / (2 * DT) * 16, n / 2 % DT); },
                           [&](int n, const bf16x8& x) {
                             const int dt = n / 2 % DT, u = n / (2 * DT);
                             f32x16& acc = n & 1 ? dkacc[dt] : dvacc[dt];
                             acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x, n & 1 ? dsf[u] : pf[u], acc, 0, 0, 0);
                           });
    }
    if (qb + 1 < qb_hi) store_rows(st ^ 1);
    wait_loads_and_barrier();
  }
  // merge the two halves' sums, dV first: the odd one hands over through LDS (64 KiB, all block tiles are free)
  float* xch = (float*)&lds.block[0][0][0] + rg * (DT * 16) * 64;
  bf16_t* dKp = f.d_qkv + m.qkv + (long long)key * f.ld + D;
#pragma unroll
  for (int which = 0; which < 2; ++which) {
    f32x16 (&acc)[DT] = which == 0 ? dvacc : dkacc;
    if (which == 1) __syncthreads();
    if (par == 1) {
#pragma unroll
      for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int r = 0; r < 16; ++r) xch[(dt * 16 + r) * 64 + lane] = acc[dt][r];
    }
    __syncthreads();
    if (par == 0 && key < f.s) {
      const float w = which == 0 ? 1.0f : f.scale;
#pragma unroll
      for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          float o[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) o[e] = key < s ? (acc[dt][4 * c + e] + xch[(dt * 16 + 4 * c + e) * 64 + lane]) * w : 0.f;
          u32x2 x = {pack2_bf16(o[0], o[1]), pack2_bf16(o[2], o[3])};
          *(u32x2*)(dKp + (which == 0 ? D : 0) + dt * 32 + 8 * c + 4 * g) = x;
        }
    }
  }
}

template <size_t A, size_t B>
constexpr size_t larger() { return A > B ? A : B; }

// Both kinds in one grid ordered by loop length, longest first, the kinds alternating: x = (matrix, kind), y = rank.
template <int D>
__global__ __launch_bounds__(256, D == 64 ? 2 : 1) void masked_bwd_kernel(SelectedArgs a) {
  __shared__ __attribute__((aligned(1024))) char lds[larger<sizeof(MaskedDqLds<D, 2>), sizeof(MaskedDkvLds<D>)>()];
  const int rank = blockIdx.y, mm = blockIdx.x >> 1, ntiles = gridDim.y;
  if (blockIdx.x & 1) masked_dq_body<D, 2>(a, *(MaskedDqLds<D, 2>*)lds, ntiles - 1 - rank, mm);
  else masked_dkv_body<D, 2>(a, *(MaskedDkvLds<D>*)lds, rank, mm);
}
__global__ __launch_bounds__(512, 2) void masked_bwd_wide_kernel(SelectedArgs a) {
  __shared__ __attribute__((aligned(1024))) char lds[larger<sizeof(MaskedWideLds), sizeof(MaskedDqLds<128, 4>)>()];
  const int rank = blockIdx.y, mm = blockIdx.x >> 1, ntiles = gridDim.y;
  if (blockIdx.x & 1) masked_dq_body<128, 4>(a, *(MaskedDqLds<128, 4>*)lds, ntiles - 1 - rank, mm);
  else masked_dkv_wide_body(a, *(MaskedWideLds*)lds, rank, mm);
}

template <int D>
void fwd_launch(const SelectedArgs& a, int mats, hipStream_t st) {
  // 64-row workgroups as long as all of them run at once, as in the attention with changed scores; the bits are the same
  const bool wide = (long long)((a.f.s + BLK - 1) / BLK) * mats > num_cus() * (D == 64 ? 2 : 1);
  if (wide) masked_fwd_kernel<D, 4><<<dim3(mats, (a.f.s + 127) / 128), 512, 0, st>>>(a);
  else masked_fwd_kernel<D, 2><<<dim3(mats, (a.f.s + BLK - 1) / BLK), 256, 0, st>>>(a);
}
template <int D>
void bwd_launch(const SelectedArgs& a, int mats, hipStream_t st) {
  masked_prepare_kernel<D><<<dim3((a.f.s + kPrepared - 1) / kPrepared, mats), 256, 0, st>>>(a);
  if constexpr (D == 128) {
    // the two forms add dK and dV up in different orders: the choice follows one device's matrices, whatever the launch covers
    if (2ll * ((a.f.s + BLK - 1) / BLK) * a.nmat > num_cus()) {
      masked_bwd_wide_kernel<<<dim3(2 * mats, (a.f.s + 127) / 128), 512, 0, st>>>(a);
      return;
    }
  }
  masked_bwd_kernel<D><<<dim3(2 * mats, (a.f.s + BLK - 1) / BLK), 256, 0, st>>>(a);
}

}  // namespace

void launch_selected_masked(const SelectedArgs& a, int mats, int d, bool bwd, hipStream_t st) {
  if (bwd) {
    if (d == 64) bwd_launch<64>(a, mats, st);
    else bwd_launch<128>(a, mats, st);
  } else {
    if (d == 64) fwd_launch<64>(a, mats, st);
    else fwd_launch<128>(a, mats, st);
  }
}

}  // namespace optimus
