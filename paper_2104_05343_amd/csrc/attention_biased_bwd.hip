// Backward of the attention with changed scores (attention_biased_kernel.hpp): dQ and the table's gradient by workgroups that own
// queries, dK and dV by workgroups that own keys, both kinds in one grid as in the attention without changes.
#include "attention_biased_kernel.hpp"

namespace optimus {
namespace {

// The sums of dS over the buckets, of one wavefront.  A lane owns a bucket (and the one 64 further).  A 32 x 32 tile that lies in the
// last bucket as a whole is summed lane by lane; another one is summed along its 63 diagonals first.  Eight keys at a time go to LDS,
// each moved by its place, so that the diagonals are columns, which a lane each adds up; places that no score reaches stay zero.
// (Adding into 63 places with LDS's float additions took some 6000 clk a tile: 8 sequences of 8 heads, s = 2048, width 64, causal,
// backward 426 us, so 240, without the table's gradient 227.)
constexpr int kSkew = 41;   // places of a key: 39 diagonals, zeros behind them; of the halves' rows, four apart, in different banks
constexpr int kSkewed = 8 * kSkew;
struct BucketSums {
  double own[2], far_pos, far_neg;   // (a few additions a tile, each tile a tree of fp32 ones)
  int lo[2], hi[2];      // distances of the lane's buckets
  int far, back;
  float* skewed;         // LDS of the wavefront: [8][kSkew], and [64] behind it
  float* line;
  __device__ __forceinline__ void init(const BiasedArgs& a, float* lds, const int* first_, int lane) {
    skewed = lds;
    line = lds + kSkewed;
    own[0] = own[1] = far_pos = far_neg = 0.0;
    far = a.far; back = a.two_sided ? a.far : 0;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const int b = lane + 64 * k;
      lo[k] = 1; hi[k] = 0;
      if (b < a.side) {
        lo[k] = b == 0 && !a.two_sided ? -0x40000000 : first_[b];
        hi[k] = b + 1 < a.side ? first_[b + 1] - 1 : 0x40000000;
      } else if (b < a.buckets) {   // (two-sided) distances below zero
        const int n = b - a.side;
        lo[k] = n + 1 < a.side ? -(first_[n + 1] - 1) : -0x40000000;
        hi[k] = -max(first_[n], 1);
      }
    }
    for (int k = lane; k < kSkewed; k += 64) skewed[k] = 0.f;
  }
  // ds: the tile's scores, whose distances are base .. base + 62
  __device__ __forceinline__ void add(const f32x16& ds, int base, int g, int lane, bool wide) {
    if (base >= far || base + 62 <= -back) {
      float t[8];
#pragma unroll
      for (int r = 0; r < 8; ++r) t[r] = ds[r] + ds[r + 8];
      const float sum = ((t[0] + t[1]) + (t[2] + t[3])) + ((t[4] + t[5]) + (t[6] + t[7]));
      if (base >= far) far_pos += sum;
      else far_neg += sum;
      return;
    }
    // key 8c + 4g + e against query t: diagonal t - key + 31, place t - (4g + e) + 7 of row 4g + e
    float* to_place = skewed + 4 * g * kSkew + (lane & 31) - 4 * g + 7;
    float run = 0.f;
#pragma unroll
    for (int c = 0; c < 4; ++c) {
#pragma unroll
      for (int e = 0; e < 4; ++e) to_place[e * (kSkew - 1)] = ds[4 * c + e];
      __builtin_amdgcn_wave_barrier();
      const int place = lane - 24 + 8 * c;   // of the lane's diagonal
      const float* column = skewed + (place >= 0 && place < 39 ? place : 39);
      float x[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) x[k] = column[k * kSkew];
      run += ((x[0] + x[1]) + (x[2] + x[3])) + ((x[4] + x[5]) + (x[6] + x[7]));
      __builtin_amdgcn_wave_barrier();
    }
    line[lane] = run;   // (63 diagonals: the last place is zero)
    __builtin_amdgcn_wave_barrier();
    // A lane adds its buckets' diagonals up, eight reads in flight.  (Differences of one running sum over all of them are shorter, but
    // leave a small bucket the rounding errors of its neighbours.)
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      if (k == 1 && !wide) break;
      const int from = max(lo[k] - base, 0), to = min(hi[k] - base, 62);
      for (int d = from; d <= to; d += 8) {
        float x[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = line[d + e <= to ? d + e : 63];
        own[k] += ((x[0] + x[1]) + (x[2] + x[3])) + ((x[4] + x[5]) + (x[6] + x[7]));
      }
    }
    __builtin_amdgcn_wave_barrier();
  }
  __device__ __forceinline__ void finish(const BiasedArgs& a, int lane) {   // the far sums to their buckets' lanes
#pragma unroll
    for (int step = 1; step < 64; step <<= 1) {
      far_pos += __shfl_xor(far_pos, step);
      far_neg += __shfl_xor(far_neg, step);
    }
    const int pos = a.side - 1, neg = a.two_sided ? a.buckets - 1 : 0;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      if (lane + 64 * k == pos) own[k] += far_pos;
      if (lane + 64 * k == neg) own[k] += far_neg;
    }
  }
};

// 128-row workgroups of width 64 are for sequences without documents (attn_biased_bwd_wide) and compiled without them: 16 matrices of
// 4096, causal, 149 us; with the branches for documents 158.
template <int D, int NRG>
constexpr bool no_documents() { return D == 64 && NRG == 4; }

template <int D, int NRG, int BIAS>
struct DqLds {
  bf16_t tile[2][2][PAIR * D];   // [stage][K, V]
  BiasLds<BIAS> bias;
  alignas(16) int key_docs[2 * NRG][BLK];   // (read sixteen bytes at a time)
  float sums[BIAS == 2 ? 2 * NRG : 1][BIAS == 2 ? kSkewed + 64 : 1];   // BucketSums; at the end the buckets (128)
};
template <int D, int NRG, int BIAS>
struct DkvLds {
  bf16_t tile[2][2][PAIR * D];   // [stage][Q, dO]
  BiasLds<BIAS> bias;
  alignas(16) float l[2][PAIR];   // (read sixteen bytes at a time, as the next two)
  alignas(16) float d[2][PAIR];
  alignas(16) int docs[2][PAIR];
};

// P = 2^x is at most 1: beyond it (the instruction's own clamp, which costs nothing) lies what the rounding of a log-sum-exp beyond some
// millions makes of it, in the end an infinity that would turn gradients of zero into NaN.
__device__ __forceinline__ float weight_of(float x) { return __builtin_amdgcn_fmed3f(__builtin_amdgcn_exp2f(x), 0.f, 1.f); }

// log-sum-exp of a row -> what is subtracted from its scores.  Of a row without pairs +infinity, which makes every P of it zero.
__device__ __forceinline__ float lse2_of(float lse) { return lse == -INFINITY ? INFINITY : lse * LOG2E; }

template <int D, int NRG, int CAP, int BIAS>
__device__ __forceinline__ void biased_dq_body(const BiasedArgs& a, DqLds<D, NRG, BIAS>& lds, int tile, int mat, int dev) {
  constexpr int KS = D / 16, DT = D / 32, BQ = NRG * 32;
  const FusedArgs& f = a.f;
  const int tid = threadIdx.x, lane = tid & 63, g = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int rg = wave % NRG, par = wave / NRG;
  const int s = f.s;
  Matrix m = matrix_of<D>(a, mat, dev);
  if (no_documents<D, NRG>()) m.docs = nullptr;
  const bf16_t* Qp = f.qkv + m.qkv;
  const bf16_t* Kp = Qp + D;
  const bf16_t* Vp = Qp + 2 * D;
  const int q0 = tile * BQ + rg * 32;
  const int query = q0 + (lane & 31);
  const int qrow = min(query, s - 1);
  const int qdoc = m.docs ? m.docs[qrow] : 0;
  bf16x8 qf[KS], dof[KS];
#pragma unroll
  for (int ks = 0; ks < KS; ++ks) {
    qf[ks] = *(const bf16x8*)(Qp + (long long)qrow * f.ld + ks * 16 + g * 8);
    dof[ks] = *(const bf16x8*)(f.d_attn + m.attn + (long long)qrow * f.ldo + ks * 16 + g * 8);
  }
  const float delta = f.delta[m.vec + qrow], lse = f.lse[m.vec + qrow];

  const int wg_hi = min(tile * BQ + BQ, s) - 1;
  int kb_lo = 0, kb_hi = a.causal ? max(wg_hi, m.prefix - 1) / BLK + 1 : a.nblk;
  if (m.docs) live_blocks(m.blocks, tile * BQ / BLK, wg_hi / BLK, kb_lo, kb_hi);
  const int it_lo = kb_lo / 2, n_it = (kb_hi + 1) / 2;
  const int wave_last = q0 >= s ? -1 : a.causal ? max(min(q0 + 31, s - 1), m.prefix - 1) : s - 1;
  const int limit = a.causal ? max(qrow, m.prefix - 1) : s - 1;
  const i32x4_t none = {0x7fffffff, -1, 0, 0};
  const i32x4_t own = m.docs && q0 < s ? m.blocks[q0 / BLK] : none;

  f32x16 dqacc[DT];
#pragma unroll
  for (int dt = 0; dt < DT; ++dt) dqacc[dt] = zero16();

  const unsigned in_rows = lds_address(lds.tile) + lane_rows<D>(lane), in_cols = lds_address(lds.tile) + lane_cols<D>(lane);
  RowLoader<D, 2 * NRG, PAIR> ldr;
  ldr.init(f.ld, wave, lane);
  struct Pair { i32x4_t even, odd; };
  auto pair_of = [&](int it) {
    Pair p = {none, none};
    if (m.docs) {
      if (2 * it < a.nblk) p.even = m.blocks[2 * it];
      if (2 * it + 1 < a.nblk) p.odd = m.blocks[2 * it + 1];
    }
    return p;
  };
  auto issue = [&](int it, int st, const Pair& p) {
    const int* docs = p.even.z | p.odd.z ? m.docs : nullptr;
    ldr.issue(Kp, it * PAIR, s, lds.tile[st][0], docs);
    ldr.issue(Vp, it * PAIR, s, lds.tile[st][1], docs);
  };
  Pair cur = pair_of(it_lo), next = pair_of(it_lo + 1);
  int first_doc = 0;
  if (it_lo < n_it) {
    if (m.docs) first_doc = m.docs[min((2 * it_lo + par) * BLK + lane, s - 1)];
    issue(it_lo, 0, cur);
  }
  // (behind the first tiles' request: it waits for loads of its own)
  const Bias bias = make_bias<BIAS>(a, m.ghead, lds.bias);
  BucketSums sums;
  const bool table_grad = BIAS == 2 && a.table_parts;
  if (BIAS == 2) sums.init(a, lds.sums[wave], lds.bias.first, lane);
  const float lse2 = query < s && qdoc >= 0 ? lse2_of(lse) : INFINITY;
  // The table's gradient is an fp32 sum: there the part of lse * log2(e) that its rounding loses is kept, in terms of the last place of
  // a number around 20 a relative error of P.  (lse2 infinite: its row has no P.)
  const float lse2_lo = BIAS == 2 && lse2 < 1e30f ? fmaf(lse, LOG2E, -lse2) + lse * 1.92596299e-8f : 0.f;
#pragma unroll
  for (int ks = 0; ks < KS; ++ks) {
    qf[ks] = zero_if(qdoc < 0, qf[ks]);
    dof[ks] = zero_if(qdoc < 0, dof[ks]);
  }
  lds.key_docs[wave][lane] = first_doc;
  wait_loads_and_barrier();
  for (int it = it_lo; it < n_it; ++it) {
    const int st = (it - it_lo) & 1;
    int next_doc = -1;
    Pair after = next;
    if (it + 1 < n_it) {
      if (m.docs) {
        next_doc = m.docs[min((2 * (it + 1) + par) * BLK + lane, s - 1)];
        after = pair_of(it + 2);
      }
      issue(it + 1, st ^ 1, next);
    }
    const int kb = 2 * it + par, kbase = kb * BLK;
    const i32x4_t blk = par ? cur.odd : cur.even;
    const bool shared = !m.docs || share_documents(blk, own);
    if (kb >= kb_lo && kb < kb_hi && kbase <= wave_last && shared) {
      const unsigned stage = (unsigned)((st * 2 * PAIR + par * BLK) * D * 2);
      const unsigned kt = in_rows + stage, kc = in_cols + stage;
      const bool masked = (a.causal ? kbase + BLK - 1 > max(q0, m.prefix - 1) : kbase + BLK > s) || (m.docs && !one_document(blk, own));
#pragma unroll
      for (int t2 = 0; t2 < 2; ++t2) {
        f32x16 sacc = zero16(), pacc = zero16();
        pipelined<2 * KS, 2>([&](int n) { return rows_at<D>(kt, (n & 1 ? PAIR : 0) + t2 * 32, n / 2); },
                            [&](int n, const bf16x8& x) {
                              f32x16& acc = n & 1 ? pacc : sacc;
                              acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x, n & 1 ? dof[n / 2] : qf[n / 2], acc, 0, 0, 0);
                            });
        const int k0 = kbase + t2 * 32, dist0 = query - k0 - 4 * g;
        // the table's gradient wants dS before the tanh's part: that waits in `part` then; else it goes into dP first
        f32x16 part;
        if (CAP) tanh16<CAP, BIAS == 2>(sacc, a);
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          pacc[r] -= delta;
          if (CAP && BIAS != 2) pacc[r] *= fmaf(-sacc[r], sacc[r], 1.0f);
          if (CAP && BIAS == 2) part[r] = fmaf(-sacc[r], sacc[r], 1.0f);
        }
        const int lo = q0 - k0 - 31;
        if (masked || !plain_tile<BIAS>(bias, lo, lo + 62)) {
          any16<CAP, BIAS, -1, BIAS == 2>(sacc, a, bias, dist0, k0 + 4 * g, limit, &lds.key_docs[wave][t2 * 32 + 4 * g], qdoc, lse2, lse2_lo);
#pragma unroll
          for (int r = 0; r < 16; ++r) sacc[r] = weight_of(BIAS == 2 ? sacc[r] : sacc[r] - lse2) * pacc[r];  // dS^T
        } else {
          float w, c;
          plain_weights<CAP, BIAS>(a, bias, lo, w, c);
          plain16<CAP, BIAS, -1>(sacc, a, bias, dist0, lo);
          c -= BIAS == 2 ? lse2_lo : lse2;
#pragma unroll
          for (int r = 0; r < 16; ++r)
            sacc[r] = weight_of(BIAS == 2 ? fmaf(sacc[r], w, -lse2) + fmaf(sacc[r], a.weight_lo, c) : fmaf(sacc[r], w, c)) * pacc[r];
        }
        if (BIAS == 2 && table_grad) sums.add(sacc, lo, g, lane, a.buckets > 64);
        if (CAP && BIAS == 2) {
#pragma unroll
          for (int r = 0; r < 16; ++r) sacc[r] *= part[r];
        }
        const bf16x8 dsf[2] = {pack_acc<0>(sacc), pack_acc<1>(sacc)};
        pipelined<2 * DT, 2>([&](int n) { return cols_at<D>(kc, t2 * 32 + n / DT * 16, n % DT); },
                            [&](int n, const bf16x8& x) {
                              const int dt = n % DT;
                              dqacc[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x, dsf[n / DT], dqacc[dt], 0, 0, 0);
                            });
      }
    }
    if (m.docs && it + 1 < n_it) lds.key_docs[wave][lane] = next_doc;
    cur = next;
    next = after;
    wait_loads_and_barrier();
  }
  float* xch = (float*)&lds.tile[0][0][0] + rg * (DT * 16) * 64;
  if (par == 1) {
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
      for (int r = 0; r < 16; ++r) xch[(dt * 16 + r) * 64 + lane] = dqacc[dt][r];
  }
  if (BIAS == 2 && table_grad) {   // (in the wavefront's own place)
    sums.finish(a, lane);
    lds.sums[wave][lane] = (float)sums.own[0];
    lds.sums[wave][64 + lane] = (float)sums.own[1];
  }
  __syncthreads();
  if (BIAS == 2 && table_grad && tid < a.buckets) {
    float sum = 0.f;
#pragma unroll
    for (int w = 0; w < 2 * NRG; ++w) sum += lds.sums[w][tid];
    a.table_parts[(((long long)dev * a.nb * f.nh + mat) * a.ntiles + tile) * a.buckets + tid] = sum;
  }
  if (par == 0 && query < s) {
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

// 32 x 32 scores S (rows: queries q0 .., columns: keys) and dP = dO V^T in accumulators -> P and dS (the gradient of Q K^T) in their place.
// l, d, docs: of the 32 queries.  (dP - rowsum) (1 - tanh^2) comes before the scores, so that the tanh needs no place of its own.
// first: query from which on the key is seen.
template <int CAP, int BIAS>
__device__ __forceinline__ void biased_dkv_scores(f32x16& sacc, f32x16& pacc, const float* l, const float* d, const int* docs, int q0, int k0, int key,
                                                  int first, int kdoc, bool masked, const BiasedArgs& a, const Bias& bias, int g) {
  if (CAP) tanh16<CAP>(sacc, a);
#pragma unroll
  for (int c = 0; c < 4; ++c) {
    const float4 d4 = *(const float4*)(d + 8 * c + 4 * g);
    const float dv[4] = {d4.x, d4.y, d4.z, d4.w};
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int r = 4 * c + e;
      pacc[r] -= dv[e];
      if (CAP) pacc[r] *= fmaf(-sacc[r], sacc[r], 1.0f);
    }
  }
  const int lo = q0 - k0 - 31, dist0 = q0 + 4 * g - key;
  float w = 1.0f, c0 = 0.f;
  if (masked || !plain_tile<BIAS>(bias, lo, lo + 62)) {
    any16<CAP, BIAS, 1>(sacc, a, bias, dist0, q0 + 4 * g, first, docs + 4 * g, kdoc);
  } else {
    plain_weights<CAP, BIAS>(a, bias, lo, w, c0);
    plain16<CAP, BIAS, 1>(sacc, a, bias, dist0, lo);
  }
#pragma unroll
  for (int c = 0; c < 4; ++c) {
    const float4 l4 = *(const float4*)(l + 8 * c + 4 * g);
    const float lv[4] = {l4.x, l4.y, l4.z, l4.w};
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int r = 4 * c + e;
      const float p = weight_of(fmaf(sacc[r], w, BIAS == 2 ? c0 - lv[e] : -lv[e]));   // (of a row without pairs, and past the end: 0)
      sacc[r] = p;
      pacc[r] *= p;
    }
  }
}

template <int D, int NRG, int CAP, int BIAS>
__device__ __forceinline__ void biased_dkv_body(const BiasedArgs& a, DkvLds<D, NRG, BIAS>& lds, int tile, int mat, int dev) {
  constexpr int KS = D / 16, DT = D / 32, BKW = NRG * 32;
  const FusedArgs& f = a.f;
  const int tid = threadIdx.x, lane = tid & 63, g = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int rg = wave % NRG, par = wave / NRG;
  const int s = f.s;
  Matrix m = matrix_of<D>(a, mat, dev);
  if (no_documents<D, NRG>()) m.docs = nullptr;
  const bf16_t* Qp = f.qkv + m.qkv;
  const bf16_t* Kp = Qp + D;
  const bf16_t* Vp = Qp + 2 * D;
  const bf16_t* Gp = f.d_attn + m.attn;
  const float* Lp = f.lse + m.vec;
  const float* Dp = f.delta + m.vec;
  const int kt0 = tile * BKW, k0 = kt0 + rg * 32;
  const int key = k0 + (lane & 31);
  const int krow = min(key, s - 1);
  const int kdoc = m.docs ? m.docs[krow] : 0;
  const int first = a.causal && key >= m.prefix ? key : 0;   // query from which on the key is seen
  bf16x8 kf[KS], vf[KS];
#pragma unroll
  for (int ks = 0; ks < KS; ++ks) {
    kf[ks] = *(const bf16x8*)(Kp + (long long)krow * f.ld + ks * 16 + g * 8);
    vf[ks] = *(const bf16x8*)(Vp + (long long)krow * f.ld + ks * 16 + g * 8);
  }
  // the first block with a query that sees the workgroup's first key
  int qb_lo = a.causal && kt0 >= m.prefix ? kt0 / BLK : 0, qb_hi = a.nblk;
  if (m.docs) live_blocks(m.blocks, kt0 / BLK, (min(kt0 + BKW, s) - 1) / BLK, qb_lo, qb_hi);
  const int it_lo = qb_lo / 2, n_it = (qb_hi + 1) / 2;
  const i32x4_t none = {0x7fffffff, -1, 0, 0};
  const i32x4_t own = m.docs && k0 < s ? m.blocks[k0 / BLK] : none;

  f32x16 dkacc[DT], dvacc[DT];
#pragma unroll
  for (int dt = 0; dt < DT; ++dt) {
    dkacc[dt] = zero16();
    dvacc[dt] = zero16();
  }
  const unsigned in_rows = lds_address(lds.tile) + lane_rows<D>(lane), in_cols = lds_address(lds.tile) + lane_cols<D>(lane);
  RowLoader<D, 2 * NRG, PAIR> ldq, ldg;
  ldq.init(f.ld, wave, lane);
  ldg.init(f.ldo, wave, lane);
  struct Pair { i32x4_t even, odd; };
  auto pair_of = [&](int it) {
    Pair p = {none, none};
    if (m.docs) {
      if (2 * it < a.nblk) p.even = m.blocks[2 * it];
      if (2 * it + 1 < a.nblk) p.odd = m.blocks[2 * it + 1];
    }
    return p;
  };
  // the queries' numbers go through registers and reach LDS at the end of an iteration: stored at its top, they would wait for their
  // loads and for the tiles requested before them
  float next_l = 0.f, next_d = 0.f;
  int next_doc = 0;
  auto load_rows = [&](int it) {
    if (tid < PAIR) {
      const int at = min(it * PAIR + tid, s - 1);
      if (m.docs) next_doc = m.docs[at];
      next_l = Lp[at];
      next_d = Dp[at];
    }
  };
  auto store_rows = [&](int it, int st) {   // (past the end as padding)
    if (tid < PAIR) {
      lds.l[st][tid] = next_doc < 0 || it * PAIR + tid >= s ? INFINITY : lse2_of(next_l);
      lds.d[st][tid] = next_d;
      lds.docs[st][tid] = next_doc;
    }
  };
  auto issue = [&](int it, int st, const Pair& p) {
    const int* docs = p.even.z | p.odd.z ? m.docs : nullptr;
    ldq.issue(Qp, it * PAIR, s, lds.tile[st][0], docs);
    ldg.issue(Gp, it * PAIR, s, lds.tile[st][1], docs);
  };
  Pair cur = pair_of(it_lo), next = pair_of(it_lo + 1);
  if (it_lo < n_it) {
    load_rows(it_lo);
    issue(it_lo, 0, cur);
  }
  const Bias bias = make_bias<BIAS>(a, m.ghead, lds.bias);
#pragma unroll
  for (int ks = 0; ks < KS; ++ks) {
    kf[ks] = zero_if(kdoc < 0, kf[ks]);
    vf[ks] = zero_if(kdoc < 0, vf[ks]);
  }
  store_rows(it_lo, 0);
  wait_loads_and_barrier();
  for (int it = it_lo; it < n_it; ++it) {
    const int st = (it - it_lo) & 1;
    Pair after = next;
    if (it + 1 < n_it) {
      load_rows(it + 1);
      if (m.docs) after = pair_of(it + 2);
      issue(it + 1, st ^ 1, next);
    }
    const int qb = 2 * it + par, qbase = qb * BLK;
    const i32x4_t blk = par ? cur.odd : cur.even;
    const bool shared = !m.docs || share_documents(blk, own);
    if (k0 < s && qb >= qb_lo && qb < qb_hi && (!a.causal || qbase + BLK - 1 >= k0 || k0 < m.prefix) && shared) {
      const unsigned stage = (unsigned)((st * 2 * PAIR + par * BLK) * D * 2);
      const unsigned qt = in_rows + stage, qc = in_cols + stage;
      const bool masked = (a.causal && qbase < k0 + 31 && k0 + 31 >= m.prefix) || (m.docs && !one_document(blk, own));
      // 32 queries at a time: with the scores of all 64 live, fragments on their way have no registers
#pragma unroll
      for (int t2 = 0; t2 < 2; ++t2) {
        f32x16 sacc = zero16(), pacc = zero16();
        pipelined<2 * KS, 2>([&](int n) { return rows_at<D>(qt, (n & 1 ? PAIR : 0) + t2 * 32, n / 2); },
                            [&](int n, const bf16x8& x) {
                              f32x16& acc = n & 1 ? pacc : sacc;
                              acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x, n & 1 ? vf[n / 2] : kf[n / 2], acc, 0, 0, 0);
                            });
        const int at = par * BLK + t2 * 32;
        biased_dkv_scores<CAP, BIAS>(sacc, pacc, lds.l[st] + at, lds.d[st] + at, lds.docs[st] + at, qbase + t2 * 32, k0, key, first, kdoc,
                                     masked, a, bias, g);
        const bf16x8 pf[2] = {pack_acc<0>(sacc), pack_acc<1>(sacc)}, dsf[2] = {pack_acc<0>(pacc), pack_acc<1>(pacc)};
        pipelined<4 * DT, 2>([&](int n) { return cols_at<D>(qc, (n & 1 ? 0 : PAIR) + t2 * 32 + n / (2 * DT) * 16, n / 2 % DT); },
                            [&](int n, const bf16x8& x) {
                              const int dt = n / 2 % DT, u = n / (2 * DT);
                              f32x16& acc = n & 1 ? dkacc[dt] : dvacc[dt];
                              acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x, n & 1 ? dsf[u] : pf[u], acc, 0, 0, 0);
                            });
      }
    }
    if (it + 1 < n_it) store_rows(it + 1, st ^ 1);
    cur = next;
    next = after;
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
  if (par == 0 && key < s) {
    bf16_t* dKp = f.d_qkv + m.qkv + (long long)key * f.ld + D;
    bf16_t* dVp = dKp + D;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        float k4[4], v4[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          k4[e] = (dkacc[dt][4 * c + e] + xch[(dt * 16 + 4 * c + e) * 64 + lane]) * f.scale;
          v4[e] = dvacc[dt][4 * c + e] + xch[((DT + dt) * 16 + 4 * c + e) * 64 + lane];
        }
        u32x2 wk = {pack2_bf16(k4[0], k4[1]), pack2_bf16(k4[2], k4[3])};
        u32x2 wv = {pack2_bf16(v4[0], v4[1]), pack2_bf16(v4[2], v4[3])};
        *(u32x2*)(dKp + dt * 32 + 8 * c + 4 * g) = wk;
        *(u32x2*)(dVp + dt * 32 + 8 * c + 4 * g) = wv;
      }
  }
}

// Head width 128, 128 keys per workgroup, eight wavefronts: as without changes, the own V rows and half of the K fragments stay in
// LDS, blocks come one at a time, a wavefront takes one 32-query half (par) of every block.
template <int BIAS>
struct WideDkvLds {
  bf16_t block[2][2][BLK * 128];   // [stage][Q, dO]
  bf16_t v[128 * 128], k[128 * 128];
  BiasLds<BIAS> bias;
  alignas(16) float l[2][BLK];
  alignas(16) float d[2][BLK];
  alignas(16) int docs[2][BLK];
};
template <int CAP, int BIAS>
__device__ __forceinline__ void biased_dkv_wide_body(const BiasedArgs& a, WideDkvLds<BIAS>& lds, int tile, int mat, int dev) {
  constexpr int D = 128, KS = D / 16, DT = D / 32, BKW = 128, KREG = KS / 2;   // KREG: K fragments kept in registers
  const FusedArgs& f = a.f;
  const int tid = threadIdx.x, lane = tid & 63, g = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int rg = wave & 3, par = wave >> 2;
  const int s = f.s;
  const Matrix m = matrix_of<D>(a, mat, dev);
  const bf16_t* Qp = f.qkv + m.qkv;
  const bf16_t* Kp = Qp + D;
  const bf16_t* Gp = f.d_attn + m.attn;
  const float* Lp = f.lse + m.vec;
  const float* Dp = f.delta + m.vec;
  const int kt0 = tile * BKW, k0 = kt0 + rg * 32;
  const int key = k0 + (lane & 31);
  const int krow = min(key, s - 1);
  const int kdoc = m.docs ? m.docs[krow] : 0;
  const int first = a.causal && key >= m.prefix ? key : 0;   // query from which on the key is seen
  bf16x8 kf[KREG];
#pragma unroll
  for (int ks = 0; ks < KREG; ++ks) kf[ks] = *(const bf16x8*)(Kp + (long long)krow * f.ld + ks * 16 + g * 8);
  const int last_blk = (min(kt0 + BKW, s) - 1) / BLK;
  {
    const int* docs = m.docs && m.blocks[kt0 / BLK].z | m.blocks[last_blk].z ? m.docs : nullptr;
    RowLoader<D, 8, BKW> own;
    own.init(f.ld, wave, lane);
    own.issue(Qp + 2 * D, kt0, s, lds.v, docs);
    own.issue(Kp, kt0, s, lds.k, docs);
  }
  int qb_lo = a.causal && kt0 >= m.prefix ? kt0 / BLK : 0, qb_hi = a.nblk;
  if (m.docs) live_blocks(m.blocks, kt0 / BLK, last_blk, qb_lo, qb_hi);
  const i32x4_t none = {0x7fffffff, -1, 0, 0};
  const i32x4_t own_docs = m.docs && k0 < s ? m.blocks[k0 / BLK] : none;

  f32x16 dkacc[DT], dvacc[DT];
#pragma unroll
  for (int dt = 0; dt < DT; ++dt) {
    dkacc[dt] = zero16();
    dvacc[dt] = zero16();
  }
  // (a wavefront's 32 rows of a block, and its own 32 rows of V and K)
  const unsigned in_rows = lds_address(lds.block) + lane_rows<D>(lane) + par * 32 * D * 2, in_cols = lds_address(lds.block) + lane_cols<D>(lane) + par * 32 * D * 2;
  const unsigned own_rows = lds_address(lds.v) + lane_rows<D>(lane) + rg * 32 * D * 2;
  RowLoader<D, 8, BLK> ldq, ldg;
  ldq.init(f.ld, wave, lane);
  ldg.init(f.ldo, wave, lane);
  auto block_of = [&](int qb) { return m.docs && qb < a.nblk ? (i32x4_t)m.blocks[qb] : none; };
  float next_l = 0.f, next_d = 0.f;
  int next_doc = 0;
  auto load_block = [&](int qb, int st, i32x4_t blk) {
    if (tid < BLK) {
      const int at = min(qb * BLK + tid, s - 1);
      if (m.docs) next_doc = m.docs[at];
      next_l = Lp[at];
      next_d = Dp[at];
    }
    const int* docs = blk.z ? m.docs : nullptr;
    ldq.issue(Qp, qb * BLK, s, lds.block[st][0], docs);
    ldg.issue(Gp, qb * BLK, s, lds.block[st][1], docs);
  };
  auto store_rows = [&](int qb, int st) {   // (past the end as padding)
    if (tid < BLK) {
      lds.l[st][tid] = next_doc < 0 || qb * BLK + tid >= s ? INFINITY : lse2_of(next_l);
      lds.d[st][tid] = next_d;
      lds.docs[st][tid] = next_doc;
    }
  };
  i32x4_t cur = block_of(qb_lo), next = block_of(qb_lo + 1);
  if (qb_lo < qb_hi) {
    load_block(qb_lo, 0, cur);
  }
  const Bias bias = make_bias<BIAS>(a, m.ghead, lds.bias);
#pragma unroll
  for (int ks = 0; ks < KREG; ++ks) kf[ks] = zero_if(kdoc < 0, kf[ks]);
  store_rows(qb_lo, 0);
  wait_loads_and_barrier();
  for (int qb = qb_lo; qb < qb_hi; ++qb) {
    const int st = (qb - qb_lo) & 1;
    i32x4_t after = next;
    if (qb + 1 < qb_hi) {
      after = block_of(qb + 2);
      load_block(qb + 1, st ^ 1, next);
    }
    const int q0 = qb * BLK + par * 32;   // this wavefront's queries
    if (k0 < s && q0 < s && (!a.causal || q0 + 31 >= k0 || k0 < m.prefix) && (!m.docs || share_documents(cur, own_docs))) {
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
      biased_dkv_scores<CAP, BIAS>(sacc, pacc, lds.l[st] + par * 32, lds.d[st] + par * 32, lds.docs[st] + par * 32, q0, k0, key, first, kdoc,
                                   (a.causal && q0 < k0 + 31 && k0 + 31 >= m.prefix) || (m.docs && !one_document(cur, own_docs)), a, bias, g);
      const bf16x8 pf[2] = {pack_acc<0>(sacc), pack_acc<1>(sacc)}, dsf[2] = {pack_acc<0>(pacc), pack_acc<1>(pacc)};
      pipelined<4 * DT, 2>([&](int n) { return cols_at<D>(qc, (n & 1 ? 0 : BLK) + n / (2 * DT) * 16, n / 2 % DT); },
                          [&](int n, const bf16x8& x) {
                            const int dt = n / 2 % DT, u = n / (2 * DT);
                            f32x16& acc = n & 1 ? dkacc[dt] : dvacc[dt];
                            acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x, n & 1 ? dsf[u] : pf[u], acc, 0, 0, 0);
                          });
    }
    if (qb + 1 < qb_hi) store_rows(qb + 1, st ^ 1);
    cur = next;
    next = after;
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
    if (par == 0 && key < s) {
      const float w = which == 0 ? 1.0f : f.scale;
#pragma unroll
      for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          float o[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) o[e] = (acc[dt][4 * c + e] + xch[(dt * 16 + 4 * c + e) * 64 + lane]) * w;
          u32x2 x = {pack2_bf16(o[0], o[1]), pack2_bf16(o[2], o[3])};
          *(u32x2*)(dKp + (which == 0 ? D : 0) + dt * 32 + 8 * c + 4 * g) = x;
        }
    }
  }
}

template <size_t A, size_t B>
constexpr size_t larger() { return A > B ? A : B; }

// Both kinds in one grid ordered by loop length, longest first, the kinds alternating: x = (rank, matrix, kind), y = device.
template <int D, int CAP, int BIAS>
__global__ __launch_bounds__(256, D == 64 ? 2 : 1) void attn_biased_bwd_kernel(BiasedArgs a, int ntiles, int nmat) {
  constexpr size_t DQ = sizeof(DqLds<D, 2, BIAS>), DKV = sizeof(DkvLds<D, 2, BIAS>);
  __shared__ __attribute__((aligned(1024))) char lds[DQ > DKV ? DQ : DKV];
  const unsigned per_rank = 2u * (unsigned)nmat;
  const unsigned rank = blockIdx.x / per_rank, rem = blockIdx.x % per_rank;
  const int mat = (int)(rem >> 1), dev = (int)blockIdx.y;
  if (rem & 1) biased_dq_body<D, 2, CAP, BIAS>(a, *(DqLds<D, 2, BIAS>*)lds, ntiles - 1 - (int)rank, mat, dev);
  else biased_dkv_body<D, 2, CAP, BIAS>(a, *(DkvLds<D, 2, BIAS>*)lds, (int)rank, mat, dev);
}

// The same in workgroups of eight wavefronts and 128 rows: x = (matrix, kind), y = rank, z = device.
template <int D, int CAP, int BIAS>
__global__ __launch_bounds__(512, 2) void attn_biased_bwd_wide_kernel(BiasedArgs a) {
  const int rank = blockIdx.y, mat = blockIdx.x >> 1, kind = blockIdx.x & 1, ntiles = gridDim.y, dev = blockIdx.z;
  if constexpr (D == 128) {
    __shared__ __attribute__((aligned(1024))) char lds[larger<sizeof(WideDkvLds<BIAS>), sizeof(DqLds<D, 4, BIAS>)>()];
    if (kind) biased_dq_body<D, 4, CAP, BIAS>(a, *(DqLds<D, 4, BIAS>*)lds, ntiles - 1 - rank, mat, dev);
    else biased_dkv_wide_body<CAP, BIAS>(a, *(WideDkvLds<BIAS>*)lds, rank, mat, dev);
  } else {
    __shared__ __attribute__((aligned(1024))) char lds[larger<sizeof(DkvLds<D, 4, BIAS>), sizeof(DqLds<D, 4, BIAS>)>()];
    if (kind) biased_dq_body<D, 4, CAP, BIAS>(a, *(DqLds<D, 4, BIAS>*)lds, ntiles - 1 - rank, mat, dev);
    else biased_dkv_body<D, 4, CAP, BIAS>(a, *(DkvLds<D, 4, BIAS>*)lds, rank, mat, dev);
  }
}

// d_table[device][head][bucket]: the parts of the head's matrices and tiles, eight threads a bucket in that order, then theirs, in 64
// bits: thousands of parts of either sign.
__global__ __launch_bounds__(1024) void attn_biased_table_kernel(BiasedArgs a, float* d_table) {
  __shared__ double sums[1024];
  const int head = blockIdx.x, dev = blockIdx.y, b = threadIdx.x & 127, slice = threadIdx.x >> 7;
  const int n = a.nb * a.ntiles;
  double sum = 0.0;
  if (b < a.buckets)
    for (int p = slice; p < n; p += 8) {
      const int seq = p / a.ntiles, tile = p % a.ntiles;
      sum += a.table_parts[((((long long)dev * a.nb + seq) * a.f.nh + head) * a.ntiles + tile) * a.buckets + b];
    }
  sums[threadIdx.x] = sum;
  __syncthreads();
  if (slice == 0 && b < a.buckets) {
#pragma unroll
    for (int k = 1; k < 8; ++k) sum += sums[k * 128 + b];
    d_table[((long long)dev * a.f.nh + head) * a.buckets + b] = (float)sum;
  }
}

template <int D, int CAP, int BIAS>
void bwd_launch(const BiasedArgs& a, const AttnBiasedDesc& b, hipStream_t st) {
  const AttnFusedDesc& d = b.base;
  const int nmat = d.nb * d.nh;
  if (attn_biased_bwd_wide(b)) attn_biased_bwd_wide_kernel<D, CAP, BIAS><<<dim3(2 * nmat, a.ntiles, d.ndev), 512, 0, st>>>(a);
  else attn_biased_bwd_kernel<D, CAP, BIAS><<<dim3((unsigned)(2ll * a.ntiles * nmat), d.ndev), 256, 0, st>>>(a, a.ntiles, nmat);
}

}  // namespace

// 64-row workgroups as long as all of them run at once (one a compute unit of width 128, two of 64), and at width 64 with documents.
// 64 rows / 128 rows, us: width 128, causal, 16 matrices of 512 (256 workgroups of 64 rows) 25.3 / 25.3, 10 of 1000 without a mask (320)
// 66.5 / 37.1, 16 of 4096 457 / 256; width 64, causal, 16 of 1024 (512) 23.4 / 25.2, 16 of 2048 (1024) 60.7 / 52.0, 16 of 4096 164 / 149, 64
// of 1024 64.9 / 62.7, 64 of 2048 without a mask 312 / 287.  With a cap of 50, with the table's gradient: 16 of 2048 74.9 / 65.8, 79.8 /
// 68.5; 128 of 512 57.4 / 58.0, 72.7 / 68.6; 64 of 4096 830 / 767, 752 / 698; without a mask 64 of 2048 401 / 377, 382 / 360, 24 of 1400 97.1 /
// 103.7, 102.2 / 105.2: ahead in 86 of 100 launches of 8 to 128 matrices, by up to 15 %, and up to 7 % behind where the last round is
// short.  With documents of 700 the other way: causal, 16 of 2048 38.2 / 41.7, 16 of 4096 99 / 108, 64 of 2048 135 / 151, 64 of 4096 392 / 407,
// without a mask 673 / 677.
// The two forms add dK and dV (width 128) and the table's gradient up in different orders, so the choice follows one device's matrices,
// whatever the launch covers.
bool attn_biased_bwd_wide(const AttnBiasedDesc& b) {
  const AttnFusedDesc& d = b.base;
  const long long groups = 2ll * ((d.s + BLK - 1) / BLK) * d.nb * d.nh;
  if (d.d == 64) return groups > 2 * num_cus() && !b.documents;
  return groups > num_cus();
}

int launch_attn_biased_bwd_kernels(const BiasedArgs& given, const AttnBiasedDesc& b, hipStream_t st) {
  const AttnFusedDesc& d = b.base;
  BiasedArgs a = given;
  a.ntiles = attn_biased_bwd_wide(b) ? (d.s + 127) / 128 : (d.s + BLK - 1) / BLK;
  a.table_parts = b.d_table ? b.table_parts : nullptr;
  with_kind(b, [&](auto width, auto cap, auto bias) {
    bwd_launch<decltype(width)::value, decltype(cap)::value, decltype(bias)::value>(a, b, st);
  });
  if (a.table_parts) attn_biased_table_kernel<<<dim3(d.nh, d.ndev), 1024, 0, st>>>(a, b.d_table);
  return hip_launch_status();
}

}  // namespace optimus
