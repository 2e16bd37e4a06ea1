// Backward of the attention with changed scores (attention_biased_kernel.hpp): dQ and the table's gradient by workgroups that own
// queries, dK and dV by workgroups that own keys, both kinds in one grid as in the attention without changes.
#include "attention_biased_kernel.hpp"

namespace optimus {
namespace {

// The sums of dS over the buckets, of one wavefront.  A lane owns a bucket (and the one 64 further).  A 32 x 32 tile that lies in the
// last bucket as a whole is summed lane by lane; another one is summed along its 63 diagonals first: slot r of 32 lanes lies on 32
// diagonals, so the adds into LDS of one instruction go to different places (the halves have an array each) and come one instruction
// after the other: the same bits in every run.
struct BucketSums {
  float own[2], far_pos, far_neg;
  int lo[2], hi[2];      // distances of the lane's buckets
  int far, back;
  float* diag;           // LDS, [2][64] of the wavefront
  int* first;
  __device__ __forceinline__ void init(const BiasedArgs& a, float* diag_, const int* first_, int lane) {
    diag = diag_;
    own[0] = own[1] = far_pos = far_neg = 0.f;
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
    diag[lane] = diag[64 + lane] = 0.f;
  }
  // ds: lane's slots at distance dist0 - slot(r); the tile's distances are base .. base + 62, the lane's slot 0 at `at` = dist0 - base
  __device__ __forceinline__ void add(const f32x16& ds, int base, int at, int g, int lane, bool wide) {
    if (base >= far || base + 62 <= -back) {
      float t[8];
#pragma unroll
      for (int r = 0; r < 8; ++r) t[r] = ds[r] + ds[r + 8];
      const float sum = ((t[0] + t[1]) + (t[2] + t[3])) + ((t[4] + t[5]) + (t[6] + t[7]));
      if (base >= far) far_pos += sum;
      else far_neg += sum;
      return;
    }
    float* mine = diag + 64 * g + at;
#pragma unroll
    for (int r = 0; r < 16; ++r) __hip_atomic_fetch_add(mine - slot(r), ds[r], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WAVEFRONT);
    __builtin_amdgcn_wave_barrier();
    const float both = diag[lane] + diag[64 + lane];
    __builtin_amdgcn_wave_barrier();
    diag[lane] = both;
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      if (k == 1 && !wide) break;
      const int from = max(lo[k] - base, 0), to = min(hi[k] - base, 62);
      for (int d = from; d <= to; ++d) own[k] += diag[d];
    }
    __builtin_amdgcn_wave_barrier();
    diag[lane] = diag[64 + lane] = 0.f;
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

template <int D, int NRG, int BIAS>
struct DqLds {
  bf16_t tile[2][2][PAIR * D];   // [stage][K, V]
  BiasLds<BIAS> bias;
  int key_docs[2 * NRG][BLK];
  float diag[BIAS == 2 ? 2 * NRG : 1][128];
  int live[2];
};
template <int D, int NRG, int BIAS>
struct DkvLds {
  bf16_t tile[2][2][PAIR * D];   // [stage][Q, dO]
  BiasLds<BIAS> bias;
  float l[2][PAIR], d[2][PAIR];
  int docs[2][PAIR];
  int live[2];
};

// log-sum-exp of a row -> what is subtracted from its scores.  Of a row without pairs +infinity, which makes every P of it zero.
__device__ __forceinline__ float lse2_of(float lse) { return lse == -INFINITY ? INFINITY : lse * LOG2E; }

template <int D, int NRG, bool CAP, int BIAS>
__device__ __forceinline__ void biased_dq_body(const BiasedArgs& a, DqLds<D, NRG, BIAS>& lds, int tile, int mat, int dev) {
  constexpr int KS = D / 16, DT = D / 32, BQ = NRG * 32;
  const FusedArgs& f = a.f;
  const int tid = threadIdx.x, lane = tid & 63, g = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int rg = wave % NRG, par = wave / NRG;
  const int s = f.s;
  const Matrix m = matrix_of<D>(a, mat, dev);
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
    qf[ks] = zero_if(qdoc < 0, *(const bf16x8*)(Qp + (long long)qrow * f.ld + ks * 16 + g * 8));
    dof[ks] = zero_if(qdoc < 0, *(const bf16x8*)(f.d_attn + m.attn + (long long)qrow * f.ldo + ks * 16 + g * 8));
  }
  const float delta = f.delta[m.vec + qrow];
  const float lse2 = query < s && qdoc >= 0 ? lse2_of(f.lse[m.vec + qrow]) : INFINITY;
  const Bias<BIAS> bias = make_bias<BIAS>(a, m.ghead, lds.bias);
  BucketSums sums;
  const bool table_grad = BIAS == 2 && a.table_parts;
  if (BIAS == 2) sums.init(a, lds.diag[wave], lds.bias.first, lane);

  const int wg_hi = min(tile * BQ + BQ, s) - 1;
  int kb_lo = 0, kb_hi = a.causal ? max(wg_hi, m.prefix - 1) / BLK + 1 : a.nblk;
  if (m.docs) live_blocks(m.blocks, tile * BQ / BLK, wg_hi / BLK, kb_lo, kb_hi, lds.live);
  const int it_lo = kb_lo / 2, n_it = (kb_hi + 1) / 2;
  const int wave_last = q0 >= s ? -1 : a.causal ? max(min(q0 + 31, s - 1), m.prefix - 1) : s - 1;
  const int limit = a.causal ? max(qrow, m.prefix - 1) : s - 1;
  const i32x4_t none = {0x7fffffff, -1, 0, 0};
  const i32x4_t own = m.docs && q0 < s ? m.blocks[q0 / BLK] : none;

  f32x16 dqacc[DT];
#pragma unroll
  for (int dt = 0; dt < DT; ++dt) dqacc[dt] = zero16();

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
  if (it_lo < n_it) {
    if (m.docs) lds.key_docs[wave][lane] = m.docs[min((2 * it_lo + par) * BLK + lane, s - 1)];
    issue(it_lo, 0, cur);
  }
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
      const bf16_t* tK = lds.tile[st][0] + par * BLK * D;
      const bf16_t* tV = lds.tile[st][1] + par * BLK * D;
      const bool need_limit = a.causal ? kbase + BLK - 1 > max(q0, m.prefix - 1) : kbase + BLK > s;
      const bool need_docs = m.docs && !one_document(blk, own);
      bf16x8 dsf[2][2];
#pragma unroll
      for (int t2 = 0; t2 < 2; ++t2) {
        f32x16 sacc = zero16(), pacc = zero16();
        pipelined<2 * KS, 2>([&](int n) { return frag_rows<D>(n & 1 ? tV : tK, t2 * 32, n / 2, lane); },
                            [&](int n, const bf16x8& x) {
                              f32x16& acc = n & 1 ? pacc : sacc;
                              acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x, n & 1 ? dof[n / 2] : qf[n / 2], acc, 0, 0, 0);
                            });
        const int k0 = kbase + t2 * 32, dist0 = query - k0 - 4 * g;
        f32x16 th;
        if (CAP) {
          tanh16(sacc, a);
          th = sacc;
        }
        scores16<CAP, BIAS, -1>(sacc, a, bias, tile_bias<BIAS>(bias, dist0, q0 - k0 - 31, q0 - k0 + 31));
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const float p = __builtin_amdgcn_exp2f(sacc[r] - lse2);
          sacc[r] = p * (pacc[r] - delta);  // dS^T
        }
        if (need_limit) {
#pragma unroll
          for (int r = 0; r < 16; ++r)
            if (k0 + slot(r) + 4 * g > limit) sacc[r] = 0.f;
        }
        if (need_docs) {
#pragma unroll
          for (int c = 0; c < 4; ++c) {
            const int4 kd = *(const int4*)&lds.key_docs[wave][t2 * 32 + 8 * c + 4 * g];
            const int k4[4] = {kd.x, kd.y, kd.z, kd.w};
#pragma unroll
            for (int e = 0; e < 4; ++e)
              if (k4[e] != qdoc || qdoc < 0) sacc[4 * c + e] = 0.f;
          }
        }
        if (BIAS == 2 && table_grad) sums.add(sacc, q0 - k0 - 31, (lane & 31) + 31 - 4 * g, g, lane, a.buckets > 64);
        if (CAP) {
#pragma unroll
          for (int r = 0; r < 16; ++r) sacc[r] *= fmaf(-th[r], th[r], 1.0f);
        }
        dsf[t2][0] = pack_acc<0>(sacc);
        dsf[t2][1] = pack_acc<1>(sacc);
      }
      pipelined<4 * DT, 2>([&](int n) { return frag_cols_acc_order<D>(tK, n / DT * 16, n % DT * 32, lane); },
                          [&](int n, const bf16x8& x) {
                            const int dt = n % DT;
                            dqacc[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x, dsf[n / (2 * DT)][n / DT & 1], dqacc[dt], 0, 0, 0);
                          });
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
  if (BIAS == 2 && table_grad) {   // (the wavefront's buckets over its diagonals)
    sums.finish(a, lane);
    lds.diag[wave][lane] = sums.own[0];
    lds.diag[wave][64 + lane] = sums.own[1];
  }
  __syncthreads();
  if (BIAS == 2 && table_grad && tid < a.buckets) {
    float sum = 0.f;
#pragma unroll
    for (int w = 0; w < 2 * NRG; ++w) sum += lds.diag[w][tid];
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
// l, d, docs: of the 32 queries.
template <bool CAP, int BIAS>
__device__ __forceinline__ void biased_dkv_scores(f32x16& sacc, f32x16& pacc, const float* l, const float* d, const int* docs, int q0, int k0, int key,
                                                  int kdoc, bool need_limit, bool need_docs, int prefix, const BiasedArgs& a, const Bias<BIAS>& bias,
                                                  int g) {
  f32x16 th;
  if (CAP) {
    tanh16(sacc, a);
    th = sacc;
  }
  scores16<CAP, BIAS, 1>(sacc, a, bias, tile_bias<BIAS>(bias, q0 + 4 * g - key, q0 - k0 - 31, q0 - k0 + 31));
#pragma unroll
  for (int c = 0; c < 4; ++c) {
    const int qi = 8 * c + 4 * g;
    const float4 l4 = *(const float4*)(l + qi);
    const float4 d4 = *(const float4*)(d + qi);
    const float lv[4] = {l4.x, l4.y, l4.z, l4.w}, dv[4] = {d4.x, d4.y, d4.z, d4.w};
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int r = 4 * c + e;
      float p = __builtin_amdgcn_exp2f(sacc[r] - lv[e]);   // (of a row without pairs, and past the end: 0)
      if (need_limit && q0 + qi + e < key && key >= prefix) p = 0.f;
      sacc[r] = p;
    }
    if (need_docs) {
      const int4 o4 = *(const int4*)(docs + qi);
      const int ov[4] = {o4.x, o4.y, o4.z, o4.w};
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (ov[e] != kdoc || kdoc < 0) sacc[4 * c + e] = 0.f;
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int r = 4 * c + e;
      float ds = sacc[r] * (pacc[r] - dv[e]);
      if (CAP) ds *= fmaf(-th[r], th[r], 1.0f);
      pacc[r] = ds;
    }
  }
}

template <int D, int NRG, bool CAP, int BIAS>
__device__ __forceinline__ void biased_dkv_body(const BiasedArgs& a, DkvLds<D, NRG, BIAS>& lds, int tile, int mat, int dev) {
  constexpr int KS = D / 16, DT = D / 32, BKW = NRG * 32;
  const FusedArgs& f = a.f;
  const int tid = threadIdx.x, lane = tid & 63, g = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int rg = wave % NRG, par = wave / NRG;
  const int s = f.s;
  const Matrix m = matrix_of<D>(a, mat, dev);
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
  bf16x8 kf[KS], vf[KS];
#pragma unroll
  for (int ks = 0; ks < KS; ++ks) {
    kf[ks] = zero_if(kdoc < 0, *(const bf16x8*)(Kp + (long long)krow * f.ld + ks * 16 + g * 8));
    vf[ks] = zero_if(kdoc < 0, *(const bf16x8*)(Vp + (long long)krow * f.ld + ks * 16 + g * 8));
  }
  const Bias<BIAS> bias = make_bias<BIAS>(a, m.ghead, lds.bias);
  // the first block with a query that sees the workgroup's first key
  int qb_lo = a.causal && kt0 >= m.prefix ? kt0 / BLK : 0, qb_hi = a.nblk;
  if (m.docs) live_blocks(m.blocks, kt0 / BLK, (min(kt0 + BKW, s) - 1) / BLK, qb_lo, qb_hi, lds.live);
  const int it_lo = qb_lo / 2, n_it = (qb_hi + 1) / 2;
  const i32x4_t none = {0x7fffffff, -1, 0, 0};
  const i32x4_t own = m.docs && k0 < s ? m.blocks[k0 / BLK] : none;

  f32x16 dkacc[DT], dvacc[DT];
#pragma unroll
  for (int dt = 0; dt < DT; ++dt) {
    dkacc[dt] = zero16();
    dvacc[dt] = zero16();
  }
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
  int next_doc = -1;
  auto load_rows = [&](int it) {
    if (tid < PAIR) {
      const int row = it * PAIR + tid, at = min(row, s - 1);
      next_doc = m.docs ? m.docs[at] : 0;
      next_l = row < s ? Lp[at] : -INFINITY;
      next_d = Dp[at];
    }
  };
  auto store_rows = [&](int st) {
    if (tid < PAIR) {
      lds.l[st][tid] = next_doc < 0 ? INFINITY : lse2_of(next_l);
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
    store_rows(0);
    issue(it_lo, 0, cur);
  }
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
      const bf16_t* tQ = lds.tile[st][0] + par * BLK * D;
      const bf16_t* tG = lds.tile[st][1] + par * BLK * D;
      f32x16 sacc[2], pacc[2];
#pragma unroll
      for (int t2 = 0; t2 < 2; ++t2) {
        sacc[t2] = zero16();
        pacc[t2] = zero16();
      }
      pipelined<4 * KS, 2>([&](int n) { return frag_rows<D>(n & 1 ? tG : tQ, n / (2 * KS) * 32, n / 2 % KS, lane); },
                          [&](int n, const bf16x8& x) {
                            const int t2 = n / (2 * KS), ks = n / 2 % KS;
                            f32x16& acc = n & 1 ? pacc[t2] : sacc[t2];
                            acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x, n & 1 ? vf[ks] : kf[ks], acc, 0, 0, 0);
                          });
      const bool need_limit = a.causal && qbase < k0 + 31 && k0 + 31 >= m.prefix;
      const bool need_docs = m.docs && !one_document(blk, own);
      bf16x8 pf[2][2], dsf[2][2];
#pragma unroll
      for (int t2 = 0; t2 < 2; ++t2) {
        const int at = par * BLK + t2 * 32;
        biased_dkv_scores<CAP, BIAS>(sacc[t2], pacc[t2], lds.l[st] + at, lds.d[st] + at, lds.docs[st] + at, qbase + t2 * 32, k0, key, kdoc, need_limit,
                                     need_docs, m.prefix, a, bias, g);
        pf[t2][0] = pack_acc<0>(sacc[t2]);
        pf[t2][1] = pack_acc<1>(sacc[t2]);
        dsf[t2][0] = pack_acc<0>(pacc[t2]);
        dsf[t2][1] = pack_acc<1>(pacc[t2]);
      }
      pipelined<8 * DT, 2>([&](int n) { return frag_cols_acc_order<D>(n & 1 ? tQ : tG, n / (2 * DT) * 16, n / 2 % DT * 32, lane); },
                          [&](int n, const bf16x8& x) {
                            const int dt = n / 2 % DT, t2 = n / (4 * DT), u = n / (2 * DT) & 1;
                            f32x16& acc = n & 1 ? dkacc[dt] : dvacc[dt];
                            acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x, n & 1 ? dsf[t2][u] : pf[t2][u], acc, 0, 0, 0);
                          });
    }
    if (it + 1 < n_it) store_rows(st ^ 1);
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

// Both kinds in one grid ordered by loop length, longest first, the kinds alternating: x = (rank, matrix, kind), y = device.
template <int D, bool CAP, int BIAS>
__global__ __launch_bounds__(256, D == 64 ? 2 : 1) void attn_biased_bwd_kernel(BiasedArgs a, int ntiles, int nmat) {
  constexpr size_t DQ = sizeof(DqLds<D, 2, BIAS>), DKV = sizeof(DkvLds<D, 2, BIAS>);
  __shared__ __attribute__((aligned(1024))) char lds[DQ > DKV ? DQ : DKV];
  const unsigned per_rank = 2u * (unsigned)nmat;
  const unsigned rank = blockIdx.x / per_rank, rem = blockIdx.x % per_rank;
  const int mat = (int)(rem >> 1), dev = (int)blockIdx.y;
  if (rem & 1) biased_dq_body<D, 2, CAP, BIAS>(a, *(DqLds<D, 2, BIAS>*)lds, ntiles - 1 - (int)rank, mat, dev);
  else biased_dkv_body<D, 2, CAP, BIAS>(a, *(DkvLds<D, 2, BIAS>*)lds, (int)rank, mat, dev);
}

// d_table[device][head][bucket]: the parts of the head's matrices and tiles, added in that order by 1024 / 128 threads a bucket, then
// theirs.
__global__ __launch_bounds__(1024) void attn_biased_table_kernel(BiasedArgs a, float* d_table) {
  __shared__ float sums[1024];
  const int head = blockIdx.x, dev = blockIdx.y, b = threadIdx.x & 127, slice = threadIdx.x >> 7;
  const int n = a.nb * a.ntiles;
  float sum = 0.f;
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
    d_table[((long long)dev * a.f.nh + head) * a.buckets + b] = sum;
  }
}

template <int D, bool CAP, int BIAS>
void bwd_launch(const BiasedArgs& a, const AttnFusedDesc& d, hipStream_t st) {
  const int ntiles = (d.s + BLK - 1) / BLK, nmat = d.nb * d.nh;
  attn_biased_bwd_kernel<D, CAP, BIAS><<<dim3((unsigned)(2ll * ntiles * nmat), d.ndev), 256, 0, st>>>(a, ntiles, nmat);
}

}  // namespace

int launch_attn_biased_bwd_kernels(const BiasedArgs& given, const AttnBiasedDesc& b, hipStream_t st) {
  const AttnFusedDesc& d = b.base;
  BiasedArgs a = given;
  a.ntiles = (d.s + BLK - 1) / BLK;
  a.table_parts = b.d_table ? b.table_parts : nullptr;
  const int kind = (b.cap > 0 ? 3 : 0) + (b.table ? 2 : b.slopes ? 1 : 0);
  auto run = [&](auto width) {
    constexpr int D = decltype(width)::value;
    switch (kind) {
      case 0: bwd_launch<D, false, 0>(a, d, st); break;
      case 1: bwd_launch<D, false, 1>(a, d, st); break;
      case 2: bwd_launch<D, false, 2>(a, d, st); break;
      case 3: bwd_launch<D, true, 0>(a, d, st); break;
      case 4: bwd_launch<D, true, 1>(a, d, st); break;
      default: bwd_launch<D, true, 2>(a, d, st);
    }
  };
  if (d.d == 64) run(std::integral_constant<int, 64>());
  else run(std::integral_constant<int, 128>());
  if (a.table_parts) attn_biased_table_kernel<<<dim3(d.nh, d.ndev), 1024, 0, st>>>(a, b.d_table);
  return hip_launch_status();
}

}  // namespace optimus
