// Forward of the attention with changed scores (attention_biased_kernel.hpp), the kernel that both directions run first, the choice
// between the forms.
#include "attention_biased_kernel.hpp"

namespace optimus {
namespace {

// Forward.  NRG: row groups of 32 queries per workgroup, as in the attention without changes.  Two workgroups of 128 rows a compute unit
// of width 64, where 128 registers a lane are enough: with slopes a dozen would be spilled (16 matrices of 4096, causal, 76 us; one
// workgroup 63), with a cap beyond 64 eight.  (With a smaller one and a table eight are.)
template <int D, int NRG, int CAP, int BIAS>
__global__ __launch_bounds__(NRG * 128, D == 64 && NRG == 4 && BIAS != 1 && CAP != 2 ? 4 : NRG == 4 || D == 64 ? 2 : 1) void attn_biased_fwd_kernel(BiasedArgs a) {
  constexpr int KS = D / 16, DT = D / 32, BQ = NRG * 32, AHEAD = D == 64 ? 1 : 2;
  __shared__ __attribute__((aligned(1024))) bf16_t lds[2][2][PAIR * D];  // [stage][K, V][pair tile]
  __shared__ BiasLds<BIAS> bias_lds;
  __shared__ __attribute__((aligned(16))) int key_docs[2 * NRG][BLK];    // of the wavefront's block
  const FusedArgs& f = a.f;
  const int tid = threadIdx.x, lane = tid & 63, g = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int rg = wave % NRG, par = wave / NRG;
  const int tile = gridDim.y - 1 - blockIdx.y, s = f.s;   // the longest causal loops first
  const Matrix m = matrix_of<D>(a, blockIdx.x, blockIdx.z);
  const bf16_t* Qp = f.qkv + m.qkv;
  const bf16_t* Kp = Qp + D;
  const bf16_t* Vp = Qp + 2 * D;
  const int q0 = tile * BQ + rg * 32;
  const int query = q0 + (lane & 31);
  const int qrow = min(query, s - 1);
  const int qdoc = m.docs ? m.docs[qrow] : 0;
  bf16x8 qf[KS];
#pragma unroll
  for (int ks = 0; ks < KS; ++ks) qf[ks] = *(const bf16x8*)(Qp + (long long)qrow * f.ld + ks * 16 + g * 8);

  const int wg_hi = min(tile * BQ + BQ, s) - 1;   // last query row of the workgroup
  int kb_lo = 0, kb_hi = a.causal ? max(wg_hi, m.prefix - 1) / BLK + 1 : a.nblk;
  if (m.docs) live_blocks(m.blocks, tile * BQ / BLK, wg_hi / BLK, kb_lo, kb_hi);
  const int it_lo = kb_lo / 2, n_it = (kb_hi + 1) / 2;
  // last key that a row of the wavefront may see, and that this lane's may
  const int wave_last = q0 >= s ? -1 : a.causal ? max(min(q0 + 31, s - 1), m.prefix - 1) : s - 1;
  const int limit = a.causal ? max(qrow, m.prefix - 1) : s - 1;
  const i32x4_t none = {0x7fffffff, -1, 0, 0};
  const i32x4_t own = m.docs && q0 < s ? m.blocks[q0 / BLK] : none;

  f32x16 oacc[DT];
#pragma unroll
  for (int dt = 0; dt < DT; ++dt) oacc[dt] = zero16();
  float m_run = -INFINITY, l_run = 0.f;

  const unsigned in_rows = lds_address(lds) + lane_rows<D>(lane), in_cols = lds_address(lds) + lane_cols<D>(lane);
  RowLoader<D, 2 * NRG, PAIR> ldr;
  ldr.init(f.ld, wave, lane);
  // documents of a pair's blocks, known an iteration before they are used
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
    ldr.issue(Kp, it * PAIR, s, lds[st][0], docs);
    ldr.issue(Vp, it * PAIR, s, lds[st][1], docs);
  };
  Pair cur = pair_of(it_lo), next = pair_of(it_lo + 1);
  int first_doc = 0;
  if (it_lo < n_it) {
    if (m.docs) first_doc = m.docs[min((2 * it_lo + par) * BLK + lane, s - 1)];
    issue(it_lo, 0, cur);
  }
  // (behind the first tiles' request: it waits for loads of its own)
  const Bias bias = make_bias<BIAS>(a, m.ghead, bias_lds);
#pragma unroll
  for (int ks = 0; ks < KS; ++ks) qf[ks] = zero_if(qdoc < 0, qf[ks]);
  key_docs[wave][lane] = first_doc;
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
      const unsigned kt = in_rows + stage, vt = in_cols + stage;
      f32x16 sacc[2];
      sacc[0] = zero16();
      sacc[1] = zero16();
      pipelined<2 * KS, AHEAD>([&](int n) { return rows_at<D>(kt, n / KS * 32, n % KS); },
                               [&](int n, const bf16x8& x) {
                                 sacc[n / KS] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x, qf[n % KS], sacc[n / KS], 0, 0, 0);
                               });
      if (CAP) {
        tanh16<CAP>(sacc[0], a);
        tanh16<CAP>(sacc[1], a);
      }
      const int dist0 = query - kbase - 4 * g, lo = q0 - kbase - (BLK - 1), hi = q0 + 31 - kbase;
      float w = 1.0f, c = 0.f;
      // pairs to leave out exist only in the last blocks and where documents meet (wave-uniform tests)
      const bool masked = (a.causal ? kbase + BLK - 1 > max(q0, m.prefix - 1) : kbase + BLK > s) || (m.docs && !one_document(blk, own));
      const bool plain = !masked && plain_tile<BIAS>(bias, lo, hi);
      if (!plain) {
#pragma unroll
        for (int t2 = 0; t2 < 2; ++t2)
          any16<CAP, BIAS, -1>(sacc[t2], a, bias, dist0 - 32 * t2, kbase + 32 * t2 + 4 * g, limit, &key_docs[wave][32 * t2 + 4 * g], qdoc);
      } else {
        plain_weights<CAP, BIAS>(a, bias, lo, w, c);
        plain16<CAP, BIAS, -1>(sacc[0], a, bias, dist0, lo);
        plain16<CAP, BIAS, -1>(sacc[1], a, bias, dist0 - 32, lo);
      }
      float mx = -INFINITY;
#pragma unroll
      for (int t2 = 0; t2 < 2; ++t2)
#pragma unroll
        for (int r = 0; r < 16; ++r) mx = fmaxf(mx, sacc[t2][r]);
      // The exponents below are v w + c less the maximum without a rounding in between, and the rounded maximum is up to 2^-24 of itself
      // too small: an exponent above zero, which overflows from 2^31 on.  From 2^28 on the scores are rounded first, like the maximum.
      // (With slopes they are; a cap up to 64 has no such scores.)
      const bool large = BIAS != 1 && CAP != 1 && plain && __builtin_amdgcn_ballot_w64(fabsf(fmaf(mx, w, c)) > 0x1p28f) != 0;
      mx = fmaf(halfwave_max(mx), w, c);   // (w is positive: it commutes with the maximum)
      if (large) {
#pragma unroll
        for (int t2 = 0; t2 < 2; ++t2)
#pragma unroll
          for (int r = 0; r < 16; ++r) sacc[t2][r] = fmaf(sacc[t2][r], w, c);
        w = 1.0f;
        c = 0.f;
      }
      // The running maximum follows the block's only when that is more than 2^8 above it (see the attention without changes).  A row
      // that has met no key yet keeps -infinity, and 0 in its place where it is subtracted: its terms are exp2(-infinity) = 0.
      const bool move = __builtin_amdgcn_ballot_w64(mx > m_run + 8.0f) != 0;
      const float m_new = move ? fmaxf(m_run, mx) : m_run;
      const float m_sub = m_new == -INFINITY ? 0.f : m_new;
      const float off = c - m_sub;
      float sum = 0.f;
#pragma unroll
      for (int t2 = 0; t2 < 2; ++t2)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const float p = __builtin_amdgcn_exp2f(fmaf(sacc[t2][r], w, off));
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
    if (m.docs && it + 1 < n_it) key_docs[wave][lane] = next_doc;
    cur = next;
    next = after;
    wait_loads_and_barrier();
  }
  // merge the two parities: the odd one hands (m, l, O) over through LDS (all tiles are free after the last barrier)
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
  if (par == 0 && query < s) {
    const float m1 = xch[(DT * 16) * 64 + lane], l1 = xch[(DT * 16 + 1) * 64 + lane];
    const float top = fmaxf(m_run, m1), m_sub = top == -INFINITY ? 0.f : top;
    const float a0 = __builtin_amdgcn_exp2f(m_run - m_sub), a1 = __builtin_amdgcn_exp2f(m1 - m_sub);
    const float l = l_run * a0 + l1 * a1;
    const float inv = l == 0.f ? 0.f : 1.0f / l;   // (no pair left: zeros)
    const float w0 = a0 * inv, w1 = a1 * inv;
    bf16_t* Op = f.attn + m.attn + (long long)query * f.ldo;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        float o[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] = oacc[dt][4 * c + e] * w0 + xch[(dt * 16 + 4 * c + e) * 64 + lane] * w1;
        u32x2 w = {pack2_bf16(o[0], o[1]), pack2_bf16(o[2], o[3])};
        *(u32x2*)(Op + dt * 32 + 8 * c + 4 * g) = w;
      }
    if (g == 0) f.lse[m.vec + query] = l == 0.f ? -INFINITY : (m_sub + __log2f(l)) * LN2;
  }
}

// Ahead of the other kernels.  Workgroups y < nmat (backward): rowsum(dO * O) of every query row, 0 for padding.  The others: documents
// of every block of 64 tokens, a wavefront each.
template <int D>
__global__ __launch_bounds__(256) void attn_biased_prepare_kernel(BiasedArgs a, int nmat) {
  const FusedArgs& f = a.f;
  const int lane = threadIdx.x & 63, g = lane >> 5, wave = threadIdx.x >> 6, s = f.s;
  if ((int)blockIdx.y < nmat) {
    const Matrix m = matrix_of<D>(a, blockIdx.y, blockIdx.z);
    const int query = blockIdx.x * 128 + wave * 32 + (lane & 31);
    const int qrow = min(query, s - 1);
    float delta = 0.f;
    const bf16_t* G = f.d_attn + m.attn + (long long)qrow * f.ldo;
    const bf16_t* O = f.attn + m.attn + (long long)qrow * f.ldo;
#pragma unroll
    for (int ks = 0; ks < D / 16; ++ks) delta += delta_piece(*(const bf16x8*)(G + ks * 16 + g * 8), *(const bf16x8*)(O + ks * 16 + g * 8));
    delta = halfwave_sum(delta);
    if (m.docs && m.docs[qrow] < 0) delta = 0.f;
    if (g == 0 && query < s) f.delta[m.vec + qrow] = delta;
    return;
  }
  // sequences of the launch's device rows: device z's, the first of a row speaks for the others
  const int at = a.dev0 + (int)blockIdx.z, seq = (int)blockIdx.y - nmat;
  if (blockIdx.z > 0 && at % a.q != 0) return;
  const long long gseq = (long long)(at / a.q) * a.nb + seq;
  for (int blk = blockIdx.x * 2 + (wave & 1); blk < a.nblk && wave < 2; blk += 2 * gridDim.x) {
    const int t = blk * BLK + lane;
    const int doc = t < s ? a.documents[gseq * s + t] : 0x7fffffff;   // (past the end: no part)
    const bool pad = t < s && doc < 0;
    int lo = t < s && doc >= 0 ? doc : 0x7fffffff, hi = t < s && doc >= 0 ? doc : -1;
#pragma unroll
    for (int step = 1; step < 64; step <<= 1) {
      lo = min(lo, __shfl_xor(lo, step));
      hi = max(hi, __shfl_xor(hi, step));
    }
    const int any = __builtin_amdgcn_ballot_w64(pad) != 0;
    if (lane == 0) const_cast<i32x4_t*>(a.blocks)[gseq * a.nblk + blk] = i32x4_t{lo, hi, any, 0};
  }
}

bool desc_ok(const AttnBiasedDesc& b) {
  const AttnFusedDesc& d = b.base;
  if (!attn_fused_supported(d.d)) return false;
  if (d.s < 1 || d.nb < 1 || d.nh < 1 || d.ndev < 1 || d.ndev > 65535) return false;
  if ((long long)d.nb * d.nh + d.nb > 65535) return false;
  if (d.ld % 8 || d.ldo % 8 || d.ld < 3 * d.d * d.nh || d.ldo < d.d * d.nh) return false;
  if ((long long)((d.s + BLK - 1) / BLK) * d.nb * d.nh >= (1 << 23)) return false;   // 2^32 threads in a launch
  return (long long)PAIR * d.ld * 2 < (1ll << 31);
}

BiasedArgs make_args(const AttnBiasedDesc& b) {
  const AttnFusedDesc& d = b.base;
  BiasedArgs a = {};
  FusedArgs& f = a.f;
  f.qkv = (const bf16_t*)d.qkv; f.attn = (bf16_t*)d.attn; f.lse = d.lse;
  f.d_attn = (const bf16_t*)d.d_attn; f.d_qkv = (bf16_t*)d.d_qkv; f.delta = d.delta;
  f.s = d.s; f.nh = d.nh; f.ld = d.ld; f.ldo = d.ldo;
  f.dev_qkv = d.dev_qkv; f.dev_attn = d.dev_attn; f.dev_vec = (long long)d.nb * d.nh * d.s;
  f.scale = 1.0f / sqrtf((float)d.d);
  f.scale_log2 = (float)(1.4426950408889634 / sqrt((double)d.d));
  a.nb = d.nb; a.q = b.q; a.dev0 = b.dev0; a.causal = d.causal; a.nblk = (d.s + BLK - 1) / BLK;
  if (b.cap > 0) {
    const double inverse = 1.0 / (sqrt((double)d.d) * b.cap);
    int shift = 0;
    if (cap_form(b) == 2) frexp(inverse, &shift);
    const double in = ldexp(inverse, -shift);   // u / x
    a.cap_pre = (float)ldexp(1.0, shift);
    a.cap_log2 = (float)(b.cap * 1.4426950408889634);
    const double of[5] = {1.0, -1.0 / 3, 2.0 / 15, -17.0 / 315, 62.0 / 2835};
    double power = in;
    for (int k = 0; k < 5; ++k, power *= in * in) a.tanh_of[k] = (float)(of[k] * power);
    a.cap_exp = (float)(2.0 * in * 1.4426950408889634);
    a.cap_small = (float)(0.25 / in);
    a.weight_lo = (float)(b.cap * 1.4426950408889634 * (in / (double)a.tanh_of[0]) - (double)a.cap_log2);
  } else {
    a.weight_lo = (float)(1.4426950408889634 / sqrt((double)d.d) - (double)f.scale_log2);
  }
  a.slopes = b.slopes; a.table = b.table; a.documents = b.documents; a.prefix = b.prefix;
  a.blocks = (const i32x4_t*)b.blocks; a.table_parts = b.table_parts;
  if (b.table) {
    a.buckets = b.buckets; a.two_sided = b.two_sided;
    a.side = b.two_sided ? b.buckets / 2 : b.buckets;
    for (int k = 0; k <= a.side; ++k) a.first[k] = b.first[k];
    a.far = a.first[a.side - 1];
  }
  return a;
}

template <int D, int CAP, int BIAS>
void fwd_launch(const BiasedArgs& a, const AttnFusedDesc& d, bool big, hipStream_t st) {
  const int rows = big ? 128 : BLK;
  const dim3 grid(d.nb * d.nh, (d.s + rows - 1) / rows, d.ndev);
  if (big) attn_biased_fwd_kernel<D, 4, CAP, BIAS><<<grid, 512, 0, st>>>(a);
  else attn_biased_fwd_kernel<D, 2, CAP, BIAS><<<grid, 256, 0, st>>>(a);
}

}  // namespace

void launch_attn_biased_prepare(const BiasedArgs& a, int d, bool delta, int nmat, int ndev, hipStream_t st) {
  const int mats = delta ? nmat : 0, seqs = a.documents ? a.nb : 0;
  if (mats + seqs == 0) return;
  const dim3 grid((a.f.s + 127) / 128, mats + seqs, ndev);
  if (d == 64) attn_biased_prepare_kernel<64><<<grid, 256, 0, st>>>(a, mats);
  else attn_biased_prepare_kernel<128><<<grid, 256, 0, st>>>(a, mats);
}

// 64-row workgroups as long as all of them run at once (one a compute unit of width 128, two of 64): a wavefront has the same loop
// either way and a SIMD to itself.  64 rows / 128 rows, us: width 128, causal with a cap, 16 matrices of 1024 (256 workgroups of 64
// rows) 23.7 / 26.8, 32 of them 31.3 / 27.5; width 64, 16 of 2048 (512) 29.7 / 37.7, 64 of 1024 (1024) 27.9 / 27.1, without a mask
// 40.1 / 34.2.  The bits are the same.
bool attn_biased_fwd_wide(const AttnBiasedDesc& b) {
  const AttnFusedDesc& d = b.base;
  return (long long)((d.s + BLK - 1) / BLK) * d.nb * d.nh * d.ndev > num_cus() * (d.d == 64 ? 2 : 1);
}

int launch_attn_biased_fwd(const AttnBiasedDesc& b, hipStream_t st) {
  const AttnFusedDesc& d = b.base;
  if (!desc_ok(b) || !d.qkv || !d.attn || !d.lse) return OPTIMUS_ESHAPE;
  const BiasedArgs a = make_args(b);
  launch_attn_biased_prepare(a, d.d, false, d.nb * d.nh, d.ndev, st);
  with_kind(b, [&](auto width, auto cap, auto bias) {
    fwd_launch<decltype(width)::value, decltype(cap)::value, decltype(bias)::value>(a, d, attn_biased_fwd_wide(b), st);
  });
  return hip_launch_status();
}

int launch_attn_biased_bwd(const AttnBiasedDesc& b, hipStream_t st) {
  const AttnFusedDesc& d = b.base;
  if (!desc_ok(b) || !d.qkv || !d.attn || !d.lse || !d.d_attn || !d.d_qkv || !d.delta) return OPTIMUS_ESHAPE;
  const BiasedArgs a = make_args(b);
  launch_attn_biased_prepare(a, d.d, true, d.nb * d.nh, d.ndev, st);
  return launch_attn_biased_bwd_kernels(a, b, st);
}

}  // namespace optimus
