// Backward of the attention over chosen blocks with lists (attention_selected_kernel.hpp): dQ as the forward makes its output, a row a pair, added
// up by the query; dK and dV by workgroups that own a block's keys, or 64 or 128 of them, and walk a piece of its list.
// Up to 128 keys a block one pass makes all three gradients (selected_bwd_kernel); larger blocks take two, one for dQ, whose rows are the whole
// block's, and one for dK and dV of 64 or 128 keys (16 (sequence, head)s of
// 16384 x 128, 8 of 64 blocks of 256: 1283 us, 4423 with a mask).
#include "attention_selected_kernel.hpp"

namespace optimus {
namespace {

// P = 2^x, at most 1 (see the attention with changed scores)
__device__ __forceinline__ float weight_of(float x) { return __builtin_amdgcn_fmed3f(__builtin_amdgcn_exp2f(x), 0.f, 1.f); }
// what is subtracted from a row's scores; a row that saw nothing: +infinity, which makes every P of it zero
__device__ __forceinline__ float lse2_of(float lse) { return lse == -INFINITY ? INFINITY : lse * LOG2E; }

// dS^T of 32 keys in LDS (rows_at from kt; V 64 rows behind) against the wavefront's queries, packed as fragments
template <int D>
__device__ __forceinline__ void dq_scores(bf16x8 (&dsf)[2], unsigned kt, const bf16x8 (&qf)[D / 16], const bf16x8 (&dof)[D / 16], float lse2, float delta,
                                          float scale_log2, bool masked, int reach) {
  constexpr int KS = D / 16;
  f32x16 sacc = zero16(), pacc = zero16();
  pipelined<2 * KS, 2>([&](int n) { return rows_at<D>(kt, n & 1 ? BLK : 0, n / 2); },
                       [&](int n, const bf16x8& x) {
                         f32x16& acc = n & 1 ? pacc : sacc;
                         acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x, n & 1 ? dof[n / 2] : qf[n / 2], acc, 0, 0, 0);
                       });
  if (masked) {   // (few tiles: the asm keeps the compiler from comparing in all of them)
    asm volatile("");
#pragma unroll
    for (int r = 0; r < 16; ++r) sacc[r] = slot(r) > reach ? -INFINITY : sacc[r];
  }
#pragma unroll
  for (int r = 0; r < 16; ++r) sacc[r] = weight_of(fmaf(sacc[r], scale_log2, -lse2)) * (pacc[r] - delta);
  dsf[0] = pack_acc<0>(sacc);
  dsf[1] = pack_acc<1>(sacc);
}

// dQ rows of larger blocks: 64 keys at a time through two stages.
template <int D>
__global__ __launch_bounds__(256, 2) void selected_dq_kernel(SelectedArgs a) {
  constexpr int KS = D / 16, DT = D / 32;
  __shared__ __attribute__((aligned(1024))) bf16_t lds[2][2][BLK * D];   // [stage][K, V]
  const FusedArgs& f = a.f;
  const int tid = threadIdx.x, lane = tid & 63, g = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int unit = blockIdx.x / a.portion, matrix = blockIdx.x % a.portion, mm = a.mat0 + matrix;
  ListItem it;
  if (!list_item(a, 0, mm, unit, &it)) return;
  const SelMatrix m = selected_matrix<D>(a, mm);
  const bf16_t* Qp = f.qkv + m.qkv;
  const bf16_t* Gp = f.d_attn + m.attn;
  const int key0 = it.block * a.block, last = m.len - 1;
  const int steps = (min(a.block, m.len - key0) + BLK - 1) / BLK;
  const int rounds = (it.pairs + kQueries - 1) / kQueries;
  TileLoader<D, 4, BLK, true> ldr;
  ldr.init(f.ld, wave, lane);
  auto issue = [&](int step, int st) {
    ldr.issue(Qp + D, key0 + step * BLK, m.len, lds[st][0]);
    ldr.issue(Qp + 2 * D, key0 + step * BLK, m.len, lds[st][1]);
  };
  issue(0, 0);
  const unsigned in_rows = lds_address(lds) + lane_rows<D>(lane), in_cols = lds_address(lds) + lane_cols<D>(lane);
  const long long pairs = (long long)f.s * a.count, first = mm * pairs + it.start, out = matrix * pairs + it.start;
  const int* list = a.list + first;
  const int row = wave * 32 + (lane & 31);
  bf16x8 qf[KS], dof[KS];
  // a tile's queries are requested a tile ahead, their numbers two, and past the end too: the last one again
  int t = 0, t_next = list[min(row, it.pairs - 1)];
  float lse = 0.f, delta = 0.f;
  auto load_queries = [&](int base) {
    t = t_next;
    const bf16_t* q = Qp + (long long)t * f.ld + g * 8;
    const bf16_t* o = Gp + (long long)t * f.ldo + g * 8;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      qf[ks] = *(const bf16x8*)(q + ks * 16);
      dof[ks] = *(const bf16x8*)(o + ks * 16);
    }
    lse = f.lse[m.vec + t];
    delta = f.delta[m.vec + t];
    t_next = list[min(base + kQueries + row, it.pairs - 1)];
  };
  load_queries(0);
  wait_loads_and_barrier();
  int stage = 0;
  for (int round = 0; round < rounds; ++round) {
    const int base = round * kQueries, left = it.pairs - base - wave * 32;
    const int limit = a.causal ? min(t, last) : last;
    const float lse2 = lse2_of(lse);
    f32x16 acc[DT];
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) acc[dt] = zero16();
    for (int step = 0; step < steps; ++step, stage ^= 1) {
      if (step + 1 < steps || round + 1 < rounds) issue(step + 1 < steps ? step + 1 : 0, stage ^ 1);
      const int kbase = key0 + step * BLK;
      if (left > 0 && __builtin_amdgcn_ballot_w64(limit >= kbase) != 0) {
        const unsigned at = (unsigned)(stage * (2 * BLK * D * 2));
        const bool masked = __builtin_amdgcn_ballot_w64(limit < kbase + BLK - 1) != 0;
#pragma unroll
        for (int t2 = 0; t2 < 2; ++t2) {
          bf16x8 dsf[2];
          dq_scores<D>(dsf, in_rows + at + t2 * (32 * D * 2), qf, dof, lse2, delta, f.scale_log2, masked, limit - kbase - 32 * t2 - 4 * g);
          pipelined<2 * DT, 2>([&](int n) { return cols_at<D>(in_cols + at, t2 * 32 + n / DT * 16, n % DT); },
                               [&](int n, const bf16x8& x) {
                                 acc[n % DT] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x, dsf[n / DT], acc[n % DT], 0, 0, 0);
                               });
        }
      }
      wait_loads_and_barrier();
    }
    load_queries(base + kQueries);
    if (left > 0) {
      const long long at = out + base + wave * 32;
      store_parts<DT>(a.rows + at * D, a.units + at, acc, min(left, 32), g, lane);
    }
  }
}

// A tile of gathered rows, global -> LDS directly: rows of [.][ld] matrices by their numbers, in the layout of TileLoader.  64-bit addresses:
// a list's rows lie anywhere in the sequence.
template <int D, int NW, int ROWS>
struct GatherLoader {
  static constexpr int CH = D / 8, ROWS_PER_KIB = 64 / CH, PIECES = ROWS * D * 2 / 1024, PER = PIECES / NW;
  static_assert(PIECES % NW == 0, "tile must divide over the wavefronts");
  int number[PER], wave, lane;
  // the numbers of the tile's rows: list entries row0 .., the last one again past the end
  __device__ __forceinline__ void fetch(const int* list, int row0, int pairs) {
#pragma unroll
    for (int it = 0; it < PER; ++it) number[it] = list[min(row0 + (wave * PER + it) * ROWS_PER_KIB + lane / CH, pairs - 1)];
  }
  __device__ __forceinline__ void issue(const bf16_t* mat, int ld, bf16_t* tile) const {
    const unsigned lds_base = (unsigned)(size_t)(__attribute__((address_space(3))) bf16_t*)tile;
#pragma unroll
    for (int it = 0; it < PER; ++it) {
      const int row = (wave * PER + it) * ROWS_PER_KIB + lane / CH;
      const bf16_t* p = mat + (long long)number[it] * ld + (((lane % CH) ^ swz<D>(row)) << 3);
      const unsigned m0v = __builtin_amdgcn_readfirstlane(lds_base + (unsigned)(wave * PER + it) * 1024u);
      asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off" ::"v"(p), "s"(m0v) : "memory", "m0");
    }
  }
};

// 32 x 32 scores (rows: queries, columns: keys) and dP -> P and dS in their place.  l, d, t: of the lane's queries; masked: some are ahead of
// the key
__device__ __forceinline__ void list_scores(f32x16& sacc, f32x16& pacc, const float* l, const float* d, const int* t, float scale_log2, bool masked, int key) {
  if (masked) {   // (few tiles: the asm keeps the compiler from comparing in all of them)
    asm volatile("");
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      const int4 t4 = *(const int4*)(t + 8 * c);
      const int tv[4] = {t4.x, t4.y, t4.z, t4.w};
#pragma unroll
      for (int e = 0; e < 4; ++e) sacc[4 * c + e] = tv[e] < key ? -INFINITY : sacc[4 * c + e];
    }
  }
#pragma unroll
  for (int c = 0; c < 4; ++c) {
    const float4 l4 = *(const float4*)(l + 8 * c), d4 = *(const float4*)(d + 8 * c);
    const float lv[4] = {l4.x, l4.y, l4.z, l4.w}, dv[4] = {d4.x, d4.y, d4.z, d4.w};
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int r = 4 * c + e;
      const float p = weight_of(fmaf(sacc[r], scale_log2, -lv[e]));
      sacc[r] = p;
      pacc[r] = p * (pacc[r] - dv[e]);
    }
  }
}
__device__ __forceinline__ bool single_piece(const SelectedArgs& a, int mm, int block) {
  const int* first = a.first_item + ((long long)a.mats + mm) * (a.blocks + 1) + block;
  return first[1] - first[0] == 1;
}
// A wavefront's sums of 32 keys from k0 on: of a block's only piece dK or dV themselves, at column `col`, a row after the other through LDS of the
// wavefront's own (32 rows of D floats); else fp32 rows to `to`.
template <int D>
__device__ __forceinline__ void key_sums(const SelectedArgs& a, const SelMatrix& m, const f32x16 (&acc)[D / 32], int k0, int col, float w, bool only,
                                         float* row, float* to, int lane) {
  const int g = lane >> 5;
  if (!only) {
    store_rows<D / 32>(to, acc, m.len - k0, g, lane);
    return;
  }
#pragma unroll
  for (int r = 0; r < 16; ++r)
#pragma unroll
    for (int dt = 0; dt < D / 32; ++dt) row[(slot(r) + 4 * g) * D + dt * 32 + (lane & 31)] = acc[dt][r] * w;
  __builtin_amdgcn_wave_barrier();
  for (int k = g; k < 32; k += 2)
    write_ordered<D / 32>(a.f.d_qkv + m.qkv + (long long)(k0 + k) * a.f.ld + col, row + k * D, lane & 31, k0 + k < m.len);
  __builtin_amdgcn_wave_barrier();
}

template <int D>
struct SelDkvLds {
  bf16_t tile[2][2][PAIR * D];   // [stage][Q, dO]
  alignas(16) float l[2][PAIR];
  alignas(16) float d[2][PAIR];
  alignas(16) int t[2][PAIR];
};
// dK and dV of 64 keys from a piece of their block's list.  Wavefronts: 32 keys, every second 64 queries, as in the fused attention.
template <int D>
__global__ __launch_bounds__(256, D == 64 ? 2 : 1) void selected_dkv_kernel(SelectedArgs a) {
  constexpr int KS = D / 16, DT = D / 32, NRG = 2;
  __shared__ __attribute__((aligned(1024))) SelDkvLds<D> lds;
  const FusedArgs& f = a.f;
  const int tid = threadIdx.x, lane = tid & 63, g = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int rg = wave % NRG, par = wave / NRG;
  const int unit = blockIdx.x / a.portion, matrix = blockIdx.x % a.portion, mm = a.mat0 + matrix;
  const int tiles = a.block / BLK, item = unit / tiles, tile = unit % tiles;
  ListItem it;
  if (!list_item(a, 1, mm, item, &it)) return;
  const SelMatrix m = selected_matrix<D>(a, mm);
  const int kt0 = it.block * a.block + tile * BLK;
  if (kt0 >= m.len) return;
  const bf16_t* Qp = f.qkv + m.qkv;
  const bf16_t* Gp = f.d_attn + m.attn;
  const int k0 = kt0 + rg * 32, key = k0 + (lane & 31), krow = min(key, m.len - 1);
  bf16x8 kf[KS], vf[KS];
#pragma unroll
  for (int ks = 0; ks < KS; ++ks) {
    kf[ks] = *(const bf16x8*)(Qp + D + (long long)krow * f.ld + ks * 16 + g * 8);
    vf[ks] = *(const bf16x8*)(Qp + 2 * D + (long long)krow * f.ld + ks * 16 + g * 8);
  }
  const int* list = a.list + m.vec * a.count + it.start;
  const int n_it = (it.pairs + PAIR - 1) / PAIR;
  f32x16 dkacc[DT], dvacc[DT];
#pragma unroll
  for (int dt = 0; dt < DT; ++dt) {
    dkacc[dt] = zero16();
    dvacc[dt] = zero16();
  }
  const unsigned in_rows = lds_address(lds.tile) + lane_rows<D>(lane), in_cols = lds_address(lds.tile) + lane_cols<D>(lane);
  GatherLoader<D, 4, PAIR> ldr;
  ldr.wave = wave;
  ldr.lane = lane;
  // a row's numbers go through registers and reach LDS at the end of an iteration
  int next_t = 0, row_t = 0;
  float next_l = 0.f, next_d = 0.f;
  auto load_numbers = [&](int n) {   // of iteration n
    ldr.fetch(list, n * PAIR, it.pairs);
    if (tid < PAIR) row_t = list[min(n * PAIR + tid, it.pairs - 1)];
  };
  auto issue = [&](int st) {
    if (tid < PAIR) {
      next_t = row_t;
      next_l = f.lse[m.vec + row_t];
      next_d = f.delta[m.vec + row_t];
    }
    ldr.issue(Qp, f.ld, lds.tile[st][0]);
    ldr.issue(Gp, f.ldo, lds.tile[st][1]);
  };
  auto store_numbers = [&](int n, int st) {   // (past the end of the list: no P)
    if (tid < PAIR) {
      lds.l[st][tid] = n * PAIR + tid < it.pairs ? lse2_of(next_l) : INFINITY;
      lds.d[st][tid] = next_d;
      lds.t[st][tid] = next_t;
    }
  };
  load_numbers(0);
  issue(0);
  if (n_it > 1) load_numbers(1);
  store_numbers(0, 0);
  wait_loads_and_barrier();
  for (int n = 0; n < n_it; ++n) {
    const int st = n & 1;
    if (n + 1 < n_it) {
      issue(st ^ 1);
      if (n + 2 < n_it) load_numbers(n + 2);
    }
    const int base = n * PAIR + par * BLK;
    // (the block's own queries come first: where the first of 64 is behind the keys, all are)
    const int first_t = __builtin_amdgcn_readfirstlane(lds.t[st][par * BLK]);
    if (base < it.pairs && k0 < m.len) {
      const unsigned stage = (unsigned)((st * 2 * PAIR + par * BLK) * D * 2);
      const unsigned qt = in_rows + stage, qc = in_cols + stage;
      const bool masked = a.causal && first_t < k0 + 31;
#pragma unroll
      for (int t2 = 0; t2 < 2; ++t2) {
        f32x16 sacc = zero16(), pacc = zero16();
        pipelined<2 * KS, 2>([&](int k) { return rows_at<D>(qt, (k & 1 ? PAIR : 0) + t2 * 32, k / 2); },
                             [&](int k, const bf16x8& x) {
                               f32x16& acc = k & 1 ? pacc : sacc;
                               acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x, k & 1 ? vf[k / 2] : kf[k / 2], acc, 0, 0, 0);
                             });
        const int at = par * BLK + t2 * 32 + 4 * g;
        list_scores(sacc, pacc, lds.l[st] + at, lds.d[st] + at, lds.t[st] + at, f.scale_log2, masked, key);
        const bf16x8 pf[2] = {pack_acc<0>(sacc), pack_acc<1>(sacc)}, dsf[2] = {pack_acc<0>(pacc), pack_acc<1>(pacc)};
        pipelined<4 * DT, 2>([&](int k) { return cols_at<D>(qc, (k & 1 ? 0 : PAIR) + t2 * 32 + k / (2 * DT) * 16, k / 2 % DT); },
                             [&](int k, const bf16x8& x) {
                               const int dt = k / 2 % DT, u = k / (2 * DT);
                               f32x16& acc = k & 1 ? dkacc[dt] : dvacc[dt];
                               acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k & 1 ? dsf[u] : pf[u], x, acc, 0, 0, 0);
                             });
      }
    }
    if (n + 1 < n_it) store_numbers(n + 1, st ^ 1);
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
  if (par == 1) return;
#pragma unroll
  for (int dt = 0; dt < DT; ++dt)
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      dkacc[dt][r] += xch[(dt * 16 + r) * 64 + lane];
      dvacc[dt][r] += xch[((DT + dt) * 16 + r) * 64 + lane];
    }
  const bool only = single_piece(a, mm, it.block);
  float* to = a.key_rows + (((long long)matrix * a.most[1] + item) * tiles + tile) * (2 * BLK * D) + rg * 32 * D;
  key_sums<D>(a, m, dkacc, k0, D, f.scale, only, xch, to, lane);
  key_sums<D>(a, m, dvacc, k0, 2 * D, 1.0f, only, xch, to + BLK * D, lane);
}

// Blocks of 64 or 128 keys: all three gradients in one pass over the list, 64 queries at a time.  P and dS are computed once, with a wavefront's 32 keys
// as columns, which is what dK and dV take; dS goes through LDS as [key][query], where the transposing reads fetch it and K for dQ, a
// 32 x 32 tile (or two) a wavefront.  A lane has one query's 16 numbers of a tile, 32 columns of dQ, which get a scale of their own.
// Bound: the steps of a block of queries one after the other, two barriers, two wavefronts a SIMD.  16 (sequence, head)s of 4096 x 128, 8 of 32 blocks:
// 119 us, 640 TFLOP/s of five products (dQ in a pass of its own 83, dK and dV 95); 20 of up to 10000 x 64, 12 of 157 blocks 136 (118 and 127).
template <int D, int KEYS>
struct SelectedBwd {
  static constexpr bool WIDE = D == 128 && KEYS == 128;
  static constexpr int WAVES = WIDE ? 8 : 4, THREADS = 64 * WAVES, RG = KEYS / 32, PARW = WAVES / RG;   // RG: groups of 32 keys; PARW: wavefronts of one
  static constexpr int TILES = 2 * (D / 32) / WAVES;   // of dQ a wavefront
  static constexpr bool SMALL = D == 64 && KEYS == 64;
  static constexpr int KREG = WIDE ? 4 : D == 128 || SMALL ? 0 : D / 16, VREG = D == 128 ? 0 : D / 16;   // own fragments in registers, others in LDS
  // Wavefronts a SIMD.  SMALL: three, with K from LDS and its fragments one step ahead, 168 registers (20 (sequence, head)s of up to 10000, 12 of 157
  // blocks: 265 us a call with two, 253 with three, 271 with fragments two ahead, which spill)
  static constexpr int MOST = SMALL ? 3 : 2, AHEAD = SMALL ? 1 : 2;
  struct Lds {
    bf16_t block[2][2][BLK * D];       // [stage][Q, dO]
    bf16_t k[KEYS * D];
    bf16_t v[VREG ? 512 : KEYS * D];
    bf16_t ds[KEYS * BLK];             // [key][query of the block], laid out as a tile of width 64
    alignas(16) float l[2][BLK];
    alignas(16) float d[2][BLK];
    alignas(16) int t[2][BLK];
  };
};
// A lane's 16 numbers of a query's 32 columns from 32 dt on, with a scale of their own
template <int DT>
__device__ __forceinline__ void store_part(const f32x16& acc, int row0, int dt, __amdgpu_buffer_rsrc_t rows, __amdgpu_buffer_rsrc_t units, int lane) {
  const RowScale s = row_scale(largest_size(acc, 0.f));
  u32x4 w[2];   // (64 whole bytes of sixteen rows a store)
  pack_columns(acc, s.scale, w);
  const int at = (row0 + (lane & 15)) * (64 * DT) + dt * 64 + (lane >> 4 & 1) * 32 + (lane >> 5) * 16;
  __builtin_amdgcn_raw_buffer_store_b128(w[0], rows, at, 0, 0);
  __builtin_amdgcn_raw_buffer_store_b128(w[1], rows, at + 16 * 64 * DT, 0, 0);
  __builtin_amdgcn_raw_buffer_store_b32((int)s.unit, units, lane < 32 ? ((row0 + lane) * DT + dt) * 4 : 0x7fffffff, 0, 0);
}

template <int D, int KEYS>
__global__ __launch_bounds__((SelectedBwd<D, KEYS>::THREADS), (SelectedBwd<D, KEYS>::MOST)) void selected_bwd_kernel(SelectedArgs a) {
  typedef SelectedBwd<D, KEYS> B;
  constexpr int KS = D / 16, DT = D / 32, NW = B::WAVES, KREG = B::KREG, VREG = B::VREG;
  extern __shared__ __attribute__((aligned(1024))) char selected_bwd_lds[];   // (of a size that the compiler does not know: where it holds one wavefront
  typename B::Lds& lds = *(typename B::Lds*)selected_bwd_lds;                 // a SIMD, 512 registers are half of them moves)
  const FusedArgs& f = a.f;
  const int tid = threadIdx.x, lane = tid & 63, g = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int rg = wave % B::RG, par = wave / B::RG;
  const int item = blockIdx.x / a.portion, matrix = blockIdx.x % a.portion, mm = a.mat0 + matrix;
  ListItem it;
  if (!list_item(a, 1, mm, item, &it)) return;
  const SelMatrix m = selected_matrix<D>(a, mm);
  const int kt0 = it.block * KEYS;
  const bf16_t* Qp = f.qkv + m.qkv;
  const bf16_t* Gp = f.d_attn + m.attn;
  const int k0 = kt0 + rg * 32, key = k0 + (lane & 31), krow = min(key, m.len - 1);
  bf16x8 kf[KREG > 0 ? KREG : 1], vf[VREG > 0 ? VREG : 1];
#pragma unroll
  for (int ks = 0; ks < KREG; ++ks) kf[ks] = *(const bf16x8*)(Qp + D + (long long)krow * f.ld + ks * 16 + g * 8);
#pragma unroll
  for (int ks = 0; ks < VREG; ++ks) vf[ks] = *(const bf16x8*)(Qp + 2 * D + (long long)krow * f.ld + ks * 16 + g * 8);
  {
    TileLoader<D, NW, KEYS, true> own;   // (keys past the end of the sequence: zeros, which whatever their dS is adds nothing to dQ)
    own.init(f.ld, wave, lane);
    own.issue(Qp + D, kt0, m.len, lds.k);
    if constexpr (VREG == 0) own.issue(Qp + 2 * D, kt0, m.len, lds.v);
  }
  const long long pairs = (long long)f.s * a.count;
  const int* list = a.list + mm * pairs + it.start;
  f16_t* const rows = a.rows + (matrix * pairs + it.start) * D;
  float* const units = a.units + (matrix * pairs + it.start) * DT;
  const int n_it = (it.pairs + BLK - 1) / BLK;
  f32x16 dkacc[DT], dvacc[DT];
#pragma unroll
  for (int dt = 0; dt < DT; ++dt) {
    dkacc[dt] = zero16();
    dvacc[dt] = zero16();
  }
  const unsigned in_rows = lds_address(lds.block) + lane_rows<D>(lane), in_cols = lds_address(lds.block) + lane_cols<D>(lane);
  const unsigned own_k = lds_address(lds.k) + lane_rows<D>(lane) + rg * 32 * D * 2, own_v = lds_address(lds.v) + lane_rows<D>(lane) + rg * 32 * D * 2;
  const unsigned k_cols = lds_address(lds.k) + lane_cols<D>(lane), ds_cols = lds_address(lds.ds) + lane_cols<64>(lane);
  const int ds_row = rg * 32 + (lane & 31);
  const unsigned ds_at = lds_address(lds.ds) + (unsigned)(ds_row * 128 + (swz<64>(ds_row) << 4) + g * 8);
  const int q_half = wave / (NW / 2), dt0 = wave % (NW / 2) * B::TILES;   // of dQ
  GatherLoader<D, NW, BLK> ldr;
  ldr.wave = wave;
  ldr.lane = lane;
  // a row's numbers go through registers and reach LDS at the end of an iteration
  int next_t = 0, row_t = 0;
  float next_l = 0.f, next_d = 0.f;
  auto load_numbers = [&](int n) {   // of iteration n
    ldr.fetch(list, n * BLK, it.pairs);
    if (tid < BLK) row_t = list[min(n * BLK + tid, it.pairs - 1)];
  };
  auto issue = [&](int st) {
    if (tid < BLK) {
      next_t = row_t;
      next_l = f.lse[m.vec + row_t];
      next_d = f.delta[m.vec + row_t];
    }
    ldr.issue(Qp, f.ld, lds.block[st][0]);
    ldr.issue(Gp, f.ldo, lds.block[st][1]);
  };
  auto store_numbers = [&](int n, int st) {   // (past the end of the list: no P)
    if (tid < BLK) {
      lds.l[st][tid] = n * BLK + tid < it.pairs ? lse2_of(next_l) : INFINITY;
      lds.d[st][tid] = next_d;
      lds.t[st][tid] = next_t;
    }
  };
  load_numbers(0);
  issue(0);
  if (n_it > 1) load_numbers(1);
  store_numbers(0, 0);
  wait_loads_and_barrier();
  for (int n = 0; n < n_it; ++n) {
    const int st = n & 1;
    if (n + 1 < n_it) {
      issue(st ^ 1);
      if (n + 2 < n_it) load_numbers(n + 2);
    }
    const unsigned stage = (unsigned)(st * 2 * BLK * D * 2);
#pragma unroll
    for (int u2 = 0; u2 < 2 / B::PARW; ++u2) {
      const int half = B::PARW == 2 ? par : u2;
      if (n * BLK + half * 32 >= it.pairs) continue;   // (dQ of these rows is not stored)
      const unsigned qt = in_rows + stage + half * (32 * D * 2), qc = in_cols + stage + half * (32 * D * 2);
      // (the block's own queries come first: where the first of 32 is behind the keys, all are)
      const bool masked = a.causal && __builtin_amdgcn_readfirstlane(lds.t[st][half * 32]) < k0 + 31;
      f32x16 sacc = zero16(), pacc = zero16();
      struct Two { bf16x8 q, own; };
      pipelined<2 * KS, B::AHEAD>([&](int k) {
                             const int ks = k / 2;
                             Two x;
                             x.q = rows_at<D>(qt, k & 1 ? BLK : 0, ks);
                             if (k & 1) x.own = ks < VREG ? vf[ks < VREG ? ks : 0] : rows_at<D>(own_v, 0, ks);
                             else x.own = ks < KREG ? kf[ks < KREG ? ks : 0] : rows_at<D>(own_k, 0, ks);
                             return x;
                           },
                           [&](int k, const Two& x) {
                             f32x16& acc = k & 1 ? pacc : sacc;
                             acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x.q, x.own, acc, 0, 0, 0);
                           });
      const int at = half * 32 + 4 * g;
      list_scores(sacc, pacc, lds.l[st] + at, lds.d[st] + at, lds.t[st] + at, f.scale_log2, masked, key);
      const bf16x8 pf[2] = {pack_acc<0>(sacc), pack_acc<1>(sacc)}, dsf[2] = {pack_acc<0>(pacc), pack_acc<1>(pacc)};
#pragma unroll
      for (int c = 0; c < 4; ++c) {   // queries 8 c + 4 g .. of the lane's key
        const u32x4 w = __builtin_bit_cast(u32x4, dsf[c >> 1]);
        *(__attribute__((address_space(3))) u32x2*)(size_t)(ds_at ^ (unsigned)((half * 4 + c) << 4)) = u32x2{w[2 * (c & 1)], w[2 * (c & 1) + 1]};
      }
      pipelined<4 * DT, 2>([&](int k) { return cols_at<D>(qc, (k & 1 ? 0 : BLK) + k / (2 * DT) * 16, k / 2 % DT); },
                           [&](int k, const bf16x8& x) {
                             const int dt = k / 2 % DT, u = k / (2 * DT);
                             f32x16& acc = k & 1 ? dkacc[dt] : dvacc[dt];
                             acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k & 1 ? dsf[u] : pf[u], x, acc, 0, 0, 0);
                           });
    }
    __syncthreads();
    f32x16 dq[B::TILES];
#pragma unroll
    for (int i = 0; i < B::TILES; ++i) dq[i] = zero16();
    struct Pair { bf16x8 ds, k[B::TILES]; };
    pipelined<KEYS / 16, 2>([&](int k) {
                              Pair x;
                              x.ds = cols_at<64>(ds_cols ^ (unsigned)(q_half * 64), k * 16, 0);
#pragma unroll
                              for (int i = 0; i < B::TILES; ++i) x.k[i] = cols_at<D>(k_cols ^ (unsigned)((dt0 + i) * 64), k * 16, 0);
                              return x;
                            },
                            [&](int, const Pair& x) {
#pragma unroll
                              for (int i = 0; i < B::TILES; ++i) dq[i] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x.k[i], x.ds, dq[i], 0, 0, 0);
                            });
    if (n + 1 < n_it) store_numbers(n + 1, st ^ 1);
    // The loads into the other stage have ended, and with them the stores of the iteration before: this one's come behind the wait and stay on their way,
    // however many instructions they are.  (A wait behind them that leaves
    // just as many takes as long: 16 (sequence, head)s of 4096 x 128 165 us a call, 16 of 8192 in blocks of 64 325 for 327.)
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    const int left = __builtin_amdgcn_readfirstlane(min(it.pairs - n * BLK, BLK));
    const auto to_rows = __builtin_amdgcn_make_buffer_rsrc(rows + (long long)n * BLK * D, 0, left * (2 * D), 0x00020000);
    const auto to_units = __builtin_amdgcn_make_buffer_rsrc(units + (long long)n * BLK * DT, 0, left * (4 * DT), 0x00020000);
#pragma unroll
    for (int i = 0; i < B::TILES; ++i) store_part<DT>(dq[i], q_half * 32, dt0 + i, to_rows, to_units, lane);
    __syncthreads();
  }
  // the halves' sums of 32 keys, dV first: the odd one hands over through LDS (all block tiles are free)
  const bool only = single_piece(a, mm, it.block);
  float* xch = (float*)&lds.block[0][0][0] + rg * (DT * 16) * 64;
  float* to = a.key_rows + (((long long)matrix * a.most[1] + item) * (KEYS / BLK) + (rg >> 1)) * (2 * BLK * D) + (rg & 1) * 32 * D;
#pragma unroll
  for (int which = 0; which < 2; ++which) {
    f32x16 (&acc)[DT] = which == 0 ? dvacc : dkacc;
    if (B::PARW == 2) {
      if (which == 1) __syncthreads();
      if (par == 1) {
#pragma unroll
        for (int dt = 0; dt < DT; ++dt)
#pragma unroll
          for (int r = 0; r < 16; ++r) xch[(dt * 16 + r) * 64 + lane] = acc[dt][r];
      }
      __syncthreads();
      if (par == 0) {
#pragma unroll
        for (int dt = 0; dt < DT; ++dt)
#pragma unroll
          for (int r = 0; r < 16; ++r) acc[dt][r] += xch[(dt * 16 + r) * 64 + lane];
      }
    }
    if (par == 0) {
      if (which == 0) key_sums<D>(a, m, acc, k0, 2 * D, 1.0f, only, xch, to + BLK * D, lane);
      else key_sums<D>(a, m, acc, k0, D, f.scale, only, xch, to, lane);
    }
  }
}

// Head width 128, blocks of whole 128 keys: 128 keys, eight wavefronts, as in the attention with changed scores: own V rows and half of the K
// fragments in LDS, 64 queries at a time, a wavefront half of them.
struct SelWideLds {
  bf16_t block[2][2][BLK * 128];   // [stage][Q, dO]
  bf16_t v[128 * 128], k[128 * 128];
  alignas(16) float l[2][BLK];
  alignas(16) float d[2][BLK];
  alignas(16) int t[2][BLK];
};
__global__ __launch_bounds__(512, 2) void selected_dkv_wide_kernel(SelectedArgs a) {
  constexpr int D = 128, KS = D / 16, DT = D / 32, BKW = 128, KREG = KS / 2;
  __shared__ __attribute__((aligned(1024))) SelWideLds lds;
  const FusedArgs& f = a.f;
  const int tid = threadIdx.x, lane = tid & 63, g = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int rg = wave & 3, par = wave >> 2;
  const int unit = blockIdx.x / a.portion, matrix = blockIdx.x % a.portion, mm = a.mat0 + matrix;
  const int tiles = a.block / BKW, item = unit / tiles, tile = unit % tiles;
  ListItem it;
  if (!list_item(a, 1, mm, item, &it)) return;
  const SelMatrix m = selected_matrix<D>(a, mm);
  const int kt0 = it.block * a.block + tile * BKW;
  if (kt0 >= m.len) return;
  const bf16_t* Qp = f.qkv + m.qkv;
  const bf16_t* Gp = f.d_attn + m.attn;
  const int k0 = kt0 + rg * 32, key = k0 + (lane & 31), krow = min(key, m.len - 1);
  bf16x8 kf[KREG];
#pragma unroll
  for (int ks = 0; ks < KREG; ++ks) kf[ks] = *(const bf16x8*)(Qp + D + (long long)krow * f.ld + ks * 16 + g * 8);
  {
    TileLoader<D, 8, BKW, true> own;
    own.init(f.ld, wave, lane);
    own.issue(Qp + 2 * D, kt0, m.len, lds.v);
    own.issue(Qp + D, kt0, m.len, lds.k);
  }
  const int* list = a.list + m.vec * a.count + it.start;
  const int n_it = (it.pairs + BLK - 1) / BLK;
  f32x16 dkacc[DT], dvacc[DT];
#pragma unroll
  for (int dt = 0; dt < DT; ++dt) {
    dkacc[dt] = zero16();
    dvacc[dt] = zero16();
  }
  // (a wavefront's 32 rows of a block, and its own 32 rows of V and K)
  const unsigned in_rows = lds_address(lds.block) + lane_rows<D>(lane) + par * 32 * D * 2, in_cols = lds_address(lds.block) + lane_cols<D>(lane) + par * 32 * D * 2;
  const unsigned own_rows = lds_address(lds.v) + lane_rows<D>(lane) + rg * 32 * D * 2;
  GatherLoader<D, 8, BLK> ldr;
  ldr.wave = wave;
  ldr.lane = lane;
  int next_t = 0, row_t = 0;
  float next_l = 0.f, next_d = 0.f;
  auto load_numbers = [&](int n) {   // of iteration n
    ldr.fetch(list, n * BLK, it.pairs);
    if (tid < BLK) row_t = list[min(n * BLK + tid, it.pairs - 1)];
  };
  auto issue = [&](int st) {
    if (tid < BLK) {
      next_t = row_t;
      next_l = f.lse[m.vec + row_t];
      next_d = f.delta[m.vec + row_t];
    }
    ldr.issue(Qp, f.ld, lds.block[st][0]);
    ldr.issue(Gp, f.ldo, lds.block[st][1]);
  };
  auto store_numbers = [&](int n, int st) {   // (past the end of the list: no P)
    if (tid < BLK) {
      lds.l[st][tid] = n * BLK + tid < it.pairs ? lse2_of(next_l) : INFINITY;
      lds.d[st][tid] = next_d;
      lds.t[st][tid] = next_t;
    }
  };
  load_numbers(0);
  issue(0);
  if (n_it > 1) load_numbers(1);
  store_numbers(0, 0);
  wait_loads_and_barrier();
  for (int n = 0; n < n_it; ++n) {
    const int st = n & 1;
    if (n + 1 < n_it) {
      issue(st ^ 1);
      if (n + 2 < n_it) load_numbers(n + 2);
    }
    // (the block's own queries come first: where the first of 32 is behind the keys, all are)
    const int first_t = __builtin_amdgcn_readfirstlane(lds.t[st][par * 32]);
    if (n * BLK + par * 32 < it.pairs && k0 < m.len) {
      const unsigned stage = (unsigned)(st * 2 * BLK * D * 2);
      const unsigned qt = in_rows + stage, qc = in_cols + stage;
      const bool masked = a.causal && first_t < k0 + 31;
      f32x16 sacc = zero16(), pacc = zero16();
      struct Two { bf16x8 q, own; };
      pipelined<2 * KS, 2>([&](int k) {
                             const int ks = k / 2;
                             Two x;
                             x.q = rows_at<D>(qt, k & 1 ? BLK : 0, ks);
                             if (k & 1) x.own = rows_at<D>(own_rows, 0, ks);
                             else x.own = ks < KREG ? kf[ks < KREG ? ks : 0] : rows_at<D>(own_rows, BKW, ks);
                             return x;
                           },
                           [&](int k, const Two& x) {
                             f32x16& acc = k & 1 ? pacc : sacc;
                             acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x.q, x.own, acc, 0, 0, 0);
                           });
      list_scores(sacc, pacc, lds.l[st] + par * 32 + 4 * g, lds.d[st] + par * 32 + 4 * g, lds.t[st] + par * 32 + 4 * g, f.scale_log2, masked, key);
      const bf16x8 pf[2] = {pack_acc<0>(sacc), pack_acc<1>(sacc)}, dsf[2] = {pack_acc<0>(pacc), pack_acc<1>(pacc)};
      pipelined<4 * DT, 2>([&](int k) { return cols_at<D>(qc, (k & 1 ? 0 : BLK) + k / (2 * DT) * 16, k / 2 % DT); },
                           [&](int k, const bf16x8& x) {
                             const int dt = k / 2 % DT, u = k / (2 * DT);
                             f32x16& acc = k & 1 ? dkacc[dt] : dvacc[dt];
                             acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k & 1 ? dsf[u] : pf[u], x, acc, 0, 0, 0);
                           });
    }
    if (n + 1 < n_it) store_numbers(n + 1, st ^ 1);
    wait_loads_and_barrier();
  }
  // the two halves' sums, dV first: the odd one hands over through LDS (64 KiB, all block tiles are free)
  const bool only = single_piece(a, mm, it.block);
  float* xch = (float*)&lds.block[0][0][0] + rg * (DT * 16) * 64;
  float* to = a.key_rows + (((long long)matrix * a.most[1] + item) * (a.block / BLK) + tile * 2 + (rg >> 1)) * (2 * BLK * D) + (rg & 1) * 32 * D;
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
    if (par == 0) {
#pragma unroll
      for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[dt][r] += xch[(dt * 16 + r) * 64 + lane];
      if (which == 0) key_sums<D>(a, m, acc, k0, 2 * D, 1.0f, only, xch, to + BLK * D, lane);
      else key_sums<D>(a, m, acc, k0, D, f.scale, only, xch, to, lane);
    }
  }
}

// Sums over a key's pieces, in the order of the lists, to dK and dV; zeros where there is none.  (A single piece is written by its workgroup.)
// A half-wavefront has four of a workgroup's 32 keys, which are of one block: with eight keys a workgroup 30 us to find single pieces for most of
// 200000 keys, where few workgroups had anything to add.
template <int D>
__global__ __launch_bounds__(256) void selected_dkv_combine_kernel(SelectedArgs a) {
  constexpr int DT = D / 32, KEYS = 4;
  typedef typename RowPart<DT>::V V;
  __shared__ __attribute__((aligned(16))) float lds[8][D];
  const FusedArgs& f = a.f;
  const int half = threadIdx.x >> 5, n = threadIdx.x & 31;
  const int mm = a.mat0 + blockIdx.y, key0 = blockIdx.x * (8 * KEYS);
  const SelMatrix m = selected_matrix<D>(a, mm);
  const int v = key0 / a.block, tiles = a.block / BLK;
  const int* first = a.first_item + ((long long)a.mats + mm) * (a.blocks + 1);
  const int from = first[v], to = first[v + 1];
  const bool single = to - from == 1;
  if (single && min(key0 + 8 * KEYS, f.s) <= m.len) return;
  V dk[KEYS], dv[KEYS];
#pragma unroll
  for (int u = 0; u < KEYS; ++u)
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) dk[u][dt] = dv[u][dt] = 0.f;
  const int in_block = key0 - v * a.block + half;
  if (!single) {   // (rows past the end of the sequence are not written: read, and not used)
    for (int k = from; k < to; ++k) {
      const float* p = a.key_rows + (((long long)blockIdx.y * a.most[1] + k) * tiles + in_block / BLK) * (2 * BLK * D) + in_block % BLK * D + n * DT;
#pragma unroll
      for (int u = 0; u < KEYS; ++u) {
        dk[u] += *(const V*)(p + u * 8 * D);
        dv[u] += *(const V*)(p + BLK * D + u * 8 * D);
      }
    }
  }
#pragma unroll
  for (int u = 0; u < KEYS; ++u) {
    const int key = key0 + u * 8 + half;
    const bool write = key < f.s && (key >= m.len || !single);
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) {
      dk[u][dt] = key < m.len ? dk[u][dt] * f.scale : 0.f;
      dv[u][dt] = key < m.len ? dv[u][dt] : 0.f;
    }
    bf16_t* out = f.d_qkv + m.qkv + (long long)key * f.ld + D;
    write_row<DT>(out, dk[u], lds[half], n, write);
    write_row<DT>(out + D, dv[u], lds[half], n, write);
  }
}

template <int D, int KEYS>
void launch_joint(const SelectedArgs& a, hipStream_t st) {
  typedef SelectedBwd<D, KEYS> B;
  constexpr int lds = sizeof(typename B::Lds);
  if (lds > 65536) (void)hipFuncSetAttribute((const void*)selected_bwd_kernel<D, KEYS>, hipFuncAttributeMaxDynamicSharedMemorySize, lds);
  selected_bwd_kernel<D, KEYS><<<a.most[1] * a.portion, B::THREADS, lds, st>>>(a);
}
template <int D>
int bwd_launch(SelectedArgs a, const SelectedPlan& p, hipStream_t st) {
  const int s = a.f.s;
  if (p.joint) {
    for (a.mat0 = 0; a.mat0 < p.mats; a.mat0 += p.portion) {
      a.portion = min(p.portion, p.mats - a.mat0);
      if (a.block == 64) launch_joint<D, 64>(a, st);
      else launch_joint<D, 128>(a, st);
      launch_selected_dq_combine(a, D, true, st);
      selected_dkv_combine_kernel<D><<<dim3((s + 31) / 32, a.portion), 256, 0, st>>>(a);
      if (const int rc = hip_launch_status()) return rc;
    }
    return OPTIMUS_OK;
  }
  for (a.mat0 = 0; a.mat0 < p.mats; a.mat0 += p.portion) {
    a.portion = min(p.portion, p.mats - a.mat0);
    selected_dq_kernel<D><<<a.most[0] * a.portion, 256, 0, st>>>(a);
    launch_selected_dq_combine(a, D, false, st);
    if (const int rc = hip_launch_status()) return rc;
  }
  for (a.mat0 = 0; a.mat0 < p.mats; a.mat0 += p.key_portion) {
    const int portion = a.portion = min(p.key_portion, p.mats - a.mat0);
    bool wide = false;
    if constexpr (D == 128) wide = a.block % 128 == 0;
    if (wide) selected_dkv_wide_kernel<<<a.most[1] * (a.block / 128) * portion, 512, 0, st>>>(a);
    else selected_dkv_kernel<D><<<a.most[1] * (a.block / BLK) * portion, 256, 0, st>>>(a);
    selected_dkv_combine_kernel<D><<<dim3((s + 31) / 32, portion), 256, 0, st>>>(a);
    if (const int rc = hip_launch_status()) return rc;
  }
  return OPTIMUS_OK;
}

}  // namespace

int launch_selected_bwd_kernels(const SelectedArgs& a, const SelectedPlan& p, int d, hipStream_t st) {
  return d == 64 ? bwd_launch<64>(a, p, st) : bwd_launch<128>(a, p, st);
}

}  // namespace optimus
