// The choice of blocks for the attention over chosen blocks (attention_selected_kernel.hpp): mean keys, scores, the best of a row.
//
// The choice is that of exact scores, q . mean with both as the bf16 numbers they are; equal scores: the lower block.  The matrix cores give
// scores that are off by at most E = d 2^-23 |q| |mean| (a rounding of the running sum per product), which decides all but a few
// rows in a thousand: with x the K-th largest such score, what is above x + 2E is chosen, what is below x - 2E is not, and where more than
// the places left lie between, their scores are computed again in 64 bits (products of bf16 numbers and their sums are exact there,
// unless they span more than 2^37).
//
// A workgroup has 32 queries of one block: its wavefronts share the blocks' scores out among them, 32 at a time, into LDS, then eight lanes
// have a query each, an eighth of its scores in registers, and find a threshold with K scores above it by halving.
// Bound: arithmetic and the waits between its steps.  8 (sequence, head)s of 32768 x 128, 16 of 256 blocks: 160 us, the vector units at work half of them:
// scores some 60, the search (eleven rounds of two operations a score; a secant's nine cost as much) 30, bounds and thresholds 20, exact scores
// and output 45.  16 of 4096 x 128, 8 of 32 blocks: 18.  The means, a pass over the keys, 18 (3.7 TB/s) and 6.
#include "attention_selected_kernel.hpp"

namespace optimus {
namespace {

// Mean keys, a workgroup a block: a lane has 8 columns of every (256 / (d / 8))-th row.  Sums in 64 bits: their bf16 rounding does not depend on
// the order then.
template <int D>
__global__ __launch_bounds__(256) void block_means_kernel(SelectedArgs a) {
  constexpr int CH = D / 8, ROWS = 256 / CH;
  __shared__ double parts[3][D];
  const FusedArgs& f = a.f;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int v = blockIdx.x, mm = blockIdx.y;
  const SelMatrix m = selected_matrix<D>(a, mm);
  const int row0 = v * a.block, rows = min(a.block, m.len - row0);
  if (rows <= 0) return;
  const bf16_t* p = f.qkv + m.qkv + D + (long long)row0 * f.ld + lane % CH * 8;
  double sum[8];
#pragma unroll
  for (int k = 0; k < 8; ++k) sum[k] = 0.0;
#pragma unroll 4
  for (int r = tid / CH; r < rows; r += ROWS) {
    const u32x4 w = *(const u32x4*)(p + (long long)r * f.ld);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      sum[2 * k] += (double)__uint_as_float(w[k] << 16);
      sum[2 * k + 1] += (double)__uint_as_float(w[k] & 0xffff0000u);
    }
  }
#pragma unroll
  for (int k = 0; k < 8; ++k)
#pragma unroll
    for (int step = CH; step < 64; step <<= 1) sum[k] += __shfl_xor(sum[k], step);
  if (wave > 0 && lane < CH) {
#pragma unroll
    for (int k = 0; k < 8; ++k) parts[wave - 1][lane * 8 + k] = sum[k];
  }
  __syncthreads();
  if (wave > 0) return;
  float mean[8], size = 0.f;
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    const int c = lane % CH * 8 + k;
    sum[k] += parts[0][c] + parts[1][c] + parts[2][c];
    mean[k] = bf16_to_f32(f32_to_bf16((float)(sum[k] / rows)));
    size = fmaf(mean[k], mean[k], size);
  }
#pragma unroll
  for (int step = 1; step < CH; step <<= 1) size += __shfl_xor(size, step);
  const long long at = (long long)mm * a.blocks + v;
  if (lane < CH) {
    u32x4 w;
#pragma unroll
    for (int k = 0; k < 4; ++k) w[k] = pack2_bf16(mean[2 * k], mean[2 * k + 1]);
    *(u32x4*)(a.means + at * D + lane * 8) = w;
  }
  if (lane == 0) a.mean_sizes[at] = sqrtf(size) * 1.0001f;
}

// sums and the like over the eight lanes of a query, in all of them: neighbours, pairs, then the other four mirrored (data-parallel moves, no
// trips to LDS)
template <int CTRL>
__device__ __forceinline__ int moved(int x) { return __builtin_amdgcn_update_dpp(0, x, CTRL, 0xf, 0xf, false); }
template <int CTRL>
__device__ __forceinline__ float moved(float x) { return __uint_as_float((unsigned)moved<CTRL>((int)__float_as_uint(x))); }
template <int CTRL>
__device__ __forceinline__ double moved(double x) {
  const long long b = __double_as_longlong(x);
  const unsigned lo = (unsigned)moved<CTRL>((int)b), hi = (unsigned)moved<CTRL>((int)(b >> 32));
  return __longlong_as_double((long long)((unsigned long long)hi << 32 | lo));
}
template <int CTRL>
__device__ __forceinline__ unsigned moved(unsigned x) { return (unsigned)moved<CTRL>((int)x); }
template <class T, class F>
__device__ __forceinline__ T eight(T x, F f) {
  x = f(x, moved<0xB1>(x));
  x = f(x, moved<0x4E>(x));
  return f(x, moved<0x141>(x));
}
__device__ __forceinline__ int sum8(int x) { return eight(x, [](int p, int q) { return p + q; }); }
__device__ __forceinline__ float min8(float x) { return eight(x, [](float p, float q) { return fminf(p, q); }); }
__device__ __forceinline__ float max8(float x) { return eight(x, [](float p, float q) { return fmaxf(p, q); }); }

constexpr int kRows = 32;             // queries of a workgroup

// LDS: kept scores [kRows][kept], scores [kRows][stride], bits of chosen and of contested blocks [kRows][words], largest mean of each
// wavefront's blocks [4], rows with scores that are not finite, kept blocks [kRows][kept]
__host__ __device__ inline int score_stride(int blocks) { return (blocks + 63) / 64 * 64 + 4; }
__host__ __device__ inline int bit_words(int blocks) { return (blocks + 31) / 32; }
inline size_t select_lds(int blocks, int count) {
  return (size_t)kRows * (score_stride(blocks) * 4 + bit_words(blocks) * 8 + count * 10) + 32;
}

// NV: scores of a lane, 4 of every 32 blocks; 8 NV blocks at most.
template <int D, int NV>
__global__ __launch_bounds__(256) void select_kernel(SelectedArgs a) {
  constexpr int KS = D / 16, PART = NV < 8 ? NV : 8;   // (loops over the scores go in parts of 64 blocks, of which the front of a sequence has few)
  extern __shared__ __attribute__((aligned(16))) char dynamic[];
  const FusedArgs& f = a.f;
  const int tid = threadIdx.x, lane = tid & 63, g = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int mm = blockIdx.y, q0 = blockIdx.x * kRows;
  const SelMatrix m = selected_matrix<D>(a, mm);
  const int own = q0 / a.block;                       // (blocks are multiples of 64 keys)
  const int have = (m.len + a.block - 1) / a.block;   // blocks with keys
  const int others = a.causal ? min(own, have) : have;   // candidates, the own block among them without a mask
  const int K = a.count - 1;
  const int stride = score_stride(a.blocks), words = bit_words(a.blocks);
  double* kept = (double*)dynamic;
  float* scores = (float*)(kept + kRows * a.count);
  unsigned* bits = (unsigned*)(scores + kRows * stride);
  unsigned* contested = bits + kRows * words;
  float* sizes = (float*)(contested + kRows * words);
  unsigned* wild_rows = (unsigned*)(sizes + 4);
  unsigned short* kept_block = (unsigned short*)(wild_rows + 4);
  const int row = tid >> 3, e = tid & 7, t = q0 + row;   // eight lanes a query
  int* out = a.chosen + (m.vec + t) * a.count;
  const bool query = t < m.len;
  const int eligible = a.causal ? others : others - 1;
  if (K == 0 || eligible <= K || q0 >= m.len) {   // (a workgroup's queries are of one block) the own one, or all of them
    if (t < f.s) {
      const int n = !query ? 0 : K == 0 ? 1 : eligible + 1, first = K == 0 ? own : 0;
      for (int k = e; k < a.count; k += 8) out[k] = k < n ? first + k : -1;
    }
    return;
  }
  // (one wait for the workgroup: everything that is loaded is on its way before it)
  for (int k = tid; k < kRows * words; k += 256) contested[k] = 0;
  float mean_size = 0.f, q_size = 0.f;
  for (int v = tid; v < others; v += 256) mean_size = fmaxf(mean_size, a.mean_sizes[(long long)mm * a.blocks + v]);
  const bf16_t* Q = f.qkv + m.qkv + (long long)min(t, m.len - 1) * f.ld + e * (D / 8);
  u32x4 qw[D / 64];
#pragma unroll
  for (int k = 0; k < D / 64; ++k) qw[k] = *(const u32x4*)(Q + 8 * k);
  // Scores, 32 blocks a wavefront at a time; of no candidate: NaN, which is neither above nor below a threshold, largest nor least.
  {
    const int qrow = min(q0 + (lane & 31), m.len - 1);
    const bf16_t* P = f.qkv + m.qkv + (long long)qrow * f.ld + g * 8;
    bf16x8 qf[KS];
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) qf[ks] = *(const bf16x8*)(P + ks * 16);
    const bf16_t* means = a.means + (long long)mm * a.blocks * D;
    unsigned long long bad = 0;
    const int end = (others + 8 * PART - 1) / (8 * PART) * (8 * PART);
    bf16x8 mf[KS];   // (the next 32 means are on their way while these are used)
    auto load_means = [&](int v0) {
      const bf16_t* p = means + (long long)min(v0 + (lane & 31), others - 1) * D + g * 8;
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) mf[ks] = *(const bf16x8*)(p + ks * 16);
    };
    load_means(wave * 32);
    for (int v0 = wave * 32; v0 < end; v0 += 128) {
      f32x16 acc = zero16();
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(mf[ks], qf[ks], acc, 0, 0, 0);
      load_means(v0 + 128);
      float zero = 0.f;
#pragma unroll
      for (int r = 0; r < 16; ++r) zero = fmaf(acc[r], 0.f, zero);   // (an infinity or NaN: NaN)
      bad |= __builtin_amdgcn_ballot_w64(!(zero == 0.f));
      if (v0 + 32 > others || (own >= v0 && own < v0 + 32)) {
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const int v = v0 + slot(r) + 4 * g;
          acc[r] = v < others && v != own ? acc[r] : NAN;
        }
      }
#pragma unroll
      for (int c = 0; c < 4; ++c)
        *(float4*)(scores + (lane & 31) * stride + v0 + 8 * c + 4 * g) = make_float4(acc[4 * c], acc[4 * c + 1], acc[4 * c + 2], acc[4 * c + 3]);
    }
    if (lane == 0) wild_rows[wave] = (unsigned)bad | (unsigned)(bad >> 32);
  }
  // E of the row: a query's size by its eight lanes, the largest mean by the workgroup
#pragma unroll
  for (int step = 1; step < 64; step <<= 1) mean_size = fmaxf(mean_size, __shfl_xor(mean_size, step));
  if (lane == 0) sizes[wave] = mean_size;
  float q[D / 8];
#pragma unroll
  for (int k = 0; k < D / 8; ++k) {
    const unsigned w = qw[k / 8][k / 2 % 4];
    q[k] = __uint_as_float(k & 1 ? w & 0xffff0000u : w << 16);
    q_size = fmaf(q[k], q[k], q_size);
  }
  q_size = sqrtf(eight(q_size, [](float p, float q) { return p + q; })) * 1.0001f;
  __syncthreads();
  mean_size = fmaxf(fmaxf(sizes[0], sizes[1]), fmaxf(sizes[2], sizes[3]));
  const float error = q_size * mean_size * (D * 1.1920929e-7f);
  // wild: a score or the bound is not finite, or too small for the bound: all scores are computed again
  const bool wild = !(error < 1e30f) || error < 1e-30f || q_size < 1e-25f || mean_size < 1e-25f || ((wild_rows[0] | wild_rows[1] | wild_rows[2] | wild_rows[3]) >> row & 1);
  // a lane's scores: of blocks 4 e + j of every 32
  const float* mine = scores + row * stride + 4 * e;
  float x[NV];
  float lo = INFINITY, hi = -INFINITY;
#pragma unroll
  for (int p = 0; p < NV; p += PART) {
    if (8 * p < others) {
#pragma unroll
      for (int k = p; k < p + PART; k += 4) {
        const float4 y = *(const float4*)(mine + 8 * k);
        x[k] = y.x;
        x[k + 1] = y.y;
        x[k + 2] = y.z;
        x[k + 3] = y.w;
      }
#pragma unroll
      for (int k = p; k < p + PART; ++k) {
        lo = fminf(lo, x[k]);
        hi = fmaxf(hi, x[k]);
      }
    } else {
#pragma unroll
      for (int k = p; k < p + PART; ++k) x[k] = NAN;
    }
  }
  lo = min8(lo);
  hi = max8(hi);
  // a threshold with K scores from it on: halving [lo, hi), from lo on at least K are (all), from hi fewer (a step above the largest)
  float cut = lo;
  bool found = wild || !query;
  hi += fabsf(hi) * 1e-6f + 1e-37f;
  for (int round = 0; round < 40 && __builtin_amdgcn_ballot_w64(!found) != 0; ++round) {
    const float middle = 0.5f * lo + 0.5f * hi;
    int n = 0;
#pragma unroll
    for (int p = 0; p < NV; p += PART)
      if (8 * p < others) {
#pragma unroll
        for (int k = p; k < p + PART; ++k) n += x[k] >= middle ? 1 : 0;
      }
    n = sum8(n);
    lo = !found && n >= K ? middle : lo;
    hi = !found && n < K ? middle : hi;
    cut = found ? cut : lo;
    found = found || n == K;
  }
  // The K-th score is the least from `cut` on.  Where K are from there on, and the next one is further away than both can be off together,
  // they are the choice.
  float least = INFINITY, next = -INFINITY;
#pragma unroll
  for (int p = 0; p < NV; p += PART)
    if (8 * p < others) {
#pragma unroll
      for (int k = p; k < p + PART; ++k) {
        least = fminf(least, x[k] >= cut ? x[k] : INFINITY);
        next = fmaxf(next, x[k] >= cut ? -INFINITY : x[k]);
      }
    }
  least = min8(least);
  next = max8(next);
  const bool separated = found && !wild;
  bool decided = separated && least - next > 2.0f * error;
  float above = (separated ? least : hi) + 2.0f * error, below = least - 2.0f * error;
  int n_above = 0;
  if (__builtin_amdgcn_ballot_w64(query && !decided) != 0) {
    // Else what is above the K-th (or `hi`, where no threshold divides the scores) by twice the error is chosen, what is as far below the least
    // is not, and as many of the scores between as there are places left.
    if (wild) {
      above = INFINITY;
      below = -INFINITY;
    }
    int n_below = 0;   // scores from `below` on
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      const int v = 32 * (k >> 2) + 4 * e + (k & 3);
      const bool candidate = v < others && v != own;
      n_above += candidate && x[k] > above ? 1 : 0;
      n_below += candidate && !(x[k] < below) ? 1 : 0;
    }
    n_above = wild ? 0 : sum8(n_above);
    n_below = sum8(n_below);
    if (!decided && n_below == K) {
      decided = true;
      cut = below;
    }
    const bool open = query && !decided;
#pragma unroll
    for (int k = 0; k < NV; ++k) {   // the bits of what is left to the exact scores
      const int v = 32 * (k >> 2) + 4 * e + (k & 3);
      if (open && v < others && v != own && !(x[k] < below) && (wild || !(x[k] > above))) atomicOr(&contested[row * words + (v >> 5)], 1u << (v & 31));
    }
  }
  // The bits of what is chosen so far, from a threshold on (decided) or above one: four of a word each lane.
  {
    const float from = !query || wild ? NAN : decided ? cut : above;   // (NaN: none)
    const bool over = !decided;
#pragma unroll
    for (int w = 0; w < NV / 4; ++w) {
      unsigned word = 0;
      if (32 * w < others) {
#pragma unroll
        for (int j = 3; j >= 0; --j) word = 2 * word + (x[4 * w + j] >= from ? 1 : 0);
        if (over) {   // (what equals the threshold is contested)
          word = 0;
#pragma unroll
          for (int j = 3; j >= 0; --j) word = 2 * word + (x[4 * w + j] > from ? 1 : 0);
        }
        word = eight(word << (4 * e), [](unsigned p, unsigned q) { return p | q; });
      }
      if (own >> 5 == w && query) word |= 1u << (own & 31);
      if (e == 0 && w < words) bits[row * words + w] = word;
    }
  }
  __builtin_amdgcn_wave_barrier();
  if (__builtin_amdgcn_ballot_w64(query && !decided) != 0) {
    // exact scores, in the order of the blocks, the best ones kept: one that is not above the worst kept is out (equal: the lower block stays)
    const int places = query && !decided ? K - n_above : 0;
    double* best = kept + row * a.count;
    unsigned short* block_of = kept_block + row * a.count;
    int n = 0, worst_at = 0, word = -1;
    double worst = 0.0;
    unsigned left = 0;
    const bf16_t* means = a.means + (long long)mm * a.blocks * D + e * (D / 8);
    while (true) {   // a query's next block each, until none has one
      while (left == 0 && word + 1 < words) left = contested[row * words + ++word];
      const bool contest = left != 0;
      if (__builtin_amdgcn_ballot_w64(contest) == 0) break;
      const int v = contest ? word * 32 + __builtin_ctz(left) : 0;
      left &= left - 1;
      double score = 0.0;
#pragma unroll
      for (int k = 0; k < D / 64; ++k) {
        const u32x4 w = *(const u32x4*)(means + (long long)v * D + 8 * k);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          score += (double)q[8 * k + 2 * j] * (double)__uint_as_float(w[j] << 16);
          score += (double)q[8 * k + 2 * j + 1] * (double)__uint_as_float(w[j] & 0xffff0000u);
        }
      }
      score = eight(score, [](double p, double q) { return p + q; });
      if (score != score) score = -INFINITY;   // (a score that is no number is below all)
      if (contest && n < places) {
        if (e == 0) {
          best[n] = score;
          block_of[n] = (unsigned short)v;
        }
        ++n;
      } else if (contest && score > worst) {
        if (e == 0) {
          best[worst_at] = score;
          block_of[worst_at] = (unsigned short)v;
        }
      } else {
        continue;
      }
      __builtin_amdgcn_wave_barrier();
      if (n == places) {   // the worst kept: the lowest score, of equal ones the last block
        double w = INFINITY;
        int at = -1, of = -1;
        for (int k = e; k < n; k += 8) {
          const double y = best[k];
          const int b = block_of[k];
          if (at < 0 || y < w || (y == w && b > of)) {
            w = y;
            at = k;
            of = b;
          }
        }
#pragma unroll
        for (int step = 1; step < 8; step <<= 1) {
          const double y = __shfl_xor(w, step);
          const int other = __shfl_xor(at, step), b = __shfl_xor(of, step);
          if (other >= 0 && (at < 0 || y < w || (y == w && b > of))) {
            w = y;
            at = other;
            of = b;
          }
        }
        worst = w;
        worst_at = at;
      }
    }
    __builtin_amdgcn_wave_barrier();
    for (int k = e; k < n; k += 8) {
      const int v = block_of[k];
      atomicOr(&bits[row * words + (v >> 5)], 1u << (v & 31));
    }
    __builtin_amdgcn_wave_barrier();
  }
  // the row's blocks in order: a lane has a run of words, those of lower lanes come first
  if (t >= f.s) return;
  const int each = (words + 7) / 8, from = min(e * each, words), to = min(from + each, words);
  int n = 0;
  for (int w = from; w < to; ++w) n += __popc(bits[row * words + w]);
  int before = n;
#pragma unroll
  for (int step = 1; step < 8; step <<= 1) {
    const int y = __shfl_up(before, step, 8);
    if (e >= step) before += y;
  }
  const int all = __shfl(before, 7, 8);
  int k = before - n;
  for (int w = from; w < to; ++w)
    for (unsigned left = bits[row * words + w]; left; left &= left - 1) out[k++] = w * 32 + __builtin_ctz(left);
  for (int r = all + e; r < a.count; r += 8) out[r] = -1;
}

template <int D, int NV>
void select_launch(const SelectedArgs& a, int mats, hipStream_t st) {
  const size_t lds = select_lds(a.blocks, a.count);
  if (lds > 65536) (void)hipFuncSetAttribute((const void*)select_kernel<D, NV>, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
  select_kernel<D, NV><<<dim3((a.f.s + kRows - 1) / kRows, mats), 256, lds, st>>>(a);
}
template <int D>
void choose(const SelectedArgs& a, int mats, hipStream_t st) {
  // (every block is chosen, or the own one alone: no scores)
  if (a.count > 1 && a.count < a.blocks) block_means_kernel<D><<<dim3(a.blocks, mats), 256, 0, st>>>(a);
  if (a.blocks <= 32) select_launch<D, 4>(a, mats, st);
  else if (a.blocks <= 64) select_launch<D, 8>(a, mats, st);
  else if (a.blocks <= 128) select_launch<D, 16>(a, mats, st);
  else if (a.blocks <= 256) select_launch<D, 32>(a, mats, st);
  else if (a.blocks <= 512) select_launch<D, 64>(a, mats, st);
  else select_launch<D, 128>(a, mats, st);
  static_assert(kMostBlocks <= 8 * 128, "a lane's scores");
}

size_t round256(size_t x) { return (x + 255) & ~(size_t)255; }

}  // namespace

size_t attn_select_ws_bytes(const AttnSelectedDesc& b) {
  const AttnFusedDesc& d = b.base;
  const size_t means = (size_t)d.ndev * d.nb * d.nh * ((d.s + b.block - 1) / b.block);
  return round256(means * d.d * 2) + round256(means * 4);
}

int launch_attn_select(const AttnSelectedDesc& b, hipStream_t st) {
  const AttnFusedDesc& d = b.base;
  SelectedArgs a = {};
  a.f.qkv = (const bf16_t*)d.qkv;
  a.f.s = d.s; a.f.nh = d.nh; a.f.ld = d.ld; a.f.ldo = d.ldo;
  a.f.dev_qkv = d.dev_qkv; a.f.dev_attn = d.dev_attn;
  a.chosen = b.chosen; a.lengths = b.lengths;
  a.nb = d.nb; a.nmat = d.nb * d.nh; a.q = b.q; a.dev0 = b.dev0; a.causal = d.causal;
  a.block = b.block; a.count = b.count; a.blocks = (d.s + b.block - 1) / b.block;
  const int mats = d.ndev * a.nmat;
  a.means = (bf16_t*)b.ws;
  a.mean_sizes = (float*)((char*)b.ws + round256((size_t)mats * a.blocks * d.d * 2));
  if (d.d == 64) choose<64>(a, mats, st);
  else choose<128>(a, mats, st);
  return hip_launch_status();
}

}  // namespace optimus
