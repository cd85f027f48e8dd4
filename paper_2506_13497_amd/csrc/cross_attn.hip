// Cross-attention of packed requests: sequence b's queries (rows q_off[b] .. q_off[b+1]-1) attend to its own encoder states (rows
// kv_off[b] .. kv_off[b+1]-1, less those that a mask takes out):
//     o_i = sum_j p_ij v_j / sum_j p_ij,  p_ij = exp(scale q_i . k_j),  lse_i = log sum_j p_ij;  no state: o_i = 0, lse_i = -inf.
// H query heads share H_kv key heads in runs of H / H_kv.  Lengths are read on the device, so a captured launch serves others.
//
// Work split.  A row is a query of one head; the rows of a key head are (query, head of its group) in that order, so that grouped heads share
// the K and V tiles that are fetched.  A wavefront takes 32 rows, a workgroup a run of rows of one sequence and key head and all of the
// sequence's keys in tiles of 64, or a part of these tiles where rows are few (see cross_attn_parts): the parts' sums then meet in a second
// launch.  The host knows only the totals, so the grid has floor(rows / run) + B slots a key head, which is enough for any lengths, and a
// workgroup finds its sequence by summing up the runs of all of them, 64 at a time; slots left over end there.
//
// Matrix cores as in the dense attention: S^T = K Q^T (a lane owns one query and 16 of 32 keys), then O^T = V^T P^T with P^T, rounded to
// bf16, straight from the accumulators and V^T through the transposing LDS read.  The sums of P and O are fp32; P is rounded because the
// matrix instruction takes two operands of one type and V is bf16.  One running maximum a query, moved only when a score exceeds it by
// 2^8 in the exponent, so that most tiles rescale nothing.
//
// K and V tiles go through registers into two LDS stages in turn (one barrier a tile), because values of rows that a mask takes out, rows of
// other sequences and columns past the head dim have to be zeros: a weight of zero times an infinity would be NaN.
#include "ddit_common.hpp"

#include <algorithm>

namespace {

typedef unsigned int uintx4 __attribute__((ext_vector_type(4)));
typedef unsigned int uintx2 __attribute__((ext_vector_type(2)));
typedef short shortx4 __attribute__((ext_vector_type(4)));
typedef short shortx8 __attribute__((ext_vector_type(8)));
typedef __attribute__((address_space(3))) shortx4 *lds_s4_ptr_t;

constexpr int KT = 64;   // keys of a tile

struct CrossParams {
  const bf16_t *q, *k, *v;
  int64_t ld_q, ld_kv, ld_o;
  const int *q_off, *kv_off;
  const uint8_t *mask;
  int B, q_rows, kv_rows, H, group, dh;   // group: query heads of a key head
  float scale, scale_log2, rebase;        // log2(e) * scale; 8 / scale_log2
  bf16_t *o; float *lse;
  int run;                                // rows of a slot: a multiple of the kernel's row tile
  int parts;
  float *part_o, *part_ml;                // parts > 1: fp32 [parts][q_rows][H][dh] and [parts][q_rows][H][2] (maximum, sum)
};

// What slot `slot` of runs of `run` rows stands for: rows [begin, end) of a sequence that starts at query q_first, and its encoder states
// [kv_begin, kv_end); false: nothing.  Offsets outside the arrays are cut off there, and sums of runs stop at 2^30 (far past every slot), so that offsets that
// decrease lead nowhere outside either.
struct Slot { int q_first, begin, end, kv_begin, kv_end; };
__device__ __forceinline__ bool find_slot(const CrossParams &p, unsigned slot, int run, Slot &at) {
  const int lane = threadIdx.x & 63;
  unsigned before = 0;
  for (int b0 = 0; b0 < p.B; b0 += 64) {
    const int i = std::min(b0 + lane, p.B - 1);
    const int q0 = p.q_off[i], q1 = p.q_off[i + 1], k0 = p.kv_off[i], k1 = p.kv_off[i + 1];
    const int from = std::min(std::max(q0, 0), p.q_rows), to = std::min(std::max(q1, from), p.q_rows);
    const int rows = (to - from) * p.group;
    const unsigned runs = b0 + lane < p.B ? ((unsigned)rows + run - 1) / (unsigned)run : 0u;
    unsigned sum = runs;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const unsigned up = (unsigned)__shfl_up((int)sum, d, 64);
      if (lane >= d) sum = std::min(sum + up, 1u << 30);
    }
    const uint64_t past = __ballot(before + sum > slot);
    if (past) {
      const int who = __ffsll((unsigned long long)past) - 1;
      const unsigned ahead = before + (unsigned)__builtin_amdgcn_readlane((int)(sum - runs), who);   // runs of the sequences before
      at.q_first = __builtin_amdgcn_readlane(from, who);
      at.begin = (int)(slot - ahead) * run;
      at.end = std::min(at.begin + run, __builtin_amdgcn_readlane(rows, who));
      at.kv_begin = std::min(std::max(__builtin_amdgcn_readlane(k0, who), 0), p.kv_rows);
      at.kv_end = std::min(std::max(__builtin_amdgcn_readlane(k1, who), at.kv_begin), p.kv_rows);
      return true;
    }
    before += (unsigned)__builtin_amdgcn_readlane((int)sum, 63);
  }
  return false;
}

template <int KS, int ST_>
struct CrossCfg {
  static constexpr int ST = ST_;                     // LDS stages: key sequences of up to ST tiles are fetched once
  static constexpr int CH = 2 * KS;                  // 16-byte pieces of a K row: the head dim padded to 16 KS
  static constexpr int DT = (KS + 1) / 2;            // 32-row tiles of V^T
  static constexpr int KP = CH * 16 + 16;            // K row pitch: an odd number of pieces, so 16 rows lie in different banks
  static constexpr int VP = KS == 8 ? 320 : 192;     // V row pitch: an odd number of 64 bytes, so the four keys of a transposing read do
  static constexpr int VOFF = KT * KP;
  static constexpr int STAGE = KT * (KP + VP);
  static constexpr int SMEM = ST * STAGE + ST * 8;   // and the valid keys of every stage
  static_assert(DT * 64 <= VP && SMEM <= 160 * 1024, "a V row is read to the end of its last tile");
};

template <int KS, int NW, int ST>
__global__ __launch_bounds__(64 * NW) void k_cross_attn(CrossParams p) {
  using C = CrossCfg<KS, ST>;
  constexpr int QT = 32 * NW, CJ = (KT * C::CH + 64 * NW - 1) / (64 * NW);   // pieces of a tile that a thread stages
  extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, l32 = lane & 31, lh = lane >> 5;
  Slot slot;
  if (!find_slot(p, blockIdx.x, p.run, slot)) return;
  const int h0 = blockIdx.y * p.group;   // first of the key head's query heads
  const int n_keys = slot.kv_end - slot.kv_begin, all = (n_keys + KT - 1) / KT;
  const int t_begin = (int)((int64_t)all * blockIdx.z / p.parts), t_end = (int)((int64_t)all * (blockIdx.z + 1) / p.parts);
  const int n_tiles = t_end - t_begin, pieces = p.dh >> 3;

  bf16x8 qn[KS];   // the next row tile's fragments
  auto fetch_q = [&](int r0) {
    const int r = std::min(r0 + wave * 32 + l32, slot.end - 1), q = r / p.group;
    const bf16_t *row = p.q + (int64_t)(slot.q_first + q) * p.ld_q + (h0 + r - q * p.group) * p.dh;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
#pragma unroll
      for (int e = 0; e < 8; ++e) qn[ks][e] = (bf16_t)0.f;
      if (2 * ks + lh < pieces) qn[ks] = *reinterpret_cast<const bf16x8 *>(row + 16 * ks + 8 * lh);
    }
  };
  fetch_q(slot.begin);

  const int64_t kv_at = (int64_t)slot.kv_begin * p.ld_kv + blockIdx.y * p.dh;
  const bf16_t *const kbase = p.k + kv_at, *const vbase = p.v + kv_at;
  const uint8_t *const mask = p.mask ? p.mask + slot.kv_begin : nullptr;
  struct Pieces { uintx4 k[CJ], v[CJ]; uint64_t bits; };
  auto fetch = [&](int tile, Pieces &x) {
#pragma unroll
    for (int j = 0; j < CJ; ++j) {
      const int i = tid + 64 * NW * j, row = i / C::CH, c = i - row * C::CH, key = tile * KT + row;
      x.k[j] = x.v[j] = uintx4{0u, 0u, 0u, 0u};
      if (row < KT && c < pieces && key < n_keys) {
        x.k[j] = *reinterpret_cast<const uintx4 *>(kbase + (int64_t)key * p.ld_kv + c * 8);
        x.v[j] = *reinterpret_cast<const uintx4 *>(vbase + (int64_t)key * p.ld_kv + c * 8);
      }
    }
    const int key = tile * KT + lane;
    x.bits = __ballot(key < n_keys && (!mask || mask[key]));   // one bit a key
  };
  auto put = [&](int st, const Pieces &x) {
    unsigned char *const at = smem + st * C::STAGE;
#pragma unroll
    for (int j = 0; j < CJ; ++j) {
      const int i = tid + 64 * NW * j, row = i / C::CH, c = i - row * C::CH;
      if (row < KT) {
        *reinterpret_cast<uintx4 *>(at + row * C::KP + c * 16) = x.k[j];   // zeros past the head dim
        *reinterpret_cast<uintx4 *>(at + C::VOFF + row * C::VP + c * 16) = (x.bits >> row) & 1 ? x.v[j] : uintx4{0u, 0u, 0u, 0u};
      }
    }
    if (tid == 0) reinterpret_cast<uint64_t *>(smem + ST * C::STAGE)[st] = x.bits;
  };
  floatx16 o[C::DT];
  float m_run, l_run;
  bf16x8 qf[KS];
  // transposing reads: this lane supplies the 8 bytes of key tr_key at feature tr_d of a 16 keys x 32 features block
  const int tr = C::VOFF + (4 * lh + ((lane & 15) >> 2)) * C::VP + (16 * ((lane >> 4) & 1) + 4 * (lane & 3)) * 2;
  auto begin = [&]() {
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) qf[ks] = qn[ks];
#pragma unroll
    for (int d = 0; d < C::DT; ++d)
#pragma unroll
      for (int e = 0; e < 16; ++e) o[d][e] = 0.f;
    m_run = -INFINITY; l_run = 0.f;
  };
  auto step = [&](int st) {
    const unsigned char *const at = smem + st * C::STAGE;
    floatx16 s[2];
#pragma unroll
    for (int kt = 0; kt < 2; ++kt) {
#pragma unroll
      for (int e = 0; e < 16; ++e) s[kt][e] = 0.f;
#pragma unroll
      for (int ks = 0; ks < KS; ++ks)
        s[kt] = mfma32(*reinterpret_cast<const bf16x8 *>(at + (kt * 32 + l32) * C::KP + (2 * ks + lh) * 16), qf[ks], s[kt]);
    }
    const uint64_t bits = reinterpret_cast<const uint64_t *>(smem + ST * C::STAGE)[st];
    const unsigned lo_bits = (unsigned)__builtin_amdgcn_readfirstlane((int)(unsigned)bits);
    const unsigned hi_bits = (unsigned)__builtin_amdgcn_readfirstlane((int)(unsigned)(bits >> 32));
    if ((lo_bits & hi_bits) != ~0u) {
#pragma unroll
      for (int kt = 0; kt < 2; ++kt) {
        const unsigned w = (kt ? hi_bits : lo_bits) >> (4 * lh);
#pragma unroll
        for (int e = 0; e < 16; ++e) s[kt][e] = (w >> (8 * (e >> 2) + (e & 3))) & 1u ? s[kt][e] : -INFINITY;
      }
    }
    float mx = s[0][0];
#pragma unroll
    for (int e = 1; e < 16; ++e) mx = fmaxf(mx, s[0][e]);
#pragma unroll
    for (int e = 0; e < 16; ++e) mx = fmaxf(mx, s[1][e]);
    mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
    const bool move = mx > m_run + p.rebase;
    if (__ballot(move)) {
      const float alpha = move ? __builtin_amdgcn_exp2f((m_run - mx) * p.scale_log2) : 1.f;   // 0 the first time
      if (move) m_run = mx;
      l_run *= alpha;
#pragma unroll
      for (int d = 0; d < C::DT; ++d)
#pragma unroll
        for (int e = 0; e < 16; ++e) o[d][e] *= alpha;
    }
    const float ref = m_run == -INFINITY ? 0.f : m_run * p.scale_log2;
    bf16x8 pf[4];
    float sum = 0.f;
#pragma unroll
    for (int kt = 0; kt < 2; ++kt)
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const float w = __builtin_amdgcn_exp2f(__builtin_fmaf(s[kt][e], p.scale_log2, -ref));
        sum += w;
        pf[2 * kt + (e >> 3)][e & 7] = (bf16_t)w;
      }
    l_run += sum;
#pragma unroll
    for (int kc = 0; kc < 4; ++kc)
#pragma unroll
      for (int d = 0; d < C::DT; ++d) {
        const unsigned char *const va = at + tr + kc * 16 * C::VP + d * 64;
        const shortx4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4_ptr_t)va);
        const shortx4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4_ptr_t)(va + 8 * C::VP));
        o[d] = mfma32(__builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7)), pf[kc], o[d]);
      }
  };
  auto finish = [&](int r0) {
    const int r = r0 + wave * 32 + l32, q = r / p.group, h = h0 + r - q * p.group;
    const bool in = r < slot.end;
    const int64_t token = slot.q_first + q;
    l_run += __shfl_xor(l_run, 32, 64);
    if (p.parts > 1) {
      if (in) {
        const int64_t at = (blockIdx.z * (int64_t)p.q_rows + token) * p.H + h;
#pragma unroll
        for (int d = 0; d < C::DT; ++d)
#pragma unroll
          for (int g = 0; g < 4; ++g) {
            const int col = 32 * d + 8 * g + 4 * lh;
            if (col < p.dh) {
              floatx4 v;
#pragma unroll
              for (int e = 0; e < 4; ++e) v[e] = o[d][4 * g + e];
              *reinterpret_cast<floatx4 *>(p.part_o + at * p.dh + col) = v;
            }
          }
        if (lh == 0) *reinterpret_cast<float2 *>(p.part_ml + 2 * at) = make_float2(m_run, l_run);
      }
      return;
    }
    const float inv = l_run == 0.f ? 0.f : 1.f / l_run;
    bf16_t *const orow = p.o + token * p.ld_o + h * p.dh;
#pragma unroll
    for (int d = 0; d < C::DT; ++d)
#pragma unroll
      for (int g = 0; g < 4; g += 2) {
        // lanes l and l ^ 32 hold the two halves of 8 features each: the lower lane collects those of group g, the upper those of g + 1
        bf16x4 x0, x1;
#pragma unroll
        for (int e = 0; e < 4; ++e) { x0[e] = (bf16_t)(o[d][4 * g + e] * inv); x1[e] = (bf16_t)(o[d][4 * g + 4 + e] * inv); }
        const uintx2 own = __builtin_bit_cast(uintx2, lh ? x1 : x0), give = __builtin_bit_cast(uintx2, lh ? x0 : x1);
        uintx2 got;
        got[0] = (unsigned)__shfl_xor((int)give[0], 32, 64);
        got[1] = (unsigned)__shfl_xor((int)give[1], 32, 64);
        const uintx4 v = lh ? uintx4{got[0], got[1], own[0], own[1]} : uintx4{own[0], own[1], got[0], got[1]};
        const int col = 32 * d + 8 * (g + lh);
        if (in && col < p.dh) *reinterpret_cast<uintx4 *>(orow + col) = v;
      }
    if (p.lse && lh == 0 && in)
      p.lse[token * p.H + h] = l_run == 0.f ? -INFINITY : __builtin_fmaf(m_run, p.scale, __builtin_amdgcn_logf(l_run) * 0.6931471805599453f);
  };

  if (n_tiles <= ST) {
    // everything is fetched once, and the workgroup walks over its row tiles with no further barrier
    {
      Pieces x[ST];
#pragma unroll
      for (int t = 0; t < ST; ++t)
        if (t < n_tiles) fetch(t_begin + t, x[t]);
#pragma unroll
      for (int t = 0; t < ST; ++t)
        if (t < n_tiles) put(t, x[t]);
    }
    __syncthreads();
    for (int r0 = slot.begin; r0 < slot.end; r0 += QT) {
      begin();
      if (r0 + QT < slot.end) fetch_q(r0 + QT);
      if (r0 + wave * 32 >= slot.end) break;   // a wavefront without rows, in the run's last tile
      for (int t = 0; t < n_tiles; ++t) step(t);
      finish(r0);
    }
  } else {
    for (int r0 = slot.begin; r0 < slot.end; r0 += QT) {
      Pieces x;
      begin();
      if (r0 + QT < slot.end) fetch_q(r0 + QT);
      fetch(t_begin, x);
      if (r0 != slot.begin) __syncthreads();   // the tiles of the rows before are done with
      put(0, x);
      __syncthreads();
      for (int t = 0; t < n_tiles; ++t) {
        if (t + 1 < n_tiles) fetch(t_begin + t + 1, x);
        step(t & 1);
        if (t + 1 < n_tiles) put((t + 1) & 1, x);
        __syncthreads();
      }
      finish(r0);
    }
  }
}

// The parts' sums of 4 rows of a key head meet, a wavefront a row: a lane looks after one part's maximum and sum first, then after two
// features.  A part without weight is left out (its place in part_o may hold anything).
__global__ __launch_bounds__(256) void k_cross_join(CrossParams p) {
  Slot slot;
  if (!find_slot(p, blockIdx.x, 4, slot)) return;
  const int lane = threadIdx.x & 63, r = slot.begin + (threadIdx.x >> 6), q = r / p.group;
  if (r >= slot.end) return;
  const int h = blockIdx.y * p.group + r - q * p.group;
  const int64_t token = slot.q_first + q, step = (int64_t)p.q_rows * p.H, at = token * p.H + h;
  float2 ml = make_float2(-INFINITY, 0.f);
  if (lane < p.parts) ml = reinterpret_cast<const float2 *>(p.part_ml)[at + lane * step];
  float top = ml.x;
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) top = fmaxf(top, __shfl_xor(top, d, 64));
  const float weight = ml.y == 0.f ? 0.f : __builtin_amdgcn_exp2f((ml.x - top) * p.scale_log2);
  const float l = wave_sum(ml.y * weight), inv = l == 0.f ? 0.f : 1.f / l;
  const int c = std::min(2 * lane, p.dh - 2);
  float2 a = make_float2(0.f, 0.f);

  for (int z = 0; z < p.parts; ++z) {
    const float w = __uint_as_float((unsigned)__builtin_amdgcn_readlane((int)__float_as_uint(weight), z));
    const float2 v = *reinterpret_cast<const float2 *>(p.part_o + (at + z * step) * p.dh + c);
    a.x += w == 0.f ? 0.f : v.x * w;
    a.y += w == 0.f ? 0.f : v.y * w;
  }
  if (2 * lane < p.dh) {
    bf16x2 v;
    v[0] = (bf16_t)(a.x * inv); v[1] = (bf16_t)(a.y * inv);
    *reinterpret_cast<bf16x2 *>(p.o + token * p.ld_o + h * p.dh + c) = v;
  }
  if (p.lse && lane == 0) p.lse[at] = l == 0.f ? -INFINITY : __builtin_fmaf(top, p.scale, __builtin_amdgcn_logf(l) * 0.6931471805599453f);
}

template <int KS, int NW, int ST>
int launch_as(const CrossParams &p, hipStream_t s) {
  constexpr int smem = CrossCfg<KS, ST>::SMEM;
  static std::atomic<uint64_t> allowed;
  const int rc = ddit::allow_dynamic_lds(reinterpret_cast<const void *>(&k_cross_attn<KS, NW, ST>), smem, &allowed);
  if (rc != 0) return rc;
  const unsigned slots = (unsigned)((int64_t)p.q_rows * p.group / p.run + p.B);
  hipLaunchKernelGGL((k_cross_attn<KS, NW, ST>), dim3(slots, (unsigned)(p.H / p.group), (unsigned)p.parts), dim3(64 * NW), smem, s, p);
  return ddit::hip_fail(hipGetLastError(), "packed cross-attention launch");
}
template <int KS>
int launch_form(int waves, const CrossParams &p, hipStream_t s) {
  if (waves == 1) return launch_as<KS, 1, 2>(p, s);
  if (waves == 4) return launch_as<KS, 4, 2>(p, s);
  return launch_as<KS, 8, KS == 8 ? 4 : 5>(p, s);
}

// Wavefronts of a workgroup, for `rows` rows a key head
int waves_for(int B, int64_t rows, int H_kv) {
  if (rows <= (int64_t)64 * B) return 1;
  return (rows / 256 + B) * H_kv >= 1024 ? 8 : 4;
}

}  // namespace

namespace ddit {

// From the totals alone, since the lengths are on the device, and for the whole chip whatever device is current, since the answer sizes workspaces.
int cross_attn_parts(int B, int64_t q_rows, int64_t kv_rows, int H, int H_kv) {
  const int64_t rows = q_rows * (H / H_kv), units = (rows / (32 * waves_for(B, rows, H_kv)) + B) * H_kv;
  return (int)std::max<int64_t>(1, std::min<int64_t>({(int64_t)32, 1024 / units, kv_rows / 128}));
}

int launch_cross_attn(const CrossAttnArgs &a, hipStream_t s) {
  if (a.q_rows == 0) return 0;
  CrossParams p;
  p.q = reinterpret_cast<const bf16_t *>(a.q); p.k = reinterpret_cast<const bf16_t *>(a.k); p.v = reinterpret_cast<const bf16_t *>(a.v);
  p.ld_q = a.ld_q; p.ld_kv = a.ld_kv; p.ld_o = a.ld_o; p.q_off = a.q_off; p.kv_off = a.kv_off; p.mask = a.mask;
  p.B = a.B; p.q_rows = (int)a.q_rows; p.kv_rows = (int)a.kv_rows; p.H = a.H; p.group = a.H / a.H_kv; p.dh = a.dh;
  p.scale = a.scale; p.scale_log2 = a.scale * 1.4426950408889634f; p.rebase = 8.f / p.scale_log2;
  p.o = reinterpret_cast<bf16_t *>(a.o); p.lse = a.lse;
  p.parts = cross_attn_parts(a.B, a.q_rows, a.kv_rows, a.H, a.H_kv);
  p.part_o = a.scratch;
  p.part_ml = p.parts > 1 ? a.scratch + (int64_t)p.parts * a.q_rows * a.H * a.dh : nullptr;
  const int64_t rows = a.q_rows * p.group;
  const int waves = waves_for(a.B, rows, a.H_kv);
  p.run = 32 * waves;
  if (waves == 8) p.run *= (int)std::max<int64_t>(1, std::min<int64_t>(8, rows * a.H_kv / (256 * 4 * device_cus())));
  const int rc = p.dh <= 64 ? launch_form<4>(waves, p, s) : p.dh <= 80 ? launch_form<5>(waves, p, s) : p.dh <= 96 ? launch_form<6>(waves, p, s)
                                                                                                              : launch_form<8>(waves, p, s);
  if (rc != 0 || p.parts == 1) return rc;
  hipLaunchKernelGGL(k_cross_join, dim3((unsigned)(rows / 4 + p.B), (unsigned)a.H_kv), dim3(256), 0, s, p);
  return hip_fail(hipGetLastError(), "packed cross-attention join");
}

}  // namespace ddit
