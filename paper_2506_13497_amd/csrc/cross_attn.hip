// Cross-attention of packed requests: sequence b's queries (rows q_off[b] .. q_off[b+1]-1) attend to its own encoder states (rows
// kv_off[b] .. kv_off[b+1]-1, less those that a mask takes out):
//     o_i = sum_j p_ij v_j / sum_j p_ij,  p_ij = exp(scale q_i . k_j),  lse_i = log sum_j p_ij;  no state: o_i = 0, lse_i = -inf.
// H query heads share H_kv key heads in runs of H / H_kv.  Lengths are read on the device, so a captured launch serves others.
//
// Work split.  A workgroup takes QT = 32 NW queries of one sequence and head, a wavefront 32 of them, and all of the sequence's keys
// in tiles of 64, or a part of these tiles where queries are few (see launch): the parts' sums then meet in a second launch.  The host knows
// only the total of the rows, so the grid has floor(q_rows / QT) + B slots a head, which is enough for any lengths, and a workgroup finds
// its sequence by summing up the tiles of all of them, 64 at a time; slots left over end there.
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
  int parts;
  float *part_o, *part_ml;                // parts > 1: fp32 [parts][q_rows][H][dh] and [parts][q_rows][H][2] (maximum, sum)
};

// Sequence, first query and end of the queries of tile `slot`, with QT queries a tile; false: there is none.  Offsets outside the arrays are
// cut off there, and sums of tiles stop at 2^30 (far past every slot), so that offsets that decrease lead nowhere outside either.
template <int QT>
__device__ __forceinline__ bool find_tile(const CrossParams &p, unsigned slot, int &b, int &q_begin, int &q_end) {
  const int lane = threadIdx.x & 63;
  unsigned before = 0;
  for (int b0 = 0; b0 < p.B; b0 += 64) {
    const int i = b0 + lane;
    int from = 0, to = 0;
    if (i < p.B) {
      from = std::min(std::max(p.q_off[i], 0), p.q_rows);
      to = std::min(std::max(p.q_off[i + 1], from), p.q_rows);
    }
    const unsigned tiles = (unsigned)(to - from + QT - 1) / QT;
    unsigned sum = tiles;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const unsigned up = (unsigned)__shfl_up((int)sum, d, 64);
      if (lane >= d) sum = std::min(sum + up, 1u << 30);
    }
    const uint64_t past = __ballot(before + sum > slot);
    if (past) {
      const int at = __ffsll((unsigned long long)past) - 1;
      const unsigned ahead = before + (unsigned)__shfl((int)(sum - tiles), at, 64);   // tiles of the sequences before
      b = b0 + at;
      q_begin = __shfl(from, at, 64) + (int)(slot - ahead) * QT;
      q_end = std::min(q_begin + QT, __shfl(to, at, 64));
      return true;
    }
    before += (unsigned)__shfl((int)sum, 63, 64);
  }
  return false;
}

template <int KS>
struct CrossCfg {
  static constexpr int CH = 2 * KS;                  // 16-byte pieces of a staged row: the head dim padded to 16 KS
  static constexpr int DT = (KS + 1) / 2;            // 32-row tiles of V^T
  static constexpr int KP = CH * 16 + 16;            // K row pitch: an odd number of pieces, so 16 rows lie in different banks
  static constexpr int VP = KS == 8 ? 320 : 192;     // V row pitch: an odd number of 64 bytes, so the four keys of a transposing read do
  static constexpr int VOFF = KT * KP;
  static constexpr int STAGE = KT * (KP + VP);
  static_assert(DT * 64 <= VP, "a V row is read to the end of its last tile");
};

template <int KS, int NW>
__global__ __launch_bounds__(64 * NW) void k_cross_attn(CrossParams p) {
  using C = CrossCfg<KS>;
  constexpr int QT = 32 * NW, CJ = (KT * C::CH + 64 * NW - 1) / (64 * NW);   // pieces of a tile that a thread stages
  extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, l32 = lane & 31, lh = lane >> 5;
  const int h = blockIdx.y;
  int b, q_begin, q_end;
  if (!find_tile<QT>(p, blockIdx.x, b, q_begin, q_end)) return;
  const int kv_begin = std::min(std::max(p.kv_off[b], 0), p.kv_rows);
  const int kv_end = std::min(std::max(p.kv_off[b + 1], kv_begin), p.kv_rows);
  const int all = (kv_end - kv_begin + KT - 1) / KT;
  const int t_begin = (int)((int64_t)all * blockIdx.z / p.parts), t_end = (int)((int64_t)all * (blockIdx.z + 1) / p.parts);
  const int pieces = p.dh >> 3;

  const int qi = q_begin + wave * 32 + l32;
  bf16x8 qf[KS];
  {
    const bf16_t *row = p.q + (int64_t)std::min(qi, q_end - 1) * p.ld_q + h * p.dh;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
#pragma unroll
      for (int e = 0; e < 8; ++e) qf[ks][e] = (bf16_t)0.f;
      if (2 * ks + lh < pieces) qf[ks] = *reinterpret_cast<const bf16x8 *>(row + 16 * ks + 8 * lh);
    }
  }

  const bf16_t *const kbase = p.k + (int64_t)kv_begin * p.ld_kv + (h / p.group) * p.dh;
  const bf16_t *const vbase = p.v + (int64_t)kv_begin * p.ld_kv + (h / p.group) * p.dh;
  const int n_keys = kv_end - kv_begin;
  const uint8_t *const mask = p.mask ? p.mask + kv_begin : nullptr;
  uintx4 kr[CJ], vr[CJ];
  auto fetch = [&](int tile) {
#pragma unroll
    for (int j = 0; j < CJ; ++j) {
      const int i = tid + 64 * NW * j, row = i / C::CH, c = i - row * C::CH, key = tile * KT + row;
      kr[j] = vr[j] = uintx4{0u, 0u, 0u, 0u};
      if (row < KT && c < pieces && key < n_keys) {
        kr[j] = *reinterpret_cast<const uintx4 *>(kbase + (int64_t)key * p.ld_kv + c * 8);
        vr[j] = *reinterpret_cast<const uintx4 *>(vbase + (int64_t)key * p.ld_kv + c * 8);
      }
    }
  };
  auto put = [&](int st, uint64_t valid) {
    unsigned char *const at = smem + st * C::STAGE;
#pragma unroll
    for (int j = 0; j < CJ; ++j) {
      const int i = tid + 64 * NW * j, row = i / C::CH, c = i - row * C::CH;
      if (row < KT) {
        *reinterpret_cast<uintx4 *>(at + row * C::KP + c * 16) = kr[j];
        *reinterpret_cast<uintx4 *>(at + C::VOFF + row * C::VP + c * 16) = (valid >> row) & 1 ? vr[j] : uintx4{0u, 0u, 0u, 0u};
      }
    }
  };
  // a wavefront's view of a tile: one bit a key
  auto keys_of = [&](int tile) {
    const int key = tile * KT + lane;
    return __ballot(key < n_keys && (!mask || mask[key]));
  };

  floatx16 o[C::DT];
#pragma unroll
  for (int d = 0; d < C::DT; ++d)
#pragma unroll
    for (int e = 0; e < 16; ++e) o[d][e] = 0.f;
  float m_run = -INFINITY, l_run = 0.f;
  // transposing reads: this lane supplies the 8 bytes of key tr_key at feature tr_d of a 16 keys x 32 features block
  const int tr = C::VOFF + (4 * lh + ((lane & 15) >> 2)) * C::VP + (16 * ((lane >> 4) & 1) + 4 * (lane & 3)) * 2;

  uint64_t bits = 0;
  if (t_begin < t_end) {
    fetch(t_begin);
    bits = keys_of(t_begin);
    put(0, bits);
  }
  __syncthreads();
  for (int t = t_begin; t < t_end; ++t) {
    const int st = (t - t_begin) & 1;
    const unsigned char *const at = smem + st * C::STAGE;
    uint64_t bits_next = 0;
    if (t + 1 < t_end) {
      fetch(t + 1);
      bits_next = keys_of(t + 1);
    }
    floatx16 s[2];
#pragma unroll
    for (int kt = 0; kt < 2; ++kt) {
#pragma unroll
      for (int e = 0; e < 16; ++e) s[kt][e] = 0.f;
#pragma unroll
      for (int ks = 0; ks < KS; ++ks)
        s[kt] = mfma32(*reinterpret_cast<const bf16x8 *>(at + (kt * 32 + l32) * C::KP + (2 * ks + lh) * 16), qf[ks], s[kt]);
    }
    if (bits != ~(uint64_t)0) {
#pragma unroll
      for (int kt = 0; kt < 2; ++kt) {
        const unsigned w = (unsigned)(bits >> (32 * kt)) >> (4 * lh);
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
    if (t + 1 < t_end) put(st ^ 1, bits_next);
    bits = bits_next;
    __syncthreads();
  }
  l_run += __shfl_xor(l_run, 32, 64);

  if (p.parts > 1) {
    if (qi < q_end) {
      const int64_t at = ((int64_t)blockIdx.z * p.q_rows + qi) * p.H + h;
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
      if (lh == 0) { p.part_ml[2 * at] = m_run; p.part_ml[2 * at + 1] = l_run; }
    }
    return;
  }
  const float inv = l_run == 0.f ? 0.f : 1.f / l_run;
  bf16_t *const orow = p.o + (int64_t)qi * p.ld_o + h * p.dh;
#pragma unroll
  for (int d = 0; d < C::DT; ++d)
#pragma unroll
    for (int g = 0; g < 4; g += 2) {
      // lanes l and l ^ 32 hold the two halves of 8 features each: the lower lane collects those of group g, the upper those of g + 1
      uintx2 own, give;
      bf16x4 x0, x1;
#pragma unroll
      for (int e = 0; e < 4; ++e) { x0[e] = (bf16_t)(o[d][4 * g + e] * inv); x1[e] = (bf16_t)(o[d][4 * g + 4 + e] * inv); }
      own = __builtin_bit_cast(uintx2, lh ? x1 : x0);
      give = __builtin_bit_cast(uintx2, lh ? x0 : x1);
      uintx2 got;
      got[0] = (unsigned)__shfl_xor((int)give[0], 32, 64);
      got[1] = (unsigned)__shfl_xor((int)give[1], 32, 64);
      const uintx4 v = lh ? uintx4{got[0], got[1], own[0], own[1]} : uintx4{own[0], own[1], got[0], got[1]};
      const int col = 32 * d + 8 * (g + lh);
      if (qi < q_end && col < p.dh) *reinterpret_cast<uintx4 *>(orow + col) = v;
    }
  if (p.lse && lh == 0 && qi < q_end)
    p.lse[(int64_t)qi * p.H + h] = l_run == 0.f ? -INFINITY : __builtin_fmaf(m_run, p.scale, __builtin_amdgcn_logf(l_run) * 0.6931471805599453f);
}

// The parts' sums of 32 queries and one head meet: eight threads a query.  Each part's maximum is its reference; a part without keys has
// no weight.
__global__ __launch_bounds__(256) void k_cross_join(CrossParams p) {
  const int h = blockIdx.y;
  int b, q_begin, q_end;
  if (!find_tile<32>(p, blockIdx.x, b, q_begin, q_end)) return;
  const int qi = q_begin + (threadIdx.x >> 3), sub = threadIdx.x & 7;
  if (qi >= q_end) return;
  const int64_t step = (int64_t)p.q_rows * p.H, at = (int64_t)qi * p.H + h;
  float top = -INFINITY;
  for (int z = 0; z < p.parts; ++z) top = fmaxf(top, p.part_ml[2 * (at + z * step)]);
  if (top == -INFINITY) top = 0.f;
  float l = 0.f;
  for (int z = 0; z < p.parts; ++z)
    l += p.part_ml[2 * (at + z * step) + 1] * __builtin_amdgcn_exp2f((p.part_ml[2 * (at + z * step)] - top) * p.scale_log2);
  const float inv = l == 0.f ? 0.f : 1.f / l;
  for (int c = sub * 8; c < p.dh; c += 64) {
    floatx4 a = {0.f, 0.f, 0.f, 0.f}, a1 = a;
    for (int z = 0; z < p.parts; ++z) {
      const float w = __builtin_amdgcn_exp2f((p.part_ml[2 * (at + z * step)] - top) * p.scale_log2);
      const floatx4 *src = reinterpret_cast<const floatx4 *>(p.part_o + (at + z * step) * p.dh + c);
      a += src[0] * w;
      a1 += src[1] * w;
    }
    bf16x8 v;
#pragma unroll
    for (int e = 0; e < 4; ++e) { v[e] = (bf16_t)(a[e] * inv); v[e + 4] = (bf16_t)(a1[e] * inv); }
    *reinterpret_cast<bf16x8 *>(p.o + (int64_t)qi * p.ld_o + h * p.dh + c) = v;
  }
  if (p.lse && sub == 0) p.lse[at] = l == 0.f ? -INFINITY : __builtin_fmaf(top, p.scale, __builtin_amdgcn_logf(l) * 0.6931471805599453f);
}

template <int KS, int NW>
int launch_as(const CrossParams &p, hipStream_t s) {
  constexpr int smem = 2 * CrossCfg<KS>::STAGE;
  static std::atomic<uint64_t> allowed;
  const int rc = ddit::allow_dynamic_lds(reinterpret_cast<const void *>(&k_cross_attn<KS, NW>), smem, &allowed);
  if (rc != 0) return rc;
  const unsigned slots = (unsigned)(p.q_rows / (32 * NW) + p.B);
  hipLaunchKernelGGL((k_cross_attn<KS, NW>), dim3(slots, (unsigned)p.H, (unsigned)p.parts), dim3(64 * NW), smem, s, p);
  return ddit::hip_fail(hipGetLastError(), "packed cross-attention launch");
}
template <int NW>
int launch_dh(const CrossParams &p, hipStream_t s) {
  if (p.dh <= 64) return launch_as<4, NW>(p, s);
  if (p.dh <= 80) return launch_as<5, NW>(p, s);
  if (p.dh <= 96) return launch_as<6, NW>(p, s);
  return launch_as<8, NW>(p, s);
}

// Queries a workgroup takes: 32 where sequences have few on average.
bool few_queries(int B, int64_t q_rows) { return q_rows <= (int64_t)64 * B; }

}  // namespace

namespace ddit {

// From the totals alone, since the lengths are on the device, and for the whole chip whatever device is current, since the answer sizes workspaces.
int cross_attn_parts(int B, int64_t q_rows, int64_t kv_rows, int H) {
  const int64_t units = (q_rows / (few_queries(B, q_rows) ? 32 : 128) + B) * H, keys = kv_rows / B;
  return (int)std::max<int64_t>(1, std::min<int64_t>({(int64_t)16, 1024 / units, keys / 128}));
}

int launch_cross_attn(const CrossAttnArgs &a, hipStream_t s) {
  if (a.q_rows == 0) return 0;
  CrossParams p;
  p.q = reinterpret_cast<const bf16_t *>(a.q); p.k = reinterpret_cast<const bf16_t *>(a.k); p.v = reinterpret_cast<const bf16_t *>(a.v);
  p.ld_q = a.ld_q; p.ld_kv = a.ld_kv; p.ld_o = a.ld_o; p.q_off = a.q_off; p.kv_off = a.kv_off; p.mask = a.mask;
  p.B = a.B; p.q_rows = (int)a.q_rows; p.kv_rows = (int)a.kv_rows; p.H = a.H; p.group = a.H / a.H_kv; p.dh = a.dh;
  p.scale = a.scale; p.scale_log2 = a.scale * 1.4426950408889634f; p.rebase = 8.f / p.scale_log2;
  p.o = reinterpret_cast<bf16_t *>(a.o); p.lse = a.lse;
  p.parts = cross_attn_parts(a.B, a.q_rows, a.kv_rows, a.H);
  p.part_o = a.scratch;
  p.part_ml = p.parts > 1 ? a.scratch + (int64_t)p.parts * a.q_rows * a.H * a.dh : nullptr;
  int rc = few_queries(a.B, a.q_rows) ? launch_dh<1>(p, s) : launch_dh<4>(p, s);
  if (rc != 0 || p.parts == 1) return rc;
  hipLaunchKernelGGL(k_cross_join, dim3((unsigned)(p.q_rows / 32 + p.B), (unsigned)p.H), dim3(256), 0, s, p);
  return hip_fail(hipGetLastError(), "packed cross-attention join");
}

}  // namespace ddit
