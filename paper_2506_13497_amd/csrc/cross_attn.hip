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
// K and V tiles go through registers into LDS, because values of rows that a mask takes out, rows of other sequences and columns past the head
// dim have to be zeros: a weight of zero times an infinity would be NaN.  Up to 320 keys (256 of 128 features) are fetched once, and every
// wavefront walks over its row tiles with no further barrier; longer sequences stream through two stages, one barrier a tile.
//
// Bound, 2 x 48600 queries x 300 states x 16 heads of 72 (215 us, 620 TFLOP/s): the vector arithmetic of the softmax, at the clock that the
// board's power leaves.  A wavefront issues 245 vector instructions a key tile, with its share of a row tile's begin and end, beside 22
// matrix instructions of 32 clocks: vector issue takes 63 % of the SIMDs' time and the matrix cores 39 %, at 1400 W (the cap) and 1.93 of 2.4
// GHz; wavefronts wait on loads and stores 29 % of theirs.  One state takes 150 us, 64 as long: up to two key tiles the rows of q and o
// bound it (a row of one head is 144 bytes, parts of two or three lines).  192 states take 168, 256 184, 320 212.
#include "ddit_common.hpp"

#include <algorithm>

namespace {

typedef unsigned int uintx4 __attribute__((ext_vector_type(4)));
typedef unsigned int uintx2 __attribute__((ext_vector_type(2)));
typedef short shortx4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) shortx4 *lds_s4_ptr_t;

constexpr int KT = 64;   // keys of a tile

// Lanes l and l + 32 exchange: the upper lanes' a against the lower lanes' b.
struct Swapped { unsigned a, b; };
__device__ __forceinline__ Swapped swap_halves(unsigned a, unsigned b) {
  const uintx2 r = __builtin_bit_cast(uintx2, __builtin_amdgcn_permlane32_swap(a, b, false, false));
  return {r[0], r[1]};
}

// The same within the halves: lanes 16-31 and 48-63 of a against lanes 0-15 and 32-47 of b.
__device__ __forceinline__ Swapped swap_quarters(unsigned a, unsigned b) {
  const uintx2 r = __builtin_bit_cast(uintx2, __builtin_amdgcn_permlane16_swap(a, b, false, false));
  return {r[0], r[1]};
}

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
// [kv_begin, kv_end); false: nothing.  Offsets outside the arrays are cut off there, and sums of runs stop at 2^30 (far past every slot), so
// that offsets that decrease lead nowhere outside either.
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
  static constexpr int VOFF = ST == 1 ? 0 : KT * KP; // (with one stage K stays in registers)
  static constexpr int STAGE = VOFF + KT * VP;
  static constexpr int SMEM = ST * STAGE + ST * 8;   // and the valid keys of every stage
  static_assert(DT * 64 <= VP && SMEM <= 160 * 1024, "a V row is read to the end of its last tile");
};

// PARTS: a part of the keys, whose sums go to part_o and part_ml
template <int KS, int NW, int ST, bool PARTS>
__global__ __launch_bounds__(64 * NW) void k_cross_attn(CrossParams p) {
  using C = CrossCfg<KS, ST>;
  constexpr int QT = 32 * NW, CJ = (KT * C::CH + 64 * NW - 1) / (64 * NW);   // pieces of a tile that a thread stages
  extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, l32 = lane & 31, lh = lane >> 5;
  // Workgroups are dealt out to the 8 XCDs in turn.  The heads of a slot come one after the other on one XCD: a row of one head is 2 dh bytes
  // of the token's, so heads share the cache lines of q and o, which its L2 puts together.  So do a slot's parts of the keys: where few slots
  // have long encodings, an XCD reads all of a request's K and V by itself and others are idle.
  const int H_kv = p.H / p.group, i0 = blockIdx.x >> 3, i1 = i0 / H_kv, kv_head = i0 - i1 * H_kv;
  const int i2 = PARTS ? i1 / p.parts : i1, part = PARTS ? i1 - i2 * p.parts : 0;
  Slot slot;
  if (!find_slot(p, (unsigned)i2 * 8 + (blockIdx.x & 7), p.run, slot)) return;
  const int h0 = kv_head * p.group;   // first of the key head's query heads
  const int n_keys = slot.kv_end - slot.kv_begin, all = (n_keys + KT - 1) / KT;
  const int t_begin = PARTS ? (int)((int64_t)all * part / p.parts) : 0, t_end = PARTS ? (int)((int64_t)all * (part + 1) / p.parts) : all;
  const int n_tiles = t_end - t_begin, pieces = p.dh >> 3;

  // Everything is loaded through buffers: what lies past an end, or is sent there, comes as zeros, and every lane loads, so that waits can count.
  constexpr unsigned NOWHERE = 0x80000000u;
  auto buffer = [](const void *at, int64_t bytes) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<void *>(at), 0, (int)std::min<int64_t>(bytes, 0x7fffffff), 0x00020000);
  };
  constexpr bool Q_AHEAD = NW == 8 && KS <= 6;   // (with wider heads, or three wavefronts a SIMD, the registers are full)
  bf16x8 qf[KS], qn[Q_AHEAD ? KS : 1];
  auto fetch_q = [&](int r0, bf16x8 (&to)[KS]) {   // rows past the end: the last one again
    const int r = std::min(r0 + l32, slot.end - 1), q0 = std::min(r0, slot.end - 1) / p.group, q = r / p.group;
    const __amdgpu_buffer_rsrc_t src = buffer(p.q + (slot.q_first + q0) * p.ld_q + h0 * p.dh, 0x7fffffff);
    const unsigned at = ((unsigned)(q - q0) * (unsigned)p.ld_q + (unsigned)((r - q * p.group) * p.dh + 8 * lh)) * 2u;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks)
      to[ks] = __builtin_bit_cast(bf16x8, __builtin_amdgcn_raw_buffer_load_b128(src, 2 * ks + lh < pieces ? at + ks * 32 : NOWHERE, 0, 0));
  };
  const int r_first = __builtin_amdgcn_readfirstlane(slot.begin + wave * 32);   // this wavefront's rows of the first row tile
  if constexpr (Q_AHEAD) fetch_q(r_first, qn);

  const int64_t kv_at = (int64_t)slot.kv_begin * p.ld_kv + kv_head * p.dh;
  const bf16_t *const kbase = p.k + kv_at, *const vbase = p.v + kv_at;
  // What a thread holds of a tile: pieces to stage of K and V, or, where a wavefront is alone, its K fragments as they are.
  constexpr bool ALONE = NW == 1;
  constexpr int NQ = 2 * KS, NPV = 4 * C::DT;   // matrix instructions of a tile's scores and of its share of O
  struct Pieces { uintx4 k[ALONE ? NQ : CJ], v[CJ]; uint64_t bits; };
  unsigned piece_at[CJ];
#pragma unroll
  for (int j = 0; j < CJ; ++j) {
    const int i = tid + 64 * NW * j, row = i / C::CH, c = i - row * C::CH;
    piece_at[j] = row < KT && c < pieces ? ((unsigned)row * (unsigned)p.ld_kv + c * 8) * 2u : NOWHERE;
  }
  // (the whole offset is the lane's own: whether a scalar one counts where a buffer's end is checked is described both ways)
  const unsigned frag_at[2] = {((unsigned)l32 * (unsigned)p.ld_kv + 8 * lh) * 2u, ((unsigned)(32 + l32) * (unsigned)p.ld_kv + 8 * lh) * 2u};
  auto fetch = [&](int tile, Pieces &x) {
    const int left = std::min(n_keys - tile * KT, KT);
    const int64_t bytes = ((int64_t)(left - 1) * p.ld_kv + p.dh) * 2, at = (int64_t)tile * KT * p.ld_kv;
    const __amdgpu_buffer_rsrc_t ksrc = buffer(kbase + at, bytes), vsrc = buffer(vbase + at, bytes);
    if constexpr (ALONE) {
#pragma unroll
      for (int q = 0; q < NQ; ++q)   // key 32 (q % 2) + l32, k-step q / 2
        x.k[q] = __builtin_amdgcn_raw_buffer_load_b128(ksrc, 2 * (q >> 1) + lh < pieces ? frag_at[q & 1] + (q >> 1) * 32 : NOWHERE, 0, 0);
    }
#pragma unroll
    for (int j = 0; j < CJ; ++j) {
      if constexpr (!ALONE) x.k[j] = __builtin_amdgcn_raw_buffer_load_b128(ksrc, piece_at[j], 0, 0);
      x.v[j] = __builtin_amdgcn_raw_buffer_load_b128(vsrc, piece_at[j], 0, 0);
    }
    unsigned valid = lane < left;   // one bit a key
    if (p.mask) valid = __builtin_amdgcn_raw_buffer_load_b8(buffer(p.mask + slot.kv_begin + tile * KT, left), lane, 0, 0);
    x.bits = __ballot(valid != 0);
  };
  auto put = [&](int st, const Pieces &x) {
    unsigned char *const at = smem + st * C::STAGE;
#pragma unroll
    for (int j = 0; j < CJ; ++j) {
      const int i = tid + 64 * NW * j, row = i / C::CH, c = i - row * C::CH;
      if (row < KT) {
        if constexpr (!ALONE) *reinterpret_cast<uintx4 *>(at + row * C::KP + c * 16) = x.k[j];   // zeros past the head dim
        *reinterpret_cast<uintx4 *>(at + C::VOFF + row * C::VP + c * 16) = (x.bits >> row) & 1 ? x.v[j] : uintx4{0u, 0u, 0u, 0u};
      }
    }
    if (!ALONE && tid == 0) reinterpret_cast<uint64_t *>(smem + ST * C::STAGE)[st] = x.bits;
  };

  floatx16 o[C::DT];
  float m_run, l_run;
  // transposing reads: this lane supplies the 8 bytes of key tr_key at feature tr_d of a 16 keys x 32 features block
  const int tr = C::VOFF + (4 * lh + ((lane & 15) >> 2)) * C::VP + (16 * ((lane >> 4) & 1) + 4 * (lane & 3)) * 2;
  auto begin = [&](int r0) {
    if constexpr (Q_AHEAD) {
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) qf[ks] = qn[ks];
      fetch_q(r0 + QT, qn);
    } else {
      fetch_q(r0, qf);
    }
#pragma unroll
    for (int d = 0; d < C::DT; ++d)
#pragma unroll
      for (int e = 0; e < 16; ++e) o[d][e] = 0.f;
    m_run = -INFINITY; l_run = 0.f;
  };
  // Where a tile's fragments lie: K of key 32 (q % 2) + l32, k-step q / 2
  auto k_frag = [&](int st, int q) {
    return *reinterpret_cast<const bf16x8 *>(smem + st * C::STAGE + ((q & 1) * 32 + l32) * C::KP + (2 * (q >> 1) + lh) * 16);
  };
  auto valid_of = [&](int st) { return reinterpret_cast<const uint64_t *>(smem + ST * C::STAGE)[st]; };
  auto scores = [&](int st, floatx16 (&s)[2]) {
#pragma unroll
    for (int kt = 0; kt < 2; ++kt)
#pragma unroll
      for (int e = 0; e < 16; ++e) s[kt][e] = 0.f;
#pragma unroll
    for (int q = 0; q < NQ; ++q) s[q & 1] = mfma32(k_frag(st, q), qf[q >> 1], s[q & 1]);
  };
  // One tile: softmax of its scores and O^T += V^T P^T.  A wavefront issues in order, so the matrix instructions are threaded by hand through
  // the vector arithmetic, which takes longer than they do: one after every two exponentials, as soon as its 16 keys' weights are there.  V
  // fragments are read a chunk of 16 keys ahead.  (The next tile's scores in between as well, and room for them, changed nothing for 64 to 80
  // features and spilled registers above: 2 x 48600 x 256 took a tenth longer with heads of 96, a third with heads of 128.)
  auto step = [&](int st, uint64_t bits, floatx16 (&s)[2]) {
    const unsigned valid[2] = {(unsigned)__builtin_amdgcn_readfirstlane((int)(unsigned)bits), (unsigned)__builtin_amdgcn_readfirstlane((int)(unsigned)(bits >> 32))};
    if ((valid[0] & valid[1]) != ~0u) {
#pragma unroll
      for (int kt = 0; kt < 2; ++kt) {
        const int w = (int)(valid[kt] >> (4 * lh));
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const int keep = __builtin_amdgcn_sbfe(w, 8 * (e >> 2) + (e & 3), 1);   // all ones or none
          s[kt][e] = __int_as_float((__float_as_int(s[kt][e]) & keep) | (0xff800000 & ~keep));
        }
      }
    }
    float mx = fmaxf(s[0][0], s[0][1]);
#pragma unroll
    for (int e = 2; e < 16; ++e) mx = fmaxf(mx, s[0][e]);
#pragma unroll
    for (int e = 0; e < 16; ++e) mx = fmaxf(mx, s[1][e]);
    const Swapped both = swap_halves(__float_as_uint(mx), __float_as_uint(mx));
    mx = fmaxf(__uint_as_float(both.a), __uint_as_float(both.b));
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
    // exp2(s c - m c) with one rounding less: fine while m c, rounded once for all scores, is off by at most 2^-13.  Further out the
    // maximum comes off first, before the difference is scaled, or its rounding error would swamp the exponent, and m c leave fp32.
    float ref = m_run == -INFINITY ? 0.f : m_run * p.scale_log2;
    if (__ballot(__builtin_fabsf(ref) > 4096.f)) {
      const float off = m_run == -INFINITY ? 0.f : m_run;
#pragma unroll
      for (int e = 0; e < 16; ++e) { s[0][e] -= off; s[1][e] -= off; }
      ref = 0.f;
    }
    const unsigned char *const va = smem + st * C::STAGE + tr;
    bf16x8 pf[4], vf[2][C::DT];
    auto v_frags = [&](int kc) {
#pragma unroll
      for (int d = 0; d < C::DT; ++d) {
        const shortx4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4_ptr_t)(va + kc * 16 * C::VP + d * 64));
        const shortx4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4_ptr_t)(va + (kc * 16 + 8) * C::VP + d * 64));
        vf[kc & 1][d] = __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
      }
    };
    auto update = [&](int v) {   // the v-th of the tile's matrix instructions
      const int kc = v / C::DT, d = v - kc * C::DT;
      if (d == 0 && kc < 3) v_frags(kc + 1);
      o[d] = mfma32(vf[kc & 1][d], pf[kc], o[d]);
    };
    v_frags(0);
    __builtin_amdgcn_sched_barrier(0);
    float sum = 0.f;
    int v = 0;
#pragma unroll
    for (int g = 0; g < 16; ++g) {
#pragma unroll
      for (int e = 2 * g; e < 2 * g + 2; ++e) {
        const float w = __builtin_amdgcn_exp2f(__builtin_fmaf(s[e >> 4][e & 15], p.scale_log2, -ref));
        sum += w;
        pf[e >> 3][e & 7] = (bf16_t)w;
      }
      __builtin_amdgcn_sched_barrier(0);
      if (g >= 4 * (v / C::DT) + 3) update(v++);
      __builtin_amdgcn_sched_barrier(0);
    }
#pragma unroll
    for (int w = 0; w < NPV; ++w)
      if (w >= v) update(w);
    l_run += sum;
  };
  auto finish = [&](int r0) {
    const int r = r0 + l32, q = r / p.group, h = h0 + r - q * p.group;
    const bool in = r < slot.end;
    const int64_t token = slot.q_first + q;
    l_run += __shfl_xor(l_run, 32, 64);
    if constexpr (PARTS) {
      if (in) {
        const int64_t at = (part * (int64_t)p.q_rows + token) * p.H + h;
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
    // Lanes without a row, or past the head dim, store past the end of the buffer, which drops it: the same stores for every tile, so that
    // where the next queries were asked for before them (Q_AHEAD) the wait for those need not be one for all stores.  The other forms ask in
    // begin, behind these stores, and wait for both.
    const float inv = l_run == 0.f ? 0.f : 1.f / l_run;
    const int q0 = r0 / p.group;   // first token of the tile
    const __amdgpu_buffer_rsrc_t r_o = buffer(p.o + (slot.q_first + q0) * p.ld_o + h0 * p.dh, 0x7fffffff);
    const unsigned o_at = in ? ((unsigned)(q - q0) * (unsigned)p.ld_o + (unsigned)((h - h0) * p.dh)) * 2u : NOWHERE;
    // Of 32 features lanes l and l + 32 hold groups of four in turn.  Two exchanges make it four lanes a row with eight features each, so that
    // a store writes 64 bytes of 16 rows in place of 32 bytes of 32.
    const unsigned at_lo = (unsigned)__shfl((int)o_at, lane & 15, 64), at_hi = (unsigned)__shfl((int)o_at, 16 + (lane & 15), 64);
    const int col_lane = 8 * (2 * ((lane >> 4) & 1) + lh);
#pragma unroll
    for (int d = 0; d < C::DT; ++d) {
      uintx4 v[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        bf16x4 x0, x1;
#pragma unroll
        for (int e = 0; e < 4; ++e) { x0[e] = (bf16_t)(o[d][8 * i + e] * inv); x1[e] = (bf16_t)(o[d][8 * i + 4 + e] * inv); }
        const uintx2 y0 = __builtin_bit_cast(uintx2, x0), y1 = __builtin_bit_cast(uintx2, x1);
        const Swapped w0 = swap_halves(y0[0], y1[0]), w1 = swap_halves(y0[1], y1[1]);
        v[i] = uintx4{w0.a, w1.a, w0.b, w1.b};
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const Swapped w = swap_quarters(v[0][i], v[1][i]);
        v[0][i] = w.a; v[1][i] = w.b;
      }
      const int col = 32 * d + col_lane;
      const bool is = col < p.dh;
      __builtin_amdgcn_raw_buffer_store_b128(v[0], r_o, is && at_lo != NOWHERE ? at_lo + col * 2u : NOWHERE, 0, 0);
      __builtin_amdgcn_raw_buffer_store_b128(v[1], r_o, is && at_hi != NOWHERE ? at_hi + col * 2u : NOWHERE, 0, 0);
    }
    const __amdgpu_buffer_rsrc_t r_l = buffer(p.lse ? p.lse + (int64_t)(slot.q_first + q0) * p.H + h0 : nullptr, p.lse ? 0x7fffffff : 0);
    const float lse = l_run == 0.f ? -INFINITY : __builtin_fmaf(m_run, p.scale, __builtin_amdgcn_logf(l_run) * 0.6931471805599453f);
    __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(lse), r_l, in && lh == 0 ? ((unsigned)(q - q0) * p.H + (h - h0)) * 4u : NOWHERE, 0, 0);
  };

  if constexpr (ALONE) {
    // one wavefront, whose LDS operations stay in order: no barrier, one stage for V, and K straight into registers; the next tile is on its
    // way during the softmax of this one
    Pieces x;
    if (n_tiles > 0) fetch(t_begin, x);
    begin(r_first);
    for (int t = 0; t < n_tiles; ++t) {
      floatx16 sc[2];
#pragma unroll
      for (int kt = 0; kt < 2; ++kt)
#pragma unroll
        for (int e = 0; e < 16; ++e) sc[kt][e] = 0.f;
#pragma unroll
      for (int q = 0; q < NQ; ++q) sc[q & 1] = mfma32(__builtin_bit_cast(bf16x8, x.k[q]), qf[q >> 1], sc[q & 1]);
      put(0, x);
      const uint64_t bits = x.bits;
      if (t + 1 < n_tiles) fetch(t_begin + t + 1, x);
      step(0, bits, sc);
    }
    finish(r_first);
  } else if (n_tiles <= ST) {
    // everything is fetched once, and every wavefront walks over its row tiles with no further barrier
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
    for (int r0 = r_first; r0 < slot.end; r0 += QT) {
      begin(r0);
      for (int t = 0; t < n_tiles; ++t) {
        floatx16 sc[2];
        scores(t, sc);
        step(t, valid_of(t), sc);
      }
      finish(r0);
    }
  } else {
    for (int r0 = r_first; r0 - wave * 32 < slot.end; r0 += QT) {   // wavefronts without rows come along for the barriers
      Pieces x;
      begin(r0);
      fetch(t_begin, x);
      if (r0 != r_first) __syncthreads();   // the tiles of the rows before are done with
      put(0, x);
      __syncthreads();
      for (int t = 0; t < n_tiles; ++t) {
        if (t + 1 < n_tiles) fetch(t_begin + t + 1, x);
        floatx16 sc[2];
        scores(t & 1, sc);
        step(t & 1, valid_of(t & 1), sc);
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
  for (int z0 = 0; z0 < p.parts; z0 += 8) {
    float2 v[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = *reinterpret_cast<const float2 *>(p.part_o + (at + std::min(z0 + j, p.parts - 1) * step) * p.dh + c);
#pragma unroll
    for (int j = 0; j < 8; ++j) {   // lanes past the parts have no weight
      const float w = __uint_as_float((unsigned)__builtin_amdgcn_readlane((int)__float_as_uint(weight), z0 + j));
      a.x += w == 0.f ? 0.f : v[j].x * w;
      a.y += w == 0.f ? 0.f : v[j].y * w;
    }
  }
  if (2 * lane < p.dh) {
    bf16x2 v;
    v[0] = (bf16_t)(a.x * inv); v[1] = (bf16_t)(a.y * inv);
    *reinterpret_cast<bf16x2 *>(p.o + token * p.ld_o + h * p.dh + c) = v;
  }
  if (p.lse && lane == 0) p.lse[at] = l == 0.f ? -INFINITY : __builtin_fmaf(top, p.scale, __builtin_amdgcn_logf(l) * 0.6931471805599453f);
}

template <int KS, int NW, int ST, bool PARTS>
int launch_as(const CrossParams &p, hipStream_t s) {
  const unsigned slots = (unsigned)((int64_t)p.q_rows * p.group / p.run + p.B);
  const int64_t blocks = (int64_t)((slots + 7) / 8 * 8) * (p.H / p.group) * p.parts;
  if (blocks * 64 * NW > 0xffffffff) {   // a launch counts its work-items in 32 bits
    ddit::set_error("packed cross-attention: %lld workgroups of %d threads: too many", (long long)blocks, 64 * NW);
    return -2;
  }
  constexpr int smem = CrossCfg<KS, ST>::SMEM;
  static std::atomic<uint64_t> allowed;
  const int rc = ddit::allow_dynamic_lds(reinterpret_cast<const void *>(&k_cross_attn<KS, NW, ST, PARTS>), smem, &allowed);
  if (rc != 0) return rc;
  hipLaunchKernelGGL((k_cross_attn<KS, NW, ST, PARTS>), dim3((unsigned)blocks), dim3(64 * NW), smem, s, p);
  return ddit::hip_fail(hipGetLastError(), "packed cross-attention launch");
}
template <int KS>
int launch_form(int waves, const CrossParams &p, hipStream_t s) {
  constexpr int ST = KS == 8 ? 4 : 5;   // as many stages as the LDS holds
  if (waves == 1) return p.parts > 1 ? launch_as<KS, 1, 1, true>(p, s) : launch_as<KS, 1, 1, false>(p, s);
  if constexpr (KS <= 6)
    if (waves == 12) return launch_as<KS, 12, ST, false>(p, s);
  return p.parts > 1 ? launch_as<KS, 8, ST, true>(p, s) : launch_as<KS, 8, ST, false>(p, s);
}

// One wavefront a workgroup where sequences have few of the `rows` rows a key head, on average.
bool lone_wavefronts(int B, int64_t rows) { return rows <= (int64_t)64 * B; }

}  // namespace

namespace ddit {

// From the totals alone, since the lengths are on the device, and for the whole chip whatever device is current, since the answer sizes workspaces:
// parts of 128 keys and more, as many as make one round of the chip (a workgroup of eight wavefronts fills a CU, four of one do).  One part / as
// taken, us in a captured graph: 22 queries of 16 heads of 72 x 1024 states 25.5 / 15.1 (8 parts), x 2048 46.5 / 20 (16), 1 x 4096 of 128 on 4
// key heads 115 / 22 (32), 2000 x 4096 of 8 heads 99 / 53 (4).  From 1024 states in all on, a border that leaves time: 22 x 485 take 14.4 in one
// part and 12.7 in three, 22 x 1000 25.3 and, in eight, 15.1; and 17 x 4096, whose rows want eight wavefronts, 39 in 32 parts and 26 in eight.
int cross_attn_parts(int B, int64_t q_rows, int64_t kv_rows, int H, int H_kv) {
  const int64_t rows = q_rows * (H / H_kv);
  const bool lone = lone_wavefronts(B, rows);
  const int64_t units = (rows / (lone ? 32 : 256) + B) * H_kv;
  if (kv_rows < 1024) return 1;
  return (int)std::max<int64_t>(1, std::min<int64_t>({(int64_t)32, (lone ? 1024 : 256) / units, kv_rows / 128}));
}

CrossForm cross_attn_form(int B, int64_t q_rows, int64_t kv_rows, int H, int H_kv, int dh, int cus) {
  const int64_t rows = q_rows * (H / H_kv);
  CrossForm f;
  f.parts = cross_attn_parts(B, q_rows, kv_rows, H, H_kv);
  // Three wavefronts a SIMD for heads whose registers allow it, from two rounds of the device on (256 rows a workgroup of eight); else two.
  // us, 8 / 12, 16 heads of 72: 2304 rows x 300 states 14.1 / 15.3, 6480 23.6 / 26.5, 8192 (the border) 24.5 / 28.5, 12960 39.9 / 40.6, 2 x 48600
  // 236 / 215, 48600 x 1024 351 / 311; 2 x 48600 x 256 of 64 159 / 152, of 96 209 / 200, of 128 257 / 402.
  f.waves = lone_wavefronts(B, rows) ? 1 : f.parts == 1 && dh <= 96 && rows * H_kv >= (int64_t)512 * cus ? 12 : 8;
  f.run = 32 * f.waves;
  if (f.waves > 1 && f.parts == 1) {
    // row tiles a workgroup walks over: a round of the chip takes that many and about one more for its set-up; counted for sequences of one length
    int64_t best = 0, cost = INT64_MAX;
    for (int64_t m = 1; m <= 16; ++m) {
      const int64_t run = B * f.run * m, blocks = B * ((rows + run - 1) / run) * H_kv, c = (blocks + cus - 1) / cus * (m + 1);
      if (c < cost) { cost = c; best = m; }
    }
    f.run *= (int)best;
  }
  return f;
}

int launch_cross_attn(const CrossAttnArgs &a, hipStream_t s) {
  if (a.q_rows == 0) return 0;
  CrossParams p;
  p.q = reinterpret_cast<const bf16_t *>(a.q); p.k = reinterpret_cast<const bf16_t *>(a.k); p.v = reinterpret_cast<const bf16_t *>(a.v);
  p.ld_q = a.ld_q; p.ld_kv = a.ld_kv; p.ld_o = a.ld_o; p.q_off = a.q_off; p.kv_off = a.kv_off; p.mask = a.mask;
  p.B = a.B; p.q_rows = (int)a.q_rows; p.kv_rows = (int)a.kv_rows; p.H = a.H; p.group = a.H / a.H_kv; p.dh = a.dh;
  p.scale = a.scale; p.scale_log2 = a.scale * 1.4426950408889634f; p.rebase = std::min(8.f / p.scale_log2, 1e30f);
  p.o = reinterpret_cast<bf16_t *>(a.o); p.lse = a.lse;
  const CrossForm f = cross_attn_form(a.B, a.q_rows, a.kv_rows, a.H, a.H_kv, a.dh, device_cus());
  p.parts = f.parts; p.run = f.run;
  p.part_o = a.scratch;
  p.part_ml = p.parts > 1 ? a.scratch + (int64_t)p.parts * a.q_rows * a.H * a.dh : nullptr;
  const int rc = p.dh <= 64 ? launch_form<4>(f.waves, p, s) : p.dh <= 80 ? launch_form<5>(f.waves, p, s) : p.dh <= 96 ? launch_form<6>(f.waves, p, s)
                                                                                                                  : launch_form<8>(f.waves, p, s);
  if (rc != 0 || p.parts == 1) return rc;
  hipLaunchKernelGGL(k_cross_join, dim3((unsigned)(a.q_rows * p.group / 4 + p.B), (unsigned)a.H_kv), dim3(256), 0, s, p);
  return hip_fail(hipGetLastError(), "packed cross-attention join");
}

}  // namespace ddit
