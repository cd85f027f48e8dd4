// Linears in microscaled 4-bit floating point: quantisation, its inverse, and the product on the matrix cores.
//
// Format.  A value is one of +-{0, 0.5, 1, 1.5, 2, 3, 4, 6} (sign, two exponent bits, one mantissa bit) times a power of two that 32
// consecutive values of k share: 2^(byte - 127), byte = max(E - 2, 0) where E is the exponent field of the block's largest
// magnitude (so that this one lies in [4, 8) and is at most rounded down to 6), 255 = NaN for a block that holds an Inf or a NaN.
// Values are rounded to nearest, ties to the even code, and saturate at 6.
//
// Layout, of activations and weights alike: k is cut into panels of 128 (the last one padded with zeros), and a panel holds 64
// bytes of codes and 4 of scales for every row, one row behind the other.  A tile of rows in a panel is then one contiguous run of
// memory: whole cache lines, whatever k is, and no k tail in the product.
#include "ddit_common.hpp"

#include <algorithm>

namespace {

typedef unsigned int uintx4 __attribute__((ext_vector_type(4)));
typedef unsigned int uintx2 __attribute__((ext_vector_type(2)));
typedef int intx4 __attribute__((ext_vector_type(4)));
typedef int intx8 __attribute__((ext_vector_type(8)));
typedef __attribute__((address_space(3))) void *lds_ptr_t;

// 2^(byte - 127) as a float; byte 0 is a subnormal one
__device__ __forceinline__ float scale_value(unsigned byte) { return __uint_as_float(byte ? byte << 23 : 1u << 22); }

// the largest magnitude among eight bf16 values, by its bits: an Inf or a NaN is above every finite value
__device__ __forceinline__ unsigned top_of(uintx4 v, unsigned top) {
#pragma unroll
  for (int i = 0; i < 4; ++i) top = max(top, max(v[i] & 0x7fffu, (v[i] >> 16) & 0x7fffu));
  return top;
}
__device__ __forceinline__ unsigned scale_byte(unsigned top) {
  const unsigned e = top >> 7;
  return e == 255 ? 255u : e < 2 ? 0u : e - 2;
}
// the codes of eight bf16 values, the first in the lowest bits; zeros in a NaN block
__device__ __forceinline__ unsigned mx4_encode(uintx4 v, unsigned byte) {
  const float scale = scale_value(byte);
  unsigned c = 0;
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2, (unsigned)v[0]), scale, 0);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2, (unsigned)v[1]), scale, 1);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2, (unsigned)v[2]), scale, 2);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2, (unsigned)v[3]), scale, 3);
  return byte == 255 ? 0u : c;
}

// Sixteen lanes take a row's panel (256 bytes of bf16 in, 64 + 4 out), a wavefront four rows of it, so what it reads and writes
// is contiguous per row and in one piece.  Bound: memory, 2 + 17/32 bytes a value.
constexpr int Q_ROWS = 4;   // row groups of a thread: as many loads in flight
__global__ __launch_bounds__(256) void k_mx4_quantize(const bf16_t *__restrict__ x, int64_t ld_x, int64_t rows, int k, int panels,
                                                      unsigned *__restrict__ codes, unsigned *__restrict__ scales) {
  const int panel = blockIdx.x % panels;
  const int64_t row0 = (int64_t)(blockIdx.x / panels) * (16 * Q_ROWS) + (threadIdx.x >> 4);
  const int l16 = threadIdx.x & 15, col = panel * 128 + l16 * 8;
  uintx4 v[Q_ROWS];
#pragma unroll
  for (int i = 0; i < Q_ROWS; ++i) {
    const int64_t row = row0 + 16 * i;
    v[i] = uintx4{0u, 0u, 0u, 0u};
    if (row < rows && col < k) v[i] = *reinterpret_cast<const uintx4 *>(x + row * ld_x + col);
  }
#pragma unroll
  for (int i = 0; i < Q_ROWS; ++i) {
    const int64_t row = row0 + 16 * i;
    unsigned top = top_of(v[i], 0);
    top = max(top, (unsigned)__shfl_xor((int)top, 1, 64));
    top = max(top, (unsigned)__shfl_xor((int)top, 2, 64));
    const unsigned byte = scale_byte(top), c = mx4_encode(v[i], byte);
    // the four blocks' bytes meet in the first lane of the sixteen
    unsigned four = byte << (8 * (l16 >> 2));
    four |= (unsigned)__shfl_xor((int)four, 4, 64);
    four |= (unsigned)__shfl_xor((int)four, 8, 64);
    if (row < rows) {
      codes[((int64_t)panel * rows + row) * 16 + l16] = c;
      if (l16 == 0) scales[(int64_t)panel * rows + row] = four;
    }
  }
}

__device__ __forceinline__ float mx4_decode(unsigned code, float scale) {
  const unsigned mag = code & 7u;
  // 0, 0.5, then (1 + m / 2) 2^(e - 1)
  const float v = mag < 2 ? 0.5f * (float)mag : __uint_as_float(((mag >> 1) + 126u) << 23 | (mag & 1u) << 22);
  return (code & 8u ? -v : v) * scale;
}

__global__ __launch_bounds__(256) void k_mx4_dequantize(const unsigned *__restrict__ codes, const uint8_t *__restrict__ scales, int64_t rows,
                                                        int k, int panels, bf16_t *__restrict__ out, int64_t ld_out) {
  const int panel = blockIdx.x % panels;
  const int64_t row0 = (int64_t)(blockIdx.x / panels) * (16 * Q_ROWS) + (threadIdx.x >> 4);
  const int l16 = threadIdx.x & 15, col = panel * 128 + l16 * 8;
  if (col >= k) return;
  unsigned c[Q_ROWS], byte[Q_ROWS];
#pragma unroll
  for (int i = 0; i < Q_ROWS; ++i) {
    const int64_t at = (int64_t)panel * rows + std::min<int64_t>(row0 + 16 * i, rows - 1);
    c[i] = codes[at * 16 + l16];
    byte[i] = scales[at * 4 + (l16 >> 2)];
  }
#pragma unroll
  for (int i = 0; i < Q_ROWS; ++i) {
    const int64_t row = row0 + 16 * i;
    const float scale = byte[i] == 255 ? __uint_as_float(0x7fc00000u) : scale_value(byte[i]);
    typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
    bf16x8_t o;
#pragma unroll
    for (int e = 0; e < 8; ++e) o[e] = (bf16_t)mx4_decode((c[i] >> (4 * e)) & 15u, scale);   // exact: bf16 holds every such value
    if (row < rows) *reinterpret_cast<bf16x8_t *>(out + row * ld_out + col) = o;
  }
}

// ------------------------------------------------------------------------------------------------ product
struct Mx4Params {
  const uint8_t *uc, *us, *wc, *ws;
  const bf16_t *bias;
  int64_t N; int n; int panels;
  bf16_t *out; int64_t ld_out;
  const float *resid; float *resid_out;
  const float *gate_tab, *gate_c6; int64_t gate_c6_stride;
  int64_t tokens_per_sample;
  int tiles_m, tiles_n, group_w;
};

__device__ __forceinline__ void lds_barrier() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }
template <int N>
__device__ __forceinline__ void wait_vmcnt() {
  static_assert(N >= 0 && N < 64, "the counter has 6 bits");
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}

// Direct load global -> LDS.  The host's pass knows no 16-byte form of it and would drop a kernel that names one, without a word.
#if defined(__HIP_DEVICE_COMPILE__)
#define MX4_LOAD_TO_LDS(...) __builtin_amdgcn_raw_ptr_buffer_load_lds(__VA_ARGS__)
#else
#define MX4_LOAD_TO_LDS(r, at, size, lane_offset, ...) ((void)(r), (void)(at), (void)(lane_offset))
#endif

// v_mfma_scale_f32_32x32x64_f8f6f4 on 4-bit operands: lane l holds 32 consecutive k, one scaled block, of row l % 32: k half l / 32.
// SEL: byte of the scale registers.  The result lies as that of the bf16 instruction.
template <int SEL>
__device__ __forceinline__ floatx16 mfma_mx4(intx4 a, int sa, intx4 b, int sb, floatx16 c) {
  const intx8 A = {a[0], a[1], a[2], a[3], 0, 0, 0, 0}, B = {b[0], b[1], b[2], b[3], 0, 0, 0, 0};
  return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(A, B, c, 4, 4, SEL, sa, SEL, sb);
}

template <int BM_, int BN_, int WGM_, int WGN_, int NS_, int PER_CU_, int PK_ = 1>
struct Mx4Cfg {
  static constexpr int BM = BM_, BN = BN_, WGM = WGM_, WGN = WGN_, NS = NS_, PER_CU = PER_CU_;
  static constexpr int PK = PK_;                             // panels of a stage
  static constexpr int NW = WGM * WGN, TM = BM / (32 * WGM), TN = BN / (32 * WGN);
  static constexpr int SC = (BM + BN) * 64;                  // scales behind the codes
  static constexpr int PANEL = (BM + BN) * 68, STAGE = PK * PANEL;
  static constexpr int NC = (BM + BN) / 16, NSC = (BM + BN) / 64;   // wave-wide loads of codes (16 rows) and scales (64 rows)
  static constexpr int CJ = (NC + NW - 1) / NW, SJ = (NSC + NW - 1) / NW, NJ = PK * (CJ + SJ);
  static constexpr int PITCH_B = TN * 64 + 16, PITCH_F = 32 * 4 + 16;   // staged rows of the epilogues
  static constexpr int EPI_WAVE = 32 * (PITCH_B > PITCH_F ? PITCH_B : PITCH_F);
  static constexpr int SMEM = NS * STAGE + NW * EPI_WAVE;
  static_assert(BM % 64 == 0 && BN % 64 == 0 && SMEM * PER_CU <= 160 * 1024, "");
  // vector-memory operations of a wavefront that may be under way while it waits for a panel: the loads of later panels, and for
  // the first panels of a tile, which were asked for before the epilogue of the tile before, that epilogue's stores
  static constexpr int AHEAD = (NS - 2) * NJ;
  static constexpr int STORES = TM * 2 * TN;
  static constexpr int AHEAD_FIRST = AHEAD + STORES < 63 ? AHEAD + STORES : 63;
  static_assert(NS >= 2 && AHEAD < 63, "the counter has 6 bits");
};

// Tile `round` of this workgroup; false: none.  Workgroups are dealt out to the 8 XCDs in turn; each XCD takes a run of the sequence, in
// which group_w feature tiles (whose codes stay in its L2) change fastest and token panels next.
__device__ __forceinline__ bool tile_of(const Mx4Params &p, int round, int &tile_m, int &tile_n) {
  const int total = p.tiles_m * p.tiles_n, xcd = blockIdx.x & 7, q8 = total >> 3, r8 = total & 7;
  const int i = round * (int)(gridDim.x >> 3) + (int)(blockIdx.x >> 3);
  if (i >= q8 + (xcd < r8 ? 1 : 0)) return false;
  const int tile = xcd * q8 + (xcd < r8 ? xcd : r8) + i;
  const int gsz = p.tiles_m * p.group_w, full = p.tiles_n / p.group_w;
  int g = tile / gsz, bw = p.group_w;
  if (g >= full) { g = full; bw = p.tiles_n - full * p.group_w; }
  const int r = tile - g * gsz;
  tile_m = r / bw;
  tile_n = g * p.group_w + (r - tile_m * bw);
  return true;
}

// BM x BN tiles of out = u W^T, a run of them a workgroup, a wavefront TM x TN matrix tiles of each.  W is the first operand, so a lane ends
// up with four consecutive features of one token per accumulator group.  k runs in panels through a ring of NS stages, each filled by
// direct global -> LDS loads NS - 1 panels ahead; the stream of panels runs on into the workgroup's next tile, whose first panels
// thus arrive ahead of the stores of this one.  A row's four 16-byte pieces are stored in the order piece ^ (row / 4 % 4), which spreads
// the 16 rows that an LDS read serves at a time over all banks; the loads fetch them from there.
// Bound, 48600 x 4608 x 1152 with GELU (213 us, 2.4 PFLOP/s; bf16 out 183): the board's power, 1400 W (the cap) at 1.96 of 2.4 GHz (bf16 out
// 1.76), with no unit busy all of the time: vector issue 53 % of the SIMDs' (GELU and the epilogue), the matrix cores 29 %, the LDS 28 % of
// the CUs' time.  The residual update of 48600 x 1152 x 4608 (243 us, 2.1 PFLOP/s) comes to 1385 W at 2.29 GHz and waits: matrix cores 24 %,
// wavefronts on loads and stores 30 % of their time.  Rows leave through LDS in pieces of 128 bytes: whole lines.  Straight from the registers,
// after lane exchanges, in pieces of 64 bytes, they took 4 % longer with GELU, a quarter longer without and 16 to 40 % longer in the
// residual update.  Reading the next step's fragments under the products of this one: 0 to 6 % longer.
template <class C, int EPI>
__global__ __launch_bounds__(64 * C::NW, C::NW * C::PER_CU / 4) void k_mx4_gemm(Mx4Params p) {
  constexpr int BM = C::BM, BN = C::BN, NW = C::NW, TM = C::TM, TN = C::TN, NS = C::NS;
  extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int l32 = lane & 31, lh = lane >> 5;
  const int wm = wave / C::WGN, wn = wave % C::WGN;
  int tile_m, tile_n;
  if (!tile_of(p, 0, tile_m, tile_n)) return;

  // ---- the stream of loads: tile ld_round, panel ld_panel comes next.  Rows past the end re-read the last one, and past the last tile the
  // last panel comes again, into a stage that nobody reads any more.
  int ld_round = 0, ld_panel = 0, ld_st = 0;
  unsigned vc[C::CJ], vs[C::SJ];
  auto ld_tile = [&](int tm, int tn) {
    const int64_t row0 = (int64_t)tm * BM;
    const int col0 = tn * BN;
    auto row_of = [&](int r) { return (unsigned)(r < BM ? std::min(row0 + r, p.N - 1) : (int64_t)std::min(col0 + r - BM, p.n - 1)); };
#pragma unroll
    for (int j = 0; j < C::CJ; ++j) {
      const int i = std::min(wave + NW * j, C::NC - 1), r = lane >> 2, piece = (lane & 3) ^ (r >> 2);
      vc[j] = row_of(i * 16 + r) * 64u + piece * 16u;
    }
#pragma unroll
    for (int j = 0; j < C::SJ; ++j) vs[j] = row_of(std::min(wave + NW * j, C::NSC - 1) * 64 + lane) * 4u;
  };
  auto issue = [&]() {
    // (the panel is in the buffers' bases: loads to LDS take no scalar offset here)
#pragma unroll
    for (int sub = 0; sub < C::PK; ++sub) {
      const int64_t from = C::PK == 1 ? ld_panel : std::min(ld_panel + sub, p.panels - 1);
      const __amdgpu_buffer_rsrc_t r_uc = __builtin_amdgcn_make_buffer_rsrc((void *)(p.uc + from * p.N * 64), 0, -1, 0x00020000);
      const __amdgpu_buffer_rsrc_t r_wc = __builtin_amdgcn_make_buffer_rsrc((void *)(p.wc + from * p.n * 64), 0, -1, 0x00020000);
      const __amdgpu_buffer_rsrc_t r_us = __builtin_amdgcn_make_buffer_rsrc((void *)(p.us + from * p.N * 4), 0, -1, 0x00020000);
      const __amdgpu_buffer_rsrc_t r_ws = __builtin_amdgcn_make_buffer_rsrc((void *)(p.ws + from * p.n * 4), 0, -1, 0x00020000);
      unsigned char *const at = smem + ld_st * C::STAGE + sub * C::PANEL;
#pragma unroll
      for (int j = 0; j < C::CJ; ++j) {
        const int i = std::min(wave + NW * j, C::NC - 1);
        if (i * 16 < BM) MX4_LOAD_TO_LDS(r_uc, (lds_ptr_t)(at + i * 1024), 16, vc[j], 0, 0, 0);
        else MX4_LOAD_TO_LDS(r_wc, (lds_ptr_t)(at + i * 1024), 16, vc[j], 0, 0, 0);
      }
#pragma unroll
      for (int j = 0; j < C::SJ; ++j) {
        const int i = std::min(wave + NW * j, C::NSC - 1);
        if (i * 64 < BM) MX4_LOAD_TO_LDS(r_us, (lds_ptr_t)(at + C::SC + i * 256), 4, vs[j], 0, 0, 0);
        else MX4_LOAD_TO_LDS(r_ws, (lds_ptr_t)(at + C::SC + i * 256), 4, vs[j], 0, 0, 0);
      }
    }
    ld_st = ld_st + 1 == NS ? 0 : ld_st + 1;
    if (ld_panel + C::PK < p.panels) {
      ld_panel += C::PK;
    } else {
      int tm, tn;
      if (tile_of(p, ld_round + 1, tm, tn)) {
        ++ld_round; ld_panel = 0;
        ld_tile(tm, tn);
      }
    }
  };

  // the tile's bias at this lane's features
  bf16x4 bias[TN][4];
  auto fetch_bias = [&](int tn) {
#pragma unroll
    for (int a = 0; a < TN; ++a)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
#pragma unroll
        for (int e = 0; e < 4; ++e) bias[a][g][e] = (bf16_t)0.f;
        if (p.bias) bias[a][g] = *reinterpret_cast<const bf16x4 *>(p.bias + std::min(tn * BN + (wn * TN + a) * 32 + 8 * g + 4 * lh, p.n - 4));
      }
  };

  const int f = (l32 >> 2) & 3;
  const int off0 = l32 * 64 + ((lh ^ f) << 4), off1 = l32 * 64 + (((2 + lh) ^ f) << 4);
  const int base_u = wm * TM * 2048, base_w = BM * 64 + wn * TN * 2048;
  const int sc_u = C::SC + (wm * TM * 32 + l32) * 4, sc_w = C::SC + (BM + wn * TN * 32 + l32) * 4;

  ld_tile(tile_m, tile_n);
  fetch_bias(tile_n);
#pragma unroll
  for (int s = 0; s < NS - 1; ++s) issue();
  int st = 0;
  for (int round = 0;; ++round) {
    floatx16 acc[TN][TM];
#pragma unroll
    for (int a = 0; a < TN; ++a)
#pragma unroll
      for (int b = 0; b < TM; ++b)
#pragma unroll
        for (int e = 0; e < 16; ++e) acc[a][b][e] = (float)bias[a][e >> 2][e & 3];
    auto multiply = [&](const unsigned char *at) {
      int su[TM], sw[TN];
      intx4 uf[2][TM], wf[2][TN];
#pragma unroll
      for (int b = 0; b < TM; ++b) su[b] = *reinterpret_cast<const int *>(at + sc_u + b * 128);
#pragma unroll
      for (int a = 0; a < TN; ++a) sw[a] = *reinterpret_cast<const int *>(at + sc_w + a * 128);
#pragma unroll
      for (int s = 0; s < 2; ++s) {
#pragma unroll
        for (int b = 0; b < TM; ++b) uf[s][b] = *reinterpret_cast<const intx4 *>(at + base_u + b * 2048 + (s ? off1 : off0));
#pragma unroll
        for (int a = 0; a < TN; ++a) wf[s][a] = *reinterpret_cast<const intx4 *>(at + base_w + a * 2048 + (s ? off1 : off0));
      }
      // this lane's block of the first step into byte 0, of the second into byte 2
#pragma unroll
      for (int b = 0; b < TM; ++b) su[b] = (unsigned)su[b] >> (8 * lh);
#pragma unroll
      for (int a = 0; a < TN; ++a) sw[a] = (unsigned)sw[a] >> (8 * lh);
#pragma unroll
      for (int a = 0; a < TN; ++a)
#pragma unroll
        for (int b = 0; b < TM; ++b) acc[a][b] = mfma_mx4<0>(wf[0][a], sw[a], uf[0][b], su[b], acc[a][b]);
#pragma unroll
      for (int a = 0; a < TN; ++a)
#pragma unroll
        for (int b = 0; b < TM; ++b) acc[a][b] = mfma_mx4<2>(wf[1][a], sw[a], uf[1][b], su[b], acc[a][b]);
    };
    for (int panel = 0, step = 0; panel < p.panels; panel += C::PK, ++step) {
      if (round > 0 && step < NS - 1) wait_vmcnt<C::AHEAD_FIRST>();
      else wait_vmcnt<C::AHEAD>();
      lds_barrier();   // this stage is complete, and everybody is done with the one before, which is filled next
      issue();
      const unsigned char *const at = smem + st * C::STAGE;
      if (C::PK == 1 || panel + C::PK <= p.panels) {
#pragma unroll
        for (int sub = 0; sub < C::PK; ++sub) multiply(at + sub * C::PANEL);
      } else {
        for (int sub = 0; panel + sub < p.panels; ++sub) multiply(at + sub * C::PANEL);
      }
      st = st + 1 == NS ? 0 : st + 1;
    }

    int next_m = 0, next_n = 0;
    const bool more = tile_of(p, round + 1, next_m, next_n);
    if (more) fetch_bias(next_n);
    // ---- epilogue: each wavefront stages its rows in LDS of its own, so that memory is written in whole row pieces.  Lanes past an
    // edge store past the end of their buffer, which drops it: the number of stores is the same in every tile.
    unsigned char *const stg = smem + NS * C::STAGE + wave * C::EPI_WAVE;
    const int64_t row_w = (int64_t)tile_m * BM + wm * TM * 32;
    const int col_w = tile_n * BN + wn * TN * 32;
    constexpr unsigned NOWHERE = 0x80000000u;
    if constexpr (EPI < 2) {
#pragma unroll
      for (int b = 0; b < TM; ++b) {
#pragma unroll
        for (int a = 0; a < TN; ++a)
#pragma unroll
          for (int g = 0; g < 4; ++g) {
            bf16x4 o;
#pragma unroll
            for (int e = 0; e < 4; ++e) o[e] = (bf16_t)(EPI == 1 ? gelu_tanh_f(acc[a][b][4 * g + e]) : acc[a][b][4 * g + e]);
            *reinterpret_cast<bf16x4 *>(stg + l32 * C::PITCH_B + (a * 32 + 8 * g + 4 * lh) * 2) = o;
          }
        const __amdgpu_buffer_rsrc_t r_out = __builtin_amdgcn_make_buffer_rsrc((void *)(p.out + (row_w + b * 32) * p.ld_out + col_w), 0, 0x7fffffff, 0x00020000);
#pragma unroll
        for (int i = 0; i < 2 * TN; ++i) {
          const int idx = lane + 64 * i, r = idx / (TN * 4), c = idx - r * (TN * 4);
          const uintx4 v = *reinterpret_cast<const uintx4 *>(stg + r * C::PITCH_B + c * 16);
          const bool in = row_w + b * 32 + r < p.N && col_w + c * 8 < p.n;
          __builtin_amdgcn_raw_buffer_store_b128(v, r_out, in ? ((unsigned)r * (unsigned)p.ld_out + c * 8) * 2u : NOWHERE, 0, 2);   // streaming
        }
      }
    } else {
      const int r8 = lane >> 3, f4 = (lane & 7) * 4;
      const int64_t row_last = std::min(row_w + TM * 32, p.N) - 1;
      const int64_t smp0 = p.gate_tab ? std::min(row_w, p.N - 1) / p.tokens_per_sample : 0;
      const bool one = !p.gate_tab || smp0 == row_last / p.tokens_per_sample || row_last < row_w;
      floatx4 gate[TN];
      auto gate_at = [&](int64_t smp, int a) {
        floatx4 g = {1.f, 1.f, 1.f, 1.f};
        if (p.gate_tab) {
          const int col = std::min(col_w + a * 32 + f4, p.n - 4);
          g = *reinterpret_cast<const floatx4 *>(p.gate_tab + col);
          const floatx4 c = *reinterpret_cast<const floatx4 *>(p.gate_c6 + smp * p.gate_c6_stride + col);
#pragma unroll
          for (int e = 0; e < 4; ++e) g[e] += c[e];
        }
        return g;
      };
      // rows of the stream, one matrix tile ahead of their use: loads and stores complete in order, so a tile's loads are issued before the
      // stores of the one before
      constexpr int T = TM * TN;
      floatx4 x[2][4];
      auto fetch_x = [&](int t) {
        const int b = t / TN, a = t % TN;
#pragma unroll
        for (int i = 0; i < 4; ++i)
          x[t & 1][i] = *reinterpret_cast<const floatx4 *>(p.resid + std::min(row_w + b * 32 + 8 * i + r8, p.N - 1) * p.n +
                                                           std::min(col_w + a * 32 + f4, p.n - 4));
      };
      fetch_x(0);
#pragma unroll
      for (int a = 0; a < TN; ++a) gate[a] = gate_at(smp0, a);
#pragma unroll
      for (int t = 0; t < T; ++t) {
        const int b = t / TN, a = t % TN;
        if (t + 1 < T) fetch_x(t + 1);
        const __amdgpu_buffer_rsrc_t r_x = __builtin_amdgcn_make_buffer_rsrc((void *)(p.resid_out + (row_w + b * 32) * p.n + col_w), 0, 0x7fffffff, 0x00020000);
        const __amdgpu_buffer_rsrc_t r_out =
            __builtin_amdgcn_make_buffer_rsrc((void *)(p.out ? p.out + (row_w + b * 32) * p.ld_out + col_w : nullptr), 0, p.out ? 0x7fffffff : 0, 0x00020000);
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          floatx4 v;
#pragma unroll
          for (int e = 0; e < 4; ++e) v[e] = acc[a][b][4 * g + e];
          *reinterpret_cast<floatx4 *>(stg + l32 * C::PITCH_F + (8 * g + 4 * lh) * 4) = v;
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const floatx4 y = *reinterpret_cast<const floatx4 *>(stg + (8 * i + r8) * C::PITCH_F + f4 * 4);
          const int64_t tok = row_w + b * 32 + 8 * i + r8;
          const bool in = tok < p.N && col_w + a * 32 + f4 < p.n;
          floatx4 g = gate[a];
          if (!one) g = gate_at(std::min(tok, p.N - 1) / p.tokens_per_sample, a);
          floatx4 v = x[t & 1][i];
          bf16x4 o;
#pragma unroll
          for (int e = 0; e < 4; ++e) { v[e] = __builtin_fmaf(g[e], y[e], v[e]); o[e] = (bf16_t)v[e]; }
          __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(uintx4, v), r_x, in ? ((unsigned)(8 * i + r8) * (unsigned)p.n + a * 32 + f4) * 4u : NOWHERE, 0, 0);
          __builtin_amdgcn_raw_buffer_store_b64(__builtin_bit_cast(uintx2, o), r_out, in ? ((unsigned)(8 * i + r8) * (unsigned)p.ld_out + a * 32 + f4) * 2u : NOWHERE, 0, 2);
        }
      }
    }
    if (!more) break;
    tile_m = next_m; tile_n = next_n;
  }
  wait_vmcnt<0>();   // no load is under way into LDS that may have another owner soon
}

// Few tokens: one launch for quantisation and product.  A workgroup takes 16 features and up to 16 TB tokens, its eight wavefronts every
// eighth panel each, and their sums meet in LDS.  v_mfma_scale_f32_16x16x128_f8f6f4 wants of lane l one block of row l % 16, block l / 16:
// of W that is 16 bytes, and a wavefront's load is one contiguous kilobyte, straight into registers; of u it is 32 bf16 values, which the
// lane quantises by itself.  Bound: the latency of these loads; every byte of W is read once.
template <int SEL>
__device__ __forceinline__ floatx4 mfma_mx4_16(intx4 a, int sa, intx4 b, int sb, floatx4 c) {
  const intx8 A = {a[0], a[1], a[2], a[3], 0, 0, 0, 0}, B = {b[0], b[1], b[2], b[3], 0, 0, 0, 0};
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(A, B, c, 4, 4, SEL, sa, SEL, sb);
}
constexpr int FEW_NW = 8, FEW_DEPTH = 2;   // wavefronts; panels of a wavefront under way
template <int TB, bool CODES, int EPI>
__global__ __launch_bounds__(64 * FEW_NW) void k_mx4_few(Mx4Params p, const bf16_t *__restrict__ u, int64_t ld_u, int k) {
  __shared__ floatx4 sums[FEW_NW][TB][64];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, l16 = lane & 15, blk = lane >> 4;
  const int col0 = blockIdx.x * 16, w_row = std::min(col0 + l16, p.n - 1);
  int u_row[TB];
#pragma unroll
  for (int b = 0; b < TB; ++b) u_row[b] = std::min(16 * b + l16, (int)p.N - 1);
  floatx4 acc[TB];
#pragma unroll
  for (int b = 0; b < TB; ++b) acc[b] = floatx4{0.f, 0.f, 0.f, 0.f};
  intx4 wc[FEW_DEPTH], uc[FEW_DEPTH][CODES ? TB : 1];
  uintx4 uv[FEW_DEPTH][CODES ? 1 : TB][4];
  int ws[FEW_DEPTH], us[FEW_DEPTH][TB];
  auto fetch = [&](int i, int panel) {
    const int64_t w_at = (int64_t)panel * p.n + w_row;
    wc[i] = *reinterpret_cast<const intx4 *>(p.wc + w_at * 64 + blk * 16);
    ws[i] = p.ws[w_at * 4 + blk];
#pragma unroll
    for (int b = 0; b < TB; ++b) {
      if constexpr (CODES) {
        const int64_t u_at = (int64_t)panel * p.N + u_row[b];
        uc[i][b] = *reinterpret_cast<const intx4 *>(p.uc + u_at * 64 + blk * 16);
        us[i][b] = p.us[u_at * 4 + blk];
      } else {
        const bf16_t *row = u + u_row[b] * ld_u;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int col = panel * 128 + blk * 32 + 8 * j;
          uv[i][b][j] = uintx4{0u, 0u, 0u, 0u};
          if (col < k) uv[i][b][j] = *reinterpret_cast<const uintx4 *>(row + col);
        }
      }
    }
  };
#pragma unroll
  for (int i = 0; i < FEW_DEPTH; ++i)
    if (wave + FEW_NW * i < p.panels) fetch(i, wave + FEW_NW * i);
  for (int panel0 = wave; panel0 < p.panels; panel0 += FEW_NW * FEW_DEPTH) {
#pragma unroll
    for (int i = 0; i < FEW_DEPTH; ++i) {
      const int panel = panel0 + FEW_NW * i;
      if (panel >= p.panels) break;
#pragma unroll
      for (int b = 0; b < TB; ++b) {
        intx4 c;
        int byte;
        if constexpr (CODES) {
          c = uc[i][b]; byte = us[i][b];
        } else {
          unsigned top = 0;
#pragma unroll
          for (int j = 0; j < 4; ++j) top = top_of(uv[i][b][j], top);
          byte = (int)scale_byte(top);
#pragma unroll
          for (int j = 0; j < 4; ++j) c[j] = (int)mx4_encode(uv[i][b][j], (unsigned)byte);
        }
        acc[b] = mfma_mx4_16<0>(wc[i], ws[i], c, byte, acc[b]);
      }
      if (panel + FEW_NW * FEW_DEPTH < p.panels) fetch(i, panel + FEW_NW * FEW_DEPTH);
    }
  }
#pragma unroll
  for (int b = 0; b < TB; ++b) sums[wave][b][lane] = acc[b];
  __syncthreads();
  // lane l holds features 4 (l / 16) .. + 3 of token l % 16
  if (wave >= TB) return;
  const int tok = 16 * wave + l16, col = col0 + 4 * blk;
  if (tok >= p.N || col >= p.n) return;
  floatx4 y = sums[0][wave][lane];
#pragma unroll
  for (int w = 1; w < FEW_NW; ++w) y += sums[w][wave][lane];
  if (p.bias) {
    const bf16x4 v = *reinterpret_cast<const bf16x4 *>(p.bias + col);
#pragma unroll
    for (int e = 0; e < 4; ++e) y[e] += (float)v[e];
  }
  bf16x4 o;
  if constexpr (EPI == 2) {
    floatx4 g = {1.f, 1.f, 1.f, 1.f}, x = *reinterpret_cast<const floatx4 *>(p.resid + (int64_t)tok * p.n + col);
    if (p.gate_tab) {
      const floatx4 t = *reinterpret_cast<const floatx4 *>(p.gate_tab + col);
      const floatx4 c = *reinterpret_cast<const floatx4 *>(p.gate_c6 + tok / p.tokens_per_sample * p.gate_c6_stride + col);
#pragma unroll
      for (int e = 0; e < 4; ++e) g[e] = t[e] + c[e];
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) { x[e] = __builtin_fmaf(g[e], y[e], x[e]); o[e] = (bf16_t)x[e]; }
    *reinterpret_cast<floatx4 *>(p.resid_out + (int64_t)tok * p.n + col) = x;
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) o[e] = (bf16_t)(EPI == 1 ? gelu_tanh_f(y[e]) : y[e]);
  }
  if (EPI != 2 || p.out) *reinterpret_cast<bf16x4 *>(p.out + tok * p.ld_out + col) = o;
}

template <int TB, bool CODES>
int launch_few_as(int epi, const Mx4Params &p, const bf16_t *u, int64_t ld_u, int k, hipStream_t s) {
  const dim3 grid((unsigned)((p.n + 15) / 16)), block(64 * FEW_NW);
  if (epi == 0) hipLaunchKernelGGL((k_mx4_few<TB, CODES, 0>), grid, block, 0, s, p, u, ld_u, k);
  else if (epi == 1) hipLaunchKernelGGL((k_mx4_few<TB, CODES, 1>), grid, block, 0, s, p, u, ld_u, k);
  else hipLaunchKernelGGL((k_mx4_few<TB, CODES, 2>), grid, block, 0, s, p, u, ld_u, k);
  return ddit::hip_fail(hipGetLastError(), "mx4 linear launch (few tokens)");
}
template <bool CODES>
int launch_few(int epi, const Mx4Params &p, const bf16_t *u, int64_t ld_u, int k, hipStream_t s) {
  return p.N <= 16 ? launch_few_as<1, CODES>(epi, p, u, ld_u, k, s) : launch_few_as<2, CODES>(epi, p, u, ld_u, k, s);
}

// Every workgroup quantises all tokens, so with more than 16 of them it pays where workgroups are few.  us in a captured graph, one launch / two:
// 16 tokens of 1152 x 1152 3.7 / 7.1, 6912 x 1152 5.0 / 7.2, 1152 x 4608 7.3 / 13.1; 32 tokens 5.4 / 7.2, 9.4 / 7.3, 12.2 / 13.6 and of
// 2304 x 1152, past the border, 5.5 / 7.2; 64 tokens 8.8 / 7.5, 16.7 / 7.6, 22.7 / 13.8.
bool few_tokens(int64_t N, int n) { return N <= 16 || (N <= 32 && n <= 2048); }

template <class C, int EPI>
int launch_as(const Mx4Params &p, unsigned grid, hipStream_t s) {
  static std::atomic<uint64_t> allowed;
  const int rc = ddit::allow_dynamic_lds(reinterpret_cast<const void *>(&k_mx4_gemm<C, EPI>), C::SMEM, &allowed);
  if (rc != 0) return rc;
  hipLaunchKernelGGL((k_mx4_gemm<C, EPI>), dim3(grid), dim3(64 * C::NW), C::SMEM, s, p);
  return ddit::hip_fail(hipGetLastError(), "mx4 linear launch");
}
template <class C, bool RESIDUAL = true, bool DENSE = true>
int launch_tile(int epi, Mx4Params p, hipStream_t s) {
  p.tiles_m = (int)((p.N + C::BM - 1) / C::BM);
  p.tiles_n = (p.n + C::BN - 1) / C::BN;
  if ((int64_t)p.tiles_m * p.tiles_n > 0x7fffffff - 8) { ddit::set_error("mx4 linear: too many output tiles"); return -2; }
  // feature tiles of a group: their codes stay in an XCD's L2 while the token panels pass
  p.group_w = std::max(1, std::min(p.tiles_n, (int)((2 << 20) / ((int64_t)C::BN * p.panels * 64))));
  const int total = p.tiles_m * p.tiles_n, grid = std::min((total + 7) / 8, std::max(1, ddit::device_cus() * C::PER_CU / 8)) * 8;
  if constexpr (RESIDUAL)
    if (epi == 2) return launch_as<C, 2>(p, grid, s);
  if constexpr (DENSE)
    if (epi != 2) return epi == 0 ? launch_as<C, 0>(p, grid, s) : launch_as<C, 1>(p, grid, s);
  return -2;   // not reached: the caller picks a tile that has the epilogue
}

}  // namespace

namespace ddit {

int launch_mx4_quantize(const void *x, int64_t ld_x, int64_t rows, int k, void *codes, void *scales, hipStream_t s) {
  if (rows == 0) return 0;
  const int64_t panels = mx4_panels(k), blocks = (rows + 16 * Q_ROWS - 1) / (16 * Q_ROWS) * panels;
  hipLaunchKernelGGL(k_mx4_quantize, dim3((unsigned)blocks), dim3(256), 0, s, reinterpret_cast<const bf16_t *>(x), ld_x, rows, k, (int)panels,
                     reinterpret_cast<unsigned *>(codes), reinterpret_cast<unsigned *>(scales));
  return hip_fail(hipGetLastError(), "mx4_quantize launch");
}

int launch_mx4_dequantize(const void *codes, const void *scales, int64_t rows, int k, void *out, int64_t ld_out, hipStream_t s) {
  if (rows == 0) return 0;
  const int64_t panels = mx4_panels(k), blocks = (rows + 16 * Q_ROWS - 1) / (16 * Q_ROWS) * panels;
  hipLaunchKernelGGL(k_mx4_dequantize, dim3((unsigned)blocks), dim3(256), 0, s, reinterpret_cast<const unsigned *>(codes),
                     reinterpret_cast<const uint8_t *>(scales), rows, k, (int)panels, reinterpret_cast<bf16_t *>(out), ld_out);
  return hip_fail(hipGetLastError(), "mx4_dequantize launch");
}

bool mx4_one_launch(int64_t N, int n) { return few_tokens(N, n); }

Mx4Form mx4_form(int epilogue, int64_t N, int n, int cus) {
  if (few_tokens(N, n)) return {N <= 16 ? 16 : 32, 16};
  // Tiles of 128 x 128, three workgroups a CU, as soon as every CU has one: their epilogues run under the others' products.  The residual
  // update holds rows of the stream too and takes two a CU, and from two rounds of the chip on 256 x 256, which draws fewer operands
  // through the L2.  us, 64 x 64 / 128 x 128 / 256 x 256, u in codes: with GELU 2304 x 4608 x 1152 20.8 / 12.3 / 15.4, 12960 101 / 59.8 / 57.9, 48600
  // 370 / 213 / 202; bf16 out 300 x 2304 x 1152 5.2 / 6.5 / 11.8, 12960 x 1152 x 1152 27.5 / 14.2 / 15.3, 48600 x 1152 x 4608 - / 145 / 151,
  // 48600 x 4608 x 1152 350 / 183 / 168; residual 2304 x 1152 x 4608 20.3 / 20.8 / 40.9, 6480 44 / 30 / 44, 12960 87 / 59 / 60, 48600 387 / 264 / 243.
  // So many tokens of many features and a short k would gain 5 to 8 % from 256 x 256 without a stream too, which is not compiled.  With two panels
  // between barriers in place of one the small tile takes, 300 x 1152 x 4608, 10.1 in place of 10.9 and, residual, 6480 44 in place of 49.
  const int64_t t128 = ((N + 127) / 128) * ((n + 127) / 128), t256 = ((N + 255) / 256) * ((n + 255) / 256);
  if (t128 < cus) return {64, 64};
  if (epilogue != 2 || t256 < 2 * cus) return {128, 128};
  return {256, 256};
}

int launch_mx4_gemm(int epilogue, const Mx4GemmArgs &a, hipStream_t s) {
  if (a.N == 0) return 0;
  Mx4Params p;
  p.uc = reinterpret_cast<const uint8_t *>(a.u_codes); p.us = reinterpret_cast<const uint8_t *>(a.u_scales);
  p.wc = reinterpret_cast<const uint8_t *>(a.w_codes); p.ws = reinterpret_cast<const uint8_t *>(a.w_scales);
  p.bias = reinterpret_cast<const bf16_t *>(a.bias);
  p.N = a.N; p.n = a.n; p.panels = (int)mx4_panels(a.k);
  p.out = reinterpret_cast<bf16_t *>(a.out); p.ld_out = a.ld_out; p.resid = a.resid; p.resid_out = a.resid_out;
  p.gate_tab = a.gate_tab; p.gate_c6 = a.gate_c6; p.gate_c6_stride = a.gate_c6_stride; p.tokens_per_sample = a.tokens_per_sample;
  const Mx4Form f = mx4_form(epilogue, a.N, a.n, device_cus());
  if (f.cols == 16) {
    if (a.u) return launch_few<false>(epilogue, p, reinterpret_cast<const bf16_t *>(a.u), a.ld_u, a.k, s);
    return launch_few<true>(epilogue, p, nullptr, 0, a.k, s);
  }
  if (f.cols == 64) return launch_tile<Mx4Cfg<64, 64, 2, 2, 2, 3, 2>>(epilogue, p, s);
  if (f.cols == 256) return launch_tile<Mx4Cfg<256, 256, 2, 4, 3, 1>, true, false>(epilogue, p, s);
  if (epilogue != 2) return launch_tile<Mx4Cfg<128, 128, 2, 2, 2, 3>, false, true>(epilogue, p, s);
  return launch_tile<Mx4Cfg<128, 128, 2, 2, 3, 2>, true, false>(epilogue, p, s);
}

}  // namespace ddit
