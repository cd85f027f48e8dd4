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
typedef int intx4 __attribute__((ext_vector_type(4)));
typedef int intx8 __attribute__((ext_vector_type(8)));
typedef __attribute__((address_space(3))) void *lds_ptr_t;

// 2^(byte - 127) as a float; byte 0 is a subnormal one
__device__ __forceinline__ float scale_value(unsigned byte) { return __uint_as_float(byte ? byte << 23 : 1u << 22); }

// Eight bf16 values of a lane, four lanes a block: -> the block's scale byte and the lane's codes, the first in the lowest bits.
__device__ __forceinline__ unsigned mx4_encode(uintx4 v, unsigned &byte) {
  // the largest magnitude by its bits: an Inf or a NaN is above every finite value
  unsigned top = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) top = max(top, max(v[i] & 0x7fffu, (v[i] >> 16) & 0x7fffu));
  top = max(top, (unsigned)__shfl_xor((int)top, 1, 64));
  top = max(top, (unsigned)__shfl_xor((int)top, 2, 64));
  const unsigned e = top >> 7;
  byte = e == 255 ? 255u : e < 2 ? 0u : e - 2;
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
    unsigned byte;
    const unsigned c = mx4_encode(v[i], byte);
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
#define MX4_LOAD_TO_LDS(r, at, size, lane_offset, offset, ...) ((void)(r), (void)(at), (void)(lane_offset), (void)(offset))
#endif

// v_mfma_scale_f32_32x32x64_f8f6f4 on 4-bit operands: lane l holds 32 consecutive k, one scaled block, of row l % 32: k half l / 32.
// SEL: byte of the scale registers.  The result lies as that of the bf16 instruction.
template <int SEL>
__device__ __forceinline__ floatx16 mfma_mx4(intx4 a, int sa, intx4 b, int sb, floatx16 c) {
  const intx8 A = {a[0], a[1], a[2], a[3], 0, 0, 0, 0}, B = {b[0], b[1], b[2], b[3], 0, 0, 0, 0};
  return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(A, B, c, 4, 4, SEL, sa, SEL, sb);
}

template <int BM_, int BN_, int WGM_, int WGN_, int NS_>
struct Mx4Cfg {
  static constexpr int BM = BM_, BN = BN_, WGM = WGM_, WGN = WGN_, NS = NS_;
  static constexpr int NW = WGM * WGN, TM = BM / (32 * WGM), TN = BN / (32 * WGN);
  static constexpr int SC = (BM + BN) * 64;                  // scales behind the codes
  static constexpr int STAGE = (BM + BN) * 68;
  static constexpr int NC = (BM + BN) / 16, NSC = (BM + BN) / 64;   // wave-wide loads of codes (16 rows) and scales (64 rows)
  static constexpr int CJ = (NC + NW - 1) / NW, SJ = (NSC + NW - 1) / NW, NJ = CJ + SJ;
  static constexpr int PITCH_B = TN * 64 + 16, PITCH_F = 32 * 4 + 16;   // staged rows of the epilogues
  static constexpr int EPI_WAVE = 32 * (PITCH_B > PITCH_F ? PITCH_B : PITCH_F);
  static constexpr int SMEM = NS * STAGE > NW * EPI_WAVE ? NS * STAGE : NW * EPI_WAVE;
  static_assert(BM % 64 == 0 && BN % 64 == 0 && (NS - 1) * NJ < 64, "");
};

// One BM x BN tile of out = u W^T a workgroup, a wavefront TM x TN matrix tiles of it.  W is the first operand, so a lane ends up with
// four consecutive features of one token per accumulator group.  k runs in panels through a ring of NS stages, each filled by direct
// global -> LDS loads NS - 1 panels ahead.  A row's four 16-byte pieces are stored in the order piece ^ (row / 4 % 4), which spreads
// the 16 rows that an LDS read serves at a time over all banks; the loads fetch them from there.
template <class C, int EPI>
__global__ __launch_bounds__(64 * C::NW) void k_mx4_gemm(Mx4Params p) {
  constexpr int BM = C::BM, BN = C::BN, NW = C::NW, TM = C::TM, TN = C::TN, NS = C::NS;
  extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int l32 = lane & 31, lh = lane >> 5;
  const int wm = wave / C::WGN, wn = wave % C::WGN;
  // tiles: runs of the sequence on one XCD (workgroups are dealt out round-robin); in groups of group_w feature tiles, token panels outside
  int tile;
  {
    const int total = p.tiles_m * p.tiles_n, xcd = blockIdx.x & 7, q8 = total >> 3, r8 = total & 7;
    tile = xcd * q8 + (xcd < r8 ? xcd : r8) + (blockIdx.x >> 3);
  }
  int tile_m, tile_n;
  {
    const int gsz = p.tiles_m * p.group_w, full = p.tiles_n / p.group_w;
    int g = tile / gsz, bw = p.group_w;
    if (g >= full) { g = full; bw = p.tiles_n - full * p.group_w; }
    const int r = tile - g * gsz;
    tile_m = r / bw;
    tile_n = g * p.group_w + (r - tile_m * bw);
  }
  const int64_t row0 = (int64_t)tile_m * BM;
  const int col0 = tile_n * BN;

  // ---- loads: rows past the end re-read the last one
  auto u_row = [&](int r) { return (unsigned)(row0 + r < p.N ? row0 + r : p.N - 1); };
  auto w_row = [&](int r) { return (unsigned)(col0 + r < p.n ? col0 + r : p.n - 1); };
  unsigned vc[C::CJ], vs[C::SJ];
#pragma unroll
  for (int j = 0; j < C::CJ; ++j) {
    const int i = std::min(wave + NW * j, C::NC - 1), r = (lane >> 2), piece = (lane & 3) ^ (r >> 2);
    const int row = i * 16 + r;
    vc[j] = (row < BM ? u_row(row) : w_row(row - BM)) * 64u + piece * 16u;
  }
#pragma unroll
  for (int j = 0; j < C::SJ; ++j) {
    const int row = std::min(wave + NW * j, C::NSC - 1) * 64 + lane;
    vs[j] = (row < BM ? u_row(row) : w_row(row - BM)) * 4u;
  }
  auto issue = [&](int panel, int st) {
    const __amdgpu_buffer_rsrc_t r_uc = __builtin_amdgcn_make_buffer_rsrc((void *)p.uc, 0, -1, 0x00020000);
    const __amdgpu_buffer_rsrc_t r_wc = __builtin_amdgcn_make_buffer_rsrc((void *)p.wc, 0, -1, 0x00020000);
    const __amdgpu_buffer_rsrc_t r_us = __builtin_amdgcn_make_buffer_rsrc((void *)p.us, 0, -1, 0x00020000);
    const __amdgpu_buffer_rsrc_t r_ws = __builtin_amdgcn_make_buffer_rsrc((void *)p.ws, 0, -1, 0x00020000);
    const unsigned pc_u = (unsigned)((int64_t)panel * p.N * 64), pc_w = (unsigned)panel * (unsigned)p.n * 64u;
    unsigned char *const at = smem + st * C::STAGE;
#pragma unroll
    for (int j = 0; j < C::CJ; ++j) {
      const int i = std::min(wave + NW * j, C::NC - 1);
      if (i * 16 < BM) MX4_LOAD_TO_LDS(r_uc, (lds_ptr_t)(at + i * 1024), 16, vc[j], pc_u, 0, 0);
      else MX4_LOAD_TO_LDS(r_wc, (lds_ptr_t)(at + i * 1024), 16, vc[j], pc_w, 0, 0);
    }
#pragma unroll
    for (int j = 0; j < C::SJ; ++j) {
      const int i = std::min(wave + NW * j, C::NSC - 1);
      if (i * 64 < BM) MX4_LOAD_TO_LDS(r_us, (lds_ptr_t)(at + C::SC + i * 256), 4, vs[j], pc_u >> 4, 0, 0);
      else MX4_LOAD_TO_LDS(r_ws, (lds_ptr_t)(at + C::SC + i * 256), 4, vs[j], pc_w >> 4, 0, 0);
    }
  };

  floatx16 acc[TN][TM];
#pragma unroll
  for (int a = 0; a < TN; ++a)
#pragma unroll
    for (int b = 0; b < TM; ++b)
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[a][b][e] = 0.f;
  const int f = (l32 >> 2) & 3;
  const int off0 = l32 * 64 + ((lh ^ f) << 4), off1 = l32 * 64 + (((2 + lh) ^ f) << 4);
  const int base_u = wm * TM * 2048, base_w = BM * 64 + wn * TN * 2048;
  const int sc_u = C::SC + (wm * TM * 32 + l32) * 4, sc_w = C::SC + (BM + wn * TN * 32 + l32) * 4;

#pragma unroll
  for (int s = 0; s < NS - 1; ++s) issue(std::min(s, p.panels - 1), s);
  int st = 0, st_in = NS - 1;
  for (int panel = 0; panel < p.panels; ++panel) {
    wait_vmcnt<(NS - 2) * C::NJ>();
    lds_barrier();   // this panel is complete, and everybody is done with the one before, whose stage is filled next
    issue(std::min(panel + NS - 1, p.panels - 1), st_in);
    const unsigned char *const at = smem + st * C::STAGE;
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
    st = st + 1 == NS ? 0 : st + 1;
    st_in = st_in + 1 == NS ? 0 : st_in + 1;
  }
  wait_vmcnt<0>();
  lds_barrier();

  // ---- epilogue: each wavefront stages its rows in LDS of its own, so that memory is written in whole row pieces
  unsigned char *const stg = smem + wave * C::EPI_WAVE;
  const int64_t row_w = row0 + wm * TM * 32;
  const int col_w = col0 + wn * TN * 32;
  floatx4 bias[TN][4];
#pragma unroll
  for (int a = 0; a < TN; ++a)
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      bias[a][g] = floatx4{0.f, 0.f, 0.f, 0.f};
      if (p.bias) {
        const int c = std::min(col_w + a * 32 + 8 * g + 4 * lh, p.n - 4);
        const bf16x4 v = *reinterpret_cast<const bf16x4 *>(p.bias + c);
#pragma unroll
        for (int e = 0; e < 4; ++e) bias[a][g][e] = (float)v[e];
      }
    }
  if constexpr (EPI < 2) {
#pragma unroll
    for (int b = 0; b < TM; ++b) {
#pragma unroll
      for (int a = 0; a < TN; ++a)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          bf16x4 o;
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            float v = acc[a][b][4 * g + e] + bias[a][g][e];
            if (EPI == 1) v = gelu_tanh_f(v);
            o[e] = (bf16_t)v;
          }
          *reinterpret_cast<bf16x4 *>(stg + l32 * C::PITCH_B + (a * 32 + 8 * g + 4 * lh) * 2) = o;
        }
#pragma unroll
      for (int i = 0; i < 2 * TN; ++i) {
        const int idx = lane + 64 * i, r = idx / (TN * 4), c = idx - r * (TN * 4);
        const uintx4 v = *reinterpret_cast<const uintx4 *>(stg + r * C::PITCH_B + c * 16);
        const int64_t tok = row_w + b * 32 + r;
        const int col = col_w + c * 8;
        if (tok < p.N && col < p.n) __builtin_nontemporal_store(v, reinterpret_cast<uintx4 *>(p.out + tok * p.ld_out + col));
      }
    }
  } else {
    const int r8 = lane >> 3, f4 = (lane & 7) * 4;
#pragma unroll
    for (int a = 0; a < TN; ++a) {
      const int col = col_w + a * 32 + f4;
      const bool in = col < p.n;
#pragma unroll
      for (int b = 0; b < TM; ++b) {
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          floatx4 v;
#pragma unroll
          for (int e = 0; e < 4; ++e) v[e] = acc[a][b][4 * g + e] + bias[a][g][e];
          *reinterpret_cast<floatx4 *>(stg + l32 * C::PITCH_F + (8 * g + 4 * lh) * 4) = v;
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const floatx4 y = *reinterpret_cast<const floatx4 *>(stg + (8 * i + r8) * C::PITCH_F + f4 * 4);
          const int64_t tok = row_w + b * 32 + 8 * i + r8;
          if (tok < p.N && in) {
            floatx4 x = *reinterpret_cast<const floatx4 *>(p.resid + tok * p.n + col);
            floatx4 g = {1.f, 1.f, 1.f, 1.f};
            if (p.gate_tab) {
              g = *reinterpret_cast<const floatx4 *>(p.gate_tab + col);
              g += *reinterpret_cast<const floatx4 *>(p.gate_c6 + tok / p.tokens_per_sample * p.gate_c6_stride + col);
            }
            bf16x4 o;
#pragma unroll
            for (int e = 0; e < 4; ++e) { x[e] = __builtin_fmaf(g[e], y[e], x[e]); o[e] = (bf16_t)x[e]; }
            *reinterpret_cast<floatx4 *>(p.resid_out + tok * p.n + col) = x;
            if (p.out) *reinterpret_cast<bf16x4 *>(p.out + tok * p.ld_out + col) = o;
          }
        }
      }
    }
  }
}

template <class C, int EPI>
int launch_as(const Mx4Params &p, hipStream_t s) {
  static std::atomic<uint64_t> allowed;
  const int rc = ddit::allow_dynamic_lds(reinterpret_cast<const void *>(&k_mx4_gemm<C, EPI>), C::SMEM, &allowed);
  if (rc != 0) return rc;
  hipLaunchKernelGGL((k_mx4_gemm<C, EPI>), dim3((unsigned)(p.tiles_m * p.tiles_n)), dim3(64 * C::NW), C::SMEM, s, p);
  return ddit::hip_fail(hipGetLastError(), "mx4 linear launch");
}
template <class C>
int launch_tile(int epi, Mx4Params p, hipStream_t s) {
  p.tiles_m = (int)((p.N + C::BM - 1) / C::BM);
  p.tiles_n = (p.n + C::BN - 1) / C::BN;
  // feature tiles of a group: their codes stay in an XCD's L2 while the token panels pass
  p.group_w = std::max(1, std::min(p.tiles_n, (int)((2 << 20) / ((int64_t)C::BN * p.panels * 64))));
  return epi == 0 ? launch_as<C, 0>(p, s) : epi == 1 ? launch_as<C, 1>(p, s) : launch_as<C, 2>(p, s);
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

int launch_mx4_gemm(int epilogue, const Mx4GemmArgs &a, hipStream_t s) {
  if (a.N == 0) return 0;
  Mx4Params p;
  p.uc = reinterpret_cast<const uint8_t *>(a.u_codes); p.us = reinterpret_cast<const uint8_t *>(a.u_scales);
  p.wc = reinterpret_cast<const uint8_t *>(a.w_codes); p.ws = reinterpret_cast<const uint8_t *>(a.w_scales);
  p.bias = reinterpret_cast<const bf16_t *>(a.bias);
  p.N = a.N; p.n = a.n; p.panels = (int)mx4_panels(a.k);
  p.out = reinterpret_cast<bf16_t *>(a.out); p.ld_out = a.ld_out; p.resid = a.resid; p.resid_out = a.resid_out;
  p.gate_tab = a.gate_tab; p.gate_c6 = a.gate_c6; p.gate_c6_stride = a.gate_c6_stride; p.tokens_per_sample = a.tokens_per_sample;
  if ((a.N + 127) / 128 * ((a.n + 127) / 128) >= 512) return launch_tile<Mx4Cfg<256, 256, 2, 4, 4>>(epilogue, p, s);
  return launch_tile<Mx4Cfg<64, 64, 2, 2, 4>>(epilogue, p, s);
}

}  // namespace ddit
