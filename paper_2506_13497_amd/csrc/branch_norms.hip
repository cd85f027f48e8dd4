// Norms on both sides of a residual branch, in one pass over the stream:
//     x' = r x + gate_b * Norm(f) * g_post          (fp32)
//     h  = bf16( Norm(x') * g_pre * (1 + scale_b) + shift_b )
// f is the branch's output (bf16), x the residual stream (fp32), h the input of the next branch.  Norm is a LayerNorm
// without affine of its own (biased variance, from the deviations) or an RMS norm; every sum is fp32.
//
// Bound: memory, 12 bytes a feature (2 of f, 4 + 4 of the stream, 2 of h).  A row stays in registers from its load to its
// stores; the next row of the same wavefront is on its way meanwhile.  What is common to a sample's rows - gate * g_post,
// g_pre * (1 + scale), shift: up to eight vectors to read for three to keep - is formed once per workgroup and kept in LDS,
// so workgroups take runs of consecutive rows, cut where the sample changes.
// One wavefront a row up to 2048 features; four share a row above, and below where rows are fewer than four a CU.
// Measured: 48600 x 1152 139 us, 4.8 TB/s (a plain copy of that size 4.6 to 4.7), 12960 x 1152 40 us (29 with its operands in the memory-side
// cache), 256 x 256 4.8 us; four wavefronts a row: 12960 x 2304 88 us (4.1 TB/s), x 4096 142 (4.5), x 8192 332 (3.8; 96 KB of vectors leave one
// workgroup a CU).
#include "ddit_common.hpp"

#include <algorithm>
#include <atomic>

namespace {

struct NormsParams {
  const bf16_t *f; int64_t ld_f;
  const bf16_t *g_post, *g_pre;      // [D] or null
  const float *x; float *x_out;
  float r;
  const float *gate_tab, *gate_c6;   // row of the table, row in c6 (of sample 0), or null
  const float *mod_tab, *mod_c6;     // shift row; the scale row follows it
  int64_t c6_stride;
  int64_t N, tps;
  int D;
  float eps;
  bf16_t *out; int64_t ld_out;       // null: the stream's update alone
};

// The sum over a row.  Four wavefronts that share it meet in LDS, in two places used in turn: one is written again only
// behind the barrier of the other, which everybody reaches after reading the first.
template <int W>
__device__ __forceinline__ float row_sum(float v, float *red, int &turn, int wave) {
  v = wave_sum(v);
  if constexpr (W > 1) {
    float *const at = red + turn * W;
    turn ^= 1;
    if ((threadIdx.x & 63) == 0) at[wave] = v;
    __syncthreads();
    v = at[0];
#pragma unroll
    for (int w = 1; w < W; ++w) v += at[w];
  }
  return v;
}

template <int W, int CHUNKS, bool RMS>
__global__ __launch_bounds__(256) void k_branch_norms(NormsParams p) {
  extern __shared__ __attribute__((aligned(16))) float4 vec[];   // [3][nchunk]: gate * g_post, g_pre * (1 + scale), shift
  __shared__ float red[2 * W];
  int turn = 0;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int nchunk = p.D >> 2;
  const int c0 = W == 1 ? lane : (int)threadIdx.x;
  constexpr int STEP = 64 * W;
  const int64_t begin = p.N * (int64_t)blockIdx.x / gridDim.x, end = p.N * ((int64_t)blockIdx.x + 1) / gridDim.x;
  const bool by_sample = p.gate_tab || p.mod_tab;

  float4 xv[CHUNKS], xn[CHUNKS];
  bf16x4 fn[CHUNKS];
  auto load_row = [&](int64_t row) {
    const float4 *xr = reinterpret_cast<const float4 *>(p.x + row * (int64_t)p.D);
    const bf16x4 *fr = reinterpret_cast<const bf16x4 *>(p.f + row * p.ld_f);
#pragma unroll
    for (int j = 0; j < CHUNKS; ++j) {
      const int c = c0 + STEP * j;
      xn[j] = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int e = 0; e < 4; ++e) fn[j][e] = (bf16_t)0.f;
      if (c < nchunk) { xn[j] = xr[c]; fn[j] = fr[c]; }
    }
  };
  // v -> normalised v; elements past the row are zero before and are not used after
  auto normalise = [&](float4 (&v)[CHUNKS]) {
    if constexpr (!RMS) {
      float s = 0.f;
#pragma unroll
      for (int j = 0; j < CHUNKS; ++j) s += (v[j].x + v[j].y) + (v[j].z + v[j].w);
      const float mean = row_sum<W>(s, red, turn, wave) / (float)p.D;
#pragma unroll
      for (int j = 0; j < CHUNKS; ++j)
        if (c0 + STEP * j < nchunk) { v[j].x -= mean; v[j].y -= mean; v[j].z -= mean; v[j].w -= mean; }
    }
    float ss = 0.f;
#pragma unroll
    for (int j = 0; j < CHUNKS; ++j) ss += (v[j].x * v[j].x + v[j].y * v[j].y) + (v[j].z * v[j].z + v[j].w * v[j].w);
    const float rstd = rsqrtf(row_sum<W>(ss, red, turn, wave) / (float)p.D + p.eps);
#pragma unroll
    for (int j = 0; j < CHUNKS; ++j) { v[j].x *= rstd; v[j].y *= rstd; v[j].z *= rstd; v[j].w *= rstd; }
  };

  const int64_t mine = W == 1 ? wave : 0;
  constexpr int ROWS_A_PASS = W == 1 ? 4 : 1;
  for (int64_t seg = begin; seg < end;) {
    const int64_t b = by_sample ? seg / p.tps : 0;
    int64_t seg_end = end;
    if (by_sample && (b + 1) * p.tps < end) seg_end = (b + 1) * p.tps;
    int64_t row = seg + mine;
    if (row < seg_end) load_row(row);
    if (seg != begin) __syncthreads();   // the rows before are done with the vectors
    for (int c = threadIdx.x; c < nchunk; c += 256) {
      float4 g = make_float4(1.f, 1.f, 1.f, 1.f), s = g, t = make_float4(0.f, 0.f, 0.f, 0.f);
      if (p.gate_tab) {
        const float4 a = reinterpret_cast<const float4 *>(p.gate_tab)[c];
        const float4 k = reinterpret_cast<const float4 *>(p.gate_c6 + b * p.c6_stride)[c];
        g = make_float4(a.x + k.x, a.y + k.y, a.z + k.z, a.w + k.w);
      }
      if (p.g_post) {
        const bf16x4 w = reinterpret_cast<const bf16x4 *>(p.g_post)[c];
        g.x *= (float)w[0]; g.y *= (float)w[1]; g.z *= (float)w[2]; g.w *= (float)w[3];
      }
      if (p.mod_tab) {
        const float4 a = reinterpret_cast<const float4 *>(p.mod_tab)[c];
        const float4 k = reinterpret_cast<const float4 *>(p.mod_c6 + b * p.c6_stride)[c];
        const float4 a1 = reinterpret_cast<const float4 *>(p.mod_tab + p.D)[c];
        const float4 k1 = reinterpret_cast<const float4 *>(p.mod_c6 + b * p.c6_stride + p.D)[c];
        t = make_float4(a.x + k.x, a.y + k.y, a.z + k.z, a.w + k.w);
        s = make_float4(1.f + (a1.x + k1.x), 1.f + (a1.y + k1.y), 1.f + (a1.z + k1.z), 1.f + (a1.w + k1.w));
      }
      if (p.g_pre) {
        const bf16x4 w = reinterpret_cast<const bf16x4 *>(p.g_pre)[c];
        s.x *= (float)w[0]; s.y *= (float)w[1]; s.z *= (float)w[2]; s.w *= (float)w[3];
      }
      vec[c] = g; vec[nchunk + c] = s; vec[2 * nchunk + c] = t;
    }
    __syncthreads();
    for (; row < seg_end; row += ROWS_A_PASS) {
      float4 bv[CHUNKS];
#pragma unroll
      for (int j = 0; j < CHUNKS; ++j) {
        xv[j] = xn[j];
        bv[j] = make_float4((float)fn[j][0], (float)fn[j][1], (float)fn[j][2], (float)fn[j][3]);
      }
      if (row + ROWS_A_PASS < seg_end) load_row(row + ROWS_A_PASS);
      normalise(bv);
      float4 *xw = reinterpret_cast<float4 *>(p.x_out + row * (int64_t)p.D);
#pragma unroll
      for (int j = 0; j < CHUNKS; ++j) {
        const int c = c0 + STEP * j;
        if (c < nchunk) {
          const float4 g = vec[c];
          xv[j].x = __builtin_fmaf(g.x, bv[j].x, p.r * xv[j].x);
          xv[j].y = __builtin_fmaf(g.y, bv[j].y, p.r * xv[j].y);
          xv[j].z = __builtin_fmaf(g.z, bv[j].z, p.r * xv[j].z);
          xv[j].w = __builtin_fmaf(g.w, bv[j].w, p.r * xv[j].w);
          xw[c] = xv[j];
        }
      }
      if (p.out) {
        normalise(xv);
        bf16x4 *orow = reinterpret_cast<bf16x4 *>(p.out + row * p.ld_out);
#pragma unroll
        for (int j = 0; j < CHUNKS; ++j) {
          const int c = c0 + STEP * j;
          if (c < nchunk) {
            const float4 s = vec[nchunk + c], t = vec[2 * nchunk + c];
            bf16x4 o;
            o[0] = (bf16_t)__builtin_fmaf(xv[j].x, s.x, t.x);
            o[1] = (bf16_t)__builtin_fmaf(xv[j].y, s.y, t.y);
            o[2] = (bf16_t)__builtin_fmaf(xv[j].z, s.z, t.z);
            o[3] = (bf16_t)__builtin_fmaf(xv[j].w, s.w, t.w);
            orow[c] = o;
          }
        }
      }
    }
    seg = seg_end;
  }
}

template <int W, int CHUNKS, bool RMS>
int launch_kind(const NormsParams &p, int64_t blocks, hipStream_t s) {
  const unsigned lds = 3u * (unsigned)p.D * 4u;   // at most 96 KB
  static std::atomic<uint64_t> allowed;
  if (lds > 48 * 1024) {
    const int rc = ddit::allow_dynamic_lds(reinterpret_cast<const void *>(&k_branch_norms<W, CHUNKS, RMS>), 3 * 8192 * 4, &allowed);
    if (rc != 0) return rc;
  }
  hipLaunchKernelGGL((k_branch_norms<W, CHUNKS, RMS>), dim3((unsigned)blocks), dim3(256), lds, s, p);
  return 0;
}
template <int W, int CHUNKS>
int launch_norms(const NormsParams &p, int norm, int64_t blocks, hipStream_t s) {
  return norm == 1 ? launch_kind<W, CHUNKS, true>(p, blocks, s) : launch_kind<W, CHUNKS, false>(p, blocks, s);
}

}  // namespace

namespace ddit {

int launch_branch_norms(const BranchNormsArgs &a, hipStream_t s) {
  if (a.N == 0) return 0;
  NormsParams p;
  p.f = reinterpret_cast<const bf16_t *>(a.f); p.ld_f = a.ld_f;
  p.g_post = reinterpret_cast<const bf16_t *>(a.g_post); p.g_pre = reinterpret_cast<const bf16_t *>(a.g_pre);
  p.x = a.x; p.x_out = a.x_out; p.r = a.residual_scale;
  p.gate_tab = a.gate_tab; p.gate_c6 = a.gate_c6; p.mod_tab = a.mod_tab; p.mod_c6 = a.mod_c6;
  p.c6_stride = 6 * (int64_t)a.D; p.N = a.N; p.tps = a.tokens_per_sample; p.D = a.D; p.eps = a.eps;
  p.out = reinterpret_cast<bf16_t *>(a.out); p.ld_out = a.ld_out;
  const int64_t cus = device_cus();
  int rc;
  if (a.D > 2048 || (a.D >= 512 && a.N < 4 * cus)) {
    const int64_t blocks = std::min<int64_t>(a.N, 8 * cus);
    if (a.D <= 2048) rc = launch_norms<4, 2>(p, a.norm, blocks, s);
    else if (a.D <= 4096) rc = launch_norms<4, 4>(p, a.norm, blocks, s);
    else rc = launch_norms<4, 8>(p, a.norm, blocks, s);
  } else {
    const int64_t blocks = std::min<int64_t>((a.N + 3) / 4, 8 * cus);
    if (a.D <= 512) rc = launch_norms<1, 2>(p, a.norm, blocks, s);
    else if (a.D <= 1280) rc = launch_norms<1, 5>(p, a.norm, blocks, s);
    else rc = launch_norms<1, 8>(p, a.norm, blocks, s);
  }
  return rc != 0 ? rc : hip_fail(hipGetLastError(), "branch_norms launch");
}

}  // namespace ddit
