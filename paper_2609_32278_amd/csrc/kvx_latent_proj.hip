// Products with the per-head weights of latent attention, gfx950: queries into the latent
// space and sums out of it (absorbed form), cached rows to keys and values (expanded form).
// Operands are bf16, sums float32, each result is rounded once: to bf16, the operand of what follows.
#include <cmath>

#include "kvx_latent_tile.h"

namespace kvx {
namespace {

constexpr int kThreads = 256;
constexpr int kSlice = 128;  // latent dims per workgroup of the query product

// q' = W_uk^T q, as (W_uk^T) q^T: W's rows run along the latent dims, so its operand is read
// transposed from LDS.  Workgroup: 64 tokens, one head, 128 latent dims.  Bound by latency (its
// waves wait 61% of their cycles): a workgroup is one chain of loads, a barrier, few products and
// stores, and every wave of every 128-dim slice reads the queries again.  900 tokens of 32 heads
// 30 us, 1.6 TB/s of the 48 MB that have to go in and out; counted, 189 MB of requests to L2 and
// 81 MB to HBM (37 us with results of 8 bytes a lane and loads of queries behind the barrier).
template <int LAT, int D>
__global__ __launch_bounds__(kThreads) void latent_absorb_kernel(LatentProjParams p) {
  constexpr int IN = D + kLatRope, OUT = LAT + kLatRope;
  constexpr int WB = kSlice * 2 + 32;  // LDS row
  __shared__ __attribute__((aligned(16))) uint8_t wl[D * WB];
  const LatentRows rows = listed(p, p.rows);
  const int hd = blockIdx.y, s0 = blockIdx.z * kSlice;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, n = lane & 15, g = lane >> 4;
  const uint16_t* w = p.w + (size_t)hd * D * LAT + s0;
  constexpr int WL = D * (kSlice / 8) / kThreads;
  uint4 wr[WL];
#pragma unroll
  for (int j = 0; j < WL; j++) {
    const int i = j * kThreads + tid;
    wr[j] = *(const uint4*)(w + (size_t)(i / (kSlice / 8)) * LAT + i % (kSlice / 8) * 8);
  }
  const uint16_t* q[4];
  bf16x8 x[4][D / 32];  // all on their way before the first is used
#pragma unroll
  for (int tb = 0; tb < 4; tb++) {
    const int t = tb * 16 + n;
    q[tb] = p.in + ((size_t)(rows.row0 + (t < rows.ntok ? t : 0)) * p.num_q_heads + hd) * IN;
#pragma unroll
    for (int ks = 0; ks < D / 32; ks++) x[tb][ks] = *(const bf16x8*)(q[tb] + ks * 32 + 8 * g);
  }
#pragma unroll
  for (int j = 0; j < WL; j++) {
    const int i = j * kThreads + tid;
    *(uint4*)(wl + i / (kSlice / 8) * WB + i % (kSlice / 8) * 16) = wr[j];
  }
  __syncthreads();
  f32x4 acc[4][2];
#pragma unroll
  for (int tb = 0; tb < 4; tb++) acc[tb][0] = acc[tb][1] = f32x4{};
#pragma unroll
  for (int ks = 0; ks < D / 32; ks++) {
    bf16x8 a[2];
#pragma unroll
    for (int b = 0; b < 2; b++) {
      s16x4 h[2];
#pragma unroll
      for (int e = 0; e < 2; e++)
        h[e] = read_tr(wl + (ks * 32 + 8 * g + 4 * e + n / 4) * WB + (wave * 32 + (n % 4) * 8 + b * 4) * 2);
      a[b] = join(h[0], h[1]);
    }
#pragma unroll
    for (int tb = 0; tb < 4; tb++)
#pragma unroll
      for (int b = 0; b < 2; b++)
        acc[tb][b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a[b], x[tb][ks], acc[tb][b], 0, 0, 0);
  }
#pragma unroll
  for (int tb = 0; tb < 4; tb++) {
    const int t = tb * 16 + n;
    if (t >= rows.ntok) continue;
    uint16_t* dst = p.out + ((size_t)(rows.own0 + t) * p.num_q_heads + hd) * OUT;
    // the columns were read so that a lane's two blocks are 8 dims side by side
    *(uint4*)(dst + s0 + wave * 32 + 8 * g) =
        make_uint4(pack_bf16(acc[tb][0][0], acc[tb][0][1]), pack_bf16(acc[tb][0][2], acc[tb][0][3]),
                   pack_bf16(acc[tb][1][0], acc[tb][1][1]), pack_bf16(acc[tb][1][2], acc[tb][1][3]));
    if (blockIdx.z == 0) {  // the rotated dims follow: 8 chunks, two of them per (wave, g) of waves 0
      if (wave == 0) {
#pragma unroll
        for (int c = 0; c < 2; c++) *(uint4*)(dst + LAT + (2 * g + c) * 8) = *(const uint4*)(q[tb] + D + (2 * g + c) * 8);
      }
    }
  }
}

// o = W_uv (sum), as W_uv o^T; both operands run along the latent dims.  Workgroup: 64
// tokens, one head.  Bound by latency: 900 tokens of 32 heads are 480 workgroups, two a CU, each
// a chain of loads and products whose four waves all read the sums.  28 us, 1.5 TB/s of the 41 MB
// that have to go in and out; counted, 112 MB of requests to L2 and 69 MB to HBM.
template <int LAT, int D>
__global__ __launch_bounds__(kThreads) void latent_output_kernel(LatentProjParams p) {
  constexpr int NB = D / 64;  // 16-row blocks of W per wave
  const LatentRows rows = listed(p, p.rows);
  const int hd = blockIdx.y;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, n = lane & 15, g = lane >> 4;
  // rows of W so that a lane's results are 4 NB dims side by side
  const uint16_t* w = p.w + ((size_t)hd * D + wave * (D / 4) + n / 4 * (4 * NB) + n % 4) * LAT + 8 * g;
  const uint16_t* x[4];
  f32x4 acc[4][NB];
#pragma unroll
  for (int tb = 0; tb < 4; tb++) {
    const int t = tb * 16 + n;
    x[tb] = p.in + ((size_t)(rows.own0 + (t < rows.ntok ? t : 0)) * p.num_q_heads + hd) * LAT + 8 * g;
#pragma unroll
    for (int b = 0; b < NB; b++) acc[tb][b] = f32x4{};
  }
#pragma unroll 8
  for (int ks = 0; ks < LAT / 32; ks++) {
    bf16x8 a[NB];
#pragma unroll
    for (int b = 0; b < NB; b++) a[b] = *(const bf16x8*)(w + b * 4 * LAT + ks * 32);
#pragma unroll
    for (int tb = 0; tb < 4; tb++) {
      const bf16x8 y = *(const bf16x8*)(x[tb] + ks * 32);
#pragma unroll
      for (int b = 0; b < NB; b++) acc[tb][b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a[b], y, acc[tb][b], 0, 0, 0);
    }
  }
#pragma unroll
  for (int tb = 0; tb < 4; tb++) {
    const int t = tb * 16 + n;
    if (t >= rows.ntok) continue;
    uint16_t* dst = p.out + ((size_t)(rows.row0 + t) * p.num_q_heads + hd) * D + wave * (D / 4) + 4 * NB * g;
    if (p.lse_out != nullptr && wave == 0 && g == 0)
      p.lse_out[(size_t)(rows.row0 + t) * p.num_q_heads + hd] = p.lse_in[(size_t)(rows.own0 + t) * p.num_q_heads + hd];
#pragma unroll
    for (int b = 0; b < NB; b++) {
      uint2 y;
      y.x = pack_bf16(acc[tb][b][0], acc[tb][b][1]);
      y.y = pack_bf16(acc[tb][b][2], acc[tb][b][3]);
      *(uint2*)(dst + b * 4) = y;
    }
  }
}

// Keys and values of cached tokens: (tokens x latent) times (latent x 2 head_dim) per head.
// Workgroup = 4 waves of 64 tokens each, whose latents stay in registers (the accumulator
// half) while the weights of one head after the other, W_uk and W_uv in turn, come through
// LDS: 128 latent dims of one of them a stage, four stages, so that a stage is loaded under
// the products of the two before and operand reads run on across the border.  A wave's results
// are 32 x 32 blocks, four of a weight's rows by two of tokens: each operand read feeds two
// products, half of what LDS can deliver (tokens through LDS as well, shared by two waves: reads
// at the rate of the products, 1260 us where this takes 1044; three
// stages 1071).  Bound by the matrix unit: 246k tokens x 16 heads at 0.99 PFLOP/s.
//
// LDS layout of a stage: for each 64 of its dims, groups of 8 weight rows, [8 rows][128 bytes]
// each, filled by one wave-wide direct load; 16-byte chunk c of row r is stored at
// c ^ wswz(r): the rows that 16 lanes read together differ in row bits 1, 2 and 4.
constexpr int kExpStages = 4;
__device__ __forceinline__ int wswz(int r) { return ((r >> 1) & 3) | ((r >> 2) & 4); }

template <int LAT, int D, bool FP8>
__global__ __launch_bounds__(kThreads, 1) void latent_expand_kernel(LatentExpandParams p) {
  constexpr int MB = D / 32;        // 32-row blocks of a weight
  constexpr int KS = LAT / 16;      // steps of 16 latent dims
  constexpr int SK = 8;             // ... of a stage
  constexpr int STEPS = KS / SK;    // stages of a weight
  constexpr int N = SK * MB;        // operand reads of a stage
  constexpr int AK = 6;             // reads ahead of their products
  constexpr int STAGE = D * 256, PIECES = D / 16;  // bytes; loads of a wave
  __shared__ __attribute__((aligned(1024))) uint8_t lds[kExpStages * STAGE];
  const LatentExpandUnit u = listed(p, p.units);
  const int head0 = blockIdx.y * p.heads_per, heads = p.heads - head0 < p.heads_per ? p.heads - head0 : p.heads_per;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n = lane & 31, h = lane >> 5;
  const int32_t* ids = p.pool.page_ids + u.page_base;
  const int last = u.key_end - 1;

  const int w_off = (lane >> 3) * (LAT * 2) + (((lane & 7) ^ ((lane >> 4) & 3)) << 4);
  const uint32_t base = lds_address(lds);
  const int total = heads * 2 * STEPS;
  // stage i: head head0 + i / (2 STEPS), W_uk or W_uv, latent dims 128 (i % STEPS) ..
  auto issue = [&](int i, uint32_t to) {
    const int hd = head0 + i / (2 * STEPS);
    const uint16_t* w = (i / STEPS & 1 ? p.w_uv : p.w_uk) + (size_t)hd * D * LAT + i % STEPS * 128;
#pragma unroll
    for (int j = 0; j < PIECES; j++) {
      const int q = wave * PIECES + j, sub = q / (D / 8), gr = q % (D / 8);
      lds_load_1k((const uint8_t*)(w + gr * 8 * LAT + sub * 64), w_off ^ ((gr >> 1) & 1) << 6, to + q * 1024);
    }
  };
  issue(0, base);
  issue(1, base + STAGE);
  issue(2, base + 2 * STAGE);

  if (p.rx != nullptr && blockIdx.y == 0) {
    for (int i = tid; i < u.nrows * 8; i += kThreads) {
      const int r = i / 8, c = i % 8, key = u.key0 + r < last ? u.key0 + r : last;
      const uint8_t* page = p.pool.base + (int64_t)ids[key / kPageSize] * p.pool.page_bytes;
      const uint8_t* src = FP8 ? page + kPageSize * LAT + (key % kPageSize) * (2 * kLatRope)
                               : page + (key % kPageSize) * (2 * (LAT + kLatRope)) + 2 * LAT;
      *(uint4*)(p.rx + (size_t)(u.x_row + r) * kLatRope + c * 8) = *(const uint4*)(src + c * 16);
    }
  }

  // Latents: 8 values of step ks are chunk 4 (ks / 2) + 2 h + ks % 2, so that a lane's values of
  // two steps are side by side (16 codes of an 8-bit pool).
  bf16x8 x[2][KS];
#pragma unroll
  for (int t = 0; t < 2; t++) {
    const int r = u.key0 + wave * 64 + t * 32 + n, key = r < last ? r : last, slot = key % kPageSize;
    const uint8_t* page = p.pool.base + (int64_t)ids[key / kPageSize] * p.pool.page_bytes;
#pragma unroll
    for (int j = 0; j < KS / 2; j++) {
      if constexpr (FP8) {
        const uint4 codes = *(const uint4*)(page + slot * LAT + j * 32 + h * 16);
        const uint8_t sc = page[kPageSize * (LAT + 2 * kLatRope) + latent_scale_at(LAT, slot, j / 2)];
        const float s = __uint_as_float((uint32_t)sc << 23);
        const uint32_t w[4] = {codes.x, codes.y, codes.z, codes.w};
        uint32_t y[8];
#pragma unroll
        for (int e = 0; e < 4; e++) {
          y[2 * e] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[e], s, false));
          y[2 * e + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[e], s, true));
        }
        x[t][2 * j] = __builtin_bit_cast(bf16x8, make_uint4(y[0], y[1], y[2], y[3]));
        x[t][2 * j + 1] = __builtin_bit_cast(bf16x8, make_uint4(y[4], y[5], y[6], y[7]));
      } else {
        const uint4* src = (const uint4*)(page + slot * (2 * (LAT + kLatRope)) + j * 64 + h * 32);
        x[t][2 * j] = __builtin_bit_cast(bf16x8, src[0]);
        x[t][2 * j + 1] = __builtin_bit_cast(bf16x8, src[1]);
      }
    }
  }
#pragma unroll
  for (int t = 0; t < 2; t++)
#pragma unroll
    for (int ks = 0; ks < KS; ks++) keep_in_acc(x[t][ks]);

  // Weight row of MFMA row m: lane (n, h) of the result then holds 16 values side by side.
  const int mw = (n & 3) | ((n & 4) << 2) | ((n >> 1) & 12);
  uint32_t wat[4];
#pragma unroll
  for (int ks = 0; ks < 4; ks++) {
    wat[ks] = base + mw * 128 + (((4 * (ks / 2) + 2 * h + ks % 2) ^ wswz(mw)) << 4);
    opaque(wat[ks]);
  }
  bf16x8 ka[AK + 1];
  auto read = [&](uint32_t st, int j) {  // 32-row block j % MB of step j / MB
    const int ks = j / MB;
    return read_b128(lds_at(wat[ks & 3] + st) + (ks >> 2) * (D * 128) + j % MB * 4096);
  };
  wait_vmcnt<0>();
  __syncthreads();
#pragma unroll
  for (int j = 0; j < AK; j++) ka[j] = read(0, j);
  // Results are packed at the end of a weight and stored, a piece at a time, beside the first
  // products of the next.
  constexpr int STORES = 4 * MB;
  const bool stores = wave * 64 < u.nrows;  // uniform: rows come in multiples of 64
  uint32_t y[2][MB][8];
  uint16_t* out = nullptr;
  auto store = [&](int k) {
    const int t = k / (2 * MB), b = k / 2 % MB, e = k % 2 * 4;
    *(uint4*)(out + (size_t)t * 32 * D + b * 32 + e * 2) = make_uint4(y[t][b][e], y[t][b][e + 1], y[t][b][e + 2], y[t][b][e + 3]);
  };
  uint32_t st = 0;
  int i = 0;
  for (int hv = 0; hv < heads * 2; hv++) {
    const bool pending = hv > 0 && stores;
    f32x16 acc[MB][2];
#pragma unroll
    for (int b = 0; b < MB; b++) acc[b][0] = acc[b][1] = f32x16{};
#pragma unroll
    for (int s = 0; s < STEPS; s++, i++) {
      const uint32_t next = st == (kExpStages - 1) * STAGE ? 0 : st + STAGE;
#pragma unroll
      for (int j = 0; j < N; j++) {
        const int at = s * N + j;
        if (j == N - AK) {
          // Stage i + 1 is whole, and every wave is past stage i - 1, whose place i + 3 takes.
          // Newer than its loads are those of stage i + 2 and the stores since.
          __builtin_amdgcn_sched_barrier(0);
          if (i + 2 >= total) wait_vmcnt<0>();
          else if (s < 2 && pending) wait_vmcnt<PIECES + STORES>();
          else wait_vmcnt<PIECES>();
          __syncthreads();
          if (i + 3 < total) issue(i + 3, base + (st == 0 ? (kExpStages - 1) * STAGE : st - STAGE));
          __builtin_amdgcn_sched_barrier(0);
        }
        ka[(at + AK) % (AK + 1)] = j + AK < N ? read(st, j + AK) : read(next, j + AK - N);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int t = 0; t < 2; t++)
          acc[j % MB][t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ka[at % (AK + 1)], x[t][s * SK + j / MB],
                                                                   acc[j % MB][t], 0, 0, 0);
        if (s == 0) {
#pragma unroll
          for (int k = 0; k < STORES; k++)
            if (k * (N - AK) / STORES == j && pending) store(k);
        }
        __builtin_amdgcn_sched_barrier(0);
      }
      st = next;
    }
    // the next weight's first operands keep their places whatever STEPS N modulo AK + 1 is
    bf16x8 keep[AK];
#pragma unroll
    for (int j = 0; j < AK; j++) keep[j] = ka[(STEPS * N + j) % (AK + 1)];
#pragma unroll
    for (int j = 0; j < AK; j++) ka[j] = keep[j];
    const int hd = head0 + hv / 2;
    out = (hv & 1 ? p.vx : p.kx) + ((size_t)hd * p.x_rows + u.x_row + wave * 64 + n) * D + 16 * h;
#pragma unroll
    for (int t = 0; t < 2; t++)
#pragma unroll
      for (int b = 0; b < MB; b++)
#pragma unroll
        for (int e = 0; e < 8; e++) {
          y[t][b][e] = pack_bf16(acc[b][t][2 * e], acc[b][t][2 * e + 1]);
          formed(y[t][b][e]);
        }
  }
  if (stores)
#pragma unroll
    for (int k = 0; k < STORES; k++) store(k);
}

}  // namespace

hipError_t launch_latent_absorb(const LatentProjParams& p, int64_t n_rows, int latent_dim, int head_dim,
                                hipStream_t stream) {
  if (n_rows <= 0) return hipSuccess;
  const dim3 grid((unsigned)n_rows, p.num_q_heads, latent_dim / kSlice), block(kThreads);
  if (latent_dim == 512) {
    if (head_dim == 128) hipLaunchKernelGGL((latent_absorb_kernel<512, 128>), grid, block, 0, stream, p);
    else hipLaunchKernelGGL((latent_absorb_kernel<512, 64>), grid, block, 0, stream, p);
  } else {
    if (head_dim == 128) hipLaunchKernelGGL((latent_absorb_kernel<256, 128>), grid, block, 0, stream, p);
    else hipLaunchKernelGGL((latent_absorb_kernel<256, 64>), grid, block, 0, stream, p);
  }
  return hipGetLastError();
}

hipError_t launch_latent_output(const LatentProjParams& p, int64_t n_rows, int latent_dim, int head_dim,
                                hipStream_t stream) {
  if (n_rows <= 0) return hipSuccess;
  const dim3 grid((unsigned)n_rows, p.num_q_heads), block(kThreads);
  if (latent_dim == 512) {
    if (head_dim == 128) hipLaunchKernelGGL((latent_output_kernel<512, 128>), grid, block, 0, stream, p);
    else hipLaunchKernelGGL((latent_output_kernel<512, 64>), grid, block, 0, stream, p);
  } else {
    if (head_dim == 128) hipLaunchKernelGGL((latent_output_kernel<256, 128>), grid, block, 0, stream, p);
    else hipLaunchKernelGGL((latent_output_kernel<256, 64>), grid, block, 0, stream, p);
  }
  return hipGetLastError();
}

template <int LAT, int D>
static void expand_by_type(const LatentExpandParams& p, dim3 grid, bool fp8, hipStream_t stream) {
  if (fp8) hipLaunchKernelGGL((latent_expand_kernel<LAT, D, true>), grid, dim3(kThreads), 0, stream, p);
  else hipLaunchKernelGGL((latent_expand_kernel<LAT, D, false>), grid, dim3(kThreads), 0, stream, p);
}

hipError_t launch_latent_expand(const LatentExpandParams& p0, int64_t n_units, int latent_dim, int head_dim, bool fp8,
                                hipStream_t stream) {
  if (n_units <= 0) return hipSuccess;
  LatentExpandParams p = p0;
  // Heads per workgroup: the number that ends first, where one workgroup a CU takes a head at
  // a time and half a head's time to load its tokens
  double least = HUGE_VAL;
  for (int32_t per = 1; per <= p.heads; per++) {
    const int64_t wgs = n_units * ((p.heads + per - 1) / per);
    const double t = (double)((wgs + 255) / 256) * (per + 0.5);
    if (t <= least) {
      least = t;
      p.heads_per = per;
    }
  }
  const dim3 grid((unsigned)n_units, (unsigned)((p.heads + p.heads_per - 1) / p.heads_per));
  if (latent_dim == 512) {
    if (head_dim == 128) expand_by_type<512, 128>(p, grid, fp8, stream);
    else expand_by_type<512, 64>(p, grid, fp8, stream);
  } else {
    if (head_dim == 128) expand_by_type<256, 128>(p, grid, fp8, stream);
    else expand_by_type<256, 64>(p, grid, fp8, stream);
  }
  return hipGetLastError();
}

}  // namespace kvx
