// Microscaled 4-bit rounding, the norm that stands before a projection, and the codes as values.
//
// mx_quant: u = post . (c_b H_b (pre . x)) in fp32 (the prologue's butterfly and stage order, each
// product one rounding), then per block of 32 channels the scale 2^e, e = floor(log2 max |u|) - 2, and
// the nearest E2M1 value of u 2^-e.  No reduction is wider than a block, so rows are not looked
// at: threads take 16-channel chunks of all rows in a row, and a b-block is b / 16 lanes of a
// 16-lane group, as in the prologue.  Bound by memory and by the vector unit alike: 4095 x 16384 bf16 (170 MB) takes 32 us in a
// graph with b = 128, 5.4 TB/s, what a large copy reaches, but 26 us without a rotation (caches hold part of such a repeated
// call's rows); a wave issues 362 vector instructions for 16 channels a lane (SQ_INSTS_VALU), a SIMD one in 3.1 of its busy cycles.
// One fold 39 us and both 42 (a trace of eager calls: 37, 44, 58): 17 instructions each, and most of it waiting (a wave's cycles grow
// by 25% and 73%, all and three quarters of that in SQ_WAIT_ANY), since every row reads them again from the L2, 4 bytes a channel
// to its own 2.5.
// Two rows a thread share the folds, 1 to 4 us less, but take 5 to 10% more for every call under 30 us, and four rows are slower
// still.  16384 x 2048 fp32 25 us, 6.2 TB/s.  50 x 1024 takes 2.7 us, of which a launch with a load and a store is 2.2.
//
// norm: h = bf16(x + r); s = 1 / sqrt(mean h^2 + eps) with the sum and the root in fp64 (a bf16's
// square is exact there and the sum all but exact, so s does not depend on the order and the codes can
// be reproduced bit for bit; in fp32 every order gives other last bits, and other codes next to a
// tie); y = (h s) w; then the prologue's transform and rounding, or mx_quant's.  A row stays in
// registers between its two reductions, so it is read once.  Bound by memory: 16383 x 4096 to 8 bits with a residual (470 MB)
// 89 us in a graph, 5.3 TB/s (to 4 bits 85, microscaled 88); 816 x 2048 5.4 us, 50 x 1024 3.7.  One row of 2048 takes 3.7 us: the
// rows' way from memory, the sum over lanes and waves (lane moves instead of the LDS crossbar, 0.3 us), fp64 division and root, the
// gain's way, the largest value.
//
// read: code times scale in fp32, rounded to bf16 (microscaled values are exact in it).  16383 x 4096 8-bit codes (201 MB) 32 us in
// a graph, 6.3 TB/s, 35 after the norm that wrote them; microscaled 4095 x 16384 (170 MB) 27 us, 6.3 TB/s.
#include "fq_codes.hpp"
#include "fq_launch.hpp"
#include "fq_mx.hpp"

namespace fq {

namespace {

struct MxQuantParams {
  const void *x;
  int64_t ldx;
  const float *pre, *post;
  int64_t M, row0;      // rows of the whole call, first row of this launch
  uint32_t chunks;      // chunks of this launch
  uint32_t per_row;     // chunks of a row
  uint32_t magic;       // floor(x / per_row) = (x magic) >> 23 for x < 2^12
  int log2b;
  float cb;
  uint8_t *codes;
  uint32_t *scales;
};

constexpr int kQuantThreads = 256;

template <typename Tin>
__global__ __launch_bounds__(kQuantThreads) void mx_quant_kernel(MxQuantParams p) {
  const int tid = threadIdx.x, tau = tid & 15;
  const uint32_t first = blockIdx.x * (uint32_t)kQuantThreads;
  const uint32_t row_first = first / p.per_row;
  const uint32_t x = first - row_first * p.per_row + (uint32_t)((tid & ~15) | mx_chunk(tau));
  const uint32_t down = (x * p.magic) >> 23;
  const int chunk = (int)(x - down * p.per_row);
  const bool in = first + (uint32_t)((tid & ~15) | mx_chunk(tau)) < p.chunks;  // whole steps: per_row is a multiple of 8
  const int64_t row = p.row0 + (in ? row_first + down : 0);

  Chunk<Tin> raw;
  load_chunk<Tin>(p.x, row * p.ldx + (int64_t)chunk * 16, raw);
  float v[1][16];
  unpack_chunk<Tin>(raw, v[0]);
  if (p.pre) {
    float4 m[4];
    load_mult(p.pre, chunk, m);
    mul_chunk(v[0], m);
  }
  if (p.log2b) {
    const float f = mx_transform<1>(v, p.log2b, tau) * p.cb;
#pragma unroll
    for (int i = 0; i < 16; ++i) v[0][i] *= f;
  }
  if (p.post) {
    float4 m[4];
    load_mult(p.post, chunk, m);
    mul_chunk(v[0], m);
  }
  const uint32_t byte = mx_scale_byte(block_max(v[0]));
  const uint2 code = mx_pack16(v[0], byte);
  const uint32_t word = step_scales(byte, tau);
  if (in) {
    *reinterpret_cast<uint2 *>(p.codes + (row * p.per_row + chunk) * 8) = code;
    if ((tau & 11) == 0) p.scales[mx_scale_word(row, p.M, chunk >> 3)] = word;
  }
}

// ---------------- norm ----------------

struct NormParams {
  NormArgs a;
  int64_t row0;  // first row of this launch
  int log2b, tpr_log2;
  float qf;
};

// The other lane's double, halves through the lane moves of 32 bits.
template <int M>
__device__ __forceinline__ double lane_xor_f64(double v) {
  const uint64_t u = __builtin_bit_cast(uint64_t, v);
  const uint32_t lo = __float_as_uint(lane_xor<M>(__uint_as_float((uint32_t)u)));
  const uint32_t hi = __float_as_uint(lane_xor<M>(__uint_as_float((uint32_t)(u >> 32))));
  return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}

// A row is held by TPR = 2^tpr_log2 >= 16 consecutive threads, thread tau owning CPT chunks
// c TPR + mx_chunk(tau).
template <int CPT, int NT, int OUT>
__global__ __launch_bounds__(NT) void norm_quant_kernel(NormParams p) {
  constexpr int NWAVES = NT / kWave;
  __shared__ double red_sum[NWAVES];
  __shared__ float red_max[NWAVES];
  const int tid = threadIdx.x;
  const int TPR = 1 << p.tpr_log2;
  const int row_local = tid >> p.tpr_log2;
  const int tau = tid & (TPR - 1), t16 = tid & 15;
  const int lam = (tau & ~15) | mx_chunk(t16);
  const int64_t row = p.row0 + (int64_t)blockIdx.x * (NT >> p.tpr_log2) + row_local;
  const bool row_ok = row < p.a.M;
  const int nchunks = p.a.K >> 4;
  const int w0 = (row_local << p.tpr_log2) / kWave, nw = TPR / kWave;

  Chunk<uint16_t> raw[CPT], res[CPT];
#pragma unroll
  for (int c = 0; c < CPT; ++c) {
    const int j = c * TPR + lam;
    const bool in = row_ok && j < nchunks;
#pragma unroll
    for (int i = 0; i < 2; ++i) raw[c].u[i] = res[c].u[i] = make_uint4(0, 0, 0, 0);
    if (in) {
      load_chunk<uint16_t>(p.a.x, row * p.a.ldx + (int64_t)j * 16, raw[c]);
      if (p.a.residual) load_chunk<uint16_t>(p.a.residual, row * p.a.ldr + (int64_t)j * 16, res[c]);
    }
  }

  // the gain asked for before the sum where few rows hide its way (16384 channels, 816 rows 23.5 -> 22.3 us); with a chunk
  // a thread its registers cost more (816 rows of 2048 6.0 us, else 5.4)
  constexpr bool EARLY = CPT > 1;
  float4 gain[CPT][4];
  auto load_gain = [&] {
#pragma unroll
    for (int c = 0; c < CPT; ++c) load_mult(p.a.weight, c * TPR + lam < nchunks ? c * TPR + lam : 0, gain[c]);
  };
  if (EARLY) load_gain();

  float v[CPT][16];
  double sum = 0.0;
#pragma unroll
  for (int c = 0; c < CPT; ++c) {
    const int j = c * TPR + lam;
    unpack_chunk<uint16_t>(raw[c], v[c]);
    if (p.a.residual) {
      float r[16];
      unpack_chunk<uint16_t>(res[c], r);
      uint32_t h[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        h[i] = f32_to_bf16(v[c][2 * i] + r[2 * i]) | (f32_to_bf16(v[c][2 * i + 1] + r[2 * i + 1]) << 16);
        v[c][2 * i] = bf16_lo(h[i]);
        v[c][2 * i + 1] = bf16_hi(h[i]);
      }
      if (p.a.sum && row_ok && j < nchunks) {
        uint4 *out = reinterpret_cast<uint4 *>(static_cast<uint16_t *>(p.a.sum) + row * p.a.lds + (int64_t)j * 16);
        out[0] = make_uint4(h[0], h[1], h[2], h[3]);
        out[1] = make_uint4(h[4], h[5], h[6], h[7]);
      }
    }
#pragma unroll
    for (int i = 0; i < 16; ++i) sum = __builtin_fma((double)v[c][i], (double)v[c][i], sum);
  }
  // the row's sum: its lanes, then its waves
  const int lim = TPR < kWave ? TPR : kWave;
  sum += lane_xor_f64<1>(sum);
  sum += lane_xor_f64<2>(sum);
  sum += lane_xor_f64<4>(sum);
  sum += lane_xor_f64<8>(sum);
  if (lim > 16) sum += lane_xor_f64<16>(sum);
  if (lim > 32) sum += __shfl_xor(sum, 32, kWave);
  if (TPR > kWave) {
    if ((tid & (kWave - 1)) == 0) red_sum[tid / kWave] = sum;
    __syncthreads();
    sum = red_sum[w0];
    for (int w = 1; w < nw; ++w) sum += red_sum[w0 + w];
  }
  const float scale = (float)(1.0 / __builtin_sqrt(sum / (double)p.a.K + (double)p.a.eps));

  if (!EARLY) load_gain();
#pragma unroll
  for (int c = 0; c < CPT; ++c) {
#pragma unroll
    for (int i = 0; i < 16; ++i) v[c][i] *= scale;
    mul_chunk(v[c], gain[c]);
  }
  const float sgn = mx_transform<CPT>(v, p.log2b, t16);
  if constexpr (OUT == kOutMx) {
    if (p.log2b) {
      const float f = sgn * p.a.cb;
#pragma unroll
      for (int c = 0; c < CPT; ++c)
#pragma unroll
        for (int i = 0; i < 16; ++i) v[c][i] *= f;
    }
  }
  if (p.a.post) {
#pragma unroll
    for (int c = 0; c < CPT; ++c) {
      const int j = c * TPR + lam;
      float4 m[4];
      load_mult(p.a.post, j < nchunks ? j : 0, m);
      mul_chunk(v[c], m);
    }
  }

  if constexpr (OUT == kOutMx) {
#pragma unroll
    for (int c = 0; c < CPT; ++c) {
      const int j = c * TPR + lam;
      const uint32_t byte = mx_scale_byte(block_max(v[c]));
      const uint2 code = mx_pack16(v[c], byte);
      const uint32_t word = step_scales(byte, t16);
      if (row_ok && j < nchunks) {
        *reinterpret_cast<uint2 *>(p.a.codes + (row * nchunks + j) * 8) = code;
        if ((t16 & 11) == 0) reinterpret_cast<uint32_t *>(p.a.scales)[mx_scale_word(row, p.a.M, j >> 3)] = word;
      }
    }
  } else {
    float amax = 0.0f;
#pragma unroll
    for (int c = 0; c < CPT; ++c)
      if (c * TPR + lam < nchunks) {
#pragma unroll
        for (int i = 0; i < 16; i += 2) amax = abs_maximum(amax, v[c][i], v[c][i + 1]);
      }
    amax = maximum(amax, lane_xor<1>(amax));
    amax = maximum(amax, lane_xor<2>(amax));
    amax = maximum(amax, lane_xor<4>(amax));
    amax = maximum(amax, lane_xor<8>(amax));
    if (lim > 16) amax = maximum(amax, lane_xor<16>(amax));
    if (lim > 32) amax = maximum(amax, __shfl_xor(amax, 32, kWave));
    if (TPR > kWave) {
      if ((tid & (kWave - 1)) == 0) red_max[tid / kWave] = amax;
      __syncthreads();
      amax = red_max[w0];
      for (int w = 1; w < nw; ++w) amax = maximum(amax, red_max[w0 + w]);
    }
    const float qf = p.qf;
    const float rA = p.a.clip_ratio * amax;
    const bool fine = amax < __builtin_inff();  // a NaN is not
    // a row of zeros, or one so small that the reciprocal overflows, has codes 0 and scale 0
    const bool some = fine && qf / rA < __builtin_inff();
    const float inv = some ? qf / rA : 0.0f;
    if (row_ok && tau == 0)
      p.a.delta[row] = some ? (rA * p.a.cb) / qf : fine ? 0.0f : __builtin_nanf("");
    if (row_ok) {
      const float lim_q = qf + 0.49f, inv_l = inv * sgn;
      const int64_t ld = OUT == kOutNibble ? p.a.K / 2 : p.a.K;
#pragma unroll
      for (int c = 0; c < CPT; ++c) {
        const int j = c * TPR + lam;
        if (j >= nchunks) continue;
        int code[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) code[i] = some ? quantize_bits(v[c][i], inv_l, lim_q) : 0;
        store_chunk_bits(p.a.codes + row * ld, j, code, OUT);
      }
    }
  }
}

// ---------------- codes as values ----------------

struct ReadParams {
  const uint8_t *codes;
  const void *scale;
  int64_t M, row0;
  uint32_t chunks, per_row, magic;
  uint16_t *values;
  int64_t ldv;
};

__device__ __forceinline__ uint32_t pack_bf16(float a, float b) { return f32_to_bf16(a) | (f32_to_bf16(b) << 16); }

// BITS: 4, 8, or 0 for microscaled codes (v_cvt_scalef32_pk_bf16_fp4, exact: two mantissa bits).
template <int BITS>
__global__ __launch_bounds__(kQuantThreads) void read_codes_kernel(ReadParams p) {
  const uint32_t first = blockIdx.x * (uint32_t)kQuantThreads;
  const uint32_t row_first = first / p.per_row;
  const uint32_t x = first - row_first * p.per_row + threadIdx.x;
  const uint32_t down = (x * p.magic) >> 23;
  const int chunk = (int)(x - down * p.per_row);
  if (first + threadIdx.x >= p.chunks) return;
  const int64_t row = p.row0 + row_first + down;
  uint32_t o[8];
  if constexpr (BITS == 8) {
    const uint4 u = *reinterpret_cast<const uint4 *>(p.codes + (row * p.per_row + chunk) * 16);
    const float d = static_cast<const float *>(p.scale)[row];
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const uint32_t q = w[i / 2] << (16 * (1 - (i & 1)));
      o[i] = pack_bf16((float)((int)(q << 8) >> 24) * d, (float)((int)q >> 24) * d);
    }
  } else {
    const uint2 u = *reinterpret_cast<const uint2 *>(p.codes + (row * p.per_row + chunk) * 8);
    const uint32_t w[2] = {u.x, u.y};
    if constexpr (BITS == 4) {
      const float d = static_cast<const float *>(p.scale)[row];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int q = (int)(w[i / 4] << (8 * (3 - (i & 3))));
        o[i] = pack_bf16((float)((q << 4) >> 28) * d, (float)(q >> 28) * d);
      }
    } else {
      const uint8_t *sc = static_cast<const uint8_t *>(p.scale);
      const uint32_t byte = sc[mx_scale_word(row, p.M, chunk >> 3) * 4 + ((chunk >> 1) & 3)];
#if defined(__HIP_DEVICE_COMPILE__)
      const float s = mx_scale_value(byte);
#define FQ_UP(i, sel) \
  o[i] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w[i / 4], s, sel))
      FQ_UP(0, 0); FQ_UP(1, 1); FQ_UP(2, 2); FQ_UP(3, 3);
      FQ_UP(4, 0); FQ_UP(5, 1); FQ_UP(6, 2); FQ_UP(7, 3);
#undef FQ_UP
#endif
      if (byte == 255) {
#pragma unroll
        for (int i = 0; i < 8; ++i) o[i] = 0x7FC07FC0u;
      }
    }
  }
  uint4 *out = reinterpret_cast<uint4 *>(p.values + row * p.ldv + (int64_t)chunk * 16);
  out[0] = make_uint4(o[0], o[1], o[2], o[3]);
  out[1] = make_uint4(o[4], o[5], o[6], o[7]);
}

// ---------------- packing of weights ----------------

// Tile (nb, kt) of 16 x 128 nibbles: lane l of a wave owns channel l % 16 and the block l / 16, 16 bytes.  Once a weight: 16384 x
// 2048 (17 MB each way) 6 us, 16384 x 16384 39 us, 6.9 TB/s (with caches), either way.
__global__ __launch_bounds__(256) void mx_pack_kernel(const uint4 *from, int64_t pieces, int ktot, int unpack, uint4 *to) {
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < pieces; i += (int64_t)gridDim.x * 256) {
    const int64_t tile = i >> 6;
    const int l = (int)(i & 63);
    const int64_t nb = tile / ktot;
    const int kt = (int)(tile - nb * ktot);
    const int64_t flat = (nb * 16 + (l & 15)) * (int64_t)ktot * 4 + kt * 4 + (l >> 4);
    if (unpack) to[flat] = from[i];
    else to[i] = from[flat];
  }
}

// The launches of a kernel over 16-channel chunks of rows: chunk numbers of one launch fit 32 bits.
template <typename F>
hipError_t over_chunks(int64_t M, int K, F launch) {
  const uint32_t per_row = (uint32_t)K / 16;
  const int64_t most = (int64_t)0xF0000000u / per_row;
  for (int64_t row0 = 0; row0 < M; row0 += most) {
    const int64_t rows = M - row0 < most ? M - row0 : most;
    const uint32_t chunks = (uint32_t)(rows * per_row);
    launch(row0, chunks, per_row, ((1u << 23) - 1) / per_row + 1, (chunks + kQuantThreads - 1) / kQuantThreads);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

template <int CPT, int NT>
hipError_t launch_norm_shape(const NormParams &p, int64_t grid, hipStream_t s) {
  switch (p.a.out_fmt) {
    case kOutNibble:
      hipLaunchKernelGGL((norm_quant_kernel<CPT, NT, kOutNibble>), dim3((unsigned)grid), dim3(NT), 0, s, p);
      break;
    case kOutInt8:
      hipLaunchKernelGGL((norm_quant_kernel<CPT, NT, kOutInt8>), dim3((unsigned)grid), dim3(NT), 0, s, p);
      break;
    case kOutMx:
      hipLaunchKernelGGL((norm_quant_kernel<CPT, NT, kOutMx>), dim3((unsigned)grid), dim3(NT), 0, s, p);
      break;
    default: return hipErrorInvalidValue;
  }
  return hipGetLastError();
}

}  // namespace

hipError_t launch_mx_quant(const MxQuantArgs &a, hipStream_t s) {
  MxQuantParams p{a.x, a.ldx, a.pre, a.post, a.M, 0, 0, 0, 0, log2_of(a.b), a.cb, a.codes,
                  reinterpret_cast<uint32_t *>(a.scales)};
  return over_chunks(a.M, a.K, [&](int64_t row0, uint32_t chunks, uint32_t per_row, uint32_t magic, uint32_t grid) {
    p.row0 = row0;
    p.chunks = chunks;
    p.per_row = per_row;
    p.magic = magic;
    if (a.x_is_f32) hipLaunchKernelGGL(mx_quant_kernel<float>, dim3(grid), dim3(kQuantThreads), 0, s, p);
    else hipLaunchKernelGGL(mx_quant_kernel<uint16_t>, dim3(grid), dim3(kQuantThreads), 0, s, p);
  });
}

hipError_t launch_norm_quant(const NormArgs &a, hipStream_t s) {
  // threads a row and chunks a thread, as the prologue's kernel
  int tpr = 16, cpt = 1, log2 = 0;
  while (tpr < a.K / 16) tpr *= 2;
  if (tpr >= 512) {
    tpr /= 2;
    cpt = 2;
  }
  const int nt = tpr > 256 ? tpr : 256;
  while ((1 << log2) < tpr) ++log2;
  NormParams p{a, 0, log2_of(a.b), log2, a.out_fmt == kOutInt8 ? 127.0f : 7.0f};
  const int64_t most = (1ll << 31) / nt * (nt / tpr);  // rows of a launch, whose threads fit 32 bits
  for (; p.row0 < a.M; p.row0 += most) {
    const int64_t rows = a.M - p.row0 < most ? a.M - p.row0 : most, grid = (rows + nt / tpr - 1) / (nt / tpr);
    const hipError_t e = nt == 256 ? cpt == 1 ? launch_norm_shape<1, 256>(p, grid, s) : launch_norm_shape<2, 256>(p, grid, s)
                         : nt == 512 ? launch_norm_shape<2, 512>(p, grid, s) : launch_norm_shape<2, 1024>(p, grid, s);
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

hipError_t launch_read_codes(const uint8_t *codes, const void *scale, int64_t M, int K, int bits, uint16_t *values,
                             int64_t ldv, hipStream_t s) {
  return over_chunks(M, K, [&](int64_t row0, uint32_t chunks, uint32_t per_row, uint32_t magic, uint32_t grid) {
    const ReadParams p{codes, scale, M, row0, chunks, per_row, magic, values, ldv};
    if (bits == 8) hipLaunchKernelGGL(read_codes_kernel<8>, dim3(grid), dim3(kQuantThreads), 0, s, p);
    else if (bits == 4) hipLaunchKernelGGL(read_codes_kernel<4>, dim3(grid), dim3(kQuantThreads), 0, s, p);
    else hipLaunchKernelGGL(read_codes_kernel<0>, dim3(grid), dim3(kQuantThreads), 0, s, p);
  });
}

hipError_t launch_mx_pack(const uint8_t *from, int64_t N, int K, bool unpack, uint8_t *to, hipStream_t s) {
  const int64_t pieces = N * (K / 32), blocks = (pieces + 255) / 256;
  hipLaunchKernelGGL(mx_pack_kernel, dim3((unsigned)(blocks < 65536 ? blocks : 65536)), dim3(256), 0, s,
                     reinterpret_cast<const uint4 *>(from), pieces, K / 128, (int)unpack, reinterpret_cast<uint4 *>(to));
  return hipGetLastError();
}

}  // namespace fq
