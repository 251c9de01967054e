// Product of microscaled 4-bit codes: y = bf16(sum over blocks 2^(ea + ew - 254) sum a w + bias) on the
// matrix instructions that take E2M1 operands with a scale byte per lane.
#include <cmath>

#include "fq_f6.hpp"
#include "fq_launch.hpp"
#include "fq_mx.hpp"

namespace fq {

namespace {

constexpr int kUnits = 256;  // compute units

// Buffers of the loads below begin where a load's step begins and end where the array's part that a workgroup reads ends, and
// no load has a scalar offset: the hardware compares a buffer's size with the vector offset only, and zeros come back for
// whatever lies behind.

// Steps of 256 channels, the last of which may have 128.
inline int steps_of(int K) { return (K / kTileK + 1) / 2; }

// 16 x 16 x 128: lane l holds row (or column) l % 16 and one block of 32 codes in four words (a format selector of 4 is
// E2M1), any four blocks in the four lane groups as long as both operands have the same; the block's scale is byte SEL
// of sa (sb).
template <int SEL>
__device__ __forceinline__ v4f mfma_mx_16(const v4i &a, int sa, const v4i &b, int sb, v4f c) {
#if defined(__HIP_DEVICE_COMPILE__)
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(v8i{a.x, a.y, a.z, a.w, 0, 0, 0, 0},
                                                          v8i{b.x, b.y, b.z, b.w, 0, 0, 0, 0}, c, 4, 4, SEL, sa, SEL, sb);
#else
  return c;
#endif
}

// The bias of the four columns of a lane's sums in join_waves, asked for before the product: behind it the load costs a
// microsecond and more.
template <int NC>
__device__ __forceinline__ float4 bias_of(const MxGemmArgs &p, int64_t n0, int cols) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), n = 16 * (wave % NC) + 4 * (lane >> 4);
  return p.bias && n < cols ? *reinterpret_cast<const float4 *>(p.bias + n0 + n) : make_float4(0.f, 0.f, 0.f, 0.f);
}

// Every wave's sums side by side; each lane's four columns of one row are added up in the order of the waves.
template <int MT, int NC, int NW>
__device__ __forceinline__ void join_waves(const v4f (&acc)[MT][NC], uint8_t *lds, const MxGemmArgs &p, float4 bias, int64_t m0, int64_t n0,
                                           int rows, int cols) {
  static_assert(NW % NC == 0, "a wave joins tiles of one column block");
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r16 = lane & 15, g = lane >> 4;
  constexpr int TILES = MT * NC;
  float4 *sums = reinterpret_cast<float4 *>(lds);
  __syncthreads();
#pragma unroll
  for (int t = 0; t < MT; ++t)
#pragma unroll
    for (int c = 0; c < NC; ++c)
      sums[(wave * TILES + t * NC + c) * 64 + lane] = make_float4(acc[t][c][0], acc[t][c][1], acc[t][c][2], acc[t][c][3]);
  __syncthreads();
  for (int tile = wave; tile < TILES; tile += NW) {
    float4 v = sums[tile * 64 + lane];
#pragma unroll
    for (int s = 1; s < NW; ++s) {
      const float4 x4 = sums[(s * TILES + tile) * 64 + lane];
      v.x += x4.x;
      v.y += x4.y;
      v.z += x4.z;
      v.w += x4.w;
    }
    const int t = tile / NC, c = tile - t * NC;
    const int m = 16 * t + r16, n = 16 * c + 4 * g;
    if (m >= rows || n >= cols) continue;
    if (p.bias) {
      v.x += bias.x;
      v.y += bias.y;
      v.z += bias.z;
      v.w += bias.w;
    }
    *reinterpret_cast<uint2 *>(p.y + (m0 + m) * p.ldy + n0 + n) =
        make_uint2(f32_to_bf16(v.x) | (f32_to_bf16(v.y) << 16), f32_to_bf16(v.z) | (f32_to_bf16(v.w) << 16));
  }
}

// Few rows: the stream of the weights.  A workgroup has 16 NC columns and 16 MT rows; its NW waves share out K in batches of
// four steps of 128 channels, ask for every load of a batch before they multiply the one ahead, and their sums meet in LDS.
//   In product i of a batch lane group g multiplies block i of step g: a lane's four scale bytes are one word, loaded once.
//   Rows go through the wave's own part of LDS: loaded in operand order (a lane a row) they come at 37 bytes a ns and compute
//   unit, four lanes a row at 120.  Weights are packed in operand order.
//   Weights are the left operand, so that a lane comes to hold four adjacent columns of one row.
// Bound by the way of the weights and by the launch (2.2 us in a graph for the smallest product): one token 2048 to 16384 (18 MB)
// 3.4 us in a graph of the same call, whose weights the caches hold, 3.7 in a trace of eager ones, 4.9 TB/s; 16384 to 2048 5.4; 50
// rows of the same 6.3 (11.8 with rows loaded in operand order and a scale word a step); 48 rows 4096 to 4096 4.1.
template <int MT, int NC, int NW>
__global__ __launch_bounds__(64 * NW) void mx_gemm_stream_kernel(MxGemmArgs p) {
  extern __shared__ __attribute__((aligned(1024))) uint8_t lds[];
  const int tid = threadIdx.x, lane = tid & 63, r16 = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  // The row blocks of a column block lie behind each other on one XCD (workgroup i runs on XCD i % 8), whose L2 then has
  // the weights for all but the first.
  const uint32_t row_blocks = (uint32_t)((p.M + 16 * MT - 1) / (16 * MT)), group = (blockIdx.x >> 3) / row_blocks;
  const int64_t n0 = ((int64_t)group * 8 + (blockIdx.x & 7)) * 16 * NC, m0 = (int64_t)((blockIdx.x >> 3) - group * row_blocks) * 16 * MT;
  if (n0 >= p.N) return;
  const int rows = min((int)p.M - (int)m0, 16 * MT), cols = min((int)p.N - (int)n0, 16 * NC);
  const int ktot = p.K / kTileK, per = ((ktot + 4 * NW - 1) / (4 * NW)) * 4;
  const int k1 = min((wave + 1) * per, ktot);
  int k0 = wave * per;

  const float4 bias = bias_of<NC>(p, n0, cols);
  // A KB of LDS has a step of 16 rows, their four pieces exchanged by (row >> 2) & 3 against bank conflicts.  What lies
  // behind the rows or columns is not stored.
  const uint8_t *a0 = p.a + m0 * (p.K / 2), *w0 = p.w + n0 / 16 * ktot * 1024;
  const int abytes = rows * (p.K / 2), wbytes = cols / 16 * ktot * 1024;
  const uint32_t avoff = (uint32_t)(lane >> 2) * (uint32_t)(p.K / 2) + ((lane & 3) ^ ((lane >> 4) & 3)) * 16u;
  const uint32_t wvoff = g * 1024u + r16 * 16u;
  const uint32_t *sa[MT], *sw[NC];
#pragma unroll
  for (int t = 0; t < MT; ++t) sa[t] = reinterpret_cast<const uint32_t *>(p.a_scale) + m0 + min(16 * t + r16, rows - 1);
#pragma unroll
  for (int c = 0; c < NC; ++c) sw[c] = reinterpret_cast<const uint32_t *>(p.w_scale) + n0 + min(16 * c + r16, cols - 1);
  struct Batch {
    v4i w[NC][4];
    uint32_t sw[NC], sa[MT];
  };
  constexpr int LOADS = 4 * MT + 4 * NC + MT + NC;
  uint8_t *mine = lds + wave * 2 * MT * 4096;
  auto load = [&](Batch &b, int buf, int at) {
    // (a batch behind the wave's share is asked of empty buffers: no branch, so that every wait knows its count)
    const int k = __builtin_amdgcn_readfirstlane(at), on = k < k1 ? -1 : 0;
    const __amdgpu_buffer_rsrc_t wr = buffer_of(w0 + k * 1024, (wbytes - k * 1024) & on);
    __amdgpu_buffer_rsrc_t ar[4];
#pragma unroll
    for (int s = 0; s < 4; ++s) {
      const int off = min(k + s, ktot - 1) * 64;
      ar[s] = buffer_of(a0 + off, (abytes - off) & on);
    }
#pragma unroll
    for (int t = 0; t < MT; ++t)
#pragma unroll
      for (int s = 0; s < 4; ++s)
        buffer_to_lds16(ar[s], avoff + (uint32_t)t * 8u * (uint32_t)p.K, 0, mine + ((buf * MT + t) * 4 + s) * 1024);
#pragma unroll
    for (int c = 0; c < NC; ++c)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        b.w[c][i] = __builtin_amdgcn_raw_buffer_load_b128(wr, wvoff + i * 256u + (uint32_t)c * (uint32_t)ktot * 1024u, 0, 0);
    const int64_t step = min(k + g, ktot - 1);
#pragma unroll
    for (int c = 0; c < NC; ++c) b.sw[c] = sw[c][step * p.N];
#pragma unroll
    for (int t = 0; t < MT; ++t) b.sa[t] = sa[t][step * p.M];
  };
  v4f acc[MT][NC];
#pragma unroll
  for (int t = 0; t < MT; ++t)
#pragma unroll
    for (int c = 0; c < NC; ++c) acc[t][c] = v4f{0.f, 0.f, 0.f, 0.f};
  auto multiply = [&](const Batch &b, int buf, int k) {
    // a step behind the wave's share: scales of 2^-127 both, and their products vanish (its codes are other steps')
    const int on = k + g < k1 ? -1 : 0;
    auto product = [&](auto which) {
      constexpr int i = decltype(which)::value;
#pragma unroll
      for (int t = 0; t < MT; ++t) {
        const v4i a = *reinterpret_cast<const v4i *>(mine + (buf * MT + t) * 4096 + g * 1024 + r16 * 64 + ((i ^ (r16 >> 2)) * 16));
#pragma unroll
        for (int c = 0; c < NC; ++c) acc[t][c] = mfma_mx_16<i>(b.w[c][i], (int)b.sw[c] & on, a, (int)b.sa[t] & on, acc[t][c]);
      }
    };
    static_for<4>(product);
  };
  Batch x, y;
  load(x, 0, k0);
  if (per <= 4) {  // a batch a wave
    wait_vmcnt<0>();
    multiply(x, 0, k0);
    k0 = k1;
  }
  for (int k = k0; k < k1; k += 8) {
    load(y, 1, k + 4);
    wait_vmcnt<LOADS>();
    multiply(x, 0, k);
    lgkm_wait_all();  // the rows are read before others take their place
    load(x, 0, k + 8);
    wait_vmcnt<LOADS>();
    multiply(y, 1, k + 4);
    lgkm_wait_all();
  }
  wait_vmcnt<0>();  // the trailing loads are over: LDS is reused

  join_waves<MT, NC, NW>(acc, lds, p, bias, m0, n0, rows, cols);
}

struct TokenParams {
  MxQuantArgs q;
  MxGemmArgs g;
  int log2b;
};

// One or two tokens from bf16: the streaming kernel with the rounding inside.  While a batch's weights are on their way, its
// wave rounds the same channels of the rows (16 lanes a 256-channel piece, as mx_quant's kernel, so the codes are the same)
// into its part of LDS.  Every workgroup rounds the rows anew, which at this height costs less than a launch: 2048 to 16384
// 4.1 us in a graph and 6.0 to 6.4 as two launches, 1024 to 4096 3.2 and 4.7, 4096 to 4096 4.3 and 5.4.  (The next batch's
// rows and weights asked for ahead cost a single batch 0.2 to 0.6 us more and saved eight 0.9.)
template <int NC, int NW>
__global__ __launch_bounds__(64 * NW) void mx_token_kernel(TokenParams p) {
  constexpr int ROOM = 4096 + 256;  // codes and scale words of 16 rows and a batch
  __shared__ __attribute__((aligned(1024))) uint8_t lds[NW * (ROOM > NC * 1024 ? ROOM : NC * 1024)];
  const int tid = threadIdx.x, lane = tid & 63, r16 = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int64_t n0 = (int64_t)blockIdx.x * 16 * NC;
  const int rows = (int)p.g.M, cols = min((int)p.g.N - (int)n0, 16 * NC);
  const int ktot = p.g.K / kTileK, per = ((ktot + 4 * NW - 1) / (4 * NW)) * 4;
  const int k0 = wave * per, k1 = min(k0 + per, ktot);

  const float4 bias = bias_of<NC>(p.g, n0, cols);
  const uint8_t *w0 = p.g.w + n0 / 16 * ktot * 1024;
  const int wbytes = cols / 16 * ktot * 1024;
  const uint32_t wvoff = g * 1024u + r16 * 16u;
  const uint32_t *sw[NC];
#pragma unroll
  for (int c = 0; c < NC; ++c) sw[c] = reinterpret_cast<const uint32_t *>(p.g.w_scale) + n0 + min(16 * c + r16, cols - 1);
  // lanes 0 to 31 hold the first row's 32 chunks of a batch, the others the second's
  const int row = lane >> 5, piece = (lane & 16) | mx_chunk(r16);
  const int64_t at = (int64_t)min(row, rows - 1) * p.q.ldx;

  struct Rows {
    Chunk<uint16_t> x;
    float4 pre[4], post[4];
  };
  struct Weights {
    v4i w[NC][4];
    uint32_t s[NC];
  };
  auto load = [&](Rows &a, Weights &b, int k) {
    const int j = min(k * 8 + piece, ktot * 8 - 1);
    load_chunk<uint16_t>(p.q.x, at + (int64_t)j * 16, a.x);
    if (p.q.pre) load_mult(p.q.pre, j, a.pre);
    if (p.q.post) load_mult(p.q.post, j, a.post);
    const __amdgpu_buffer_rsrc_t wr = buffer_of(w0 + k * 1024, wbytes - k * 1024);
#pragma unroll
    for (int c = 0; c < NC; ++c)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        b.w[c][i] = __builtin_amdgcn_raw_buffer_load_b128(wr, wvoff + i * 256u + (uint32_t)c * (uint32_t)ktot * 1024u, 0, 0);
#pragma unroll
    for (int c = 0; c < NC; ++c) b.s[c] = sw[c][(int64_t)min(k + g, ktot - 1) * p.g.N];
  };
  uint8_t *mine = lds + wave * ROOM;
  uint32_t *scales = reinterpret_cast<uint32_t *>(mine + 4096);
  auto round = [&](const Rows &a) {
    float v[1][16];
    unpack_chunk<uint16_t>(a.x, v[0]);
    if (p.q.pre) mul_chunk(v[0], a.pre);
    if (p.log2b) {
      const float f = mx_transform<1>(v, p.log2b, r16) * p.q.cb;
#pragma unroll
      for (int i = 0; i < 16; ++i) v[0][i] *= f;
    }
    if (p.q.post) mul_chunk(v[0], a.post);
    const uint32_t byte = mx_scale_byte(block_max(v[0]));
    const uint2 code = mx_pack16(v[0], byte);
    const uint32_t word = step_scales(byte, r16);
    if (row < rows) {
      *reinterpret_cast<uint2 *>(mine + (piece >> 3) * 1024 + row * 64 + (piece & 7) * 8) = code;
      if ((r16 & 11) == 0) scales[(piece >> 3) * 16 + row] = word;
    }
  };
  v4f acc[1][NC];
#pragma unroll
  for (int c = 0; c < NC; ++c) acc[0][c] = v4f{0.f, 0.f, 0.f, 0.f};
  auto multiply = [&](const Weights &b, int k) {
    const int on = k + g < k1 ? -1 : 0;  // as above
    const int r = min(r16, rows - 1);    // (the last row again for all behind it, whose outputs are not stored)
    const uint32_t sa = scales[g * 16 + r];
    auto product = [&](auto which) {
      constexpr int i = decltype(which)::value;
      const v4i a = *reinterpret_cast<const v4i *>(mine + g * 1024 + r * 64 + i * 16);
#pragma unroll
      for (int c = 0; c < NC; ++c) acc[0][c] = mfma_mx_16<i>(b.w[c][i], (int)b.s[c] & on, a, (int)sa & on, acc[0][c]);
    };
    static_for<4>(product);
  };
  Rows a;
  Weights b;
  for (int k = k0; k < k1; k += 4) {
    load(a, b, k);
    round(a);
    wave_lds_fence();
    multiply(b, k);
    wave_lds_fence();
  }
  join_waves<1, NC, NW>(acc, lds, p.g, bias, 0, n0, rows, cols);
}

// 32 x 32 x 64: lane l holds row (or column) l % 32 and block l / 32; its scale is byte SEL of sa (sb).
template <int SEL>
__device__ __forceinline__ v16f mfma_mx_32(const v4i &a, int sa, const v4i &b, int sb, v16f c) {
#if defined(__HIP_DEVICE_COMPILE__)
  return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(v8i{a.x, a.y, a.z, a.w, 0, 0, 0, 0},
                                                         v8i{b.x, b.y, b.z, b.w, 0, 0, 0, 0}, c, 4, 4, SEL, sa, SEL, sb);
#else
  return c;
#endif
}

// 4 bytes per lane (lane l -> dst + 4 l).
__device__ __forceinline__ void buffer_to_lds4(__amdgpu_buffer_rsrc_t r, uint32_t voff, void *dst) {
#if defined(__HIP_DEVICE_COMPILE__)
  __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (__attribute__((address_space(3))) void *)dst, 4, voff, 0, 0, 0);
#else
  (void)r; (void)voff; (void)dst;
#endif
}

typedef float v2f __attribute__((ext_vector_type(2)));
typedef __bf16 v2bf __attribute__((ext_vector_type(2)));

struct TileParams {
  MxGemmArgs g;
  float *partial;   // [splits][M][N], or NULL
  int tiles, ntm, ntn, splits;
  int steps;        // steps of 256 channels of a slice of K (the last slice may have fewer)
};

template <int TI, int TJ, int WM, int WN, int STAGES>
struct TileShape {
  static constexpr int NW = WM * WN, BM = 32 * TI * WM, BN = 32 * TJ * WN;
  static constexpr int A = BM * 128, B = BN * 128, S = (BM + BN) * 8, STAGE = A + B + S;
  static constexpr int STRIDE = 64 * TJ + 16;                       // bytes of a staged output row
  static constexpr int LDS = STAGES * STAGE + NW * 16 * STRIDE;
  static constexpr int IA = A / 1024 / NW, IB = B / 1024 / NW, IS_ALL = S / 256, IS = (IS_ALL + NW - 1) / NW;
  static constexpr int LPS = IA + IB + IS;
  static constexpr int PER_UNIT = 163840 / LDS;  // workgroups of a compute unit
  static_assert(IA * NW * 1024 == A && IB * NW * 1024 == B && BM % 64 == 0 && BN % 64 == 0, "whole loads");
};

// What a workgroup works on: an output tile and a piece of K, in steps of 256 channels from `first` up to `last`.
struct Piece {
  int64_t m0, n0;
  int rows, cols, first, last, split;
};

// Many rows.  Workgroups take pieces blockIdx, blockIdx + gridDim, .. and read them as one stream of steps through a ring in LDS:
// the next piece's first steps arrive while the last ones of this are multiplied and its outputs stored.
// 8191 x 4096 to 16384 with 256 x 256 tiles: 268 to 295 us by card, 3.7 to 4.1 PFLOP/s.  The matrix cores are busy 55% of the
// time, at 1.8 GHz: under random codes the card lowers its clock (the instructions alone reach 5.9 PFLOP/s with them, 8.3
// with zeros).  Of some 3100 cycles a step 2050 are a SIMD's products, and 1150 a unit's reads of LDS and stagings (SQ_LDS_IDX_ACTIVE,
// without what loads write there); waves wait 29% of theirs.  A tile's outputs, staged and stored, are 5 us of 34 in which
// nothing is multiplied.  Measured and slower: weights straight to registers (308 us), steps of 128 channels, one
// or two workgroups a unit (321), outputs stored in pieces of 64 bytes from exchanged operands (313), four waves with tiles of
// 128 x 128, and accumulators in ordinary registers (17%).
// Tiles of 64 x 64 (four waves, two workgroups a unit) are for what fills the card with no more: 382 x 256 to 2496 4.3 us (128 x
// 128 5.3), 2669 x 1280 to 320 5.7 (7.3), 816 x 2048 to 2048 8.8 (9.2); with two workgroups of 128 x 128 the larger shapes lose
// to 256 x 256 all the same.
template <int TI, int TJ, int WM, int WN, int STAGES, bool SPLIT>
__global__ __launch_bounds__(64 * WM * WN) void mx_gemm_tile_kernel(TileParams p) {
  using T = TileShape<TI, TJ, WM, WN, STAGES>;
  extern __shared__ __attribute__((aligned(1024))) uint8_t lds[];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int K = p.g.K, ktot = K / kTileK, steps_all = (ktot + 1) / 2, total = p.tiles * p.splits;
  auto piece_of = [&](int lin) {
    Piece c;
    c.split = __builtin_amdgcn_readfirstlane(lin / p.tiles);
    int tm, tn;
    tile_of(lin - c.split * p.tiles, p.tiles, p.ntm, p.ntn, tm, tn);
    c.m0 = (int64_t)__builtin_amdgcn_readfirstlane(tm) * T::BM;
    c.n0 = (int64_t)__builtin_amdgcn_readfirstlane(tn) * T::BN;
    c.rows = min((int)p.g.M - (int)c.m0, T::BM);
    c.cols = min((int)p.g.N - (int)c.n0, T::BN);
    c.first = c.split * p.steps;
    c.last = min(c.first + p.steps, steps_all);
    return c;
  };

  // Ring loads of one step: rows in KBs of 8 rows x 128 bytes, their 16-byte pieces exchanged by (row >> 1) & 7; weight
  // tiles as they lie; scale words of both halves of the step, rows then columns.  What lies behind the
  // matrices comes back as zeros.  Where K ends inside a step, the second half's codes are others' (finite, as all
  // codes) and its scale bytes are made zeros: products of 2^-254, which vanish.
  // (offsets of a load are added up where it goes out: held in registers they cost 8 and more)
  uint32_t avoff[2], lane16 = lane * 16u;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int row = (wave * T::IA + i) * 8 + (lane >> 3);
    avoff[i] = (uint32_t)row * (uint32_t)(K / 2) + ((lane & 7) ^ ((row >> 1) & 7)) * 16u;
  }

  // The step that is loaded next: it walks through this workgroup's pieces, and comes to read empty buffers.
  const int64_t msteps = p.g.M * 4, nsteps = p.g.N * 4;  // bytes of a step's scale words
  Piece from = piece_of(blockIdx.x);
  int from_lin = blockIdx.x, from_step = from.first, a_bytes, w_bytes;
  const uint8_t *from_a, *from_w, *from_sa, *from_sw;
  auto turn = [&] {
    from_a = p.g.a + from.m0 * (K / 2) + from.first * 128;
    from_w = p.g.w + from.n0 / 16 * ktot * 1024 + from.first * 2048;
    from_sa = p.g.a_scale + 2 * from.first * msteps + from.m0 * 4;
    from_sw = p.g.w_scale + 2 * from.first * nsteps + from.n0 * 4;
    a_bytes = from.rows * (K / 2) - from.first * 128;
    w_bytes = from.cols / 16 * ktot * 1024 - from.first * 2048;
  };
  turn();
  auto advance = [&] {
    from_sa += 2 * msteps;
    from_sw += 2 * nsteps;
    if (++from_step < from.last) {
      from_a += 128;
      from_w += 2048;
      a_bytes -= 128;
      w_bytes -= 2048;
      return;
    }
    from_lin += gridDim.x;
    if (from_lin < total) {
      from = piece_of(from_lin);
      from_step = from.first;
      turn();
    } else {
      from.rows = from.cols = a_bytes = w_bytes = 0;
    }
  };
  auto issue = [&](int slot, int q) {
    uint8_t *st = lds + slot * T::STAGE;
    if (q < T::IA) {
      buffer_to_lds16(buffer_of(from_a, a_bytes), avoff[q & 1] + (uint32_t)(q >> 1) * 8u * (uint32_t)K, 0, st + (wave * T::IA + q) * 1024);
    } else if (q < T::IA + T::IB) {
      const int kb = wave * T::IB + q - T::IA;
      buffer_to_lds16(buffer_of(from_w, w_bytes), lane16 + (uint32_t)(kb >> 1) * (uint32_t)ktot * 1024u + (kb & 1) * 1024u, 0,
                      st + T::A + kb * 1024);
    } else {
      const int idx = min(wave * T::IS + q - T::IA - T::IB, T::IS_ALL - 1);
      const bool is_b = idx >= T::BM / 32;
      const int j = is_b ? idx - T::BM / 32 : idx, per = (is_b ? T::BN : T::BM) / 64;
      const int h = j >= per ? 1 : 0, part = j - h * per;
      const uint8_t *src = (is_b ? from_sw : from_sa) + (h ? (is_b ? nsteps : msteps) : 0);
      const int bytes = 2 * from_step + h < ktot ? 4 * (is_b ? from.cols : from.rows) : 0;
      buffer_to_lds4(buffer_of(src, bytes), (lane16 >> 2) + (uint32_t)part * 256u, st + T::A + T::B + idx * 256);
    }
  };

  // Operands of chunk q (64 channels): lane l takes row (or column) l % 32 and block 2 q + l / 32; its scale is byte
  // 2 (q % 2) of the word of half q / 2, shifted by l / 32 bytes.
  const int u = lane >> 5, r32 = lane & 31;
  const int wm = wave / WN, wn = wave - wm * WN;
  const int arow = wm * 32 * TI + r32;
  int abase = arow * 128 + ((u ^ ((r32 >> 1) & 7)) * 16);
  int bbase = T::A + wn * TJ * 4096 + (r32 >> 4) * 2048 + u * 256 + (r32 & 15) * 16;
  int sabase = T::A + T::B + arow * 4, sbbase = T::A + T::B + T::BM * 8 + (wn * 32 * TJ + r32) * 4;
  v4i ra[2][TI], rb[2][TJ];
  int sa[2][TI], sb[2][TJ];
  constexpr int NRD = TI + TJ;
  auto read = [&](int set, int slot, int q, int r) {  // in the order the products want them
    const uint8_t *st = lds + slot * T::STAGE;
    if (r >= 1 && r <= TI) {
      ra[set][r - 1] = *reinterpret_cast<const v4i *>(st + (abase ^ (q * 32)) + (r - 1) * 4096);
      if ((q & 1) == 0) sa[q >> 1][r - 1] = *reinterpret_cast<const int *>(st + sabase + (q >> 1) * T::BM * 4 + (r - 1) * 128);
    } else {
      const int j = r == 0 ? 0 : r - TI;
      rb[set][j] = *reinterpret_cast<const v4i *>(st + bbase + (q >> 1) * 1024 + (q & 1) * 512 + j * 4096);
      if ((q & 1) == 0) sb[q >> 1][j] = *reinterpret_cast<const int *>(st + sbbase + (q >> 1) * T::BN * 4 + j * 128);
    }
  };
  v16f acc[TI][TJ];
  auto pin = [&](v16f (&a)[TJ]) {
    __builtin_amdgcn_sched_barrier(0);
#if defined(__HIP_DEVICE_COMPILE__)
#pragma unroll
    for (int j = 0; j < TJ; ++j) asm volatile("" : "+a"(a[j]));
#endif
  };
  auto clear = [&] {
#pragma unroll
    for (int i = 0; i < TI; ++i)
#pragma unroll
      for (int j = 0; j < TJ; ++j)
#pragma unroll
        for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.0f;
#pragma unroll
    for (int i = 0; i < TI; ++i) pin(acc[i]);
  };
  int there = -1;  // 0: the step's second half lies behind K
  auto product = [&](auto chunk, int i, int j) {
    constexpr int q = decltype(chunk)::value;
    // where a word is first used: its read has landed
    if (q % 2 == 0 && j == 0) sa[q >> 1][i] = (q ? sa[1][i] & there : sa[0][i]) >> (8 * u);
    if (q % 2 == 0 && i == 0) sb[q >> 1][j] = (q ? sb[1][j] & there : sb[0][j]) >> (8 * u);
    acc[i][j] = mfma_mx_32<2 * (q & 1)>(ra[q & 1][i], sa[q >> 1][i], rb[q & 1][j], sb[q >> 1][j], acc[i][j]);
  };

  // The loads of the step STAGES ahead go out behind the barrier of a step's last chunk, LATE of them in the next
  // step's first.
  constexpr int LATE = T::LPS / 2;
  int slot = 0;
  auto chunk = [&](auto c, auto end) {
    constexpr int q = decltype(c)::value;
    constexpr bool END = decltype(end)::value;
    const int next = slot == STAGES - 1 ? 0 : slot + 1, prev = slot == 0 ? STAGES - 1 : slot - 1;
    int r = 0, g = 0;
#pragma unroll
    for (int t = 0; t < TI * TJ; ++t) {
      __builtin_amdgcn_sched_barrier(0);
      product(c, t % TI, t / TI);
      __builtin_amdgcn_sched_barrier(0);
      if (END && t == 0) {
        // (pinned: the compiler would move this step's products behind the branch in there)
#pragma unroll
        for (int i = 0; i < TI; ++i) pin(acc[i]);
        advance();
        // every read of this step's slot is done; the next step's loads have landed
        wait_vmcnt<(STAGES - 2) * T::LPS>();
        lds_barrier();
      }
      constexpr int ROOM = TI * TJ > 1 ? TI * TJ - 1 : 1, PER = (NRD + ROOM - 1) / ROOM;
#pragma unroll
      for (int h = 0; h < PER; ++h)
        if (r < NRD) read((q + 1) & 1, END ? next : slot, END ? 0 : q + 1, r++);
      constexpr int LPER = (T::LPS - LATE + TI * TJ - 1) / (TI * TJ);
#pragma unroll
      for (int h = 0; h < LPER; ++h) {
        if (q == 0 && g < LATE) issue(prev, T::LPS - LATE + g++);
        if (END && g < T::LPS - LATE) issue(slot, g++);
      }
    }
    if (END) slot = next;
  };
  constexpr std::integral_constant<int, 0> C0{};
  constexpr std::integral_constant<int, 1> C1{};
  constexpr std::integral_constant<int, 2> C2{};
  constexpr std::integral_constant<int, 3> C3{};
  constexpr std::false_type mid{};
  constexpr std::true_type end{};

  Piece cur = from;
#pragma unroll
  for (int s = 0; s < STAGES; ++s) {
#pragma unroll
    for (int q = 0; q < (s == STAGES - 1 ? T::LPS - LATE : T::LPS); ++q) issue(s, q);
    if (s < STAGES - 1) advance();
  }
  wait_vmcnt<(STAGES - 2) * T::LPS + T::LPS - LATE>();
  lds_barrier();
#pragma unroll
  for (int r = 0; r < NRD; ++r) read(0, 0, 0, r);

  clear();
  for (int lin = blockIdx.x, ks = cur.first;;) {
#pragma unroll
    for (int i = 0; i < TI; ++i) pin(acc[i]);
    // the same sums made in every step, not held in a register each over the loop
    asm volatile("" : "+v"(avoff[0]), "+v"(avoff[1]), "+v"(lane16), "+v"(abase), "+v"(bbase), "+v"(sabase), "+v"(sbbase));
    there = 2 * ks + 1 < ktot ? -1 : 0;
    chunk(C0, mid);
    chunk(C1, mid);
    chunk(C2, mid);
    chunk(C3, end);
    if (++ks < cur.last) continue;

    // Lane l holds column l % 32 and rows 8 (e / 4) + 4 (l / 32) + e % 4 of each 32 x 32 tile.
    int el = lane;
    asm volatile("" : "+v"(el));  // keeps the addresses below out of the loop's registers
    const int eu = el >> 5, e32 = el & 31;
    const int rw = wm * 32 * TI, cw = wn * 32 * TJ;
    if constexpr (SPLIT) {
      const int left = cur.rows - rw - 4 * eu, n = cw + e32;
      float *out = p.partial + ((int64_t)cur.split * p.g.M + cur.m0 + rw + 4 * eu) * p.g.N + cur.n0 + n;
#pragma unroll
      for (int i = 0; i < TI; ++i) {
        pin(acc[i]);
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const int k = 32 * i + 8 * (e >> 2) + (e & 3);
#pragma unroll
          for (int j = 0; j < TJ; ++j)
            if (k < left && n + 32 * j < cur.cols) out[k * p.g.N + 32 * j] = acc[i][j][e];
        }
      }
    } else {
      // bf16 rows, 16 at a time, through the wave's own part of LDS, so that they leave in 16-byte pieces
      constexpr int CPR = 4 * TJ, ROWS = 16 / TJ;  // pieces of a row, rows of 64 lanes
      uint8_t *stage = lds + STAGES * T::STAGE + wave * 16 * T::STRIDE;
      uint8_t *to = stage + 4 * eu * T::STRIDE + e32 * 2;
      const uint8_t *of = stage + el / CPR * T::STRIDE + el % CPR * 16;
      const int n = cw + el % CPR * 8, left = n < cur.cols ? cur.rows - rw - el / CPR : 0;
      uint16_t *out = p.g.y + (cur.m0 + rw + el / CPR) * p.g.ldy + cur.n0 + n;
      float bias[TJ];
#pragma unroll
      for (int j = 0; j < TJ; ++j) {  // (816 x 2048 to 16384 takes 23.1 us with a bias and without one)
        const int m = cw + 32 * j + e32;
        bias[j] = p.g.bias && m < cur.cols ? p.g.bias[cur.n0 + m] : 0.0f;
      }
#pragma unroll
      for (int i = 0; i < 2 * TI; ++i) {
        // one group's values at a time in ordinary registers: without the pin the compiler copies all of them at once,
        // and runs out of registers for the loop
        if (i % 2 == 0) pin(acc[i / 2]);
#pragma unroll
        for (int j = 0; j < TJ; ++j)
#pragma unroll
          for (int e = 0; e < 8; e += 2) {
            v2f f{acc[i / 2][j][8 * (i & 1) + e], acc[i / 2][j][8 * (i & 1) + e + 1]};
            f.x += bias[j];
            f.y += bias[j];
            const uint32_t two = __builtin_bit_cast(uint32_t, __builtin_convertvector(f, v2bf));
            uint8_t *at = to + (8 * (e >> 2) + (e & 3)) * T::STRIDE + 64 * j;
            *reinterpret_cast<uint16_t *>(at) = (uint16_t)two;
            *reinterpret_cast<uint16_t *>(at + T::STRIDE) = (uint16_t)(two >> 16);
          }
        wave_lds_fence();
#pragma unroll
        for (int q = 0; q < TJ; ++q) {
          const int k = 16 * i + q * ROWS;
          if (k < left) *reinterpret_cast<uint4 *>(out + k * p.g.ldy) = *reinterpret_cast<const uint4 *>(of + q * ROWS * T::STRIDE);
        }
        wave_lds_fence();
      }
      __builtin_amdgcn_sched_barrier(0);
    }
    lin += gridDim.x;
    if (lin >= total) break;
    cur = piece_of(lin);
    ks = cur.first;
    clear();
  }
  wait_vmcnt<0>();  // the ring's trailing loads are over before LDS is given back
}

// The slices' sums, the bias and the rounding.
__global__ __launch_bounds__(256) void mx_join_kernel(const float *partial, int splits, const float *bias, uint16_t *y, int64_t ldy,
                                                      int64_t M, int64_t N) {
  const int64_t per = N / 8, i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= M * per) return;
  const int64_t m = i / per, n = (i - m * per) * 8;
  float v[8] = {};
  for (int s = 0; s < splits; ++s) {
    const float4 *f = reinterpret_cast<const float4 *>(partial + ((int64_t)s * M + m) * N + n);
    const float4 a = f[0], b = f[1];
    const float w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] += w[j];
  }
  uint32_t o[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    if (bias) {
      v[2 * j] += bias[n + 2 * j];
      v[2 * j + 1] += bias[n + 2 * j + 1];
    }
    o[j] = f32_to_bf16(v[2 * j]) | (f32_to_bf16(v[2 * j + 1]) << 16);
  }
  *reinterpret_cast<uint4 *>(y + m * ldy + n) = make_uint4(o[0], o[1], o[2], o[3]);
}

template <int MT, int NC, int NW>
hipError_t launch_stream(const MxGemmArgs &g, hipStream_t s) {
  constexpr int LDS = NW * (8 * MT > MT * NC ? 8 * MT : MT * NC) * 1024;
  static std::atomic<uint64_t> done{0};
  const hipError_t e = allow_dynamic_lds(&mx_gemm_stream_kernel<MT, NC, NW>, LDS, done);
  if (e != hipSuccess) return e;
  const int64_t grid = ((g.N / 16 + NC - 1) / NC + 7) / 8 * 8 * ((g.M + 16 * MT - 1) / (16 * MT));
  hipLaunchKernelGGL((mx_gemm_stream_kernel<MT, NC, NW>), dim3((unsigned)grid), dim3(64 * NW), LDS, s, g);
  return hipGetLastError();
}

template <int NC, int NW>
hipError_t launch_token(const TokenParams &p, hipStream_t s) {
  hipLaunchKernelGGL((mx_token_kernel<NC, NW>), dim3((unsigned)((p.g.N + 16 * NC - 1) / (16 * NC))), dim3(64 * NW), 0, s, p);
  return hipGetLastError();
}

template <int TI, int TJ, int WM, int WN, int STAGES, bool SPLIT>
hipError_t launch_tile(TileParams p, hipStream_t s) {
  using T = TileShape<TI, TJ, WM, WN, STAGES>;
  static std::atomic<uint64_t> done{0};
  const hipError_t e = allow_dynamic_lds(&mx_gemm_tile_kernel<TI, TJ, WM, WN, STAGES, SPLIT>, T::LDS, done);
  if (e != hipSuccess) return e;
  p.ntm = (int)((p.g.M + T::BM - 1) / T::BM);
  p.ntn = (int)((p.g.N + T::BN - 1) / T::BN);
  p.tiles = p.ntm * p.ntn;
  const int64_t total = (int64_t)p.tiles * p.splits;
  const int64_t most = kUnits * T::PER_UNIT;
  hipLaunchKernelGGL((mx_gemm_tile_kernel<TI, TJ, WM, WN, STAGES, SPLIT>), dim3((unsigned)(total < most ? total : most)), dim3(64 * T::NW),
                     T::LDS, s, p);
  return hipGetLastError();
}

template <int TI, int TJ, int WM, int WN, int STAGES>
hipError_t launch_tiles(const MxGemmArgs &g, int splits, float *ws, hipStream_t s) {
  const int steps = steps_of(g.K), per = (steps + splits - 1) / splits;
  const TileParams p{g, splits > 1 ? ws : nullptr, 0, 0, 0, splits, per};
  if (splits == 1) return launch_tile<TI, TJ, WM, WN, STAGES, false>(p, s);
  const hipError_t e = launch_tile<TI, TJ, WM, WN, STAGES, true>(p, s);
  if (e != hipSuccess) return e;
  const int64_t blocks = (g.M * (g.N / 8) + 255) / 256;
  hipLaunchKernelGGL(mx_join_kernel, dim3((unsigned)blocks), dim3(256), 0, s, ws, splits, g.bias, g.y, g.ldy, g.M, g.N);
  return hipGetLastError();
}

// The kernels to choose from, and the microseconds that a call takes by what was measured (1700 drawn sizes of 1 to
// 8191 rows, K 128 to 32768, N 64 to 32768, each with every kernel and split, in a graph of calls in a row).  On 450 other sizes of
// the same range the formulas are within 6 to 8% (tiles) and 8 to 11% of a call at the root mean square, and the kernel that they
// choose takes 1.3% more than the best of all on average, 23% at most, for a call of 3 us (48% among the 1700).
struct StreamKind {
  int mt, nc, nw;
  hipError_t (*launch)(const MxGemmArgs &, hipStream_t);
  // a call, a batch of a wave, a workgroup that a compute unit runs, a step of 128 channels of all but its first, and a
  // million outputs
  float call, batch, group, step, outputs;
};
const StreamKind kStream[] = {
    {1, 1, 2, launch_stream<1, 1, 2>, 2.84f, 0.183f, 0.031f, 0.0245f, 1.07f},
    {1, 1, 4, launch_stream<1, 1, 4>, 2.71f, 0.278f, 0.157f, 0.0241f, 0.97f},
    {1, 2, 4, launch_stream<1, 2, 4>, 2.80f, 0.426f, 0.149f, 0.0354f, 0.95f},
    {2, 1, 2, launch_stream<2, 1, 2>, 2.73f, 0.295f, 0.157f, 0.0358f, 0.75f},
    {2, 2, 8, launch_stream<2, 2, 8>, 1.17f, 1.357f, 1.695f, 0.0527f, 0.57f},
    {2, 4, 4, launch_stream<2, 4, 4>, 2.70f, 1.063f, 0.362f, 0.0733f, 1.17f},
    {4, 4, 4, launch_stream<4, 4, 4>, 1.43f, 1.654f, 1.810f, 0.1296f, 1.09f},
};
struct TileKind {
  int bm, bn, per_unit;
  hipError_t (*launch)(const MxGemmArgs &, int, float *, hipStream_t);
  // a call, a step of 256 channels alone and with all compute units at work, the outputs of a tile then; a split K's
  // second kernel, and a million bytes of partial sums
  float call, step, step_full, outputs, join, partial;
};
const TileKind kTiles[] = {
    {64, 64, TileShape<1, 1, 2, 2, 3>::PER_UNIT, launch_tiles<1, 1, 2, 2, 3>, 3.50f, 0.299f, 0.109f, 1.54f, 3.05f, 0.189f},
    {128, 128, TileShape<2, 1, 2, 4, 3>::PER_UNIT, launch_tiles<2, 1, 2, 4, 3>, 4.18f, 0.476f, 0.055f, 1.59f, 3.29f, 0.282f},
    {128, 256, TileShape<2, 2, 2, 4, 2>::PER_UNIT, launch_tiles<2, 2, 2, 4, 2>, 5.03f, 0.767f, 0.143f, 2.51f, 3.55f, 0.274f},
    {256, 256, TileShape<4, 2, 2, 4, 2>::PER_UNIT, launch_tiles<4, 2, 2, 4, 2>, 6.68f, 1.155f, 0.299f, 3.04f, 4.08f, 0.289f},
};

// One launch or two: the one rounds each batch of a wave before the product takes it, 1.2 us a batch, and pays up to three or
// four batches a wave (two waves: 2688 channels 4.9 us and 5.6, 4480 9.0 and 7.2; four waves: 8192 to 1024 outputs 6.1 and 6.1,
// to 8192 outputs 8.4 and 10.2, 16384 to 2048 11.2 and 8.0).
bool one_launch(const MxPlan &p, int64_t M, int K) {
  if (M > 2 || p.tile >= 0 || kStream[p.stream].nw > 4) return false;
  return K <= (kStream[p.stream].nw == 2 ? 3 : 4) * 512 * kStream[p.stream].nw;
}

}  // namespace

MxPlan mx_plan(int64_t M, int64_t N, int64_t K) {
  MxPlan best{0, -1, 1, false};
  float least = INFINITY;
  const int ktot = (int)K / kTileK, steps = steps_of((int)K);
  for (int i = 0; i < (int)(sizeof kStream / sizeof kStream[0]); ++i) {
    const StreamKind &k = kStream[i];
    const int64_t groups = ((N / 16 + k.nc - 1) / k.nc + 7) / 8 * 8 * ((M + 16 * k.mt - 1) / (16 * k.mt));
    if (groups * 64 * k.nw > 0xFFFFFFFF) continue;  // threads of a launch
    const float rounds = (float)((groups + kUnits - 1) / kUnits);
    const int batches = (ktot + 4 * k.nw - 1) / (4 * k.nw);
    const float t = k.call + k.batch * (float)batches + rounds * k.group + (rounds - 1.0f) * (float)ktot * k.step +
                    k.outputs * 1e-6f * (float)M * (float)N;
    if (t < least) least = t, best = MxPlan{i, -1, 1, false};
  }
  for (int i = 0; i < (int)(sizeof kTiles / sizeof kTiles[0]); ++i) {
    const TileKind &k = kTiles[i];
    for (int want = 1; want <= 8 && (want == 1 || steps / want >= 2); want *= 2) {
      const int per = (steps + want - 1) / want, splits = (steps + per - 1) / per;  // no slice is empty
      const int64_t pieces = ((M + k.bm - 1) / k.bm) * ((N + k.bn - 1) / k.bn) * splits;
      if (pieces > 0x7FFFFFFF) continue;
      const int64_t units = kUnits * k.per_unit;
      const float rounds = (float)((pieces + units - 1) / units), full = (float)pieces / (rounds * (float)units);
      float t = k.call + rounds * ((float)per * (k.step + k.step_full * full) + k.outputs * full);
      if (splits > 1) t += k.join + k.partial * (float)splits * (float)M * (float)N * 4e-6f;
      if (t < least) least = t, best = MxPlan{-1, i, splits, false};
    }
  }
  best.token = one_launch(best, M, (int)K);
  return best;
}

hipError_t launch_mx_gemm(const MxGemmArgs &g, const MxPlan &p, void *ws, hipStream_t s) {
  return p.tile < 0 ? kStream[p.stream].launch(g, s) : kTiles[p.tile].launch(g, p.splits, static_cast<float *>(ws), s);
}

// As many waves as the product's own kernel, whose sums these are then to the last bit; columns of a workgroup so that its
// waves all find room at once (2048 to 32768 outputs: 16 columns 8.8 us, 32 7.2, 64 5.5; 4096 to 4096: 4.3, 4.7 and 5.2).
hipError_t launch_mx_token(const MxQuantArgs &q, const MxGemmArgs &g, const MxPlan &plan, hipStream_t s) {
  const TokenParams p{q, g, log2_of(q.b)};
  const int nw = kStream[plan.stream].nw;
  const int64_t waves = g.N / 16 * nw;
  if (nw == 2) return waves <= 8 * kUnits ? launch_token<1, 2>(p, s) : launch_token<2, 2>(p, s);
  return waves <= 8 * kUnits ? launch_token<1, 4>(p, s) : waves <= 16 * kUnits ? launch_token<2, 4>(p, s) : launch_token<4, 4>(p, s);
}

}  // namespace fq
