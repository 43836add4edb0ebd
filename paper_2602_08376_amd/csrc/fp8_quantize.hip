// Arrays brought to 8 bits (ojbkq_quantize_fp8): e4m3 values with a
// power-of-two scale for each block of 1 or 128 rows x 128 features.
//
// All three kernels read X once and write its 8-bit form once; they are bound
// by memory.
#include "fp8_pack.h"

namespace ojbkq {
namespace {

// Rows of features, a scale to 128 of them: 16 lanes hold a block, eight
// features each, and meet by lane rotations; a wave takes four blocks of a row
// at a time, `per` times.  16384 x 8192 in fp16: 79 us, 5.1 TB/s, as a large
// copy.
template <int XT>
__global__ __launch_bounds__(256) void quantize_rows_kernel(Quantize8Args a, int per) {
  typedef typename Number<XT>::type E;
  const int lane = threadIdx.x & 63;
  const int64_t row = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (row >= a.rows) return;   // a whole wave
  const E* const src = static_cast<const E*>(a.X) + row * a.ldx;
  uint8_t* const dst = a.X8 + row * a.ld8;
  const int64_t m16 = (a.m + 15) / 16 * 16;
  const int64_t first = (int64_t)blockIdx.y * per * 512 + 8 * lane;
  for (int i = 0; i < per; ++i) {
    const int64_t k = first + 512 * i;
    Eight<E> x;
    x.load(src + k, a.m - k);
    float v[8];
    uint32_t most = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      v[e] = (float)x.v[e];
      const uint32_t s = size_key(v[e]);
      most = most > s ? most : s;
    }
    const uint32_t code = scale_code(max16(most));
    if (k < m16) *reinterpret_cast<u2*>(dst + k) = to_e4m3(v, inverse_scale(code));
    if ((lane & 15) == 0 && k < a.m) a.scales[row * a.lds + (k >> 7)] = (uint8_t)code;
  }
}

// Blocks of 128 rows x 128 features, one to a workgroup, held in registers.
// 14336 x 4096 in fp32: 51.7 us, 5.7 TB/s.
template <int XT>
__global__ __launch_bounds__(256) void quantize_blocks_kernel(Quantize8Args a) {
  typedef typename Number<XT>::type E;
  __shared__ uint32_t part[4];
  const int tid = threadIdx.x;
  const int64_t r0 = (int64_t)blockIdx.y * 128 + (tid >> 4), k = (int64_t)blockIdx.x * 128 + 8 * (tid & 15);
  Eight<E> x[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int64_t r = r0 + 16 * i;
    x[i].load(static_cast<const E*>(a.X) + (r < a.rows ? r * a.ldx + k : 0), r < a.rows ? a.m - k : 0);
  }
  uint32_t most = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i)
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const uint32_t s = size_key((float)x[i].v[e]);
      most = most > s ? most : s;
    }
  most = max16(most);
#pragma unroll
  for (int d = 16; d < 64; d *= 2) {
    const uint32_t o = __shfl_xor(most, d);
    most = most > o ? most : o;
  }
  if ((tid & 63) == 0) part[tid >> 6] = most;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < 4; ++w) most = most > part[w] ? most : part[w];
  const uint32_t code = scale_code(most);
  const float inv = inverse_scale(code);
  const int64_t m16 = (a.m + 15) / 16 * 16;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int64_t r = r0 + 16 * i;
    float v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = (float)x[i].v[e];
    if (r < a.rows && k < m16) *reinterpret_cast<u2*>(a.X8 + r * a.ld8 + k) = to_e4m3(v, inv);
  }
  if (tid == 0) a.scales[(int64_t)blockIdx.y * a.lds + blockIdx.x] = (uint8_t)code;
}

// X [m, rows], the rows (tokens) contiguous: a workgroup takes 128 features x
// TOK tokens through LDS, read there with a lane to each token, 32 features to a
// thread; the four threads of a token meet in LDS for the scale, and its 128
// bytes go out by way of LDS, so that lanes write along them too.  256 bytes of
// a feature at a time (TOK 64 for float32, 128 for 16 bits): 4096 x 32768 in
// fp16 92.8 us, 4.3 TB/s, against 95.8 with 128 bytes; float32 with 512 bytes
// 72.9 against 72.0 (4096 x 16384), its LDS leaving fewer waves.  Without the
// second pass through LDS 108.
template <int XT, int TOK>
__global__ __launch_bounds__(4 * TOK) void quantize_turned_kernel(Quantize8Args a) {
  typedef typename Number<XT>::type E;
  typedef E Vec __attribute__((ext_vector_type(8)));
  __shared__ __align__(16) E tile[128 * TOK];
  __shared__ uint32_t part[4][TOK];
  const int tid = threadIdx.x, lane = tid % TOK, wave = tid / TOK;   // (a quarter of the features)
  const int64_t t0 = (int64_t)blockIdx.x * TOK, k0 = (int64_t)blockIdx.y * 128;
  {
    const int f = tid / (TOK / 8), t = 8 * (tid % (TOK / 8));
    Eight<E> x[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int64_t k = k0 + f + 32 * i;
      const bool in = k < a.m && t0 + t < a.rows;
      x[i].load(static_cast<const E*>(a.X) + (in ? k * a.ldx + t0 + t : 0), in ? a.rows - t0 - t : 0);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) *reinterpret_cast<Vec*>(tile + (f + 32 * i) * TOK + t) = x[i].v;
  }
  __syncthreads();
  float v[32];
  uint32_t most = 0;
#pragma unroll
  for (int i = 0; i < 32; ++i) {
    v[i] = (float)tile[(32 * wave + i) * TOK + lane];
    const uint32_t s = size_key(v[i]);
    most = most > s ? most : s;
  }
  part[wave][lane] = most;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < 4; ++w) most = most > part[w][lane] ? most : part[w][lane];
  const uint32_t code = scale_code(most);
  const float inv = inverse_scale(code);
  // the tokens' 128 bytes once more through LDS, so that lanes write along them
  // (16-byte piece p of token t at p ^ (t % 8))
  uint8_t* const out = reinterpret_cast<uint8_t*>(tile);   // (every wave has its values)
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    float p[8], q[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      p[e] = v[16 * h + e];
      q[e] = v[16 * h + 8 + e];
    }
    const u2 lo = to_e4m3(p, inv), hi = to_e4m3(q, inv);
    *reinterpret_cast<uint4*>(out + 128 * lane + 16 * ((2 * wave + h) ^ (lane & 7))) =
        make_uint4(lo.x, lo.y, hi.x, hi.y);
  }
  if (wave == 0 && t0 + lane < a.rows) a.scales[(t0 + lane) * a.lds + blockIdx.y] = (uint8_t)code;
  __syncthreads();
  const int64_t m16 = (a.m + 15) / 16 * 16, k = k0 + 16 * (tid & 7);
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int r = (tid >> 3) + TOK / 2 * i;
    const int64_t t = t0 + r;
    if (t < a.rows && k < m16)
      *reinterpret_cast<uint4*>(a.X8 + t * a.ld8 + k) =
          *reinterpret_cast<const uint4*>(out + 128 * r + 16 * ((tid & 7) ^ (r & 7)));
  }
}

template <int XT>
hipError_t launch(const Quantize8Args& a, bool features_first, int block_rows, hipStream_t s) {
  const int64_t G = (a.m + kFp8Block - 1) / kFp8Block;
  if (features_first) {
    constexpr int kTok = XT == 0 ? 64 : 128;
    quantize_turned_kernel<XT, kTok><<<dim3((unsigned)((a.rows + kTok - 1) / kTok), (unsigned)G),
                                       dim3(4 * kTok), 0, s>>>(a);
  } else if (block_rows == 128) {
    // (rows <= 2^24: at most 2^17 blocks of them)
    for (int64_t r = 0; r < a.rows; r += 65535 * 128) {
      Quantize8Args b = a;
      const int64_t blocks = (a.rows - r + 127) / 128;
      b.X = static_cast<const typename Number<XT>::type*>(a.X) + r * a.ldx;
      b.X8 = a.X8 + r * a.ld8;
      b.scales = a.scales + r / 128 * a.lds;
      b.rows = a.rows - r;
      quantize_blocks_kernel<XT><<<dim3((unsigned)G, (unsigned)(blocks < 65535 ? blocks : 65535)),
                                   dim3(256), 0, s>>>(b);
    }
  } else {
    // more steps of 512 features to a wave as they leave the chip enough waves
    // (us for 1 / 2 / 4 / 8, bfloat16: 512 x 4096 3.1 / 3.2 / 3.9 / 5.4, 2000 x
    // 4096 7.0 / 6.4 / 6.8 / 8.5, 8192 x 4096 19.0 / 18.5 / 18.3 / 18.5, 8192 x
    // 14336 77.0 / 78.3 / 75.2 / 76.0)
    const int64_t steps = (a.m + 511) / 512, all = a.rows * steps;
    const int per = all >= 65536 ? 4 : all >= 8192 ? 2 : 1;
    quantize_rows_kernel<XT><<<dim3((unsigned)((a.rows + 3) / 4), (unsigned)((steps + per - 1) / per)),
                               dim3(256), 0, s>>>(a, per);
  }
  return hipGetLastError();
}

}  // namespace

hipError_t launch_quantize_fp8(const Quantize8Args& a, int xtype, bool features_first,
                               int block_rows, hipStream_t stream) {
  switch (xtype) {
    case 0: return launch<0>(a, features_first, block_rows, stream);
    case 1: return launch<1>(a, features_first, block_rows, stream);
    case 2: return launch<2>(a, features_first, block_rows, stream);
    default: return hipErrorInvalidValue;
  }
}

}  // namespace ojbkq
