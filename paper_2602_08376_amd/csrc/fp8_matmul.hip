// Products with 8-bit activations for many tokens, and the choice of the kernel
// for the sizes at hand.
//
//   expand_codes_kernel  packed codes -> e4m3 values q - z, once
//   product8_kernel      Y of e4m3 weights and activations, in tiles
#include "device.h"
#include "fp8_product.h"
#include "kernels.h"

namespace ojbkq {
namespace {

typedef int i8 __attribute__((ext_vector_type(8)));

// ---- codes in e4m3 ---------------------------------------------------------

// W8 [n, ldw] e4m3 = q - z of the packed codes: whole numbers of at most 15,
// exact in e4m3's 4 significant bits.  One thread to 32 codes (BITS words of a
// row).  Bound by memory: it writes a byte for every code.
template <int BITS>
__global__ __launch_bounds__(256) void expand_codes_kernel(Product8Args a, uint8_t* W8, int64_t ldw) {
  const int64_t runs = ldw / 32, total = a.n * runs;
  for (int64_t e = (int64_t)blockIdx.x * 256 + threadIdx.x; e < total; e += (int64_t)gridDim.x * 256) {
    const int64_t j = e / runs, u = e % runs;
    const uint32_t* const row = a.P + j * a.wpr;
    uint32_t w[BITS];
#pragma unroll
    for (int q = 0; q < BITS; ++q) w[q] = row[u * BITS + q < a.wpr ? u * BITS + q : a.wpr - 1];
    // (runs past the last feature: any group will do, they are not used)
    const uint32_t b = 32 * u < a.m ? (uint32_t)(u / 4) : 0u;
    const float z = whole_zero<BITS>(a.Z[j * a.ws_ld + b / a.ws_div]);
    u4 out[2];
#pragma unroll
    for (int d = 0; d < 8; ++d) {
      float v[4];
#pragma unroll
      for (int c = 0; c < 4; ++c) v[c] = (float)code_of<BITS>(w, 4 * d + c) - z;
      int p = __builtin_amdgcn_cvt_pk_fp8_f32(v[0], v[1], 0, false);
      p = __builtin_amdgcn_cvt_pk_fp8_f32(v[2], v[3], p, true);
      out[d >> 2][d & 3] = (uint32_t)p;
    }
    *reinterpret_cast<u4*>(W8 + j * ldw + 32 * u) = out[0];
    *reinterpret_cast<u4*>(W8 + j * ldw + 32 * u + 16) = out[1];
  }
}

// ---- tiles -----------------------------------------------------------------

// Output tile of this workgroup: each XCD (of eight, dealt workgroups round
// robin) takes a contiguous run of tiles, walked in groups of 8 channel tiles
// with the token tiles outer, so that the workgroups it runs at once share
// their panels in its L2.
__device__ __forceinline__ void tile_of(int64_t tiles_n, int64_t& tj, int64_t& tt) {
  constexpr int64_t kGroup = 8;
  const int64_t nb = gridDim.x, tiles_t = nb / tiles_n;
  int64_t t = blockIdx.x;
  if ((nb & 7) == 0) t = (t & 7) * (nb >> 3) + (t >> 3);
  const int64_t per = kGroup * tiles_t, first = (t / per) * kGroup;
  const int64_t rows = tiles_n - first < kGroup ? tiles_n - first : kGroup;
  const int64_t r = t % per;
  tj = first + r % rows;
  tt = r / rows;
}

template <class E, int N>
__device__ __forceinline__ void store_run(E* p, const float (&v)[N], int64_t left) {
  typedef E Any __attribute__((ext_vector_type(N), aligned(sizeof(E))));
  if (left >= N) {
    Any o;
#pragma unroll
    for (int e = 0; e < N; ++e) o[e] = (E)v[e];
    *reinterpret_cast<Any*>(p) = o;
  } else {
#pragma unroll
    for (int e = 0; e < N; ++e)
      if (e < left) p[e] = (E)v[e];
  }
}

// Tiles of kTile tokens x kTile channels (256 with eight waves, 128 with four),
// a block of 128 features to a stage, two stages in LDS.  A wave holds 16 NX
// tokens x 64 channels: its weights of a stage stay in registers while its
// activations pass.  Both operands go straight from memory to LDS in lines of
// 128 bytes, 16-byte chunk c of line l at slot c ^ (l % 8), which spreads the
// operand reads of 16 lines x 4 chunks over all banks.
// Line 16 x + i of the activations holds token 32 (x / 2) + 8 (i / 4) + 4 (x %
// 2) + i % 4, line 16 y + i of a wave's 64 of weights channel 4 i + y: a lane
// then ends up with runs of 8 tokens and of 4 channels, whichever is contiguous
// in Y.
// EXACT: operands brought to bf16 (with the activations' scales, exactly) and
// multiplied there.  Otherwise v_mfma_scale_f32_16x16x128_f8f6f4 takes them as
// they are, scales included, at twice the rate.
template <int NX, bool EXACT>
__global__ __launch_bounds__(64 * NX, 2) void product8_kernel(Product8Args a, int64_t tiles_n) {
  constexpr int kTile = 32 * NX;
  __shared__ __align__(16) uint8_t sX[2][kTile * 128], sW[2][kTile * 128];
  __shared__ uint32_t sxs[2][kTile];      // scales of a line for four stages
  __shared__ float sws[2][4][kTile];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int i16 = lane & 15, g4 = lane >> 4;
  const int wr = wave & 1, wc = wave >> 1;
  int64_t tj, tt;
  tile_of(tiles_n, tj, tt);
  const int64_t J0 = tj * kTile, T0 = tt * kTile;
  const int nst = (int)((a.m + 127) / 128);

  auto token_of = [](int line) {
    const int i = line & 15;
    return (line & ~31) + 8 * (i >> 2) + 4 * ((line >> 4) & 1) + (i & 3);
  };
  auto channel_of = [](int line) { return (line & ~63) + 4 * (line & 15) + ((line >> 4) & 3); };

  // load q of a wave fills lines 8 (4 wave + q) .. + 7; rows past the last one
  // repeat it (they feed only results that are not stored)
  uint32_t xoff[4], woff[4];
  const int chunk = (lane & 7) ^ (lane >> 3);
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    const int line = 8 * (4 * wave + q) + (lane >> 3);
    const int64_t t = T0 + token_of(line), j = J0 + channel_of(line);
    xoff[q] = (uint32_t)((t < a.T ? t : a.T - 1) - T0) * (uint32_t)a.ldx + 16 * chunk;
    woff[q] = (uint32_t)((j < a.n ? j : a.n - 1) - J0) * (uint32_t)a.ldw + 16 * chunk;
  }
  const uint8_t* const xbase = a.X8 + T0 * a.ldx;
  const uint8_t* const wbase = a.W8 + J0 * a.ldw;
  auto load = [&](int st, int buf) {
    const int64_t k0 = 128 * (int64_t)st;
    // a chunk past the last feature reads the row's first one; mask_tail
    // clears it
    const uint32_t back = k0 + 16 * chunk < a.m ? 0u : 16u * chunk;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      load_to_lds16(xbase + k0, xoff[q] - back, sX[buf] + 1024 * (4 * wave + q));
      load_to_lds16(wbase + k0, woff[q] - back, sW[buf] + 1024 * (4 * wave + q));
    }
  };
  // the last stage of a ragged row: everything from feature m on cleared
  auto mask_tail = [&](int st, int buf) {
    const int left = (int)(a.m - 128 * (int64_t)st);
    uint8_t* const line = (tid < kTile ? sX[buf] : sW[buf]) + 128 * (tid & (kTile - 1));
    for (int c = left / 16; c < 8; ++c) {
      u4* const p = reinterpret_cast<u4*>(line + 16 * (c ^ (tid & 7)));
      u4 v = *p;
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = features_below(v[e], 16 * c + 4 * e, left);
      *p = v;
    }
  };

  // scales of four stages, a thread to a line of either operand: read at the
  // first of the four before, in LDS at the last of them
  const int sline = tid & (kTile - 1);
  const int64_t srow = tid < kTile ? T0 + token_of(sline) : J0 + channel_of(sline);
  const bool bytes = tid < kTile || a.ws_e8m0;   // (the same for a whole wave)
  const uint8_t* const srow_at =
      tid < kTile ? a.xs + (srow < a.T ? srow : a.T - 1) * a.lds
                  : static_cast<const uint8_t*>(a.ws) +
                        ((srow < a.n ? srow : a.n - 1) >> a.ws_shift) * a.ws_ld * (a.ws_e8m0 ? 1 : 4);
  uint32_t sc[4] = {0u, 0u, 0u, 0u};
  auto fetch_scales = [&](int quad) {
    if (bytes) {
      sc[0] = *reinterpret_cast<const uint32_t*>(srow_at + 4 * quad);
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const uint32_t b = (uint32_t)(4 * quad + e < nst ? 4 * quad + e : nst - 1);
        sc[e] = reinterpret_cast<const uint32_t*>(srow_at)[b / a.ws_div];
      }
    }
  };
  auto put_scales = [&](int buf) {
    if (tid < kTile) {
      sxs[buf][sline] = sc[0];
    } else if (bytes) {
#pragma unroll
      for (int e = 0; e < 4; ++e) sws[buf][e][sline] = from_e8m0((sc[0] >> (8 * e)) & 0xffu);
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e) sws[buf][e][sline] = __uint_as_float(sc[e]);
    }
  };

  v4 acc[NX][4];
#pragma unroll
  for (int x = 0; x < NX; ++x)
#pragma unroll
    for (int y = 0; y < 4; ++y) acc[x][y] = v4{0.f, 0.f, 0.f, 0.f};

  // chunks g4 and 4 + g4 of line l: any order of the features will do, if it
  // is the same for both operands
  const int slot0 = 16 * (g4 ^ (i16 & 7));
  const int xline = 16 * NX * wr + i16, wline = 64 * wc + i16;
  auto operand = [&](const uint8_t* lines, int line, u4 (&v)[2]) {
    v[0] = *reinterpret_cast<const u4*>(lines + 128 * line + slot0);
    v[1] = *reinterpret_cast<const u4*>(lines + 128 * line + (slot0 ^ 64));
  };

  load(0, 0);
  fetch_scales(0);
  put_scales(0);
  __builtin_amdgcn_s_waitcnt(0x0f70);
  __syncthreads();
  for (int st = 0; st < nst; ++st) {
    const int cur = st & 1, sq = (st >> 2) & 1;
    if (128 * (int64_t)(st + 1) > a.m) {
      mask_tail(st, cur);
      __syncthreads();
    }
    if (st + 1 < nst) load(st + 1, cur ^ 1);
    if ((st & 3) == 0 && st + 4 < nst) fetch_scales(st / 4 + 1);
    if ((st & 3) == 3 && st + 1 < nst) put_scales(sq ^ 1);
    __builtin_amdgcn_sched_barrier(0);
    float s[4], power[4];
#pragma unroll
    for (int y = 0; y < 4; ++y) {
      const SplitScale sp = split_scale(sws[sq][st & 3][wline + 16 * y]);
      s[y] = sp.rest;
      power[y] = sp.power;
    }
    const int byte = 8 * (st & 3);
    if constexpr (EXACT) {
      b8 fw[4][4];
#pragma unroll
      for (int y = 0; y < 4; ++y) {
        u4 v[2];
        operand(sW[cur], wline + 16 * y, v);
#pragma unroll
        for (int k = 0; k < 4; ++k) fw[y][k] = to_bf16(v[k >> 1][2 * (k & 1)], v[k >> 1][2 * (k & 1) + 1], power[y]);
      }
      u4 next[2];
      operand(sX[cur], xline, next);
#pragma unroll
      for (int x = 0; x < NX; ++x) {
        const u4 v[2] = {next[0], next[1]};
        if (x + 1 < NX) operand(sX[cur], xline + 16 * (x + 1), next);
        const float sx = from_e8m0((sxs[sq][xline + 16 * x] >> byte) & 0xffu);
        v4 d[4];
#pragma unroll
        for (int y = 0; y < 4; ++y) d[y] = v4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const b8 fx = to_bf16(v[k >> 1][2 * (k & 1)], v[k >> 1][2 * (k & 1) + 1], sx);
#pragma unroll
          for (int y = 0; y < 4; ++y)
            d[y] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fx, fw[y][k], d[y], 0, 0, 0);
        }
#pragma unroll
        for (int y = 0; y < 4; ++y)
#pragma unroll
          for (int r = 0; r < 4; ++r) acc[x][y][r] = __builtin_fmaf(d[y][r], s[y], acc[x][y][r]);
        __builtin_amdgcn_sched_barrier(0);
      }
    } else {
      i8 fw[4];
      auto eight = [](const u4 (&v)[2]) {
        return __builtin_bit_cast(i8, __builtin_shufflevector(v[0], v[1], 0, 1, 2, 3, 4, 5, 6, 7));
      };
#pragma unroll
      for (int y = 0; y < 4; ++y) {
        u4 v[2];
        operand(sW[cur], wline + 16 * y, v);
        fw[y] = eight(v);
      }
      u4 next[2];
      operand(sX[cur], xline, next);
#pragma unroll
      for (int x = 0; x < NX; ++x) {
        const i8 fx = eight(next);
        if (x + 1 < NX) operand(sX[cur], xline + 16 * (x + 1), next);
        const int sx = (int)(sxs[sq][xline + 16 * x] >> byte);
#pragma unroll
        for (int y = 0; y < 4; ++y) {
          const v4 d = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(
              fx, fw[y], v4{0.f, 0.f, 0.f, 0.f}, 0, 0, 0, sx, 0,
              (int)(__float_as_uint(power[y]) >> 23));
#pragma unroll
          for (int r = 0; r < 4; ++r) acc[x][y][r] = __builtin_fmaf(d[r], s[y], acc[x][y][r]);
        }
        __builtin_amdgcn_sched_barrier(0);
      }
    }
    __builtin_amdgcn_s_waitcnt(0x0f70);
    __syncthreads();
  }

  // lane l holds tokens 4 g4 + r (lines) of channel i16 of each 16 x 16 block
  auto store = [&](auto* Y) {
    const int64_t j0 = J0 + 64 * wc + 4 * i16, t0 = T0 + 16 * NX * wr + 8 * g4;
#pragma unroll
    for (int p = 0; p < NX / 2; ++p) {
      const int64_t t = t0 + 32 * p;
      if (a.tokens_first) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          float v[4];
#pragma unroll
          for (int y = 0; y < 4; ++y) v[y] = acc[2 * p + (e >> 2)][y][e & 3];
          if (t + e < a.T) store_run(Y + (t + e) * a.ldy + j0, v, a.n - j0);
        }
      } else {
#pragma unroll
        for (int y = 0; y < 4; ++y) {
          float v[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) v[e] = acc[2 * p + (e >> 2)][y][e & 3];
          if (j0 + y < a.n) store_run(Y + (j0 + y) * a.ldy + t, v, a.T - t);
        }
      }
    }
  };
  if (a.ytype == 0) store(static_cast<float*>(a.Y));
  else if (a.ytype == 1) store(static_cast<_Float16*>(a.Y));
  else store(static_cast<__bf16*>(a.Y));
}

template <int NX>
hipError_t launch_tiles(const Product8Args& a, hipStream_t s) {
  constexpr int kTile = 32 * NX;
  const int64_t tiles_n = (a.n + kTile - 1) / kTile, tiles = tiles_n * ((a.T + kTile - 1) / kTile);
  if (tiles > 0x7fffffff) return hipErrorInvalidValue;
  const dim3 grid((unsigned)tiles), block(64 * NX);
  if (a.ytype == 0) product8_kernel<NX, true><<<grid, block, 0, s>>>(a, tiles_n);
  else product8_kernel<NX, false><<<grid, block, 0, s>>>(a, tiles_n);
  return hipGetLastError();
}

// Up to two workgroups of 64 channels x 64 tokens per CU, or up to 32 tokens.
bool few(int64_t n, int64_t m, int64_t T) {
  const int64_t blocks = (n + 63) / 64 * ((T + 63) / 64);
  return blocks <= 512 || T <= 32;
}
int64_t expanded_row(int64_t m) { return (m + 127) / 128 * 128; }

}  // namespace

size_t product8_workspace_bytes(int64_t n, int64_t m, int64_t T) {
  return few(n, m, T) ? 0 : (size_t)n * (size_t)expanded_row(m);
}

hipError_t launch_product8(const Product8Args& a, int bits, void* workspace, hipStream_t stream) {
  // (tiles address their rows with 32 bits)
  if (few(a.n, a.m, a.T) || a.ldx > (1 << 23) || (bits == 0 && a.ldw > (1 << 23)))
    return launch_product_few8(a, bits, stream);
  Product8Args b = a;
  if (bits) {
    uint8_t* const W8 = static_cast<uint8_t*>(workspace);
    b.W8 = W8;
    b.ldw = expanded_row(a.m);
    const int64_t blocks = (a.n * (b.ldw / 32) + 255) / 256;
    const dim3 grid((unsigned)(blocks < 65536 ? blocks : 65536)), block(256);
    switch (bits) {
      case 1: expand_codes_kernel<1><<<grid, block, 0, stream>>>(a, W8, b.ldw); break;
      case 2: expand_codes_kernel<2><<<grid, block, 0, stream>>>(a, W8, b.ldw); break;
      case 3: expand_codes_kernel<3><<<grid, block, 0, stream>>>(a, W8, b.ldw); break;
      case 4: expand_codes_kernel<4><<<grid, block, 0, stream>>>(a, W8, b.ldw); break;
      default: return hipErrorInvalidValue;
    }
    if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
  }
  const int64_t big = (b.n + 255) / 256 * ((b.T + 255) / 256);
  const int64_t small = (b.n + 127) / 128 * ((b.T + 127) / 128);
  return 100 * ((big + 255) / 256) <= 65 * ((small + 511) / 512) ? launch_tiles<8>(b, stream)
                                                                 : launch_tiles<4>(b, stream);
}

}  // namespace ojbkq
