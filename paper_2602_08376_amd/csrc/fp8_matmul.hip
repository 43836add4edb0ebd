// Products with 8-bit activations for many tokens, and the choice of the kernel
// for the sizes at hand.
//
//   expand_codes_kernel  packed codes -> e4m3 values q - z, once
//   product8_kernel      Y of e4m3 weights and activations, in tiles
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

// Sums are formed where they stand (the compiler moves them, with the products
// they come from, behind the branches and barriers that follow, and has to hold
// all operands until then).
__device__ __forceinline__ void pin(v4& v) { asm volatile("" : "+v"(v)); }

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
// kExact: operands brought to bf16, with the activations' scales and the powers
// of two of the weights', exactly, and multiplied there.  Otherwise
// v_mfma_scale_f32_16x16x128_f8f6f4 takes them as they are, with these scales,
// at twice the rate; kPowers: the weights' scales are powers of two, so it takes
// the sums so far as well.
enum { kPowers, kScaled, kExact };
template <int NX, int HOW>
__global__ __launch_bounds__(64 * NX, 2) void product8_kernel(Product8Args a, int64_t tiles_n) {
  constexpr int kTile = 32 * NX;
  __shared__ __align__(16) uint8_t sX[2][kTile * 128], sW[2][kTile * 128];
  // scales of four stages: of a line of activations (a byte each), of a channel
  // of weights (a float32 each, or e8m0 bytes in the first)
  __shared__ __align__(16) uint32_t sxs[2][kTile], sws[2][4][kTile];
  __shared__ __align__(16) uint8_t swp[2][4][kTile];
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

  // ---- memory to LDS --------------------------------------------------------
  // Load q of a wave fills lines 8 (4 wave + q) .. + 7; rows past the last one
  // repeat it (they feed only results that are not stored).
  const int last_t = (int)(a.T - 1 - T0 < kTile - 1 ? a.T - 1 - T0 : kTile - 1);
  const int last_j = (int)(a.n - 1 - J0 < kTile - 1 ? a.n - 1 - J0 : kTile - 1);
  const uint32_t piece = 16 * ((lane & 7) ^ (lane >> 3));
  uint32_t xoff[4], woff[4];
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    const int line = 8 * (4 * wave + q) + (lane >> 3);
    const int t = token_of(line), j = channel_of(line);
    xoff[q] = (uint32_t)(t < last_t ? t : last_t) * (uint32_t)a.ldx + piece;
    woff[q] = (uint32_t)(j < last_j ? j : last_j) * (uint32_t)a.ldw + piece;
  }
  const uint8_t* const xbase = a.X8 + T0 * a.ldx;
  const uint8_t* const wbase = a.W8 + J0 * a.ldw;
  const bool ragged = (a.m & 127) != 0;
  auto load = [&](const uint8_t* base, const uint32_t (&off)[4], int st, uint8_t* to) {
    base += 128 * (int64_t)st;
    to += 4096 * wave;
    if (ragged && st == nst - 1) {
      // a piece past the last feature reads the row's first one; mask_tail clears it
      const uint32_t back = 128 * (int64_t)st + piece < a.m ? 0u : piece;
#pragma unroll
      for (int q = 0; q < 4; ++q) load_to_lds16(base, off[q] - back, to + 1024 * q);
    } else {
#pragma unroll
      for (int q = 0; q < 4; ++q) load_to_lds16(base, off[q], to + 1024 * q);
    }
  };
  auto load_x = [&](int st) { load(xbase, xoff, st, sX[st & 1]); };
  auto load_w = [&](int st) { load(wbase, woff, st, sW[st & 1]); };
  // the last stage of a ragged row: everything from feature m on cleared
  auto mask_tail = [&](int st) {
    const int left = (int)(a.m - 128 * (int64_t)st);
    uint8_t* const line = (tid < kTile ? sX[st & 1] : sW[st & 1]) + 128 * (tid & (kTile - 1));
    for (int c = left / 16; c < 8; ++c) {
      u4* const p = reinterpret_cast<u4*>(line + 16 * (c ^ (tid & 7)));
      u4 v = *p;
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = features_below(v[e], 16 * c + 4 * e, left);
      *p = v;
    }
  };
  // a wave to 64 lines or channels (their addresses formed anew every time, not
  // held in registers)
  const bool bytes = a.ws_e8m0 != 0;
  auto load_scales = [&](int quad) {
    int w = wave;
    __asm__("" : "+s"(w));
    const int buf = quad & 1;
    if (w < kTile / 64) {
      const int t = token_of(64 * w + lane);
      load_to_lds4_at(a.xs + (T0 + (t < last_t ? t : last_t)) * a.lds + 4 * quad, &sxs[buf][64 * w]);
    } else {
      const int c0 = 64 * (w - kTile / 64), j = c0 + lane;
      const int64_t at = ((J0 + (j < last_j ? j : last_j)) >> a.ws_shift) * a.ws_ld;
      const uint8_t* const S = static_cast<const uint8_t*>(a.ws);
      if (bytes) {
        load_to_lds4_at(S + at + 4 * quad, &sws[buf][0][c0]);
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const uint32_t b = (uint32_t)(4 * quad + e < nst ? 4 * quad + e : nst - 1);
          load_to_lds4_at(S + 4 * (at + (a.ws_div == 1 ? b : b / a.ws_div)), &sws[buf][e][c0]);
        }
      }
    }
  };
  auto arrived = [&](int st) {   // stage st, of which every wave has loaded a share
    __builtin_amdgcn_s_waitcnt(0x0f70);
    __syncthreads();
    if (ragged && st == nst - 1) {
      mask_tail(st);
      __syncthreads();
    }
  };

  // ---- LDS to registers -----------------------------------------------------
  // Pieces g4 and 4 + g4 of a line: any order of the features will do, if it is
  // the same for both operands.
  const int slot0 = 16 * (g4 ^ (i16 & 7));
  const int xline = 16 * NX * wr + i16, wline = 64 * wc + i16;
  auto operand = [&](const uint8_t* lines, int line, u4 (&v)[2]) {
    v[0] = *reinterpret_cast<const u4*>(lines + 128 * line + slot0);
    v[1] = *reinterpret_cast<const u4*>(lines + 128 * line + (slot0 ^ 64));
  };
  auto xscales = [&](int st, int x) { return sxs[(st >> 2) & 1][xline + 16 * x]; };   // of four stages
  // The scales of four stages parted in place (split_scale), a thread to a
  // channel, well before the first of them.
  auto part_scales = [&](int quad) {
    if (wave < kTile / 64) return;
    const int c = tid - kTile, buf = quad & 1;
    const uint32_t first = sws[buf][0][c];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if (HOW == kPowers) {
        swp[buf][e][c] = (uint8_t)(first >> (8 * e));
        continue;
      }
      const uint32_t w = sws[buf][e][c];
      const SplitScale sp = split_scale(bytes ? from_e8m0((first >> (8 * e)) & 0xffu) : __uint_as_float(w));
      sws[buf][e][c] = __float_as_uint(sp.rest);
      swp[buf][e][c] = (uint8_t)(__float_as_uint(sp.power) >> 23);
    }
  };
  // of a lane's four channels
  auto rests = [&](int st) {
    return *reinterpret_cast<const v4*>(&sws[(st >> 2) & 1][st & 3][64 * wc + 4 * i16]);
  };
  auto powers = [&](int st) {
    return *reinterpret_cast<const uint32_t*>(&swp[(st >> 2) & 1][st & 3][64 * wc + 4 * i16]);
  };

  v4 acc[NX][4];
#pragma unroll
  for (int x = 0; x < NX; ++x)
#pragma unroll
    for (int y = 0; y < 4; ++y) acc[x][y] = v4{0.f, 0.f, 0.f, 0.f};

  load_scales(0);
  load_w(0);
  load_x(0);
  if (nst > 1) {
    load_w(1);
    load_x(1);
  }
  arrived(0);
  part_scales(0);
  __syncthreads();
  if constexpr (HOW == kExact) {
    for (int st = 0; st < nst; ++st) {
      if ((st & 3) == 0 && st + 4 < nst) load_scales(st / 4 + 1);
      if ((st & 3) == 1 && (st | 3) + 1 < nst) part_scales(st / 4 + 1);
      const v4 s = rests(st);
      const uint32_t power = powers(st);
      b8 fw[4][4];
#pragma unroll
      for (int y = 0; y < 4; ++y) {
        u4 v[2];
        operand(sW[st & 1], wline + 16 * y, v);
        const float p = __uint_as_float(((power >> (8 * y)) & 0xffu) << 23);
#pragma unroll
        for (int k = 0; k < 4; ++k)
          fw[y][k] = to_bf16(v[k >> 1][2 * (k & 1)], v[k >> 1][2 * (k & 1) + 1], p);
      }
      u4 next[2];
      operand(sX[st & 1], xline, next);
      uint32_t nsx = xscales(st, 0);
#pragma unroll
      for (int x = 0; x < NX; ++x) {
        const u4 v[2] = {next[0], next[1]};
        const float sx = from_e8m0((nsx >> (8 * (st & 3))) & 0xffu);
        if (x + 1 < NX) {
          operand(sX[st & 1], xline + 16 * (x + 1), next);
          nsx = xscales(st, x + 1);
        } else if (st + 1 < nst) {
          arrived(st + 1);
          if (st + 2 < nst) {
            load_w(st + 2);
            load_x(st + 2);
          }
        }
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
        for (int y = 0; y < 4; ++y) {
#pragma unroll
          for (int r = 0; r < 4; ++r) acc[x][y][r] = __builtin_fmaf(d[y][r], s[y], acc[x][y][r]);
          pin(acc[x][y]);
        }
        __builtin_amdgcn_sched_barrier(0);
      }
    }
  } else {
    // A product's sums take their scale two products later, beside the matrix
    // cores; the last two of a stage in the next one.  A stage's last line of
    // activations is read ahead, so the barrier stands before its products:
    // behind it the stage's buffers take the stage after the next, and the next
    // stage's first operands are read.
    auto eight = [](const u4 (&v)[2]) {
      return __builtin_bit_cast(i8, __builtin_shufflevector(v[0], v[1], 0, 1, 2, 3, 4, 5, 6, 7));
    };
    i8 fw[4];
    u4 next[2];
    v4 s = rests(0);
    uint32_t power = powers(0), next_power = 0;   // four e8m0 codes
    float last_s[2] = {0.f, 0.f};
    v4 wait[2] = {v4{0.f, 0.f, 0.f, 0.f}, v4{0.f, 0.f, 0.f, 0.f}};
    uint32_t nsx;
    auto read_w = [&](int st, int y) {
      u4 v[2];
      operand(sW[st & 1], wline + 16 * y, v);
      fw[y] = eight(v);
    };
    auto read_x = [&](int st, int x) {
      operand(sX[st & 1], xline + 16 * x, next);
      nsx = xscales(st, x);
    };
#pragma unroll
    for (int y = 0; y < 4; ++y) read_w(0, y);
    read_x(0, 0);
    for (int st = 0; st < nst; ++st) {
      if ((st & 3) == 0 && st + 4 < nst) load_scales(st / 4 + 1);
      if ((st & 3) == 1 && (st | 3) + 1 < nst) part_scales(st / 4 + 1);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int x = 0; x < NX; ++x) {
        const i8 fx = eight(next);
        const int sx = (int)(nsx >> (8 * (st & 3)));
        if (x + 1 < NX) {
          read_x(st, x + 1);
        } else {
          // (behind the last stage these read what stands there, unused)
          if (st + 1 < nst) arrived(st + 1);
          read_x(st + 1, 0);
        }
        if (x == NX / 2) next_power = powers(st + 1);
        if (x == 0 && st > 0 && st + 1 < nst) load_x(st + 1);
#pragma unroll
        for (int y = 0; y < 4; ++y) {
          constexpr v4 kZero = {0.f, 0.f, 0.f, 0.f};
          v4 d = HOW == kPowers ? acc[x][y] : kZero;
          if (y == 0) d = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(fx, fw[0], d, 0, 0, 0, sx, 0, (int)power);
          else if (y == 1) d = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(fx, fw[1], d, 0, 0, 0, sx, 1, (int)power);
          else if (y == 2) d = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(fx, fw[2], d, 0, 0, 0, sx, 2, (int)power);
          else d = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(fx, fw[3], d, 0, 0, 0, sx, 3, (int)power);
          if (x + 1 == NX) read_w(st + 1, y);
          if (HOW == kPowers) {
            acc[x][y] = d;
            pin(acc[x][y]);
            __builtin_amdgcn_sched_barrier(0);
            continue;
          }
          // (the product before the one before)
          const int px = y >= 2 ? x : (x + NX - 1) % NX, py = (y + 2) & 3;
          const float ps = x == 0 && y < 2 ? last_s[y] : s[py];
#pragma unroll
          for (int r = 0; r < 4; ++r)
            acc[px][py][r] = __builtin_fmaf(wait[y & 1][r], ps, acc[px][py][r]);
          pin(acc[px][py]);
          wait[y & 1] = d;
          __builtin_amdgcn_sched_barrier(0);
        }
        if (x + 1 == NX && st + 2 < nst) load_w(st + 2);
      }
      last_s[0] = s[2];
      last_s[1] = s[3];
      s = rests(st + 1);
      power = next_power;
    }
#pragma unroll
    for (int y = 0; y < (HOW == kPowers ? 0 : 2); ++y)
#pragma unroll
      for (int r = 0; r < 4; ++r)
        acc[NX - 1][2 + y][r] = __builtin_fmaf(wait[y][r], last_s[y], acc[NX - 1][2 + y][r]);
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
  if (a.ytype == 0) product8_kernel<NX, kExact><<<grid, block, 0, s>>>(a, tiles_n);
  else if (a.ws_e8m0) product8_kernel<NX, kPowers><<<grid, block, 0, s>>>(a, tiles_n);
  else product8_kernel<NX, kScaled><<<grid, block, 0, s>>>(a, tiles_n);
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
