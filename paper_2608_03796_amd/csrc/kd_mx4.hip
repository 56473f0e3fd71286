// HIP kernels (gfx950) of 4-bit microscaled numbers and their launchers:
//   mx4_write, mx4_read    a matrix to codes and scales, and back
//   mx4_rows               logits of few hidden rows with a head of such numbers
#include "kd_mx4.h"
#include "kd_ops.h"

namespace kd {

// ------------------------------------------------------ write and read -----
// Streams: 16 bytes and more a thread. From 64 MiB on (kMx4Big) results that nothing
// reads soon pass by the caches.
constexpr int64_t kMx4Big = (int64_t)64 << 20;
template <bool BIG, typename V>
__device__ __forceinline__ void mx4_store(V v, V* p) {
  if constexpr (BIG) __builtin_nontemporal_store(v, p);
  else *p = v;
}
template <bool BIG, typename V>
__device__ __forceinline__ V mx4_load(const V* p) {
  if constexpr (BIG) return __builtin_nontemporal_load(p);
  else return *p;
}

// Eight elements a thread, four threads a block of 32.
template <typename T, bool BIG>
__global__ __launch_bounds__(256) void k_mx4_write(const T* __restrict__ x, int64_t n8,
                                                   uint32_t* __restrict__ codes,
                                                   uint8_t* __restrict__ scales) {
  const int64_t stride = (int64_t)gridDim.x * 256;
  // (n8 is a multiple of 4: the four threads of a block run or stop together)
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n8; i += stride) {
    float v[8];
    if constexpr (sizeof(T) == 2) {
      const u32x4_t q = mx4_load<BIG>(reinterpret_cast<const u32x4_t*>(x) + i);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        v[2 * j] = __builtin_bit_cast(float, q[j] << 16);
        v[2 * j + 1] = __builtin_bit_cast(float, q[j] & 0xffff0000u);
      }
    } else {
      const f32x4_t q = mx4_load<BIG>(reinterpret_cast<const f32x4_t*>(x) + 2 * i);
      const f32x4_t r = mx4_load<BIG>(reinterpret_cast<const f32x4_t*>(x) + 2 * i + 1);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        v[j] = q[j];
        v[4 + j] = r[j];
      }
    }
    // magnitudes as bit patterns: infinities and what is not a number come last in
    // their order, so neither is lost in the maximum
    uint32_t m = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) m = max(m, __builtin_bit_cast(uint32_t, v[j]) & 0x7fffffffu);
    m = max(m, (uint32_t)__builtin_amdgcn_mov_dpp((int)m, 0xB1, 0xF, 0xF, false));
    m = max(m, (uint32_t)__builtin_amdgcn_mov_dpp((int)m, 0x4E, 0xF, 0xF, false));
    const int s = mx4_scale(m);
    codes[i] = mx4_pack8(v, s);
    if ((threadIdx.x & 3) == 0) scales[i / 4] = (uint8_t)s;
  }
}

template <typename T, bool BIG>
__global__ __launch_bounds__(256) void k_mx4_read(const uint32_t* __restrict__ codes,
                                                  const uint8_t* __restrict__ scales, int64_t n8,
                                                  T* __restrict__ x) {
  const int64_t stride = (int64_t)gridDim.x * 256;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n8; i += stride) {
    const float sc = __builtin_bit_cast(float, (uint32_t)scales[i / 4] << 23);
    const u32x4_t v = mx4_unpack8(codes[i], sc);
    if constexpr (sizeof(T) == 2) {
      mx4_store<BIG>(v, reinterpret_cast<u32x4_t*>(x) + i);
    } else {
      u32x4_t* p = reinterpret_cast<u32x4_t*>(x) + 2 * i;
      mx4_store<BIG>(u32x4_t{v[0] << 16, v[0] & 0xffff0000u, v[1] << 16, v[1] & 0xffff0000u}, p);
      mx4_store<BIG>(u32x4_t{v[2] << 16, v[2] & 0xffff0000u, v[3] << 16, v[3] & 0xffff0000u},
                     p + 1);
    }
  }
}

// ---------------------------------------------------------- few hidden rows --
// out[n, v] = sum_d h[n, d] W[v, d] for up to 16 NB rows n a workgroup, whose
// KS waves each hold 16 R rows of W (MFMA rows) and share its columns: wave w
// takes the 256-column pieces w, w + KS, ... A lane loads 16 bytes of codes at a
// time, one block of 32 columns, 64 columns' blocks apart (four lanes a 64-byte
// run of a row); the MFMAs' column order is the blocks', the same for both
// operands. H = 0: bf16 hidden rows, codes decoded to bf16 in registers (exact).
// H = 1: fp32 hidden rows as three bf16 terms (exact), the same codes thrice.
// H = 2: hidden rows in 4 bits too, both as they are (scaled MFMA). Sums are
// fp32; the waves' sums are added in LDS in order.
struct Mx4RowsArgs {
  const void* hidden;
  int64_t hld;             // bytes between hidden rows
  const uint8_t* hscales;  // H = 2
  const uint8_t *codes, *scales;
  void* out;
  int64_t ldo;             // elements between output rows
  int64_t N;
  int D, V, out_bf16;
};

__device__ __forceinline__ u32x4_t mx4_buf16(__amdgpu_buffer_rsrc_t r, uint32_t off) {
  return __builtin_bit_cast(u32x4_t, __builtin_amdgcn_raw_buffer_load_b128(r, off, 0, 0));
}

template <int H, int NB, int R>
__global__ __launch_bounds__(512) void k_mx4_rows(Mx4RowsArgs a) {
  extern __shared__ __attribute__((aligned(16))) char lds[];
  const int lane = threadIdx.x & 63, wave = wave_id(), KS = blockDim.x >> 6;
  const int m = lane & 15, g = lane >> 4;
  const int v0 = blockIdx.x * 16 * R;
  const int64_t n0 = (int64_t)blockIdx.y * 16 * NB;
  const int nb32 = a.D / kMx4Block;  // blocks of a row
  const int units = (nb32 + 7) / 8;
  const int vrows = min(16 * R, a.V - v0);
  const int nrows = (int)min((int64_t)16 * NB, a.N - n0);
  // the tile's rows only: what lies past them reads as zeros
  const __amdgpu_buffer_rsrc_t rw =
      make_rsrc(a.codes + (int64_t)v0 * (a.D / 2), (uint32_t)(vrows * (a.D / 2)));
  const __amdgpu_buffer_rsrc_t rs =
      make_rsrc(a.scales + (int64_t)v0 * nb32, (uint32_t)(vrows * nb32));
  const char* hbase = static_cast<const char*>(a.hidden) + n0 * a.hld;
  constexpr int HB = H == 0 ? 64 : H == 1 ? 128 : 16;  // bytes of a block of a hidden row

  u32x4_t cw[2][R];
  uint32_t cs[2][R];
  auto load = [&](int u) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int b = 8 * u + 4 * h + g;
      const bool in = b < nb32;  // (u past the end too)
#pragma unroll
      for (int r = 0; r < R; ++r) {
        const uint32_t row = (uint32_t)(16 * r + m);
        cw[h][r] = mx4_buf16(rw, in ? row * (uint32_t)(a.D / 2) + (uint32_t)b * 16u : kOobOffset);
        cs[h][r] = __builtin_amdgcn_raw_buffer_load_b8(
            rs, in ? row * (uint32_t)nb32 + (uint32_t)b : kOobOffset, 0, 0);
      }
    }
  };
  f32x4_t acc[R][NB];
#pragma unroll
  for (int r = 0; r < R; ++r)
#pragma unroll
    for (int q = 0; q < NB; ++q) acc[r][q] = f32x4_t{0.f, 0.f, 0.f, 0.f};

  load(wave);
  for (int u = wave; u < units; u += KS) {
    u32x4_t w[2][R];
    uint32_t s[2][R];
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int r = 0; r < R; ++r) {
        w[h][r] = cw[h][r];
        s[h][r] = cs[h][r];
      }
    load(u + KS);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int b = 8 * u + 4 * h + g;
      const bool in = b < nb32;
#pragma unroll
      for (int q = 0; q < NB; ++q) {
        const int n = 16 * q + m;
        const bool live = in && n < nrows;
        const char* p = hbase + (int64_t)n * a.hld + (int64_t)b * HB;
        if constexpr (H == 2) {
          u32x4_t hc = {0u, 0u, 0u, 0u};
          uint32_t hs = 0;
          if (live) {
            hc = *reinterpret_cast<const u32x4_t*>(p);
            hs = a.hscales[(n0 + n) * nb32 + b];
          }
#pragma unroll
          for (int r = 0; r < R; ++r)
            acc[r][q] = mfma_mx4(w[h][r], hc, acc[r][q], (int)s[h][r], (int)hs);
        } else {
          u32x4_t x[4 * (H + 1)];
#pragma unroll
          for (int i = 0; i < 4 * (H + 1); ++i) {
            x[i] = u32x4_t{0u, 0u, 0u, 0u};
            if (live) x[i] = reinterpret_cast<const u32x4_t*>(p)[i];
          }
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            u32x4_t t[3];
            if constexpr (H == 1) {
              const f32x4_t lo = __builtin_bit_cast(f32x4_t, x[2 * i]);
              const f32x4_t hi = __builtin_bit_cast(f32x4_t, x[2 * i + 1]);
              const float f[8] = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
              cut8(f, t);
            }
#pragma unroll
            for (int r = 0; r < R; ++r) {
              const float sc = __builtin_bit_cast(float, s[h][r] << 23);
              const u32x4_t wf = mx4_unpack8(w[h][r][i], sc);
              if constexpr (H == 0) {
                acc[r][q] = mfma_slot(wf, x[i], acc[r][q], (__bf16*)nullptr);
              } else {
#pragma unroll
                for (int k = 2; k >= 0; --k)
                  acc[r][q] = mfma_slot(wf, t[k], acc[r][q], (__bf16*)nullptr);
              }
            }
          }
        }
      }
    }
  }

  f32x4_t* red = reinterpret_cast<f32x4_t*>(lds);
#pragma unroll
  for (int r = 0; r < R; ++r)
#pragma unroll
    for (int q = 0; q < NB; ++q) red[((wave * R + r) * NB + q) * 64 + lane] = acc[r][q];
  __syncthreads();
  const float* rf = reinterpret_cast<const float*>(lds);
  for (int e = threadIdx.x; e < 16 * R * nrows; e += blockDim.x) {
    const int vl = e % (16 * R), n = e / (16 * R);
    if (vl >= vrows) continue;
    const int at = (((vl >> 4) * NB + (n >> 4)) * 64 + ((vl >> 2) & 3) * 16 + (n & 15)) * 4 + (vl & 3);
    float z = 0.f;
    for (int k = 0; k < KS; ++k) z += rf[k * R * NB * 256 + at];
    const int64_t o = (n0 + n) * a.ldo + v0 + vl;
    if (a.out_bf16) static_cast<__bf16*>(a.out)[o] = (__bf16)z;
    else static_cast<float*>(a.out)[o] = z;
  }
}

}  // namespace kd

using namespace kd;

static unsigned mx4_blocks(int64_t n) {
  const int64_t b = (n + 255) / 256;
  return (unsigned)(b < 16384 ? b : 16384);
}

template <typename T>
static int launch_mx4_write(const void* x, int64_t n, uint8_t* codes, uint8_t* scales,
                            hipStream_t s) {
  auto k = n * (int64_t)sizeof(T) < kMx4Big ? k_mx4_write<T, false> : k_mx4_write<T, true>;
  hipLaunchKernelGGL(k, dim3(mx4_blocks(n / 8)), dim3(256), 0, s, static_cast<const T*>(x), n / 8,
                     reinterpret_cast<uint32_t*>(codes), scales);
  return (int)hipGetLastError();
}
template <typename T>
static int launch_mx4_read(const uint8_t* codes, const uint8_t* scales, int64_t n, void* x,
                           hipStream_t s) {
  auto k = n * (int64_t)sizeof(T) < kMx4Big ? k_mx4_read<T, false> : k_mx4_read<T, true>;
  hipLaunchKernelGGL(k, dim3(mx4_blocks(n / 8)), dim3(256), 0, s,
                     reinterpret_cast<const uint32_t*>(codes), scales, n / 8, static_cast<T*>(x));
  return (int)hipGetLastError();
}

extern "C" int kd_launch_mx4_write(const void* x, int dtype, int64_t n, uint8_t* codes,
                                   uint8_t* scales, void* stream) {
  hipStream_t s = static_cast<hipStream_t>(stream);
  return dtype == 1 ? launch_mx4_write<__bf16>(x, n, codes, scales, s)
                    : launch_mx4_write<float>(x, n, codes, scales, s);
}
extern "C" int kd_launch_mx4_read(const uint8_t* codes, const uint8_t* scales, int dtype, int64_t n,
                                  void* x, void* stream) {
  hipStream_t s = static_cast<hipStream_t>(stream);
  return dtype == 1 ? launch_mx4_read<__bf16>(codes, scales, n, x, s)
                    : launch_mx4_read<float>(codes, scales, n, x, s);
}

template <int H, int NB, int R>
static int launch_mx4_rows(const Mx4RowsArgs& a, int ks, hipStream_t s) {
  const size_t lds = (size_t)ks * R * NB * 1024;
  const int64_t per = 16 * NB, ty = (a.N + per - 1) / per;
  // (the grid's second dimension holds 65535 tiles)
  for (int64_t t = 0; t < ty; t += 65535) {
    Mx4RowsArgs b = a;
    b.hidden = static_cast<const char*>(a.hidden) + t * per * a.hld;
    if (H == 2) b.hscales = a.hscales + t * per * (a.D / kMx4Block);
    b.out = static_cast<char*>(a.out) + t * per * a.ldo * (a.out_bf16 ? 2 : 4);
    b.N = a.N - t * per;
    hipLaunchKernelGGL((k_mx4_rows<H, NB, R>), dim3((a.V + 16 * R - 1) / (16 * R),
                       (unsigned)(ty - t < 65535 ? ty - t : 65535)), dim3(64 * ks), lds, s, b);
  }
  return (int)hipGetLastError();
}

template <int H>
static int launch_mx4_logits(const KdMx4Args& q, hipStream_t s) {
  Mx4RowsArgs a{};
  a.hidden = q.hidden;
  a.hld = H == 2 ? q.D / 2 : q.ld_hidden * (H == 1 ? 4 : 2);
  a.hscales = q.hscales;
  a.codes = q.codes;
  a.scales = q.scales;
  a.out = q.out;
  a.ldo = q.ld_out;
  a.N = q.N;
  a.D = (int)q.D;
  a.V = (int)q.V;
  a.out_bf16 = q.out_dtype == 1;
  const int units = (a.D / kMx4Block + 7) / 8;
  int ks = 1;
  while (ks < 8 && ks < units) ks *= 2;
  const bool small = a.V <= 16384;
  if (q.N <= 16) {
    if (small) return launch_mx4_rows<H, 1, 1>(a, ks, s);
    return launch_mx4_rows<H, 1, 2>(a, ks, s);
  }
  ks = ks > 4 ? 4 : ks;
  if (q.N <= 32) return launch_mx4_rows<H, 2, 2>(a, ks, s);
  return launch_mx4_rows<H, 4, 2>(a, ks, s);
}

extern "C" int kd_launch_mx4_logits(const KdMx4Args* a, void* stream) {
  hipStream_t s = static_cast<hipStream_t>(stream);
  switch (a->dtype) {
    case 0: return launch_mx4_logits<1>(*a, s);
    case 1: return launch_mx4_logits<0>(*a, s);
    default: return launch_mx4_logits<2>(*a, s);
  }
}
