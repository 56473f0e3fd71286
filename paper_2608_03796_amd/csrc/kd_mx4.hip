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

// ---------------------------------------------------------------- products --
struct Mx4Args {
  const void* hidden;
  int64_t hld;             // bytes between hidden rows
  const uint8_t* hscales;  // H = 2
  const uint8_t *codes, *scales;
  void* out;
  int64_t ldo;             // elements between output rows
  int64_t N;
  int D, V, out_bf16;
};

// Both kernels form out[n, v] = sum_d h[n, d] W[v, d] on matrix instructions, rows v of
// W as their rows, hidden rows n as their columns. Hidden rows: H = 0 bf16, codes
// decoded to bf16 in registers (exact); H = 1 fp32 as three bf16 terms (exact), the same
// codes thrice; H = 2 in 4 bits too, both as they are (scaled instructions). Sums are
// fp32. A lane loads 16 bytes of codes at a time, one block of 32 columns; the
// instructions' column order is the blocks', the same for both operands.

// A wave's 16 R rows of W: codes of a piece of 256 columns (8 blocks; lane (m, g) has
// block 4 h + g of row m of each 16) and their scale bytes.
template <int R>
struct Mx4Weights {
  __amdgpu_buffer_rsrc_t rw;
  const uint8_t* scales;   // of the first row
  int64_t left;            // bytes from there to the scales' end
  int vrows, nb32, pitch;
  u32x2_t sc[R], next[R];
  __device__ __forceinline__ void init(const Mx4Args& a, int v0) {
    vrows = max(0, min(16 * R, a.V - v0));
    nb32 = a.D / kMx4Block;
    pitch = a.D / 2;
    // these rows only: what lies past them reads as zeros
    rw = make_rsrc(a.codes + (int64_t)v0 * pitch, (uint32_t)(vrows * pitch));
    scales = a.scales + (int64_t)v0 * nb32;
    left = ((int64_t)a.V - v0) * nb32;
  }
  // half h of piece u, zeros from block `end` on
  __device__ __forceinline__ void load(int u, int h, int end, int m, int g, u32x4_t (&w)[R]) const {
    const int b = 8 * u + 4 * h + g;
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const uint32_t off = (uint32_t)(16 * r + m) * (uint32_t)pitch + (uint32_t)b * 16u;
      w[r] = __builtin_bit_cast(
          u32x4_t, __builtin_amdgcn_raw_buffer_load_b128(rw, b < end ? off : kOobOffset, 0, 0));
    }
  }
  // scale bytes of pieces u .. u + 3: lane (m, g) holds the 8 of piece u + g, row m. (A
  // byte a piece and lane fetched each line of the scales once a piece, as many
  // requests as the codes': one row of 131072 x 4096 81 us, now 61.)
  __device__ __forceinline__ void load_scales(int u, int m, int g) {
    const int b = 8 * (u + g);
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const int row = 16 * r + m;
      next[r] = u32x2_t{0u, 0u};
      if (row < vrows && b < nb32) {
        const int64_t at = (int64_t)row * nb32 + b;
        if (at + 8 <= left) {
          __builtin_memcpy(&next[r], scales + at, 8);
        } else {
          uint32_t w[2] = {0u, 0u};
          for (int i = 0; i < 8; ++i)
            if (b + i < nb32) w[i >> 2] |= (uint32_t)scales[at + i] << (8 * (i & 3));
          next[r] = u32x2_t{w[0], w[1]};
        }
      }
    }
  }
  // at every fourth piece u: what was loaded for it, and the loads of the next four
  __device__ __forceinline__ void turn(int u, int m, int g) {
#pragma unroll
    for (int r = 0; r < R; ++r) sc[r] = next[r];
    load_scales(u + 4, m, g);
  }
  // of block 8 u + 4 h + g, the t-th of the four pieces held. (A block past the row's
  // end may hold the next row's byte there: 0.)
  __device__ __forceinline__ uint32_t scale(int r, int u, int h, int t, int m, int g) const {
    const uint32_t x = (uint32_t)__shfl((int)sc[r][h], 16 * t + m);
    return 8 * u + 4 * h + g < nb32 ? (x >> (8 * g)) & 255u : 0u;
  }
};

// One block of columns of the lane's row of W and of its hidden row: 4 instructions
// (12 with three terms; 1 with 4-bit hidden rows). x: the hidden block, as 4
// 16-byte vectors of bf16 (of each term), or its codes.
template <int H>
__device__ __forceinline__ f32x4_t mx4_block(u32x4_t w, uint32_t s,
                                             const u32x4_t (&x)[H == 0 ? 4 : H == 1 ? 12 : 1],
                                             uint32_t hs, f32x4_t c) {
  if constexpr (H == 2) {
    return mfma_mx4(w, x[0], c, (int)s, (int)hs);
  } else {
    const float sc = __builtin_bit_cast(float, s << 23);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const u32x4_t f = mx4_unpack8(w[i], sc);
      // the smallest terms first
      if constexpr (H == 1) {
        c = mfma_slot(f, x[8 + i], c, (__bf16*)nullptr);
        c = mfma_slot(f, x[4 + i], c, (__bf16*)nullptr);
      }
      c = mfma_slot(f, x[i], c, (__bf16*)nullptr);
    }
    return c;
  }
}
// 8 fp32 elements in two vectors -> vector i of each term of a block
__device__ __forceinline__ void mx4_cut(u32x4_t lo, u32x4_t hi, u32x4_t (&t)[3]) {
  const f32x4_t a = __builtin_bit_cast(f32x4_t, lo), b = __builtin_bit_cast(f32x4_t, hi);
  const float f[8] = {a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
  cut8(f, t);
}

// Up to 16 hidden rows. Bound by reading W: a workgroup takes 16 R rows of it, whose
// columns its waves share, a range of pieces each, with the next piece's codes in flight;
// nothing of W passes through LDS. Hidden rows come from the caches. The waves' sums
// are added in LDS in order. Columns behind the last hidden row hold that row again
// (no branch around the loads) and are not stored.
template <int H, int R>
__global__ __launch_bounds__(512) void k_mx4_rows(Mx4Args a) {
  extern __shared__ __attribute__((aligned(16))) char lds[];
  const int lane = threadIdx.x & 63, wave = wave_id(), KS = blockDim.x >> 6;
  const int m = lane & 15, g = lane >> 4;
  const int v0 = blockIdx.x * 16 * R;
  const int nrows = (int)a.N;
  Mx4Weights<R> W;
  W.init(a, v0);
  const int nb32 = W.nb32, units = (nb32 + 7) / 8;
  const int per = (units + KS - 1) / KS;
  const int u0 = wave * per, u1 = min(units, u0 + per);
  constexpr int HB = H == 0 ? 64 : H == 1 ? 128 : 16;  // bytes of a block of a hidden row
  const int n = min(m, nrows - 1);
  const char* hrow = static_cast<const char*>(a.hidden) + (int64_t)n * a.hld;
  f32x4_t acc[R];
#pragma unroll
  for (int r = 0; r < R; ++r) acc[r] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  u32x4_t cw[2][R];
  W.load_scales(u0, m, g);
#pragma unroll
  for (int h = 0; h < 2; ++h) W.load(u0, h, u0 < u1 ? nb32 : 0, m, g, cw[h]);
  for (int u = u0; u < u1; ++u) {
    const int t = (u - u0) & 3;
    if (t == 0) W.turn(u, m, g);
    u32x4_t w[2][R];
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int r = 0; r < R; ++r) w[h][r] = cw[h][r];
#pragma unroll
    for (int h = 0; h < 2; ++h) W.load(u + 1, h, u + 1 < u1 ? nb32 : 0, m, g, cw[h]);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int b = 8 * u + 4 * h + g;
      const u32x4_t* p = reinterpret_cast<const u32x4_t*>(hrow + (int64_t)min(b, nb32 - 1) * HB);
      constexpr int NV = HB / 16;
      u32x4_t v[NV];
#pragma unroll
      for (int i = 0; i < NV; ++i) v[i] = p[i];
      uint32_t hs = 0;
      if constexpr (H == 2) hs = a.hscales[n * nb32 + min(b, nb32 - 1)];
      if (8 * u + 8 > nb32) {  // zeros past the row's end: codes of 0 times an infinity
        if (b >= nb32) {
          hs = 0;
#pragma unroll
          for (int i = 0; i < NV; ++i) v[i] = u32x4_t{0u, 0u, 0u, 0u};
        }
      }
      u32x4_t x[H == 0 ? 4 : H == 1 ? 12 : 1];
      if constexpr (H == 1) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          u32x4_t c[3];
          mx4_cut(v[2 * i], v[2 * i + 1], c);
#pragma unroll
          for (int k = 0; k < 3; ++k) x[4 * k + i] = c[k];
        }
      } else {
#pragma unroll
        for (int i = 0; i < NV; ++i) x[i] = v[i];
      }
#pragma unroll
      for (int r = 0; r < R; ++r)
        acc[r] = mx4_block<H>(w[h][r], W.scale(r, u, h, t, m, g), x, hs, acc[r]);
    }
  }

  f32x4_t* red = reinterpret_cast<f32x4_t*>(lds);
#pragma unroll
  for (int r = 0; r < R; ++r) red[(wave * R + r) * 64 + lane] = acc[r];
  __syncthreads();
  const float* rf = reinterpret_cast<const float*>(lds);
  for (int e = threadIdx.x; e < 16 * R * nrows; e += blockDim.x) {
    const int vl = e % (16 * R), nn = e / (16 * R);
    if (vl >= W.vrows) continue;
    const int at = ((vl >> 4) * 64 + ((vl >> 2) & 3) * 16 + nn) * 4 + (vl & 3);
    float z = 0.f;
    for (int k = 0; k < KS; ++k) z += rf[k * R * 256 + at];
    const int64_t o = nn * a.ldo + v0 + vl;
    if (a.out_bf16) static_cast<__bf16*>(a.out)[o] = (__bf16)z;
    else static_cast<float*>(a.out)[o] = z;
  }
}

// 4 consecutive logits of a row; `wide` where the rows allow 4 elements a store
__device__ __forceinline__ void mx4_put4(const Mx4Args& a, int64_t n, int v, f32x4_t z, bool wide) {
  const int64_t o = n * a.ldo + v;
  if (wide && v + 4 <= a.V) {
    if (a.out_bf16)
      *reinterpret_cast<u32x2_t*>(static_cast<__bf16*>(a.out) + o) =
          u32x2_t{pack_bf16x2(z[0], z[1]), pack_bf16x2(z[2], z[3])};
    else
      *reinterpret_cast<f32x4_t*>(static_cast<float*>(a.out) + o) = z;
    return;
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if (v + i >= a.V) break;
    if (a.out_bf16) static_cast<__bf16*>(a.out)[o + i] = (__bf16)z[i];
    else static_cast<float*>(a.out)[o + i] = z[i];
  }
}
__device__ __forceinline__ bool mx4_wide(const Mx4Args& a) {
  const uintptr_t eb = a.out_bf16 ? 2 : 4;
  return ((reinterpret_cast<uintptr_t>(a.out) | ((uintptr_t)a.ldo * eb)) & (4 * eb - 1)) == 0;
}

// 17 hidden rows and more, 16 NB a workgroup: its 8 waves take 16 R rows of W each and
// share the hidden rows' columns through LDS, a stage of 256 (fp32: 128) of them at a
// time in two buffers, one barrier a stage. Codes go from memory to registers, those of the
// next piece as soon as a half's are used.
constexpr int kMx4Stages(int H) { return H == 1 ? 2 : 1; }  // of a piece
constexpr int mx4_token_bytes(int H) {  // of a stage in LDS: fp32 as three terms of bf16
  return H == 0 ? 512 : H == 1 ? 768 : 128;
}
constexpr int mx4_stage_bytes(int H, int NB) {
  return 16 * NB * (mx4_token_bytes(H) + (H == 2 ? 8 : 0));  // 4 bits: with scales
}

template <int H, int NB, int R>
__global__ __launch_bounds__(512, NB * R <= 8 && R <= 2 ? 4 : 2) void k_mx4_wide(Mx4Args a) {
  __shared__ __attribute__((aligned(16))) char lds[2 * mx4_stage_bytes(H, NB)];
  constexpr int TB = mx4_token_bytes(H), STAGE = mx4_stage_bytes(H, NB), NST = kMx4Stages(H);
  constexpr int HB = H == 0 ? 64 : H == 1 ? 128 : 16;   // bytes of a block in memory
  constexpr int SB = 8 / NST;                           // blocks of a stage
  constexpr int PV = H == 1 ? 2 : 1;                    // 16-byte vectors of a thread's load
  constexpr int PT = SB * HB / 16 / PV;                 // loads of a token's stage
  constexpr int LT = (16 * NB * PT + 511) / 512;        // loads of a thread
  const int tid = threadIdx.x, lane = tid & 63, wave = wave_id();
  const int m = lane & 15, g = lane >> 4;
  const int v0 = (blockIdx.x * 8 + wave) * 16 * R;
  const int64_t n0 = (int64_t)blockIdx.y * 16 * NB;
  const int nrows = (int)min((int64_t)16 * NB, a.N - n0);
  Mx4Weights<R> W;
  W.init(a, min(v0, a.V));
  const int nb32 = W.nb32, units = (nb32 + 7) / 8;
  f32x4_t acc[R][NB];
#pragma unroll
  for (int r = 0; r < R; ++r)
#pragma unroll
    for (int q = 0; q < NB; ++q) acc[r][q] = f32x4_t{0.f, 0.f, 0.f, 0.f};

  // the hidden rows' stage st: load l of a thread is number tid + 512 l, PT a token
  u32x4_t hv[LT][PV];
  uint32_t hsv = 0;
  const char* hbase = static_cast<const char*>(a.hidden) + n0 * a.hld;
  auto fetch = [&](int st) {
#pragma unroll
    for (int l = 0; l < LT; ++l) {
      const int p = tid + 512 * l;
      const int tok = min(p / PT, nrows - 1), b = SB * st + (p % PT) * (16 * PV) / HB;
      const char* q = hbase + (int64_t)tok * a.hld + (int64_t)min(b, nb32 - 1) * HB +
                      (p % PT) * (16 * PV) % HB;
#pragma unroll
      for (int i = 0; i < PV; ++i) {
        hv[l][i] = reinterpret_cast<const u32x4_t*>(q)[i];
        if (b >= nb32) hv[l][i] = u32x4_t{0u, 0u, 0u, 0u};
      }
    }
    if constexpr (H == 2) {
      const int tok = min(tid >> 3, nrows - 1), b = SB * st + (tid & 7);
      hsv = a.hscales[(n0 + tok) * nb32 + min(b, nb32 - 1)];
      if (b >= nb32) hsv = 0;
    }
  };
  // to LDS: rows of TB bytes, 16-byte slots XORed with the token's low bits, which
  // leaves 8 lanes of a read (8 tokens, one slot) and of a write (8 slots of a token) in
  // 8 different ones
  auto put = [&](int buf) {
    char* s = lds + buf * STAGE;
#pragma unroll
    for (int l = 0; l < LT; ++l) {
      const int p = tid + 512 * l, tok = p / PT, slot = p % PT;
      if (16 * NB * PT % 512 != 0 && tok >= 16 * NB) continue;
      if constexpr (H == 1) {
        u32x4_t c[3];
        mx4_cut(hv[l][0], hv[l][1], c);
#pragma unroll
        for (int k = 0; k < 3; ++k)
          *reinterpret_cast<u32x4_t*>(s + tok * TB + k * 256 + ((slot ^ (tok & 7)) << 4)) = c[k];
      } else {
        *reinterpret_cast<u32x4_t*>(s + tok * TB + ((slot ^ (tok & 7)) << 4)) = hv[l][0];
      }
    }
    if constexpr (H == 2)
      if (tid < 16 * NB * 8) s[16 * NB * TB + tid] = (char)hsv;
  };

  u32x4_t w[2][R];
  W.load_scales(0, m, g);
#pragma unroll
  for (int h = 0; h < 2; ++h) W.load(0, h, nb32, m, g, w[h]);
  fetch(0);
  put(0);
  __syncthreads();
  int buf = 0;
  for (int u = 0; u < units; ++u) {
    const int t = u & 3;
    if (t == 0) W.turn(u, m, g);
#pragma unroll
    for (int st = 0; st < NST; ++st) {
      const bool more = st + 1 < NST || u + 1 < units;
      // (before the next codes: put waits for it, and not for them)
      if (more) fetch(NST * u + st + 1);
      const char* s = lds + buf * STAGE;
#pragma unroll
      for (int hh = 0; hh < 2 / NST; ++hh) {
        const int h = NST == 1 ? hh : st;
        const int sb = NST == 1 ? 4 * hh + g : g;  // block of the stage
        uint32_t ws[R];
#pragma unroll
        for (int r = 0; r < R; ++r) ws[r] = W.scale(r, u, h, t, m, g);
        if constexpr (H == 2) {
#pragma unroll
          for (int q = 0; q < NB; ++q) {
            const int tok = 16 * q + m;
            const u32x4_t x[1] = {
                *reinterpret_cast<const u32x4_t*>(s + tok * TB + ((sb ^ (tok & 7)) << 4))};
            const uint32_t hs = (uint8_t)s[16 * NB * TB + tok * 8 + sb];
#pragma unroll
            for (int r = 0; r < R; ++r) acc[r][q] = mx4_block<2>(w[h][r], ws[r], x, hs, acc[r][q]);
          }
        } else {
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            u32x4_t f[R];
#pragma unroll
            for (int r = 0; r < R; ++r)
              f[r] = mx4_unpack8(w[h][r][i], __builtin_bit_cast(float, ws[r] << 23));
#pragma unroll
            for (int q = 0; q < NB; ++q) {
              const int tok = 16 * q + m;
#pragma unroll
              for (int k = H == 1 ? 2 : 0; k >= 0; --k) {
                const u32x4_t x = *reinterpret_cast<const u32x4_t*>(
                    s + tok * TB + k * 256 + (((4 * sb + i) ^ (tok & 7)) << 4));
#pragma unroll
                for (int r = 0; r < R; ++r)
                  acc[r][q] = mfma_slot(f[r], x, acc[r][q], (__bf16*)nullptr);
              }
            }
          }
        }
        W.load(u + 1, h, nb32, m, g, w[h]);
      }
      if (more) put(buf ^ 1);
      __syncthreads();
      buf ^= 1;
    }
  }

  const bool wide = mx4_wide(a);
#pragma unroll
  for (int q = 0; q < NB; ++q) {
    const int n = 16 * q + m;
    if (n >= nrows) continue;
#pragma unroll
    for (int r = 0; r < R; ++r) mx4_put4(a, n0 + n, v0 + 16 * r + 4 * g, acc[r][q], wide);
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

template <int H, int R>
static int launch_mx4_rows(const Mx4Args& a, int ks, hipStream_t s) {
  hipLaunchKernelGGL((k_mx4_rows<H, R>), dim3((a.V + 16 * R - 1) / (16 * R)), dim3(64 * ks),
                     (size_t)ks * R * 1024, s, a);
  return (int)hipGetLastError();
}

template <int H, int NB, int R>
static int launch_mx4_wide(const Mx4Args& a, hipStream_t s) {
  const int64_t per = 16 * NB, ty = (a.N + per - 1) / per;
  // (the grid's second dimension holds 65535 tiles)
  for (int64_t t = 0; t < ty; t += 65535) {
    Mx4Args b = a;
    b.hidden = static_cast<const char*>(a.hidden) + t * per * a.hld;
    if (H == 2) b.hscales = a.hscales + t * per * (a.D / kMx4Block);
    b.out = static_cast<char*>(a.out) + t * per * a.ldo * (a.out_bf16 ? 2 : 4);
    b.N = a.N - t * per;
    hipLaunchKernelGGL((k_mx4_wide<H, NB, R>),
                       dim3((a.V + 128 * R - 1) / (128 * R),
                            (unsigned)(ty - t < 65535 ? ty - t : 65535)),
                       dim3(512), 0, s, b);
  }
  return (int)hipGetLastError();
}

template <int H>
static int launch_mx4_logits(const KdMx4Args& q, hipStream_t s) {
  Mx4Args a{};
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
  if (q.N <= 16) {
    const int units = (a.D / kMx4Block + 7) / 8;
    int ks = 1;
    while (ks < 4 && ks < units) ks *= 2;
    if (a.V <= 16384) return launch_mx4_rows<H, 1>(a, ks, s);
    return launch_mx4_rows<H, 2>(a, ks, s);
  }
  // rows of W a wave: as many as leave a workgroup for each compute unit
  constexpr int R4 = H == 1 ? 2 : 4;
  if (q.N <= 32) {
    if (a.V > 32768) return launch_mx4_wide<H, 2, R4>(a, s);
    return launch_mx4_wide<H, 2, 1>(a, s);
  }
  if (a.V > 65536) return launch_mx4_wide<H, 4, R4>(a, s);
  if (a.V > 32768) return launch_mx4_wide<H, 4, 2>(a, s);
  return launch_mx4_wide<H, 4, 1>(a, s);
}

extern "C" int kd_launch_mx4_logits(const KdMx4Args* a, void* stream) {
  hipStream_t s = static_cast<hipStream_t>(stream);
  switch (a->dtype) {
    case 0: return launch_mx4_logits<1>(*a, s);
    case 1: return launch_mx4_logits<0>(*a, s);
    default: return launch_mx4_logits<2>(*a, s);
  }
}
