// HIP kernels (gfx950) of 4-bit microscaled numbers and their launchers:
//   mx4_write, mx4_read    a matrix to codes and scales, and back
//   logits of hidden rows with a head W of such numbers, by the rule of kd_mx4_plan:
//   mx4_rows               few hidden rows, small heads
//   mx4_wide               few hidden rows
//   [mx4_terms,] mx4_scale_tiles, mx4_gemm     many, in bf16 (fp32 ones as three terms)
//   mx4_scale_tiles, mx4_gemm4                 many, in 4 bits
//   each of the last three with mx4_join where its columns are split into ranges
#include "kd_mx4.h"
#include "kd_ops.h"

namespace kd {

// ------------------------------------------------------ write and read -----
// Streams of 16 bytes a thread. Results of 64 MiB and more (kMx4Big), which nothing reads
// soon, are stored past the caches.
constexpr int64_t kMx4Big = (int64_t)64 << 20;
template <bool BIG, typename V>
__device__ __forceinline__ void mx4_store(V v, V* p) {
  if constexpr (BIG) __builtin_nontemporal_store(v, p);
  else *p = v;
}

// Eight elements a thread, four threads a block of 32. Bound by memory: 131072 x 4096 in
// bf16 230 to 244 us (medians on two cards), 5.6 to 5.9 TB/s of matrix, codes and scales;
// back 231 to 234 us, 5.8 TB/s. fp32 459 us, 5.3 TB/s, and 535 us, 4.5 TB/s.
template <typename T>
__global__ __launch_bounds__(256) void k_mx4_write(const T* __restrict__ x, int64_t n8,
                                                   uint32_t* __restrict__ codes,
                                                   uint8_t* __restrict__ scales) {
  const int64_t stride = (int64_t)gridDim.x * 256;
  // (n8 is a multiple of 4: the four threads of a block run or stop together)
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n8; i += stride) {
    float v[8];
    if constexpr (sizeof(T) == 2) {
      const u32x4_t q = reinterpret_cast<const u32x4_t*>(x)[i];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        v[2 * j] = __builtin_bit_cast(float, q[j] << 16);
        v[2 * j + 1] = __builtin_bit_cast(float, q[j] & 0xffff0000u);
      }
    } else {
      const f32x4_t q = reinterpret_cast<const f32x4_t*>(x)[2 * i];
      const f32x4_t r = reinterpret_cast<const f32x4_t*>(x)[2 * i + 1];
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
  // k_mx4_wide: pieces of 256 columns of a range, and with several ranges their sums
  // [range][N][Vp], which are joined afterwards
  int per;
  float* part;
  int64_t Vp;
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
  // requests as the codes': one row of 131072 x 4096 81 us, this way, at that time, 61.)
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

// Up to 16 hidden rows and a small W, whose workgroups would be too few if each took more
// of it. Bound by latency: 8000 x 4096 for one row 6.8 us (k_mx4_wide 19), 2000 x 1024 2.9
// (5.5); from 32000 rows of W on its hidden rows' reads cost more (16 rows of 32000 x 4096
// 26.5 us, k_mx4_wide 21). A workgroup takes 16 R rows of it, whose
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

// 4 consecutive logits of a row (stored together at any element boundary, which the
// target allows)
__device__ __forceinline__ void mx4_put4(const Mx4Args& a, int64_t n, int v, f32x4_t z) {
  const int64_t o = n * a.ldo + v;
  if (v + 4 <= a.V) {
    if (a.out_bf16) {
      const u32x2_t x = {pack_bf16x2(z[0], z[1]), pack_bf16x2(z[2], z[3])};
      __builtin_memcpy(static_cast<__bf16*>(a.out) + o, &x, 8);
    } else {
      __builtin_memcpy(static_cast<float*>(a.out) + o, &z, 16);
    }
    return;
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if (v + i >= a.V) break;
    if (a.out_bf16) static_cast<__bf16*>(a.out)[o + i] = (__bf16)z[i];
    else static_cast<float*>(a.out)[o + i] = z[i];
  }
}

// 16 NB hidden rows a workgroup: its 8 waves take 16 R rows of W each and share the hidden
// rows' columns through LDS, a stage of 256 (fp32: 128) of them at a time in two
// buffers, one barrier a stage. Where workgroups are few, the columns are split into
// ranges. Codes go from memory to registers, those of the next piece as soon as a
// half's are used. Bound by reading W while hidden rows are few: 131072 x 4096, one launch
// after the other, bf16 logits (medians), for 1 row 55 us (5.2 TB/s; reading alone 48 at
// 5.6), for 16 56, for 32 60; 64 rows 71 (77 with fp32 logits), whose MFMAs take 30 and
// which one workgroup a compute unit does not hide entirely (R = 4; fewer rows of W a wave
// read the hidden rows from LDS more often: R = 2 was a quarter slower). 4-bit rows 47, 49,
// 52, 62 us (1, 16, 32, 64), fp32 rows 70, 72, 103, 177.
constexpr int kMx4Stages(int H) { return H == 1 ? 2 : 1; }  // of a piece
constexpr int mx4_token_bytes(int H) {  // of a stage in LDS: fp32 as three terms of bf16
  return H == 0 ? 512 : H == 1 ? 768 : 128;
}
constexpr int mx4_stage_bytes(int H, int NB) {
  return 16 * NB * (mx4_token_bytes(H) + (H == 2 ? 8 : 0));  // 4 bits: with scales
}

template <int H, int NB, int R>
__global__ __launch_bounds__(512, NB * R <= 4 ? 4 : 2) void k_mx4_wide(Mx4Args a) {
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
  const int nb32 = W.nb32;
  const int ub = blockIdx.z * a.per, units = min(ub + a.per, (nb32 + 7) / 8);
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
      for (int i = 0; i < PV; ++i) hv[l][i] = reinterpret_cast<const u32x4_t*>(q)[i];
    }
    if constexpr (H == 2) {
      const int tok = min(tid >> 3, nrows - 1), b = SB * st + (tid & 7);
      hsv = a.hscales[(n0 + tok) * nb32 + min(b, nb32 - 1)];
    }
  };
  // to LDS: rows of TB bytes, 16-byte slots XORed with the token's low bits, which
  // leaves 8 lanes of a read (8 tokens, one slot) and of a write (8 slots of a token) in
  // 8 different ones. (With 64 bf16 rows a counter still gives conflicts 9% of the time; other
  // slots changed nothing.) Zeros past the rows' end (here: a choice behind the load would
  // wait for it there)
  auto put = [&](int buf, int st) {
    char* s = lds + buf * STAGE;
    if (SB * st + SB > nb32) {
#pragma unroll
      for (int l = 0; l < LT; ++l) {
        const int p = tid + 512 * l;
        if (SB * st + (p % PT) * (16 * PV) / HB >= nb32) {
#pragma unroll
          for (int i = 0; i < PV; ++i) hv[l][i] = u32x4_t{0u, 0u, 0u, 0u};
        }
      }
      if (H == 2 && SB * st + (tid & 7) >= nb32) hsv = 0;
    }
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
  W.load_scales(ub, m, g);
#pragma unroll
  for (int h = 0; h < 2; ++h) W.load(ub, h, nb32, m, g, w[h]);
  fetch(NST * ub);
  put(0, NST * ub);
  __syncthreads();
  int buf = 0;
  for (int u = ub; u < units; ++u) {
    const int t = (u - ub) & 3;
    if (t == 0) W.turn(u, m, g);
#pragma unroll
    for (int st = 0; st < NST; ++st) {
      const bool more = st + 1 < NST || u + 1 < units;
      // (before the next codes: put waits for it, and not for them)
      if (more) fetch(NST * u + st + 1);
      const char* s = lds + buf * STAGE;
      if constexpr (H == 2) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int sb = 4 * h + g;  // block of the stage
          uint32_t ws[R];
#pragma unroll
          for (int r = 0; r < R; ++r) ws[r] = W.scale(r, u, h, t, m, g);
#pragma unroll
          for (int q = 0; q < NB; ++q) {
            const int tok = 16 * q + m;
            const u32x4_t x[1] = {
                *reinterpret_cast<const u32x4_t*>(s + tok * TB + ((sb ^ (tok & 7)) << 4))};
            const uint32_t hs = (uint8_t)s[16 * NB * TB + tok * 8 + sb];
#pragma unroll
            for (int r = 0; r < R; ++r) acc[r][q] = mx4_block<2>(w[h][r], ws[r], x, hs, acc[r][q]);
          }
          W.load(u + 1, h, nb32, m, g, w[h]);
        }
      } else {
        // groups of NB R MFMAs (8 columns a lane, one term); the hidden rows and the codes
        // of a group are read and decoded while the group before it runs
        constexpr int TERMS = H == 1 ? 3 : 1, NG = 8 / NST * TERMS;
        u32x4_t x[2][NB], f[2][R];
        float sc[R];
        auto read = [&](int e) {
          const int sb = NST == 1 ? 4 * (e / 4 / TERMS) + g : g, i = e / TERMS % 4, k = TERMS - 1 - e % TERMS;
#pragma unroll
          for (int q = 0; q < NB; ++q) {
            const int tok = 16 * q + m;
            x[e & 1][q] = *reinterpret_cast<const u32x4_t*>(
                s + tok * TB + k * 256 + (((4 * sb + i) ^ (tok & 7)) << 4));
          }
        };
        auto decode = [&](int e) {
          const int h = NST == 1 ? e / 4 / TERMS : st, i = e / TERMS % 4;
          if (i == 0) {
#pragma unroll
            for (int r = 0; r < R; ++r)
              sc[r] = __builtin_bit_cast(float, W.scale(r, u, h, t, m, g) << 23);
          }
#pragma unroll
          for (int r = 0; r < R; ++r) f[e / TERMS & 1][r] = mx4_unpack8(w[h][r][i], sc[r]);
          if (i == 3) W.load(u + 1, h, nb32, m, g, w[h]);
        };
        read(0);
        decode(0);
#pragma unroll
        for (int e = 0; e < NG; ++e) {
          if (e + 1 < NG) read(e + 1);
          if (e + 1 < NG && (e + 1) % TERMS == 0) decode(e + 1);
#pragma unroll
          for (int q = 0; q < NB; ++q)
#pragma unroll
            for (int r = 0; r < R; ++r)
              acc[r][q] = mfma_slot(f[e / TERMS & 1][r], x[e & 1][q], acc[r][q], (__bf16*)nullptr);
          __builtin_amdgcn_sched_barrier(0);
        }
      }
      if (more) put(buf ^ 1, NST * u + st + 1);
      __syncthreads();
      buf ^= 1;
    }
  }

  if (a.part != nullptr) {
    a.out = a.part + blockIdx.z * a.N * a.Vp;
    a.ldo = a.Vp;
    a.out_bf16 = 0;
  }
#pragma unroll
  for (int q = 0; q < NB; ++q) {
    const int n = 16 * q + m;
    if (n >= nrows) continue;
#pragma unroll
    for (int r = 0; r < R; ++r) mx4_put4(a, n0 + n, v0 + 16 * r + 4 * g, acc[r][q]);
  }
}

// ------------------------------------------------------ many hidden rows --
// Scale bytes as the tiles below take them: of each 64 rows and 128 columns (4 blocks) 256
// bytes [g][m][b] = scale of row 16 b + m, block g, zeros past the rows and blocks that
// exist (a block of scale 2^-127 on both sides, or of a hidden row's zeros, adds
// nothing). A lane's dword then holds the four row blocks of a wave, which the scaled
// instructions select from; and 256 bytes are a wave's load.
__host__ __device__ constexpr int64_t mx4_tile_steps(int64_t D) {  // of 128 columns, even
  return (D / kMx4Block + 7) / 8 * 2;
}
__host__ __device__ constexpr int64_t mx4_tile_groups(int64_t rows) { return (rows + 255) / 256 * 4; }

// A workgroup per 64 rows and 32 steps, which pass through LDS: reads of 128 bytes of
// each row, writes of 256 (dword by dword, 16 bytes of a row at a time, 131072 x 128 took 38
// us).
constexpr int kMx4TileSteps = 32;
struct Mx4Scales {
  const uint8_t* scales;
  int64_t rows;
  uint8_t* out;
  int blocks;
};
// two matrices of as many columns: blocks [0, a.blocks) are the first one's
__global__ __launch_bounds__(256) void k_mx4_scale_tiles(Mx4Scales a, Mx4Scales b, int nb32, int T) {
  constexpr int LD = 4 * kMx4TileSteps + 4;  // bytes of a row in LDS
  __shared__ __attribute__((aligned(4))) uint8_t lds[64 * LD];
  const bool second = (int)blockIdx.x >= a.blocks;
  const uint8_t* __restrict__ scales = second ? b.scales : a.scales;
  uint8_t* __restrict__ out = second ? b.out : a.out;
  const int64_t rows = second ? b.rows : a.rows;
  const int block = (int)blockIdx.x - (second ? a.blocks : 0);
  const int per = (T + kMx4TileSteps - 1) / kMx4TileSteps;
  const int64_t G = block / per;
  const int t0 = (int)(block - G * per) * kMx4TileSteps, b0 = 4 * t0;
  // 4 bytes a thread: 32 threads a row
  const int c = (threadIdx.x & 31) * 4;
  for (int r = threadIdx.x >> 5; r < 64; r += 8) {
    const int64_t row = G * 64 + r;
    uint32_t w = 0;
    if (row < rows) {
      const uint8_t* p = scales + row * nb32 + b0 + c;
      if (b0 + c + 4 <= nb32) {
        __builtin_memcpy(&w, p, 4);
      } else {
        for (int i = 0; i < 4; ++i)
          if (b0 + c + i < nb32) w |= (uint32_t)p[i] << (8 * i);
      }
    }
    *reinterpret_cast<uint32_t*>(lds + r * LD + c) = w;
  }
  __syncthreads();
  const int m = threadIdx.x & 15, g = (threadIdx.x >> 4) & 3;
  for (int t = threadIdx.x >> 6; t < kMx4TileSteps && t0 + t < T; t += 4) {
    uint32_t w = 0;
#pragma unroll
    for (int q = 0; q < 4; ++q) w |= (uint32_t)lds[(16 * q + m) * LD + 4 * t + g] << (8 * q);
    *reinterpret_cast<uint32_t*>(out + (G * T + t0 + t) * 256 + g * 64 + m * 4) = w;
  }
}

// fp32 hidden rows as three bf16 terms a 64 columns: [N][Dp / 64][lo, mid, hi][64], zeros
// from column D to Dp
__global__ __launch_bounds__(256) void k_mx4_terms(const char* __restrict__ hidden, int64_t hld,
                                                   int64_t N, int D, int Dp, char* out) {
  const int per = Dp / 8;  // pieces of 8 columns
  const int64_t stride = (int64_t)gridDim.x * 256;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < N * per; i += stride) {
    const int64_t n = i / per;
    const int p = (int)(i - n * per);
    u32x4_t c[3] = {{0u, 0u, 0u, 0u}, {0u, 0u, 0u, 0u}, {0u, 0u, 0u, 0u}};
    if (8 * p < D) {
      const u32x4_t* q = reinterpret_cast<const u32x4_t*>(hidden + n * hld + (int64_t)p * 32);
      mx4_cut(q[0], q[1], c);
    }
    u32x4_t* o = reinterpret_cast<u32x4_t*>(out + n * Dp * 6 + (int64_t)(p >> 3) * 384 + (p & 7) * 16);
    o[0] = c[2];
    o[8] = c[1];
    o[16] = c[0];
  }
}

struct Mx4GemmArgs {
  Mx4Args o;               // N, V, D, codes and the output
  const char* hidden;      // rows of bf16 (terms), or of codes
  int64_t hld;             // bytes between them
  int hbytes;              // bytes of one
  const uint8_t *wst, *hst;  // scales as tiles (hst: 4-bit hidden rows)
  int T;                   // 128-column steps of them
  int TV, TT;              // tiles of 256 rows of W and of 32 NJ hidden rows
  int per, splits;         // 64-column steps (256 with 4-bit hidden rows) of a range; ranges
  float* part;             // [splits][N][Vp] sums of each, or null with one
  int64_t Vp;
};

// One wave-wide 4-byte-per-lane LDS-DMA load (see dma_b128)
__device__ __forceinline__ void dma_b32(i32x4_t r, uint32_t lds_addr, uint32_t voff) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dword %1, %2, 0 offen lds"
               :
               : "s"(lds_addr), "v"(voff), "s"(r)
               : "memory");
}

// Workgroups are as many as the compute units; each takes the items blockIdx.x, + gridDim.x,
// ... of a.TV a.TT tiles, range of columns after range.
template <int NJ>
__device__ __forceinline__ void mx4_item(const Mx4GemmArgs& a, int item, int& v0, int64_t& n0,
                                         int& z) {
  const int tiles = a.TV * a.TT;
  int vt, tt;
  z = __builtin_amdgcn_readfirstlane(item / tiles);
  tile_at(tile_order_xcd(item - z * tiles, tiles), a.TV, a.TT, 4, vt, tt);
  // (scalar: the divisions are the vector unit's)
  v0 = __builtin_amdgcn_readfirstlane(vt) * 256;
  n0 = (int64_t)__builtin_amdgcn_readfirstlane(tt) * 32 * NJ;
}
// acc[i][j] of wave (wv, wt): rows 64 wv + 16 i + 4 g .. + 3 of W, hidden row 16 NJ wt + 16 j + m.
// By way of LDS (2 KiB a wave, its own, so that no barrier is needed): 16 hidden rows at a
// time, whole 128-byte lines (64 logits of bf16, 32 of fp32). Stored from the accumulators,
// 32 or 64 bytes of a row at a time, the tiles' stores took 0.34 (bf16 hidden rows) and
// 0.50 ms of 4096 x 4096 x 131072. True if every lane stored every line: then the wave
// has issued NJ * (bf16 ? 2 : 4) store instructions.
__device__ __forceinline__ void mx4_wave_sync() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}
template <int NJ, bool BF16>
__device__ __forceinline__ bool mx4_lines(const Mx4Args& o, int v, int64_t n0, char* st,
                                          const f32x4_t (&acc)[4][NJ]) {
  constexpr int EB = BF16 ? 2 : 4, EV = 16 / EB, HP = BF16 ? 1 : 2;
  int lane = threadIdx.x & 63;
  // (opaque: what depends on it is formed here, not held through the main loop)
  asm volatile("" : "+v"(lane));
  const int m = lane & 15, g = lane >> 4;
  // (8 rows by 32-bit offsets; a store of 16 bytes may lie at any element boundary)
  const bool full = v + 64 <= o.V && n0 + 16 * NJ <= o.N && o.ldo < (1 << 26);
  const int t0 = lane >> 3, c = lane & 7;
  const uint32_t off = (uint32_t)(t0 * (int)o.ldo + c * EV) * EB;
#pragma unroll
  for (int j = 0; j < NJ; ++j)
#pragma unroll
    for (int p = 0; p < HP; ++p) {
      if constexpr (BF16) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
          *reinterpret_cast<u32x2_t*>(st + m * 128 + (((2 * i + (g >> 1)) ^ (m & 7)) << 4) + 8 * (g & 1)) =
              u32x2_t{pack_bf16x2(acc[i][j][0], acc[i][j][1]), pack_bf16x2(acc[i][j][2], acc[i][j][3])};
      } else {
#pragma unroll
        for (int i = 0; i < 2; ++i)
          *reinterpret_cast<f32x4_t*>(st + m * 128 + (((4 * i + g) ^ (m & 7)) << 4)) = acc[2 * p + i][j];
      }
      mx4_wave_sync();
#pragma unroll
      for (int q = 0; q < 2; ++q) {
        const int t = 8 * q + t0;
        const u32x4_t x = *reinterpret_cast<const u32x4_t*>(st + t * 128 + ((c ^ (t & 7)) << 4));
        if (full) {
          char* row = static_cast<char*>(o.out) + ((n0 + 16 * j + 8 * q) * o.ldo + v + 32 * p) * EB;
          __builtin_memcpy(row + off, &x, 16);
          continue;
        }
        const int64_t n = n0 + 16 * j + t;
        const int vv = v + 32 * p + c * EV;
        if (n >= o.N) continue;
        char* dst = static_cast<char*>(o.out) + (n * o.ldo + vv) * EB;
        if (vv + EV <= o.V) {
          __builtin_memcpy(dst, &x, 16);
        } else {
#pragma unroll
          for (int e = 0; e < EV; ++e) {
            if (vv + e >= o.V) break;
            if constexpr (BF16)
              reinterpret_cast<uint16_t*>(dst)[e] = (uint16_t)(x[e >> 1] >> (16 * (e & 1)));
            else
              reinterpret_cast<uint32_t*>(dst)[e] = x[e];
          }
        }
      }
      mx4_wave_sync();
      __builtin_amdgcn_sched_barrier(0);
    }
  return full;
}
// the wave's store instructions in flight: 0 if it has waited for them
template <int NJ>
__device__ __forceinline__ int mx4_tile_out(const Mx4GemmArgs& a, int v, int64_t n, int z, char* st,
                                            const f32x4_t (&acc)[4][NJ]) {
  Mx4Args o = a.o;
  if (a.part != nullptr) {
    o.out = a.part + (int64_t)z * o.N * a.Vp;
    o.ldo = a.Vp;
    o.out_bf16 = 0;
  }
  const bool full = o.out_bf16 ? mx4_lines<NJ, true>(o, v, n, st, acc) : mx4_lines<NJ, false>(o, v, n, st, acc);
  if (full) return o.out_bf16 ? 2 * NJ : 4 * NJ;
  KD_VMCNT(0);
  return 0;
}
// s_waitcnt vmcnt(n + the stores in flight): what was loaded before them has landed (loads
// and stores count in the order of their issue)
template <int NJ, int N>
__device__ __forceinline__ void mx4_wait(int stores) {
  if (stores == 0) KD_VMCNT(N);
  else if (stores == 2 * NJ) KD_VMCNT(N + 2 * NJ);
  else KD_VMCNT(N + 4 * NJ);
}
// MFMA pair q of 2 NJ: row block q / (NJ / 2) of W, two hidden blocks, back and forth
template <int NJ>
__device__ __forceinline__ void mx4_pair(int q, int& i, int& j0, int& j1) {
  i = q / (NJ / 2);
  const int jj = 2 * (q % (NJ / 2));
  j0 = (i & 1) ? NJ - 1 - jj : jj;
  j1 = (i & 1) ? NJ - 2 - jj : jj + 1;
}

// Tiles of 256 rows of W by 32 NJ hidden rows, bf16 hidden rows (TERMS = 1) or three
// terms each (3): 8 waves of 64 x 16 NJ. A step is 64 columns (of one term): hidden rows
// 128 bytes each in three stages, codes 32 bytes a row in two, scales of up to four steps
// in three, all by LDS-DMA two steps ahead; one barrier a step. A wave's 4 row blocks of W are
// decoded in registers between the MFMAs of the half step before their use: a block's
// codes are read from LDS twice (by two waves) and take a quarter of bf16's bytes: the LDS,
// which bounds the bf16 tiles of the loss, is active 30% of the time, the MFMAs 73% at the
// clock that power leaves. 4096 x 4096 x 131072: 2.92 ms, 1.5 PFLOP/s; with three terms 8.86
// ms, 1.5 PFLOP/s of them (k_mx4_terms 28 us).
// The steps of a workgroup's items form one sequence: a tile's last steps load the next
// tile's first ones, and its logits are stored under that tile's first step.
template <int TERMS, int NJ>
__global__ __launch_bounds__(512, 1) void k_mx4_gemm(Mx4GemmArgs a) {
  constexpr int TOK = 32 * NJ, HST = TOK * 128, CST = 256 * 32, SST = 2048;
  constexpr int NPW = NJ / 2, NP = 2 * NJ;
  __shared__ __attribute__((aligned(16))) char lds[3 * HST + 2 * CST + 3 * SST + 8 * 2048];
  char* const lc = lds + 3 * HST;
  char* const ls = lc + 2 * CST;
  const int lane = threadIdx.x & 63, wave = wave_id();
  char* const lo = ls + 3 * SST + wave * 2048;
  const int m = lane & 15, g = lane >> 4, wv = wave >> 1, wt = wave & 1;
  const int items = a.TV * a.TT * a.splits, steps = (a.o.D + 63) / 64 * TERMS, pitch = a.o.D / 2;

  // hidden rows: instruction i of the wave has rows 8 (NPW wave + i) .. + 7
  const int hslot = ((lane & 7) ^ (lane >> 3)) << 4;
  const uint32_t hoff = (uint32_t)(lane >> 3) * (uint32_t)a.hld + (uint32_t)hslot;
  // codes: rows 32 wave .. + 31, the 16-byte halves exchanged for every other 8 rows (the
  // 4-byte reads still conflict two ways, a sixth of the LDS's active time)
  const int crow = 32 * wave + (lane >> 1);
  const uint32_t coff = (uint32_t)crow * (uint32_t)pitch + (((lane & 1) ^ ((crow >> 3) & 1)) << 4);
  const uint32_t soff = (uint32_t)((wave & 3) * a.T * 256 + lane * 4);

  // the step to load next: lk of lk_end of item li, whose scales go to stage lsc
  i32x4_t rh, rc, rs;
  int li = (int)blockIdx.x, lk = 0, lk_end = 0, lsc = 2;
  auto open = [&]() {
    lk = lk_end = 0;
    if (li >= items) return;
    int v0, z;
    int64_t n0;
    mx4_item<NJ>(a, li, v0, n0, z);
    const int vrows = min(256, a.o.V - v0), nrows = (int)min((int64_t)TOK, a.o.N - n0);
    rh = rsrc_words(a.hidden + n0 * a.hld, (uint32_t)((nrows - 1) * a.hld + a.hbytes));
    rc = rsrc_words(a.o.codes + (int64_t)v0 * pitch, (uint32_t)(vrows * pitch));
    rs = rsrc_words(a.wst + (int64_t)(v0 / 64) * a.T * 256, (uint32_t)(4 * a.T * 256));
    lk = z * a.per;
    lk_end = min(lk + a.per, steps);
  };
  auto next = [&]() {
    if (++lk >= lk_end) {
      li += gridDim.x;
      open();
    }
  };
  auto dma_h = [&](int stage, int i) {
    const bool live = lk < lk_end && lk * 128 + hslot < a.hbytes;
    dma_b128(rh, __builtin_amdgcn_readfirstlane(lds_addr(lds + stage * HST) + (wave * NPW + i) * 1024),
             live ? hoff + ((uint32_t)((wave * NPW + i) * 8) * (uint32_t)a.hld + (uint32_t)lk * 128u)
                  : kOobOffset);
  };
  auto dma_c = [&](int stage) {
    dma_b128(rc, __builtin_amdgcn_readfirstlane(lds_addr(lc + stage * CST) + wave * 1024),
             lk < lk_end ? coff + (uint32_t)(lk / TERMS) * 32u : kOobOffset);
  };
  // at every fourth 64 columns: waves 0..3 the scales of two steps, 4..7 of the next two
  auto dma_s = [&]() {
    if (lk >= lk_end || lk % TERMS != 0 || (lk / TERMS & 3) != 0) return;
    lsc = lsc == 2 ? 0 : lsc + 1;
    const int t = (lk / TERMS >> 1) + (wave >> 2);
    dma_b32(rs, __builtin_amdgcn_readfirstlane(lds_addr(ls + lsc * SST) + wave * 256),
            t < a.T ? soff + (uint32_t)t * 256u : kOobOffset);
  };

  f32x4_t acc[4][NJ];
  // fragment addresses within a stage
  const int hrd = (16 * NJ * wt + m) * 128, hx = g ^ (m & 7);
  const int crd = (64 * wv + m) * 32 + 4 * g, cx = (m >> 3) & 1;
  const int srd = wv * 256 + m * 4;
  u32x4_t hf[2][NJ], wf[2][4];
  uint32_t raw[4], sc = 0;
  // half s of 64 columns number w, whose scales are in stage cs
  auto read_s = [&](int cs, int w, int s) {
    return *reinterpret_cast<const uint32_t*>(ls + cs * SST + ((w >> 1) & 1) * 1024 + srd +
                                              (2 * (w & 1) + s) * 64);
  };
  auto read_h = [&](const char* st, int s, int f) {
    return *reinterpret_cast<const u32x4_t*>(st + hrd + f * 2048 + ((hx ^ (4 * s)) << 4));
  };
  auto read_c = [&](const char* st, int s, int b) {
    return *reinterpret_cast<const uint32_t*>(st + crd + b * 512 + ((s ^ cx) << 4));
  };
  auto unpack = [&](int b) {
    const uint32_t e = b == 3 ? (sc >> 1) & 0x7f800000u : (sc << (23 - 8 * b)) & 0x7f800000u;
    return mx4_unpack8(raw[b], __builtin_bit_cast(float, e));
  };

  open();
#pragma unroll
  for (int p = 0; p < 2; ++p) {
    dma_s();
#pragma unroll
    for (int i = 0; i < NPW; ++i) dma_h(p, i);
    dma_c(p);
    next();
  }
  KD_VMCNT(0);
  __syncthreads();
  int item = (int)blockIdx.x, v0, z;
  int64_t n0;
  mx4_item<NJ>(a, item, v0, n0, z);
  int k = z * a.per, ke = min(k + a.per, steps);
  int ca = 0, cc = 0, cs = 0, stores = 0;  // stages of step k's hidden rows, codes and scales
#pragma unroll
  for (int f = 0; f < NJ; ++f) hf[0][f] = read_h(lds, 0, f);
  sc = read_s(0, k / TERMS, 0);
#pragma unroll
  for (int b = 0; b < 4; ++b) raw[b] = read_c(lc, 0, b);
#pragma unroll
  for (int b = 0; b < 4; ++b) wf[0][b] = unpack(b);
  // MFMAs of half x, reads of the other half y (half s of 64 columns w) between them
  constexpr int U0 = NP == 16 ? 8 : 4, US = NP == 16 ? 2 : 1, H0 = NP == 16 ? 4 : 2;
  auto half = [&](int q, int x, const char* hst, const char* cst, int css, int w, int s) {
    const int y = x ^ 1;
    int i, j0, j1;
    mx4_pair<NJ>(q, i, j0, j1);
    acc[i][j0] = mfma_slot(wf[x][i], hf[x][j0], acc[i][j0], (__bf16*)nullptr);
    acc[i][j1] = mfma_slot(wf[x][i], hf[x][j1], acc[i][j1], (__bf16*)nullptr);
    if (q == 0) sc = read_s(css, w, s);
    if (q < 4) raw[q] = read_c(cst, s, q);
    if (q >= H0 && q < H0 + NJ) hf[y][q - H0] = read_h(hst, s, q - H0);
    if (q >= U0 && (q - U0) % US == 0) wf[y][(q - U0) / US] = unpack((q - U0) / US);
    __builtin_amdgcn_sched_barrier(0);
  };
#pragma unroll 1
  while (true) {
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < NJ; ++j) acc[i][j] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    const int nitem = item + gridDim.x;
    int nv0 = 0, nz = 0;
    int64_t nn0 = 0;
    if (nitem < items) mx4_item<NJ>(a, nitem, nv0, nn0, nz);
#pragma unroll 1
    for (;;) {
      const int na = ca == 2 ? 0 : ca + 1, pa = ca == 0 ? 2 : ca - 1;
      // the step after this one, of the next tile behind the last (its first columns' scales
      // start a stage)
      const int kn = k + 1 < ke ? k + 1 : nz * a.per;
      const bool same = k + 1 < ke && (kn % TERMS != 0 || (kn / TERMS & 3) != 0);
      const int ncs = same ? cs : cs == 2 ? 0 : cs + 1;
      dma_s();
#pragma unroll
      for (int q = 0; q < NP; ++q) {
        if (q % 4 == 3) dma_h(pa, q / 4);
        half(q, 0, lds + ca * HST, lc + cc * CST, cs, k / TERMS, 1);
      }
      __builtin_amdgcn_s_waitcnt(0xc07f & ~0x0f00);  // lgkmcnt(0)
      mx4_wait<NJ, NPW>(stores);  // the next step landed; the hidden rows behind it may still fly
      stores = 0;
      __syncthreads();
      __builtin_amdgcn_s_setprio(1);
#pragma unroll
      for (int q = 0; q < NP; ++q) {
        if (q == 0) dma_c(cc);
        half(q, 1, lds + na * HST, lc + (cc ^ 1) * CST, ncs, kn / TERMS, 0);
      }
      __builtin_amdgcn_s_setprio(0);
      next();
      ca = na;
      cc ^= 1;
      cs = ncs;
      if (++k >= ke) break;
    }
    stores = mx4_tile_out<NJ>(a, v0 + 64 * wv, n0 + 16 * NJ * wt, z, lo, acc);
    if (nitem >= items) break;
    item = nitem;
    v0 = nv0;
    n0 = nn0;
    z = nz;
    k = z * a.per;
    ke = min(k + a.per, steps);
  }
  KD_VMCNT(0);  // loads into LDS end before the workgroup does
}

template <int OA, int OB>
__device__ __forceinline__ f32x4_t mfma_mx4_sel(const i32x8_t& x, const i32x8_t& y, f32x4_t c, int sa,
                                                int sb) {
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(x, y, c, 4, 4, OA, sa, OB, sb);
}
// one 16x16x128 step with the scales in byte ia of sa and ib of sb (constants once
// unrolled)
__device__ __forceinline__ f32x4_t mfma_mx4_at(u32x4_t a, u32x4_t b, f32x4_t c, int ia, uint32_t sa,
                                               int ib, uint32_t sb) {
  const i32x8_t x = {(int)a[0], (int)a[1], (int)a[2], (int)a[3], 0, 0, 0, 0};
  const i32x8_t y = {(int)b[0], (int)b[1], (int)b[2], (int)b[3], 0, 0, 0, 0};
  const int p = (int)sa, r = (int)sb;
  switch (4 * ia + ib) {
    case 0: return mfma_mx4_sel<0, 0>(x, y, c, p, r);
    case 1: return mfma_mx4_sel<0, 1>(x, y, c, p, r);
    case 2: return mfma_mx4_sel<0, 2>(x, y, c, p, r);
    case 3: return mfma_mx4_sel<0, 3>(x, y, c, p, r);
    case 4: return mfma_mx4_sel<1, 0>(x, y, c, p, r);
    case 5: return mfma_mx4_sel<1, 1>(x, y, c, p, r);
    case 6: return mfma_mx4_sel<1, 2>(x, y, c, p, r);
    case 7: return mfma_mx4_sel<1, 3>(x, y, c, p, r);
    case 8: return mfma_mx4_sel<2, 0>(x, y, c, p, r);
    case 9: return mfma_mx4_sel<2, 1>(x, y, c, p, r);
    case 10: return mfma_mx4_sel<2, 2>(x, y, c, p, r);
    case 11: return mfma_mx4_sel<2, 3>(x, y, c, p, r);
    case 12: return mfma_mx4_sel<3, 0>(x, y, c, p, r);
    case 13: return mfma_mx4_sel<3, 1>(x, y, c, p, r);
    case 14: return mfma_mx4_sel<3, 2>(x, y, c, p, r);
    default: return mfma_mx4_sel<3, 3>(x, y, c, p, r);
  }
}

// The same tiles with 4-bit hidden rows: a step is 256 columns, 128 bytes a row of codes in
// two stages by LDS-DMA, two scaled MFMAs a block pair. The second half of a step
// issues the loads of the step after the next, into the stage whose last
// fragments were read in its first half; the barrier between the halves waits for
// those of the next step. 4096 x 4096 x 131072: 1.10 ms, 4.0 PFLOP/s with the MFMAs 50% busy
// (from registers alone, at the clock that power leaves, these reach 5.5); 0.95 without the
// loads, 0.82 with neither these nor the fragments' reads, 0.15 of each the logits' stores.
template <int NJ>
__global__ __launch_bounds__(512, 1) void k_mx4_gemm4(Mx4GemmArgs a) {
  constexpr int TOK = 32 * NJ, HST = TOK * 128, CST = 256 * 128, SST = 8192;
  constexpr int NH = NJ / 2, NC = 4, NI = NC + NH + 1, NP = 2 * NJ;
  static_assert(NI <= NP, "a load a pair");
  __shared__ __attribute__((aligned(16))) char lds[2 * (HST + CST + SST) + 8 * 2048];
  char* const lc = lds + 2 * HST;
  char* const ls = lc + 2 * CST;
  const int lane = threadIdx.x & 63, wave = wave_id();
  char* const lo = ls + 2 * SST + wave * 2048;
  const int m = lane & 15, g = lane >> 4, wv = wave >> 1, wt = wave & 1;
  const int items = a.TV * a.TT * a.splits, steps = (a.o.D + 255) / 256, pitch = a.o.D / 2;
  const int lrow = lane >> 3, slot = ((lane & 7) ^ lrow) << 4;
  const uint32_t off = (uint32_t)lrow * (uint32_t)pitch + (uint32_t)slot;

  // the step to load next: lk of lk_end of item li
  i32x4_t rh, rc, rs;
  int li = (int)blockIdx.x, lk = 0, lk_end = 0;
  auto open = [&]() {
    lk = lk_end = 0;
    if (li >= items) return;
    int v0, z;
    int64_t n0;
    mx4_item<NJ>(a, li, v0, n0, z);
    const int vrows = min(256, a.o.V - v0), nrows = (int)min((int64_t)TOK, a.o.N - n0);
    rh = rsrc_words(a.hidden + n0 * pitch, (uint32_t)(nrows * pitch));
    rc = rsrc_words(a.o.codes + (int64_t)v0 * pitch, (uint32_t)(vrows * pitch));
    // scales: waves 0..3 a group of 64 rows of W each, 4..7 one of hidden rows; 512 bytes
    // a step by the first 32 lanes
    const int64_t group = wave >= 4 ? n0 / 64 + (wave & 3) % (TOK / 64) : v0 / 64 + wave;
    rs = rsrc_words((wave >= 4 ? a.hst : a.wst) + group * a.T * 256, (uint32_t)(a.T * 256));
    lk = z * a.per;
    lk_end = min(lk + a.per, steps);
  };
  auto next = [&]() {
    if (++lk >= lk_end) {
      li += gridDim.x;
      open();
    }
  };
  // instruction i of that step
  auto dma = [&](int st, int i) {
    const bool live = lk < lk_end;
    if (i == 0)
      dma_b128(rs, __builtin_amdgcn_readfirstlane(lds_addr(ls + st * SST) + wave * 1024),
               live && lane < 32 ? (uint32_t)(lk * 512 + lane * 16) : kOobOffset);
    else if (i <= NC)
      dma_b128(rc, __builtin_amdgcn_readfirstlane(lds_addr(lc + st * CST) + (wave * NC + i - 1) * 1024),
               live ? off + (uint32_t)((wave * NC + i - 1) * 8 * pitch + lk * 128) : kOobOffset);
    else
      dma_b128(rh, __builtin_amdgcn_readfirstlane(lds_addr(lds + st * HST) + (wave * NH + i - 1 - NC) * 1024),
               live ? off + (uint32_t)((wave * NH + i - 1 - NC) * 8 * pitch + lk * 128) : kOobOffset);
  };
  f32x4_t acc[4][NJ];
  const int hrd = (16 * NJ * wt + m) * 128, crd = (64 * wv + m) * 128, fx = g ^ (m & 7);
  u32x4_t hf[2][NJ], wf[2][4];
  uint32_t sw[2], sh[2][NJ / 4];
  // read number f of half s of the step in stage st, into set s
  constexpr int NR = 1 + NJ / 4 + 4 + NJ;
  auto read = [&](int st, int s, int f) {
    if (f == 0)
      sw[s] = *reinterpret_cast<const uint32_t*>(ls + st * SST + wv * 1024 + s * 256 + lane * 4);
    else if (f < 1 + NJ / 4)
      sh[s][f - 1] = *reinterpret_cast<const uint32_t*>(
          ls + st * SST + 4096 + ((wt * NJ / 4) + f - 1) * 1024 + s * 256 + lane * 4);
    else if (f < 5 + NJ / 4)
      wf[s][f - 1 - NJ / 4] = *reinterpret_cast<const u32x4_t*>(
          lc + st * CST + crd + (f - 1 - NJ / 4) * 2048 + ((fx ^ (4 * s)) << 4));
    else
      hf[s][f - 5 - NJ / 4] = *reinterpret_cast<const u32x4_t*>(
          lds + st * HST + hrd + (f - 5 - NJ / 4) * 2048 + ((fx ^ (4 * s)) << 4));
  };
  open();
#pragma unroll
  for (int p = 0; p < 2; ++p) {
#pragma unroll
    for (int i = 0; i < NI; ++i) dma(p, i);
    next();
  }
  KD_VMCNT(NI);
  __syncthreads();
#pragma unroll
  for (int f = 0; f < NR; ++f) read(0, 0, f);
  // MFMAs of half x, and the reads of half x ^ 1 (of the step in stage st) between them
  auto half = [&](int q, int x, int st) {
    int i, j0, j1;
    mx4_pair<NJ>(q, i, j0, j1);
    acc[i][j0] = mfma_mx4_at(wf[x][i], hf[x][j0], acc[i][j0], i, sw[x], j0 & 3, sh[x][j0 >> 2]);
    acc[i][j1] = mfma_mx4_at(wf[x][i], hf[x][j1], acc[i][j1], i, sw[x], j1 & 3, sh[x][j1 >> 2]);
#pragma unroll
    for (int f = 0; f < NR; ++f)
      if (f * NP / NR == q) read(st, x ^ 1, f);
    __builtin_amdgcn_sched_barrier(0);
  };
  int st = 0, stores = 0;
#pragma unroll 1
  for (int item = (int)blockIdx.x; item < items; item += gridDim.x) {
    int v0, z;
    int64_t n0;
    mx4_item<NJ>(a, item, v0, n0, z);
    const int ke = min((z + 1) * a.per, steps);
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < NJ; ++j) acc[i][j] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll 1
    for (int k = z * a.per; k < ke; ++k) {
#pragma unroll
      for (int q = 0; q < NP; ++q) half(q, 0, st);
      __builtin_amdgcn_s_waitcnt(0xc07f & ~0x0f00);  // lgkmcnt(0)
      mx4_wait<NJ, 0>(stores);  // the next step landed
      stores = 0;
      __syncthreads();
      __builtin_amdgcn_s_setprio(1);
#pragma unroll
      for (int q = 0; q < NP; ++q) {
        if (q < NI) dma(st, q);
        half(q, 1, st ^ 1);
      }
      __builtin_amdgcn_s_setprio(0);
      next();
      st ^= 1;
    }
    stores = mx4_tile_out<NJ>(a, v0 + 64 * wv, n0 + 16 * NJ * wt, z, lo, acc);
  }
  KD_VMCNT(0);  // loads into LDS end before the workgroup does
}

// out = the ranges' sums, in order
__global__ __launch_bounds__(256) void k_mx4_join(const float* __restrict__ part, int splits,
                                                  int64_t N, int64_t V, int64_t Vp, void* out,
                                                  int64_t ldo, int out_bf16) {
  const int64_t per = Vp / 4, stride = (int64_t)gridDim.x * 256;
  Mx4Args o{};
  o.out = out;
  o.ldo = ldo;
  o.V = (int)V;
  o.out_bf16 = out_bf16;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < N * per; i += stride) {
    const int64_t n = i / per;
    f32x4_t z = {0.f, 0.f, 0.f, 0.f};
    for (int k = 0; k < splits; ++k)
      z += reinterpret_cast<const f32x4_t*>(part)[(int64_t)k * N * per + i];
    mx4_put4(o, n, (int)(i - n * per) * 4, z);
  }
}

}  // namespace kd

using namespace kd;

// Workgroups of a stream of n pieces: a piece a thread, two where there are many (131072 x
// 4096 in bf16 written by 2048, 16384, 131072 and 262144 workgroups 269, 302, 218 and 233 us,
// read by them 254, 304, 232 and 233: the fewer, the farther apart what they touch at a time).
static unsigned mx4_blocks(int64_t n) {
  const int64_t b = (n + 255) / 256;
  const int64_t c = b <= 16384 ? b : (b + 1) / 2;
  return (unsigned)(c < (1 << 22) ? c : 1 << 22);
}

template <typename T>
static int launch_mx4_write(const void* x, int64_t n, uint8_t* codes, uint8_t* scales,
                            hipStream_t s) {
  hipLaunchKernelGGL(k_mx4_write<T>, dim3(mx4_blocks(n / 8)), dim3(256), 0, s, static_cast<const T*>(x), n / 8,
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

static int launch_mx4_join(const KdMx4Args& q, const KdMx4Plan& p, int64_t rows, void* out,
                           hipStream_t s) {
  const int64_t Vp = (q.V + 3) / 4 * 4;
  hipLaunchKernelGGL(k_mx4_join, dim3(mx4_blocks(rows * Vp / 4)), dim3(256), 0, s,
                     reinterpret_cast<const float*>(q.ws + p.off_part), p.splits, rows, q.V, Vp, out,
                     q.ld_out, q.out_dtype == 1);
  return (int)hipGetLastError();
}

// hidden rows [0, o.N) of the call, at most 65535 tiles of 16 NB
template <int H, int NB, int R>
static int launch_mx4_wide(const KdMx4Args& q, const KdMx4Plan& p, Mx4Args o, hipStream_t s) {
  o.per = p.per;
  o.Vp = (q.V + 3) / 4 * 4;
  o.part = p.splits > 1 ? reinterpret_cast<float*>(q.ws + p.off_part) : nullptr;
  hipLaunchKernelGGL((k_mx4_wide<H, NB, R>),
                     dim3((o.V + 128 * R - 1) / (128 * R), (unsigned)((o.N + 16 * NB - 1) / (16 * NB)),
                          (unsigned)p.splits),
                     dim3(512), 0, s, o);
  if (p.splits > 1) return launch_mx4_join(q, p, o.N, o.out, s);
  return (int)hipGetLastError();
}

constexpr int64_t kMx4Units = 256;  // compute units

static Mx4Scales mx4_scales(const uint8_t* scales, int64_t rows, int64_t D, void* out) {
  const int64_t per = (mx4_tile_steps(D) + kMx4TileSteps - 1) / kMx4TileSteps;
  return Mx4Scales{scales, rows, static_cast<uint8_t*>(out), (int)(mx4_tile_groups(rows) * per)};
}
static int launch_mx4_scale_tiles(const Mx4Scales& a, const Mx4Scales& b, int64_t D, hipStream_t s) {
  if (a.blocks + b.blocks == 0) return 0;
  hipLaunchKernelGGL(k_mx4_scale_tiles, dim3((unsigned)(a.blocks + b.blocks)), dim3(256), 0, s, a, b,
                     (int)(D / kMx4Block), (int)mx4_tile_steps(D));
  return (int)hipGetLastError();
}

// hidden rows of one pass; the head's scales come with the first
template <int H>
static int launch_mx4_gemm(const KdMx4Args& q, const KdMx4Plan& p, const Mx4Args& o, bool first,
                           hipStream_t s) {
  Mx4GemmArgs a{};
  a.o = o;
  a.wst = reinterpret_cast<uint8_t*>(q.ws + p.off_wst);
  a.T = (int)mx4_tile_steps(q.D);
  a.TV = (int)((q.V + 255) / 256);
  a.TT = (int)((o.N + p.tok - 1) / p.tok);
  a.per = p.per;
  a.splits = p.splits;
  a.Vp = (q.V + 3) / 4 * 4;
  a.part = p.splits > 1 ? reinterpret_cast<float*>(q.ws + p.off_part) : nullptr;
  a.hidden = static_cast<const char*>(o.hidden);
  a.hld = o.hld;
  a.hbytes = (int)(H == 2 ? q.D / 2 : q.D * 2);
  if (H == 1) {
    const int64_t Dp = (q.D + 63) / 64 * 64;
    char* t = q.ws + p.off_hidden;
    hipLaunchKernelGGL(k_mx4_terms, dim3(mx4_blocks(o.N * Dp / 8)), dim3(256), 0, s, a.hidden, o.hld,
                       o.N, (int)q.D, (int)Dp, t);
    a.hidden = t;
    a.hld = Dp * 6;
    a.hbytes = (int)(Dp * 6);
  }
  if (H == 2) a.hst = reinterpret_cast<uint8_t*>(q.ws + p.off_hidden);
  const Mx4Scales none{nullptr, 0, nullptr, 0};
  if (launch_mx4_scale_tiles(
          first ? mx4_scales(q.scales, q.V, q.D, q.ws + p.off_wst) : none,
          H == 2 ? mx4_scales(o.hscales, o.N, q.D, q.ws + p.off_hidden) : none, q.D, s) != 0)
    return 1;
  const int64_t items = (int64_t)a.TV * a.TT * p.splits;
  const dim3 grid((unsigned)(items < kMx4Units ? items : kMx4Units)), block(512);
  if constexpr (H == 2) {
    if (p.tok == 256) hipLaunchKernelGGL((k_mx4_gemm4<8>), grid, block, 0, s, a);
    else hipLaunchKernelGGL((k_mx4_gemm4<4>), grid, block, 0, s, a);
  } else {
    constexpr int TERMS = H == 1 ? 3 : 1;
    if (p.tok == 256) hipLaunchKernelGGL((k_mx4_gemm<TERMS, 8>), grid, block, 0, s, a);
    else hipLaunchKernelGGL((k_mx4_gemm<TERMS, 4>), grid, block, 0, s, a);
  }
  if (p.splits > 1) return launch_mx4_join(q, p, o.N, o.out, s);
  return (int)hipGetLastError();
}

template <int H>
static int launch_mx4_logits(const KdMx4Args& q, hipStream_t s) {
  const KdMx4Plan p = kd_mx4_plan(q.N, q.D, q.V, q.dtype, q.ld_hidden);
  Mx4Args a{};
  a.hld = H == 2 ? q.D / 2 : q.ld_hidden * (H == 1 ? 4 : 2);
  a.codes = q.codes;
  a.scales = q.scales;
  a.ldo = q.ld_out;
  a.D = (int)q.D;
  a.V = (int)q.V;
  a.out_bf16 = q.out_dtype == 1;
  for (int64_t r = 0; r < q.N; r += p.rows) {
    a.N = q.N - r < p.rows ? q.N - r : p.rows;
    a.hidden = static_cast<const char*>(q.hidden) + r * a.hld;
    if (H == 2) a.hscales = q.hscales + r * (q.D / kMx4Block);
    a.out = static_cast<char*>(q.out) + r * q.ld_out * (a.out_bf16 ? 2 : 4);
    int rc;
    if (p.kind == KD_MX4_TILES) {
      rc = launch_mx4_gemm<H>(q, p, a, r == 0, s);
    } else if (p.kind == KD_MX4_ROWS) {
      rc = p.r == 1 ? launch_mx4_rows<H, 1>(a, p.ks, s) : launch_mx4_rows<H, 2>(a, p.ks, s);
    } else if (p.nb == 1) {
      rc = p.r == 1 ? launch_mx4_wide<H, 1, 1>(q, p, a, s) : launch_mx4_wide<H, 1, 2>(q, p, a, s);
    } else if (p.nb == 2) {
      rc = p.r == 1 ? launch_mx4_wide<H, 2, 1>(q, p, a, s) : launch_mx4_wide<H, 2, 2>(q, p, a, s);
    } else if (p.r == 4) {
      rc = launch_mx4_wide<H, 4, 4>(q, p, a, s);
    } else if (p.r == 1) {
      rc = launch_mx4_wide<H, 4, 1>(q, p, a, s);
    } else {
      if constexpr (H == 2) rc = launch_mx4_wide<H, 4, 1>(q, p, a, s);
      else rc = launch_mx4_wide<H, 4, 2>(q, p, a, s);
    }
    if (rc != 0) return rc;
  }
  return 0;
}

extern "C" int kd_launch_mx4_logits(const KdMx4Args* a, void* stream) {
  hipStream_t s = static_cast<hipStream_t>(stream);
  switch (a->dtype) {
    case 0: return launch_mx4_logits<1>(*a, s);
    case 1: return launch_mx4_logits<0>(*a, s);
    default: return launch_mx4_logits<2>(*a, s);
  }
}
