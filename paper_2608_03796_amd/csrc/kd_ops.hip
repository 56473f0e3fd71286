// HIP kernels (gfx950) around the loss and their launchers:
//   top-K rows       [row_groups ->] row_select   the K largest logits of each row,
//                    as (index, value) or as entries of the teacher cache
//   teacher cache    cache_read                 entries back to (index, value)
//   checkpoints      ckpt_write, ckpt_read      hidden states in 8 bits
//   verification     seg_sums -> accept (-> rest_sums -> pick)
//                    drafted tokens against the target's probabilities
#include "kd_ckpt.h"
#include "kd_device.h"
#include "kd_ops.h"

namespace kd {

// --------------------------------------------------------------- row reads --
// A logits row is read in 16-byte vectors at 16-byte boundaries wherever the row
// starts: column v of the row has the place e = v + shift, shift = the elements
// between the boundary at or before the row and the row. Vectors that reach
// past either end of the row are read element by element; what is not of the
// row reads as -inf.
// z, or -inf where it is not a number. (The comparison has to be with z itself: of
// z > -inf the compiler makes a maximum, which is a NaN where z is a signalling one.)
__device__ __forceinline__ float number(float z) { return __builtin_isnan(z) ? -INFINITY : z; }
template <typename T>
struct Row {
  static constexpr int VPT = 16 / (int)sizeof(T);      // elements of a vector
  static constexpr int U = kSegCols / (64 * VPT);      // vectors of a lane in a segment
  static constexpr int GL = kGroupCols / VPT;          // lanes of a group
  const T* p;
  int V, shift;
  __device__ __forceinline__ Row(const void* base, int64_t offset, int V_)
      : p(static_cast<const T*>(base) + offset),
        V(V_),
        shift((int)((reinterpret_cast<uintptr_t>(p) & 15u) / sizeof(T))) {}

  // whether the vector at place e (a multiple of VPT) lies inside the row
  __device__ __forceinline__ bool inside(int e) const {
    return e >= shift && e - shift + VPT <= V;
  }
  __device__ __forceinline__ u32x4_t at(int e) const {
    return inside(e) ? *reinterpret_cast<const u32x4_t*>(p + (e - shift)) : edge(e);
  }
  __device__ __forceinline__ u32x4_t edge(int e) const {
    const int v = e - shift;
    uint32_t w[4];
    if constexpr (sizeof(T) == 2) {
      uint16_t h[8];
#pragma unroll
      for (int i = 0; i < 8; ++i)
        h[i] = (unsigned)(v + i) < (unsigned)V ? reinterpret_cast<const uint16_t*>(p)[v + i]
                                               : 0xff80;
#pragma unroll
      for (int i = 0; i < 4; ++i) w[i] = h[2 * i] | (uint32_t)h[2 * i + 1] << 16;
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        w[i] = (unsigned)(v + i) < (unsigned)V ? reinterpret_cast<const uint32_t*>(p)[v + i]
                                               : 0xff800000u;
    }
    return u32x4_t{w[0], w[1], w[2], w[3]};
  }
  // the calling wave's share of a segment: lane l holds U vectors, 64 apart
  __device__ __forceinline__ void segment(int seg, u32x4_t* x) const {
    const int lane = threadIdx.x & 63, e0 = seg * kSegCols;
    if (e0 >= shift && e0 + kSegCols - shift <= V) {
      const u32x4_t* q = reinterpret_cast<const u32x4_t*>(p + (e0 - shift)) + lane;
#pragma unroll
      for (int u = 0; u < U; ++u) x[u] = q[64 * u];
    } else {
#pragma unroll
      for (int u = 0; u < U; ++u) x[u] = at(e0 + (64 * u + lane) * VPT);
    }
  }
  // element i of a vector, as it is: maxima and med3 may return a signalling NaN or
  // drop what they had for it
  static __device__ __forceinline__ float raw(u32x4_t x, int i) {
    uint32_t b;
    if constexpr (sizeof(T) == 2) b = i & 1 ? x[i / 2] & 0xffff0000u : x[i / 2] << 16;
    else b = x[i];
    return __builtin_bit_cast(float, b);
  }
  // the same with any NaN quiet, which a maximum passes over
  static __device__ __forceinline__ float quiet(u32x4_t x, int i) {
    return __builtin_canonicalizef(raw(x, i));
  }
  // the same with any NaN as -inf
  static __device__ __forceinline__ float elt(u32x4_t x, int i) { return number(raw(x, i)); }
  __device__ __forceinline__ float one(int v) const { return number((float)p[v]); }
};

// values as unsigned numbers of the same order (-0 as +0)
__device__ __forceinline__ uint32_t order_key(float z) {
  const uint32_t b = __builtin_bit_cast(uint32_t, z + 0.f);
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float key_value(uint32_t k) {
  return __builtin_bit_cast(float, k & 0x80000000u ? k & 0x7fffffffu : ~k);
}
constexpr uint32_t kKeyNegInf = 0x007fffffu;

// 2^(log2(e) (z - m)) with m the largest of several z: 0 where z = -inf, and at
// m = +inf 1 for each z = m
__device__ __forceinline__ float exp_below(float z, float m) {
  return z == m ? 1.f : fast_exp2((z - m) * kLog2e);
}

// ------------------------------------------------------------- top-K rows ----
// Largest values of the 32 groups of the wave's segment: group i of the segment in
// lane `lane` with group_of(lane) = i, for the lanes that hold one. `top`: the lane's
// largest (of its groups).
template <typename T>
__device__ __forceinline__ float group_maxima(const u32x4_t* x, float& top) {
  constexpr int U = Row<T>::U, VPT = Row<T>::VPT, GL = Row<T>::GL;
  static_assert(U <= GL, "a lane of each group keeps each vector's maximum");
  const int lane = threadIdx.x & 63;
  float mine = -INFINITY;
  top = -INFINITY;
#pragma unroll
  for (int u = 0; u < U; ++u) {
    float m = Row<T>::elt(x[u], 0);
#pragma unroll
    for (int i = 1; i < VPT; ++i) m = fmaxf(m, Row<T>::quiet(x[u], i));
#pragma unroll
    for (int c = 0; c < (GL == 8 ? 3 : 4); ++c) m = fmaxf(m, dpp_f(m, c));
    if ((lane & (GL - 1)) == u) mine = m;
    top = fmaxf(top, m);
  }
  return mine;
}
template <typename T>
__device__ __forceinline__ int group_of(int lane) {  // -1: none
  constexpr int U = Row<T>::U, GL = Row<T>::GL;
  const int u = lane & (GL - 1);
  return u < U ? u * (64 / GL) + lane / GL : -1;
}
// sum of exp below m > -inf over the N vectors' elements of the lane
template <typename T, int N>
__device__ __forceinline__ float exp_sum(const u32x4_t* x, float m) {
  float s = 0.f;
  if (m == INFINITY) {
#pragma unroll
    for (int u = 0; u < N; ++u)
#pragma unroll
      for (int i = 0; i < Row<T>::VPT; ++i) s += Row<T>::raw(x[u], i) == m ? 1.f : 0.f;
    return s;
  }
#pragma unroll
  for (int u = 0; u < N; ++u) {
    // (a difference that is none, and what is far below, ends at 2^-200: 0 in fp32)
#pragma unroll
    for (int i = 0; i < Row<T>::VPT; ++i)
      s += fast_exp2(fmaxf((Row<T>::raw(x[u], i) - m) * kLog2e, -200.f));
    // one vector after the other: all at once the scheduler takes 100 registers
    __builtin_amdgcn_sched_barrier(0);
  }
  return s;
}

// First pass, the one that reads the logits: the largest value of each group of
// 64 columns, and with LSE the segment's maximum and sum of exp below it. A wave
// per segment, no LDS and no barrier: bound by the read (the exponentials and
// maxima take about half of the issue slots that go by at the memory's rate).
template <typename T, bool LSE>
__global__ __launch_bounds__(256) void k_row_groups(const T* __restrict__ logits, int64_t ld, int V,
                                                    int nseg, int waves, float* __restrict__ gmax,
                                                    float* __restrict__ pm,
                                                    float* __restrict__ ps) {
  const int w = blockIdx.x * 4 + wave_id();
  if (w >= waves) return;
  const int r = w / nseg, seg = w - r * nseg;
  const Row<T> row(logits, (int64_t)r * ld, V);
  u32x4_t x[Row<T>::U];
  row.segment(seg, x);
  const int lane = threadIdx.x & 63, g = group_of<T>(lane);
  float top;
  const float mine = group_maxima<T>(x, top);
  if (g >= 0) gmax[(int64_t)w * kSegGroups + g] = mine;
  if constexpr (LSE) {
    top = wave_max(top);
    const float s = wave_sum(top != -INFINITY ? exp_sum<T, Row<T>::U>(x, top) : 0.f);
    if (lane == 0) {
      pm[w] = top;
      ps[w] = s;
    }
  }
}

// Second pass, a workgroup of NT threads per row. At least K groups have a maximum
// of at least the K-th largest group maximum, so the K largest elements are among
// those that reach it, and these lie in the groups whose maximum does: about K
// groups of 64 columns are read again instead of the row. The bound is found in
// the 16 leading bits of the maxima (bf16's precision, no higher than the K-th),
// by counting them per value from the largest down: for V = 131072 and K = 100 there
// are about 105 elements that reach it. They are sorted by (value, lowest index
// first), the order of the result, so which thread collected which does not
// matter. Where more elements reach the bound than fit (many equal values), the
// K-th largest is found exactly by counting digits over the row. Columns of -inf
// never are candidates: where the row has too few others, the list is filled up
// from its first columns.
//
// kDirect (rows of up to 8 vectors a thread): the only pass. The row is held in
// registers, its groups are single vectors, and their maxima and the sum of exp
// are formed here: one launch, and groups enough for K above V / 64.
//
// kStream (rows of up to 2048 groups, with K > 512 up to 4096: their keys stand where
// the candidates will): the only pass too, the first pass's work done by the row's
// workgroup. The scattered reads of the second pass take 20 us and more
// when all rows make them at once (1 GiB of logits has left the caches by then); here
// some workgroups wait for them while others stream.
//
// The pass is latency-bound (a few dependent reads and barriers per row), so what
// counts is rows in flight, and for few rows the time of one.
constexpr int kHistBins = 2048;
constexpr int kBoundBins = 1024;
// keys of a thread in registers: all of a row held directly, or of 131072 columns
constexpr int select_keys(int NT, bool direct) { return direct || NT <= 512 ? 8 : 2; }

__host__ __device__ constexpr int select_cap(int K) {
  int c = 1024;
  while (c < 2 * K) c *= 2;
  return c;
}
// bytes of LDS: the counts of maxima, later the candidates or the digit counts; the
// list of groups
__host__ __device__ constexpr int select_lds(int G, int K) { return 8 * select_cap(K) + 2 * G; }

template <int NT>
struct SelectShared {
  int scan[NT / 64];
  int found, before;
  int n, nlist;
  float logs, sum[NT / 64], top[NT / 64];
  uint32_t whi[NT / 64];
};

// The bin of `want` (1 = the first) in the bins' order (descending or ascending),
// and the count of the bins before it; hist holds nb = 2048 or 1024 bins.
template <int NT>
__device__ __forceinline__ void find_bin(SelectShared<NT>& s, const int* hist, int nb,
                                         bool descending, int want, int& bin, int& before,
                                         int& count) {
  const int per = nb / NT, tid = threadIdx.x;
  int sum = 0;
  for (int i = 0; i < per; ++i) {
    const int b = tid * per + i;
    sum += hist[descending ? nb - 1 - b : b];
  }
  int incl = wave_incl_scan(sum);
  if ((tid & 63) == 63) s.scan[tid >> 6] = incl;
  __syncthreads();
  for (int w = 0; w < (tid >> 6); ++w) incl += s.scan[w];
  int at = incl - sum;
  if (at < want && want <= incl) {
    for (int i = 0; i < per; ++i) {
      const int b = descending ? nb - 1 - (tid * per + i) : tid * per + i;
      if (at + hist[b] >= want) {
        s.found = b;
        s.before = at;
        break;
      }
      at += hist[b];
    }
  }
  __syncthreads();
  bin = s.found;
  before = s.before;
  count = hist[bin];
  __syncthreads();
}

// lanes of the wave below this one whose bit is set
__device__ __forceinline__ int lanes_below(uint64_t b) {
  return __builtin_amdgcn_mbcnt_hi((uint32_t)(b >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)b, 0));
}

// f(in, key, v) for the VPT elements of a vector, by all lanes; `in` tells whether
// there is an element. Of the listed groups (of GL lanes), or of the whole row.
template <typename T, typename F>
__device__ __forceinline__ void vector_keys(const Row<T>& row, bool have, int e, u32x4_t x, F&& f) {
  constexpr int VPT = Row<T>::VPT;
  bool in[VPT];
  uint32_t k[VPT];
#pragma unroll
  for (int i = 0; i < VPT; ++i) {
    in[i] = have && (unsigned)(e + i - row.shift) < (unsigned)row.V;
    k[i] = order_key(Row<T>::elt(x, i));
  }
  f(in, k, e - row.shift);
}
template <typename T, int NT, int GL, typename F>
__device__ __forceinline__ void listed_vectors(const Row<T>& row, const uint16_t* list, int n,
                                               F&& f) {
  constexpr int VPT = Row<T>::VPT, GPW = 64 / GL;
  const int lane = threadIdx.x & 63, wave = wave_id();
  for (int l0 = wave * GPW; l0 < n; l0 += NT / 64 * GPW) {
    const int l = l0 + lane / GL;
    const int e = l < n ? ((int)list[l] * GL + (lane & (GL - 1))) * VPT : 0;
    vector_keys<T>(row, l < n, e, row.at(e), f);
  }
}
template <typename T, int NT, typename F>
__device__ __forceinline__ void row_vectors(const Row<T>& row, F&& f) {
  constexpr int VPT = Row<T>::VPT, R = 2;  // vectors read together
  const int end = row.shift + row.V;
  for (int e0 = threadIdx.x * VPT; e0 - (int)(threadIdx.x & 63) * VPT < end; e0 += R * NT * VPT) {
    u32x4_t x[R];
#pragma unroll
    for (int j = 0; j < R; ++j) x[j] = row.at(e0 + j * NT * VPT);
#pragma unroll
    for (int j = 0; j < R; ++j) vector_keys<T>(row, true, e0 + j * NT * VPT, x[j], f);
  }
}
// counts the lanes' bins: the first one's with one addition (most elements may be
// equal), the others' by themselves
__device__ __forceinline__ void count_bins(int* hist, bool in, int bin) {
  const uint64_t act = __builtin_amdgcn_ballot_w64(in);
  if (act == 0) return;
  const int lead = __builtin_ctzll(act), first = __builtin_amdgcn_readlane(bin, lead);
  const uint64_t same = __builtin_amdgcn_ballot_w64(in && bin == first);
  if ((int)(threadIdx.x & 63) == lead) atomicAdd(&hist[first], __popcll(same));
  if (in && bin != first) atomicAdd(&hist[bin], 1);
}

struct SelectArgs {
  const void* logits;
  int64_t ld;
  int V, K, G, nseg, logprobs;
  const float *gmax, *pm, *ps;
  int32_t* idx;
  float* value;
  uint32_t* entries;
  float* scale;
};

enum SelectMode { kFromMaxima, kDirect, kStream };
template <typename T, int NT, SelectMode MODE>
__global__ __launch_bounds__(NT) void k_row_select(SelectArgs a) {
  constexpr bool DIRECT = MODE == kDirect, STREAM = MODE == kStream;
  extern __shared__ __align__(16) char lds[];
  __shared__ SelectShared<NT> s;
  constexpr int VPT = Row<T>::VPT, GL = DIRECT ? 1 : Row<T>::GL;
  constexpr int kUnroll = select_keys(NT, DIRECT);
  const int tid = threadIdx.x, lane = tid & 63, wave = wave_id();
  const int K = a.K, G = a.G, cap = select_cap(K);
  const int64_t r = blockIdx.x;
  const Row<T> row(a.logits, r * a.ld, a.V);
  uint64_t* cand = reinterpret_cast<uint64_t*>(lds);
  int* hist = reinterpret_cast<int*>(lds);
  uint16_t* list = reinterpret_cast<uint16_t*>(lds + 8 * cap);

  // The group maxima as keys, some a thread: kept in registers where that holds all
  // of them, else read again. f(keys, first
  // group) takes keys of groups first, first + NT, ...; 0 where there is none
  const float* gm = MODE == kFromMaxima ? a.gmax + r * G : nullptr;
  uint32_t held[kUnroll];
  u32x4_t x[DIRECT ? kUnroll : 1];
  auto read_keys = [&](int i0, uint32_t* k) {
    float g[kUnroll];
#pragma unroll
    for (int j = 0; j < kUnroll; ++j) g[j] = i0 + j * NT < G ? gm[i0 + j * NT] : 0.f;
#pragma unroll
    for (int j = 0; j < kUnroll; ++j) k[j] = i0 + j * NT < G ? order_key(g[j]) : 0u;
  };
  const bool hold = MODE != kFromMaxima || G <= kUnroll * NT;
  if constexpr (DIRECT) {
#pragma unroll
    for (int j = 0; j < kUnroll; ++j) x[j] = row.at((tid + j * NT) * VPT);
#pragma unroll
    for (int j = 0; j < kUnroll; ++j) {
      float m = Row<T>::elt(x[j], 0);
#pragma unroll
      for (int i = 1; i < VPT; ++i) m = fmaxf(m, Row<T>::quiet(x[j], i));
      held[j] = tid + j * NT < G ? order_key(m) : 0u;
    }
  } else if constexpr (STREAM) {
    uint32_t* keys = reinterpret_cast<uint32_t*>(lds);
    const int g = group_of<T>(lane);
    u32x4_t y[Row<T>::U];
    float m = -INFINITY, t = 0.f;  // the wave's largest, the lane's sum of exp below it
    if (wave < a.nseg) row.segment(wave, y);
    for (int seg = wave; seg < a.nseg; seg += NT / 64) {
      u32x4_t next[Row<T>::U];
      if (seg + NT / 64 < a.nseg) row.segment(seg + NT / 64, next);
      float top;
      const float mine = group_maxima<T>(y, top);
      if (g >= 0) keys[seg * kSegGroups + g] = order_key(mine);
      if (a.logprobs) {
        top = fmaxf(wave_max(top), m);
        if (top != -INFINITY) t = t * exp_below(m, top) + exp_sum<T, Row<T>::U>(y, top);
        m = top;
      }
#pragma unroll
      for (int u = 0; u < Row<T>::U; ++u) y[u] = next[u];
    }
    if (a.logprobs) {
      t = wave_sum(t);
      if (lane == 0) {
        s.sum[wave] = t;
        s.top[wave] = m;
      }
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < kUnroll; ++j) held[j] = tid + j * NT < G ? keys[tid + j * NT] : 0u;
    __syncthreads();
  } else if (hold) {
    read_keys(tid, held);
  }
  auto all_keys = [&](auto&& f) {
    if (hold) {
      f(held, tid);
    } else {
      for (int i0 = tid; i0 - lane < G; i0 += kUnroll * NT) {
        uint32_t k[kUnroll];
        read_keys(i0, k);
        f(k, i0);
      }
    }
  };
  // the largest of them, and log of the row's sum of exp
  uint32_t hi = 0;
  all_keys([&](const uint32_t* k, int) {
#pragma unroll
    for (int j = 0; j < kUnroll; ++j) hi = max(hi, k[j]);
  });
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) hi = max(hi, (uint32_t)__shfl_xor((int)hi, o));
  if (lane == 0) s.whi[wave] = hi;
  if (tid == 0) s.n = s.nlist = 0;
  for (int i = tid; i < kBoundBins; i += NT) hist[i] = 0;
  if (MODE == kFromMaxima && a.logprobs && wave == NT / 64 - 1) {
    const float *pm = a.pm + r * a.nseg, *ps = a.ps + r * a.nseg;
    float m = -INFINITY, t = 0.f;
    for (int i = lane; i < a.nseg; i += 64) m = fmaxf(m, pm[i]);
    m = wave_max(m);
    if (m != -INFINITY)
      for (int i = lane; i < a.nseg; i += 64) t += ps[i] * exp_below(pm[i], m);
    t = wave_sum(t);
    if (lane == 0) s.logs = m != -INFINITY ? logf(t) : 0.f;
  }
  __syncthreads();
  hi = s.whi[lane % (NT / 64)];
#pragma unroll
  for (int o = NT / 128; o >= 1; o >>= 1) hi = max(hi, (uint32_t)__shfl_xor((int)hi, o));
  hi = (uint32_t)__builtin_amdgcn_readfirstlane((int)hi);
  if constexpr (DIRECT) {
    if (a.logprobs) {
      const float m = key_value(hi);
      float t = 0.f;
      if (m != -INFINITY) t = exp_sum<T, kUnroll>(x, m);
      t = wave_sum(t);
      if (lane == 0) s.sum[wave] = t;
    }
  }
  hi >>= 16;
  // the largest 16-bit prefix that K maxima reach: by counts where it lies within
  // 1022 of the largest (eight factors of two), else by halving; 0 where K groups
  // do not exist
  uint32_t t = 0;
  if (K <= G) {
    all_keys([&](const uint32_t* k, int) {
#pragma unroll
      for (int j = 0; j < kUnroll; ++j)
        if (k[j] != 0) atomicAdd(&hist[min(hi - (k[j] >> 16), (uint32_t)kBoundBins - 1)], 1);
    });
    __syncthreads();
    int bin, before, count;
    find_bin<NT>(s, hist, kBoundBins, false, K, bin, before, count);
    if (bin < kBoundBins - 1) {
      t = hi - bin;
    } else {
      uint32_t top = hi - (kBoundBins - 2);  // reached by fewer than K; 0 by all
      while (top - t > 1) {
        const uint32_t mid = (t + top) / 2;
        int c = 0;
        all_keys([&](const uint32_t* k, int) {
#pragma unroll
          for (int j = 0; j < kUnroll; ++j) c += k[j] >> 16 >= mid;
        });
#pragma unroll
        for (int o = 32; o >= 1; o >>= 1) c += __shfl_xor(c, o);
        if (lane == 0) s.scan[wave] = c;
        __syncthreads();
        c = 0;
        for (int w = 0; w < NT / 64; ++w) c += s.scan[w];
        if (c >= K) t = mid;
        else top = mid;
        __syncthreads();
      }
    }
    t <<= 16;
  }
  t = max(t, kKeyNegInf + 1);
  // the groups that reach it (a key is never 0), one reservation per wave
  all_keys([&](const uint32_t* k, int i0) {
    uint64_t b[kUnroll];
    int total = 0;
#pragma unroll
    for (int j = 0; j < kUnroll; ++j) {
      b[j] = __builtin_amdgcn_ballot_w64(k[j] != 0 && k[j] >= t);
      total += __popcll(b[j]);
    }
    int at = 0;
    if (lane == 0 && total > 0) at = atomicAdd(&s.nlist, total);
    at = __builtin_amdgcn_readfirstlane(at);
#pragma unroll
    for (int j = 0; j < kUnroll; ++j) {
      if (b[j] >> lane & 1) list[at + lanes_below(b[j])] = (uint16_t)(i0 + j * NT);
      at += __popcll(b[j]);
    }
  });
  __syncthreads();
  const int nlist = s.nlist;

  // elements with key > kth, or = kth and an index up to vcut, as candidates
  auto collect = [&](uint32_t kth, int vcut) {
    return [=](const bool* in, const uint32_t* k, int v) {
      uint64_t b[VPT];
      int total = 0;
#pragma unroll
      for (int i = 0; i < VPT; ++i) {
        b[i] = __builtin_amdgcn_ballot_w64(in[i] && (k[i] > kth || (k[i] == kth && v + i <= vcut)));
        total += __popcll(b[i]);
      }
      if (total == 0) return;
      int to = 0;
      if (lane == 0) to = atomicAdd(&s.n, total);
      to = __builtin_amdgcn_readfirstlane(to);
#pragma unroll
      for (int i = 0; i < VPT; ++i) {
        const int o = to + lanes_below(b[i]);
        if ((b[i] >> lane & 1) != 0 && o < cap)
          cand[o] = (uint64_t)k[i] << 32 | (0xffffffffu - (uint32_t)(v + i));
        to += __popcll(b[i]);
      }
    };
  };
  listed_vectors<T, NT, GL>(row, list, nlist, collect(t - 1, -1));
  __syncthreads();
  int n = s.n;
  __syncthreads();  // (before any wave adds to it again)
  if (n > cap) {
    // the K-th largest exactly: its key in digits of 11 and 5 bits, in fp32 11, 11 and
    // 10 (keys of bf16 have 16 bits of their own)
    uint32_t kth = 0;
    int want = K, ties = 0;
    constexpr int kDigits = sizeof(T) == 2 ? 2 : 3;
    constexpr int kShift[3] = {21, sizeof(T) == 2 ? 16 : 10, 0};
    constexpr uint32_t kMask[3] = {0u, 0xffe00000u, 0xfffffc00u};
#pragma unroll
    for (int d = 0; d < kDigits; ++d) {
      const int nb = d == 2 ? 1024 : kHistBins, sh = kShift[d];
      for (int i = tid; i < nb; i += NT) hist[i] = 0;
      __syncthreads();
      row_vectors<T, NT>(row, [&](const bool* in, const uint32_t* k, int) {
#pragma unroll
        for (int i = 0; i < VPT; ++i)
          count_bins(hist, in[i] && (k[i] & kMask[d]) == kth,
                     (int)(k[i] >> sh & (sizeof(T) == 2 && d == 1 ? 31 : nb - 1)));
      });
      __syncthreads();
      int bin, before;
      find_bin<NT>(s, hist, nb, true, want, bin, before, ties);
      kth |= (uint32_t)bin << sh;
      want -= before;
    }
    if (sizeof(T) == 2 && !(kth & 0x80000000u)) kth |= 0xffffu;
    // of more elements with that key than are wanted, those of the lowest indices:
    // columns in their order until there are enough
    int vcut = 0x7fffffff;
    if (ties > want) {
      int seen = 0;
      for (int e0 = 0; e0 < row.shift + row.V; e0 += NT * VPT) {
        const int e = e0 + tid * VPT;
        int mine = 0;
        uint32_t hits = 0;
        vector_keys<T>(row, true, e, row.at(e), [&](const bool* in, const uint32_t* k, int) {
#pragma unroll
          for (int i = 0; i < VPT; ++i)
            if (in[i] && k[i] == kth) {
              ++mine;
              hits |= 1u << i;
            }
        });
        int incl = wave_incl_scan(mine);
        if (lane == 63) s.scan[wave] = incl;
        __syncthreads();
        int total = 0;
        for (int w = 0; w < NT / 64; ++w) {
          if (w < wave) incl += s.scan[w];
          total += s.scan[w];
        }
        const int need = want - seen - (incl - mine);  // of this thread's, the last wanted
        if (need >= 1 && need <= mine) {
          for (int i = 1; i < need; ++i) hits &= hits - 1;
          s.found = e - row.shift + __builtin_ctz(hits);
        }
        seen += total;
        __syncthreads();
        if (seen >= want) break;
      }
      vcut = s.found;
    }
    if (tid == 0) s.n = 0;
    __syncthreads();
    row_vectors<T, NT>(row, collect(kth, vcut));
    __syncthreads();
    n = s.n;
  } else if (n < K) {
    // fewer than K above -inf: of the first K columns as many as it takes are -inf
    for (int v0 = 0; v0 < K; v0 += NT) {
      const int v = v0 + tid;
      const bool q = v < K && row.one(v) == -INFINITY;
      const uint64_t b = __builtin_amdgcn_ballot_w64(q);
      int to = 0;
      if (lane == 0 && b != 0) to = atomicAdd(&s.n, __popcll(b));
      to = __builtin_amdgcn_readfirstlane(to) + lanes_below(b);
      if (q) cand[to] = (uint64_t)kKeyNegInf << 32 | (0xffffffffu - (uint32_t)v);
    }
    __syncthreads();
    n = s.n;
  }
  // sorted, largest first: each candidate's rank among all of them, by as many
  // lanes as there are for it; or, when there are more than threads, bitonic
  if (n <= NT) {
    int per = NT, each = 1;  // places of candidates, lanes of each
    while (per / 2 >= n && each < 64) per /= 2, each *= 2;
    const int j = tid / each, sub = tid & (each - 1);
    const uint64_t c = j < n ? cand[j] : 0;
    int rank = 0;
#pragma unroll 8
    for (int i = sub; i < n; i += each) rank += cand[i] > c;
    for (int o = each / 2; o >= 1; o >>= 1) rank += __shfl_xor(rank, o);
    __syncthreads();
    if (j < n && sub == 0) cand[rank] = c;
  } else {
    int P = 2 * NT;
    while (P < n) P *= 2;
    for (int i = n + tid; i < P; i += NT) cand[i] = 0;
    for (int size = 2; size <= P; size *= 2)
      for (int st = size / 2; st > 0; st /= 2) {
        __syncthreads();
        for (int i = tid; i < P / 2; i += NT) {
          const int x = 2 * i - (i & (st - 1)), y = x + st;
          const uint64_t p = cand[x], q = cand[y];
          if ((p < q) == ((x & size) == 0)) {
            cand[x] = q;
            cand[y] = p;
          }
        }
      }
  }
  __syncthreads();

  const float z0 = key_value((uint32_t)(cand[0] >> 32));
  float logs = 0.f;
  if (a.logprobs && MODE != kFromMaxima) {
    for (int w = 0; w < NT / 64; ++w)
      logs += STREAM ? s.sum[w] * exp_below(s.top[w], z0) : s.sum[w];
    logs = z0 == -INFINITY ? 0.f : logf(logs);
  } else if (a.logprobs) {
    logs = s.logs;
  }
  if (a.value != nullptr) {
    for (int k = tid; k < K; k += NT) {
      const uint64_t c = cand[k];
      const float z = key_value((uint32_t)(c >> 32));
      const int64_t o = r * K + k;
      a.idx[o] = (int32_t)(0xffffffffu - (uint32_t)c);
      a.value[o] = !a.logprobs ? z : z == -INFINITY ? z : (z == z0 ? 0.f : z - z0) - logs;
    }
    return;
  }
  // cache entries: the kept ones come first; the steps between the first and the
  // last of them are computed in 64 bits (infinities as the largest finite value)
  const bool empty = z0 == -INFINITY;
  const float top = fminf(z0, 3.402823466e38f);
  if (wave == 0) {
    int kept = 0;
    for (int k0 = 0; k0 < K; k0 += 64) {
      const int k = k0 + lane;
      const float z = fminf(key_value((uint32_t)(cand[k < K ? k : 0] >> 32)), 3.402823466e38f);
      // (in fp32 top - 1024 is rounded to 2^-14, or 2^-13, and entries there misjudged)
      const bool near = (double)z >= (double)top - kCacheReach;
      kept += __popcll(__builtin_amdgcn_ballot_w64(!empty && k < K && near));
    }
    if (lane == 0) s.n = kept;
  }
  __syncthreads();
  const int kept = s.n;
  const double dtop = top;
  float step = 0.f;
  if (kept > 0) {
    const float low = fminf(key_value((uint32_t)(cand[kept - 1] >> 32)), 3.402823466e38f);
    step = (float)((dtop - (double)low) / kCacheCodeMax);
  }
  for (int k = tid; k < K; k += NT) {
    const uint64_t c = cand[k];
    const uint32_t v = 0xffffffffu - (uint32_t)c;
    uint32_t code = kCacheNone;
    if (k < kept) {
      const float z = fminf(key_value((uint32_t)(c >> 32)), 3.402823466e38f);
      const double q = step > 0.f ? __builtin_rint((dtop - (double)z) / (double)step) : 0.0;
      code = q < (double)kCacheCodeMax ? (uint32_t)q : (uint32_t)kCacheCodeMax;
    }
    a.entries[r * K + k] = v << kCacheCodeBits | code;
  }
  if (tid == 0) {
    a.scale[2 * r] = empty ? -INFINITY : a.logprobs ? -logs : top;
    a.scale[2 * r + 1] = step;
  }
}

// Results larger than the caches (BIG) are stored past them, and such hidden states
// read past them, so that what is read again stays: 262144 cache rows of 100 entries
// 75.6 and 58.4 us, checkpoints of 32768 x 4096 bf16 written and read 149 and 124 us.
// Small ones are wanted there by the next kernel and are not: 8192 x 4096 (64 MiB) 34
// and 37 us. Between 64 and 128 MiB the two cross.
constexpr int64_t kBigBytes = (int64_t)96 << 20;
template <bool BIG, typename V>
__device__ __forceinline__ void store_out(V v, V* p) {
  if constexpr (BIG) __builtin_nontemporal_store(v, p);
  else *p = v;
}
template <bool BIG, typename V>
__device__ __forceinline__ V load_in(const V* p) {
  if constexpr (BIG) return __builtin_nontemporal_load(p);
  else return *p;
}

// ------------------------------------------------------------ teacher cache --
// Entries back to (index, value): value = top - code * step, rounded once (the
// product is exact in the fused operation). V4: four entries a thread. BIG: see
// store_out.
template <bool V4, bool BIG>
__global__ __launch_bounds__(256) void k_cache_read(const uint32_t* __restrict__ entries,
                                                    const float* __restrict__ scale,
                                                    const int64_t* __restrict__ rows, int64_t N,
                                                    int64_t M, int K, int rows_per_block,
                                                    int32_t* __restrict__ idx,
                                                    float* __restrict__ value,
                                                    uint8_t* __restrict__ ignore) {
  constexpr int VPT = V4 ? 4 : 1;
  const int per = K / VPT;
  const int64_t stride = (int64_t)gridDim.x * rows_per_block;
  for (int64_t m0 = (int64_t)blockIdx.x * rows_per_block; m0 < M; m0 += stride) {
    const int nrow = (int)(M - m0 < rows_per_block ? M - m0 : rows_per_block);
    for (int i = threadIdx.x; i < nrow * per; i += 256) {
      const int j = i / per, q = i - j * per;
      const int64_t m = m0 + j, src = rows != nullptr ? rows[m] : m;
      const bool have = src >= 0 && src < N;
      float top = -INFINITY, step = 0.f;
      uint32_t e[VPT];
#pragma unroll
      for (int x = 0; x < VPT; ++x) e[x] = kCacheNone;
      if (have) {
        top = scale[2 * src];
        step = scale[2 * src + 1];
        const uint32_t* p = entries + src * K + q * VPT;
        if constexpr (V4) {
          const u32x4_t w = *reinterpret_cast<const u32x4_t*>(p);
#pragma unroll
          for (int x = 0; x < 4; ++x) e[x] = w[x];
        } else {
          e[0] = *p;
        }
      }
      const bool empty = top == -INFINITY;
      int32_t iv[VPT];
      float zv[VPT];
#pragma unroll
      for (int x = 0; x < VPT; ++x) {
        const int code = (int)(e[x] & ((1u << kCacheCodeBits) - 1));
        iv[x] = empty ? -1 : (int32_t)(e[x] >> kCacheCodeBits);
        zv[x] = empty ? 0.f : code == kCacheNone ? -INFINITY : fmaf(-(float)code, step, top);
      }
      const int64_t o = m * K + q * VPT;
      if constexpr (V4) {
        typedef __attribute__((__vector_size__(16))) int32_t s32x4_t;
        store_out<BIG>(s32x4_t{iv[0], iv[1], iv[2], iv[3]}, reinterpret_cast<s32x4_t*>(idx + o));
        store_out<BIG>(f32x4_t{zv[0], zv[1], zv[2], zv[3]}, reinterpret_cast<f32x4_t*>(value + o));
      } else {
        idx[o] = iv[0];
        value[o] = zv[0];
      }
      if (q == 0 && ignore != nullptr) ignore[m] = empty ? 1 : 0;
    }
  }
}

// -------------------------------------------------------------- checkpoints --
// Eight elements a thread, four threads a block of 32 (kd_ckpt.h).
template <typename T, bool BIG>
__global__ __launch_bounds__(256) void k_ckpt_write(const T* __restrict__ h, int64_t n8,
                                                    uint8_t* __restrict__ codes,
                                                    uint8_t* __restrict__ scales) {
  const int64_t stride = (int64_t)gridDim.x * 256;
  // (n8 is a multiple of 4: the four threads of a block run or stop together)
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n8; i += stride) {
    float v[8];
    if constexpr (sizeof(T) == 2) {
      const u32x4_t x = load_in<BIG>(reinterpret_cast<const u32x4_t*>(h) + i);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        v[2 * j] = __builtin_bit_cast(float, x[j] << 16);
        v[2 * j + 1] = __builtin_bit_cast(float, x[j] & 0xffff0000u);
      }
    } else {
      const f32x4_t x = load_in<BIG>(reinterpret_cast<const f32x4_t*>(h) + 2 * i);
      const f32x4_t y = load_in<BIG>(reinterpret_cast<const f32x4_t*>(h) + 2 * i + 1);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        v[j] = x[j];
        v[4 + j] = y[j];
      }
    }
    // magnitudes as bit patterns: their order has infinities and what is not a
    // number at the end, so neither is lost in the maximum
    uint32_t m = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) m = max(m, __builtin_bit_cast(uint32_t, v[j]) & 0x7fffffffu);
    m = max(m, (uint32_t)__builtin_amdgcn_mov_dpp((int)m, 0xB1, 0xF, 0xF, false));
    m = max(m, (uint32_t)__builtin_amdgcn_mov_dpp((int)m, 0x4E, 0xF, 0xF, false));
    const int s = ckpt_scale(m);
    reinterpret_cast<u32x2_t*>(codes)[i] =
        u32x2_t{ckpt_pack4(v[0], v[1], v[2], v[3], s), ckpt_pack4(v[4], v[5], v[6], v[7], s)};
    if ((threadIdx.x & 3) == 0) scales[i / 4] = (uint8_t)s;
  }
}

template <typename T, bool BIG>
__global__ __launch_bounds__(256) void k_ckpt_read(const uint8_t* __restrict__ codes,
                                                   const uint8_t* __restrict__ scales, int64_t n16,
                                                   T* __restrict__ h) {
  constexpr int VPT = 16 / (int)sizeof(T);
  const int64_t stride = (int64_t)gridDim.x * 256;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n16; i += stride)
    store_out<BIG>(ckpt_load16<T>(codes + i * VPT, scales + i * VPT / kCkptBlock, 0, 0, 0),
                   reinterpret_cast<u32x4_t*>(h) + i);
}

// ------------------------------------------------------------- verification --
// A drafted token d at place t is kept while u_t q(d) < p(d), p the target's and
// q the draft's softmax; the token behind the r kept ones is drawn by the last
// uniform number u from x = max(p - q, 0) at place r, or from p behind the last
// drafted one: the first v whose cumulative x exceeds u times the sum of x. A
// step of that sum is as small as a token's probability, and 2^17 of them stand
// side by side, so weights, sums and comparisons are in 64 bits (fp64 runs at
// the rate of unpacked fp32 here).

// s 2^y: 2^n times the exponential series of ln(2) f, |f| <= 1/2 (to degree 13: the next
// term is below 2^-57 of the result). s is 2^-1000 to 2^910, and what is below 2^-1074 is 0
// in the result only
__device__ __forceinline__ double exp2_64(double y, double s = 1.0) {
  y = fmax(y, -2200.0);
  const double n = __builtin_rint(y), g = (y - n) * 0.69314718055994530942;
  double p = 1.0 / 6227020800;
  p = fma(p, g, 1.0 / 479001600);
  p = fma(p, g, 1.0 / 39916800);
  p = fma(p, g, 1.0 / 3628800);
  p = fma(p, g, 1.0 / 362880);
  p = fma(p, g, 1.0 / 40320);
  p = fma(p, g, 1.0 / 5040);
  p = fma(p, g, 1.0 / 720);
  p = fma(p, g, 1.0 / 120);
  p = fma(p, g, 1.0 / 24);
  p = fma(p, g, 1.0 / 6);
  p = fma(p, g, 0.5);
  p = fma(p, g, 1.0);
  p = fma(p, g, 1.0);
  return __builtin_amdgcn_ldexp(p * s, (int)n);
}
// weight of z relative to m: 2^(c (z - m)); with m = +inf, 1 for z = m; 0 where
// m = -inf (nothing is left)
__device__ __forceinline__ double weight(float z, float m, double c) {
  if (z == m) return m == -INFINITY ? 0.0 : 1.0;
  return exp2_64(((double)z - (double)m) * c);
}
// a sum s of weights relative to z as one of weights relative to m. (The weight of z may be
// too small for 64 bits where the sum is not: a segment's reference may be 2^890 below its
// largest logit.)
__device__ __forceinline__ double mass(double s, float z, float m, double c) {
  if (z == m) return m == -INFINITY ? 0.0 : s;
  return s > 0.0 ? exp2_64(((double)z - (double)m) * c, s) : 0.0;
}
// Weights relative to one m, for passes over whole rows: 2^(y / 256) with y = 256 c
// (z - m) by a table of 2^(i / 256) in LDS and, for the rest of a step, the cubic that
// is 2^(x / 256) at x = 0, 1/4, 3/4 and 1 (off by at most 2^-44 of it between). y is held
// 2^18 higher, so that it is positive and its whole part and rest are an operation
// each: 8 fp64 operations and 6 others where exp2_64 with its difference, comparisons
// and sum takes 25 and 4 (segment sums of 256 x 6 rows 134 and 72 us). The rounding of y
// at 2^18 is 2^-43 of the weight; that of 256 c m, which is all weights' and grows with it,
// is kept as a factor for their sum (`fix`: without it 3e-9 at m / tau = 3e7). z is held above
// m - 990 / c, where weights no longer count (2^-990; -inf and a quiet NaN end there
// too), and below m + 900 / c. fp32 can tell these from m where `fast`: its rounding of
// them, at most 2^-24 (|m| + 990 / c) with |m| below 65536 * 990 / c, moves their weights
// by up to 2^3.9, so one that is held back stays above kHeld. Elsewhere (infinities,
// extreme tau) weight() serves.
constexpr int kTabBits = 8, kTab = 1 << kTabBits;
// 2^(i / 256) less i << 12 in its high word, and less 2^18 << 12: adding n << 12 for
// n = 2^18 + i + 256 j gives 2^(j + i / 256)
constexpr int kTabLift = 1 << 18;
constexpr double kHeld = 0x1p890;
struct Roots {
  uint64_t v[kTab];
  constexpr Roots() : v() {
    for (int i = 0; i < kTab; ++i) {
      const double x = i * (0.69314718055994530942 / kTab);
      double s = 1.0;
      for (int k = 24; k >= 1; --k) s = 1.0 + s * x / k;
      v[i] = __builtin_bit_cast(uint64_t, s) - ((uint64_t)(kTabLift + i) << (52 - kTabBits));
    }
  }
};
__device__ constexpr Roots kRoots{};
__device__ __forceinline__ void load_roots(uint64_t* tab) {
  for (int i = threadIdx.x; i < kTab; i += blockDim.x) tab[i] = kRoots.v[i];
  __syncthreads();
}
struct Weights {
  double c, cs, ms, fix;
  float m, floor, ceil;
  bool fast;
  const uint64_t* tab;
  __device__ __forceinline__ Weights(float m_, double c_, const uint64_t* t)
      : c(c_), m(m_), tab(t) {
    const double reach = 990.0 / c, big = fabs((double)m);
    fast = reach > big * (1.0 / 65536) && reach < 1e37 && big < 1e37;
    floor = (float)((double)m - reach);
    ceil = (float)((double)m + reach * (900.0 / 990.0));
    cs = (double)kTab * c;
    {
#pragma clang fp contract(off)
      // m cs = p + e exactly, and 2^18 - p = ms + d exactly
      const double p = (double)m * cs, e = __builtin_fma((double)m, cs, -p);
      ms = kTabLift - p;
      const double r = ms - kTabLift, d = (kTabLift - (ms - r)) - (p + r);
      fix = 1.0 + (d - e) * (0.69314718055994530942 / kTab);
    }
  }
  // the weight of z over `fix`
  __device__ __forceinline__ double quick(float z) const {
    const double y = fma((double)__builtin_amdgcn_fmed3f(z, floor, ceil), cs, ms);
    const double g = __builtin_amdgcn_fract(y);
    const uint32_t n = (uint32_t)(int)y;
    double p = fma(g, 3.31278488346773615534e-9, 3.66556293497395606907e-6);
    p = fma(p, g, 2.70760617448262800694e-3);
    p = fma(p, g, 1.0);
    const uint64_t e = tab[n & (kTab - 1)];
    const uint32_t high = (uint32_t)(e >> 32) + (n << (20 - kTabBits));
    return p * __builtin_bit_cast(double, (uint64_t)high << 32 | (uint32_t)e);
  }
  __device__ __forceinline__ double exact(float z) const { return weight(z, m, c); }
};

__device__ __forceinline__ double wave_sum64(double x) {
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) x += __shfl_xor(x, o);
  return x;
}
__device__ __forceinline__ double wave_incl_scan64(double x) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const double y = __shfl_up(x, o);
    if (lane >= o) x += y;
  }
  return x;
}

struct VerifyArgs {
  const void *target, *draft;
  int64_t ld_t, ld_d;
  int B, T, V, K, nseg;
  const int32_t *tokens, *didx;
  const float *dlogit, *uniform;
  const int32_t* lengths;
  double c;
  int32_t *out_tokens, *accepted;
  float* prob;
  float* segm;
  double *segs, *segr, *norm;
};
__device__ __forceinline__ int drafted(const VerifyArgs& a, int b) {
  if (a.lengths == nullptr) return a.T;
  const int n = a.lengths[b];
  return n < 0 ? 0 : n > a.T ? a.T : n;
}
__device__ __forceinline__ int64_t target_row(const VerifyArgs& a, int b, int t) {
  return (int64_t)b * (a.T + 1) + t;
}
__device__ __forceinline__ int64_t draft_row(const VerifyArgs& a, int b, int t) {
  return (int64_t)b * a.T + t;
}

// Reference m and sum of 2^(c (z - m)) of each segment of the rows in question (the
// target's, then the draft's): the pass that reads the logits, bound by its fp64
// arithmetic (8 of about 16 operations an element): 256 sequences of up to 6 rows of
// 131072 in bf16, 0.24 GB read, 73 us; the same read without the weights 44. 64 bits
// hold the weights of logits well above the reference too, so the largest of a
// quarter (bf16) or an eighth of the segment serves, the largest of all where that is
// -inf; a segment whose sum reaches kHeld, as it does where a logit was held back, is
// summed again below its largest logit.
template <typename T>
__global__ __launch_bounds__(256) void k_seg_sums(VerifyArgs a, int waves) {
  __shared__ uint64_t tab[kTab];
  load_roots(tab);
  const int w = blockIdx.x * 4 + wave_id();
  if (w >= waves) return;
  const int r = w / a.nseg, seg = w - r * a.nseg;
  const int nt = a.B * (a.T + 1);
  const bool tgt = r < nt;
  const int b = tgt ? r / (a.T + 1) : (r - nt) / a.T;
  const int t = tgt ? r - b * (a.T + 1) : r - nt - b * a.T;
  const int n = drafted(a, b);
  if (tgt ? t > n : t >= n) return;  // no one asks for this row
  const Row<T> row(tgt ? a.target : a.draft, tgt ? r * a.ld_t : (int64_t)(r - nt) * a.ld_d, a.V);
  constexpr int U = Row<T>::U, VPT = Row<T>::VPT;
  u32x4_t x[U];
  row.segment(seg, x);
  auto largest = [&](int vectors) {
    float m = -INFINITY;
#pragma unroll
    for (int u = 0; u < vectors; ++u)
#pragma unroll
      for (int i = 0; i < VPT; ++i) m = fmaxf(m, Row<T>::quiet(x[u], i));
    return wave_max(m);
  };
  float m = largest(1);
  if (m == -INFINITY) m = largest(U);
  double s = 0.0;
  if (m != -INFINITY) {
    const Weights q(m, a.c, tab);
    if (q.fast) {
      double h = 0.0;
#pragma unroll
      for (int u = 0; u < U; ++u) {
#pragma unroll
        for (int i = 0; i < VPT; i += 2) {
          s += q.quick(Row<T>::raw(x[u], i));
          h += q.quick(Row<T>::raw(x[u], i + 1));
        }
      }
      s = wave_sum64(s + h) * q.fix;
    }
    // (a signalling NaN that med3 let through makes the sum none either)
    if (!q.fast || !(s < kHeld)) {
      m = largest(U);
      s = 0.0;
#pragma unroll
      for (int u = 0; u < U; ++u)
        for (int i = 0; i < VPT; ++i) s += weight(Row<T>::elt(x[u], i), m, a.c);
      s = wave_sum64(s);
    }
  }
  if ((threadIdx.x & 63) == 0) {
    a.segm[w] = m;
    a.segs[w] = s;
  }
}

constexpr int kVerThreads = 512;
constexpr int kVerWaves = kVerThreads / 64;
constexpr int kVerMaxSegs = 513;   // of 2^20 columns
struct VerifyShared {
  double seg[kVerMaxSegs];         // mass of each segment
  double x[kSegCols];              // the segment the token is drawn from
  double scan[kVerWaves];
  double goal;                     // what the running sum has to pass in it
  int first, at;
};

// (M, S) of a row from its segments, by the calling wave
__device__ __forceinline__ void merge_row(const VerifyArgs& a, int64_t r, float& M, double& S) {
  const float* pm = a.segm + r * a.nseg;
  const double* ps = a.segs + r * a.nseg;
  const int lane = threadIdx.x & 63;
  float m = -INFINITY;
  for (int i = lane; i < a.nseg; i += 64) m = fmaxf(m, pm[i]);
  M = wave_max(m);
  double s = 0.0;
  if (M != -INFINITY)
    for (int i = lane; i < a.nseg; i += 64) s += mass(ps[i], pm[i], M, a.c);
  S = wave_sum64(s);
}

// The segment, and in it the place, that the goal falls in: sh.seg holds the
// mass of each segment. fill(seg) writes the mass of each of its places to sh.x
// (all threads). Returns the place (or -1 if no place has mass), to all threads.
template <typename F>
__device__ __forceinline__ int pick_place(VerifyShared& sh, int nseg, double u, F&& fill) {
  const int tid = threadIdx.x, lane = tid & 63;
  // segments: a wave, a run of them per lane
  if (tid < 64) {
    const int per = (nseg + 63) / 64, i0 = lane * per;
    double sum = 0.0;
    for (int i = i0; i < i0 + per && i < nseg; ++i) sum += sh.seg[i];
    const double incl = wave_incl_scan64(sum);
    const double total = __shfl(incl, 63);
    const double goal = u * total;
    double at = incl - sum;
    int first = nseg;
    double before = 0.0;
    for (int i = i0; i < i0 + per && i < nseg; ++i) {
      if (first == nseg && at + sh.seg[i] > goal) {
        first = i;
        before = at;
      }
      at += sh.seg[i];
    }
    // the first lane's find; the last segment with mass if rounding left none
    const uint64_t found = __builtin_amdgcn_ballot_w64(first < nseg);
    int last = -1;
    for (int i = i0; i < i0 + per && i < nseg; ++i)
      if (sh.seg[i] > 0.0) last = i;
    const uint64_t some = __builtin_amdgcn_ballot_w64(last >= 0);
    if (found != 0) {
      const int l = __builtin_ctzll(found);
      first = __shfl(first, l);
      before = __shfl(before, l);
    } else if (some != 0) {
      first = __shfl(last, 63 - __builtin_clzll(some));
      before = 0.0;
    }
    if (lane == 0) {
      sh.goal = found != 0 ? goal - before : INFINITY;
      sh.first = total > 0.0 ? first : nseg;
    }
  }
  __syncthreads();
  const int first = sh.first;
  if (first >= nseg) return -1;
  // within the segment the first place past the goal, else its last with mass;
  // where the segment has none after all, the next ones', then the ones' before
  for (int i = 0; i < nseg; ++i) {
    const int seg = first + i < nseg ? first + i : nseg - 1 - i;
    fill(seg);
    if (tid == 0) sh.at = kSegCols;
    __syncthreads();
    constexpr int per = kSegCols / kVerThreads;
    double v[per], sum = 0.0;
    int last = -1;
#pragma unroll
    for (int j = 0; j < per; ++j) {
      v[j] = sh.x[tid * per + j];
      sum += v[j];
      if (v[j] > 0.0) last = tid * per + j;
    }
    double incl = wave_incl_scan64(sum);
    if (lane == 63) sh.scan[tid >> 6] = incl;
    __syncthreads();
    for (int w = 0; w < (tid >> 6); ++w) incl += sh.scan[w];
    double at = incl - sum;
    const double goal = i == 0 ? sh.goal : first + i < nseg ? 0.0 : INFINITY;
    int hit = kSegCols;
#pragma unroll
    for (int j = 0; j < per; ++j) {
      at += v[j];
      if (hit == kSegCols && at > goal && v[j] > 0.0) hit = tid * per + j;
    }
    // the first lane's find is the wave's (places ascend with the lanes)
    const uint64_t any = __builtin_amdgcn_ballot_w64(hit < kSegCols);
    if (any != 0 && lane == __builtin_ctzll(any)) atomicMin(&sh.at, hit);
    __syncthreads();
    int place = sh.at;
    __syncthreads();
    if (place == kSegCols) {
      if (tid == 0) sh.at = -1;
      __syncthreads();
      const uint64_t some = __builtin_amdgcn_ballot_w64(last >= 0);
      if (some != 0 && lane == 63 - __builtin_clzll(some)) atomicMax(&sh.at, last);
      __syncthreads();
      place = sh.at;
      __syncthreads();
    }
    if (place >= 0) return seg * kSegCols + place;
  }
  return -1;
}

// What the draft leaves of p at a token, 0 up to the rounding of the two, so that a draft
// that has the target's probabilities leaves nothing. Weights far from their reference and
// the sums of fast ones are off by up to 2^-42 (kNear). Relative to the rows' largest logits,
// with sums of the same weights, probabilities are off by 2^-49 or so, and equal logits have
// equal weights (kClose).
constexpr double kNear = 0x1p-40, kClose = 0x1p-46;
__device__ __forceinline__ double excess(double p, double q, double eps) {
  return p - q > p * eps ? p - q : 0.0;
}

// the sum of the threads' x, to every thread
__device__ __forceinline__ double block_sum(VerifyShared& sh, double x) {
  x = wave_sum64(x);
  if ((threadIdx.x & 63) == 0) sh.scan[threadIdx.x >> 6] = x;
  __syncthreads();
  x = 0.0;
  for (int w = 0; w < kVerWaves; ++w) x += sh.scan[w];
  __syncthreads();
  return x;
}
// the largest of the threads' x, to every thread
__device__ __forceinline__ float block_max(VerifyShared& sh, float x) {
  x = wave_max(x);
  if ((threadIdx.x & 63) == 0) sh.scan[threadIdx.x >> 6] = x;
  __syncthreads();
  for (int w = 0; w < kVerWaves; ++w) x = fmaxf(x, (float)sh.scan[w]);
  __syncthreads();
  return x;
}
// the sum of sh.x
__device__ __forceinline__ double sum_places(VerifyShared& sh) {
  double t = 0.0;
  for (int j = threadIdx.x; j < kSegCols; j += kVerThreads) t += sh.x[j];
  return block_sum(sh, t);
}

// Where little is left (a draft rejected with a probability below 2^-10), the segments'
// sums of it are mostly the rounding of what is taken out of them: then the masses are
// formed again place by place, relative to the rows' largest logits and with their sums
// from the same weights. The question is answered by wave 0's sum of sh.seg, which all
// threads have written. One workgroup reads the row three times then: 176 us for K entries
// and 270 for a dense draft at V = 131072.
__device__ __forceinline__ bool little_left(VerifyShared& sh, int nseg, double all) {
  if (threadIdx.x < 64) {
    double t = 0.0;
    for (int i = threadIdx.x; i < nseg; i += 64) t += sh.seg[i];
    t = wave_sum64(t);
    if (threadIdx.x == 0) sh.goal = t;
  }
  __syncthreads();
  const bool little = sh.goal < all * 0x1p-10;
  __syncthreads();
  return little;
}

// place -> token, and the tokens behind it
__device__ __forceinline__ void write_tokens(const VerifyArgs& a, int b, int r, int next) {
  int32_t* out = a.out_tokens + (int64_t)b * (a.T + 1);
  for (int t = threadIdx.x; t <= a.T; t += kVerThreads)
    out[t] = t < r ? a.tokens[(int64_t)b * a.T + t] : t == r ? next : -1;
  if (threadIdx.x == 0) a.accepted[b] = r;
}

// The power of two that brings S to 1 or above, below 2: weights and sums times it are
// probabilities but for a factor below 2, and 0 where 64 bits cannot hold those. (M may be
// 2^890 below the row's largest logit, and weights relative to it go as much further.)
__device__ __forceinline__ double unit(double S) {
  return S > 0.0 ? __builtin_amdgcn_ldexp(1.0, 1 - __builtin_amdgcn_frexp_exp(S)) : 1.0;
}

// the segment's masses of the target's row: weights times f, places outside 0
template <typename T>
__device__ __forceinline__ void fill_target(VerifyShared& sh, const Row<T>& row, int seg, float M,
                                            double c, double f) {
  constexpr int VPT = Row<T>::VPT;
  for (int j = threadIdx.x; j < kSegCols / VPT; j += kVerThreads) {
    const u32x4_t x = row.at(seg * kSegCols + j * VPT);
#pragma unroll
    for (int i = 0; i < VPT; ++i) sh.x[j * VPT + i] = weight(Row<T>::elt(x, i), M, c) * f;
  }
}

// A workgroup per sequence: the places' probabilities of their tokens (a wave per
// place), the first rejected place, and with a draft of K entries the draw. The
// draft's K entries take their part of a segment's mass out of its sum: no pass
// over the vocabulary but the one segment's. Latency-bound: 9 us for one sequence,
// 17 for 256.
template <typename T, bool DENSE>
__global__ __launch_bounds__(kVerThreads) void k_accept(VerifyArgs a) {
  extern __shared__ __align__(16) char lds[];
  __shared__ VerifyShared sh;
  const int b = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = wave_id();
  const int n = drafted(a, b);
  // (S, M) of the target's row at each place; the entries' arrays behind them
  double* rowS = reinterpret_cast<double*>(lds);
  const int Kp = (a.K + 3) & ~3;
  double *em = rowS + ((a.T + 2) & ~1), *eq = em + Kp;
  int* ei = reinterpret_cast<int*>(eq + Kp);
  float* rowM = reinterpret_cast<float*>(ei + Kp);
  if (tid == 0) sh.first = n;
  __syncthreads();
  if (a.prob != nullptr)
    for (int t = n + tid; t < a.T; t += kVerThreads) a.prob[draft_row(a, b, t)] = 0.f;
  for (int t = wave; t <= n; t += kVerWaves) {
    const int64_t rt = target_row(a, b, t), rd = draft_row(a, b, t);
    // what the place needs is read first: these reads and the segments' are cold and
    // each takes microseconds
    constexpr int R = 2;  // entries of a lane in registers (K up to 128)
    int d = -1, iv[R] = {-1, -1};
    float zt = -INFINITY, zd = -INFINITY, lv[R] = {-INFINITY, -INFINITY};
    const float* l = a.dlogit + rd * a.K;
    const int32_t* ix = a.didx + rd * a.K;
    if (t < n) {
      d = a.tokens[rd];
      if constexpr (!DENSE) {
#pragma unroll
        for (int j = 0; j < R; ++j)
          if (lane + 64 * j < a.K) {
            lv[j] = number(l[lane + 64 * j]);
            iv[j] = ix[lane + 64 * j];
          }
      }
      if ((unsigned)d < (unsigned)a.V) {
        zt = Row<T>(a.target, rt * a.ld_t, a.V).one(d);
        if constexpr (DENSE) zd = Row<T>(a.draft, rd * a.ld_d, a.V).one(d);
      }
    }
    float M;
    double S;
    merge_row(a, rt, M, S);
    if (lane == 0) {
      rowM[t] = M;
      rowS[t] = S;
    }
    if (t == n) break;
    const bool known = (unsigned)d < (unsigned)a.V;
    const double p = known && S > 0.0 ? weight(zt, M, a.c) / S : 0.0;
    double q = 0.0;
    if constexpr (DENSE) {
      merge_row(a, (int64_t)a.B * (a.T + 1) + rd, M, S);
      q = known && S > 0.0 ? weight(zd, M, a.c) / S : 0.0;
    } else {
      float m = -INFINITY;
#pragma unroll
      for (int j = 0; j < R; ++j) m = fmaxf(m, lv[j]);
      for (int k = lane + 64 * R; k < a.K; k += 64) m = fmaxf(m, number(l[k]));
      m = wave_max(m);
      double s = 0.0, w = 0.0;
      auto entry = [&](float lk, int v) {
        const double e = weight(lk, m, a.c);
        s += e;
        if (v == d) w += e;
      };
#pragma unroll
      for (int j = 0; j < R; ++j)
        if (lane + 64 * j < a.K) entry(lv[j], iv[j]);
      for (int k = lane + 64 * R; k < a.K; k += 64) entry(number(l[k]), ix[k]);
      s = wave_sum64(s);
      w = wave_sum64(w);
      q = known && s > 0.0 ? w / s : 0.0;
    }
    if (lane == 0) {
      const double u = a.uniform[target_row(a, b, t)];
      if (!(u * q < p)) atomicMin(&sh.first, t);
      if (a.prob != nullptr)
        a.prob[rd] = q > 0.0 ? (float)fmin(p / q, 1.0) : p > 0.0 ? 1.f : 0.f;
    }
  }
  __syncthreads();
  const int r = sh.first;
  __syncthreads();
  const int64_t rt = target_row(a, b, r);
  float M = rowM[r];
  double f = unit(rowS[r]), S = rowS[r] * f, eps = kNear;
  if constexpr (DENSE) {
    if (wave == 0 && r < n) {
      float Md;
      double Sd;
      merge_row(a, (int64_t)a.B * (a.T + 1) + draft_row(a, b, r), Md, Sd);
      if (lane == 0) {
        a.norm[4 * b + 2] = Md;
        a.norm[4 * b + 3] = Sd;
      }
    }
    if (tid == 0) {
      a.norm[4 * b] = M;
      a.norm[4 * b + 1] = rowS[r];
      a.accepted[b] = r;
    }
    return;
  }
  const Row<T> row(a.target, rt * a.ld_t, a.V);
  const float* pm = a.segm + rt * a.nseg;
  const double* ps = a.segs + rt * a.nseg;
  // entries of the draft at the rejected place: q (eq) and the target's weight (em) at
  // the first of each index (one that repeats counts once, with the sum), else 0
  const bool rest = r < n && S > 0.0;
  // lanes of each of `count` sums, over a workgroup: powers of two up to a wave
  auto lanes_each = [](int count) {
    int each = 1;
    while (each < 64 && count * each * 2 <= kVerThreads) each *= 2;
    return each;
  };
  if (rest) {
    const float* l = a.dlogit + draft_row(a, b, r) * a.K;
    const int32_t* ix = a.didx + draft_row(a, b, r) * a.K;
    float m = -INFINITY;
    for (int k = lane; k < a.K; k += 64) m = fmaxf(m, number(l[k]));  // (each wave for itself)
    m = wave_max(m);
    double s = 0.0;
    for (int k = lane; k < a.K; k += 64) s += weight(number(l[k]), m, a.c);
    s = wave_sum64(s);
    for (int k = tid; k < Kp; k += kVerThreads) {
      const bool entry = k < a.K;
      em[k] = entry && s > 0.0 ? weight(number(l[k]), m, a.c) / s : 0.0;
      const int v = entry ? ix[k] : -1;
      ei[k] = (unsigned)v < (unsigned)a.V ? v : -1;
      eq[k] = 0.0;
    }
    __syncthreads();
    // (each lane sums over every each-th four of the entries)
    typedef __attribute__((__vector_size__(16))) int s32x4_t;
    const int each = lanes_each(a.K), sub = tid & (each - 1);
    for (int k0 = 0; k0 < a.K; k0 += kVerThreads / each) {
      const int k = k0 + tid / each;
      double q = 0.0;
      int again = 0;
      const int v = k < a.K ? ei[k] : -1;
      if (v >= 0) {
#pragma unroll 4
        for (int j = 4 * sub; j < Kp; j += 4 * each) {
          const s32x4_t w = *reinterpret_cast<const s32x4_t*>(ei + j);
#pragma unroll
          for (int x = 0; x < 4; ++x)
            if (w[x] == v) {
              q += em[j + x];
              again |= j + x < k;
            }
        }
      }
      for (int o = each / 2; o >= 1; o >>= 1) {
        q += __shfl_xor(q, o);
        again |= __shfl_xor(again, o);
      }
      if (v >= 0 && sub == 0 && again == 0) eq[k] = q;
    }
    __syncthreads();
    for (int k = tid; k < Kp; k += kVerThreads)
      em[k] = eq[k] > 0.0 ? weight(row.one(ei[k]), M, a.c) * f : 0.0;
    __syncthreads();
  }
  {
    typedef __attribute__((__vector_size__(16))) int s32x4_t;
    const int each = lanes_each(a.nseg), sub = tid & (each - 1);
    for (int i0 = 0; i0 < a.nseg; i0 += kVerThreads / each) {
      const int i = i0 + tid / each;
      double take = 0.0;
      if (rest && i < a.nseg) {
        // columns of segment i, -1 being of none
        const int v0 = max(i * kSegCols - row.shift, 0), v1 = (i + 1) * kSegCols - row.shift;
#pragma unroll 4
        for (int k = 4 * sub; k < Kp; k += 4 * each) {
          const s32x4_t w = *reinterpret_cast<const s32x4_t*>(ei + k);
#pragma unroll
          for (int x = 0; x < 4; ++x)
            if (w[x] >= v0 && w[x] < v1) take += fmin(eq[k + x] * S, em[k + x]);
        }
      }
      for (int o = each / 2; o >= 1; o >>= 1) take += __shfl_xor(take, o);
      if (sub == 0 && i < a.nseg) {
        // (where the rounding leaves nothing of a sum that was taken from, its places
        // may still hold a little, which a random number of 0 asks for)
        const double left = mass(ps[i] * f, pm[i], M, a.c) - take;
        sh.seg[i] = left > 0.0 ? left : take > 0.0 ? 0x1p-1000 : 0.0;
      }
    }
  }
  __syncthreads();
  const double u = a.uniform[target_row(a, b, a.T)];
  // the masses of a segment's places, in sh.x
  auto fill = [&](int seg) {
    fill_target<T>(sh, row, seg, M, a.c, f);
    __syncthreads();
    if (rest)
      for (int k = tid; k < a.K; k += kVerThreads) {
        const int e = ei[k] + row.shift - seg * kSegCols;
        if (eq[k] > 0.0 && (unsigned)e < (unsigned)kSegCols) sh.x[e] = excess(em[k], eq[k] * S, eps);
      }
    __syncthreads();
  };
  if (rest && little_left(sh, a.nseg, S)) {
    constexpr int VPT = Row<T>::VPT;
    const int end = a.nseg * kSegCols;
    float m = -INFINITY;
    for (int e = tid * VPT; e < end; e += kVerThreads * VPT) {
      const u32x4_t x = row.at(e);
      for (int i = 0; i < VPT; ++i) m = fmaxf(m, Row<T>::elt(x, i));
    }
    M = block_max(sh, m);
    double t = 0.0;
    for (int e = tid * VPT; e < end; e += kVerThreads * VPT) {
      const u32x4_t x = row.at(e);
      for (int i = 0; i < VPT; ++i) t += weight(Row<T>::elt(x, i), M, a.c);
    }
    S = block_sum(sh, t);
    f = 1.0;
    eps = kClose;
    for (int k = tid; k < Kp; k += kVerThreads)
      em[k] = eq[k] > 0.0 ? weight(row.one(ei[k]), M, a.c) : 0.0;
    __syncthreads();
    for (int seg = 0; seg < a.nseg; ++seg) {
      fill(seg);
      const double t = sum_places(sh);
      if (tid == 0) sh.seg[seg] = t;
    }
    __syncthreads();
  }
  int place = pick_place(sh, a.nseg, u, fill);
  if (place < 0 && rest) {
    // p does not exceed q anywhere: from p
    for (int i = tid; i < a.nseg; i += kVerThreads) sh.seg[i] = mass(ps[i] * f, pm[i], M, a.c);
    __syncthreads();
    place = pick_place(sh, a.nseg, u, [&](int seg) {
      fill_target<T>(sh, row, seg, M, a.c, f);
      __syncthreads();
    });
  }
  write_tokens(a, b, r, place < 0 ? -1 : place - row.shift);
}

// the masses of a dense draft's rejected row: max(p - q, 0), p where nothing was
// rejected; places count from the target row's boundary
struct RestRow {
  Weights t, d;
  double it, id;  // 1 / S
  double eps = kNear;
  bool rest;
  __device__ __forceinline__ RestRow(const VerifyArgs& a, int b, bool rest_, const uint64_t* tab)
      : t((float)a.norm[4 * b], a.c, tab),
        d(rest_ ? (float)a.norm[4 * b + 2] : 0.f, a.c, tab),
        it(a.norm[4 * b + 1] > 0.0 ? 1.0 / a.norm[4 * b + 1] : 0.0),
        id(rest_ && a.norm[4 * b + 3] > 0.0 ? 1.0 / a.norm[4 * b + 3] : 0.0),
        rest(rest_) {}
  __device__ __forceinline__ bool fast() const { return t.fast && d.fast; }
  __device__ __forceinline__ double quick(float zt, float zd) const {
    return fmax(t.quick(zt) * (it * t.fix) - d.quick(zd) * (id * d.fix), 0.0);
  }
  __device__ __forceinline__ double exact(float zt, float zd) const {
    const double p = t.exact(zt) * it;
    return rest ? excess(p, d.exact(zd) * id, eps) : p;
  }
};
// vector of the draft's row at the target's place e (its own boundary may differ)
template <typename T>
__device__ __forceinline__ u32x4_t draft_at(const Row<T>& d, int e, int shift) {
  if (d.shift == shift) return d.at(e);
  constexpr int VPT = Row<T>::VPT;
  uint32_t w[4];
  const int v = e - shift;
  if constexpr (sizeof(T) == 2) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint16_t* h = reinterpret_cast<const uint16_t*>(d.p);
      const uint32_t x = (unsigned)(v + 2 * i) < (unsigned)d.V ? h[v + 2 * i] : 0xff80u;
      const uint32_t y = (unsigned)(v + 2 * i + 1) < (unsigned)d.V ? h[v + 2 * i + 1] : 0xff80u;
      w[i] = x | y << 16;
    }
  } else {
#pragma unroll
    for (int i = 0; i < VPT; ++i)
      w[i] = (unsigned)(v + i) < (unsigned)d.V ? reinterpret_cast<const uint32_t*>(d.p)[v + i]
                                               : 0xff800000u;
  }
  return u32x4_t{w[0], w[1], w[2], w[3]};
}

// Dense draft: the mass of each segment at the place where the sequence ended, a
// workgroup per segment (two rows with an exponential each: the few segments of a
// small batch are spread over more of the chip). Nothing rejected: the target's
// own sums serve.
template <typename T>
__global__ __launch_bounds__(256) void k_rest_sums(VerifyArgs a) {
  __shared__ uint64_t tab[kTab];
  __shared__ double part[4];
  load_roots(tab);
  const int b = blockIdx.x / a.nseg, seg = blockIdx.x - b * a.nseg;
  const int r = a.accepted[b];
  if (r >= drafted(a, b)) return;
  const RestRow m(a, b, true, tab);
  const Row<T> row(a.target, target_row(a, b, r) * a.ld_t, a.V);
  const Row<T> dr(a.draft, draft_row(a, b, r) * a.ld_d, a.V);
  constexpr int VPT = Row<T>::VPT;
  double s = 0.0;
  for (int e = threadIdx.x * VPT; e < kSegCols; e += 256 * VPT) {
    const u32x4_t x = row.at(seg * kSegCols + e);
    const u32x4_t y = draft_at<T>(dr, seg * kSegCols + e, row.shift);
    if (m.fast()) {
#pragma unroll
      for (int i = 0; i < VPT; ++i) s += m.quick(Row<T>::elt(x, i), Row<T>::elt(y, i));
    } else {
      for (int i = 0; i < VPT; ++i) s += m.exact(Row<T>::elt(x, i), Row<T>::elt(y, i));
    }
  }
  s = wave_sum64(s);
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = s;
  __syncthreads();
  if (threadIdx.x == 0) a.segr[blockIdx.x] = (part[0] + part[1]) + (part[2] + part[3]);
}

template <typename T>
__global__ __launch_bounds__(kVerThreads) void k_pick(VerifyArgs a) {
  __shared__ VerifyShared sh;
  const int b = blockIdx.x, tid = threadIdx.x;
  const int r = a.accepted[b];
  const bool rest = r < drafted(a, b);
  const int64_t rt = target_row(a, b, r);
  const Row<T> row(a.target, rt * a.ld_t, a.V);
  const Row<T> dr(a.draft, draft_row(a, b, rest ? r : 0) * a.ld_d, a.V);
  RestRow m(a, b, rest, nullptr);
  const float* pm = a.segm + rt * a.nseg;
  const double* ps = a.segs + rt * a.nseg;
  for (int i = tid; i < a.nseg; i += kVerThreads)
    sh.seg[i] = rest        ? a.segr[(int64_t)b * a.nseg + i]
                : m.it > 0.0 ? mass(ps[i] * m.it, pm[i], m.t.m, a.c)
                             : 0.0;
  __syncthreads();
  const double u = a.uniform[target_row(a, b, a.T)];
  constexpr int VPT = Row<T>::VPT;
  auto fill = [&](int seg) {
    for (int j = tid; j < kSegCols / VPT; j += kVerThreads) {
      const int e = seg * kSegCols + j * VPT;
      const u32x4_t x = row.at(e);
      const u32x4_t y = rest ? draft_at<T>(dr, e, row.shift) : x;
#pragma unroll
      for (int i = 0; i < VPT; ++i)
        sh.x[j * VPT + i] = m.exact(Row<T>::elt(x, i), Row<T>::elt(y, i));
    }
    __syncthreads();
  };
  if (rest && m.it > 0.0 && little_left(sh, a.nseg, 1.0)) {
    const int end = a.nseg * kSegCols;
    float mt = -INFINITY, md = -INFINITY;
    for (int e = tid * VPT; e < end; e += kVerThreads * VPT) {
      const u32x4_t x = row.at(e), y = draft_at<T>(dr, e, row.shift);
      for (int i = 0; i < VPT; ++i) {
        mt = fmaxf(mt, Row<T>::elt(x, i));
        md = fmaxf(md, Row<T>::elt(y, i));
      }
    }
    m.t.m = block_max(sh, mt);
    m.d.m = block_max(sh, md);
    m.eps = kClose;
    double st = 0.0, sd = 0.0;
    for (int e = tid * VPT; e < end; e += kVerThreads * VPT) {
      const u32x4_t x = row.at(e), y = draft_at<T>(dr, e, row.shift);
      for (int i = 0; i < VPT; ++i) {
        st += m.t.exact(Row<T>::elt(x, i));
        sd += m.d.exact(Row<T>::elt(y, i));
      }
    }
    st = block_sum(sh, st);
    sd = block_sum(sh, sd);
    m.it = 1.0 / st;
    m.id = sd > 0.0 ? 1.0 / sd : 0.0;
    for (int seg = 0; seg < a.nseg; ++seg) {
      fill(seg);
      const double t = sum_places(sh);
      if (tid == 0) sh.seg[seg] = t;
    }
    __syncthreads();
  }
  int place = pick_place(sh, a.nseg, u, fill);
  if (place < 0 && rest && m.it > 0.0) {
    for (int i = tid; i < a.nseg; i += kVerThreads) sh.seg[i] = mass(ps[i] * m.it, pm[i], m.t.m, a.c);
    __syncthreads();
    place = pick_place(sh, a.nseg, u, [&](int seg) {
      fill_target<T>(sh, row, seg, m.t.m, a.c, m.it);
      __syncthreads();
    });
  }
  write_tokens(a, b, r, place < 0 ? -1 : place - row.shift);
}

}  // namespace kd

// ================================================================ launchers ==
using namespace kd;

// How rows are selected from (us for all of it, top 64 or 100, with the read back):
//  * up to 256 rows: 1024 threads a row in the second pass. One row of 131072 in fp32
//    11.1 (256 threads 15.7), 256 rows bf16 25.5 (30.0), 300 rows 33.9 (32.7).
//  * rows that 8 vectors a thread hold: one pass, the row in registers (8192 rows of
//    4000 166 in two passes, 87).
//  * more rows: each streamed by its own workgroup. Long ones (48 segments, about
//    100000 columns) by 512 threads: 300 rows 28.8 (two passes 32.7), 777 50.1 (53.0),
//    4096 192 (236; 256 threads 203). Shorter ones by 256 threads once there are 1536:
//    8000 rows of 50257 169 (208; 512 threads 198). In fp32 with log-probabilities the
//    two cross there: 1300 rows of 50257 61.7 (56.0), 1800 80.0 (79.6), 2200 91.9 (99.4);
//    in bf16 streaming is between 4% slower and 9% faster from 600 rows to 1800.
//  * else two passes, 256 threads a row in the second.
constexpr int64_t kSelectFewRows = 256, kSelectStreamRows = 1536;
constexpr int kSelectLongSegs = 48;

template <typename T>
static int launch_topk(const KdTopkArgs& a, hipStream_t s) {
  const T* x = static_cast<const T*>(a.logits);
  SelectArgs q{a.logits, a.ld, a.V, a.K, 0, a.nseg, a.logprobs, a.gmax, a.pm, a.ps,
               a.idx, a.value, a.entries, a.scale};
  const dim3 rows((unsigned)a.rows);
  const bool wide = a.rows <= kSelectFewRows;
  // vectors of a row, wherever it starts
  constexpr int VPT = Row<T>::VPT;
  const int vectors = (a.V + 2 * (VPT - 1)) / VPT;
  if (vectors <= (wide ? 1024 * select_keys(1024, true) : 256 * select_keys(256, true))) {
    q.G = vectors;
    const size_t lds = select_lds(q.G, a.K);
    if (wide)
      hipLaunchKernelGGL((k_row_select<T, 1024, kDirect>), rows, dim3(1024), lds, s, q);
    else
      hipLaunchKernelGGL((k_row_select<T, 256, kDirect>), rows, dim3(256), lds, s, q);
    return (int)hipGetLastError();
  }
  q.G = a.nseg * kSegGroups;
  const size_t lds = select_lds(q.G, a.K);
  // (the keys of a streamed row stand where its candidates will, then in registers)
  auto streams = [&](int threads) {
    return !wide && 4 * q.G <= 8 * select_cap(a.K) && q.G <= threads * select_keys(threads, true);
  };
  if (streams(512) && a.nseg >= kSelectLongSegs) {
    hipLaunchKernelGGL((k_row_select<T, 512, kStream>), rows, dim3(512), lds, s, q);
    return (int)hipGetLastError();
  }
  if (streams(256) && a.rows >= kSelectStreamRows) {
    hipLaunchKernelGGL((k_row_select<T, 256, kStream>), rows, dim3(256), lds, s, q);
    return (int)hipGetLastError();
  }
  const int64_t waves = a.rows * a.nseg;
  const dim3 grid((unsigned)((waves + 3) / 4));
  if (a.logprobs)
    hipLaunchKernelGGL((k_row_groups<T, true>), grid, dim3(256), 0, s, x, a.ld, a.V, a.nseg,
                       (int)waves, a.gmax, a.pm, a.ps);
  else
    hipLaunchKernelGGL((k_row_groups<T, false>), grid, dim3(256), 0, s, x, a.ld, a.V, a.nseg,
                       (int)waves, a.gmax, (float*)nullptr, (float*)nullptr);
  if (wide)
    hipLaunchKernelGGL((k_row_select<T, 1024, kFromMaxima>), rows, dim3(1024), lds, s, q);
  else
    hipLaunchKernelGGL((k_row_select<T, 256, kFromMaxima>), rows, dim3(256), lds, s, q);
  return (int)hipGetLastError();
}

extern "C" int kd_launch_topk(const KdTopkArgs* a, void* stream) {
  hipStream_t s = static_cast<hipStream_t>(stream);
  return a->dtype == 1 ? launch_topk<__bf16>(*a, s) : launch_topk<float>(*a, s);
}

extern "C" int kd_launch_cache_read(const KdCacheReadArgs* a, void* stream) {
  hipStream_t s = static_cast<hipStream_t>(stream);
  const bool v4 = a->K % 4 == 0 && (((uintptr_t)a->entries | (uintptr_t)a->idx |
                                     (uintptr_t)a->value) & 15u) == 0;
  // rows of a block: about 1024 pieces, at most 64 rows
  const int per = v4 ? a->K / 4 : a->K;
  const int rpb = per >= 1024 ? 1 : 1024 / per > 64 ? 64 : 1024 / per;
  const int64_t blocks = (a->M + rpb - 1) / rpb;
  const dim3 grid((unsigned)(blocks < (1 << 20) ? blocks : 1 << 20));
  auto k = !v4                                        ? k_cache_read<false, false>
           : a->M * (int64_t)a->K * 8 < kBigBytes ? k_cache_read<true, false>
                                                      : k_cache_read<true, true>;
  hipLaunchKernelGGL(k, grid, dim3(256), 0, s, a->entries, a->scale, a->rows, a->N, a->M, a->K,
                     rpb, a->idx, a->value, a->ignore);
  return (int)hipGetLastError();
}

static unsigned stream_blocks(int64_t threads) {
  const int64_t b = (threads + 255) / 256;
  return (unsigned)(b < 16384 ? b : 16384);
}

template <typename T>
static int launch_ckpt_write(const void* hidden, int64_t n, uint8_t* codes, uint8_t* scales,
                             hipStream_t s) {
  auto k = n * (int64_t)sizeof(T) < kBigBytes ? k_ckpt_write<T, false> : k_ckpt_write<T, true>;
  hipLaunchKernelGGL(k, dim3(stream_blocks(n / 8)), dim3(256), 0, s, static_cast<const T*>(hidden),
                     n / 8, codes, scales);
  return (int)hipGetLastError();
}
template <typename T>
static int launch_ckpt_read(const uint8_t* codes, const uint8_t* scales, int64_t n, void* hidden,
                            hipStream_t s) {
  auto k = n * (int64_t)sizeof(T) < kBigBytes ? k_ckpt_read<T, false> : k_ckpt_read<T, true>;
  const int64_t n16 = n * (int64_t)sizeof(T) / 16;
  hipLaunchKernelGGL(k, dim3(stream_blocks(n16)), dim3(256), 0, s, codes, scales, n16,
                     static_cast<T*>(hidden));
  return (int)hipGetLastError();
}

extern "C" int kd_launch_ckpt_write(const void* hidden, int dtype, int64_t n, uint8_t* codes,
                                    uint8_t* scales, void* stream) {
  hipStream_t s = static_cast<hipStream_t>(stream);
  return dtype == 1 ? launch_ckpt_write<__bf16>(hidden, n, codes, scales, s)
                    : launch_ckpt_write<float>(hidden, n, codes, scales, s);
}

extern "C" int kd_launch_ckpt_read(const uint8_t* codes, const uint8_t* scales, int dtype,
                                   int64_t n, void* hidden, void* stream) {
  hipStream_t s = static_cast<hipStream_t>(stream);
  return dtype == 1 ? launch_ckpt_read<__bf16>(codes, scales, n, hidden, s)
                    : launch_ckpt_read<float>(codes, scales, n, hidden, s);
}

template <typename T>
static int launch_verify(const KdVerifyArgs& q, hipStream_t s) {
  const VerifyArgs a{q.target, q.draft, q.ld_t, q.ld_d, q.B, q.T, q.V, q.K, q.nseg,
                     q.tokens, q.didx, q.dlogit, q.uniform, q.lengths, q.c, q.out_tokens,
                     q.accepted, q.prob, q.segm, q.segs, q.segr, q.norm};
  const bool dense = q.draft != nullptr;
  const int64_t waves = ((int64_t)q.B * (q.T + 1) + (dense ? (int64_t)q.B * q.T : 0)) * q.nseg;
  hipLaunchKernelGGL(k_seg_sums<T>, dim3((unsigned)((waves + 3) / 4)), dim3(256), 0, s, a,
                     (int)waves);
  if (!dense) {
    const size_t lds = (size_t)((q.K + 3) & ~3) * 20 + (size_t)(q.T + 2) * 12;
    hipLaunchKernelGGL((k_accept<T, false>), dim3(q.B), dim3(kVerThreads), lds, s, a);
    return (int)hipGetLastError();
  }
  hipLaunchKernelGGL((k_accept<T, true>), dim3(q.B), dim3(kVerThreads), (size_t)(q.T + 2) * 12, s,
                     a);
  hipLaunchKernelGGL(k_rest_sums<T>, dim3((unsigned)(q.B * q.nseg)), dim3(256), 0, s, a);
  hipLaunchKernelGGL(k_pick<T>, dim3(q.B), dim3(kVerThreads), 0, s, a);
  return (int)hipGetLastError();
}

extern "C" int kd_launch_verify(const KdVerifyArgs* a, void* stream) {
  hipStream_t s = static_cast<hipStream_t>(stream);
  return a->dtype == 1 ? launch_verify<__bf16>(*a, s) : launch_verify<float>(*a, s);
}
