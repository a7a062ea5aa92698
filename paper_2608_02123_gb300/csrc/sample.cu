// pctree_sample: the target's token at every row of its logits, from given
// random numbers, with temperature, top-k, top-p and min-p.
//
// A row belongs to a cluster of up to eight CTAs, each of which keeps its slice
// of the row in shared memory: the logits are read from memory once, and every
// later pass (maximum, weights, selection, draw) runs on shared memory, with
// the CTAs' results exchanged through distributed shared memory.
//
// Weights w = exp((z - max) / T) are summed as integers in units of 2^-45 of
// the largest weight, so sums are exact and in any order the same.  A token is
// drawn where the cumulative weight passes u * total: with 10^5 borders between
// tokens, a relative error d of the cumulative weights moves one of them past
// the random number in 10^5 d of all rows, so single-precision exponentials
// would miss a token in a few rows of a thousand.  Two forms of the weight:
//   light  2^(n/128) from a table in 31-bit fixed point, times 1 + s, s the
//          rest of at most 1/256 octave by a cubic: relative error 2^-30.5,
//          independent from token to token;
//   fine   the same with every term carried as a float pair: 2^-41.
// Tokens above 2^-12 of the total use the fine form (there are at most 4096);
// the errors of the light ones then add up to at most 2^-36.5 of the total.
//
// Selection: every filter keeps a head of the order (z desc, index asc), which
// is the set of keys K >= K* for K = (z, -index) as one 64-bit integer, K* the
// largest key whose head reaches a target count (top-k) or weight (top-p).
// The logits are binned linearly below the maximum (512 bins over 16 octaves
// of weight, over all 46 where that is too few); the bin that the target falls
// in is gathered and ranked.  A bin too full for that (long runs of equal
// logits) is left to a bisection over the keys.
#include "kv_rows.cuh"
#include "sm103_ptx.cuh"

namespace pct {
namespace {

constexpr int kSmpThreads = 512;
constexpr int kSmpWarps = kSmpThreads / 32;
constexpr int kSmpMaxCluster = 8;
constexpr int kSmpBins = 512;
constexpr int kSmpList = 512;               // gathered keys of a bin
constexpr int kSmpMaxV = 1 << 18;           // sums of 2^45-scaled weights fit 64 bits
constexpr int kOctaves = 46;                // below: weight 0
constexpr int kNarrow = 16;                 // octaves of the first binning
constexpr float kMagic = 12582912.0f;       // 1.5 * 2^23: adds as round to integer
constexpr float kMagic2 = 0.0234375f;       // 1.5 * 2^-6: rounds to 2^-29
constexpr float kLn2 = 0.693147180559945f / 128.0f;

// 2^(j/128) by the exponential series, at compile time: in 31-bit fixed point,
// as a float and the rest of that float.
struct Pow2Table {
  uint32_t fix[128];
  float hi[128], lo[128];
};
constexpr Pow2Table make_pow2() {
  Pow2Table t{};
  for (int j = 0; j < 128; ++j) {
    const double x = j * (0.693147180559945309417232 / 128);
    double term = 1.0, sum = 1.0;
    for (int i = 1; i < 30; ++i) {
      term *= x / i;
      sum += term;
    }
    t.fix[j] = static_cast<uint32_t>(sum * 2147483648.0 + 0.5);
    t.hi[j] = static_cast<float>(sum);
    t.lo[j] = static_cast<float>(sum - static_cast<double>(t.hi[j]));
  }
  return t;
}
__device__ const Pow2Table kPow2 = make_pow2();

struct SampleArgs {
  const void* logits;
  const float* uniform;
  const float* temperature;
  const int32_t* top_k;
  const float* top_p;
  const float* min_p;
  const int32_t* n_rows;
  int32_t* tokens;
  int32_t* status;
  long long row_stride;
  int V, group, slice;                      // slice: elements per CTA of the cluster
};

// What a row's passes need, the same in every CTA of its cluster.
struct RowFacts {
  float c_hi, c_lo;                         // 128 log2(e) / T
  float base;                               // subtracted from z before scaling
  float m;                                  // max - base
  float cut;                                // z - base below it has weight 0
  float fine_from;                          // z - base from it on uses the fine form
  int k0;                                   // round(m * 128 log2(e) / T)
};

struct alignas(16) SampleShared {
  uint64_t bar;
  RowFacts row;
  float warp_max[kSmpWarps];
  float cta_max[kSmpMaxCluster];
  int cta_first[kSmpMaxCluster];            // lowest index of the maximum (T = 0)
  unsigned long long warp_sum[kSmpMaxCluster * kSmpWarps];
  // found by the leader, written to every CTA
  int bin;                                  // -1: the target lies past the bins
  unsigned long long above_n, above_w;      // count and weight before the bin
  unsigned long long border, border_w;      // K* and the weight of its head
  unsigned long long total_w;               // weight of all bins
  unsigned list_n;
  unsigned long long part_n[kSmpMaxCluster], part_w[kSmpMaxCluster];
  unsigned long long red[2 * kSmpWarps];
  // the leader's sum of all CTAs' bins
  unsigned bin_n[kSmpBins];
  unsigned long long bin_w[kSmpBins];
  union {
    unsigned hist[4][kSmpBins];             // count, weight in 15-bit limbs
    struct {
      unsigned long long key[kSmpList], w[kSmpList];
    } list;
  };
  uint2 tab[128][16];                       // light table, a column per lane pair
};

template <typename T>
__device__ __forceinline__ T* cluster_ptr(T* p, int rank) {
  uint64_t r;
  asm volatile("mapa.u64 %0, %1, %2;" : "=l"(r) : "l"(reinterpret_cast<uint64_t>(p)), "r"(rank));
  return reinterpret_cast<T*>(r);
}

// Barrier of the cluster's CTAs, with the warp's lanes together.
__device__ __forceinline__ void csync() {
  __syncwarp();
  cluster_sync();
}

__device__ __forceinline__ unsigned long long light_weight(const SampleShared* S,
                                                           const RowFacts& f, float x) {
  const float t = fmaf(x, f.c_hi, kMagic);
  const float kf = t - kMagic;
  float r = fmaf(x, f.c_hi, -kf);
  r = fmaf(x, f.c_lo, r);
  float p = fmaf(r, kLn2 * kLn2 * kLn2 / 6.0f, kLn2 * kLn2 / 2.0f);
  p = fmaf(r, p, kLn2);
  const float s = r * p;
  const int n = __float_as_int(t) - 0x4b400000 - f.k0;      // <= 0
  const uint2 e = S->tab[n & 127][threadIdx.x & 15];
  const float b = fmaf(__uint_as_float(e.y), s, kMagic2);
  const uint32_t w = e.x + (static_cast<uint32_t>(__float_as_int(b)) << 2);
  const int sh = -(n >> 7);
  return ((static_cast<unsigned long long>(w) << 14) + ((1ull << sh) >> 1)) >> sh;
}

__device__ __forceinline__ unsigned long long fine_weight(const RowFacts& f, float x) {
  const float ph = x * f.c_hi;
  const float pl = fmaf(x, f.c_lo, fmaf(x, f.c_hi, -ph));
  const float kf = rintf(ph);
  const float r = (ph - kf) + pl;                           // |r| <= 1/2 (and a little)
  const float rl = pl - (r - (ph - kf));
  // y = r ln2 / 128 as a pair
  constexpr float l_hi = 0.00541521234810352325f;           // ln2 / 128 to float, and its rest
  constexpr float l_lo = static_cast<float>(0.693147180559945309417 / 128.0 -
                                            static_cast<double>(l_hi));
  const float yh = r * l_hi;
  const float yl = fmaf(r, l_hi, -yh) + fmaf(r, l_lo, rl * l_hi);
  const float sl = fmaf(yh * yh, fmaf(yh, fmaf(yh, 1.0f / 24.0f, 1.0f / 6.0f), 0.5f), yl);
  const int n = static_cast<int>(kf) - f.k0;
  const int j = n & 127;
  const float th = kPow2.hi[j], tl = kPow2.lo[j];
  const float q = th * yh;
  const float rest = fmaf(th, yh, -q) + fmaf(th, sl, tl);
  const float unit = 35184372088832.0f;                     // 2^45
  const long long w = __float2ll_rn(th * unit) + __float2ll_rn(q * unit) +
                      __float2ll_rn(rest * unit);
  const int sh = -(n >> 7);
  return (static_cast<unsigned long long>(w) + ((1ull << sh) >> 1)) >> sh;
}

__device__ __forceinline__ unsigned long long weight(const SampleShared* S, const RowFacts& f,
                                                     float x) {
  if (x < f.cut) return 0ull;
  return x >= f.fine_from ? fine_weight(f, x) : light_weight(S, f, x);
}

// Order (z desc, index asc) as integers, largest first.
__device__ __forceinline__ unsigned long long order_key(float z, int index) {
  const unsigned b = __float_as_uint(z + 0.0f);             // -0 ranks as 0
  const unsigned o = (b & 0x80000000u) ? ~b : b | 0x80000000u;
  return (static_cast<unsigned long long>(o) << 32) | (0xffffffffu - static_cast<unsigned>(index));
}

__device__ __forceinline__ unsigned long long warp_sum64(unsigned long long v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(kFull, v, o);
  return v;
}

template <int DT>
struct Elem;
template <>
struct Elem<PCTREE_F32> {
  using type = float;
  static constexpr int kVec = 4;
  static __device__ __forceinline__ float low() { return -INFINITY; }
  static __device__ __forceinline__ void unpack(const uint4& v, float (&x)[4]) {
    x[0] = __uint_as_float(v.x);
    x[1] = __uint_as_float(v.y);
    x[2] = __uint_as_float(v.z);
    x[3] = __uint_as_float(v.w);
  }
};
template <bool F16>
struct Elem16 {
  using type = uint16_t;
  static constexpr int kVec = 8;
  static __device__ __forceinline__ uint16_t low() { return F16 ? 0xfc00 : 0xff80; }
  static __device__ __forceinline__ void unpack(const uint4& v, float (&x)[8]) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float2 p = unpack16<F16>(w[e]);
      x[2 * e] = p.x;
      x[2 * e + 1] = p.y;
    }
  }
};
template <>
struct Elem<PCTREE_BF16> : Elem16<false> {};
template <>
struct Elem<PCTREE_F16> : Elem16<true> {};

template <int DT>
__global__ void __launch_bounds__(kSmpThreads) sample_kernel(SampleArgs a) {
  using E = Elem<DT>;
  using T = typename E::type;
  constexpr int kVec = E::kVec;
  extern __shared__ __align__(16) uint8_t smem[];
  SampleShared* S = reinterpret_cast<SampleShared*>(smem);
  T* data = reinterpret_cast<T*>(smem + sizeof(SampleShared));
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int n_cta = static_cast<int>(a.V + a.slice - 1) / a.slice;   // = the cluster's size
  const int rank = static_cast<int>(cluster_ctarank());
  const int row = blockIdx.x / n_cta;
  SampleShared* L = cluster_ptr(S, 0);                      // the leader's
  pdl_launch_dependents();
  if (tid == 0) {
    mbar_init(&S->bar, 1);
    fence_barrier_init();
  }
  for (int i = tid; i < 128 * 16; i += kSmpThreads) {
    const int j = i >> 4;
    S->tab[j][i & 15] = make_uint2(
        kPow2.fix[j] - (static_cast<uint32_t>(__float_as_int(kMagic2)) << 2),
        __float_as_uint(kPow2.hi[j]));
  }
  pdl_wait();
  const int g = row / a.group;
  if (a.n_rows != nullptr && row - g * a.group >= a.n_rows[g]) {
    if (rank == 0 && tid == 0) a.tokens[row] = -1;
    return;                                                 // the whole cluster
  }
  // ---------------- the slice into shared memory ----------------
  const int e0 = rank * a.slice, n_el = min(a.slice, a.V - e0);
  const T* src = static_cast<const T*>(a.logits) + row * a.row_stride + e0;
  // element i lies at data[pad + i], so that global and shared addresses agree
  // modulo 16 bytes; the vectors' places outside the slice hold -inf
  const int pad = static_cast<int>((reinterpret_cast<uintptr_t>(src) & 15u) / sizeof(T));
  const int n_vec = (pad + n_el + kVec - 1) / kVec;
  const int head = pad == 0 ? 0 : min(n_el, kVec - pad);
  const int body = (n_el - head) / kVec;                    // whole vectors
  __syncthreads();
  if (tid == 0 && body > 0) {
    mbar_arrive_expect_tx(&S->bar, static_cast<uint32_t>(body) * 16u);
    const uint32_t bar = smem_u32(&S->bar);
    const T* from = src + head;
    uint32_t to = smem_u32(data + pad + head);
    for (int left = body; left > 0;) {
      const int v = left < 1024 ? left : 1024;              // 16 KB a copy
      asm volatile(
          "cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::
              "r"(to), "l"(reinterpret_cast<uint64_t>(from)), "r"(v * 16), "r"(bar)
          : "memory");
      to += v * 16;
      from += v * kVec;
      left -= v;
    }
  }
  if (tid < head) data[pad + tid] = src[tid];
  const int tail0 = head + body * kVec;
  if (tid >= 32 && tid < 32 + n_el - tail0) data[pad + tail0 + tid - 32] = src[tail0 + tid - 32];
  if (tid >= 64 && tid < 64 + pad) data[tid - 64] = E::low();
  if (tid >= 96 && tid < 96 + n_vec * kVec - pad - n_el) data[pad + n_el + tid - 96] = E::low();
  // the row's parameters
  const float temp = a.temperature != nullptr ? a.temperature[g] : 1.0f;
  const int top_k = a.top_k != nullptr ? a.top_k[g] : 0;
  const float top_p = a.top_p != nullptr ? a.top_p[g] : 1.0f;
  const float min_p = a.min_p != nullptr ? a.min_p[g] : 0.0f;
  const float u = a.uniform[row];
  const bool params_ok = (temp == 0.0f || (temp >= 1e-6f && temp <= 1e6f)) && top_p > 0.0f &&
                         min_p >= 0.0f && min_p <= 1.0f && u >= 0.0f && u < 1.0f;
  bool landed = true;
  if (body > 0) {
    volatile int never = 0;
    landed = mbar_wait_bounded(&S->bar, 0, &never, 1000000000ull);
  }
  __syncthreads();
  // each warp has a run of the slice's vectors
  const int per_warp = (n_vec + kSmpWarps - 1) / kSmpWarps;
  const int v0 = min(n_vec, warp * per_warp), v1 = min(n_vec, v0 + per_warp);
  const uint4* vec = reinterpret_cast<const uint4*>(data);
  const int first = e0 - pad;                               // row index of data[0]

  // ---------------- maximum ----------------
  float m = -INFINITY;
  for (int v = v0 + lane; v < v1; v += 32) {
    float x[kVec];
    E::unpack(vec[v], x);
#pragma unroll
    for (int e = 0; e < kVec; ++e) m = max_nan(m, x[e]);
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) m = max_nan(m, __shfl_xor_sync(kFull, m, o));
  if (lane == 0) S->warp_max[warp] = m;
  __syncthreads();
  // every CTA of the cluster has started before its memory is written
  csync();
  if (warp == 0) {
    m = lane < kSmpWarps ? S->warp_max[lane] : -INFINITY;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) m = max_nan(m, __shfl_xor_sync(kFull, m, o));
    if (!landed) m = __int_as_float(0x7fc00000);
    if (lane < n_cta) cluster_ptr(S, lane)->cta_max[rank] = m;
  }
  csync();
  m = S->cta_max[0];
  for (int c = 1; c < n_cta; ++c) m = max_nan(m, S->cta_max[c]);
  if (!params_ok || !(fabsf(m) < INFINITY)) {
    if (rank == 0 && tid == 0) {
      a.tokens[row] = -1;
      if (a.status != nullptr)
        atomicCAS(a.status, 0, !params_ok ? PCTREE_ERR_INVALID_ARG : PCTREE_ERR_NONFINITE);
    }
    return;
  }
  if (temp == 0.0f) {                                       // the lowest index of the maximum
    int at = 0x7fffffff;
    for (int v = v0 + lane; v < v1; v += 32) {
      float x[kVec];
      E::unpack(vec[v], x);
#pragma unroll
      for (int e = 0; e < kVec; ++e)
        if (x[e] == m) at = min(at, first + v * kVec + e);
    }
    at = __reduce_min_sync(kFull, at);
    int* best = reinterpret_cast<int*>(S->red);
    if (lane == 0) best[warp] = at;
    __syncthreads();
    if (tid == 0) {
      for (int w = 1; w < kSmpWarps; ++w) at = min(at, best[w]);
      L->cta_first[rank] = at;
    }
    csync();
    if (rank == 0 && tid == 0) {
      for (int c = 0; c < n_cta; ++c) at = min(at, S->cta_first[c]);
      a.tokens[row] = at;
    }
    return;
  }

  // ---------------- the row's facts ----------------
  if (tid == 0) {
    const double c = 128.0 * 1.4426950408889634074 / static_cast<double>(temp);
    RowFacts f;
    f.c_hi = static_cast<float>(c);
    f.c_lo = static_cast<float>(c - static_cast<double>(f.c_hi));
    // Scaled logits of more than 2^14 lose digits: subtract the maximum first.
    // Logits that still have a weight are then within a factor of two of it,
    // so the difference is exact.
    f.base = fabsf(m) * f.c_hi > 16384.0f ? m : 0.0f;
    f.m = m - f.base;
    f.k0 = __float_as_int(fmaf(f.m, f.c_hi, kMagic)) - 0x4b400000;
    f.cut = static_cast<float>(static_cast<double>(f.m) - kOctaves * 128.0 / c);
    f.fine_from = -INFINITY;
    S->row = f;
  }
  __syncthreads();
  RowFacts f = S->row;
  const bool by_k = top_k > 0 && top_k < a.V, by_p = top_p < 1.0f;

  // sums the cluster's values (one per thread) for everyone
  auto cluster_total = [&](unsigned long long v) -> unsigned long long {
    v = warp_sum64(v);
    if (lane == 0) S->red[warp] = v;
    __syncthreads();
    if (warp == 0) {
      v = warp_sum64(lane < kSmpWarps ? S->red[lane] : 0ull);
      if (lane < n_cta) cluster_ptr(S, lane)->part_w[rank] = v;
    }
    csync();
    unsigned long long t = 0;
    for (int c = 0; c < n_cta; ++c) t += S->part_w[c];
    csync();                                         // part_w may be written again
    return t;
  };

  unsigned long long all_w = 0;                             // weight of the whole row
  unsigned long long mine = 0;                              // of this lane's elements
  if (!by_k) {
    for (int v = v0 + lane; v < v1; v += 32) {
      float x[kVec];
      E::unpack(vec[v], x);
#pragma unroll
      for (int e = 0; e < kVec; ++e) {
        const float z = x[e] - f.base;
        if (z >= f.cut) mine += light_weight(S, f, z);
      }
    }
    const unsigned long long z0 = cluster_total(mine);
    // fine weights from 2^-12 of the total on
    if (tid == 0)
      S->row.fine_from = static_cast<float>(
          static_cast<double>(f.m) +
          (log2(static_cast<double>(z0)) - 45.0 - 12.0) * 128.0 / static_cast<double>(f.c_hi));
    __syncthreads();
    f.fine_from = S->row.fine_from;
    for (int v = v0 + lane; v < v1; v += 32) {
      float x[kVec];
      E::unpack(vec[v], x);
#pragma unroll
      for (int e = 0; e < kVec; ++e) {
        const float z = x[e] - f.base;
        if (z >= f.fine_from && z >= f.cut) mine += fine_weight(f, z) - light_weight(S, f, z);
      }
    }
    if (by_p) all_w = cluster_total(mine);
  }

  // ---------------- selection ----------------
  unsigned long long border = 0;                            // keep keys >= border
  float bin_scale = 0.0f;
  auto bin_of = [&](float z) -> unsigned {
    return __float_as_uint(fmaf(f.m - z, bin_scale, 8388608.0f)) - 0x4b000000u;
  };
  auto build_bins = [&](int octaves) {
    bin_scale = f.c_hi * (static_cast<float>(kSmpBins) / (128.0f * octaves));
    for (int i = tid; i < 4 * kSmpBins; i += kSmpThreads) (&S->hist[0][0])[i] = 0;
    __syncthreads();
    for (int v = v0 + lane; v < v1; v += 32) {
      float x[kVec];
      E::unpack(vec[v], x);
#pragma unroll
      for (int e = 0; e < kVec; ++e) {
        const float z = x[e] - f.base;
        if (z >= f.cut) {
          const unsigned b = bin_of(z);
          if (b < kSmpBins) {
            const unsigned long long w = weight(S, f, z);
            atomicAdd(&S->hist[0][b], 1u);
            atomicAdd(&S->hist[1][b], static_cast<unsigned>(w) & 0x7fffu);
            atomicAdd(&S->hist[2][b], static_cast<unsigned>(w >> 15) & 0x7fffu);
            atomicAdd(&S->hist[3][b], static_cast<unsigned>(w >> 30));
          }
        }
      }
    }
    csync();
    // each CTA adds up a share of the bins, for the leader
    const int share = kSmpBins / kSmpMaxCluster;
    for (int s = rank; s < kSmpMaxCluster; s += n_cta) {
      for (int i = tid; i < share; i += kSmpThreads) {
        const int b = s * share + i;
        unsigned n = 0;
        unsigned long long w = 0;
        for (int c = 0; c < n_cta; ++c) {
          const SampleShared* R = cluster_ptr(S, c);
          n += R->hist[0][b];
          w += R->hist[1][b] + (static_cast<unsigned long long>(R->hist[2][b]) << 15) +
               (static_cast<unsigned long long>(R->hist[3][b]) << 30);
        }
        L->bin_n[b] = n;
        L->bin_w[b] = w;
      }
    }
    csync();
  };
  // the bin in which the bins' sum reaches `target` (counts or weights)
  auto find_bin = [&](unsigned long long target, bool weights) {
    if (rank == 0 && warp == 0) {
      constexpr int kPer = kSmpBins / 32;
      unsigned long long n = 0, w = 0;
      for (int i = 0; i < kPer; ++i) {
        n += S->bin_n[lane * kPer + i];
        w += S->bin_w[lane * kPer + i];
      }
      unsigned long long n_in = n, w_in = w;                // inclusive over lanes
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const unsigned long long pn = __shfl_up_sync(kFull, n_in, o);
        const unsigned long long pw = __shfl_up_sync(kFull, w_in, o);
        if (lane >= o) {
          n_in += pn;
          w_in += pw;
        }
      }
      const unsigned reach = __ballot_sync(kFull, (weights ? w_in : n_in) >= target);
      const unsigned long long total = __shfl_sync(kFull, w_in, 31);
      if (reach == 0) {
        if (lane == 0)
          for (int c = 0; c < n_cta; ++c) {
            cluster_ptr(S, c)->bin = -1;
            cluster_ptr(S, c)->total_w = total;
          }
      } else if (lane == __ffs(reach) - 1) {
        unsigned long long an = n_in - n, aw = w_in - w;
        int b = lane * kPer;
        while (b < lane * kPer + kPer - 1 &&
               (weights ? aw + S->bin_w[b] : an + S->bin_n[b]) < target) {
          an += S->bin_n[b];
          aw += S->bin_w[b];
          ++b;
        }
        for (int c = 0; c < n_cta; ++c) {
          SampleShared* R = cluster_ptr(S, c);
          R->bin = b;
          R->above_n = an;
          R->above_w = aw;
          R->total_w = total;
          R->list_n = 0;
        }
      }
    }
    csync();
  };
  // K* of `target` and the weight of its head, once find_bin has found its bin
  auto resolve = [&](unsigned long long target, bool weights) {
    const unsigned bin = static_cast<unsigned>(S->bin);
    for (int v = v0 + lane; v < v1; v += 32) {
      float x[kVec];
      E::unpack(vec[v], x);
#pragma unroll
      for (int e = 0; e < kVec; ++e) {
        const float z = x[e] - f.base;
        if (z >= f.cut && bin_of(z) == bin) {
          const unsigned at = atomicAdd(&L->list_n, 1u);
          if (at < kSmpList) {
            L->list.key[at] = order_key(x[e], first + v * kVec + e);
            L->list.w[at] = weight(S, f, z);
          }
        }
      }
    }
    csync();
    const unsigned n = L->list_n;
    csync();
    if (n <= kSmpList) {
      if (rank == 0 && tid < n) {
        const unsigned long long key = S->list.key[tid], own = S->list.w[tid];
        unsigned long long hn = S->above_n, hw = S->above_w;   // up to and with this key
        for (unsigned i = 0; i < n; ++i)
          if (S->list.key[i] >= key) {
            ++hn;
            hw += S->list.w[i];
          }
        const bool here = weights ? hw >= target && hw - own < target : hn == target;
        if (here)
          for (int c = 0; c < n_cta; ++c) {
            cluster_ptr(S, c)->border = key;
            cluster_ptr(S, c)->border_w = hw;
          }
      }
      csync();
      return;
    }
    // too many keys in the bin: K* bit by bit, the largest key whose head
    // reaches the target
    unsigned long long key = 0, key_w = 0;
    for (int bit = 63; bit >= 0; --bit) {
      const unsigned long long trial = key | (1ull << bit);
      unsigned long long hn = 0, hw = 0;
      for (int v = v0 + lane; v < v1; v += 32) {
        float x[kVec];
        E::unpack(vec[v], x);
#pragma unroll
        for (int e = 0; e < kVec; ++e) {
          const float z = x[e] - f.base;
          if (z >= f.cut && order_key(x[e], first + v * kVec + e) >= trial) {
            ++hn;
            hw += weight(S, f, z);
          }
        }
      }
      hw = cluster_total(hw);
      if (!weights) hn = cluster_total(hn);
      if ((weights ? hw : hn) >= target) {
        key = trial;
        key_w = hw;
      }
    }
    if (tid == 0) {
      S->border = key;
      S->border_w = key_w;
    }
    __syncthreads();
  };

  if (by_k || by_p) {
    build_bins(kNarrow);
    bool wide = false;
    if (by_k) {
      find_bin(static_cast<unsigned long long>(top_k), false);
      if (S->bin < 0) {
        wide = true;
        build_bins(kOctaves);
        find_bin(static_cast<unsigned long long>(top_k), false);
      }
      if (S->bin >= 0) {
        resolve(static_cast<unsigned long long>(top_k), false);
        border = S->border;
        all_w = S->border_w;
      } else {
        all_w = S->total_w;                                 // all that have a weight
      }
    }
    if (by_p) {
      double want = ceil(static_cast<double>(top_p) * static_cast<double>(all_w));
      unsigned long long target = static_cast<unsigned long long>(want);
      if (target < 1) target = 1;
      if (target > all_w) target = all_w;
      csync();                                       // the results above are read
      find_bin(target, true);
      if (S->bin < 0 && !wide) {
        build_bins(kOctaves);
        find_bin(target, true);
      }
      if (S->bin >= 0) {
        resolve(target, true);
        const unsigned long long b = S->border;
        border = b > border ? b : border;
      }
    }
  }
  if (min_p > 0.0f) {
    // the smallest float z with exp((z - max) / T) >= min_p
    if (tid == 0) {
      const double from = static_cast<double>(m) +
                          static_cast<double>(temp) * log(static_cast<double>(min_p));
      float z = static_cast<float>(from);
      if (static_cast<double>(z) < from) z = nextafterf(z, INFINITY);
      S->red[0] = order_key(fminf(z, m), 0x7fffffff);
    }
    __syncthreads();
    const unsigned long long b = S->red[0];
    border = b > border ? b : border;
    __syncthreads();
  }

  // ---------------- draw ----------------
  const bool filtered = border != 0;
  const unsigned ob = static_cast<unsigned>(border >> 32);
  const float border_z = __uint_as_float((ob & 0x80000000u) ? ob & 0x7fffffffu : ~ob);
  auto kept = [&](float z, int index) {
    return z > border_z || (z == border_z && order_key(z, index) >= border);
  };
  if (filtered || by_k) {
    mine = 0;
    for (int v = v0 + lane; v < v1; v += 32) {
      float x[kVec];
      E::unpack(vec[v], x);
#pragma unroll
      for (int e = 0; e < kVec; ++e)
        if (!filtered || kept(x[e], first + v * kVec + e)) mine += weight(S, f, x[e] - f.base);
    }
  }
  mine = warp_sum64(mine);
  if (lane < n_cta) cluster_ptr(S, lane)->warp_sum[rank * kSmpWarps + warp] = mine;
  csync();
  // the warp in whose run the cumulative weight passes u * total
  constexpr int kPer = kSmpMaxCluster * kSmpWarps / 32;     // runs a lane adds up
  unsigned long long lane_in = 0, upto[kPer];
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    const int x = lane * kPer + i;
    lane_in += x < n_cta * kSmpWarps ? S->warp_sum[x] : 0ull;
    upto[i] = lane_in;
  }
  unsigned long long scan = lane_in;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const unsigned long long p = __shfl_up_sync(kFull, scan, o);
    if (lane >= o) scan += p;
  }
  const unsigned long long total = __shfl_sync(kFull, scan, 31);
  const int self = rank * kSmpWarps + warp;                 // this warp's run
  unsigned long long before = 0;
#pragma unroll
  for (int i = 0; i < kPer; ++i)
    if (i == self % kPer) before = scan - lane_in + upto[i];
  before = __shfl_sync(kFull, before, self / kPer) - mine;
  const unsigned long long target =
      static_cast<unsigned long long>(static_cast<double>(u) * static_cast<double>(total));
  if (before > target || before + mine <= target) return;
  unsigned long long cum = before;
  for (int vb = v0; vb < v1; vb += 32) {
    const int v = vb + lane;
    float x[kVec];
    unsigned long long w[kVec], sum = 0;
    if (v < v1) E::unpack(vec[v], x);
#pragma unroll
    for (int e = 0; e < kVec; ++e) {
      w[e] = 0;
      if (v < v1 && (!filtered || kept(x[e], first + v * kVec + e)))
        w[e] = weight(S, f, x[e] - f.base);
      sum += w[e];
    }
    unsigned long long in = sum;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const unsigned long long p = __shfl_up_sync(kFull, in, o);
      if (lane >= o) in += p;
    }
    const unsigned pass = __ballot_sync(kFull, cum + in > target);
    if (pass != 0) {
      if (lane == __ffs(pass) - 1) {
        unsigned long long c = cum + in - sum;
        int token = -1;
#pragma unroll
        for (int e = 0; e < kVec; ++e) {
          c += w[e];
          if (token < 0 && c > target) token = first + v * kVec + e;
        }
        a.tokens[row] = token;
      }
      return;
    }
    cum += __shfl_sync(kFull, in, 31);
  }
}

pctree_status sample_check(const pctree_sample_config* c) {
  if (c == nullptr) return PCTREE_ERR_INVALID_ARG;
  if (c->rows < 1 || c->V < 1 || c->group < 1 || c->row_stride < c->V)
    return PCTREE_ERR_INVALID_ARG;
  if (c->dtype != PCTREE_F32 && c->dtype != PCTREE_BF16 && c->dtype != PCTREE_F16)
    return PCTREE_ERR_INVALID_ARG;
  if (c->V > kSmpMaxV || c->rows > (1 << 27) || c->row_stride > (1ll << 40))
    return PCTREE_ERR_UNSUPPORTED;
  return PCTREE_OK;
}

}  // namespace
}  // namespace pct

extern "C" {

pctree_status pctree_sample(const pctree_sample_config* cfg, const void* logits,
                            const float* uniform, const float* temperature,
                            const int32_t* top_k, const float* top_p, const float* min_p,
                            const int32_t* n_rows, int32_t* tokens, int32_t* status,
                            void* stream) {
  using namespace pct;
  NvtxRange range("pctree_sample");
  pctree_status st = sample_check(cfg);
  if (st != PCTREE_OK) return st;
  const pctree_sample_config& c = *cfg;
  const int el = c.dtype == PCTREE_F32 ? 4 : 2;
  if (logits == nullptr || uniform == nullptr || tokens == nullptr ||
      (reinterpret_cast<uintptr_t>(logits) & (el - 1)) != 0)
    return PCTREE_ERR_INVALID_ARG;
  int num_sms = 0;
  st = device_facts(&num_sms);
  if (st != PCTREE_OK) return st;
  // CTAs per row: slices of at most 80 KB (two CTAs an SM), and of at least
  // 8 KB
  int ctas = 1;
  while (ctas < kSmpMaxCluster &&
         static_cast<long long>(c.V) * el > ctas * 8192ll)
    ctas *= 2;
  const int vec = 16 / el;
  SampleArgs a{};
  a.slice = ((c.V + ctas - 1) / ctas + vec - 1) / vec * vec;
  ctas = (c.V + a.slice - 1) / a.slice;
  a.logits = logits;
  a.uniform = uniform;
  a.temperature = temperature;
  a.top_k = top_k;
  a.top_p = top_p;
  a.min_p = min_p;
  a.n_rows = n_rows;
  a.tokens = tokens;
  a.status = status;
  a.row_stride = c.row_stride;
  a.V = c.V;
  a.group = c.group;
  const size_t bytes = sizeof(SampleShared) + static_cast<size_t>(a.slice + 2 * vec) * el;
  const void* fn = c.dtype == PCTREE_F32    ? reinterpret_cast<const void*>(sample_kernel<PCTREE_F32>)
                   : c.dtype == PCTREE_BF16 ? reinterpret_cast<const void*>(sample_kernel<PCTREE_BF16>)
                                            : reinterpret_cast<const void*>(sample_kernel<PCTREE_F16>);
  constexpr size_t kMost = sizeof(SampleShared) + (kSmpMaxV / kSmpMaxCluster + 8) * 4;
  static_assert(kMost <= 227 * 1024, "shared memory per CTA");
  static SmemLimit limits[3];
  if (limits[c.dtype].ensure(fn, kMost) != cudaSuccess) return PCTREE_ERR_CUDA;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = static_cast<unsigned>(ctas);
  attr[1].val.clusterDim.y = 1;
  attr[1].val.clusterDim.z = 1;
  cudaLaunchConfig_t lc = {};
  lc.gridDim = dim3(static_cast<unsigned>(c.rows) * ctas);
  lc.blockDim = dim3(kSmpThreads);
  lc.dynamicSmemBytes = bytes;
  lc.stream = static_cast<cudaStream_t>(stream);
  lc.attrs = attr;
  lc.numAttrs = 2;
  void* params[] = {&a};
  return cudaLaunchKernelExC(&lc, fn, params) == cudaSuccess ? PCTREE_OK : PCTREE_ERR_CUDA;
}

}  // extern "C"
