// pctree_sample: the target's token at every row of its logits, from given
// random numbers, with temperature, top-k, top-p and min-p.
//
// Two placements of a row, the same code:
//   cluster  (few rows) a row belongs to up to 16 CTAs, each of which keeps
//            its slice in shared memory: logits are read once, and the CTAs'
//            results meet through distributed shared memory;
//   stream   (many rows) a row belongs to one CTA, which reads it from memory
//            in the first pass and from L2 in the others: no cluster barriers,
//            and as many rows in flight as L2 holds (4096 rows of 151936 bf16
//            logits, mixed filters: 2745 us by clusters, 599 by streams when
//            these came).
//
// Weights w = exp((z - max) / T) are summed as integers in units of 2^-45 of
// the largest weight, so sums are exact and in any order the same.  A token is
// drawn where the cumulative weight passes u * total: with 10^5 borders between
// tokens, a relative error d of the cumulative weights moves one of them past
// the random number in 10^5 d of all rows, so single-precision exponentials
// would miss a token in a few rows of a thousand.  Two forms of the weight:
//   light  2^(n/128) from a table in 31-bit fixed point, times 1 + s, s the
//          rest of at most 1/256 octave by a cubic, whose product is rounded to
//          units of 2^-29: relative error at most 2^-29.4, 2^-31.2 on average,
//          the same for equal logits;
//   fine   the same with every term carried as a float pair: 2^-39.5.
// Tokens above 2^-12 of the total use the fine form (there are at most 4096).  The
// errors of the light ones move a border by at most half of 2^-29.4 of the total
// (all of one sign on one side of it).  Errors of different logits are as good as
// independent: 2^-35 in rows of drawn bf16 logits (some 600 values among 151936), 2^-37
// of f16 or f32 ones, a chance of 10^-6 and 2 10^-7 a row that the random number lies
// between a border and its place.
//
// Selection: every filter keeps a head of the order (z desc, index asc).
//   Few candidates: where a logit is known that nothing kept is below, the
//   logits from it on (a little over top_k of them) are ranked against one
//   another by one CTA, with their exact weights.
//   Else a head is the set of keys K >= K* for K = (z, -index) as one 64-bit
//   integer, K* the largest key whose head reaches a target count (top-k) or
//   weight (top-p): the logits are binned linearly below the maximum, by count
//   and by weight in single precision; the bins that the target can fall in
//   are gathered and ranked on top of the exact sums above them.  Bins too full
//   for that (flat rows, long runs of equal logits) are searched digit by digit,
//   nine bits of the key a pass.
//
// What bounds it (one GB300, us, 4096 streamed rows of 151936 bf16 logits; one
// read of them at the measured copy rate is 184): rows with top-k 50 220 and with
// min-p 209, HBM; plain ones 645, of which the light weights take 400, some 13
// integer instructions a logit at half rate; top-p 0.95 alone 1240, the sum,
// then the bins' atomics and the weights of what is kept.  A single row of f32
// logits takes 26, a chain of passes and barriers of 16 CTAs.
#include "kv_rows.cuh"
#include "sm103_ptx.cuh"

namespace pct {
namespace {

constexpr int kSmpThreads = 512;
constexpr int kSmpWarps = kSmpThreads / 32;
constexpr int kSmpMaxCluster = 16;
constexpr int kSmpAhead = 6;                // vectors of a lane per noted maximum
constexpr int kSmpBins = 512;
constexpr int kSmpList = 512;               // gathered keys of a bin
constexpr int kSmpMaxGroups = 512;          // groups of lanes whose maxima are ranked
constexpr int kSmpCand = 640;               // candidates one CTA can rank
constexpr int kSmpMaxV = 1 << 18;           // sums of 2^45-scaled weights fit 64 bits
constexpr int kOctaves = 46;                // below the largest: weight 0
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

// What a row's passes need, the same in every CTA of its cluster.  Logits are
// taken relative to `base`.
struct RowFacts {
  float c_hi, c_lo;                         // 128 log2(e) / T
  float base;
  float m;                                  // the maximum
  float cut;                                // 46 octaves below: weight 0 from here down
  float fine_from;                          // from it on the fine form
  float min_z;                              // min_p keeps logits (not relative) from it on
  int k;                                    // round(m * 128 log2(e) / T)
};

struct alignas(16) SampleShared {
  uint64_t bar;
  RowFacts row;
  float warp_max[kSmpMaxCluster * kSmpWarps];       // of every warp of the cluster
  float group_max[kSmpMaxGroups];           // of every group of lanes
  float from;                               // logits from it on are candidates
  int cta_first[kSmpMaxCluster];            // lowest index of the maximum (T = 0)
  unsigned cta_n[kSmpMaxCluster];           // candidates of every CTA
  unsigned long long warp_sum[kSmpMaxCluster * kSmpWarps];
  int bin0, bin1;                           // the bins a target can fall in (-1: past all)
  unsigned long long border, border_w;      // K* and the weight of its head
  int found;
  unsigned long long kept_w[kSmpWarps];     // of the list, by the warps of their runs
  unsigned list_n, local_n;
  int run;                                  // the warp whose run holds the token (-1: none)
  unsigned long long run_before;            // the weight before that run
  unsigned long long part[2][kSmpMaxCluster];
  unsigned long long red[kSmpWarps];
  union {
    struct {                                // one CTA's candidates
      unsigned long long key[kSmpCand], w[kSmpCand];
    } cand;
    struct {
      unsigned bin_n[kSmpBins], bin_w[kSmpBins];    // the leader's sum of all CTAs' bins
      union {
        unsigned hist[2][kSmpBins];         // count, weight in 2^-32 of the total
        struct {
          unsigned long long key[kSmpList], w[kSmpList];
          unsigned char owner[kSmpList];    // the warp, of all CTAs'
        } list;
      };
    };
  };
  int pending[kSmpWarps][64];               // a warp's elements, until 32 are together
  uint2 tab[128][16];                       // light table, a column per lane pair
};

template <bool STREAM, typename T>
__device__ __forceinline__ T* cluster_ptr(T* p, int rank) {
  if constexpr (STREAM) {
    return p;
  } else {
    uint64_t r;
    asm volatile("mapa.u64 %0, %1, %2;" : "=l"(r) : "l"(reinterpret_cast<uint64_t>(p)), "r"(rank));
    return reinterpret_cast<T*>(r);
  }
}

// The two halves of csync below.
__device__ __forceinline__ void cluster_arrive() {
  asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
}
__device__ __forceinline__ void cluster_wait() {
  asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}

// Barrier of the row's CTAs, with the warp's lanes together.
template <bool STREAM>
__device__ __forceinline__ void csync() {
  if constexpr (STREAM) {
    __syncthreads();
  } else {
    __syncwarp();
    cluster_sync();
  }
}

// v * 2^(32 - n) cut off, 0 from n = 64 on.
__device__ __forceinline__ unsigned long long high_shifted(uint32_t v, uint32_t n) {
  unsigned long long r;
  asm("{\n\t.reg .b64 t;\n\tmov.b64 t, {%1, %2};\n\tshr.u64 %0, t, %3;\n\t}"
      : "=l"(r) : "r"(0u), "r"(v), "r"(n));
  return r;
}

// Light weights of two logits (relative to base, or -inf) in units of 2^-46,
// cut off: rounded to units of 2^-45 they are (w + 1) / 2.  Logits so far below
// that t leaves [2^23, 2^24) need no clamp: its bits, as an integer, are then
// so far from kMagic's that n shifts all of v out.
__device__ __forceinline__ void light_halves(const SampleShared* S, const RowFacts& f, float x0,
                                             float x1, unsigned long long& w0,
                                             unsigned long long& w1) {
  const uint64_t x = pack2(x0, x1), c = pack2(f.c_hi, f.c_hi);
  const uint64_t t = fma2(x, c, pack2(kMagic, kMagic));
  const uint64_t nk = fma2(t, pack2(-1.0f, -1.0f), pack2(kMagic, kMagic));
  uint64_t r = fma2(x, c, nk);
  r = fma2(x, pack2(f.c_lo, f.c_lo), r);
  constexpr float a2 = kLn2 * kLn2 / 2.0f, a3 = kLn2 * kLn2 * kLn2 / 6.0f;
  uint64_t p = fma2(r, pack2(a3, a3), pack2(a2, a2));
  p = fma2(r, p, pack2(kLn2, kLn2));
  const uint64_t s = mul2(r, p);
  float t0, t1;
  unpack2(t, t0, t1);
  // round(x c) - k <= 0 is -(128 sh - j), sh = ceil of its 128th part, and the
  // table is stored backwards; n = 128 (sh + 17) + 127 - j, for a shift from the
  // upper word
  const uint32_t top = static_cast<uint32_t>(f.k) + 0x4b400000u + 127u + 17u * 128u;
  const uint32_t n0 = top - __float_as_uint(t0), n1 = top - __float_as_uint(t1);
  const uint2 e0 = S->tab[n0 & 127][threadIdx.x & 15], e1 = S->tab[n1 & 127][threadIdx.x & 15];
  float b0, b1;
  unpack2(fma2(pack2(__uint_as_float(e0.y), __uint_as_float(e1.y)), s, pack2(kMagic2, kMagic2)),
          b0, b1);
  const uint32_t v0 = e0.x + (static_cast<uint32_t>(__float_as_int(b0)) << 2);
  const uint32_t v1 = e1.x + (static_cast<uint32_t>(__float_as_int(b1)) << 2);
  w0 = high_shifted(v0, n0 >> 7);
  w1 = high_shifted(v1, n1 >> 7);
}
__device__ __forceinline__ void light_weights(const SampleShared* S, const RowFacts& f, float x0,
                                              float x1, unsigned long long& w0,
                                              unsigned long long& w1) {
  light_halves(S, f, x0, x1, w0, w1);
  w0 = (w0 + 1) >> 1;
  w1 = (w1 + 1) >> 1;
}

__device__ __noinline__ unsigned long long fine_weight(const RowFacts& f, float x) {
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
  const int n = static_cast<int>(kf) - f.k;
  const int j = n & 127;
  const float th = kPow2.hi[j], tl = kPow2.lo[j];
  // (th + tl)(1 + yh + sl) = th + q + rest in units of 2^-45: th's bits, q in units
  // of 2^-30 and what is left (tl yh is up to 2^-32.7; tl sl is below 2^-42)
  const float q = th * yh;
  const int qi = __float2int_rn(q * 1073741824.0f);
  const float rest = fmaf(static_cast<float>(qi), -1.0f / 1073741824.0f, q) +
                     (fmaf(th, yh, -q) + fmaf(th, sl, fmaf(tl, yh, tl)));
  const long long w =
      (static_cast<long long>((__float_as_uint(th) & 0x7fffffu) | 0x800000u) << 22) +
      (static_cast<long long>(qi) << 15) + __float2int_rn(rest * 35184372088832.0f);
  const int sh = -(n >> 7);
  return (static_cast<unsigned long long>(w) + ((1ull << sh) >> 1)) >> sh;
}


// Order (z desc, index asc) as integers, largest first.
__device__ __forceinline__ unsigned long long order_key(float z, int index) {
  const unsigned b = __float_as_uint(z + 0.0f);             // -0 ranks as 0
  const unsigned o = (b & 0x80000000u) ? ~b : b | 0x80000000u;
  return (static_cast<unsigned long long>(o) << 32) | (0xffffffffu - static_cast<unsigned>(index));
}

// x in [0, 1) as a 64-bit fraction (exact from 2^-41 on).
__device__ __forceinline__ unsigned long long fraction64(float x) {
  const unsigned b = __float_as_uint(x);
  const int e = static_cast<int>(b >> 23);
  const unsigned long long m = (b & 0x7fffffu) | 0x800000u;
  return e >= 86 ? m << (e - 86) : e > 62 ? m >> (86 - e) : 0ull;
}
// The smallest weight that reaches p of `all`, and the place of u in `total`.
__device__ __forceinline__ unsigned long long reach_of(float p, unsigned long long all) {
  const unsigned long long f = fraction64(p);
  const unsigned long long t = __umul64hi(f, all) + (f * all != 0 ? 1ull : 0ull);
  return t < 1 ? 1 : t;
}
__device__ __forceinline__ unsigned long long place_of(float u, unsigned long long total) {
  return __umul64hi(fraction64(u), total);
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
  static constexpr int kLowBits = 0;        // of a float that the type has not
  static constexpr int kVec = 4;
  static __device__ __forceinline__ float low() { return -INFINITY; }
  static __device__ __forceinline__ uint4 low_vec() {
    return make_uint4(0xff800000u, 0xff800000u, 0xff800000u, 0xff800000u);
  }
  // the largest of a vector's elements and `m` (NaN if any is)
  using Max = float;
  static __device__ __forceinline__ Max join(Max a, Max b) { return max_nan(a, b); }
  static __device__ __forceinline__ Max none() { return -INFINITY; }
  static __device__ __forceinline__ Max larger(const uint4& v, Max m) {
    m = max_nan(m, __uint_as_float(v.x), __uint_as_float(v.y));
    return max_nan(m, __uint_as_float(v.z), __uint_as_float(v.w));
  }
  static __device__ __forceinline__ float value(Max m) { return m; }
  // the first two elements, which leave the vector
  static __device__ __forceinline__ float2 next2(uint4& v) {
    const float2 x = make_float2(__uint_as_float(v.x), __uint_as_float(v.y));
    v.x = v.z;
    v.y = v.w;
    return x;
  }
  static __device__ __forceinline__ float one(float v) { return v; }
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
  static constexpr int kLowBits = F16 ? 13 : 16;
  static constexpr int kVec = 8;
  static __device__ __forceinline__ uint16_t low() { return F16 ? 0xfc00 : 0xff80; }
  static __device__ __forceinline__ uint4 low_vec() {
    constexpr uint32_t two = F16 ? 0xfc00fc00u : 0xff80ff80u;
    return make_uint4(two, two, two, two);
  }
  // (pairs: even and odd elements)
  using Max = uint32_t;
  static __device__ __forceinline__ Max none() { return low_vec().x; }
  static __device__ __forceinline__ Max max2(Max a, Max b) {
    Max r;
    if constexpr (F16) asm("max.NaN.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    else asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
  }
  static __device__ __forceinline__ Max join(Max a, Max b) { return max2(a, b); }
  static __device__ __forceinline__ Max larger(const uint4& v, Max m) {
    return max2(max2(max2(v.x, v.y), max2(v.z, v.w)), m);
  }
  static __device__ __forceinline__ float value(Max m) {
    const float2 p = unpack16<F16>(m);
    return max_nan(p.x, p.y);
  }
  static __device__ __forceinline__ float2 next2(uint4& v) {
    const float2 x = unpack16<F16>(v.x);
    v.x = v.y;
    v.y = v.z;
    v.z = v.w;
    return x;
  }
  static __device__ __forceinline__ float one(uint16_t v) { return unpack16<F16>(v).x; }
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

// The weights of a lane's logits: the light form of all without branches (so
// that the chains overlap), then the fine form of the few that use it.
template <int N>
__device__ __forceinline__ void weights(const SampleShared* S, const RowFacts& f,
                                        const float (&x)[N], unsigned long long (&w)[N]) {
  bool fine = false;
#pragma unroll
  for (int e = 0; e < N; e += 2) {
    const float z0 = x[e] - f.base, z1 = x[e + 1] - f.base;
    light_weights(S, f, z0, z1, w[e], w[e + 1]);
    fine |= z0 >= f.fine_from || z1 >= f.fine_from;
  }
  if (fine) {
#pragma unroll 1
    for (int e = 0; e < N; ++e) {
      float z = 0.0f;
#pragma unroll
      for (int i = 0; i < N; ++i)
        if (i == e) z = x[i] - f.base;
      if (z >= f.fine_from) {
        const unsigned long long v = fine_weight(f, z);
#pragma unroll
        for (int i = 0; i < N; ++i)
          if (i == e) w[i] = v;
      }
    }
  }
}

__device__ __forceinline__ unsigned long long weight(const SampleShared* S, const RowFacts& f,
                                                     float x) {
  const float z = x - f.base;
  if (z >= f.fine_from) return fine_weight(f, z);
  unsigned long long w, same;
  light_weights(S, f, z, z, w, same);
  return w;
}

static_assert(kSmpBins == kSmpThreads && kSmpMaxV == 1 << 18, "digits: a bin a thread");

// Maxima a lane of a streamed row notes.
__host__ __device__ constexpr int notes_of(int n_vec) {
  return ((n_vec + kSmpWarps - 1) / kSmpWarps + 32 * kSmpAhead - 1) / (32 * kSmpAhead);
}

template <int DT, bool STREAM>
__global__ void __launch_bounds__(kSmpThreads, 2) sample_kernel(SampleArgs a) {
  using E = Elem<DT>;
  using T = typename E::type;
  constexpr int kVec = E::kVec;
  extern __shared__ __align__(16) uint8_t smem[];
  SampleShared* S = reinterpret_cast<SampleShared*>(smem);
  T* data = reinterpret_cast<T*>(smem + sizeof(SampleShared));
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int n_cta = STREAM ? 1 : (a.V + a.slice - 1) / a.slice;       // = the cluster's size
  const int rank = STREAM ? 0 : static_cast<int>(cluster_ctarank());
  const int row = blockIdx.x / n_cta;
  SampleShared* L = cluster_ptr<STREAM>(S, 0);              // the leader's
  pdl_launch_dependents();
  if (tid == 0) {
    mbar_init(&S->bar, 1);
    fence_barrier_init();
    S->list_n = 0;
    S->local_n = 0;
    S->run = -1;
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
  const int pad =
      STREAM ? 0 : static_cast<int>((reinterpret_cast<uintptr_t>(src) & 15u) / sizeof(T));
  const int n_vec = (pad + n_el + kVec - 1) / kVec;
  const int head = pad == 0 ? 0 : min(n_el, kVec - pad);
  const int body = STREAM ? 0 : (n_el - head) / kVec;       // whole vectors
  __syncthreads();
  if constexpr (!STREAM) cluster_arrive();                  // this CTA has started
  if constexpr (!STREAM) {
    if (tid == 0 && body > 0) {
      mbar_arrive_expect_tx(&S->bar, static_cast<uint32_t>(body) * 16u);
      const uint32_t bar = smem_u32(&S->bar);
      const T* from = src + head;
      uint32_t to = smem_u32(data + pad + head);
      for (int left = body; left > 0;) {
        const int v = left < 1024 ? left : 1024;            // 16 KB a copy
        asm volatile(
            "cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, "
            "[%3];" ::"r"(to), "l"(reinterpret_cast<uint64_t>(from)), "r"(v * 16), "r"(bar)
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
  }
  // the row's parameters
  const float temp = a.temperature != nullptr ? a.temperature[g] : 1.0f;
  const int top_k = a.top_k != nullptr ? a.top_k[g] : 0;
  const float top_p = a.top_p != nullptr ? a.top_p[g] : 1.0f;
  const float min_p = a.min_p != nullptr ? a.min_p[g] : 0.0f;
  const float u = a.uniform[row];
  const bool params_ok = (temp == 0.0f || (temp >= 1e-6f && temp <= 1e6f)) && top_p > 0.0f &&
                         min_p >= 0.0f && min_p <= 1.0f && u >= 0.0f && u < 1.0f;
  const bool by_k = top_k > 0 && top_k < a.V, by_p = top_p < 1.0f, by_m = min_p > 0.0f;
  // lanes per group of the maxima that bound the top_k-th logit (0: too many):
  // of G groups in the row, about -G ln(1 - top_k / G) logits reach the
  // top_k-th largest maximum
  int group_lanes = 0;
  if (by_k && temp > 0.0f) {
#pragma unroll
    for (int lanes = 1; lanes <= 32; lanes *= 2) {
      const int groups = n_cta * (kSmpThreads / lanes);
      if (groups <= kSmpMaxGroups &&
          top_k <= (groups <= 128 ? groups / 16 * 15 : groups / 8 * 5))
        group_lanes = lanes;
    }
  }
  const bool few = group_lanes != 0 || (by_m && (!by_k || !by_p));
  const float octave = temp * 0.693147181f;                 // of weight, in logits
  // the scale, and min_p's border below the maximum (one thread: 64-bit
  // arithmetic of a whole CTA would take longer than a pass over the row)
  double c = 1.0, below = 0.0;
  if (tid == 0 && params_ok && temp > 0.0f) {
    c = 128.0 * 1.4426950408889634074 / static_cast<double>(temp);
    if (by_m) below = static_cast<double>(temp) * log(static_cast<double>(min_p));
  }
  auto make_table = [&]() {
    for (int i = tid; i < 128 * 16; i += kSmpThreads) {
      const int q = i >> 4, j = 127 - q;
      S->tab[q][i & 15] = make_uint2(
          kPow2.fix[j] - (static_cast<uint32_t>(__float_as_int(kMagic2)) << 2),
          __float_as_uint(kPow2.hi[j]));
    }
  };
  const bool all_light = temp > 0.0f && !by_k && (by_p || !by_m);   // weights of the whole row
  if (all_light) make_table();
  bool landed = true;
  if (body > 0) {
    volatile int never = 0;
    landed = mbar_wait_bounded(&S->bar, 0, &never, 1000000000ull);
  }
  __syncthreads();
  // each warp has a run of the slice's vectors
  const int per_warp = (n_vec + kSmpWarps - 1) / kSmpWarps;
  const int v0 = min(n_vec, warp * per_warp), v1 = min(n_vec, v0 + per_warp);
  const uint4* vec = STREAM ? reinterpret_cast<const uint4*>(src)
                            : reinterpret_cast<const uint4*>(data);
  const int first = e0 - pad;                               // row index of data[0]
  // fn(vector, row index of its first element) over the lane's vectors, the
  // next load ahead of the work; lanes past the run's end (and those that do not
  // read) get -inf, so the warp stays together.
  auto pass = [&](auto&& fn, bool reads = true) {
    auto load = [&](int v) { return v < v1 && reads ? vec[v] : E::low_vec(); };
    uint4 next = load(v0 + lane);
#pragma unroll 1
    for (int vb = v0; vb < v1; vb += 32) {
      const uint4 now = next;
      next = load(vb + 32 + lane);
      fn(now, first + (vb + lane) * kVec);
    }
  };

  // ---------------- maximum ----------------
  // A streamed row's lanes also note the maxima of kSmpAhead vectors each: later
  // passes for few logits then read only where one is.
  typename E::Max largest = E::none();
  typename E::Max* noted = reinterpret_cast<typename E::Max*>(data) + tid;
  if constexpr (STREAM) {
    int note = 0;
#pragma unroll 1
    for (int vb = v0; vb < v1; vb += 32 * kSmpAhead, note += kSmpThreads) {
      uint4 raw[kSmpAhead];
#pragma unroll
      for (int i = 0; i < kSmpAhead; ++i) {
        const int v = vb + i * 32 + lane;
        raw[i] = v < v1 ? vec[v] : E::low_vec();
      }
      typename E::Max here = E::none();
#pragma unroll
      for (int i = 0; i < kSmpAhead; ++i) here = E::larger(raw[i], here);
      noted[note] = here;
      largest = E::join(largest, here);
    }
  } else {
    pass([&](const uint4& raw, int) { largest = E::larger(raw, largest); });
  }
  float m = E::value(largest);
  if (!landed) m = __int_as_float(0x7fc00000);
  const float m1 = m;
  // pass over at least the vectors with a logit that is wanted (monotone)
  auto sparse_pass = [&](auto&& wanted, auto&& fn) {
    if (!__any_sync(kFull, wanted(m1))) return;             // none in this warp's run
    if constexpr (STREAM) {
      // places (kSmpAhead vectors of a lane) are listed until 30 are known; then
      // each lane loads one vector of each of six
      static_assert(kSmpAhead == 6, "five places a load, six loads");
      int* list = reinterpret_cast<int*>(data) + notes_of(n_vec) * kSmpThreads + warp * 64;
      const int of = lane / 6, at = lane - of * 6;          // lanes 30 and 31: none
      int n = 0;
      auto read = [&]() {
        uint4 raw[6];
        int v[6];
#pragma unroll
        for (int i = 0; i < 6; ++i) {
          const int x = i * 5 + of;
          const int place = of < 5 && x < n ? list[x] : 0;
          v[i] = v0 + ((place >> 5) * kSmpAhead + at) * 32 + (place & 31);
          raw[i] = of < 5 && x < n && v[i] < v1 ? vec[v[i]] : E::low_vec();
        }
#pragma unroll
        for (int i = 0; i < 6; ++i)
          if (i * 5 < n) fn(raw[i], first + v[i] * kVec);
      };
      int note = 0;
#pragma unroll 1
      for (int vb = v0; vb < v1; vb += 32 * kSmpAhead, ++note) {
        const bool hit = wanted(E::value(noted[note * kSmpThreads]));
        const unsigned who = __ballot_sync(kFull, hit);
        if (hit) list[n + __popc(who & ((1u << lane) - 1u))] = note * 32 + lane;
        n += __popc(who);
        __syncwarp();
        while (n >= 30) {
          read();
          const int rest = list[30 + lane];
          __syncwarp();
          list[lane] = rest;
          __syncwarp();
          n -= 30;
        }
      }
      if (n > 0) read();
    } else {
      pass(fn, wanted(m1));
    }
  };
  float mg = m;                                             // of this lane's group
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    m = max_nan(m, __shfl_xor_sync(kFull, m, o));
    if (2 * o == group_lanes) mg = m;
  }
  const float mw = m;                                       // of this warp's run
  // every CTA of the cluster has started before its memory is written
  if constexpr (!STREAM) {
    __syncwarp();
    cluster_wait();
  }
  if (lane < n_cta) cluster_ptr<STREAM>(S, lane)->warp_max[rank * kSmpWarps + warp] = mw;
  const int own_group = group_lanes == 0 ? 0 : (rank * kSmpThreads + tid) / group_lanes;
  if (group_lanes != 0 && group_lanes != 32) {
    for (int r = lane & (group_lanes - 1); r < n_cta; r += group_lanes)
      cluster_ptr<STREAM>(S, r)->group_max[own_group] = mg;
  }
  csync<STREAM>();
  m = -INFINITY;
  for (int i = lane; i < n_cta * kSmpWarps; i += 32) m = max_nan(m, S->warp_max[i]);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) m = max_nan(m, __shfl_xor_sync(kFull, m, o));
  if (!params_ok || !(fabsf(m) < INFINITY)) {
    if (rank == 0 && tid == 0) {
      a.tokens[row] = -1;
      if (a.status != nullptr)
        atomicCAS(a.status, 0, !landed      ? PCTREE_ERR_TIMEOUT
                               : !params_ok ? PCTREE_ERR_INVALID_ARG
                                            : PCTREE_ERR_NONFINITE);
    }
    return;
  }
  if (temp == 0.0f) {                                       // the lowest index of the maximum
    int at = 0x7fffffff;
    sparse_pass([&](float x) { return x == m; }, [&](const uint4& raw, int i0) {
      if (E::value(E::larger(raw, E::none())) != m) return;
      float x[kVec];
      E::unpack(raw, x);
#pragma unroll
      for (int e = 0; e < kVec; ++e)
        if (x[e] == m) at = min(at, i0 + e);
    });
    at = __reduce_min_sync(kFull, at);
    int* best = reinterpret_cast<int*>(S->red);
    if (lane == 0) best[warp] = at;
    __syncthreads();
    if (tid == 0) {
      for (int w = 1; w < kSmpWarps; ++w) at = min(at, best[w]);
      L->cta_first[rank] = at;
    }
    csync<STREAM>();
    if (rank == 0 && tid == 0) {
      for (int r = 0; r < n_cta; ++r) at = min(at, S->cta_first[r]);
      a.tokens[row] = at;
    }
    return;
  }

  // ---------------- the row's facts ----------------
  if (tid == 0) {
    RowFacts f;
    f.c_hi = static_cast<float>(c);
    f.c_lo = static_cast<float>(c - static_cast<double>(f.c_hi));
    // Scaled logits of more than 2^14 lose digits: subtract the maximum first.
    // Logits that still have a weight are then within a factor of two of it,
    // so the difference is exact.
    f.base = fabsf(m) * f.c_hi > 16384.0f ? m : 0.0f;
    f.m = m - f.base;
    f.k = __float_as_int(fmaf(f.m, f.c_hi, kMagic)) - 0x4b400000;
    f.cut = f.m - kOctaves * octave;
    f.fine_from = f.cut;
    f.min_z = -INFINITY;
    if (by_m) {
      // the smallest float z with exp((z - max) / T) >= min_p
      const double from = static_cast<double>(m) + below;
      float z = static_cast<float>(from);
      if (static_cast<double>(z) < from) z = nextafterf(z, INFINITY);
      f.min_z = fminf(z, m);
    }
    S->row = f;
  }
  __syncthreads();
  RowFacts f = S->row;

  // Element `index` of the row (of this CTA's slice).
  auto element = [&](int index) { return E::one(reinterpret_cast<const T*>(vec)[index - first]); };
  // Gathers the elements of the lanes' `hits` (bits, from index i0) until every
  // lane has one, so that little of a warp idles where few are wanted; then
  // fn(element, its index, whether the lane has one) by the whole warp.
  int waiting = 0;
  int* pending = S->pending[warp];
  auto gather = [&](unsigned hits, int i0, auto&& fn) {
    for (;;) {
      const unsigned who = __ballot_sync(kFull, hits != 0);
      if (who == 0) return;
      if (hits != 0) {
        pending[waiting + __popc(who & ((1u << lane) - 1u))] = i0 + __ffs(hits) - 1;
        hits &= hits - 1;
      }
      waiting += __popc(who);
      __syncwarp();
      if (waiting >= 32) {
        fn(element(pending[lane]), pending[lane], true);
        const int rest = pending[32 + lane];
        __syncwarp();
        pending[lane] = rest;
        waiting -= 32;
        __syncwarp();
      }
    }
  };
  auto gather_rest = [&](auto&& fn) {
    const bool have = lane < waiting;
    fn(have ? element(pending[lane]) : -INFINITY, have ? pending[lane] : 0, have);
    waiting = 0;
    __syncwarp();
  };
  // sums the cluster's values (one per thread) for everyone; the next sum but
  // one writes the same words, with a barrier in between
  int sums = 0;
  auto cluster_total = [&](unsigned long long v) -> unsigned long long {
    unsigned long long* part = S->part[sums++ & 1];
    v = warp_sum64(v);
    if (lane == 0) S->red[warp] = v;
    __syncthreads();
    if (warp == 0) {
      v = warp_sum64(lane < kSmpWarps ? S->red[lane] : 0ull);
      if (lane < n_cta) cluster_ptr<STREAM>(part, lane)[rank] = v;
    }
    csync<STREAM>();
    unsigned long long t = 0;
    for (int r = 0; r < n_cta; ++r) t += part[r];
    return t;
  };
  // the weight of the whole row: light weights of all, then the fine form of
  // those above 2^-12 of the total; leaves this lane's sum in `mine`
  unsigned long long all_w = 0, mine = 0;
  auto sum_all = [&]() {
    // two logits at a time: the loop stays in the innermost instruction cache
    // (the sum of rounded weights is the sum of w + (w & 1), halved)
    mine = 0;
    unsigned odd = 0;
    pass([&](uint4 raw, int) {
#pragma unroll 1
      for (int i = 0; i < kVec / 2; ++i) {
        const float2 x = E::next2(raw);
        unsigned long long w0, w1;
        light_halves(S, f, x.x - f.base, x.y - f.base, w0, w1);
        mine += w0 + w1;
        odd += (static_cast<unsigned>(w0) & 1u) + (static_cast<unsigned>(w1) & 1u);
      }
    });
    mine = (mine + odd) >> 1;
    const unsigned long long rough = cluster_total(mine);
    f.fine_from =
        fmaxf(f.cut, f.m + (log2f(static_cast<float>(rough)) - 57.0f) * octave);
    auto more = [&](float x, int, bool have) {
      if (!have) return;
      const float z = x - f.base;
      unsigned long long w0, w1;
      light_weights(S, f, z, z, w0, w1);
      mine += fine_weight(f, z) - w0;
    };
    auto is_fine = [&](float x) { return x - f.base >= f.fine_from; };
    sparse_pass(is_fine, [&](const uint4& raw, int i0) {
      unsigned hits = 0;
      if (is_fine(E::value(E::larger(raw, E::none())))) {
        float x[kVec];
        E::unpack(raw, x);
#pragma unroll
        for (int e = 0; e < kVec; ++e) hits |= (is_fine(x[e]) ? 1u : 0u) << e;
      }
      gather(hits, i0, more);
    });
    gather_rest(more);
    if (by_k || by_p) all_w = cluster_total(mine);          // else the draw adds up
  };
  if (all_light) sum_all();

  // ---------------- few candidates: one CTA alone ----------------
  // A logit that nothing kept is below: min_p's border; for top_k the top_k-th
  // largest of the maxima of disjoint groups, which as many logits reach (a
  // little over top_k of them, while there are more groups than that).
  if (few) {
    float from = -INFINITY;
    if (group_lanes == 32) {
      // every CTA ranks all warps' maxima (16 to 256), 32 to 2 threads each
      const int n = n_cta * kSmpWarps, split = kSmpThreads / n, i = tid / split;
      const float x = i < n ? S->warp_max[i] : -INFINITY;
      int ahead = 0;
      for (int j = tid % split; j < n; j += split) {
        const float y = S->warp_max[j];
        ahead += y > x || (y == x && j < i) ? 1 : 0;
      }
      for (int o = 1; o < split; o <<= 1) ahead += __shfl_xor_sync(kFull, ahead, o);
      if (i < n && tid % split == 0 && ahead == top_k - 1) S->from = x;
      __syncthreads();
      from = S->from;
    } else if (group_lanes != 0) {
      // a group's lanes rank its maximum, for all CTAs
      const int n = n_cta * (kSmpThreads / group_lanes);
      int ahead = 0;
      for (int j = lane & (group_lanes - 1); j < n; j += group_lanes) {
        const float y = S->group_max[j];
        ahead += y > mg || (y == mg && j < own_group) ? 1 : 0;
      }
      for (int o = 1; o < group_lanes; o <<= 1) ahead += __shfl_xor_sync(kFull, ahead, o);
      if ((lane & (group_lanes - 1)) == 0 && ahead == top_k - 1)
        for (int r = 0; r < n_cta; ++r) cluster_ptr<STREAM>(S, r)->from = mg;
      csync<STREAM>();
      from = S->from;
    }
    // (top_p needs the weight of all that top_k leaves)
    if (by_m && (group_lanes == 0 || !by_p)) from = fmaxf(from, f.min_z);
    unsigned mine_n = 0;
    sparse_pass([&](float x) { return x >= from; }, [&](const uint4& raw, int i0) {
      if (E::value(E::larger(raw, E::none())) >= from) {
        float x[kVec];
        E::unpack(raw, x);
        unsigned hits = 0;
#pragma unroll
        for (int e = 0; e < kVec; ++e)
          hits |= (x[e] >= from && x[e] - f.base >= f.cut ? 1u : 0u) << e;
        const unsigned n = __popc(hits);
        if (n != 0) {
          mine_n += n;
          unsigned at = atomicAdd(&L->list_n, n);
#pragma unroll
          for (int e = 0; e < kVec; ++e)
            if ((hits >> e) & 1u) {
              if (at < kSmpCand) L->cand.key[at] = order_key(x[e], i0 + e);
              ++at;
            }
        }
      }
      __syncwarp();
    });
    mine_n = __reduce_add_sync(kFull, mine_n);
    if (lane == 0 && mine_n != 0) atomicAdd(&S->local_n, mine_n);
    __syncthreads();
    if (tid < n_cta) cluster_ptr<STREAM>(S, tid)->cta_n[rank] = S->local_n;
    csync<STREAM>();
    unsigned n = 0;
    for (int r = 0; r < n_cta; ++r) n += S->cta_n[r];
    if (n <= kSmpCand) {
      if (rank != 0) return;
      // threads per candidate (a power of two), so that few are ranked fast
      int split = 1;
      while (split < 32 && n * split * 2 <= kSmpThreads) split *= 2;
      const int per = kSmpThreads / split, sub = tid & (split - 1);
      for (unsigned i = tid; i < n; i += kSmpThreads) {
        const unsigned o = static_cast<unsigned>(S->cand.key[i] >> 32);
        S->cand.w[i] = fine_weight(
            f, __uint_as_float((o & 0x80000000u) ? o & 0x7fffffffu : ~o) - f.base);
      }
      __syncthreads();
      auto over_split = [&](unsigned long long v) {
        for (int o = 1; o < split; o <<= 1) v += __shfl_xor_sync(kFull, v, o);
        return v;
      };
      constexpr int kMine = (kSmpCand + kSmpThreads - 1) / kSmpThreads;
      unsigned hn[kMine];                                   // count and weight of the head
      unsigned long long hw[kMine];                         // that ends at a candidate
#pragma unroll
      for (int t = 0; t < kMine; ++t) {
        const unsigned i = tid / split + t * per;
        const unsigned long long key = i < n ? S->cand.key[i] : ~0ull;
        unsigned long long w = 0;
        unsigned c1 = 0;
        if (t * per < static_cast<int>(n))
          for (unsigned j = sub; j < n; j += split)
            if (S->cand.key[j] >= key) {
              ++c1;
              w += S->cand.w[j];
            }
        hw[t] = over_split(w);
        hn[t] = static_cast<unsigned>(over_split(c1));
      }
      if (by_k) {
        const unsigned last = min(static_cast<unsigned>(top_k), n);
#pragma unroll
        for (int t = 0; t < kMine; ++t)
          if (tid / split + t * per < n && hn[t] == last && sub == 0) S->border_w = hw[t];
        __syncthreads();
        all_w = S->border_w;
      }
      const unsigned long long want = by_p ? reach_of(top_p, all_w) : ~0ull;
      const unsigned long long least = by_m ? order_key(f.min_z, 0x7fffffff) : 0ull;
      unsigned long long own[kMine], sum = 0;
#pragma unroll
      for (int t = 0; t < kMine; ++t) {
        const unsigned i = tid / split + t * per;
        own[t] = i < n ? S->cand.w[i] : 0ull;
        if (i < n && ((by_k && hn[t] > static_cast<unsigned>(top_k)) ||
                      hw[t] - own[t] >= want || S->cand.key[i] < least))
          own[t] = 0;
        if (sub == 0) sum += own[t];
      }
      __syncthreads();                                      // the weights have been read
#pragma unroll
      for (int t = 0; t < kMine; ++t) {
        const unsigned i = tid / split + t * per;
        if (i < n && sub == 0) S->cand.w[i] = own[t];
      }
      sum = warp_sum64(sum);
      if (lane == 0) S->red[warp] = sum;
      __syncthreads();
      unsigned long long total = 0;
#pragma unroll
      for (int w = 0; w < kSmpWarps; ++w) total += S->red[w];
      const unsigned long long target = place_of(u, total);
      // ascending index is descending lower half of the key
#pragma unroll
      for (int t = 0; t < kMine; ++t) {
        const unsigned i = tid / split + t * per;
        const unsigned place = i < n ? static_cast<unsigned>(S->cand.key[i]) : ~0u;
        unsigned long long w = 0;
        if (t * per < static_cast<int>(n))
          for (unsigned j = sub; j < n; j += split)
            if (static_cast<unsigned>(S->cand.key[j]) >= place) w += S->cand.w[j];
        w = over_split(w);
        if (i < n && sub == 0 && w > target && w - own[t] <= target)
          a.tokens[row] = static_cast<int>(0xffffffffu - place);
      }
      return;
    }
    // too many: every CTA selects among its own, below
    csync<STREAM>();
  }

  // ---------------- selection by bins ----------------
  const bool no_total = by_k && !by_p && top_k <= a.V / 8;
  if (!all_light) {
    make_table();
    __syncthreads();
    // a count needs no total; the fine weights of a few kept logits cost less
    // than the light ones of all
    if (no_total) f.fine_from = f.cut;
    else sum_all();
  }
  unsigned long long border = 0;                            // keep keys >= border
  bool summed = !no_total;                                  // `mine` is of what is kept
  if (by_k || by_p) {
    // top-p alone: as many octaves as tokens below them cannot reach half of
    // 1 - top_p of the weight, were all of them that heavy
    const int octaves =
        by_k ? kOctaves
             : max(4, min(kOctaves, 2 + static_cast<int>(ceilf(
                                        45.0f + log2f(static_cast<float>(a.V)) -
                                        log2f((1.0f - top_p) * static_cast<float>(all_w))))));
    const float bin_scale = f.c_hi * (static_cast<float>(kSmpBins) / (128.0f * octaves));
    // 2^23 + the bin of a logit `below` the maximum (monotone; a bin below
    // kSmpBins is above the cut)
    auto place = [&](float below) { return fmaf(below, bin_scale, 8388608.0f); };
    // weights in 2^-31.9 of the total, in single precision: off by at most half
    // a unit a token and 2^-18 of their sum
    // (the exact weights are relative to 2^(k/128), not to the maximum's)
    const float log_total = log2f(static_cast<float>(all_w)) - 45.0f;
    const float scale2 = f.c_hi * (1.0f / 128.0f);
    const float log_unit =
        31.9f - log_total +
        fmaf(f.m, f.c_lo, fmaf(f.m, f.c_hi, -static_cast<float>(f.k))) * (1.0f / 128.0f);
    const unsigned long long unit_total = 4007346184ull;    // 2^31.9
    const unsigned long long slack = (unit_total >> 18) + a.V / 2 + 4096;
    for (int i = tid; i < 2 * kSmpBins; i += kSmpThreads) (&S->hist[0][0])[i] = 0;
    __syncthreads();
    pass([&](const uint4& raw, int) {
      float x[kVec];
      E::unpack(raw, x);
#pragma unroll
      for (int e = 0; e < kVec; ++e) {
        const float below = m - x[e];
        const unsigned b = __float_as_uint(place(below)) - 0x4b000000u;
        if (b < kSmpBins) {
          if (by_p)
            atomicAdd(&S->hist[1][b], __float2uint_rn(ex2_approx(fmaf(below, -scale2, log_unit))));
          if (by_k) atomicAdd(&S->hist[0][b], 1u);
        }
      }
    });
    csync<STREAM>();
    // each CTA adds up a share of the bins, for the leader
    constexpr int share = kSmpBins / 16;
    for (int i = rank * share + tid; i < kSmpBins; i += kSmpThreads) {
      // (a CTA takes every n_cta-th share)
      const int s = i / share;
      if (s % n_cta != rank && !STREAM) continue;
      unsigned n = 0, w = 0;
      for (int r = 0; r < n_cta; ++r) {
        const SampleShared* R = cluster_ptr<STREAM>(S, r);
        n += R->hist[0][i];
        w += R->hist[1][i];
      }
      L->bin_n[i] = n;
      L->bin_w[i] = w;
    }
    csync<STREAM>();
    // the bins in which the head of `target` (a count, or a weight in units)
    // can end, give or take `loose`
    auto find_bins = [&](unsigned long long target, bool by_weight, unsigned long long loose) {
      if (rank == 0 && warp == 0) {
        const unsigned* bins = by_weight ? S->bin_w : S->bin_n;
        unsigned long long base = 0;
        int b0 = -1, b1 = -1;
        for (int b = 0; b < kSmpBins; b += 32) {
          unsigned long long in = bins[b + lane];
#pragma unroll
          for (int o = 1; o < 32; o <<= 1) {
            const unsigned long long p = __shfl_up_sync(kFull, in, o);
            if (lane >= o) in += p;
          }
          in += base;
          const unsigned lo = __ballot_sync(kFull, in + loose >= target);
          const unsigned hi = __ballot_sync(kFull, in >= target + loose);
          if (b0 < 0 && lo != 0) b0 = b + __ffs(lo) - 1;
          if (b1 < 0 && hi != 0) b1 = b + __ffs(hi) - 1;
          base = __shfl_sync(kFull, in, 31);
        }
        if (by_weight && b1 < 0) b1 = kSmpBins - 1;
        if (lane < n_cta) {
          SampleShared* R = cluster_ptr<STREAM>(S, lane);
          R->bin0 = b0;
          R->bin1 = b1;
          R->list_n = 0;
          R->found = 0;
        }
      }
      if (tid < kSmpWarps) S->kept_w[tid] = 0;
      csync<STREAM>();
    };
    // K* of `target` (a count, or an exact weight) and the weight of its head,
    // once its bins are known
    auto resolve = [&](unsigned long long target, bool by_weight) {
      // bin < b0 is above, b0 <= bin <= b1 in the list
      const float to_b0 = 8388608.0f + static_cast<float>(S->bin0);
      const float to_b1 = 8388608.0f + static_cast<float>(S->bin1);
      unsigned long long above_w = 0;
      unsigned above = 0;
      // what the logits of the bins, and those above, are not below: a bin's
      // place, at its upper end
      auto logit_at = [&](float t) { return f.base + (f.m - (t - 8388608.0f) / bin_scale); };
      const float from = logit_at(to_b1 + 1.0f);
      auto more = [&](float x, int index, bool have) {
        const float t = place(m - x);
        if (have && t < to_b0) {
          ++above;
          above_w += weight(S, f, x);
        } else if (have && t <= to_b1) {
          const unsigned at = atomicAdd(&L->list_n, 1u);
          if (at < kSmpList) {
            L->list.key[at] = order_key(x, index);
            L->list.w[at] = weight(S, f, x);
            L->list.owner[at] = static_cast<unsigned char>(rank * kSmpWarps + warp);
          }
        }
        __syncwarp();
      };
      pass([&](const uint4& raw, int i0) {
        float x[kVec];
        E::unpack(raw, x);
        unsigned hits = 0;
#pragma unroll
        for (int e = 0; e < kVec; ++e) hits |= (x[e] >= from ? 1u : 0u) << e;
        gather(hits, i0, more);
      });
      gather_rest(more);
      mine = above_w;
      above_w = cluster_total(above_w);
      const unsigned long long above_n = by_weight ? 0 : cluster_total(above);
      const unsigned n = S->list_n;                         // (the leader's counts)
      if (rank == 0 && n <= kSmpList) {
        // a power of two of threads per key
        int split = 1;
        while (split < 32 && n * split * 2 <= kSmpThreads) split *= 2;
        const unsigned k = tid / split;
        const unsigned long long key = k < n ? S->list.key[k] : ~0ull;
        const unsigned long long own = k < n ? S->list.w[k] : 0ull;
        unsigned long long hn = 0, hw = 0;                  // up to and with this key
        if (k < n)
          for (unsigned i = tid & (split - 1); i < n; i += split)
            if (S->list.key[i] >= key) {
              ++hn;
              hw += S->list.w[i];
            }
        for (int o = 1; o < split; o <<= 1) {
          hn += __shfl_xor_sync(kFull, hn, o);
          hw += __shfl_xor_sync(kFull, hw, o);
        }
        hn += above_n;
        hw += above_w;
        if ((tid & (split - 1)) == 0 && k < n &&
            (by_weight ? hw >= target && hw - own < target : hn == target)) {
          for (int r = 0; r < n_cta; ++r) {
            SampleShared* R = cluster_ptr<STREAM>(S, r);
            R->border = key;
            R->border_w = hw;
            R->found = 1;
          }
        }
        __syncthreads();
        // the weights kept of the list, to the warps whose runs they are of
        if (S->found != 0 && tid < n && S->list.key[tid] >= S->border) {
          const int owner = S->list.owner[tid];
          atomicAdd(&cluster_ptr<STREAM>(S, owner / kSmpWarps)->kept_w[owner % kSmpWarps],
                    S->list.w[tid]);
        }
      }
      csync<STREAM>();
      if (S->found != 0) {
        if (lane == 0) mine += S->kept_w[warp];
        return;
      }
      // Too many keys in the bins (a flat row, or long runs of equal logits): K*
      // by nine bits a pass from the highest, a key as a short number: the order
      // of the logit (without the bits that its type has not) from the bins' end
      // on, and 2^18 - 1 - index
      const float to = logit_at(to_b0 - 1.0f);              // and not above
      auto order_of = [&](float x) {
        return static_cast<unsigned>(order_key(x, 0) >> 32) >> E::kLowBits;
      };
      const unsigned o_end = order_of(from);
      auto in_bins = [&](float x) {
        const float t = place(m - x);
        return t >= to_b0 && t <= to_b1;
      };
      auto short_key = [&](float x, int index) {
        return static_cast<unsigned long long>(order_of(x) - o_end) << 18 |
               static_cast<unsigned>(kSmpMaxV - 1 - index);
      };
      const int bits = 18 + 32 - __clz(order_of(to) - o_end);
      unsigned long long base = by_weight ? above_w : above_n;       // of what is above
      unsigned long long digits = 0;                        // K*'s, so far
#pragma unroll 1
      for (int shift = (bits - 1) / 9 * 9; shift >= 0; shift -= 9) {
        for (int i = tid; i < 2 * kSmpBins; i += kSmpThreads) (&S->hist[0][0])[i] = 0;
        __syncthreads();
        if (tid == 0) {
          S->bin0 = 0;
          S->border_w = base;
        }
        auto add = [&](int d, unsigned long long v) {       // 64 bits in two words
          const unsigned lo = static_cast<unsigned>(v);
          const unsigned old = atomicAdd(&S->hist[0][d], lo);
          atomicAdd(&S->hist[1][d], static_cast<unsigned>(v >> 32) + (old + lo < old ? 1u : 0u));
        };
        auto count = [&](float x, int index, bool have) {
          const unsigned long long key = short_key(x, index);
          const bool in = have && in_bins(x) && (key >> (shift + 9)) == digits;
          const unsigned who = __ballot_sync(kFull, in);
          if (who == 0) return;
          unsigned long long v = 0;
          if (in) v = by_weight ? weight(S, f, x) : 1ull;
          const int d = static_cast<int>(key >> shift) & (kSmpBins - 1);
          const int d0 = __shfl_sync(kFull, d, __ffs(who) - 1);
          if (__any_sync(kFull, in && d != d0)) {
            if (in) add(d, v);
          } else {                                          // one digit: one addition
            v = warp_sum64(v);
            if (lane == 0) add(d0, v);
          }
        };
        pass([&](const uint4& raw, int i0) {
          float x[kVec];
          E::unpack(raw, x);
          unsigned in = 0;
#pragma unroll
          for (int e = 0; e < kVec; ++e) in |= (x[e] >= from && x[e] <= to ? 1u : 0u) << e;
          gather(in, i0, count);
        });
        gather_rest(count);
        csync<STREAM>();
        // the digit with which the target is reached, the same in every CTA
        const int d = kSmpBins - 1 - tid;
        unsigned long long own = 0;
        for (int r = 0; r < n_cta; ++r) {
          const SampleShared* R = cluster_ptr<STREAM>(S, r);
          own += (static_cast<unsigned long long>(R->hist[1][d]) << 32) + R->hist[0][d];
        }
        unsigned long long upto = own;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
          const unsigned long long p = __shfl_up_sync(kFull, upto, o);
          if (lane >= o) upto += p;
        }
        if (lane == 31) S->red[warp] = upto;
        __syncthreads();
        upto += base;
        for (int w = 0; w < warp; ++w) upto += S->red[w];
        if (upto >= target && upto - own < target) {
          S->bin0 = d;
          S->border_w = upto - own;
        }
        csync<STREAM>();
        digits = digits << 9 | static_cast<unsigned>(S->bin0);
        base = S->border_w;
      }
      auto more_kept = [&](float x, int index, bool have) {
        if (have && in_bins(x) && short_key(x, index) >= digits) mine += weight(S, f, x);
      };
      pass([&](const uint4& raw, int i0) {           // the weights kept of the bins
        float x[kVec];
        E::unpack(raw, x);
        unsigned in = 0;
#pragma unroll
        for (int e = 0; e < kVec; ++e) in |= (x[e] >= from && x[e] <= to ? 1u : 0u) << e;
        gather(in, i0, more_kept);
      });
      gather_rest(more_kept);
      above_w = cluster_total(mine);
      if (tid == 0) {
        const unsigned o = (static_cast<unsigned>(digits >> 18) + o_end) << E::kLowBits;
        // (the bits that the type has not are ones in the order of negative logits)
        const unsigned rest = (o & 0x80000000u) != 0 ? 0u : (1u << E::kLowBits) - 1u;
        S->border = static_cast<unsigned long long>(o | rest) << 32 |
                    (0xffffffffu - (kSmpMaxV - 1) + static_cast<unsigned>(digits & (kSmpMaxV - 1)));
        S->border_w = above_w;
      }
      __syncthreads();
    };
    if (by_k) {
      find_bins(static_cast<unsigned long long>(top_k), false, 0);
      if (S->bin1 >= 0) {                                   // else fewer have a weight
        resolve(static_cast<unsigned long long>(top_k), false);
        summed = true;
        border = S->border;
        all_w = S->border_w;
      }
      csync<STREAM>();                                      // the results are read
    }
    if (by_p) {
      const unsigned long long target = reach_of(top_p, all_w);
      // in the bins' units
      const float scaled = static_cast<float>(target) * exp2f(31.9f - log_total - 45.0f);
      find_bins(static_cast<unsigned long long>(scaled), true, slack);
      resolve(target, true);
      const unsigned long long b = S->border;
      border = b > border ? b : border;
    }
  }
  if (by_m) {
    const unsigned long long least = order_key(f.min_z, 0x7fffffff);
    if (least > border) {
      border = least;
      summed = false;
    }
  }

  // ---------------- draw ----------------
  const unsigned ob = static_cast<unsigned>(border >> 32);
  const float border_z = border == 0 ? -INFINITY
                                     : __uint_as_float((ob & 0x80000000u) ? ob & 0x7fffffffu : ~ob);
  auto kept = [&](float z, int index) {
    return z > border_z || (z == border_z && order_key(z, index) >= border);
  };
  if (!summed) {
    mine = 0;
    pass([&](const uint4& raw, int i0) {
      float x[kVec];
      E::unpack(raw, x);
      unsigned keep = 0;
#pragma unroll
      for (int e = 0; e < kVec; ++e) keep |= (kept(x[e], i0 + e) ? 1u : 0u) << e;
      if (!__any_sync(kFull, keep != 0)) return;
      unsigned long long w[kVec];
      weights(S, f, x, w);
#pragma unroll
      for (int e = 0; e < kVec; ++e) mine += (keep >> e) & 1u ? w[e] : 0ull;
    });
  }
  mine = warp_sum64(mine);
  if (lane < n_cta) cluster_ptr<STREAM>(S, lane)->warp_sum[rank * kSmpWarps + warp] = mine;
  csync<STREAM>();
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
  const unsigned long long target = place_of(u, total);
  // that warp's run, divided among the CTA's warps
  if (lane == 0 && before <= target && before + mine > target) {
    S->run = warp;
    S->run_before = before;
  }
  __syncthreads();
  if (S->run < 0) return;
  const int r0 = min(n_vec, S->run * per_warp), r1 = min(n_vec, r0 + per_warp);
  const int part = (r1 - r0 + kSmpWarps - 1) / kSmpWarps;
  const int s0 = min(r1, r0 + warp * part), s1 = min(r1, s0 + part);
  auto kept_weights = [&](int vb, int v1, unsigned long long (&w)[kVec]) {
    const int v = vb + lane;
    float x[kVec];
    E::unpack(v < v1 ? vec[v] : E::low_vec(), x);
    weights(S, f, x, w);
    unsigned long long sum = 0;
#pragma unroll
    for (int e = 0; e < kVec; ++e) {
      if (!kept(x[e], first + v * kVec + e)) w[e] = 0;
      sum += w[e];
    }
    return sum;
  };
  unsigned long long w[kVec], part_w = 0;
  for (int vb = s0; vb < s1; vb += 32) part_w += kept_weights(vb, s1, w);
  part_w = warp_sum64(part_w);
  if (lane == 0) S->red[warp] = part_w;
  __syncthreads();
  unsigned long long cum = S->run_before;
  for (int i = 0; i < warp; ++i) cum += S->red[i];
  if (cum > target || cum + part_w <= target) return;
  for (int vb = s0; vb < s1; vb += 32) {
    const unsigned long long sum = kept_weights(vb, s1, w);
    unsigned long long in = sum;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const unsigned long long p = __shfl_up_sync(kFull, in, o);
      if (lane >= o) in += p;
    }
    const unsigned past = __ballot_sync(kFull, cum + in > target);
    if (past != 0) {
      if (lane == __ffs(past) - 1) {
        unsigned long long at = cum + in - sum;
        int token = -1;
#pragma unroll
        for (int e = 0; e < kVec; ++e) {
          at += w[e];
          if (token < 0 && at > target) token = first + (vb + lane) * kVec + e;
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

// Resident rows of the streamed placement: what a second pass finds in L2.
constexpr size_t kStreamBytes = 104u << 20;

template <int DT, bool STREAM>
const void* sample_fn() {
  return reinterpret_cast<const void*>(sample_kernel<DT, STREAM>);
}
const void* sample_fn(int dtype, bool streamed) {
  return dtype == PCTREE_F32
             ? (streamed ? sample_fn<PCTREE_F32, true>() : sample_fn<PCTREE_F32, false>())
         : dtype == PCTREE_BF16
             ? (streamed ? sample_fn<PCTREE_BF16, true>() : sample_fn<PCTREE_BF16, false>())
             : (streamed ? sample_fn<PCTREE_F16, true>() : sample_fn<PCTREE_F16, false>());
}

// Bytes of a slice with which two CTAs of a cluster placement share an SM.
constexpr size_t kSmpSlice = 228 * 1024 / 2 - 1024 - 64 - sizeof(SampleShared);
constexpr size_t kSampleSmem = sizeof(SampleShared) + (kSmpMaxV / 8 + 8) * 4;
static_assert(kSampleSmem <= 227 * 1024 && kSampleSmem >= 120 * 1024, "shared memory per CTA");

// Whether clusters of 16 CTAs (more than is portable) fit on the current
// device; asked once per device and type.
bool wide_clusters(int dtype) {
  static std::mutex mu;
  static signed char known[64][3];
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return false;
  std::lock_guard<std::mutex> lk(mu);
  signed char& k = known[dev][dtype];
  if (k == 0) {
    const void* fn = sample_fn(dtype, false);
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = 16;
    attr[0].val.clusterDim.y = 1;
    attr[0].val.clusterDim.z = 1;
    cudaLaunchConfig_t lc = {};
    lc.gridDim = dim3(16);
    lc.blockDim = dim3(kSmpThreads);
    lc.dynamicSmemBytes = sizeof(SampleShared) + (kSmpMaxV / 16 + 8) * 4;
    lc.attrs = attr;
    lc.numAttrs = 1;
    int clusters = 0;
    const bool asked =
        cudaFuncSetAttribute(fn, cudaFuncAttributeMaxDynamicSharedMemorySize,
                             static_cast<int>(kSampleSmem)) == cudaSuccess &&
        cudaFuncSetAttribute(fn, cudaFuncAttributeNonPortableClusterSizeAllowed, 1) ==
            cudaSuccess &&
        cudaOccupancyMaxActiveClusters(&clusters, fn, &lc) == cudaSuccess;
    if (!asked) {                                // no answer to keep
      (void)cudaGetLastError();
      return false;
    }
    k = clusters > 0 ? 1 : -1;
  }
  return k > 0;
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
  const int vec = 16 / el;
  const size_t row_bytes = static_cast<size_t>(c.V) * el;
  // streamed: whole 16-byte vectors, (two CTAs an SM, or one) the rows in flight
  // in L2, and rows for 3/5 of the SMs (us, clusters / streams, bf16 logits,
  // plain | top-p 0.95 | top-k 50: 64 rows of 151936 46 / 57 | 87 / 170 | 29 / 26,
  // 96 rows 58 / 58 | 126 / 165 | 36 / 29, 152 rows 79 / 58 | 170 / 171 | 44 / 29;
  // 64 rows of 65536 32 / 38 | 51 / 65 | 26 / 25, 96 rows 41 / 35 | 68 / 68 | 29 /
  // 23; f32 logits and shorter rows cross there too)
  const bool aligned = (reinterpret_cast<uintptr_t>(logits) & 15u) == 0 && c.V % vec == 0 &&
                       (c.row_stride * el) % 16 == 0;
  const int per_sm = row_bytes * 2 * num_sms <= kStreamBytes ? 2 : 1;
  const bool streamed =
      aligned && row_bytes * num_sms <= kStreamBytes && c.rows * 5ll >= num_sms * 3ll;
  // cluster: slices of at least 8 KB, up to eight of them, 16 while the SMs
  // have room (one row of 151936 f32: 35.8 us by eight, 29.9 by 16)
  int ctas = 1;
  SampleArgs a{};
  size_t bytes = sizeof(SampleShared);
  if (streamed) {
    a.slice = c.V;
    bytes += static_cast<size_t>(notes_of(c.V / vec)) * kSmpThreads * 4 + kSmpWarps * 64 * 4;
    // a size that keeps a second CTA off the SM
    if (per_sm == 1 && bytes < 120 * 1024) bytes = 120 * 1024;
  } else {
    const int most = c.rows * 16ll <= num_sms && wide_clusters(c.dtype) ? 16 : 8;
    while (ctas < most && row_bytes > ctas * 8192ull) ctas *= 2;
    // fewer where that keeps all rows on the GPU at once, two CTAs an SM (61
    // rows of 32003 f16 logits: 20 us by eight, 11.3 by four)
    while (ctas > 1 && static_cast<long long>(c.rows) * ctas > 2 * num_sms &&
           row_bytes <= ctas / 2 * kSmpSlice)
      ctas /= 2;
    a.slice = ((c.V + ctas - 1) / ctas + vec - 1) / vec * vec;
    ctas = (c.V + a.slice - 1) / a.slice;
    bytes += static_cast<size_t>(a.slice + 2 * vec) * el;
  }
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
  const void* fn = sample_fn(c.dtype, streamed);
  static SmemLimit limits[2][3];
  if (limits[streamed][c.dtype].ensure(fn, kSampleSmem) != cudaSuccess) return PCTREE_ERR_CUDA;
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
  lc.numAttrs = streamed ? 1 : 2;
  void* params[] = {&a};
  return cudaLaunchKernelExC(&lc, fn, params) == cudaSuccess ? PCTREE_OK : PCTREE_ERR_CUDA;
}

}  // extern "C"
