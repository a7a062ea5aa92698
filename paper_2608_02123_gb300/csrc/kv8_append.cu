// pctree_kv8_append: per-head norms of queries and keys, their rotation, and the
// append of keys and values to an 8-bit cache.
//
// The lanes, angles and loads are those of pctree_kv_append: a head is D/16 lanes
// of a warp, 16 elements each as two 8-element pieces that hold whole rotation
// pairs, and angles are 64-bit fractions of a turn.  What differs is the end: the
// largest magnitude of the block's new rows gives the block's power-of-two scale.
//
// Two kinds of work, each a warp's:
//   rows    a run of a row's heads.  With a scale per slot (scale_block 1) keys
//           and values are among them, since their scale is found in the row.
//   blocks  with larger blocks: a block of one request's new slots, keys or
//           values of the heads that fit a warp.  Its rows are read twice, for
//           the maximum and for the codes (the second time from L1), four rows'
//           loads in flight.  Sines and cosines of a CTA's blocks are found once,
//           in shared memory.  Earlier slots of the request in the block are
//           divided by what their scale has to grow.
//
// What bounds it (one GB300, us): prompts (fp16, blocks of 16, 311 MB) 90, 0.51 of the
// measured copy rate: instructions, with four warps on a quarter of an SM (of 15000
// rows of 16 and 2 x 16 heads in blocks of 16, 89: 20 are the queries, 14 the keys'
// rotation; the same in blocks of one slot, read once, 68); trees (blocks of one, 87
// MB) 31, as the append in 16 bits: the rows a warp takes one after the other.  Angles
// by every warp for its own heads 99.7; blocks by a team of warps that keep their
// rows in registers 99.6, chains 17.0 instead of 14.
#include "kv8.cuh"
#include "sm103_ptx.cuh"

namespace pct {
namespace {

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;
constexpr int kCtas = 2;            // an SM
constexpr int kAhead = 4;           // heads or rows a lane has loads in flight for
constexpr int kBlocks = 32;         // that a CTA takes at once, at most

struct Kv8AppendArgs {
  KvRows rows;
  Kv8Blocks blocks;
  const uint16_t* q;
  const uint16_t* k;
  const uint16_t* v;
  const uint16_t* q_weight;
  const uint16_t* k_weight;
  const double* inv_freq;
  const int32_t* positions;
  uint8_t* cache[2];                // keys, values
  uint8_t* scale[2];
  uint16_t* q_out;
  int32_t* status;
  long long q_stride, k_stride, v_stride;
  int Hq, Hkv, rotary, interleaved;
  int heads;                        // of a row's run: Hq, and 2 Hkv with a scale per slot
  int parts, heads_per_part;        // runs of heads a row is divided into
  int groups;                       // warps that a block's keys (values) take; 0: no blocks
  float eps, rope_scale;
};

struct Kv8AppendShared {
  unsigned long long turn[128];                  // fraction of a turn per position
  alignas(16) float weight[2][128];              // of queries and keys
  int start[PCTREE_KV_MAX_BATCH], end[PCTREE_KV_MAX_BATCH], prefix[PCTREE_KV_MAX_BATCH];
  int upto[PCTREE_KV_MAX_BATCH];                 // blocks of requests 0 .. r
  int blocks;                                    // of all; -1: too many rows
  // a CTA's blocks: their requests, pages (-1: none), first and last new slots
  int r[kBlocks], page[kBlocks], base[kBlocks], first[kBlocks], stop[kBlocks];
};

// Sines and cosines of the blocks' rows, [row][sin, cos][pair].
constexpr int kTableRows = 128;
using AngleTable = float[kTableRows][2][64];

// A lane's share of a head: two pieces of eight elements, two at a time.
struct Piece2 {
  uint64_t a[4], b[4];
};

// The angles of a position for the eight pairs of this lane, found by the warp's
// groups together.
template <int S>
__device__ __forceinline__ void angles(const unsigned long long* turn, long long pos, int s,
                                       int group, float rope_scale, uint64_t (&cs)[4],
                                       uint64_t (&sn)[4]) {
  constexpr int kGroups = 32 / S, kOwn = 8 / kGroups;
  float c_own[kOwn], s_own[kOwn];
#pragma unroll
  for (int e = 0; e < kOwn; ++e) {
    const unsigned long long ph =
        static_cast<unsigned long long>(pos) * turn[8 * s + group * kOwn + e];
    // half turns in [-1, 1)
    const float x = static_cast<float>(static_cast<int>(ph >> 32)) * (1.0f / 2147483648.0f);
    sincospif(x, &s_own[e], &c_own[e]);
    s_own[e] *= rope_scale;
    c_own[e] *= rope_scale;
  }
#pragma unroll
  for (int e = 0; e < 8; e += 2) {
    float c[2], t[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int from = ((e + i) / kOwn) * S + s;
      c[i] = __shfl_sync(kFull, c_own[(e + i) % kOwn], from);
      t[i] = __shfl_sync(kFull, s_own[(e + i) % kOwn], from);
    }
    cs[e / 2] = pack2(c[0], c[1]);
    sn[e / 2] = pack2(t[0], t[1]);
  }
}

__device__ __forceinline__ uint64_t negated2(uint64_t x) { return x ^ 0x8000000080000000ull; }

// (a, b) -> (a cos - b sin, b cos + a sin): the pieces are the pairs' halves, or
// hold whole pairs if interleaved (angles 0..3 in the first, 4..7 in the second).
__device__ __forceinline__ void rotate(Piece2& f, const uint64_t (&cs)[4], const uint64_t (&sn)[4],
                                       bool interleaved) {
  if (interleaved) {
    auto turned = [](uint64_t ab, float c, float t) {
      float x, y;
      unpack2(ab, x, y);
      return fma2(pack2(y, x), pack2(-t, t), mul2(ab, pack2(c, c)));
    };
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      float c, d, t, v;
      unpack2(cs[e / 2], c, d);
      unpack2(sn[e / 2], t, v);
      f.a[e] = turned(f.a[e], (e & 1) ? d : c, (e & 1) ? v : t);
      unpack2(cs[2 + e / 2], c, d);
      unpack2(sn[2 + e / 2], t, v);
      f.b[e] = turned(f.b[e], (e & 1) ? d : c, (e & 1) ? v : t);
    }
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const uint64_t p = f.a[e];
      f.a[e] = fma2(f.b[e], negated2(sn[e]), mul2(p, cs[e]));
      f.b[e] = fma2(p, sn[e], mul2(f.b[e], cs[e]));
    }
  }
}

template <bool F16>
__device__ __forceinline__ Piece2 widened(const uint4& x0, const uint4& x1) {
  Piece2 f;
  const uint32_t w0[4] = {x0.x, x0.y, x0.z, x0.w}, w1[4] = {x1.x, x1.y, x1.z, x1.w};
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const float2 lo = unpack16<F16>(w0[e]), hi = unpack16<F16>(w1[e]);
    f.a[e] = pack2(lo.x, lo.y);
    f.b[e] = pack2(hi.x, hi.y);
  }
  return f;
}

// The sum over a head of the squares of this lane's elements (all lanes call it).
template <int S>
__device__ __forceinline__ float head_square(const Piece2& f) {
  uint64_t sum2 = 0;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    sum2 = fma2(f.a[e], f.a[e], sum2);
    sum2 = fma2(f.b[e], f.b[e], sum2);
  }
  float sum, odd;
  unpack2(sum2, sum, odd);
  sum += odd;
#pragma unroll
  for (int o = S / 2; o > 0; o >>= 1) sum += __shfl_xor_sync(kFull, sum, o);
  return sum;
}

__device__ __forceinline__ void scaled(Piece2& f, float inv, const float* w0, const float* w1) {
  const uint64_t inv2 = pack2(inv, inv);
  const ulonglong2* g0 = reinterpret_cast<const ulonglong2*>(w0);
  const ulonglong2* g1 = reinterpret_cast<const ulonglong2*>(w1);
#pragma unroll
  for (int e = 0; e < 4; e += 2) {
    const ulonglong2 p = g0[e / 2], q = g1[e / 2];
    f.a[e] = mul2(mul2(f.a[e], inv2), p.x);
    f.a[e + 1] = mul2(mul2(f.a[e + 1], inv2), p.y);
    f.b[e] = mul2(mul2(f.b[e], inv2), q.x);
    f.b[e + 1] = mul2(mul2(f.b[e + 1], inv2), q.y);
  }
}

// Turns what is not finite into NaN (whose code is NaN) and returns the largest
// finite magnitude; `bad` is set if there is any.
__device__ __forceinline__ float finite_top(Piece2& f, bool& bad) {
  const uint64_t minus1 = pack2(-1.0f, -1.0f);
  float top = 0.0f;
  uint64_t any = 0;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    uint64_t& x = e < 4 ? f.a[e & 3] : f.b[e & 3];
    const uint64_t t = fma2(x, minus1, x);       // 0, or NaN
    any = add2(any, t);
    x = add2(x, t);
    float lo, hi;
    unpack2(x, lo, hi);
    top = fmaxf(top, fmaxf(fabsf(lo), fabsf(hi)));   // (NaN is dropped)
  }
  float a0, a1;
  unpack2(any, a0, a1);
  bad = bad || !(a0 == 0.0f && a1 == 0.0f);
  return top;
}

template <bool F16>
__device__ __forceinline__ uint4 narrowed(const uint64_t (&f)[4]) {
  uint32_t w[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    float lo, hi;
    unpack2(f[e], lo, hi);
    w[e] = pack16<F16>(lo, hi);
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}

// A piece's codes, `by` the reciprocal of the scale.
__device__ __forceinline__ uint2 coded(const uint64_t (&f)[4], float by) {
  const uint64_t by2 = pack2(by, by);
  uint32_t w[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    float lo, hi;
    unpack2(mul2(f[e], by2), lo, hi);
    w[e] = codes2(lo, hi);
  }
  return make_uint2(w[0] | w[1] << 16, w[2] | w[3] << 16);
}

template <bool F16, int D>
__global__ void __launch_bounds__(kThreads, kCtas) kv8_append_kernel(Kv8AppendArgs a) {
  constexpr int S = D / 16;                      // lanes per head
  constexpr int kGroups = 32 / S;                // heads side by side in a warp
  __shared__ Kv8AppendShared sh;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int s = lane % S, group = lane / S;
  const int half = a.rotary / 2;
  pdl_launch_dependents();
  pdl_wait();
  auto report = [&](int code) {
    if (a.status != nullptr) atomicCAS(a.status, 0, code);
  };
  for (int i = half + threadIdx.x; i < 128; i += kThreads) sh.turn[i] = 0;
  for (int i = threadIdx.x; i < 2 * D; i += kThreads) {
    const uint16_t* w = i < D ? a.q_weight : a.k_weight;
    const int d = i < D ? i : i - D;
    sh.weight[i < D ? 0 : 1][d] = w != nullptr ? unpack16<F16>(w[d]).x : 1.0f;
  }
  for (int i = threadIdx.x; i < half; i += kThreads) {
    double t = a.inv_freq[i] * 0.15915494309189533577;   // 1 / (2 pi)
    if (!(fabs(t) < INFINITY)) {
      t = 0.0;
      if (blockIdx.x == 0) report(PCTREE_ERR_INVALID_ARG);
    }
    // the fraction in [-0.5, 0.5] as a signed 64-bit integer, twice over
    sh.turn[i] =
        static_cast<unsigned long long>(__double2ll_rn((t - rint(t)) * 9223372036854775808.0)) << 1;
  }
  // number of the block that holds a slot, over all pages of a request
  auto block_of = [&](int slot) {
    const int entry = div_by(slot, a.blocks.page);
    return entry * a.blocks.per_page + ((slot - entry * a.rows.page_size) >> a.blocks.shift);
  };
  for (int r = threadIdx.x; r < a.rows.batch; r += kThreads) {
    const int start = a.rows.row_start[r], n = a.rows.n_rows[r], prefix = a.rows.prefix_len[r];
    const bool ok = kv_request_ok(a.rows, start, n, prefix);
    if (!ok && blockIdx.x == 0) report(PCTREE_ERR_INVALID_ARG);
    sh.start[r] = start;
    sh.end[r] = ok ? start + n : start;
    sh.prefix[r] = prefix;
    sh.upto[r] = ok && n > 0 ? block_of(prefix + n - 1) - block_of(prefix) + 1 : 0;
  }
  __syncthreads();
  if (a.groups > 0) {
    if (warp == 0) {
      int base = 0;
      long long rows = 0;
      for (int r0 = 0; r0 < a.rows.batch; r0 += 32) {
        const int r = r0 + lane;
        int w = r < a.rows.batch ? sh.upto[r] : 0;
        rows += r < a.rows.batch ? sh.end[r] - sh.start[r] : 0;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
          const int p = __shfl_up_sync(kFull, w, o);
          if (lane >= o) w += p;
        }
        if (r < a.rows.batch) sh.upto[r] = base + w;
        base += __shfl_sync(kFull, w, 31);
      }
      // more rows than there are: requests overlap, and their blocks may be more
      // than an int counts
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) rows += __shfl_xor_sync(kFull, rows, o);
      if (lane == 0) sh.blocks = rows > a.rows.total_rows ? -1 : base;
    }
    __syncthreads();
    if (sh.blocks < 0) {
      if (blockIdx.x == 0 && threadIdx.x == 0) report(PCTREE_ERR_INVALID_ARG);
      return;
    }
  }
  const long long blocks = a.groups > 0 ? sh.blocks : 0;
  const bool rotated = s < a.rotary / 16;
  const int c0 = rotated && !a.interleaved ? s : 2 * s;
  const int c1 = rotated && !a.interleaved ? s + a.rotary / 16
                                           : 2 * s + 1;
  // (dims past rotary_dim: pieces 2 s and 2 s + 1 lie past it, since
  // s >= rotary_dim / 16)
  const long long row_items = static_cast<long long>(a.rows.total_rows) * a.parts;
  bool bad = false;                              // a key or value is not finite
  for (long long item = static_cast<long long>(blockIdx.x) * kWarps + warp; item < row_items;
       item += static_cast<long long>(gridDim.x) * kWarps) {
    // ---------------- a run of a row's heads ----------------
    const int row = static_cast<int>(item / a.parts);
    const int part = static_cast<int>(item - static_cast<long long>(row) * a.parts);
    int r = -1;
    for (int b = 0; b < a.rows.batch; b += 32) {
      const int x = b + lane;
      const unsigned in = __ballot_sync(
          kFull, x < a.rows.batch && row >= sh.start[x] && row < sh.end[x]);
      if (in != 0) {
        r = b + __ffs(in) - 1;
        break;
      }
    }
    if (r < 0) continue;                       // a row of no request
    const int h_end = min(a.heads, (part + 1) * a.heads_per_part);
    const uint16_t* q_row = a.q + row * a.q_stride;
    const uint16_t* k_row = a.k + row * a.k_stride;
    const uint16_t* v_row = a.v + row * a.v_stride;
    uint4 x0[kAhead], x1[kAhead];
    auto load = [&](int hb) {
#pragma unroll
      for (int u = 0; u < kAhead; ++u) {
        const int h = hb + u * kGroups + group;
        const bool is_v = h >= a.Hq + a.Hkv;
        const uint16_t* src = h < a.Hq ? q_row + h * D
                              : !is_v  ? k_row + (h - a.Hq) * D
                                       : v_row + (h - a.Hq - a.Hkv) * D;
        if (h < h_end) {
          x0[u] = *reinterpret_cast<const uint4*>(src + (is_v ? 2 * s : c0) * 8);
          x1[u] = *reinterpret_cast<const uint4*>(src + (is_v ? 2 * s + 1 : c1) * 8);
        } else {
          x0[u] = x1[u] = make_uint4(0, 0, 0, 0);
        }
      }
    };
    // the first heads are under way while the place and the angles are found
    load(part * a.heads_per_part);
    const int slot = sh.prefix[r] + row - sh.start[r];
    int page = 0, off = 0;
    if (a.groups == 0) {
      const int entry = div_by(slot, a.blocks.page);
      off = slot - entry * a.rows.page_size;
      page = kv_page(a.rows, r, entry);
      if (page < 0 && lane == 0) report(PCTREE_ERR_INVALID_ARG);
    }
    const long long place = (static_cast<long long>(page) * a.rows.page_size + off) * a.Hkv;
    uint64_t cs[4], sn[4];
    if (a.rotary > 0)
      angles<S>(sh.turn, a.positions != nullptr ? a.positions[row] : slot, s, group,
                a.rope_scale, cs, sn);
    // every lane runs the same number of rounds: the reductions are warp-wide
    for (int hb = part * a.heads_per_part;;) {
#pragma unroll
      for (int u = 0; u < kAhead; ++u) {
        const int h = hb + u * kGroups + group;
        const bool is_q = h < a.Hq, is_v = h >= a.Hq + a.Hkv;
        Piece2 f = widened<F16>(x0[u], x1[u]);
        const float sum = head_square<S>(f);
        if (!is_v) {
          if ((is_q ? a.q_weight : a.k_weight) != nullptr)
            scaled(f, rsqrtf(sum * (1.0f / D) + a.eps), &sh.weight[is_q ? 0 : 1][c0 * 8],
                   &sh.weight[is_q ? 0 : 1][c1 * 8]);
          if (rotated) rotate(f, cs, sn, a.interleaved != 0);
        }
        if (a.groups == 0) {                   // (the reductions are warp-wide)
          const bool code = !is_q && h < h_end && page >= 0;
          bool odd = false;
          float top = is_q ? 0.0f : finite_top(f, odd);
#pragma unroll
          for (int o = S / 2; o > 0; o >>= 1)
            top = fmaxf(top, __shfl_xor_sync(kFull, top, o));
          if (code) {
            const int kv = is_v ? 1 : 0, hk = h - a.Hq - kv * a.Hkv;
            const int e = least_exp(top);
            const float by = exp2_of(-e);
            uint8_t* dst = a.cache[kv] + (place + hk) * D;
            *reinterpret_cast<uint2*>(dst + (is_v ? 2 * s : c0) * 8) = coded(f.a, by);
            *reinterpret_cast<uint2*>(dst + (is_v ? 2 * s + 1 : c1) * 8) = coded(f.b, by);
            if (s == 0) a.scale[kv][place + hk] = static_cast<uint8_t>(e + kExpBias);
            bad = bad || odd;
          }
        }
        if (is_q && h < h_end) {
          uint16_t* dst = a.q_out + (static_cast<size_t>(row) * a.Hq + h) * D;
          *reinterpret_cast<uint4*>(dst + c0 * 8) = narrowed<F16>(f.a);
          *reinterpret_cast<uint4*>(dst + c1 * 8) = narrowed<F16>(f.b);
        }
      }
      hb += kGroups * kAhead;
      if (hb >= h_end) break;
      load(hb);
    }
  }
  // ---------------- keys or values of blocks ----------------
  // as many at a time as give every CTA some, and as the table holds
  extern __shared__ float4 dynamic[];
  AngleTable& table = *reinterpret_cast<AngleTable*>(dynamic);
  const int block_slots = 1 << a.blocks.shift;
  const int nb = static_cast<int>(
      min(static_cast<long long>(min(kBlocks, kTableRows >> a.blocks.shift)),
          max(1ll, (blocks + gridDim.x - 1) / gridDim.x)));
  for (long long b_first = static_cast<long long>(blockIdx.x) * nb; b_first < blocks;
       b_first += static_cast<long long>(gridDim.x) * nb) {
    const int here = static_cast<int>(min(static_cast<long long>(nb), blocks - b_first));
    __syncthreads();                             // the blocks before are done
    if (threadIdx.x < here) {
      const int nth = static_cast<int>(b_first) + threadIdx.x;
      int lo = 0, hi = a.rows.batch - 1;         // the request that holds it
      while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (sh.upto[mid] <= nth) lo = mid + 1; else hi = mid;
      }
      const int prefix = sh.prefix[lo], last = prefix + sh.end[lo] - sh.start[lo];
      const int block = block_of(prefix) + nth - (lo > 0 ? sh.upto[lo - 1] : 0);
      const int entry = block / a.blocks.per_page;
      const int base = entry * a.rows.page_size +
                       ((block - entry * a.blocks.per_page) << a.blocks.shift);
      const int page = kv_page(a.rows, lo, entry);
      if (page < 0) report(PCTREE_ERR_INVALID_ARG);
      sh.r[threadIdx.x] = lo;
      sh.page[threadIdx.x] = page;
      sh.base[threadIdx.x] = base;
      sh.first[threadIdx.x] = max(base, prefix);
      sh.stop[threadIdx.x] =
          min(min(base + block_slots, (entry + 1) * a.rows.page_size), last);
    }
    __syncthreads();
    if (a.rotary > 0) {
      for (int i = threadIdx.x; i < (here << a.blocks.shift) * half; i += kThreads) {
        const int row = i / half, pair = i - row * half;
        const int b = row >> a.blocks.shift, slot = sh.base[b] + (row & (block_slots - 1));
        if (slot < sh.first[b] || slot >= sh.stop[b]) continue;
        const int r = sh.r[b];
        const long long pos = a.positions != nullptr
                                  ? a.positions[sh.start[r] + slot - sh.prefix[r]] : slot;
        const unsigned long long ph = static_cast<unsigned long long>(pos) * sh.turn[pair];
        float sine, cosine;                      // (half turns in [-1, 1))
        sincospif(static_cast<float>(static_cast<int>(ph >> 32)) * (1.0f / 2147483648.0f), &sine,
                  &cosine);
        table[row][0][pair] = sine * a.rope_scale;
        table[row][1][pair] = cosine * a.rope_scale;
      }
      __syncthreads();
    }
    for (int task = warp; task < here * 2 * a.groups; task += kWarps) {
      const int b = task / (2 * a.groups), part = task - b * 2 * a.groups;
      const int kv = part >= a.groups ? 1 : 0, g = part - kv * a.groups;
      const int page = sh.page[b];
      if (page < 0) continue;
      const int r = sh.r[b], base = sh.base[b], first = sh.first[b], stop = sh.stop[b];
      const int prefix = sh.prefix[r];
      const int entry = div_by(base, a.blocks.page), page0 = entry * a.rows.page_size;
      const int hk = g * kGroups + group;
      const bool mine = hk < a.Hkv;
      const int b0 = kv ? 2 * s : c0, b1 = kv ? 2 * s + 1 : c1;
      const uint16_t* src = (kv ? a.v : a.k) + hk * D;
      const long long stride = kv ? a.v_stride : a.k_stride;
      const int row0 = sh.start[r] - prefix;     // row of slot 0
      const bool norm = kv == 0 && a.k_weight != nullptr, turn = kv == 0 && rotated;
      float top = 0.0f;
      int e = 0;
      uint8_t* dst = a.cache[kv] +
                     (static_cast<long long>(page) * a.rows.page_size * a.Hkv + hk) * D;
      uint8_t* scale = a.scale[kv] +
                       (static_cast<long long>(page) * a.blocks.per_page +
                        ((base - page0) >> a.blocks.shift)) * a.Hkv + hk;
      // the largest magnitude, then the codes
#pragma unroll 1
      for (int pass = 0; pass < 2; ++pass) {
#pragma unroll 1
        for (int x = first; x < stop; x += kAhead) {
          uint4 x0[kAhead], x1[kAhead];
#pragma unroll
          for (int u = 0; u < kAhead; ++u) {
            if (mine && x + u < stop) {
              const uint16_t* p = src + (row0 + x + u) * stride;
              x0[u] = *reinterpret_cast<const uint4*>(p + b0 * 8);
              x1[u] = *reinterpret_cast<const uint4*>(p + b1 * 8);
            } else {
              x0[u] = x1[u] = make_uint4(0, 0, 0, 0);
            }
          }
#pragma unroll
          for (int u = 0; u < kAhead; ++u) {
            if (x + u >= stop) break;            // (the same for the whole warp)
            Piece2 f = widened<F16>(x0[u], x1[u]);
            if (norm)
              scaled(f, rsqrtf(head_square<S>(f) * (1.0f / D) + a.eps), &sh.weight[1][c0 * 8],
                     &sh.weight[1][c1 * 8]);
            if (turn) {
              const auto& angle = table[(b << a.blocks.shift) + x + u - base];
              uint64_t cs[4], sn[4];
#pragma unroll
              for (int i = 0; i < 4; i += 2) {
                const ulonglong2 q = *reinterpret_cast<const ulonglong2*>(&angle[0][8 * s + 2 * i]);
                const ulonglong2 c = *reinterpret_cast<const ulonglong2*>(&angle[1][8 * s + 2 * i]);
                sn[i] = q.x;
                sn[i + 1] = q.y;
                cs[i] = c.x;
                cs[i + 1] = c.y;
              }
              rotate(f, cs, sn, a.interleaved != 0);
            }
            bool odd = false;
            const float t = finite_top(f, odd);
            if (pass == 0) {
              top = fmaxf(top, t);
              bad = bad || (mine && odd);
            } else if (mine) {
              const float by = exp2_of(-e);
              uint8_t* to = dst + static_cast<long long>(x + u - page0) * a.Hkv * D;
              *reinterpret_cast<uint2*>(to + b0 * 8) = coded(f.a, by);
              *reinterpret_cast<uint2*>(to + b1 * 8) = coded(f.b, by);
            }
          }
        }
        if (pass == 1) break;
#pragma unroll
        for (int o = S / 2; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(kFull, top, o));
        e = least_exp(top);
        if (base < prefix && mine) {
          // earlier slots of the request: their scale stays or grows
          const int old = scale_exp(*scale);
          e = max(e, old);
          if (e > old) {
            const float by = exp2_of(old - e);
            for (int x = base; x < prefix; ++x) {
              uint4* p = reinterpret_cast<uint4*>(
                  dst + static_cast<long long>(x - page0) * a.Hkv * D + s * 16);
              *p = rescaled16(*p, by);
            }
          }
        }
        __syncwarp();                            // all lanes have read the scale
        if (mine && s == 0) *scale = static_cast<uint8_t>(e + kExpBias);
      }
    }
  }
  if (__any_sync(kFull, bad) && lane == 0) report(PCTREE_ERR_NONFINITE);
}

pctree_status append8_check(const pctree_kv8_append_config* c) {
  if (c == nullptr) return PCTREE_ERR_INVALID_ARG;
  if (c->Hq < 0 || c->D < 1 || c->rotary_dim < 0 || c->rotary_dim > c->D ||
      c->rotary_dim % 16 != 0 || (c->interleaved != 0 && c->interleaved != 1) ||
      !(c->eps >= 0.0f) || !(c->eps < 1e30f) || !(c->rope_scale > -1e30f) ||
      !(c->rope_scale < 1e30f))
    return PCTREE_ERR_INVALID_ARG;
  const pctree_status st = kv_check(c->batch, c->total_rows, c->Hkv, c->page_size, c->n_pages,
                                    c->max_pages, c->dtype);
  if (st != PCTREE_OK) return st;
  if (!kv8_block_ok(c->scale_block)) return PCTREE_ERR_INVALID_ARG;
  if ((c->D != 64 && c->D != 128) || c->Hq > 65535) return PCTREE_ERR_UNSUPPORTED;
  const int64_t most = 1ll << 40;
  if (c->k_stride % 8 != 0 || c->v_stride % 8 != 0 || c->q_stride % 8 != 0 ||
      c->k_stride < static_cast<int64_t>(c->Hkv) * c->D ||
      c->v_stride < static_cast<int64_t>(c->Hkv) * c->D ||
      c->q_stride < static_cast<int64_t>(c->Hq) * c->D || c->k_stride > most ||
      c->v_stride > most || c->q_stride > most)
    return PCTREE_ERR_INVALID_ARG;
  return PCTREE_OK;
}

// The kernel, ready to be launched with the table; NULL if it cannot be.
template <bool F16, int D>
const void* append8_kernel() {
  static SmemLimit limit;
  const void* fn = reinterpret_cast<const void*>(kv8_append_kernel<F16, D>);
  return limit.ensure(fn, sizeof(AngleTable)) == cudaSuccess ? fn : nullptr;
}

}  // namespace
}  // namespace pct

extern "C" {

pctree_status pctree_kv8_append(const pctree_kv8_append_config* cfg, const void* q, const void* k,
                                const void* v, const void* q_weight, const void* k_weight,
                                const double* inv_freq, const int32_t* positions,
                                const int32_t* row_start, const int32_t* n_rows,
                                const int32_t* prefix_len, const int32_t* page_table,
                                void* k_cache, void* v_cache, void* k_scale, void* v_scale,
                                void* q_out, int32_t* status, void* stream) {
  using namespace pct;
  NvtxRange range("pctree_kv8_append");
  pctree_status st = append8_check(cfg);
  if (st != PCTREE_OK) return st;
  const pctree_kv8_append_config& c = *cfg;
  if (k == nullptr || v == nullptr || k_cache == nullptr || v_cache == nullptr ||
      k_scale == nullptr || v_scale == nullptr || row_start == nullptr || n_rows == nullptr ||
      prefix_len == nullptr || (c.Hq > 0 && (q == nullptr || q_out == nullptr)) ||
      (c.rotary_dim > 0 && inv_freq == nullptr) || !kv_al16(q) || !kv_al16(k) || !kv_al16(v) ||
      !kv_al16(q_weight) || !kv_al16(k_weight) || !kv_al16(k_cache) || !kv_al16(v_cache) ||
      !kv_al16(q_out) || (reinterpret_cast<uintptr_t>(inv_freq) & 7u) != 0 ||
      !kv_table_ok(page_table, c.batch, c.n_pages, c.max_pages))
    return PCTREE_ERR_INVALID_ARG;
  if (c.Hq > 0) {
    // rows are written while others are still read
    const size_t el = 2, n = static_cast<size_t>(c.total_rows);
    const char* o0 = static_cast<const char*>(q_out);
    const char* o1 = o0 + n * c.Hq * c.D * el;
    const struct { const void* p; int64_t stride; int heads; } in[3] = {
        {q, c.q_stride, c.Hq}, {k, c.k_stride, c.Hkv}, {v, c.v_stride, c.Hkv}};
    for (const auto& t : in) {
      const char* p0 = static_cast<const char*>(t.p);
      const char* p1 =
          p0 + ((n - 1) * static_cast<size_t>(t.stride) + static_cast<size_t>(t.heads) * c.D) * el;
      if (p0 < o1 && o0 < p1) return PCTREE_ERR_INVALID_ARG;
    }
  }
  int num_sms = 0;
  st = device_facts(&num_sms);
  if (st != PCTREE_OK) return st;
  Kv8AppendArgs a{};
  a.rows = {row_start, n_rows, prefix_len, page_table, c.batch, c.total_rows,
            c.page_size, c.n_pages, c.max_pages};
  a.blocks = kv8_blocks(c.page_size, c.scale_block);
  a.q = static_cast<const uint16_t*>(q);
  a.k = static_cast<const uint16_t*>(k);
  a.v = static_cast<const uint16_t*>(v);
  a.q_weight = static_cast<const uint16_t*>(q_weight);
  a.k_weight = static_cast<const uint16_t*>(k_weight);
  a.inv_freq = inv_freq;
  a.positions = positions;
  a.cache[0] = static_cast<uint8_t*>(k_cache);
  a.cache[1] = static_cast<uint8_t*>(v_cache);
  a.scale[0] = static_cast<uint8_t*>(k_scale);
  a.scale[1] = static_cast<uint8_t*>(v_scale);
  a.q_out = static_cast<uint16_t*>(q_out);
  a.status = status;
  a.q_stride = c.q_stride;
  a.k_stride = c.k_stride;
  a.v_stride = c.v_stride;
  a.Hq = c.Hq;
  a.Hkv = c.Hkv;
  a.rotary = c.rotary_dim;
  a.interleaved = c.interleaved;
  a.eps = c.eps;
  a.rope_scale = c.rope_scale;
  const int side = 512 / c.D;                    // heads side by side in a warp
  a.groups = c.scale_block == 1 ? 0 : (c.Hkv + side - 1) / side;
  a.heads = c.Hq + (c.scale_block == 1 ? 2 * c.Hkv : 0);
  // runs of heads: all that the SMs' warps take at once while rows are few, whole
  // rows (one set of sines and cosines) once there are enough
  const long long warps = static_cast<long long>(num_sms) * kWarps * kCtas;
  if (a.heads > 0) {
    long long parts = warps > c.total_rows ? warps / c.total_rows : 1;
    const int most = (a.heads + side - 1) / side;
    if (parts > most) parts = most;
    a.heads_per_part = (a.heads + static_cast<int>(parts) - 1) / static_cast<int>(parts);
    a.heads_per_part = (a.heads_per_part + side - 1) / side * side;
    a.parts = (a.heads + a.heads_per_part - 1) / a.heads_per_part;
  }
  // (every block has a new row)
  const long long items = static_cast<long long>(c.total_rows) * (a.parts + 2 * a.groups);
  long long ctas = (items + kWarps - 1) / kWarps;
  if (ctas > num_sms * kCtas) ctas = num_sms * kCtas;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cudaLaunchConfig_t lc = {};
  lc.gridDim = dim3(static_cast<unsigned>(ctas));
  lc.blockDim = dim3(kThreads);
  lc.dynamicSmemBytes = a.groups > 0 && c.rotary_dim > 0 ? sizeof(AngleTable) : 0;
  lc.stream = static_cast<cudaStream_t>(stream);
  lc.attrs = attr;
  lc.numAttrs = 1;
  const bool f16 = c.dtype == PCTREE_F16;
  const void* fn = c.D == 64 ? (f16 ? append8_kernel<true, 64>() : append8_kernel<false, 64>())
                             : (f16 ? append8_kernel<true, 128>() : append8_kernel<false, 128>());
  if (fn == nullptr) return PCTREE_ERR_CUDA;
  void* params[] = {&a};
  return cudaLaunchKernelExC(&lc, fn, params) == cudaSuccess ? PCTREE_OK : PCTREE_ERR_CUDA;
}

}  // extern "C"
