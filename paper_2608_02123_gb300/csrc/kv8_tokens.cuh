// Attention over a cache in 8 bits for requests of one new row: a unit is the G
// query heads of a row that share a KV head, few against a tile of 128 rows.
//
// Every warp works for itself on 16 keys at a time, from registers: with m16n8k16
// products whose first operand is the cache, S^T = K Q^T has the keys as its rows
// and the query heads as its (8) columns, and O^T += V^T P^T the dims.  Since the
// products' inner index may be permuted as long as both sides agree, a lane's
// share of K is 16 neighbouring dims of a key and of V 16 neighbouring dims of
// four keys: codes are widened where they were loaded, without shared memory.
// (tcgen05 would take them from there, widened, for tiles of 128 rows of which G
// are real: the kernel for many rows takes 230 us for the batch below.)
//
// P is 2^7 times the probability relative to the running maximum of the scores, by
// ex2.approx (2^-22 of it), and its row's sum adds it in float32.  For the product, in float16, V's scales are
// relative to the largest exponent the warp has met.  Where those of 32 keys are at
// most 3 below it, P takes them, 2^-3 .. 1, and V is the codes themselves (11 bits
// of P down to 2^-18 of the maximum, and 2^-29 of it).  Else V takes as many as
// float16 holds exactly with every code, 15, and P the rest: never more than 7, with
// 11 bits down to 2^-14 and 2^-25 of the maximum, as the type has for the probability
// itself.
//
// A CTA's pieces are kv_pieces.cuh's, planned by every warp alike; a piece's keys
// are dealt out among its warps, whose (max, sum, O) are added up in order.
//
// What bounds it (one GB300, us; tokens of 32 requests over up to 8192 slots, 40
// query and 8 KV heads of 128 dims, 431 MB): 84.5 to 86.6 by box, 0.74 of the
// measured copy rate; some 350 instructions a tile of 16 keys, 5 cycles each, by the
// three warps of a quarter of an SM.  Groups of 9 to 16 heads have eight warps: 119 to
// 121 where eight heads take 96 (L2 flushed).  Before: each lane finding its key's place twice over (16 keys at a time)
// 99; a scale or page number that is looked at where it is read 104; sixteen warps of
// one tile ahead 107.  Not kept: a unit of all KV heads of a row (neighbouring memory
// at the same time) 114; codes through L1 132; the codes of no key from an array of
// zeros instead of predicated loads 87.
#pragma once

#include <cfloat>
#include <type_traits>

#include "kv8.cuh"
#include "kv_pieces.cuh"

namespace pct {
namespace {

struct Kv8AttnArgs {
  Units units;
  Kv8Blocks blocks;
  const uint16_t* q;
  const uint8_t* cache[2];                   // keys, values
  const uint8_t* scale[2];
  const int32_t* parent;                     // NULL: causal
  uint16_t* out;
  float* part_o;                             // as in JoinArgs
  float2* part_ml;
  PieceJoin* join;
  int32_t* status;
  long long q_stride;
  int Hq, G;
  int tile_rows;                             // a unit's first rows; the rest are tile 1's
  FastDiv by_G;
  float scale_log2;
};

__device__ __forceinline__ void report(int32_t* status, int code) {
  if (status != nullptr) atomicCAS(status, 0, code);
}

// Threads for NT groups of 8 query heads: as many as their registers allow.
__host__ __device__ constexpr int token_threads(int NT) { return NT == 1 ? 384 : 256; }
__host__ __device__ constexpr int token_warps(int NT) { return token_threads(NT) / 32; }
constexpr int kTokenBlock = 128;             // keys per block of work
constexpr int kTokenHeads = 16;              // query heads of a unit, at most
constexpr float kTokenBits = 7.0f;           // P is 2^7 times what it is relative to
constexpr int kTokenLift = 3;                // of V's exponents that P takes where all are near

// D (+)= A B of 16 x 8 x 16 float16 values, float32 sums.
__device__ __forceinline__ void mma_f16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2,
                                        uint32_t a3, uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, "
      "{%0,%1,%2,%3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// The softmax scale of a row of Q times 2^e: a normal number, so that neither a masked
// score's infinity nor a score of 0 becomes NaN.  (Below the smallest all scores are 0
// but for 2^-80; past the largest those that are not equal are 2^70 apart.)
__device__ __forceinline__ float row_scale(float scale_log2, int e) {
  return fminf(fmaxf(scale_log2 * exp2_of(e), FLT_MIN), FLT_MAX);
}

// Two float16 values times a float16 pair.
__device__ __forceinline__ uint32_t mul_h2(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("mul.rn.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}

// 2^e as float16, e in -15 .. 7.
__device__ __forceinline__ uint16_t half_exp(int e) {
  return static_cast<uint16_t>(e >= -14 ? (e + 15) << 10 : 0x200);
}
__device__ __forceinline__ uint32_t transposed8x8(uint32_t x) {
  uint32_t r;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(x));
  return r;
}

// N words, or zeros if not wanted.  (Predicated inside: a branch around the load
// would end in a copy of its result, which waits for it.)
template <int N>
__device__ __forceinline__ void load_if(uint32_t (&v)[N], bool wanted, const uint8_t* p) {
  if constexpr (N == 4) {
    asm volatile(
        "{\n .reg .pred p;\n setp.ne.u32 p, %5, 0;\n mov.u32 %0, 0;\n mov.u32 %1, 0;\n"
        " mov.u32 %2, 0;\n mov.u32 %3, 0;\n"
        " @p ld.global.nc.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];\n}\n"
        : "=&r"(v[0]), "=&r"(v[1]), "=&r"(v[2]), "=&r"(v[3])
        : "l"(p), "r"(static_cast<uint32_t>(wanted)));
  } else {
    asm volatile(
        "{\n .reg .pred p;\n setp.ne.u32 p, %3, 0;\n mov.u32 %0, 0;\n mov.u32 %1, 0;\n"
        " @p ld.global.nc.L1::no_allocate.v2.u32 {%0,%1}, [%2];\n}\n"
        : "=&r"(v[0]), "=&r"(v[1])
        : "l"(p), "r"(static_cast<uint32_t>(wanted)));
  }
}

__device__ __forceinline__ int load_int_if(bool wanted, const int32_t* p, int otherwise) {
  int v;
  asm volatile(
      "{\n .reg .pred p;\n setp.ne.u32 p, %2, 0;\n mov.u32 %0, %3;\n"
      " @p ld.global.nc.u32 %0, [%1];\n}\n"
      : "=&r"(v)
      : "l"(p), "r"(static_cast<uint32_t>(wanted)), "r"(otherwise));
  return v;
}
__device__ __forceinline__ uint32_t load_byte_if(bool wanted, const uint8_t* p,
                                                 uint32_t otherwise) {
  uint32_t v;
  asm volatile(
      "{\n .reg .pred p;\n setp.ne.u32 p, %2, 0;\n mov.u32 %0, %3;\n"
      " @p ld.global.nc.u8 %0, [%1];\n}\n"
      : "=&r"(v)
      : "l"(p), "r"(static_cast<uint32_t>(wanted)), "r"(otherwise));
  return v;
}

template <int D, int NT>
struct TokenShared {
  float o[token_warps(NT)][8 * NT][D + 4];
  float m[token_warps(NT)][8 * NT], l[token_warps(NT)][8 * NT];
  unsigned upto[PCTREE_KV_MAX_BATCH];
  int16_t par[PCTREE_ATTN_MAX_N];
  uint32_t path[PCTREE_ATTN_MAX_N / 32];         // the row and its ancestors
};

// NT: groups of 8 query heads.
template <int D, bool F16, int NT>
__global__ void __launch_bounds__(token_threads(NT), 1) kv8_token_kernel(Kv8AttnArgs a) {
  constexpr int kC = D / 64;                     // 16-byte chunks of a key's row a lane has
  constexpr int kVWords = D / 32;                // words of V a lane has of a key
  constexpr int kTiles = D / 16;                 // of O^T's rows
  extern __shared__ uint8_t smem_raw[];
  TokenShared<D, NT>& sh = *reinterpret_cast<TokenShared<D, NT>*>(smem_raw);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int g = lane >> 2, t = lane & 3;
  const KvRows& rows = a.units.rows;
  const int Hkv = a.units.Hkv;
  pdl_launch_dependents();
  pdl_wait();
  count_work<token_threads(NT)>(a.units, sh.upto, [&](int code) {
    if (blockIdx.x == 0) report(a.status, code);
  });

  auto piece = [&](const Piece& it) -> bool {
    // this lane's share of Q: head g, the dims of its chunks
    uint32_t qf[NT][kC][4][2];
    float sc[NT][2];                             // of the heads 2 t and 2 t + 1 (log2 units)
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      const int h = 8 * n + g;
      float row_sc = a.scale_log2;
      const uint16_t* q =
          a.q + it.row0 * a.q_stride + (it.kvh * a.G + min(h, a.G - 1)) * D + t * 16;
      uint32_t top2 = 0;
#pragma unroll
      for (int c = 0; c < kC; ++c) {
        const uint4 lo = *reinterpret_cast<const uint4*>(q + c * 64);
        const uint4 hi = *reinterpret_cast<const uint4*>(q + c * 64 + 8);
        const uint32_t w[8] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          qf[n][c][i / 2][i & 1] = h < a.G ? w[i] : 0;
          top2 = __vmaxu2(top2, w[i] & 0x7fff7fffu);
        }
      }
      if constexpr (!F16) {
        // to float16: the row's largest to 2^14 .. 2^15 (as in the kernel for many rows)
        top2 = __vmaxu2(top2, __shfl_xor_sync(kFull, top2, 1));
        top2 = __vmaxu2(top2, __shfl_xor_sync(kFull, top2, 2));
        const int top = static_cast<int>(max(top2 >> 16, top2 & 0xffffu) >> 7) - 127;
        const int e = max(-100, min(126, top)) - 14;
        const float by = exp2_of(-e);
        row_sc = row_scale(row_sc, e);
#pragma unroll
        for (int c = 0; c < kC; ++c)
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const float2 f = unpack16<false>(qf[n][c][i / 2][i & 1]);
            qf[n][c][i / 2][i & 1] = pack16<true>(f.x * by, f.y * by);
          }
      }
      sc[n][0] = __shfl_sync(kFull, row_sc, 8 * t);
      sc[n][1] = __shfl_sync(kFull, row_sc, 8 * t + 4);
    }
    float o[NT][kTiles][4];                      // times 2^-e_ref
    float m[NT][2], l[NT][2];
    int e_ref = kMinExp;                         // the largest exponent of V so far
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      m[n][0] = m[n][1] = -INFINITY;
      l[n][0] = l[n][1] = 0.0f;
#pragma unroll
      for (int i = 0; i < kTiles; ++i) o[n][i][0] = o[n][i][1] = o[n][i][2] = o[n][i][3] = 0.0f;
    }
    const int stop = min(it.key_end, it.b1 * kTokenBlock);
    int edge = stop;                             // from here on not every key is seen
    if (a.parent != nullptr) {
      const int32_t* parent = a.parent + it.row0 - it.j0;
      for (int i = threadIdx.x; i <= it.j0; i += token_threads(NT)) {
        int p = parent[i];
        if (p < -1 || p >= i) {                  // parents precede children
          report(a.status, PCTREE_ERR_INVALID_ARG);
          p = -1;
        }
        sh.par[i] = static_cast<int16_t>(p);
      }
      __syncthreads();
      if (warp == 0) {
        uint32_t word = 0;                       // lane i finds word i
        for (int i = it.j0; i >= 0; i = sh.par[i])
          if (i >> 5 == lane) word |= 1u << (i & 31);
        if (lane < PCTREE_ATTN_MAX_N / 32) sh.path[lane] = word;
      }
      __syncthreads();
      edge = min(edge, it.prefix);
    }
    // Keys come to a warp 32 at a time, as two tiles of 16; lane i finds the place and
    // the scales of key i, none where the row does not see it and in pages that are
    // none.  Codes are on their way from 32 keys ahead, page numbers from 32 more.
    constexpr uint32_t kNone = 0xffffffffu;
    struct Ahead {
      uint32_t k[2][kC][4], v[4][kVWords];
    };
    int page = 0;                                // as it is in the table
    auto find_page = [&](int key0) {
      const int key = key0 + lane;
      page = load_int_if(
          key < stop && rows.page_table != nullptr,
          rows.page_table + static_cast<size_t>(it.r) * rows.max_pages + div_by(key, a.blocks.page),
          it.r);
    };
    uint32_t at = kNone, k_byte = kExpBias, v_byte = kExpBias;
    bool seen = false;
    auto find = [&](int key0) {
      const int key = key0 + lane;
      seen = key < stop;
      bool is = seen && page >= 0 && page < rows.n_pages;
      if (seen && !is) report(a.status, PCTREE_ERR_INVALID_ARG);
      if (a.parent != nullptr && key0 + 32 > edge) {
        const int node = key - it.prefix;
        if (seen && node >= 0) seen = (sh.path[node >> 5] >> (node & 31)) & 1u;
        is = is && seen;
      }
      const int off = key - div_by(key, a.blocks.page) * rows.page_size;
      at = is ? (static_cast<uint32_t>(page) * rows.page_size + off) * Hkv + it.kvh : kNone;
      const long long s = (static_cast<long long>(page) * a.blocks.per_page +
                           (off >> a.blocks.shift)) * Hkv + it.kvh;
      k_byte = load_byte_if(is, a.scale[0] + s, kExpBias);
      v_byte = load_byte_if(is, a.scale[1] + s, kExpBias);
    };
    // codes of the keys from lane `half` on
    auto load_k = [&](Ahead& x, int half) {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const uint32_t p = __shfl_sync(kFull, at, half + g + 8 * i);
#pragma unroll
        for (int c = 0; c < kC; ++c)
          load_if<4>(x.k[i][c], p != kNone,
                     a.cache[0] + static_cast<size_t>(p) * D + c * 64 + t * 16);
      }
    };
    auto load_v = [&](Ahead& x, int half) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t p = __shfl_sync(kFull, at, half + 2 * t + (i & 1) + 8 * (i >> 1));
        load_if<kVWords>(x.v[i], p != kNone,
                         a.cache[1] + static_cast<size_t>(p) * D + g * (D / 8));
      }
    };
    const int first = it.b0 * kTokenBlock + warp * 32;
    constexpr int kStep = 32 * token_warps(NT);
    // Of a lane's key: K's scale as the upper half of a float, the part of V's that P
    // takes as the lower half (0: not seen); V's own part; whether there is any.
    uint32_t here = 0, v_part = 0;
    bool parted = false;
    // one tile, whose registers then take the one 32 keys on
    auto step = [&](Ahead& cur, int key0, int half) {
      float s[NT][4];
#pragma unroll
      for (int n = 0; n < NT; ++n) s[n][0] = s[n][1] = s[n][2] = s[n][3] = 0.0f;
#pragma unroll
      for (int c = 0; c < kC; ++c)
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          const uint32_t x = cur.k[0][c][w], y = cur.k[1][c][w];
          const uint32_t a0 = halves2(x), a1 = halves2(y), a2 = halves2(x >> 16),
                         a3 = halves2(y >> 16);
#pragma unroll
          for (int n = 0; n < NT; ++n) mma_f16(s[n], a0, a1, a2, a3, qf[n][c][w][0], qf[n][c][w][1]);
        }
      load_k(cur, half);
      // scores with K's scales; keys not seen are -inf
      uint32_t p16[NT][2];
      float k_by[2], p_by[2];
      bool hide[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const uint32_t by = __shfl_sync(kFull, here, half + g + 8 * i);
        k_by[i] = __uint_as_float(by & 0xffff0000u);
        p_by[i] = __uint_as_float(by << 16);
        hide[i] = key0 + 16 > edge && p_by[i] == 0.0f;
      }
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        // (x: scores; d: relative to the reference)
        float x[4], d[4];
        bool look = false;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          x[i] = (s[n][i] * k_by[i >> 1]) * sc[n][i & 1];
          if (hide[i >> 1]) x[i] = -INFINITY;
          const float ref = m[n][i & 1] == -INFINITY ? 0.0f : m[n][i & 1];
          d[i] = x[i] - ref;
          look = look || d[i] > (m[n][i & 1] == -INFINITY ? -INFINITY : 8.0f);
        }
        if (__any_sync(kFull, look)) {
#pragma unroll
          for (int r = 0; r < 2; ++r) {
            float top = fmaxf(x[r], x[2 + r]);
#pragma unroll
            for (int o2 = 4; o2 < 32; o2 <<= 1) top = fmaxf(top, __shfl_xor_sync(kFull, top, o2));
            if (top > m[n][r]) {
              const float alpha = ex2_approx(m[n][r] - top);
              m[n][r] = top;
              d[r] = x[r] - top;
              d[2 + r] = x[2 + r] - top;
              l[n][r] *= alpha;
#pragma unroll
              for (int i = 0; i < kTiles; ++i) {
                o[n][i][r] *= alpha;
                o[n][i][2 + r] *= alpha;
              }
            }
          }
        }
        float p[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          p[i] = ex2_approx(d[i] + kTokenBits);
          l[n][i & 1] += p[i];
        }
        p16[n][0] = transposed8x8(pack16<true>(p[0] * p_by[0], p[1] * p_by[0]));
        p16[n][1] = transposed8x8(pack16<true>(p[2] * p_by[1], p[3] * p_by[1]));
      }
      // V^T P^T: pairs of keys of a dim, two dims a word
      auto product = [&](auto with_parts) {
        uint32_t part[2] = {0, 0};               // of V's scales, pairs of keys
        if constexpr (with_parts.value) {
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            const uint32_t lo = __shfl_sync(kFull, v_part, half + 2 * t + 8 * i);
            part[i] = lo | __shfl_sync(kFull, v_part, half + 2 * t + 1 + 8 * i) << 16;
          }
        }
        auto halves = [&](uint32_t codes, int i) {
          const uint32_t h = halves2(codes);
          if constexpr (with_parts.value) return mul_h2(h, part[i]);
          return h;
        };
#pragma unroll
        for (int w = 0; w < kVWords; ++w)
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            const uint32_t sel = j == 0 ? 0x5140u : 0x7362u;
            const uint32_t lo = __byte_perm(cur.v[0][w], cur.v[1][w], sel);
            const uint32_t hi = __byte_perm(cur.v[2][w], cur.v[3][w], sel);
            const uint32_t a0 = halves(lo, 0), a1 = halves(lo >> 16, 0), a2 = halves(hi, 1),
                           a3 = halves(hi >> 16, 1);
#pragma unroll
            for (int n = 0; n < NT; ++n)
              mma_f16(o[n][2 * w + j], a0, a1, a2, a3, p16[n][0], p16[n][1]);
          }
      };
      if (parted) product(std::true_type{}); else product(std::false_type{});
      load_v(cur, half);
    };
    // the scales of the 32 keys that come next
    auto take_scales = [&]() {
      if (!scale_ok(k_byte) || !scale_ok(v_byte)) report(a.status, PCTREE_ERR_INVALID_ARG);
      const bool none = at == kNone;             // no codes: any scale does
      const int e = none ? kMinExp : scale_exp(v_byte);
      const int top = __reduce_max_sync(kFull, e);
      if (top > e_ref) {
        const float by = exp2_of(e_ref - top);
        e_ref = top;
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int i = 0; i < kTiles; ++i)
#pragma unroll
            for (int r = 0; r < 4; ++r) o[n][i][r] *= by;
      }
      const int off = none ? 0 : e - e_ref;      // -22 .. 0
      parted = __any_sync(kFull, off < -kTokenLift);
      const int p_exp = parted ? min(0, off - kMinExp) : off;
      v_part = half_exp(off - p_exp);            // (-15 .. 0: exact with every code)
      here = __float_as_uint(exp2_of(scale_exp(k_byte))) |
             (seen ? __float_as_uint(exp2_of(p_exp)) >> 16 : 0u);
    };
    Ahead x0, x1;
    find_page(first);
    find(first);
    find_page(first + kStep);
    load_k(x0, 0);
    load_v(x0, 0);
    load_k(x1, 16);
    load_v(x1, 16);
#pragma unroll 1
    for (int key0 = first; key0 < stop; key0 += kStep) {
      take_scales();
      find(key0 + kStep);
      find_page(key0 + 2 * kStep);
      step(x0, key0, 0);
      if (key0 + 16 < stop) step(x1, key0 + 16, 16);
    }
    // the warps' parts, in order
    const float f = exp2_of(e_ref);
#pragma unroll
    for (int n = 0; n < NT; ++n) {
#pragma unroll
      for (int r = 0; r < 2; ++r) {
#pragma unroll
        for (int d = 4; d < 32; d <<= 1) l[n][r] += __shfl_xor_sync(kFull, l[n][r], d);
        const int h = 8 * n + 2 * t + r;
        if (g == 0) {
          sh.m[warp][h] = m[n][r];
          sh.l[warp][h] = l[n][r];
        }
#pragma unroll
        for (int i = 0; i < kTiles; ++i)
          *reinterpret_cast<float2*>(&sh.o[warp][h][g * (D / 8) + 2 * i]) =
              make_float2(o[n][i][r] * f, o[n][i][2 + r] * f);
      }
    }
    __syncthreads();
    const bool whole = it.b0 == 0 && it.b1 == it.nblk;
    const size_t part = static_cast<size_t>(blockIdx.x) * 2 + (it.b0 == 0 ? 1 : 0);
    constexpr int kQuads = D / 4;
    for (int i = threadIdx.x; i < a.G * kQuads; i += token_threads(NT)) {
      const int h = i / kQuads, d = (i - h * kQuads) * 4;
      float top = -INFINITY, sum = 0.0f;
#pragma unroll
      for (int w = 0; w < token_warps(NT); ++w)
        if (sh.l[w][h] != 0.0f) top = fmaxf(top, sh.m[w][h]);
      float4 y = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
      for (int w = 0; w < token_warps(NT); ++w) {
        const float lw = sh.l[w][h];
        if (lw == 0.0f) continue;                // (no finite score, or no keys)
        const float f = exp2f(sh.m[w][h] - top);
        const float4 v = *reinterpret_cast<const float4*>(&sh.o[w][h][d]);
        sum = fmaf(lw, f, sum);
        y.x = fmaf(v.x, f, y.x);
        y.y = fmaf(v.y, f, y.y);
        y.z = fmaf(v.z, f, y.z);
        y.w = fmaf(v.w, f, y.w);
      }
      if (whole) {
        const float inv = 1.0f / sum;            // (no finite score, sum = 0: NaN)
        *reinterpret_cast<uint2*>(a.out + (static_cast<size_t>(it.row0) * a.Hq + it.kvh * a.G + h) * D +
                                  d) = make_uint2(pack16<F16>(y.x * inv, y.y * inv),
                                                  pack16<F16>(y.z * inv, y.w * inv));
      } else {
        reinterpret_cast<float4*>(a.part_o)[(part * kQuads + d / 4) * kUnitRows + h] = y;
        if (d == 0) a.part_ml[part * kUnitRows + h] = make_float2(sum != 0.0f ? top : -INFINITY, sum);
      }
    }
    __syncthreads();
    return true;
  };
  PieceJoin join;
  plan_pieces(a.units, sh.upto, join, piece);
  if (threadIdx.x == 0) a.join[blockIdx.x] = join;
}

template <int D, bool F16, int NT>
cudaError_t launch_tokens(cudaLaunchConfig_t lc, const Kv8AttnArgs& a) {
  static SmemLimit limit;
  const cudaError_t e = limit.ensure(reinterpret_cast<const void*>(kv8_token_kernel<D, F16, NT>),
                                     sizeof(TokenShared<D, NT>));
  if (e != cudaSuccess) return e;
  lc.blockDim = dim3(token_threads(NT));
  lc.dynamicSmemBytes = sizeof(TokenShared<D, NT>);
  return cudaLaunchKernelEx(&lc, kv8_token_kernel<D, F16, NT>, a);
}

}  // namespace
}  // namespace pct
