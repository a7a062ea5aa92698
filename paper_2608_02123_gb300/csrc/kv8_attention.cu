// pctree_kv8_attention: grouped-query attention of new rows of several requests
// (tokens, chains, packed trees, prompts) over a paged or contiguous cache of
// 8-bit codes with a power-of-two scale per block of slots and head.
//
// Units, pieces and joins are kv_pieces.cuh's.  A unit has up to two tiles of rows;
// a tile's rows are (row, query head of the group) pairs, R = G * tile_rows <= 128.
// Keys come in blocks of 64 consecutive slots, gathered slot by slot, so pages of
// any size fill a block, and are brought and widened once for both tiles.
//
//   warp 0        planner: the CTA's pieces, in order, up to kItemRing ahead
//   warp 1        S issuer: S = Q K^T (tcgen05.mma, M = 128, N = 64) of each tile
//                 into one of its two TMEM buffers
//   warp 2        PV issuer: O += P V of each tile (P read from TMEM)
//   warp 3        where the keys of a block lie and what scales they have, up to
//                 kPlaceRing blocks ahead
//   warps 4..7    the next unit's Q as it is and its rows' ancestors, once the last S
//                 of a piece is done; then O of the finished piece to rows of out or
//                 to the piece's partial
//   warps 8..15   softmax, four warps a tile and a thread a row: Q to float16, then S
//                 is read from TMEM, masked and scaled, P = 2^(s - m_used) written
//                 back over it
//   warps 16..19  K, and warps 20..23 V: codes to shared memory two blocks ahead,
//                 16 bytes a thread and copy, and to float16 (128-byte swizzle, 64
//                 dims a half)
// All waits are bounded (1 s; those for a whole piece 1 s without a block) and end
// in PCTREE_ERR_TIMEOUT.
//
// Numbers: code * 2^e is exact in float16 for every exponent of the format, so the
// products' K and V are the cache's values.  A bfloat16 row of Q is multiplied by
// a power of two that brings its largest element to 2^14 .. 2^15 (exact in float16
// but for elements below 2^-31 of the largest, and those to 2^-39 of it); the power
// goes into the row's softmax scale.  P is 2^7 times the probability relative to the
// row's running maximum, by ex2.approx (2^-22 of it), in float16 (11 bits; down to
// 2^-31 of the maximum): far keys of a long context that are each small against the
// first are not lost.  (A product's operands have one type, and float16 holds V
// exactly.  P's rounding is below that of a bfloat16 output; to a float16 output's
// error it adds a fifth.)  Row sums add the unrounded values.
//
// What bounds it (one GB300, us; 40 query and 8 KV heads of 128 dims, bf16):
//   four prompts of up to 4096 rows 874 to 884 by box (0.48 PFLOP/s), packed trees of 32
//   requests 197 to 200.  With longer prefixes a block of 64 keys costs
//   2950 cycles for two tiles (at the 2070 MHz sampled meanwhile), of which the
//   products take 1280 (S, M = 128, N = 64, reads 6 KB of shared memory a product: 48
//   cycles instead of 32), the widening's traffic (64 KB) 512, and a softmax warp's
//   chain 2300: two warps on an SM's quarter issue an instruction in some 7 cycles
//   each, and the roles' code, 140 KB, is more than the instruction cache holds.  That
//   is 506 us of the prompts' (354 blocks a CTA) and 89 of the trees' (62); the rest
//   is 18 to 25 us for each of a CTA's 14 and 5 pieces: queries, first block, output;
//   16 chains of 8 rows (32 query heads) 35: one tile, 16 to 32 of its 128 rows real;
//   2100 cycles a block.
// Steps that were measured (prompts): codes to registers with a branch around each
// load, which waits for it, 4583; places and scales by a warp of their own 1589;
// copies to shared memory 1290; two tiles a block of K and V 1216; Q in place by
// asynchronous copies, to float16 by its tile's softmax warps 870.  Not kept: codes in
// registers two blocks ahead instead of the copies 997; one warpgroup for K and V both
// 2147; the rescaling of O unrolled (instructions that run rarely come from memory)
// 1370.
#include <algorithm>
#include <atomic>

#include "kv8_tokens.cuh"

namespace pct {
namespace {

constexpr int kBK = 64;                      // keys per block
constexpr int kQHalf = 128 * 128;            // bytes of 128 rows x 64 halves
constexpr int kKHalf = kBK * 128;            // of a block's
constexpr uint64_t kLimitNs = 1000000000ull;
constexpr int kThreads = 768;
constexpr int kSlots = 6;                    // K and V blocks in the ring, in turn
constexpr int kAhead = 2;                    // blocks of codes under way
constexpr int kItemRing = 8;
constexpr int kPlaceRing = 4;
constexpr uint32_t kTmemCols = 512;
// Registers a thread: of the launch, and what the groups of four warps make of
// them (their sum must not exceed the launch's).
constexpr int kRegsLaunch = 80, kRegsIssue = 48, kRegsSoftmax = 112, kRegsConvert = 64;
static_assert(kRegsLaunch * kThreads <= 65536 &&
                  kRegsIssue + kRegsLaunch + 2 * kRegsSoftmax + 2 * kRegsConvert <=
                      kRegsLaunch * (kThreads / 128),
              "registers");
constexpr uint32_t kOCol = 4 * kBK;          // S of tile t, buffer b: column (2 t + b) * kBK
constexpr float kPBits = 7.0f;               // P is 2^7 times what it is relative to

// A block's keys: places (slot * Hkv + head, or kNowhere) and scales (float16, of
// K and of V).
constexpr uint32_t kNowhere = 0xffffffffu;
struct Places {
  uint32_t at[kBK];
  uint32_t by[kBK];                          // V's in the upper half
  int key0, all, ring;                       // keys below `all` are seen by every row
  int keys;                                  // 0: no more blocks
};

struct Tail {
  uint64_t place_full[kPlaceRing], place_empty[kPlaceRing];
  // (raw: by place in the item ring, whose places are given back after the wait for
  // it: a warp without a part in a piece cannot fall a phase behind; full: by tile)
  uint64_t q_raw[kItemRing], q_full[2], q_empty;
  uint64_t kv_full[kSlots], kv_empty[kSlots];
  uint64_t s_full[2][2], p_full[2][2], p_empty[2][2];      // [tile][buffer]
  uint64_t o_full[2], o_empty[2];            // [tile]
  uint64_t item_full[kItemRing], item_empty[kItemRing];
  uint64_t done, out_sync;
  uint32_t tmem_base;
  int abort;
  int blocks;                                // multiplied so far (see wwait_long)
  Piece item[kItemRing];
  Places places[kPlaceRing];
  float row_l[2][128], row_m[2][128];        // [tile]
  float row_scale[2][128];                   // of Q's rows (log2 units), [tile]
  // keys with NaN values that only some rows of the unit see, by place in the item
  // ring: a bit each, counted from the first key that not every row sees
  uint32_t bad[kItemRing][PCTREE_ATTN_MAX_N / 32];
  int16_t par[PCTREE_ATTN_MAX_N];
  uint32_t path[2][256][PCTREE_ATTN_MAX_N / 32];   // rows' ancestors, by piece parity
  alignas(16) uint8_t stage[4][32 * 32];
  unsigned upto[PCTREE_KV_MAX_BATCH];        // work of requests 0 .. r
};

template <int N>
__device__ __forceinline__ void set_registers_up() {
  asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(N));
}
template <int N>
__device__ __forceinline__ void set_registers_down() {
  asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(N));
}

__device__ __forceinline__ void tmem_st_x8(uint32_t taddr, const uint32_t (&r)[8]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"r"(taddr),
      "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7])
      : "memory");
}
__device__ __forceinline__ void tmem_st_x16(uint32_t taddr, const uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], "
      "{%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};" ::"r"(taddr),
      "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]),
      "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]),
      "r"(r[15])
      : "memory");
}
// D[tmem] (+)= A[tmem] * B[smem] (see tc_mma_bf16): A's 16 K elements are 8
// columns of 16-bit pairs.
__device__ __forceinline__ void tc_mma_tmem_a(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc,
                                              uint32_t accumulate) {
  asm volatile(
      "{\n .reg .pred p;\n setp.ne.b32 p, %4, 0;\n"
      " tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n}\n" ::"r"(d),
      "r"(a), "l"(b), "r"(idesc), "r"(accumulate)
      : "memory");
}
// Instruction descriptor with float16 operands.
__host__ __device__ constexpr uint32_t idesc_f16(int M, int N) {
  return idesc_bf16_f32(M, N) & ~((1u << 7) | (1u << 10));
}

// An asynchronous copy of 16 bytes (zeros if not wanted) to shared memory.
__device__ __forceinline__ void copy16_if(bool wanted, void* dst, const uint8_t* p) {
  asm volatile(
      "cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(smem_u32(dst)), "l"(p),
      "r"(wanted ? 16 : 0)
      : "memory");
}
__device__ __forceinline__ void copies_commit() {
  asm volatile("cp.async.commit_group;" ::: "memory");
}
template <int N>
__device__ __forceinline__ void copies_wait() {
  asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}

// Whether a word holds the code NaN (a carry into the byte's top bit).
__device__ __forceinline__ uint32_t nan_tops(uint32_t w) {
  return ((w & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u;
}
__device__ __forceinline__ bool any_nan(const uint4& x) {
  return (nan_tops(x.x) | nan_tops(x.y) | nan_tops(x.z) | nan_tops(x.w)) != 0;
}

// Sixteen codes of V with the NaN among them replaced by 0, their key noted.
__device__ __noinline__ uint4 without_nan(uint4 x, Tail* T, int ring, int key) {
  uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) w[i] &= ~((nan_tops(w[i]) >> 7) * 0xffu);   // 0xff in those bytes
  atomicOr(&T->bad[ring][key >> 5], 1u << (key & 31));
  return make_uint4(w[0], w[1], w[2], w[3]);
}
// Which of sixteen codes are NaN, a bit each.
__device__ __forceinline__ uint32_t nan_bits(const uint4& x) {
  const uint32_t w[4] = {x.x, x.y, x.z, x.w};
  uint32_t bits = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t nan = (nan_tops(w[i]) >> 7) * 0xffu;
    bits |= (((nan & 0x08040201u) * 0x01010101u) >> 24 & 15u) << (4 * i);
  }
  return bits;
}

// Scores (in log2 units) whose floats are half an octave apart: from here on the
// softmax's fused product would differ from its reference, a rounded product, by
// powers of two that P's type does not hold.
constexpr float kWideScore = 4194304.0f;

// The 64 scores of a block at TMEM columns s_col .. (those not in `see` are
// -inf) become what, times sc, is the rounded score less the reference.
__device__ __noinline__ void wide_scores(uint32_t s_col, float sc, float mref, uint64_t see) {
  const float inv = 1.0f / sc;
#pragma unroll 1
  for (int c = 0; c < 64; c += 8) {
    uint32_t y[8];
    tmem_ld_32x32b_x8(s_col + c, y);
    tmem_ld_wait();
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const float x = (see >> (c + k)) & 1 ? __uint_as_float(y[k]) : -INFINITY;
      y[k] = __float_as_uint((__fmul_rn(x, sc) - mref) * inv);
    }
    tmem_st_x8(s_col + c, y);
  }
  tmem_st_wait();
}

__device__ __forceinline__ bool wait_one(Tail* T, uint64_t* bar, uint32_t parity) {
  return mbar_wait_bounded(bar, parity, &T->abort, kLimitNs);
}
// By a whole warp; and one that lasts as long as pieces do: over once no block has
// been multiplied for the limit.
__device__ __forceinline__ bool wwait(Tail* T, uint64_t* bar, uint32_t parity) {
  return __all_sync(kFull, wait_one(T, bar, parity));
}
__device__ __forceinline__ bool wwait_long(Tail* T, uint64_t* bar, uint32_t parity) {
  volatile int* blocks = &T->blocks;
  for (;;) {
    const int before = *blocks;
    if (wwait(T, bar, parity)) return true;
    if (__any_sync(kFull, *static_cast<volatile int*>(&T->abort) != 0) ||
        __all_sync(kFull, *blocks == before))
      return false;
  }
}

template <int D, bool F16>
__global__ void __launch_bounds__(kThreads, 1) kv8_attn_kernel(Kv8AttnArgs a) {
  constexpr int kHalves = D / 64;
  constexpr int kQBytes = kHalves * kQHalf, kKBytes = kHalves * kKHalf;
  constexpr int kCodeBytes = kBK * D;              // of a block's K or V
  extern __shared__ uint8_t smem_raw[];
  uint8_t* sm = reinterpret_cast<uint8_t*>(
      (reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~static_cast<uintptr_t>(1023));
  uint8_t* sq = sm;                                // [tile]
  uint8_t* skv = sq + 2 * kQBytes;                 // ring
  uint8_t* codes = skv + kSlots * kKBytes;         // [K, V][kAhead][row of a thread][128][16]
  Tail* T = reinterpret_cast<Tail*>(codes + 2 * kAhead * kCodeBytes);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

  // ---------------- set-up ----------------
  if (threadIdx.x == 0) {
    for (int s = 0; s < kSlots; ++s) {
      mbar_init(&T->kv_full[s], 4);
      mbar_init(&T->kv_empty[s], 1);
    }
    mbar_init(&T->q_empty, 1);
    for (int s = 0; s < 2; ++s) {
      mbar_init(&T->q_full[s], 4);
      for (int t = 0; t < 2; ++t) {
        mbar_init(&T->s_full[t][s], 1);
        mbar_init(&T->p_full[t][s], 4);
        mbar_init(&T->p_empty[t][s], 1);
      }
      mbar_init(&T->o_full[s], 1 + 4);
      mbar_init(&T->o_empty[s], 4);
    }
    for (int s = 0; s < kItemRing; ++s) {
      mbar_init(&T->q_raw[s], 4);
      mbar_init(&T->item_full[s], 1);
      mbar_init(&T->item_empty[s], 2 + 1 + 4 + 8);
    }
    for (int s = 0; s < kPlaceRing; ++s) {
      mbar_init(&T->place_full[s], 1);
      mbar_init(&T->place_empty[s], 8);
    }
    mbar_init(&T->done, 2);
    mbar_init(&T->out_sync, 4);
    T->abort = 0;
    T->blocks = 0;
    fence_barrier_init();
  }
  // rows past a tile's are never written: zero them once
  {
    const int R = a.G * a.tile_rows, zq = (128 - R) * 8;
    for (int i = threadIdx.x; i < 2 * kHalves * zq; i += kThreads) {
      const int h = i / zq, rem = i - h * zq;
      *reinterpret_cast<uint4*>(sq + h * kQHalf + (R + rem / 8) * 128 + (rem % 8) * 16) =
          make_uint4(0, 0, 0, 0);
    }
  }
  fence_proxy_async_smem();
  if (warp == 1) tmem_alloc(&T->tmem_base, kTmemCols);
  pdl_launch_dependents();
  pdl_wait();
  count_work<kThreads>(a.units, T->upto, [&](int code) {
    if (blockIdx.x == 0) report(a.status, code);
  });
  tc_fence_before_sync();
  __syncthreads();
  tc_fence_after_sync();

  auto give_up = [&]() {
    *static_cast<volatile int*>(&T->abort) = 1;
    report(a.status, PCTREE_ERR_TIMEOUT);
  };
  auto fetch_one = [&](int k, Piece& it) -> bool {
    const int s = k % kItemRing;
    if (!wait_one(T, &T->item_full[s], (k / kItemRing) & 1)) return false;
    it = T->item[s];
    mbar_arrive(&T->item_empty[s]);
    return true;
  };
  // (peek leaves the place taken)
  auto peek_warp = [&](int k, Piece& it) -> bool {
    const int s = k % kItemRing;
    if (!wwait_long(T, &T->item_full[s], (k / kItemRing) & 1)) return false;
    it = T->item[s];
    return true;
  };
  auto release_warp = [&](int k) {
    __syncwarp();
    if (lane == 0) mbar_arrive(&T->item_empty[k % kItemRing]);
  };

  if (warp < 4) {
    set_registers_down<kRegsIssue>();
    const uint32_t tmem = T->tmem_base;
    if (warp == 1 && lane == 0) {
      // ---------------- S issuer ----------------
      constexpr uint32_t idS = idesc_f16(128, kBK);
      const uint64_t q_desc = desc_kmajor_sw128(smem_u32(sq));
      const uint64_t k_desc = desc_kmajor_sw128(smem_u32(skv));
      int g = 0, gt[2] = {0, 0}, kt[2] = {0, 0};   // blocks, of each tile; pieces of each
      bool ok = true;
      Piece it;
      for (int k = 0; ok; ++k) {
        if (!(ok = fetch_one(k, it)) || it.nblk == 0) break;
        const int tiles = it.n_rows > a.tile_rows ? 2 : 1;
        for (int b = it.b0; ok && b < it.b1; ++b, ++g) {
          const int slot = (2 * g) % kSlots;
          if (!(ok = wait_one(T, &T->kv_full[slot], (2 * g / kSlots) & 1))) break;
          const uint64_t kd = k_desc + slot * (kKBytes >> 4);
#pragma unroll 1
          for (int t = 0; t < tiles; ++t) {
            const int n = t == 0 ? gt[0]++ : gt[1]++, sb = n & 1;
            ok = wait_one(T, &T->p_empty[t][sb], ((n >> 1) & 1) ^ 1) &&
                 (b > it.b0 || wait_one(T, &T->q_full[t], (t == 0 ? kt[0]++ : kt[1]++) & 1));
            if (!ok) break;
            tc_fence_after_sync();
#pragma unroll
            for (int kk = 0; kk < D / 16; ++kk)
              tc_mma_bf16(tmem + (2 * t + sb) * kBK,
                          q_desc + ((t * kQBytes + (kk >> 2) * kQHalf + (kk & 3) * 32) >> 4),
                          kd + (((kk >> 2) * kKHalf + (kk & 3) * 32) >> 4), idS, kk > 0 ? 1u : 0u);
            tc_commit(&T->s_full[t][sb]);
          }
          tc_commit(&T->kv_empty[slot]);
        }
        tc_commit(&T->q_empty);
      }
      if (!ok) give_up();
      tc_commit(&T->done);
      volatile int never = 0;
      (void)mbar_wait_bounded(&T->done, 0, &never, kLimitNs);
    } else if (warp == 2 && lane == 0) {
      // ---------------- PV issuer ----------------
      constexpr uint32_t idO = idesc_f16(128, D) | (1u << 16);   // B MN-major
      const uint64_t v_desc = desc_mnmajor_sw128(smem_u32(skv), kKHalf, 1024);
      int g = 0, gt[2] = {0, 0}, kt[2] = {0, 0};   // blocks, of each tile; pieces of each
      bool ok = true;
      volatile int* blocks = &T->blocks;
      Piece it;
      for (int k = 0; ok; ++k) {
        if (!(ok = fetch_one(k, it)) || it.nblk == 0) break;
        const int tiles = it.n_rows > a.tile_rows ? 2 : 1;
        for (int b = it.b0; ok && b < it.b1; ++b, ++g) {
          const int slot = (2 * g + 1) % kSlots;
          if (!(ok = wait_one(T, &T->kv_full[slot], ((2 * g + 1) / kSlots) & 1))) break;
          const uint64_t vd = v_desc + slot * (kKBytes >> 4);
#pragma unroll 1
          for (int t = 0; t < tiles; ++t) {
            const int n = t == 0 ? gt[0]++ : gt[1]++, sb = n & 1;
            ok = wait_one(T, &T->p_full[t][sb], (n >> 1) & 1) &&
                 (b > it.b0 ||                     // the last piece's O has been read
                  wait_one(T, &T->o_empty[t], ((t == 0 ? kt[0]++ : kt[1]++) & 1) ^ 1));
            if (!ok) break;
            tc_fence_after_sync();
#pragma unroll
            for (int kk = 0; kk < kBK / 16; ++kk)
              tc_mma_tmem_a(tmem + kOCol + t * D, tmem + (2 * t + sb) * kBK + kk * 8,
                            vd + ((16 * kk * 128) >> 4), idO, (b > it.b0 || kk > 0) ? 1u : 0u);
            tc_commit(&T->p_empty[t][sb]);
            if (b + 1 == it.b1) tc_commit(&T->o_full[t]);
          }
          *blocks = g + 1;
          tc_commit(&T->kv_empty[slot]);
        }
      }
      if (!ok) give_up();
      tc_commit(&T->done);
      volatile int never = 0;
      (void)mbar_wait_bounded(&T->done, 0, &never, kLimitNs);
    } else if (warp == 0) {
      // ---------------- planner ----------------
      int k = 0;
      auto post = [&](const Piece& it) -> bool {   // lane 0 writes the k-th piece
        const int s = k % kItemRing;
        if (!wwait_long(T, &T->item_empty[s], ((k / kItemRing) & 1) ^ 1)) return false;
        if (lane < PCTREE_ATTN_MAX_N / 32) T->bad[s][lane] = 0;
        __syncwarp();
        if (lane == 0) {
          T->item[s] = it;
          mbar_arrive(&T->item_full[s]);
        }
        __syncwarp();
        ++k;
        return true;
      };
      PieceJoin join;
      bool ok = plan_pieces(a.units, T->upto, join, post);
      if (lane == 0) a.join[blockIdx.x] = join;
      if (ok) {
        Piece end = {};
        ok = post(end);
      }
      if (!ok && lane == 0) give_up();
    } else if (warp == 3) {
      // ---------------- places and scales of the keys ----------------
      // Two keys a lane.  Page numbers are read a block ahead of their use, and a
      // block's scales are under way while the block before it is written down.
      constexpr int kKeys = kBK / 32;
      const KvRows& rows = a.units.rows;
      const int Hkv = a.units.Hkv;
      Piece it;
      int k = 0, b = 0, left = 0;                  // pieces fetched; block, blocks left of it
      bool ok = true;
      struct Block {
        int r, kvh, key0, key_end, all, ring;
      };
      auto next_block = [&](Block& x) {            // no keys: no more
        x = Block{};
        if (left == 0) {
          if (k < 0 || !ok) return;
          if (!(ok = peek_warp(k, it))) return;
          release_warp(k);
          if (it.nblk == 0) {
            k = -1;
            return;
          }
          ++k;
          b = it.b0;
          left = it.b1 - it.b0;
        }
        x.r = it.r;
        x.kvh = it.kvh;
        x.key0 = b * kBK;
        x.key_end = it.key_end;
        x.all = a.parent != nullptr ? it.prefix : it.prefix + it.j0 + 1;
        x.ring = (k - 1) % kItemRing;
        ++b;
        --left;
      };
      int page[kKeys];                             // of the block whose scales come next
      auto find_pages = [&](const Block& x) {
#pragma unroll
        for (int i = 0; i < kKeys; ++i) {
          const int key = x.key0 + i * 32 + lane;
          page[i] = key < x.key_end ? kv_page(rows, x.r, div_by(key, a.blocks.page)) : -2;
        }
      };
      uint32_t sk[kKeys], sv[kKeys];               // scales' bytes, under way
      Block cur;
      next_block(cur);
      find_pages(cur);
      for (int g = 0; ok; ++g) {
        // the g-th block's places (without keys: the end); then the scales of the
        // block before it, which are there by now
        const int st = g % kPlaceRing;
        if (!(ok = wwait(T, &T->place_empty[st], ((g / kPlaceRing) & 1) ^ 1))) break;
        uint32_t tk[kKeys], tv[kKeys];
#pragma unroll
        for (int i = 0; i < kKeys; ++i) {
          uint32_t at = kNowhere;
          tk[i] = tv[i] = kExpBias;
          if (page[i] >= 0) {
            const int key = cur.key0 + i * 32 + lane;
            const int off = key - div_by(key, a.blocks.page) * rows.page_size;
            at = (static_cast<uint32_t>(page[i]) * rows.page_size + off) * Hkv + cur.kvh;
            const long long sc = (static_cast<long long>(page[i]) * a.blocks.per_page +
                                  (off >> a.blocks.shift)) * Hkv + cur.kvh;
            tk[i] = __ldg(a.scale[0] + sc);
            tv[i] = __ldg(a.scale[1] + sc);
          } else if (page[i] == -1) {
            report(a.status, PCTREE_ERR_INVALID_ARG);
          }
          T->places[st].at[i * 32 + lane] = at;
        }
        const bool end = cur.key_end == 0;
        if (lane == 0) {
          T->places[st].key0 = cur.key0;
          T->places[st].all = cur.all;
          T->places[st].ring = cur.ring;
          T->places[st].keys = end ? 0 : kBK;
        }
        if (!end) {
          next_block(cur);
          if (!ok) break;
          find_pages(cur);
        }
        if (g > 0) {
          Places& p = T->places[(g - 1) % kPlaceRing];
          bool fine = true;
#pragma unroll
          for (int i = 0; i < kKeys; ++i) {
            p.by[i * 32 + lane] = half_exp(scale_exp(sk[i])) |
                                  static_cast<uint32_t>(half_exp(scale_exp(sv[i]))) << 16;
            fine = fine && scale_ok(sk[i]) && scale_ok(sv[i]);
          }
          if (!fine) report(a.status, PCTREE_ERR_INVALID_ARG);
          __syncwarp();
          if (lane == 0) mbar_arrive(&T->place_full[(g - 1) % kPlaceRing]);
        }
        if (end) {
          __syncwarp();
          if (lane == 0) mbar_arrive(&T->place_full[st]);
          break;
        }
#pragma unroll
        for (int i = 0; i < kKeys; ++i) {
          sk[i] = tk[i];
          sv[i] = tv[i];
        }
      }
      if (!ok && lane == 0) give_up();
    }
  } else if (warp < 8) {
    // ---------------- Q in, O out ----------------
    const uint32_t tmem = T->tmem_base;
    const int quad = warp & 3;
    const int t = quad * 32 + lane;
    const int R = a.G * a.tile_rows;
    uint8_t* stg = T->stage[quad];
    // a barrier of these four warps that gives up as other waits do
    int syncs = 0;
    auto together = [&]() -> bool {
      __syncwarp();
      if (lane == 0) mbar_arrive(&T->out_sync);
      return wwait(T, &T->out_sync, syncs++ & 1);
    };
    // the k-th piece's tiles; false: given up
    auto bring_q = [&](int k, const Piece& it) -> bool {
      const int qb = k & 1;
      constexpr int kLanes = D / 8;                // lanes of a row
      constexpr int kRows = 128 / kLanes;          // rows at a time
      const int c = t % kLanes;
      const int rows = it.n_rows * a.G;            // of both tiles, one behind the other
      const uint16_t* q = a.q + it.row0 * a.q_stride + it.kvh * a.G * D + c * 8;
      auto place_of = [&](int row) {               // of a row of the unit
        const int n = div_by(row, a.by_G);
        return reinterpret_cast<const uint8_t*>(q + n * a.q_stride + (row - n * a.G) * D);
      };
      if (!wwait_long(T, &T->q_empty, (k & 1) ^ 1)) return false;
      // rows past the last one's are zeros up to the end of their tile
      const int all = it.n_rows > a.tile_rows ? 2 * R : R;
#pragma unroll 2
      for (int row = t / kLanes; row < all; row += kRows) {
        const int tile = row >= R ? 1 : 0, in = row - tile * R;
        copy16_if(row < rows,
                  sq + tile * kQBytes + (c >> 3) * kQHalf + in * 128 + (((c & 7) ^ (in & 7)) * 16),
                  place_of(min(row, rows - 1)));
      }
      copies_commit();
      if (a.parent != nullptr) {
        // ancestors of the unit's rows, from the parents of the request's first rows
        const int n = it.j0 + it.n_rows;
        const int32_t* parent = a.parent + it.row0 - it.j0;
        if (!together()) return false;
        for (int i = t; i < n; i += 128) {
          int p = parent[i];
          if (p < -1 || p >= i) {                  // parents precede children
            report(a.status, PCTREE_ERR_INVALID_ARG);
            p = -1;
          }
          T->par[i] = static_cast<int16_t>(p);
        }
        if (!together()) return false;
        for (int j = t; j < it.n_rows; j += 128) {
          uint32_t* path = T->path[qb][j];
          for (int i = 0; i < PCTREE_ATTN_MAX_N / 32; ++i) path[i] = 0;
          for (int m = it.j0 + j; m >= 0; m = T->par[m]) path[m >> 5] |= 1u << (m & 31);
        }
      }
      copies_wait<0>();
      fence_proxy_async_smem();
      __syncwarp();
      if (lane == 0) mbar_arrive(&T->q_raw[k % kItemRing]);
      return true;
    };
    Piece it;
    bool ok = peek_warp(0, it);
    if (ok && it.nblk != 0) ok = bring_q(0, it);
    int kt[2] = {0, 0};                            // pieces of each tile
    for (int k = 0; ok && it.nblk != 0; ++k) {
      Piece next;
      if (!(ok = peek_warp(k + 1, next))) break;
      if (next.nblk != 0 && !(ok = bring_q(k + 1, next))) break;
      const bool whole = it.b0 == 0 && it.b1 == it.nblk;
      const int ring = k % kItemRing;
      const size_t part = static_cast<size_t>(blockIdx.x) * 2 + (it.b0 == 0 ? 1 : 0);
      const int tiles = it.n_rows > a.tile_rows ? 2 : 1;
#pragma unroll 1
      for (int tile = 0; tile < tiles; ++tile) {
        if (!(ok = wwait_long(T, &T->o_full[tile], (tile == 0 ? kt[0]++ : kt[1]++) & 1))) break;
        tc_fence_after_sync();
        uint32_t any_bad = 0;
        for (int i = 0; i < PCTREE_ATTN_MAX_N / 32; ++i) any_bad |= T->bad[ring][i];
        const int nl = tile * a.tile_rows + div_by(t, a.by_G);   // row of the unit
        const int n_end = min(it.n_rows, (tile + 1) * a.tile_rows);
        // (rows of the next tile lie past this one's R)
        const bool in_tile = t < R && nl < n_end;
        const float l = T->row_l[tile][t];
        const float inv = whole ? 1.0f / l : 1.0f;   // (no finite score, l = 0: NaN)
        const int slot = tile * R + t;               // of the unit's rows
        if (!whole && in_tile)
          a.part_ml[part * kUnitRows + slot] =
              make_float2(l != 0.0f ? T->row_m[tile][t] : -INFINITY, l);
        const uint32_t o_col = tmem + (static_cast<uint32_t>(quad * 32) << 16) + kOCol + tile * D;
#pragma unroll 1
        for (int c = 0; c < D / 16; ++c) {
          uint32_t y[16];
          tmem_ld_32x32b_x16(o_col + c * 16, y);
          tmem_ld_wait();
          float f[16];
#pragma unroll
          for (int i = 0; i < 16; ++i) f[i] = __uint_as_float(y[i]) * inv;
          if (l == 0.0f && !whole) {
#pragma unroll
            for (int i = 0; i < 16; ++i) f[i] = 0.0f;
          }
          if (any_bad != 0) {
            // NaN values that were taken out of V reach the rows that see their keys:
            // the codes are looked at once more
            const int first = a.parent != nullptr ? it.prefix : it.prefix + it.j0 + 1;
            uint32_t nan = 0;
            for (int i = 0; i < PCTREE_ATTN_MAX_N / 32; ++i) {
              uint32_t keys = T->bad[ring][i] &
                              (a.parent != nullptr     ? T->path[k & 1][min(nl, 255)][i]
                               : nl >= 32 * (i + 1) ? ~0u
                               : nl > 32 * i        ? (1u << (nl - 32 * i)) - 1
                                                    : 0u);
              for (; in_tile && keys != 0; keys &= keys - 1) {
                const int key = first + 32 * i + __ffs(keys) - 1;
                const int entry = div_by(key, a.blocks.page);
                const long long at =
                    (static_cast<long long>(kv_page(a.units.rows, it.r, entry)) *
                         a.units.rows.page_size + key - entry * a.units.rows.page_size) *
                        a.units.Hkv + it.kvh;
                // (a page that is none has no NaN)
                nan |= nan_bits(__ldg(reinterpret_cast<const uint4*>(a.cache[1] + at * D + c * 16)));
              }
            }
#pragma unroll
            for (int i = 0; i < 16; ++i)
              if ((nan >> i) & 1u) f[i] = __int_as_float(0x7fc00000);
            __syncwarp();
          }
          if (c == D / 16 - 1) {
            tc_fence_before_sync();
            __syncwarp();
            if (lane == 0) mbar_arrive(&T->o_empty[tile]);
          }
          if (!whole) {
            float4* po =
                reinterpret_cast<float4*>(a.part_o) + (part * (D / 4) + c * 4) * kUnitRows + slot;
            if (in_tile) {
#pragma unroll
              for (int i = 0; i < 4; ++i)
                po[i * kUnitRows] = make_float4(f[4 * i], f[4 * i + 1], f[4 * i + 2], f[4 * i + 3]);
            }
            continue;
          }
          // through shared memory: two neighbouring lanes store a row's 32 bytes
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            uint32_t w[4];
#pragma unroll
            for (int h = 0; h < 4; ++h) w[h] = pack16<F16>(f[i * 8 + 2 * h], f[i * 8 + 2 * h + 1]);
            *reinterpret_cast<uint4*>(stg + lane * 32 + ((i ^ (lane >> 2)) & 1) * 16) =
                make_uint4(w[0], w[1], w[2], w[3]);
          }
          __syncwarp();
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            const int row = 16 * i + (lane >> 1), ti = quad * 32 + row, ni = div_by(ti, a.by_G);
            const uint4 v = *reinterpret_cast<const uint4*>(
                stg + row * 32 + (((lane & 1) ^ (row >> 2)) & 1) * 16);
            if (ti < R && tile * a.tile_rows + ni < n_end)
              *reinterpret_cast<uint4*>(
                  a.out + ((static_cast<size_t>(it.row0) + tile * a.tile_rows + ni) * a.Hq +
                           it.kvh * a.G + ti - ni * a.G) * D + c * 16 + (lane & 1) * 8) = v;
          }
          __syncwarp();
        }
      }
      // (a piece's ancestors are read up to here: they are replaced after)
      if (!ok || !(ok = together())) break;
      release_warp(k);
      it = next;
    }
    copies_wait<0>();                              // copies land before the CTA may exit
    if (!ok && lane == 0) give_up();
  } else if (warp < 16) {
    // ---------------- softmax, a thread per row of a tile ----------------
    set_registers_up<kRegsSoftmax>();
    const uint32_t tmem = T->tmem_base;
    const int tile = (warp - 8) >> 2;
    const int quad = warp & 3;
    const int t = quad * 32 + lane;
    const int nl = tile * a.tile_rows + div_by(t, a.by_G);     // row of the unit
    const uint32_t lane_base = tmem + (static_cast<uint32_t>(quad * 32) << 16);
    const uint32_t o_col = lane_base + kOCol + tile * D;
    int g = 0, kt = 0;                             // this tile's blocks and pieces
    bool ok = true;
    Piece it;
    for (int k = 0; ok; ++k) {
      if (!(ok = peek_warp(k, it))) break;
      if (it.nblk == 0) {
        release_warp(k);
        break;
      }
      if (!(ok = wwait_long(T, &T->q_raw[k % kItemRing], (k / kItemRing) & 1))) break;
      release_warp(k);
      if (it.n_rows <= tile * a.tile_rows) continue;
      float sc = a.scale_log2;
      if constexpr (!F16) {
        // this warp's 32 rows of the tile to float16, the row's largest to 2^14 .. 2^15
        constexpr int kLanes = D / 8, kRows = 32 / kLanes;
        const int c = lane % kLanes;
#pragma unroll 2
        for (int r0 = 0; r0 < 32; r0 += kRows) {
          const int row = quad * 32 + r0 + lane / kLanes;
          uint4* at = reinterpret_cast<uint4*>(sq + tile * kQBytes + (c >> 3) * kQHalf + row * 128 +
                                               (((c & 7) ^ (row & 7)) * 16));
          const uint4 x = *at;
          uint32_t w[4] = {x.x, x.y, x.z, x.w};
          // (magnitudes of bfloat16 are ordered as the integers they are)
          uint32_t top2 = 0;
#pragma unroll
          for (int i = 0; i < 4; ++i) top2 = __vmaxu2(top2, w[i] & 0x7fff7fffu);
#pragma unroll
          for (int o = kLanes / 2; o > 0; o >>= 1)
            top2 = __vmaxu2(top2, __shfl_xor_sync(kFull, top2, o));
          const int top = static_cast<int>(max(top2 >> 16, top2 & 0xffffu) >> 7) - 127;
          // (a row with an infinity or NaN is NaN in the end, whatever its others are)
          const int e = max(-100, min(126, top)) - 14;
          const float by = exp2_of(-e);
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float2 f = unpack16<false>(w[i]);
            w[i] = pack16<true>(f.x * by, f.y * by);
          }
          *at = make_uint4(w[0], w[1], w[2], w[3]);
          if (c == 0) T->row_scale[tile][row] = row_scale(a.scale_log2, e);
        }
        fence_proxy_async_smem();
        __syncwarp();
        sc = T->row_scale[tile][t];
      }
      if (lane == 0) mbar_arrive(&T->q_full[tile]);
      // keys this row sees: slots below `end`, and of those from the prefix on (in
      // a tree) its ancestors
      const int end = min(it.key_end, it.prefix + it.j0 + nl + 1);
      float m_used = -INFINITY, l_sum = 0.0f;
      float over = -INFINITY;                      // a maximum above it needs a look
      for (int b = it.b0; b < it.b1; ++b, ++g) {
        const int sb = g & 1;
        const int key0 = b * kBK;
        const int seen = end - key0;
        uint64_t see = seen >= 64 ? ~0ull : seen <= 0 ? 0ull : (1ull << seen) - 1;
        if (a.parent != nullptr && key0 + 64 > it.prefix && see != 0) {
          const int node = key0 - it.prefix;       // > -64: the first key's place in the tree
          const uint32_t* path = T->path[k & 1][min(nl, 255)];
          auto word = [&](int i) -> uint64_t {
            return i >= 0 && i < PCTREE_ATTN_MAX_N / 32 ? path[i] : 0u;
          };
          const int w0 = node >> 5, sh = node & 31;
          const uint64_t lo = word(w0) | word(w0 + 1) << 32, hi = word(w0 + 2);
          uint64_t anc = sh == 0 ? lo : lo >> sh | hi << (64 - sh);
          if (node < 0) anc |= (1ull << -node) - 1;   // slots of the prefix
          see &= anc;
        }
        if (!(ok = wwait(T, &T->s_full[tile][sb], (g >> 1) & 1))) break;
        tc_fence_after_sync();
        const uint32_t s_col = lane_base + (2 * tile + sb) * kBK;
        float x[64];
        bool shifted = false;
        // The scores, and once more if the reference has moved: the rescaling of O
        // takes their registers.  (Loops, not copies of the code: instructions that
        // run rarely come from memory.)
#pragma unroll 1
        for (bool again = false;; again = true) {
          uint32_t* xu = reinterpret_cast<uint32_t*>(x);
#pragma unroll
          for (int c = 0; c < 2; ++c)
            tmem_ld_32x32b_x32(s_col + c * 32,
                               *reinterpret_cast<uint32_t(*)[32]>(xu + c * 32));
          tmem_ld_wait();
          // keys the row may not see become -inf
          if (__any_sync(kFull, see != ~0ull)) {
            const uint32_t s0 = static_cast<uint32_t>(see), s1 = static_cast<uint32_t>(see >> 32);
#pragma unroll
            for (int i = 0; i < 32; ++i) {
              x[i] = (s0 >> i) & 1u ? x[i] : -INFINITY;
              x[32 + i] = (s1 >> i) & 1u ? x[32 + i] : -INFINITY;
            }
          }
          if (again) break;
          float m8[8];
#pragma unroll
          for (int u = 0; u < 8; ++u) m8[u] = x[u];
#pragma unroll
          for (int k2 = 8; k2 < 64; ++k2) m8[k2 & 7] = fmaxf(m8[k2 & 7], x[k2]);
          const float mx = fmaxf(fmaxf(fmaxf(m8[0], m8[1]), fmaxf(m8[2], m8[3])),
                           fmaxf(fmaxf(m8[4], m8[5]), fmaxf(m8[6], m8[7]))) * sc;
          if (!__any_sync(kFull, mx > over)) break;
          const bool mine = mx > m_used + 8.0f;
          const float alpha = mine ? ex2_approx(m_used - mx) : 1.0f;
          if (b > it.b0) {
            if (!(ok = wwait(T, &T->p_empty[tile][(g - 1) & 1], ((g - 1) >> 1) & 1))) break;
            tc_fence_after_sync();
            const uint64_t alpha2 = pack2(alpha, alpha);
#pragma unroll 1
            for (int c = 0; c < D; c += 32) {
              uint32_t y[32];
              tmem_ld_32x32b_x32(o_col + c, y);
              tmem_ld_wait();
#pragma unroll
              for (int k2 = 0; k2 < 32; k2 += 2) {
                float y0, y1;
                unpack2(mul2(pack2(__uint_as_float(y[k2]), __uint_as_float(y[k2 + 1])), alpha2),
                        y0, y1);
                y[k2] = __float_as_uint(y0);
                y[k2 + 1] = __float_as_uint(y1);
              }
              tmem_st_32x32b_x32(o_col + c, y);
            }
            tmem_st_wait();
          }
          if (mine) {
            l_sum *= alpha;
            m_used = mx;
          }
          const bool wide = fabsf(m_used) > kWideScore && m_used > -INFINITY;
          over = wide ? -INFINITY : m_used + 8.0f;
          shifted = __any_sync(kFull, wide);
          if (shifted) wide_scores(s_col, sc, m_used == -INFINITY ? 0.0f : m_used, see);
        }
        if (!ok) break;
        const float mref = (shifted || m_used == -INFINITY ? 0.0f : m_used) - kPBits;
        const uint64_t sc2 = pack2(sc, sc), nm2 = pack2(-mref, -mref);
        uint64_t ls[4] = {0, 0, 0, 0};
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          uint32_t pk[16];
#pragma unroll
          for (int h = 0; h < 16; ++h) {
            float e0, e1;
            unpack2(fma2(pack2(x[c * 32 + 2 * h], x[c * 32 + 2 * h + 1]), sc2, nm2), e0, e1);
            const float p0 = ex2_approx(e0), p1 = ex2_approx(e1);
            ls[h & 3] = add2(ls[h & 3], pack2(p0, p1));
            pk[h] = pack16<true>(p0, p1);
          }
          tmem_st_x16(s_col + c * 16, pk);
        }
        tmem_st_wait();
        {
          float s0, s1;
          unpack2(add2(add2(ls[0], ls[1]), add2(ls[2], ls[3])), s0, s1);
          l_sum += s0 + s1;
        }
        tc_fence_before_sync();
        __syncwarp();
        if (lane == 0) mbar_arrive(&T->p_full[tile][sb]);
      }
      if (!ok) break;
      if (!(ok = wwait(T, &T->o_empty[tile], (kt++ & 1) ^ 1))) break;
      T->row_l[tile][t] = l_sum;
      T->row_m[tile][t] = m_used;
      __syncwarp();
      if (lane == 0) mbar_arrive(&T->o_full[tile]);
    }
    if (!ok && lane == 0) give_up();
  } else {
    // ---------------- K or V: codes to float16 ----------------
    set_registers_down<kRegsConvert>();
    const int is_v = (warp - 16) >> 2, wq = warp & 3;
    const uint8_t* cache = a.cache[is_v];
    constexpr int kRows = 128 / (D / 16);          // rows the four warps bring at a time
    constexpr int kU = kBK / kRows;                // rows a thread brings of a block
    // 16 bytes of a row a lane; eight neighbouring lanes have four groups of one
    // half of two neighbouring rows, whose 16-byte places in the swizzled tile are
    // all different
    const int c4 = lane & 3;                       // group of 16 dims in its half
    const int half = kHalves == 2 ? (lane >> 3) & 1 : 0;
    const int row_in = wq * (kRows / 4) + ((lane >> 2) & 1) +
                       2 * (kHalves == 2 ? lane >> 4 : lane >> 3);
    const int dim0 = half * 64 + c4 * 16;
    // (rows kRows apart are multiples of 8 apart: the same swizzle)
    uint8_t* mine = skv + half * kKHalf + row_in * 128;
    const int lo16 = ((2 * c4) ^ (row_in & 7)) * 16, hi16 = ((2 * c4 + 1) ^ (row_in & 7)) * 16;
    uint8_t* raw = codes + is_v * kAhead * kCodeBytes + (threadIdx.x & 127) * 16;
    cache += dim0;
    // codes of a block's rows on their way (one group of copies)
    auto load = [&](const Places& p, uint8_t* dst) {
#pragma unroll
      for (int u = 0; u < kU; ++u) {
        const uint32_t at = p.at[u * kRows + row_in];
        const bool is = at != kNowhere;
        copy16_if(is, dst + u * 128 * 16, cache + static_cast<size_t>(is ? at : 0) * D);
      }
      copies_commit();
    };
    // places of the g-th block, if there is one (past the end: an empty group)
    bool ok = true, more = true;
    auto ahead = [&](int g) -> bool {
      if (more) {
        const int st = g % kPlaceRing;
        if (!wwait_long(T, &T->place_full[st], (g / kPlaceRing) & 1)) return false;
        more = T->places[st].keys > 0;
        if (more) {
          load(T->places[st], raw + (g % kAhead) * kCodeBytes);
          return true;
        }
      }
      copies_commit();
      return true;
    };
    int n = 0;                                     // blocks whose codes are under way or here
    for (; ok && n < kAhead; ++n) {
      ok = ahead(n);
      if (!more) break;
    }
    int total = more ? 1 << 30 : n;
    if (!more)
      for (int i = n; i < kAhead; ++i) copies_commit();
    for (int g = 0; ok && g < total; ++g) {
      const Places& cur = T->places[g % kPlaceRing];
      const int place = 2 * g + is_v, slot = place % kSlots;
      if (!(ok = wwait(T, &T->kv_empty[slot], ((place / kSlots) & 1) ^ 1))) break;
      copies_wait<kAhead - 1>();
      const uint8_t* src = raw + (g % kAhead) * kCodeBytes;
      uint4 x[kU];
      uint32_t by[kU];
#pragma unroll
      for (int u = 0; u < kU; ++u) {
        x[u] = *reinterpret_cast<const uint4*>(src + u * 128 * 16);
        by[u] = (cur.by[u * kRows + row_in] >> (16 * is_v) & 0xffffu) * 0x10001u;
      }
      if (is_v != 0 && cur.key0 + kBK > cur.all) {
        // keys that not every row sees: their NaN values are taken out, the keys noted
#pragma unroll
        for (int u = 0; u < kU; ++u) {
          const int key = cur.key0 + u * kRows + row_in - cur.all;
          if (key >= 0 && any_nan(x[u])) x[u] = without_nan(x[u], T, cur.ring, key);
        }
      }
      uint8_t* dst = mine + slot * kKBytes;
#pragma unroll
      for (int u = 0; u < kU; ++u) {
        const uint32_t w[4] = {x[u].x, x[u].y, x[u].z, x[u].w};
        uint32_t h[8];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          h[2 * i] = mul_h2(halves2(w[i]), by[u]);
          h[2 * i + 1] = mul_h2(halves2(w[i] >> 16), by[u]);
        }
        *reinterpret_cast<uint4*>(dst + u * kRows * 128 + lo16) =
            make_uint4(h[0], h[1], h[2], h[3]);
        *reinterpret_cast<uint4*>(dst + u * kRows * 128 + hi16) =
            make_uint4(h[4], h[5], h[6], h[7]);
      }
      fence_proxy_async_smem();
      __syncwarp();
      if (lane == 0) {
        mbar_arrive(&T->kv_full[slot]);
        mbar_arrive(&T->place_empty[g % kPlaceRing]);
      }
      if (total == 1 << 30) {
        ok = ahead(g + kAhead);
        if (!more) total = g + kAhead;
      } else {
        copies_commit();
      }
    }
    copies_wait<0>();                              // copies land before the CTA may exit
    if (!ok && lane == 0) give_up();
  }
  // ---------------- teardown ----------------
  __syncwarp();
  tc_fence_before_sync();
  __syncthreads();
  tc_fence_after_sync();
  if (warp == 1) tmem_dealloc(T->tmem_base, kTmemCols);
}

// Rows per unit: one where requests have one row each, on average (a tile's rows
// are multiplied whether or not they are the request's), else as many as fit in two
// tiles.
int rows_per_tile(const pctree_kv8_attn_config& c) { return 128 / (c.Hq / c.Hkv); }
int rows_per_unit(const pctree_kv8_attn_config& c) {
  const int fit = 2 * rows_per_tile(c);
  return c.total_rows <= c.batch ? 1 : fit < c.total_rows ? fit : c.total_rows;
}

// Whether the planner can count the most work a configuration can have in 32
// bits.
bool work_ok(const pctree_kv8_attn_config& c) {
  const long long units = c.total_rows / rows_per_unit(c) + 1ll + c.batch;
  const long long blocks =
      (static_cast<long long>(c.max_pages) * c.page_size + kBK - 1) / kBK + kUnitCharge;
  return units * blocks < (1ll << 32) / c.Hkv - 1024;
}

// Whether a 32-bit number tells all heads of all slots apart (a plane of 2^32 heads
// of 64 codes alone would fill the memory of a GB300).
bool places_ok(const pctree_kv8_attn_config& c) {
  return static_cast<long long>(c.n_pages) * c.page_size <= 0xfffffffell / c.Hkv;
}

pctree_status attn8_check(const pctree_kv8_attn_config* c) {
  if (c == nullptr) return PCTREE_ERR_INVALID_ARG;
  if (c->Hq < 1 || c->D < 1 || !(c->scale > 0.0f) || !(c->scale < 1e30f))
    return PCTREE_ERR_INVALID_ARG;
  const pctree_status st = kv_check(c->batch, c->total_rows, c->Hkv, c->page_size, c->n_pages,
                                    c->max_pages, c->dtype);
  if (st != PCTREE_OK) return st;
  if (!kv8_block_ok(c->scale_block) || c->Hq % c->Hkv != 0 || c->q_stride % 8 != 0 ||
      c->q_stride < static_cast<int64_t>(c->Hq) * c->D)
    return PCTREE_ERR_INVALID_ARG;
  if ((c->D != 64 && c->D != 128) || c->Hq / c->Hkv > 128 || c->q_stride > (1ll << 38) ||
      !work_ok(*c) || !places_ok(*c))
    return PCTREE_ERR_UNSUPPORTED;
  return PCTREE_OK;
}

// Whether a tile of one row's heads fits the token kernel.
bool takes_tokens(const pctree_kv8_attn_config& c) {
  return rows_per_unit(c) == 1 && c.Hq / c.Hkv <= kTokenHeads;
}

template <int D, bool F16>
pctree_status attn8_launch(const Kv8AttnArgs& a, bool tokens, int num_sms, cudaStream_t stream) {
  constexpr size_t smem = (D / 64) * static_cast<size_t>(2 * kQHalf + kSlots * kKHalf) +
                          2 * kAhead * static_cast<size_t>(kBK) * D + sizeof(Tail) + 1024;
  static_assert(smem <= 227 * 1024, "shared memory per CTA");
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cudaLaunchConfig_t lc = {};
  const unsigned ctas = static_cast<unsigned>(num_sms < kMaxCtas ? num_sms : kMaxCtas);
  lc.gridDim = dim3(ctas);
  lc.stream = stream;
  lc.attrs = attr;
  lc.numAttrs = 1;
  if (tokens) {
    const cudaError_t e = a.G <= 8 ? launch_tokens<D, F16, 1>(lc, a) : launch_tokens<D, F16, 2>(lc, a);
    if (e != cudaSuccess) return PCTREE_ERR_CUDA;
  } else {
    static SmemLimit limit;
    const void* fn = reinterpret_cast<const void*>(kv8_attn_kernel<D, F16>);
    if (limit.ensure(fn, smem) != cudaSuccess) return PCTREE_ERR_CUDA;
    // (a launch with fewer registers would leave the softmax waiting for its own; a
    // query that fails is asked again by the next call)
    static std::atomic<bool> registers{false};
    if (!registers.load(std::memory_order_relaxed)) {
      cudaFuncAttributes f;
      if (cudaFuncGetAttributes(&f, fn) != cudaSuccess) {
        (void)cudaGetLastError();
        return PCTREE_ERR_CUDA;
      }
      if (f.numRegs < kRegsLaunch) return PCTREE_ERR_CUDA;
      registers.store(true, std::memory_order_relaxed);
    }
    lc.blockDim = dim3(kThreads);
    lc.dynamicSmemBytes = smem;
    if (cudaLaunchKernelEx(&lc, kv8_attn_kernel<D, F16>, a) != cudaSuccess) return PCTREE_ERR_CUDA;
  }
  const JoinArgs j = {a.part_o, a.part_ml, a.join, a.out, a.G, a.Hq};
  lc.gridDim = dim3(ctas, kJoinCtas);
  lc.blockDim = dim3(kJoinThreads);
  lc.dynamicSmemBytes = 0;
  return cudaLaunchKernelEx(&lc, join_pieces_kernel<D, F16>, j) == cudaSuccess ? PCTREE_OK
                                                                              : PCTREE_ERR_CUDA;
}

}  // namespace
}  // namespace pct

extern "C" {

size_t pctree_kv8_attention_workspace_bytes(const pctree_kv8_attn_config* cfg) {
  if (pct::attn8_check(cfg) != PCTREE_OK) return 0;
  return pct::piece_ws(cfg->D).total;
}

pctree_status pctree_kv8_attention(const pctree_kv8_attn_config* cfg, const void* q,
                                   const void* k_cache, const void* v_cache, const void* k_scale,
                                   const void* v_scale, const int32_t* row_start,
                                   const int32_t* n_rows, const int32_t* prefix_len,
                                   const int32_t* page_table, const int32_t* parent, void* out,
                                   void* workspace, size_t workspace_bytes, int32_t* status,
                                   void* stream_ptr) {
  using namespace pct;
  NvtxRange range("pctree_kv8_attention");
  pctree_status st = attn8_check(cfg);
  if (st != PCTREE_OK) return st;
  const pctree_kv8_attn_config& c = *cfg;
  if (q == nullptr || k_cache == nullptr || v_cache == nullptr || k_scale == nullptr ||
      v_scale == nullptr || row_start == nullptr || n_rows == nullptr || prefix_len == nullptr ||
      out == nullptr || !kv_al16(q) || !kv_al16(k_cache) || !kv_al16(v_cache) || !kv_al16(out) ||
      !kv_table_ok(page_table, c.batch, c.n_pages, c.max_pages))
    return PCTREE_ERR_INVALID_ARG;
  {
    const char* q0 = static_cast<const char*>(q);
    const char* q1 = q0 + ((c.total_rows - 1) * static_cast<size_t>(c.q_stride) +
                           static_cast<size_t>(c.Hq) * c.D) * 2;
    const char* o0 = static_cast<const char*>(out);
    const char* o1 = o0 + static_cast<size_t>(c.total_rows) * c.Hq * c.D * 2;
    if (q0 < o1 && o0 < q1) return PCTREE_ERR_INVALID_ARG;   // overlap
  }
  const PieceWs w = piece_ws(c.D);
  if (workspace == nullptr || workspace_bytes < w.total ||
      (reinterpret_cast<uintptr_t>(workspace) & 255u) != 0)
    return PCTREE_ERR_WORKSPACE;
  int num_sms = 0;
  st = device_facts(&num_sms);
  if (st != PCTREE_OK) return st;
  Kv8AttnArgs a{};
  a.units = {{row_start, n_rows, prefix_len, page_table, c.batch, c.total_rows, c.page_size,
              c.n_pages, c.max_pages},
             c.Hkv, rows_per_unit(c), parent != nullptr ? PCTREE_ATTN_MAX_N : 1 << 30, kBK};
  a.blocks = kv8_blocks(c.page_size, c.scale_block);
  a.q = static_cast<const uint16_t*>(q);
  a.cache[0] = static_cast<const uint8_t*>(k_cache);
  a.cache[1] = static_cast<const uint8_t*>(v_cache);
  a.scale[0] = static_cast<const uint8_t*>(k_scale);
  a.scale[1] = static_cast<const uint8_t*>(v_scale);
  a.parent = parent;
  a.out = static_cast<uint16_t*>(out);
  unsigned char* ws = static_cast<unsigned char*>(workspace);
  a.part_o = reinterpret_cast<float*>(ws + w.part_o);
  a.part_ml = reinterpret_cast<float2*>(ws + w.part_ml);
  a.join = reinterpret_cast<PieceJoin*>(ws + w.join);
  a.status = status;
  a.q_stride = c.q_stride;
  a.Hq = c.Hq;
  a.G = c.Hq / c.Hkv;
  a.by_G = fast_div(a.G);
  a.tile_rows = std::min(rows_per_tile(c), a.units.npt);
  a.scale_log2 = static_cast<float>(static_cast<double>(c.scale) * 1.4426950408889634);
  cudaStream_t stream = static_cast<cudaStream_t>(stream_ptr);
  const bool f16 = c.dtype == PCTREE_F16, tokens = takes_tokens(c);
  if (tokens) a.units.block_keys = kTokenBlock;
  if (c.D == 64)
    return f16 ? attn8_launch<64, true>(a, tokens, num_sms, stream)
               : attn8_launch<64, false>(a, tokens, num_sms, stream);
  return f16 ? attn8_launch<128, true>(a, tokens, num_sms, stream)
             : attn8_launch<128, false>(a, tokens, num_sms, stream);
}

}  // extern "C"
