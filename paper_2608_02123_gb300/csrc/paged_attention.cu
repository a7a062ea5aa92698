// pctree_paged_attention: causal grouped-query attention of new rows of several
// requests over a paged or contiguous cache.
//
// Work: a unit is a request, a KV head and a tile of its rows; a tile's rows
// are (row, query head of the group) pairs, row-major: R = G * rows_per_tile
// <= 128, so the G query heads sharing a KV head read each K/V block once.  A
// unit's keys are cut into blocks of at most 128 (whole pages, or parts of
// one).  All units' blocks, plus a fixed charge per unit, are one line of
// work, and CTA c takes the c-th of gridDim.x equal stretches of it: every SM
// gets the same number of blocks whatever the requests' lengths, known only on
// the device.  A stretch may begin and end inside a unit; such a piece writes
// (max, sum, unnormalised O) of its rows, and a second kernel joins the pieces
// in order.
//
//   warp 0      TMA producer, all lanes: the tile's Q (two buffers), then K and
//               V blocks (128-byte swizzle, 64 dims a half) into a ring; a lane
//               issues the copies of one page
//   warp 1      S issuer: S_b = Q K_b^T (tcgen05.mma, M = N = 128) into one of
//               two TMEM buffers
//   warp 2      PV issuer: O_h += P_b V_b over each half h of the block's keys
//               (P read from TMEM)
//   warp 3      planner: the CTA's pieces, in order, up to kItemRing ahead
//   warps 4..7  output: the two O of a finished piece, combined, to rows of out
//               or the piece's partial, while the softmax goes on
//   warps 8..15 softmax, two threads per tile row, 64 keys of a block each with
//               its own running maximum, sum and O: S is read from TMEM once,
//               masked and scaled, P = 2^(s - m_used) written back over it
// All waits are bounded (1 s; those for a whole piece 1 s without a block) and end
// in PCTREE_ERR_TIMEOUT.
//
// What bounds it (one GB300, us; 40 query and 8 KV heads of 128 dims, bf16):
//   tokens of 32 requests over up to 8192 slots: HBM, 854 MB in 141, 0.89 of
//   the measured copy rate;
//   four prompts of up to 4096 rows: K and V into the SMs, 64 KB a block for
//   every tile, 458 in pages of 64 (0.93 PFLOP/s), 485 of 32, 591 of 16, whose
//   24 TMA boxes a block cost ~30 ns each, 668 of 8;
//   a token of one request: two launches and one block's chain, 14.4.
// K and V in turn (K a block ahead: 450 -> 471 in pages of 64, 588 -> 603 of 16), one box for
// both halves of the dims in small pages (pages of 8: 253 -> 183 for tokens),
// pieces of equal length (a unit a CTA leaves SMs idle at the end).  Every CTA
// loads for itself: copies that multicast a block to the tiles of a cluster
// would halve those bytes, but the library is also that of runs on several GPUs.
#include "kv_rows.cuh"
#include "sm103_ptx.cuh"

namespace pct {
namespace {

constexpr int kBK = 128;                     // keys per block
constexpr int kHalfBytes = 128 * 128;        // 128 rows x 64 elements
constexpr uint64_t kLimitNs = 1000000000ull;
constexpr int kThreads = 512;
constexpr int kSlots = 4;                    // K or V blocks in the ring
constexpr int kItemRing = 4;
constexpr int kMaxBad = 64;                  // 16-byte places of V told apart (clean_v)
constexpr int kMaxCtas = 152;                // SMs of a GB300: partials the workspace holds
constexpr uint32_t kTmemCols = 512;
constexpr uint32_t kOCol = 2 * kBK;
constexpr int kUnitCharge = 1;               // blocks' worth of a unit's fixed cost
constexpr int kMinStretch = 2;               // of work per CTA

// A piece of a unit: blocks b0 .. b1-1 of the nblk of a tile whose keys end at
// key_end.  nblk = 0: no more pieces.
struct Item {
  int r, kvh, row0, n_rows, j0, prefix, key_end, b0, b1, nblk;
};

// How the pieces of a unit are joined: written by the CTA whose stretch ends
// inside the unit and holds its first block.
struct Join {
  int pieces;                                // 0: nothing to join at this CTA
  int kvh, row0, n_rows;
};

struct PagedArgs {
  KvRows rows;
  uint16_t* out;
  float* part_o;          // [CTA][2][D / 4][128 rows][4]
  float2* part_ml;        // [CTA][2][128]  (max in log2 units, sum)
  Join* join;             // [CTA]
  int32_t* status;
  int Hq, Hkv, G, npt;
  int packed;             // pages per block (page_size 8 .. 64), 0: parts of pages
  int page_blocks;        // blocks per page if not packed
  int box_rows;           // rows of a K/V box: a page, or part of one
  // Rows of the groups in which K and V lie in a ring slot, [group][64-dim half]
  // [row]: 128 (each half in one piece), or box_rows where one box brings both
  // halves of the dims.  A group of V is at least 8 keys, of K 8 or all (the
  // 8-key steps of an MMA operand are equally far apart).
  int k_group, v_group;
  float scale_log2;
};

// Bytes from the start of a slot to key r of its V (first half of the dims).
__device__ __forceinline__ int v_place_of(int r, int group, int halves) {
  return ((r & -group) * halves + (r & (group - 1))) * 128;
}

// Eight values (16 bytes of V) with a NaN or infinity among them: key (counted
// from the first that not every row of the tile sees), place of the eight in
// the row, and for each value 0 (finite), 1 (+inf), 2 (-inf) or 3 (NaN).  The
// non-finite ones are replaced by 0.  Returns 0 if all are finite.
template <bool F16>
__device__ __forceinline__ uint32_t bad_entry(uint4& v, int key, int place) {
  constexpr uint32_t top = F16 ? 0x7c00u : 0x7f80u;
  uint32_t w[4] = {v.x, v.y, v.z, v.w};
  uint32_t kinds = 0;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const uint32_t x = (w[e >> 1] >> (16 * (e & 1))) & 0xffffu;
    if ((x & top) == top) {
      kinds |= ((x & (0x7fffu ^ top)) != 0 ? 3u : (x & 0x8000u) != 0 ? 2u : 1u) << (2 * e);
      w[e >> 1] &= ~(0xffffu << (16 * (e & 1)));
    }
  }
  v = make_uint4(w[0], w[1], w[2], w[3]);
  return kinds == 0 ? 0u
                    : kinds | static_cast<uint32_t>(place) << 16 | static_cast<uint32_t>(key) << 20;
}

// Places of the g-th block's K and V in the ring's sequence.
__device__ __forceinline__ int k_place(int g) { return 2 * g; }
__device__ __forceinline__ int v_place(int g) { return 2 * g + 1; }

struct Tail {
  uint64_t q_full[2], q_empty[2];
  uint64_t kv_full[kSlots], kv_empty[kSlots];
  uint64_t s_full[2], p_full[2], p_empty[2];
  uint64_t o_full, o_empty;
  uint64_t item_full[kItemRing], item_empty[kItemRing];
  uint64_t done;
  uint32_t tmem_base;
  int abort;
  int blocks;                                // multiplied so far (see wwait_long)
  Item item[kItemRing];
  float row_l[2][128], row_m[2][128];
  // Non-finite values at keys that only some rows of the piece's tile see, by
  // piece parity and output warp (each resets its own copy): entries of
  // bad_entry, their number and the first such key.
  int bad_n[2][4], bad_first[2][4];
  uint32_t bad[2][4][kMaxBad];
  alignas(16) uint8_t stage[4][32 * 64];
  unsigned upto[PCTREE_KV_MAX_BATCH];        // work of requests 0 .. r (the host checks the sum)
  int start[PCTREE_KV_MAX_BATCH], n[PCTREE_KV_MAX_BATCH], prefix[PCTREE_KV_MAX_BATCH];
};

// Blocks that hold the keys 0 .. end-1, the first key of block b, and the keys
// it may hold.
__device__ __forceinline__ int blocks_of(const PagedArgs& a, int end) {
  if (a.packed) return (end + kBK - 1) / kBK;
  const int pages = end / a.rows.page_size;
  return pages * a.page_blocks + (end - pages * a.rows.page_size + kBK - 1) / kBK;
}
__device__ __forceinline__ int block_key(const PagedArgs& a, int b, int& cap) {
  cap = kBK;
  if (a.packed) return b * kBK;
  const int page = b / a.page_blocks, off = (b - page * a.page_blocks) * kBK;
  cap = min(kBK, a.rows.page_size - off);
  return page * a.rows.page_size + off;
}

__device__ __forceinline__ void report(int32_t* status, int code) {
  if (status != nullptr) atomicCAS(status, 0, code);
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

// Instruction descriptors: the operand types are bits 7 and 10 (0: f16).
template <bool F16>
__host__ __device__ constexpr uint32_t idesc(int M, int N) {
  return idesc_bf16_f32(M, N) & (F16 ? ~((1u << 7) | (1u << 10)) : ~0u);
}

// Readies a V block whose keys `valid` .. 127 no row of the tile sees and whose
// keys by_some .. valid - 1 only some rows do (see its call; not inline: its
// registers would be the loop's).  rel0: key 0 counted from the first key that
// not every row sees.
template <int HALVES, bool F16>
__device__ __noinline__ void clean_v(uint8_t* v, Tail* T, int parity, int thread, int valid,
                                     int by_some, int rel0, int group) {
  const int n16 = (kBK - valid) * 8;
  for (int i = thread; i < HALVES * n16; i += 256) {
    const int vh = i >= n16 ? 1 : 0, rem = i - vh * n16;
    *reinterpret_cast<uint4*>(v + v_place_of(valid + rem / 8, group, HALVES) + vh * group * 128 +
                              (rem % 8) * 16) = make_uint4(0, 0, 0, 0);
  }
  for (int i = thread; i < (valid - by_some) * 8 * HALVES; i += 256) {
    const int key = by_some + i / (8 * HALVES), place = i % (8 * HALVES);
    // (the 128-byte rows are swizzled: 16-byte place p of row r at p ^ (r & 7))
    const int at = v_place_of(key, group, HALVES) + (place >> 3) * group * 128;
    uint4* p = reinterpret_cast<uint4*>(v + at + (((place & 7) ^ ((at >> 7) & 7)) * 16));
    uint4 x = *p;
    const uint32_t entry = bad_entry<F16>(x, rel0 + key, place);
    if (entry != 0) {
      *p = x;
      for (int q = 0; q < 4; ++q) {
        atomicMin(&T->bad_first[parity][q], rel0 + key);
        const int n = atomicAdd(&T->bad_n[parity][q], 1);
        if (n < kMaxBad) T->bad[parity][q][n] = entry;
      }
    }
  }
}

// Scores (in log2 units) whose floats are half an octave apart: from here on the
// softmax's fused product would differ from its reference, a rounded product, by
// powers of two that P's type does not hold.
constexpr float kWideScore = 4194304.0f;

// The 64 scores of a block half at TMEM columns s_col .. (those from `seen` on are
// -inf) become what, times sc, is the rounded score less the reference.  (Not
// inline: in the loop it cost prompts 6 %.)
__device__ __noinline__ void wide_scores(uint32_t s_col, float sc, float mref, int seen) {
  const float inv = 1.0f / sc;
#pragma unroll 1
  for (int c = 0; c < 64; c += 8) {
    uint32_t y[8];
    tmem_ld_32x32b_x8(s_col + c, y);
    tmem_ld_wait();
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const float x = c + k < seen ? __uint_as_float(y[k]) : -INFINITY;
      y[k] = __float_as_uint((__fmul_rn(x, sc) - mref) * inv);
    }
    tmem_st_x8(s_col + c, y);
  }
  tmem_st_wait();
}

template <int D, bool F16>
__global__ void __maxnreg__(112)
paged_attn_kernel(const __grid_constant__ CUtensorMap tm_q,
                  const __grid_constant__ CUtensorMap tm_k,
                  const __grid_constant__ CUtensorMap tm_v, PagedArgs a) {
  constexpr int kHalves = D / 64;
  constexpr int kTileBytes = kHalves * kHalfBytes;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* sm = reinterpret_cast<uint8_t*>(
      (reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~static_cast<uintptr_t>(1023));
  uint8_t* sq = sm;                                // Q buffer of the k-th piece: k & 1
  uint8_t* skv = sm + 2 * kTileBytes;              // ring
  Tail* T = reinterpret_cast<Tail*>(skv + kSlots * kTileBytes);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int R = a.G * a.npt;                       // rows of a tile
  volatile int* abort_v = &T->abort;

  // ---------------- set-up ----------------
  if (threadIdx.x == 0) {
    for (int s = 0; s < kSlots; ++s) {
      mbar_init(&T->kv_full[s], 1);
      mbar_init(&T->kv_empty[s], 1);
    }
    for (int s = 0; s < 2; ++s) {
      mbar_init(&T->q_full[s], 1);
      mbar_init(&T->q_empty[s], 1);
      mbar_init(&T->s_full[s], 1);
      mbar_init(&T->p_full[s], 8);
      mbar_init(&T->p_empty[s], 1);
    }
    for (int s = 0; s < kItemRing; ++s) {
      mbar_init(&T->item_full[s], 1);
      mbar_init(&T->item_empty[s], 3 + 4 + 8);
    }
    mbar_init(&T->o_full, 1 + 8);
    mbar_init(&T->o_empty, 4);
    mbar_init(&T->done, 2);
    T->abort = 0;
    T->blocks = 0;
    for (int i = 0; i < 8; ++i) {
      T->bad_n[i >> 2][i & 3] = 0;
      T->bad_first[i >> 2][i & 3] = kBK;
    }
    fence_barrier_init();
    tma_prefetch_desc(&tm_q);
    tma_prefetch_desc(&tm_k);
    tma_prefetch_desc(&tm_v);
  }
  // rows R..127 of the Q buffers are never loaded: zero them once
  const int zq = (128 - R) * 8;
  for (int i = threadIdx.x; i < 2 * kHalves * zq; i += kThreads) {
    const int h = i / zq, rem = i - h * zq;
    *reinterpret_cast<uint4*>(sq + h * kHalfBytes + (R + rem / 8) * 128 + (rem % 8) * 16) =
        make_uint4(0, 0, 0, 0);
  }
  fence_proxy_async_smem();
  if (warp == 1) tmem_alloc(&T->tmem_base, kTmemCols);
  pdl_launch_dependents();
  pdl_wait();
  // the requests and the work of each: a thread each, but a warp where there are
  // several tiles
  for (int r = threadIdx.x; r < a.rows.batch; r += kThreads) {
    const int start = a.rows.row_start[r], prefix = a.rows.prefix_len[r];
    int n = a.rows.n_rows[r];
    if (!kv_request_ok(a.rows, start, n, prefix)) {
      if (blockIdx.x == 0) report(a.status, PCTREE_ERR_INVALID_ARG);
      n = 0;
    }
    T->start[r] = start;
    T->n[r] = n;
    T->prefix[r] = prefix;
    if (n <= a.npt) T->upto[r] = n > 0 ? (blocks_of(a, prefix + n) + kUnitCharge) * a.Hkv : 0;
  }
  __syncthreads();
  constexpr int kWarps = kThreads / 32;
  for (int r0 = warp; r0 < a.rows.batch; r0 += kThreads) {   // every kWarps-th is this warp's
    const int mine = r0 + lane * kWarps;
    unsigned several =
        __ballot_sync(kFull, mine < a.rows.batch && T->n[min(mine, a.rows.batch - 1)] > a.npt);
    for (; several != 0; several &= several - 1) {
      const int r = r0 + (__ffs(several) - 1) * kWarps;
      const int n = T->n[r], prefix = T->prefix[r];
      unsigned w = 0;
      for (int j = lane * a.npt; j < n; j += 32 * a.npt)
        w += blocks_of(a, prefix + min(n, j + a.npt)) + kUnitCharge;
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) w += __shfl_xor_sync(kFull, w, o);
      if (lane == 0) T->upto[r] = w * a.Hkv;
    }
  }
  __syncthreads();
  if (warp == 0) {
    unsigned base = 0;
    long long n_all = 0;
    for (int r0 = 0; r0 < a.rows.batch; r0 += 32) {
      const int r = r0 + lane;
      unsigned w = r < a.rows.batch ? T->upto[r] : 0;
      n_all += r < a.rows.batch ? T->n[r] : 0;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const unsigned p = __shfl_up_sync(kFull, w, o);
        if (lane >= o) w += p;
      }
      if (r < a.rows.batch) T->upto[r] = base + w;
      base += __shfl_sync(kFull, w, 31);
    }
    // More rows than there are: requests overlap, and their work may be more than
    // the host has checked.  Nothing is done.
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) n_all += __shfl_xor_sync(kFull, n_all, o);
    if (n_all > a.rows.total_rows) {
      for (int r = lane; r < a.rows.batch; r += 32) T->upto[r] = 0;
      if (blockIdx.x == 0 && lane == 0) report(a.status, PCTREE_ERR_INVALID_ARG);
    }
  }
  tc_fence_before_sync();
  __syncthreads();
  tc_fence_after_sync();
  const uint32_t tmem = T->tmem_base;

  auto wwait = [&](uint64_t* bar, uint32_t parity) -> bool {
    return __all_sync(kFull, mbar_wait_bounded(bar, parity, abort_v, kLimitNs));
  };
  // a wait that lasts as long as pieces do: over once no block has been multiplied
  // for the limit
  auto wwait_long = [&](uint64_t* bar, uint32_t parity) -> bool {
    volatile int* blocks = &T->blocks;
    for (;;) {
      const int before = *blocks;
      if (wwait(bar, parity)) return true;
      if (__any_sync(kFull, *abort_v != 0) || __all_sync(kFull, *blocks == before)) return false;
    }
  };
  auto give_up = [&]() {
    *abort_v = 1;
    report(a.status, PCTREE_ERR_TIMEOUT);
  };
  auto fetch_one = [&](int k, Item& it) -> bool {
    const int s = k % kItemRing;
    if (!mbar_wait_bounded(&T->item_full[s], (k / kItemRing) & 1, abort_v, kLimitNs)) return false;
    it = T->item[s];
    mbar_arrive(&T->item_empty[s]);
    return true;
  };
  auto fetch_warp = [&](int k, Item& it) -> bool {
    const int s = k % kItemRing;
    if (!wwait(&T->item_full[s], (k / kItemRing) & 1)) return false;
    it = T->item[s];
    __syncwarp();
    if (lane == 0) mbar_arrive(&T->item_empty[s]);
    return true;
  };

  if (warp == 0) {
    // ---------------- TMA producer ----------------
    // K_0 V_0 K_1 V_1 ..., place k_place(g) and v_place(g) of the ring's sequence
    struct Box {
      int page, off, boxes, kvh;                   // this lane's box of a block
    };
    int g = 0, q = 0, k = 0, b = 0;                // blocks, Q tiles, items fetched, block
    bool ok = true;
    Item it;
    it.b1 = 0;
    auto next_block = [&](Box& x) {                // false: no more, or not ok
      if (b >= it.b1) {
        if (!(ok = fetch_warp(k++, it)) || it.nblk == 0) return false;
        b = it.b0;
        const int qb = q & 1;
        if (!(ok = wwait(&T->q_empty[qb], ((q >> 1) & 1) ^ 1))) return false;
        if (lane == 0) {
          mbar_arrive_expect_tx(&T->q_full[qb], static_cast<uint32_t>(kHalves * R) * 128u);
          for (int h = 0; h < kHalves; ++h)
            tma_load_3d(sq + qb * kTileBytes + h * kHalfBytes, &tm_q, &T->q_full[qb], 64 * h,
                        it.kvh * a.G, it.row0);
        }
        ++q;
      }
      x.page = -1;
      x.off = 0;
      x.kvh = it.kvh;
      const int rows = a.box_rows;
      if (a.packed) {
        x.boxes = (min(kBK, it.key_end - b * kBK) + rows - 1) / rows;
        if (lane < x.boxes) x.page = kv_page(a.rows, it.r, b * a.packed + lane);
      } else {
        const int entry = b / a.page_blocks;
        x.off = (b - entry * a.page_blocks) * kBK;
        x.boxes = (min(kBK, a.rows.page_size - x.off) + rows - 1) / rows;
        x.off += lane * rows;
        if (lane < x.boxes) x.page = kv_page(a.rows, it.r, entry);
      }
      if (lane < x.boxes && x.page < 0) {
        report(a.status, PCTREE_ERR_INVALID_ARG);
        x.page = a.rows.n_pages;                   // past the tensor: zeros
      }
      ++b;
      return true;
    };
    auto load = [&](const CUtensorMap* map, const Box& x, int place) {
      const int slot = place % kSlots;
      if (!(ok = wwait(&T->kv_empty[slot], ((place / kSlots) & 1) ^ 1))) return;
      const bool both = kHalves == 2 && (map == &tm_k ? a.k_group : a.v_group) != kBK;
      uint8_t* dst = skv + slot * kTileBytes + lane * a.box_rows * (both ? 256 : 128);
      if (lane == 0)
        mbar_arrive_expect_tx(&T->kv_full[slot],
                              static_cast<uint32_t>(kHalves * x.boxes * a.box_rows) * 128u);
      __syncwarp();
      if (lane < x.boxes) {
        if (both) {
          tma_load_5d(dst, map, &T->kv_full[slot], 0, x.off, 0, x.kvh, x.page);
        } else {
#pragma unroll
          for (int h = 0; h < kHalves; ++h)
            tma_load_5d(dst + h * kHalfBytes, map, &T->kv_full[slot], 0, x.off, h, x.kvh, x.page);
        }
      }
    };
    Box cur;
    int k_issued = 0, v_issued = 0;
    for (; ok && next_block(cur); ++g) {
      load(&tm_k, cur, k_place(g));
      if (!ok) break;
      ++k_issued;
      load(&tm_v, cur, v_place(g));
      if (!ok) break;
      ++v_issued;
    }
    __syncwarp();
    if (lane == 0) {
      if (!ok) give_up();
      // copies still in flight land before the CTA may exit
      volatile int never = 0;
      for (int slot = 0; slot < kSlots; ++slot) {  // each slot's last place
        int last = -1;
        for (int x = max(0, k_issued - kSlots); x < k_issued; ++x)
          if (k_place(x) % kSlots == slot) last = max(last, k_place(x));
        for (int x = max(0, v_issued - kSlots); x < v_issued; ++x)
          if (v_place(x) % kSlots == slot) last = max(last, v_place(x));
        if (last >= 0)
          (void)mbar_wait_bounded(&T->kv_full[slot], (last / kSlots) & 1, &never, kLimitNs);
      }
      for (int x = q > 2 ? q - 2 : 0; x < q; ++x)
        (void)mbar_wait_bounded(&T->q_full[x & 1], (x >> 1) & 1, &never, kLimitNs);
    }
  } else if (warp == 1 && lane == 0) {
    // ---------------- S issuer ----------------
    constexpr uint32_t idS = idesc<F16>(128, kBK);
    int q = 0, g = 0;
    const uint64_t q_desc = desc_kmajor_sw128(smem_u32(sq));
    // 8 keys are a row group; groups of 8 with both halves are twice as far apart
    const bool k_both = kHalves == 2 && a.k_group == 8;
    const uint64_t k_desc = desc_kmajor_sw128(smem_u32(skv)) +
                            (k_both ? static_cast<uint64_t>(1024 >> 4) << 32 : 0ull);
    const int k_half = (k_both ? 1024 : kHalfBytes) >> 4;
    bool ok = true;
    Item it;
    for (int k = 0; ok; ++k) {
      if (!(ok = fetch_one(k, it)) || it.nblk == 0) break;
      const int qb = q & 1;
      if (!(ok = mbar_wait_bounded(&T->q_full[qb], (q >> 1) & 1, abort_v, kLimitNs))) break;
      ++q;
      const uint64_t qd = q_desc + qb * (kTileBytes >> 4);
      for (int b = it.b0; b < it.b1; ++b, ++g) {
        const int sb = g & 1, slot = k_place(g) % kSlots;
        ok = mbar_wait_bounded(&T->kv_full[slot], (k_place(g) / kSlots) & 1, abort_v, kLimitNs) &&
             mbar_wait_bounded(&T->p_empty[sb], ((g >> 1) & 1) ^ 1, abort_v, kLimitNs);
        if (!ok) break;
        const uint64_t kd = k_desc + slot * (kTileBytes >> 4);
        tc_fence_after_sync();
#pragma unroll
        for (int kk = 0; kk < D / 16; ++kk) {
          const int q_off = ((kk >> 2) * kHalfBytes + (kk & 3) * 32) >> 4;
          const int k_off = (kk >> 2) * k_half + (kk & 3) * 2;
          tc_mma_bf16(tmem + sb * kBK, qd + q_off, kd + k_off, idS, kk > 0 ? 1u : 0u);
        }
        tc_commit(&T->s_full[sb]);
        tc_commit(&T->kv_empty[slot]);
      }
      tc_commit(&T->q_empty[qb]);
    }
    if (!ok) give_up();
    tc_commit(&T->done);
    volatile int never = 0;
    (void)mbar_wait_bounded(&T->done, 0, &never, kLimitNs);
  } else if (warp == 2 && lane == 0) {
    // ---------------- PV issuer ----------------
    constexpr uint32_t idO = idesc<F16>(128, D) | (1u << 16);   // B MN-major
    int g = 0;
    // (with groups of 8 keys the next 8 are in the next group)
    const uint64_t v_desc = desc_mnmajor_sw128(smem_u32(skv), a.v_group * 128,
                                               kHalves == 2 && a.v_group == 8 ? 2048 : 1024);
    int v_off[kBK / 16];                           // of every 16 keys in a slot
#pragma unroll
    for (int kk = 0; kk < kBK / 16; ++kk) v_off[kk] = v_place_of(16 * kk, a.v_group, kHalves) >> 4;
    bool ok = true;
    volatile int* blocks = &T->blocks;
    Item it;
    for (int k = 0; ok; ++k) {
      if (!(ok = fetch_one(k, it)) || it.nblk == 0) break;
      for (int b = it.b0; b < it.b1; ++b, ++g) {
        const int sb = g & 1, slot = v_place(g) % kSlots;
        ok = mbar_wait_bounded(&T->kv_full[slot], (v_place(g) / kSlots) & 1, abort_v, kLimitNs) &&
             mbar_wait_bounded(&T->p_full[sb], (g >> 1) & 1, abort_v, kLimitNs) &&
             (b > it.b0 ||                         // the last piece's O has been read
              mbar_wait_bounded(&T->o_empty, (k & 1) ^ 1, abort_v, kLimitNs));
        if (!ok) break;
        const uint64_t vd = v_desc + slot * (kTileBytes >> 4);
        tc_fence_after_sync();
#pragma unroll
        for (int kk = 0; kk < kBK / 16; ++kk) {
          const int h = kk >> 2;
          tc_mma_tmem_a(tmem + kOCol + h * D, tmem + sb * kBK + h * 64 + (kk & 3) * 8,
                        vd + v_off[kk], idO,
                        (b > it.b0 || (kk & 3) > 0) ? 1u : 0u);
        }
        tc_commit(&T->p_empty[sb]);
        if (b + 1 == it.b1) tc_commit(&T->o_full);
        *blocks = g + 1;
        tc_commit(&T->kv_empty[slot]);
      }
    }
    if (!ok) give_up();
    tc_commit(&T->done);
    volatile int never = 0;
    (void)mbar_wait_bounded(&T->done, 0, &never, kLimitNs);
  } else if (warp == 3) {
    // ---------------- planner ----------------
    const unsigned total = T->upto[a.rows.batch - 1];
    const unsigned places = gridDim.x, place = blockIdx.x;
    const unsigned stretch = max((total + places - 1) / places, static_cast<unsigned>(kMinStretch));
    // (place * stretch is at most total + places * kMinStretch)
    unsigned x = place * stretch;
    const unsigned x_end = min(total, x + stretch);
    Join join = {0, 0, 0, 0};
    int k = 0;
    bool ok = true;
    auto post = [&](const Item& it) {              // lane 0 writes the k-th piece
      const int s = k % kItemRing;
      if (!(ok = wwait_long(&T->item_empty[s], ((k / kItemRing) & 1) ^ 1))) return;
      if (lane == 0) {
        T->item[s] = it;
        mbar_arrive(&T->item_full[s]);
      }
      __syncwarp();
      ++k;
    };
    if (x < x_end) {
      // the request, KV head and tile that hold place x of the line
      int lo = 0, hi = a.rows.batch - 1;
      while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (T->upto[mid] <= x) lo = mid + 1; else hi = mid;
      }
      int r = lo, kvh = 0, tile = 0;
      int start = 0, n = 0, prefix = 0;
      auto load = [&]() {
        start = T->start[r];
        n = T->n[r];
        prefix = T->prefix[r];
      };
      load();
      const unsigned before = r > 0 ? T->upto[r - 1] : 0;
      const unsigned per_head = (T->upto[r] - before) / a.Hkv;
      unsigned in = x - before;                    // place inside the head's tiles
      kvh = static_cast<int>(in / per_head);
      in -= kvh * per_head;
      for (;;) {
        const int j = (tile + lane) * a.npt;
        const unsigned cost = j < n ? blocks_of(a, prefix + min(n, j + a.npt)) + kUnitCharge : 0;
        unsigned c = cost;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
          const unsigned p = __shfl_up_sync(kFull, c, o);
          if (lane >= o) c += p;
        }
        const unsigned past = __ballot_sync(kFull, c > in);
        if (past != 0) {
          const int l = __ffs(past) - 1;
          in -= __shfl_sync(kFull, c - cost, l);
          tile += l;
          break;
        }
        in -= __shfl_sync(kFull, c, 31);
        tile += 32;
      }
      while (ok && x < x_end) {
        const int j0 = tile * a.npt;
        Item it;
        it.r = r;
        it.kvh = kvh;
        it.row0 = start + j0;
        it.n_rows = min(n - j0, a.npt);
        it.j0 = j0;
        it.prefix = prefix;
        it.key_end = prefix + min(n, j0 + a.npt);
        it.nblk = blocks_of(a, it.key_end);
        const unsigned left = it.nblk + kUnitCharge - in;
        const unsigned take = min(left, x_end - x);
        it.b0 = max(0, static_cast<int>(in) - kUnitCharge);
        it.b1 = max(0, static_cast<int>(in + take) - kUnitCharge);
        if (it.b1 > it.b0) {
          if (it.b0 == 0 && it.b1 < it.nblk) {
            // joined from here: the unit's end lies `left` past x
            join.pieces = static_cast<int>((x + left - 1) / stretch - place) + 1;
            join.kvh = kvh;
            join.row0 = it.row0;
            join.n_rows = it.n_rows;
          }
          post(it);
        }
        x += take;
        in = 0;
        ++tile;
        if (x < x_end && tile * a.npt >= n) {
          tile = 0;
          if (++kvh == a.Hkv) {
            kvh = 0;
            do ++r; while (T->upto[r] <= x);       // requests without work
            load();
          }
        }
      }
    }
    if (lane == 0) a.join[blockIdx.x] = join;
    if (ok) {
      Item end = {};
      post(end);
    }
    if (!ok && lane == 0) give_up();
  } else if (warp >= 4 && warp < 8) {
    // ---------------- output, one thread per tile row ----------------
    const int quad = warp & 3;
    const int t = quad * 32 + lane;
    const uint32_t lane_base = tmem + (static_cast<uint32_t>(quad * 32) << 16);
    uint8_t* stg = T->stage[quad];
    // the rows this lane stores (8 i + lane / 4 of the warp's 32, piece lane %
    // 4 of a 64-byte segment): their places in the tile
    int out_nl[4], out_off[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int ti = quad * 32 + 8 * i + (lane >> 2), ni = ti / a.G;
      out_nl[i] = ti < R ? ni : 0x7fffffff;
      out_off[i] = (ni * a.Hq + ti - ni * a.G) * D + (lane & 3) * 8;
    }
    bool ok = true;
    Item it;
    for (int k = 0;; ++k) {
      if (!(ok = fetch_warp(k, it)) || it.nblk == 0) break;
      if (!(ok = wwait_long(&T->o_full, k & 1))) break;
      tc_fence_after_sync();
      uint16_t* oitem = a.out + (static_cast<size_t>(it.row0) * a.Hq + it.kvh * a.G) * D;
      const bool whole = it.b0 == 0 && it.b1 == it.nblk;
      const int n_bad = T->bad_n[k & 1][quad];
      const size_t part = static_cast<size_t>(blockIdx.x) * 2 + (it.b0 == 0 ? 1 : 0);
      // the halves' sums and O relative to the larger of their references
      const float l0 = T->row_l[0][t], l1 = T->row_l[1][t];
      const float m0 = l0 != 0.0f ? T->row_m[0][t] : -INFINITY;
      const float m1 = l1 != 0.0f ? T->row_m[1][t] : -INFINITY;
      const float m = fmaxf(m0, m1);
      float f0 = l0 != 0.0f ? exp2f(m0 - m) : 0.0f;
      float f1 = l1 != 0.0f ? exp2f(m1 - m) : 0.0f;
      const float l = l0 * f0 + l1 * f1;
      const uint32_t o_col = lane_base + kOCol;
      if (whole) {                                 // (no finite score, l = 0: NaN)
        const float inv = 1.0f / l;
        f0 *= inv;
        f1 *= inv;
      }
      const bool in_tile = t / a.G < it.n_rows && t < R;
      if (!whole && in_tile)
        a.part_ml[part * 128 + t] = make_float2(l != 0.0f ? m : -INFINITY, l);
#pragma unroll 1
      for (int c = 0; c < D / 32; ++c) {
        float y[32];
        {
          uint32_t y0[32], y1[32];
          tmem_ld_32x32b_x32(o_col + c * 32, y0);
          tmem_ld_32x32b_x32(o_col + D + c * 32, y1);
          tmem_ld_wait();
#pragma unroll
          for (int i = 0; i < 32; i += 2) {
            const uint64_t a0 = pack2(__uint_as_float(y0[i]), __uint_as_float(y0[i + 1]));
            const uint64_t a1 = pack2(__uint_as_float(y1[i]), __uint_as_float(y1[i + 1]));
            unpack2(fma2(a0, pack2(f0, f0), mul2(a1, pack2(f1, f1))), y[i], y[i + 1]);
          }
        }
        // values taken out of V reach the rows that see their keys
        if (n_bad != 0) {
          uint32_t pos = 0, neg = 0, nan = 0;
          const int seen = t / a.G - 1;            // the last such key the row sees
          for (int i = 0; i < min(n_bad, kMaxBad); ++i) {
            const uint32_t e = T->bad[k & 1][quad][i];
            const int place = (e >> 16) & 15;
            if (static_cast<int>(e >> 20) > seen || place / 4 != c) continue;
            for (int x = 0; x < 8; ++x) {
              const uint32_t kind = (e >> (2 * x)) & 3u, bit = 1u << ((place & 3) * 8 + x);
              if (kind == 1) pos |= bit;
              if (kind == 2) neg |= bit;
              if (kind == 3) nan |= bit;
            }
          }
          if (n_bad > kMaxBad && T->bad_first[k & 1][quad] <= seen) nan = 0xffffffffu;
          // (added: y may be NaN or the opposite infinity already)
#pragma unroll
          for (int i = 0; i < 32; ++i) {
            if ((pos >> i) & 1u) y[i] += INFINITY;
            if ((neg >> i) & 1u) y[i] -= INFINITY;
            if ((nan >> i) & 1u) y[i] = __int_as_float(0x7fc00000);
          }
          __syncwarp();
          if (c == D / 32 - 1 && lane == 0) {
            T->bad_n[k & 1][quad] = 0;
            T->bad_first[k & 1][quad] = kBK;
          }
        }
        if (c == D / 32 - 1) {
          tc_fence_before_sync();
          __syncwarp();
          if (lane == 0) mbar_arrive(&T->o_empty);
        }
        if (!whole) {
          float4* po = reinterpret_cast<float4*>(a.part_o) + part * (D / 4) * 128 + c * 8 * 128 + t;
          if (in_tile) {
#pragma unroll
            for (int q = 0; q < 8; ++q)
              po[q * 128] = make_float4(y[4 * q], y[4 * q + 1], y[4 * q + 2], y[4 * q + 3]);
          }
          continue;
        }
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          uint32_t w[4];
#pragma unroll
          for (int h = 0; h < 4; ++h) w[h] = pack16<F16>(y[q * 8 + 2 * h], y[q * 8 + 2 * h + 1]);
          *reinterpret_cast<uint4*>(stg + lane * 64 + ((q ^ (lane >> 1)) & 3) * 16) =
              make_uint4(w[0], w[1], w[2], w[3]);
        }
        __syncwarp();
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int row = 8 * i + (lane >> 2);
          const uint4 v = *reinterpret_cast<const uint4*>(
              stg + row * 64 + (((lane & 3) ^ (row >> 1)) & 3) * 16);
          if (out_nl[i] < it.n_rows) *reinterpret_cast<uint4*>(oitem + out_off[i] + c * 32) = v;
        }
        __syncwarp();
      }
    }
    if (!ok && lane == 0) give_up();
  } else if (warp >= 8) {
    // ---------------- softmax, two threads per tile row ----------------
    const int half = (warp - 8) >> 2;
    const int quad = warp & 3;
    const int t = quad * 32 + lane;
    const int nl = t / a.G;
    const uint32_t lane_base = tmem + (static_cast<uint32_t>(quad * 32) << 16);
    const uint32_t o_col = lane_base + kOCol + half * D;
    const float sc = a.scale_log2;
    int g = 0;
    bool ok = true;
    Item it;
    for (int k = 0; ok; ++k) {
      if (!(ok = fetch_warp(k, it)) || it.nblk == 0) break;
      // keys this row sees: slots below `end`
      const int end = min(it.key_end, it.prefix + it.j0 + nl + 1);
      float m_used = -INFINITY, l_sum = 0.0f;
      float over = -INFINITY;                      // a maximum above it needs a look
      for (int b = it.b0; b < it.b1; ++b, ++g) {
        const int sb = g & 1;
        int cap;
        const int key0 = block_key(a, b, cap);
        if (!(ok = wwait(&T->s_full[sb], (g >> 1) & 1))) break;
        tc_fence_after_sync();
        const uint32_t s_col = lane_base + sb * kBK + half * 64;
        float x[64];
        {
          uint32_t* xu = reinterpret_cast<uint32_t*>(x);
#pragma unroll
          for (int c = 0; c < 2; ++c)
            tmem_ld_32x32b_x32(s_col + c * 32,
                               *reinterpret_cast<uint32_t(*)[32]>(xu + c * 32));
          tmem_ld_wait();
        }
        // keys the row may not see become -inf
        const int seen = min(cap, end - key0) - half * 64;
        if (__any_sync(kFull, seen < 64)) {
#pragma unroll
          for (int k2 = 0; k2 < 64; ++k2) x[k2] = k2 < seen ? x[k2] : -INFINITY;
        }
        float m8[8];
#pragma unroll
        for (int u = 0; u < 8; ++u) m8[u] = x[u];
#pragma unroll
        for (int k2 = 8; k2 < 64; ++k2) m8[k2 & 7] = fmaxf(m8[k2 & 7], x[k2]);
        const float mx = fmaxf(fmaxf(fmaxf(m8[0], m8[1]), fmaxf(m8[2], m8[3])),
                         fmaxf(fmaxf(m8[4], m8[5]), fmaxf(m8[6], m8[7]))) * sc;
        bool shifted = false;
        if (__any_sync(kFull, mx > over)) {
          const bool mine = mx > m_used + 8.0f;
          const float alpha = mine ? ex2_approx(m_used - mx) : 1.0f;
          if (b > it.b0) {
            if (!(ok = wwait(&T->p_empty[(g - 1) & 1], ((g - 1) >> 1) & 1))) break;
            tc_fence_after_sync();
#pragma unroll 2
            for (int c = 0; c < D / 8; ++c) {
              uint32_t y[8];
              tmem_ld_32x32b_x8(o_col + c * 8, y);
              tmem_ld_wait();
#pragma unroll
              for (int k2 = 0; k2 < 8; ++k2)
                y[k2] = __float_as_uint(__uint_as_float(y[k2]) * alpha);
              tmem_st_x8(o_col + c * 8, y);
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
          if (shifted) {
            wide_scores(s_col, sc, m_used == -INFINITY ? 0.0f : m_used, seen);
#pragma unroll
            for (int c = 0; c < 2; ++c)
              tmem_ld_32x32b_x32(s_col + c * 32,
                                 *reinterpret_cast<uint32_t(*)[32]>(
                                     reinterpret_cast<uint32_t*>(x) + c * 32));
            tmem_ld_wait();
          }
        }
        const float mref = shifted || m_used == -INFINITY ? 0.0f : m_used;
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
            pk[h] = pack16<F16>(p0, p1);
          }
          tmem_st_x16(s_col + c * 16, pk);
        }
        tmem_st_wait();
        {
          float s0, s1;
          unpack2(add2(add2(ls[0], ls[1]), add2(ls[2], ls[3])), s0, s1);
          l_sum += s0 + s1;
        }
        // V rows no row of the tile sees hold anything: zero them, so that
        // 0 * (non-finite) cannot reach O.  Those that only some rows see (the
        // tile's own keys) must not reach the others either: their non-finite
        // values are taken out and noted for the output warps.
        const int valid = min(cap, max(0, it.prefix + it.j0 + it.n_rows - key0));
        const int by_some = max(0, it.prefix + it.j0 + 1 - key0);
        if (min(valid, by_some) < kBK) {
          const int xv = v_place(g);
          if (!(ok = wwait(&T->kv_full[xv % kSlots], (xv / kSlots) & 1))) break;
          uint8_t* v = skv + (xv % kSlots) * kTileBytes;
          clean_v<D / 64, F16>(v, T, k & 1, half * 128 + t, valid, by_some,
                               key0 - (it.prefix + it.j0 + 1), a.v_group);
          fence_proxy_async_smem();
        }
        tc_fence_before_sync();
        __syncwarp();
        if (lane == 0) mbar_arrive(&T->p_full[sb]);
      }
      if (!ok) break;
      if (!(ok = wwait(&T->o_empty, (k & 1) ^ 1))) break;
      T->row_l[half][t] = l_sum;
      T->row_m[half][t] = m_used;
      __syncwarp();
      if (lane == 0) mbar_arrive(&T->o_full);
    }
    if (!ok && lane == 0) give_up();
  }
  // ---------------- teardown ----------------
  __syncwarp();
  tc_fence_before_sync();
  __syncthreads();
  tc_fence_after_sync();
  if (warp == 1) tmem_dealloc(tmem, kTmemCols);
}

// Joins the pieces of the units that end in another CTA than they began in: a
// thread has four dims of a row at a time.  Few CTAs, since most find nothing to
// join (152 x 32 of them took 3 us of a batch of short chains).
constexpr int kJoinThreads = 256;
constexpr int kJoinCtas = 4;                 // per CTA of the attention

template <int D, bool F16>
__global__ void __launch_bounds__(kJoinThreads, 4) paged_join_kernel(PagedArgs a) {
  pdl_launch_dependents();
  pdl_wait();
  const int c0 = blockIdx.x;
  const Join j = a.join[c0];
  if (j.pieces == 0) return;
  constexpr int kQuads = D / 4;
  const float4* po = reinterpret_cast<const float4*>(a.part_o);
  const int n = j.n_rows * a.G * kQuads;
  for (int i = blockIdx.y * kJoinThreads + threadIdx.x; i < n; i += kJoinCtas * kJoinThreads) {
    // neighbouring threads have neighbouring dims (their stores) of a row
    const int row = i / kQuads, quad = i - row * kQuads;
    const int nl = row / a.G, g = row - nl * a.G;
    float m = -INFINITY, lsum = 0.0f;
    float4 acc = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    for (int s0 = 0; s0 < j.pieces; s0 += 4) {
      float2 w[4];
      float4 v[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const bool in = s0 + u < j.pieces;
        // the first piece is its CTA's last, every other one its CTA's first
        const size_t part =
            static_cast<size_t>(c0 + s0 + u) * 2 + (s0 + u == 0 ? 1 : 0);
        w[u] = in ? a.part_ml[part * 128 + row] : make_float2(-INFINITY, 0.0f);
        v[u] = in ? po[(part * kQuads + quad) * 128 + row] : acc;
      }
      float mn = m;
#pragma unroll
      for (int u = 0; u < 4; ++u)
        if (w[u].y != 0.0f) mn = fmaxf(mn, w[u].x);
      const float f0 = mn > m && m > -INFINITY ? exp2f(m - mn) : 1.0f;
      lsum *= f0;
      acc.x *= f0;
      acc.y *= f0;
      acc.z *= f0;
      acc.w *= f0;
      m = mn;
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        if (w[u].y != 0.0f) {
          const float f = exp2f(w[u].x - m);
          lsum = fmaf(w[u].y, f, lsum);
          acc.x = fmaf(v[u].x, f, acc.x);
          acc.y = fmaf(v[u].y, f, acc.y);
          acc.z = fmaf(v[u].z, f, acc.z);
          acc.w = fmaf(v[u].w, f, acc.w);
        }
      }
    }
    const float inv = 1.0f / lsum;               // (no finite score, lsum = 0: NaN)
    uint16_t* orow =
        a.out + ((static_cast<size_t>(j.row0) + nl) * a.Hq + j.kvh * a.G + g) * D + quad * 4;
    *reinterpret_cast<uint2*>(orow) = make_uint2(pack16<F16>(acc.x * inv, acc.y * inv),
                                                 pack16<F16>(acc.z * inv, acc.w * inv));
  }
}

// Rows per tile: one where requests have one row each, on average (a tile's
// rows are loaded whether or not they are the request's), else as many as fit.
int rows_per_tile(const pctree_paged_attn_config& c) {
  const int fit = 128 / (c.Hq / c.Hkv);
  return c.total_rows <= c.batch ? 1 : fit < c.total_rows ? fit : c.total_rows;
}

// Pages per block of keys where several fill one, else 0.
int packed_pages(int page_size) {
  return page_size == 8 || page_size == 16 || page_size == 32 || page_size == 64 ? kBK / page_size
                                                                                 : 0;
}

// Whether the planner can count the most work a configuration can have in 32
// bits.
bool paged_work_ok(const pctree_paged_attn_config& c) {
  const long long units = c.total_rows / rows_per_tile(c) + 1ll + c.batch;
  const long long blocks =
      (packed_pages(c.page_size) != 0
           ? (static_cast<long long>(c.max_pages) * c.page_size + kBK - 1) / kBK
           : static_cast<long long>(c.max_pages) * ((c.page_size + kBK - 1) / kBK)) + kUnitCharge;
  return units * blocks < (1ll << 32) / c.Hkv - 1024;
}

pctree_status paged_check(const pctree_paged_attn_config* c) {
  if (c == nullptr) return PCTREE_ERR_INVALID_ARG;
  if (c->Hq < 1 || c->D < 1 || !(c->scale > 0.0f) || !(c->scale < 1e30f))
    return PCTREE_ERR_INVALID_ARG;
  const pctree_status st = kv_check(c->batch, c->total_rows, c->Hkv, c->page_size, c->n_pages,
                                    c->max_pages, c->dtype);
  if (st != PCTREE_OK) return st;
  if (c->Hq % c->Hkv != 0 || c->q_stride % 8 != 0 ||
      c->q_stride < static_cast<int64_t>(c->Hq) * c->D)
    return PCTREE_ERR_INVALID_ARG;
  if ((c->D != 64 && c->D != 128) || c->Hq / c->Hkv > 128 || c->q_stride > (1ll << 38) ||
      !paged_work_ok(*c))
    return PCTREE_ERR_UNSUPPORTED;
  return PCTREE_OK;
}

struct PagedWs {
  size_t part_o, part_ml, join, total;
};
PagedWs paged_ws(const pctree_paged_attn_config& c) {
  PagedWs w{};
  const size_t slots = static_cast<size_t>(kMaxCtas) * 2 * 128;
  w.part_o = 0;
  w.part_ml = w.part_o + slots * c.D * sizeof(float);
  w.join = w.part_ml + slots * sizeof(float2);
  w.total = (w.join + kMaxCtas * sizeof(Join) + 255) & ~static_cast<size_t>(255);
  return w;
}

template <int D, bool F16>
pctree_status paged_launch(const CUtensorMap& tm_q, const CUtensorMap& tm_k,
                           const CUtensorMap& tm_v, const PagedArgs& a, int num_sms,
                           cudaStream_t stream) {
  constexpr size_t smem =
      (2 + kSlots) * (D / 64) * static_cast<size_t>(kHalfBytes) + sizeof(Tail) + 1024;
  static_assert(smem <= 227 * 1024, "shared memory per CTA");
  static SmemLimit limit;
  const void* fn = reinterpret_cast<const void*>(paged_attn_kernel<D, F16>);
  if (limit.ensure(fn, smem) != cudaSuccess) return PCTREE_ERR_CUDA;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cudaLaunchConfig_t lc = {};
  const unsigned ctas = static_cast<unsigned>(num_sms < kMaxCtas ? num_sms : kMaxCtas);
  lc.gridDim = dim3(ctas);
  lc.blockDim = dim3(kThreads);
  lc.dynamicSmemBytes = smem;
  lc.stream = stream;
  lc.attrs = attr;
  lc.numAttrs = 1;
  if (cudaLaunchKernelEx(&lc, paged_attn_kernel<D, F16>, tm_q, tm_k, tm_v, a) != cudaSuccess)
    return PCTREE_ERR_CUDA;
  lc.gridDim = dim3(ctas, kJoinCtas);
  lc.blockDim = dim3(kJoinThreads);
  lc.dynamicSmemBytes = 0;
  return cudaLaunchKernelEx(&lc, paged_join_kernel<D, F16>, a) == cudaSuccess ? PCTREE_OK
                                                                             : PCTREE_ERR_CUDA;
}

}  // namespace
}  // namespace pct

extern "C" {

size_t pctree_paged_attention_workspace_bytes(const pctree_paged_attn_config* cfg) {
  if (pct::paged_check(cfg) != PCTREE_OK) return 0;
  return pct::paged_ws(*cfg).total;
}

pctree_status pctree_paged_attention(const pctree_paged_attn_config* cfg, const void* q,
                                     const void* k_cache, const void* v_cache,
                                     const int32_t* row_start, const int32_t* n_rows,
                                     const int32_t* prefix_len, const int32_t* page_table,
                                     void* out, void* workspace, size_t workspace_bytes,
                                     int32_t* status, void* stream_ptr) {
  using namespace pct;
  NvtxRange range("pctree_paged_attention");
  pctree_status st = paged_check(cfg);
  if (st != PCTREE_OK) return st;
  const pctree_paged_attn_config& c = *cfg;
  if (q == nullptr || k_cache == nullptr || v_cache == nullptr || row_start == nullptr ||
      n_rows == nullptr || prefix_len == nullptr || out == nullptr || !kv_al16(q) ||
      !kv_al16(k_cache) || !kv_al16(v_cache) || !kv_al16(out) ||
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
  const PagedWs w = paged_ws(c);
  if (workspace == nullptr || workspace_bytes < w.total ||
      (reinterpret_cast<uintptr_t>(workspace) & 255u) != 0)
    return PCTREE_ERR_WORKSPACE;
  int num_sms = 0;
  st = device_facts(&num_sms);
  if (st != PCTREE_OK) return st;
  PagedArgs a{};
  a.rows = {row_start, n_rows, prefix_len, page_table, c.batch, c.total_rows,
            c.page_size, c.n_pages, c.max_pages};
  a.out = static_cast<uint16_t*>(out);
  unsigned char* ws = static_cast<unsigned char*>(workspace);
  a.part_o = reinterpret_cast<float*>(ws + w.part_o);
  a.part_ml = reinterpret_cast<float2*>(ws + w.part_ml);
  a.join = reinterpret_cast<Join*>(ws + w.join);
  a.status = status;
  a.Hq = c.Hq;
  a.Hkv = c.Hkv;
  a.G = c.Hq / c.Hkv;
  a.npt = rows_per_tile(c);
  a.packed = packed_pages(c.page_size);
  a.page_blocks = (c.page_size + kBK - 1) / kBK;
  a.box_rows = c.page_size < kBK ? c.page_size : kBK;
  a.v_group = a.packed != 0 && a.box_rows < kBK ? a.box_rows : kBK;
  a.k_group = a.v_group == 8 ? 8 : kBK;
  a.scale_log2 = static_cast<float>(static_cast<double>(c.scale) * 1.4426950408889634);
  CUtensorMap tm_q, tm_k, tm_v;
  const uint64_t D = static_cast<uint64_t>(c.D), head = D * 2;   // bytes of one head row
  {
    const uint64_t dims[3] = {D, static_cast<uint64_t>(c.Hq), static_cast<uint64_t>(c.total_rows)};
    const uint64_t str[2] = {head, static_cast<uint64_t>(c.q_stride) * 2};
    const uint32_t box[3] = {64, static_cast<uint32_t>(a.G), static_cast<uint32_t>(a.npt)};
    st = encode_bf16_map_nd(&tm_q, q, 3, dims, str, box);
    if (st != PCTREE_OK) return st;
  }
  {
    // 64 dims, slots of a page, halves of the dims, heads, pages
    const uint64_t dims[5] = {64, static_cast<uint64_t>(c.page_size), D / 64,
                              static_cast<uint64_t>(c.Hkv), static_cast<uint64_t>(c.n_pages)};
    const uint64_t str[4] = {head * c.Hkv, 128, head, head * c.Hkv * c.page_size};
    const uint32_t rows = static_cast<uint32_t>(a.box_rows);
    const uint32_t half = 1, all = static_cast<uint32_t>(c.D / 64);
    const uint32_t k_box[5] = {64, rows, a.k_group == kBK ? half : all, 1, 1};
    const uint32_t v_box[5] = {64, rows, a.v_group == kBK ? half : all, 1, 1};
    st = encode_bf16_map_nd(&tm_k, k_cache, 5, dims, str, k_box);
    if (st != PCTREE_OK) return st;
    st = encode_bf16_map_nd(&tm_v, v_cache, 5, dims, str, v_box);
    if (st != PCTREE_OK) return st;
  }
  cudaStream_t stream = static_cast<cudaStream_t>(stream_ptr);
  const bool f16 = c.dtype == PCTREE_F16;
  if (c.D == 64)
    return f16 ? paged_launch<64, true>(tm_q, tm_k, tm_v, a, num_sms, stream)
               : paged_launch<64, false>(tm_q, tm_k, tm_v, a, num_sms, stream);
  return f16 ? paged_launch<128, true>(tm_q, tm_k, tm_v, a, num_sms, stream)
             : paged_launch<128, false>(tm_q, tm_k, tm_v, a, num_sms, stream);
}

}  // extern "C"
