// How attention over the rows of several requests is divided among CTAs.
//
// A unit is a request, a KV head and a tile of `npt` of its rows; its keys are cut
// into blocks.  All units' blocks, plus a fixed charge per unit, are one line of
// work, and CTA c takes the c-th of gridDim.x equal stretches of it, so that every
// SM gets the same number of blocks whatever the requests' lengths, which are
// known only on the device.  A stretch may begin and end inside a unit: such a
// piece writes (max, sum, unnormalised O) of its rows, and join_pieces adds the
// pieces of a unit up in order.
#pragma once

#include "kv_rows.cuh"
#include "sm103_ptx.cuh"

namespace pct {

constexpr int kUnitCharge = 1;               // blocks' worth of a unit's fixed cost
constexpr int kMinStretch = 2;               // of work per CTA
constexpr int kMaxCtas = 152;                // SMs of a GB300: partials a workspace holds
constexpr int kUnitRows = 256;               // (row, query head) pairs of a unit, at most

// A piece of a unit: blocks b0 .. b1-1 of the nblk of a tile whose keys end at
// key_end.  nblk = 0: no more pieces.
struct Piece {
  int r, kvh, row0, n_rows, j0, prefix, key_end, b0, b1, nblk;
};

// How the pieces of a unit are joined: written by the CTA whose stretch ends
// inside the unit and holds its first block.
struct PieceJoin {
  int pieces;                                // 0: nothing to join at this CTA
  int kvh, row0, n_rows;
};

// Units of rows over a cache: npt rows a tile, at most max_rows rows a request,
// blocks of block_keys consecutive slots.
struct Units {
  KvRows rows;
  int Hkv, npt, max_rows, block_keys;
  __device__ __forceinline__ int blocks(int end) const {
    return (end + block_keys - 1) / block_keys;
  }
};

// The work of requests 0 .. r in upto[r] (shared memory), by all kThreads threads
// of the CTA; bad(code) is called by one thread for every request that is left
// out.  Ends with a barrier.
template <int kThreads, class Bad>
__device__ __forceinline__ void count_work(const Units& u, unsigned* upto, Bad bad) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int batch = u.rows.batch;
  constexpr int kWarps = kThreads / 32;
  constexpr unsigned kSeveral = 0xffffffffu;     // tiles, to be counted by a warp
  for (int r = threadIdx.x; r < batch; r += kThreads) {
    const int start = u.rows.row_start[r], prefix = u.rows.prefix_len[r];
    int n = u.rows.n_rows[r];
    if (!kv_request_ok(u.rows, start, n, prefix) || n > u.max_rows) {
      bad(PCTREE_ERR_INVALID_ARG);
      n = 0;
    }
    upto[r] = n <= 0       ? 0u
              : n <= u.npt ? static_cast<unsigned>((u.blocks(prefix + n) + kUnitCharge) * u.Hkv)
                           : kSeveral;
  }
  __syncthreads();
  for (int r0 = warp; r0 < batch; r0 += kThreads) {          // every kWarps-th is this warp's
    const int mine = r0 + lane * kWarps;
    unsigned several = __ballot_sync(kFull, mine < batch && upto[min(mine, batch - 1)] == kSeveral);
    for (; several != 0; several &= several - 1) {
      const int r = r0 + (__ffs(several) - 1) * kWarps;
      const int n = u.rows.n_rows[r], prefix = u.rows.prefix_len[r];
      unsigned w = 0;
      for (int j = lane * u.npt; j < n; j += 32 * u.npt)
        w += u.blocks(prefix + min(n, j + u.npt)) + kUnitCharge;
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) w += __shfl_xor_sync(kFull, w, o);
      __syncwarp();
      if (lane == 0) upto[r] = w * u.Hkv;
    }
  }
  __syncthreads();
  if (warp == 0) {
    unsigned base = 0;
    long long n_all = 0;
    for (int r0 = 0; r0 < batch; r0 += 32) {
      const int r = r0 + lane;
      unsigned w = r < batch ? upto[r] : 0;
      n_all += w != 0 ? u.rows.n_rows[r] : 0;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const unsigned p = __shfl_up_sync(kFull, w, o);
        if (lane >= o) w += p;
      }
      if (r < batch) upto[r] = base + w;
      base += __shfl_sync(kFull, w, 31);
    }
    // More rows than there are: requests overlap, and their work may be more than
    // the host has checked.  Nothing is done.
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) n_all += __shfl_xor_sync(kFull, n_all, o);
    if (n_all > u.rows.total_rows) {
      for (int r = lane; r < batch; r += 32) upto[r] = 0;
      if (lane == 0) bad(PCTREE_ERR_INVALID_ARG);
    }
  }
  __syncthreads();
}

// One warp: this CTA's pieces, in order, each given to post (false: stop).
template <class Post>
__device__ __forceinline__ bool plan_pieces(const Units& u, const unsigned* upto, PieceJoin& join,
                                            Post post) {
  const int lane = threadIdx.x & 31, npt = u.npt;
  const unsigned total = upto[u.rows.batch - 1];
  const unsigned places = gridDim.x, place = blockIdx.x;
  const unsigned stretch = max((total + places - 1) / places, static_cast<unsigned>(kMinStretch));
  // (place * stretch is at most total + places * kMinStretch)
  unsigned x = place * stretch;
  const unsigned x_end = min(total, x + stretch);
  join = {0, 0, 0, 0};
  if (x >= x_end) return true;
  // the request, KV head and tile that hold place x of the line
  int lo = 0, hi = u.rows.batch - 1;
  while (lo < hi) {
    const int mid = (lo + hi) >> 1;
    if (upto[mid] <= x) lo = mid + 1; else hi = mid;
  }
  int r = lo, tile = 0;
  int start = u.rows.row_start[r], n = u.rows.n_rows[r], prefix = u.rows.prefix_len[r];
  const unsigned before = r > 0 ? upto[r - 1] : 0;
  const unsigned per_head = (upto[r] - before) / u.Hkv;
  unsigned in = x - before;                      // place inside the head's tiles
  int kvh = static_cast<int>(in / per_head);
  in -= kvh * per_head;
  for (;;) {
    const int j = (tile + lane) * npt;
    const unsigned cost = j < n ? u.blocks(prefix + min(n, j + npt)) + kUnitCharge : 0;
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
  while (x < x_end) {
    const int j0 = tile * npt;
    Piece it;
    it.r = r;
    it.kvh = kvh;
    it.row0 = start + j0;
    it.n_rows = min(n - j0, npt);
    it.j0 = j0;
    it.prefix = prefix;
    it.key_end = prefix + min(n, j0 + npt);
    it.nblk = u.blocks(it.key_end);
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
      if (!post(it)) return false;
    }
    x += take;
    in = 0;
    ++tile;
    if (x < x_end && tile * npt >= n) {
      tile = 0;
      if (++kvh == u.Hkv) {
        kvh = 0;
        do ++r; while (upto[r] <= x);            // requests without work
        start = u.rows.row_start[r];
        n = u.rows.n_rows[r];
        prefix = u.rows.prefix_len[r];
      }
    }
  }
  return true;
}

struct JoinArgs {
  const float* part_o;    // [CTA][2][D / 4][kUnitRows][4]; a CTA's first piece, its last
  const float2* part_ml;  // [CTA][2][kUnitRows]  (max in log2 units, sum)
  const PieceJoin* join;  // [CTA]
  uint16_t* out;
  int G, Hq;
};

// Joins the pieces of the units that end in another CTA than they began in: a
// thread has four dims of a row at a time.  Few CTAs, since most find nothing to
// join.
constexpr int kJoinThreads = 256;
constexpr int kJoinCtas = 4;                 // per CTA of the attention

template <int D, bool F16>
__global__ void __launch_bounds__(kJoinThreads, 4) join_pieces_kernel(JoinArgs a) {
  pdl_launch_dependents();
  pdl_wait();
  const int c0 = blockIdx.x;
  const PieceJoin j = a.join[c0];
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
        const size_t part = static_cast<size_t>(c0 + s0 + u) * 2 + (s0 + u == 0 ? 1 : 0);
        w[u] = in ? a.part_ml[part * kUnitRows + row] : make_float2(-INFINITY, 0.0f);
        v[u] = in ? po[(part * kQuads + quad) * kUnitRows + row] : acc;
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

// Workspace of a pieces' kernel and its join.
struct PieceWs {
  size_t part_o, part_ml, join, total;
};
inline PieceWs piece_ws(int D) {
  PieceWs w{};
  const size_t slots = static_cast<size_t>(kMaxCtas) * 2 * kUnitRows;
  w.part_o = 0;
  w.part_ml = w.part_o + slots * D * sizeof(float);
  w.join = w.part_ml + slots * sizeof(float2);
  w.total = (w.join + kMaxCtas * sizeof(PieceJoin) + 255) & ~static_cast<size_t>(255);
  return w;
}

}  // namespace pct
