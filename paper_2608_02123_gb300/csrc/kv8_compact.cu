// pctree_kv8_compact: the accepted path's rows of an 8-bit cache, moved behind
// the verified prefix in all layers.
//
// A block of slots that accepted rows go to gets the largest scale of the rows
// that it then holds: codes of a smaller scale are divided by the quotient, a
// power of two (exact but for subnormal codes).  a[j] >= j, so rows are moved in
// ascending order with a window's sources read before its slots are written; a
// later source lies behind every slot written before it.
//
// A warp moves one head of a request, layer and plane: 16 bytes a lane, 32 / (D /
// 16) rows side by side, all rows of a window of up to 32 slots in flight.
//
// What bounds it (one GB300, us): 32 requests of 40 layers (53 MB) 29.4, 0.26 of the
// measured copy rate: a warp's chain of dependent reads (path, pages, scales, codes),
// with three CTAs an SM; four of 64 registers spill (30.5), two have too few warps
// (35.0), and a warp's items of one request, with one look at its path, lie apart in
// memory from its neighbours' (36.0).
#include "kv8.cuh"
#include "sm103_ptx.cuh"

namespace pct {
namespace {

constexpr int kCompactThreads = 256;
constexpr int kCompactWarps = kCompactThreads / 32;

struct Kv8CompactArgs {
  KvRows rows;                               // (row_start, n_rows unused)
  Kv8Blocks blocks;
  const int32_t* accepted_idx;
  const int32_t* accepted_len;
  uint8_t* cache[2];
  uint8_t* scale[2];
  int32_t* status;
  long long cache_layer, scale_layer;        // bytes from layer to layer
  long long items;
  int B, N, layers, Hkv;
};

template <int D>
__global__ void __launch_bounds__(kCompactThreads, 3) kv8_compact_kernel(Kv8CompactArgs a) {
  constexpr int S = D / 16;                  // lanes per row
  constexpr int kRows = 32 / S;              // rows side by side
  const int lane = threadIdx.x & 31;
  const int s = lane % S, part = lane / S;
  pdl_launch_dependents();
  pdl_wait();
  for (long long item = static_cast<long long>(blockIdx.x) * kCompactWarps + (threadIdx.x >> 5);
       item < a.items; item += static_cast<long long>(gridDim.x) * kCompactWarps) {
    // head, plane, layer, request: neighbouring warps have neighbouring bytes
    const int h = static_cast<int>(item % a.Hkv);
    long long rest = item / a.Hkv;
    const int plane = static_cast<int>(rest & 1);
    rest >>= 1;
    const int layer = static_cast<int>(rest % a.layers);
    const int r = static_cast<int>(rest / a.layers);
    const int T = a.rows.prefix_len[r], L = a.accepted_len[r];
    const int32_t* idx = a.accepted_idx + static_cast<size_t>(r) * (a.B + 1);
    // place of a slot and of its scale; false if its page is no page
    auto find = [&](int slot, long long& place, long long& at) {
      const int entry = div_by(slot, a.blocks.page), off = slot - entry * a.rows.page_size;
      const int page = kv_page(a.rows, r, entry);
      place = static_cast<long long>(page) * a.rows.page_size + off;
      at = static_cast<long long>(page) * a.blocks.per_page + (off >> a.blocks.shift);
      return page >= 0;
    };
    const int slots = a.rows.max_pages * a.rows.page_size;     // <= 2^30
    bool bad = L < 0 || L > a.B || T < 0 || T >= slots;
    if (!bad)
      for (int j = lane; j <= L; j += 32) {
        const int x = idx[j];
        long long place, at;
        // (the tree may be smaller than N: its rows' slots must be there, and j <= x)
        bad = bad || x < j || x >= a.N || x >= slots - T || (j == 0 ? x != 0 : x <= idx[j - 1]) ||
              !find(T + j, place, at) || !find(T + x, place, at);
      }
    if (__any_sync(kFull, bad)) {
      if (lane == 0 && a.status != nullptr) atomicCAS(a.status, 0, PCTREE_ERR_INVALID_ARG);
      continue;
    }
    uint8_t* cache = a.cache[plane] + layer * a.cache_layer + h * D + s * 16;
    uint8_t* scale = a.scale[plane] + layer * a.scale_layer + h;
    const int block = 1 << a.blocks.shift, end = T + L + 1;
    // start of the block that holds a slot
    auto block_start = [&](int slot) {
      const int off = slot - div_by(slot, a.blocks.page) * a.rows.page_size;
      return slot - (off & (block - 1));
    };
    for (int w0 = block_start(T), w1; w0 < end; w0 = w1) {
      // whole blocks of together at most 32 slots, or a larger block
      if (block <= 32) {
        w1 = block_start(w0 + 32);
      } else {
        const int entry = div_by(w0, a.blocks.page);
        w1 = min(w0 + block, (entry + 1) * a.rows.page_size);
      }
      const int stop = min(w1, end);
      int most = 0;                          // of a larger block: its largest source's byte
      if (block > 32) {
        for (int x = w0 + lane; x < stop; x += 32) {
          long long place, at;
          find(x < T ? x : T + idx[x - T], place, at);
          most = max(most, static_cast<int>(scale[at * a.Hkv]));
        }
        most = __reduce_max_sync(kFull, most);
      }
      for (int x0 = w0; x0 < stop; x0 += 32) {
        // a lane finds one slot's places, then rows go to S lanes each
        const int x = x0 + lane;
        const bool in = x < stop;
        const int src = !in ? 0 : x < T ? x : T + idx[x - T];
        long long to = -1, to_at = -1, of = -1, of_at = -1;
        if (in) {
          find(x, to, to_at);
          find(src, of, of_at);
        }
        const int old = in ? scale[of_at * a.Hkv] : 0;
        int now = most;
        if (block <= 32) {
          const int id = in ? block_start(x) : -1;
          const unsigned same = __match_any_sync(kFull, id);
          now = __reduce_max_sync(same, old);
        }
        // 0: stays as it is; else the codes' factor
        const float by = !in || (src == x && old == now)
                             ? 0.0f
                             : exp2_of(max(-126, scale_exp(old) - scale_exp(now)));
        uint4 code[S];
#pragma unroll
        for (int u = 0; u < S; ++u) {
          const int from = u * kRows + part;
          const long long p = __shfl_sync(kFull, of, from);
          const float f = __shfl_sync(kFull, by, from);
          if (f != 0.0f) code[u] = *reinterpret_cast<const uint4*>(cache + p * a.Hkv * D);
        }
        __syncwarp();
#pragma unroll
        for (int u = 0; u < S; ++u) {
          const int from = u * kRows + part;
          const long long p = __shfl_sync(kFull, to, from);
          const float f = __shfl_sync(kFull, by, from);
          if (f != 0.0f)
            *reinterpret_cast<uint4*>(cache + p * a.Hkv * D) =
                f == 1.0f ? code[u] : rescaled16(code[u], f);
        }
        __syncwarp();
        // a block's scale, once none of its codes is still to be read
        if (in && x0 + 32 >= stop && scale[to_at * a.Hkv] != now)
          scale[to_at * a.Hkv] = static_cast<uint8_t>(now);
        __syncwarp();
      }
    }
  }
}

pctree_status compact_check(const pctree_kv8_compact_config* c) {
  if (c == nullptr || c->B < 0 || c->N < 1 || c->layers < 1 || c->D < 1)
    return PCTREE_ERR_INVALID_ARG;
  const pctree_status st = kv_check(c->batch, 1, c->Hkv, c->page_size, c->n_pages, c->max_pages,
                                    PCTREE_BF16);
  if (st != PCTREE_OK) return st;
  if (!kv8_block_ok(c->scale_block)) return PCTREE_ERR_INVALID_ARG;
  if (static_cast<long long>(c->max_pages) * c->page_size < c->N) return PCTREE_ERR_INVALID_ARG;
  if ((c->D != 64 && c->D != 128) || c->B > (1 << 20) || c->layers > (1 << 20))
    return PCTREE_ERR_UNSUPPORTED;
  const Kv8Blocks b = kv8_blocks(c->page_size, c->scale_block);
  const long long slot = static_cast<long long>(c->Hkv) * c->D;
  if (c->layers > 1 &&
      (c->cache_layer_stride % 16 != 0 ||
       c->cache_layer_stride / slot / c->page_size < c->n_pages ||
       c->scale_layer_stride / c->Hkv / b.per_page < c->n_pages))
    return PCTREE_ERR_INVALID_ARG;
  return PCTREE_OK;
}

}  // namespace
}  // namespace pct

extern "C" {

pctree_status pctree_kv8_compact(const pctree_kv8_compact_config* cfg,
                                 const int32_t* accepted_idx, const int32_t* accepted_len,
                                 const int32_t* prefix_len, const int32_t* page_table,
                                 void* k_cache, void* v_cache, void* k_scale, void* v_scale,
                                 int32_t* status, void* stream) {
  using namespace pct;
  NvtxRange range("pctree_kv8_compact");
  pctree_status st = compact_check(cfg);
  if (st != PCTREE_OK) return st;
  const pctree_kv8_compact_config& c = *cfg;
  if (accepted_idx == nullptr || accepted_len == nullptr || prefix_len == nullptr ||
      k_cache == nullptr || v_cache == nullptr || k_scale == nullptr || v_scale == nullptr ||
      !kv_al16(k_cache) || !kv_al16(v_cache) ||
      !kv_table_ok(page_table, c.batch, c.n_pages, c.max_pages))
    return PCTREE_ERR_INVALID_ARG;
  int num_sms = 0;
  st = device_facts(&num_sms);
  if (st != PCTREE_OK) return st;
  Kv8CompactArgs a{};
  a.rows = {nullptr, nullptr, prefix_len, page_table, c.batch, 1, c.page_size, c.n_pages,
            c.max_pages};
  a.blocks = kv8_blocks(c.page_size, c.scale_block);
  a.accepted_idx = accepted_idx;
  a.accepted_len = accepted_len;
  a.cache[0] = static_cast<uint8_t*>(k_cache);
  a.cache[1] = static_cast<uint8_t*>(v_cache);
  a.scale[0] = static_cast<uint8_t*>(k_scale);
  a.scale[1] = static_cast<uint8_t*>(v_scale);
  a.status = status;
  a.cache_layer = c.cache_layer_stride;
  a.scale_layer = c.scale_layer_stride;
  a.items = static_cast<long long>(c.batch) * c.layers * 2 * c.Hkv;
  a.B = c.B;
  a.N = c.N;
  a.layers = c.layers;
  a.Hkv = c.Hkv;
  long long ctas = (a.items + kCompactWarps - 1) / kCompactWarps;
  if (ctas > 3ll * num_sms) ctas = 3ll * num_sms;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cudaLaunchConfig_t lc = {};
  lc.gridDim = dim3(static_cast<unsigned>(ctas));
  lc.blockDim = dim3(kCompactThreads);
  lc.stream = static_cast<cudaStream_t>(stream);
  lc.attrs = attr;
  lc.numAttrs = 1;
  const void* fn = c.D == 64 ? reinterpret_cast<const void*>(kv8_compact_kernel<64>)
                             : reinterpret_cast<const void*>(kv8_compact_kernel<128>);
  void* params[] = {&a};
  return cudaLaunchKernelExC(&lc, fn, params) == cudaSuccess ? PCTREE_OK : PCTREE_ERR_CUDA;
}

}  // extern "C"
