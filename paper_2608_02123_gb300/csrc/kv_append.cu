// pctree_kv_append: per-head norms and the position rotation of new rows'
// queries and keys, and the append of keys and values to a paged or
// contiguous cache.
//
// A head is D/16 lanes of a warp, 16 elements each as two 16-byte pieces: the
// two halves of 8 rotation pairs (pieces s and s + rotary_dim/16 of a head
// whose pairs are (i, i + rotary_dim/2), else two pieces side by side), so a
// pair never leaves its lane and the norm is one shuffle reduction over the
// head's lanes.  A warp takes a run of a row's heads, queries, keys and values
// alike: the sines and cosines of the row's position are computed once for all
// of them (8 a lane).
//
// Angles: inv_freq / (2 pi) is held as a 64-bit fraction of a turn, so
// position * fraction wraps modulo one turn by itself, in integers; what is
// left is exact to position * 2^-53 turns, for any position.
//
// What bounds it: HBM for prompts (each element is read and written once: 370
// MB in 65 us, 0.84 of the measured copy rate), the launch for single tokens;
// in between (trees of 32 requests, 89 MB in 26.6 us) the rows a warp takes one
// after the other.  Four heads of loads ahead of the arithmetic and two CTAs an
// SM (us, trees / prompts): 26.6 / 65.2; two heads and three CTAs 33.1 / 70.2;
// six heads 27.1 / 64.0; eight and one CTA 35.5 / 89.6.  Arithmetic goes two
// elements at a time (before: 28.2 / 70.5).
#include "kv_rows.cuh"
#include "sm103_ptx.cuh"

namespace pct {
namespace {

constexpr int kAppendThreads = 256;
constexpr int kAppendWarps = kAppendThreads / 32;
constexpr int kAppendCtas = 2;      // an SM: 113 registers a thread
constexpr int kHeadsAhead = 4;      // heads a lane has loads in flight for

struct AppendArgs {
  KvRows rows;
  const uint16_t* q;
  const uint16_t* k;
  const uint16_t* v;
  const uint16_t* q_weight;
  const uint16_t* k_weight;
  const double* inv_freq;
  const int32_t* positions;
  uint16_t* k_cache;
  uint16_t* v_cache;
  uint16_t* q_out;
  int32_t* status;
  long long q_stride, k_stride, v_stride;
  int Hq, Hkv, rotary, interleaved;
  int parts, heads_per_part;        // runs of heads a row is divided into
  float eps, scale;
};

struct AppendShared {
  unsigned long long turn[128];                  // fraction of a turn per position
  alignas(16) float weight[2][256];              // of queries and keys
  int start[PCTREE_KV_MAX_BATCH], end[PCTREE_KV_MAX_BATCH], prefix[PCTREE_KV_MAX_BATCH];
};

template <bool F16, int D>
__global__ void __launch_bounds__(kAppendThreads, kAppendCtas) kv_append_kernel(AppendArgs a) {
  constexpr int S = D / 16;                      // lanes per head
  constexpr int kGroups = 32 / S;                // heads side by side in a warp
  __shared__ AppendShared sh;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int s = lane % S, group = lane / S;
  const int half = a.rotary / 2;
  pdl_launch_dependents();
  pdl_wait();
  for (int i = half + threadIdx.x; i < 128; i += kAppendThreads) sh.turn[i] = 0;
  for (int i = threadIdx.x; i < 2 * D; i += kAppendThreads) {
    const uint16_t* w = i < D ? a.q_weight : a.k_weight;
    const int d = i < D ? i : i - D;
    sh.weight[i < D ? 0 : 1][d] = w != nullptr ? unpack16<F16>(w[d]).x : 1.0f;
  }
  for (int i = threadIdx.x; i < half; i += kAppendThreads) {
    double t = a.inv_freq[i] * 0.15915494309189533577;   // 1 / (2 pi)
    if (!(fabs(t) < INFINITY)) {
      t = 0.0;
      if (blockIdx.x == 0 && a.status != nullptr) atomicCAS(a.status, 0, PCTREE_ERR_INVALID_ARG);
    }
    // the fraction in [-0.5, 0.5] as a signed 64-bit integer, twice over
    sh.turn[i] =
        static_cast<unsigned long long>(__double2ll_rn((t - rint(t)) * 9223372036854775808.0)) << 1;
  }
  for (int r = threadIdx.x; r < a.rows.batch; r += kAppendThreads) {
    const int start = a.rows.row_start[r], n = a.rows.n_rows[r], prefix = a.rows.prefix_len[r];
    const bool ok = kv_request_ok(a.rows, start, n, prefix);
    if (!ok && blockIdx.x == 0 && a.status != nullptr)
      atomicCAS(a.status, 0, PCTREE_ERR_INVALID_ARG);
    sh.start[r] = start;
    sh.end[r] = ok ? start + n : start;
    sh.prefix[r] = prefix;
  }
  __syncthreads();
  const int heads = a.Hq + 2 * a.Hkv;
  const bool rotated = s < a.rotary / 16;
  const int c0 = rotated && !a.interleaved ? s : 2 * s;
  const int c1 = rotated && !a.interleaved ? s + a.rotary / 16
                                           : 2 * s + 1;
  // (dims past rotary_dim: pieces 2 s and 2 s + 1 lie past it, since
  // s >= rotary_dim / 16)
  const long long items = static_cast<long long>(a.rows.total_rows) * a.parts;
  for (long long item = static_cast<long long>(blockIdx.x) * kAppendWarps + warp; item < items;
       item += static_cast<long long>(gridDim.x) * kAppendWarps) {
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
    if (r < 0) continue;                         // a row of no request
    const int h_end = min(heads, (part + 1) * a.heads_per_part);
    const uint16_t* q_row = a.q + row * a.q_stride;
    const uint16_t* k_row = a.k + row * a.k_stride;
    const uint16_t* v_row = a.v + row * a.v_stride;
    uint4 x0[kHeadsAhead], x1[kHeadsAhead];
    auto load = [&](int hb) {
#pragma unroll
      for (int u = 0; u < kHeadsAhead; ++u) {
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
    const int entry = slot / a.rows.page_size;
    const int page = kv_page(a.rows, r, entry);
    if (page < 0 && lane == 0 && a.status != nullptr)
      atomicCAS(a.status, 0, PCTREE_ERR_INVALID_ARG);
    const size_t place =
        (static_cast<size_t>(page < 0 ? 0 : page) * a.rows.page_size +
         (slot - entry * a.rows.page_size)) * a.Hkv * D;
    // the head lanes' eight angles, each worked out by one of the warp's groups
    uint64_t cs[4], sn[4], ns[4];                // cos, sin and -sin, in pairs
    if (a.rotary > 0) {
      constexpr int kOwn = 8 / kGroups;
      const long long pos = a.positions != nullptr ? a.positions[row] : slot;
      float c_own[kOwn], s_own[kOwn];
#pragma unroll
      for (int e = 0; e < kOwn; ++e) {
        const unsigned long long ph =
            static_cast<unsigned long long>(pos) * sh.turn[8 * s + group * kOwn + e];
        // half turns in [-1, 1)
        const float x = static_cast<float>(static_cast<int>(ph >> 32)) * (1.0f / 2147483648.0f);
        sincospif(x, &s_own[e], &c_own[e]);
        s_own[e] *= a.scale;
        c_own[e] *= a.scale;
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
        ns[e / 2] = pack2(-t[0], -t[1]);
      }
    }
    // every lane runs the same number of rounds: the reductions are warp-wide
    for (int hb = part * a.heads_per_part;;) {
#pragma unroll
      for (int u = 0; u < kHeadsAhead; ++u) {
        const int h = hb + u * kGroups + group;
        const bool is_q = h < a.Hq, is_v = h >= a.Hq + a.Hkv;
        const bool norm = (is_q ? a.q_weight : a.k_weight) != nullptr;
        uint64_t f0[4], f1[4];                   // the two pieces, two elements at a time
        uint64_t sum2 = 0;
        const uint32_t w0[4] = {x0[u].x, x0[u].y, x0[u].z, x0[u].w};
        const uint32_t w1[4] = {x1[u].x, x1[u].y, x1[u].z, x1[u].w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float2 lo = unpack16<F16>(w0[e]), hi = unpack16<F16>(w1[e]);
          f0[e] = pack2(lo.x, lo.y);
          f1[e] = pack2(hi.x, hi.y);
          sum2 = fma2(f0[e], f0[e], sum2);
          sum2 = fma2(f1[e], f1[e], sum2);
        }
        float sum, odd;
        unpack2(sum2, sum, odd);
        sum += odd;
#pragma unroll
        for (int o = S / 2; o > 0; o >>= 1) sum += __shfl_xor_sync(kFull, sum, o);
        if (h >= h_end) continue;
        if (!is_v && (norm || rotated)) {
          if (norm) {
            const float inv = rsqrtf(sum * (1.0f / D) + a.eps);
            const uint64_t inv2 = pack2(inv, inv);
            const ulonglong2* g0 = reinterpret_cast<const ulonglong2*>(&sh.weight[is_q ? 0 : 1][c0 * 8]);
            const ulonglong2* g1 = reinterpret_cast<const ulonglong2*>(&sh.weight[is_q ? 0 : 1][c1 * 8]);
#pragma unroll
            for (int e = 0; e < 4; e += 2) {
              const ulonglong2 p = g0[e / 2], q = g1[e / 2];
              f0[e] = mul2(mul2(f0[e], inv2), p.x);
              f0[e + 1] = mul2(mul2(f0[e + 1], inv2), p.y);
              f1[e] = mul2(mul2(f1[e], inv2), q.x);
              f1[e + 1] = mul2(mul2(f1[e + 1], inv2), q.y);
            }
          }
          if (rotated) {
            if (a.interleaved) {
              // a piece's element pairs are rotation pairs: piece 0 has the
              // angles 0..3, piece 1 the angles 4..7
              auto turn = [](uint64_t ab, float c, float t) {
                float x, y;
                unpack2(ab, x, y);
                return fma2(pack2(y, x), pack2(-t, t), mul2(ab, pack2(c, c)));
              };
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                float c, d, t, v;
                unpack2(cs[e / 2], c, d);
                unpack2(sn[e / 2], t, v);
                f0[e] = turn(f0[e], (e & 1) ? d : c, (e & 1) ? v : t);
                unpack2(cs[2 + e / 2], c, d);
                unpack2(sn[2 + e / 2], t, v);
                f1[e] = turn(f1[e], (e & 1) ? d : c, (e & 1) ? v : t);
              }
            } else {
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                const uint64_t p = f0[e];
                f0[e] = fma2(f1[e], ns[e], mul2(p, cs[e]));
                f1[e] = fma2(p, sn[e], mul2(f1[e], cs[e]));
              }
            }
          }
          auto packed = [](const uint64_t(&f)[4]) {
            uint32_t w[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              float lo, hi;
              unpack2(f[e], lo, hi);
              w[e] = pack16<F16>(lo, hi);
            }
            return make_uint4(w[0], w[1], w[2], w[3]);
          };
          x0[u] = packed(f0);
          x1[u] = packed(f1);
        }
        uint16_t* dst = is_q    ? a.q_out + (static_cast<size_t>(row) * a.Hq + h) * D
                        : !is_v ? a.k_cache + place + (h - a.Hq) * D
                                : a.v_cache + place + (h - a.Hq - a.Hkv) * D;
        if (is_q || page >= 0) {
          *reinterpret_cast<uint4*>(dst + (is_v ? 2 * s : c0) * 8) = x0[u];
          *reinterpret_cast<uint4*>(dst + (is_v ? 2 * s + 1 : c1) * 8) = x1[u];
        }
      }
      hb += kGroups * kHeadsAhead;
      if (hb >= h_end) break;
      load(hb);
    }
  }
}

pctree_status append_check(const pctree_append_config* c) {
  if (c == nullptr) return PCTREE_ERR_INVALID_ARG;
  if (c->Hq < 0 || c->D < 1 || c->rotary_dim < 0 || c->rotary_dim > c->D ||
      c->rotary_dim % 16 != 0 || (c->interleaved != 0 && c->interleaved != 1) ||
      !(c->eps >= 0.0f) || !(c->eps < 1e30f) || !(c->rope_scale > -1e30f) ||
      !(c->rope_scale < 1e30f))
    return PCTREE_ERR_INVALID_ARG;
  const pctree_status st = kv_check(c->batch, c->total_rows, c->Hkv, c->page_size, c->n_pages,
                                    c->max_pages, c->dtype);
  if (st != PCTREE_OK) return st;
  if ((c->D != 64 && c->D != 128 && c->D != 256) || c->Hq > 65535) return PCTREE_ERR_UNSUPPORTED;
  const int64_t most = 1ll << 40;
  if (c->k_stride % 8 != 0 || c->v_stride % 8 != 0 || c->q_stride % 8 != 0 ||
      c->k_stride < static_cast<int64_t>(c->Hkv) * c->D ||
      c->v_stride < static_cast<int64_t>(c->Hkv) * c->D ||
      c->q_stride < static_cast<int64_t>(c->Hq) * c->D || c->k_stride > most ||
      c->v_stride > most || c->q_stride > most)
    return PCTREE_ERR_INVALID_ARG;
  return PCTREE_OK;
}

template <bool F16>
const void* append_kernel(int D) {
  return D == 64    ? reinterpret_cast<const void*>(kv_append_kernel<F16, 64>)
         : D == 128 ? reinterpret_cast<const void*>(kv_append_kernel<F16, 128>)
                    : reinterpret_cast<const void*>(kv_append_kernel<F16, 256>);
}

}  // namespace
}  // namespace pct

extern "C" {

pctree_status pctree_kv_append(const pctree_append_config* cfg, const void* q, const void* k,
                               const void* v, const void* q_weight, const void* k_weight,
                               const double* inv_freq, const int32_t* positions,
                               const int32_t* row_start, const int32_t* n_rows,
                               const int32_t* prefix_len, const int32_t* page_table,
                               void* k_cache, void* v_cache, void* q_out, int32_t* status,
                               void* stream) {
  using namespace pct;
  NvtxRange range("pctree_kv_append");
  pctree_status st = append_check(cfg);
  if (st != PCTREE_OK) return st;
  const pctree_append_config& c = *cfg;
  if (k == nullptr || v == nullptr || k_cache == nullptr || v_cache == nullptr ||
      row_start == nullptr || n_rows == nullptr || prefix_len == nullptr ||
      (c.Hq > 0 && (q == nullptr || q_out == nullptr)) ||
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
  AppendArgs a{};
  a.rows = {row_start, n_rows, prefix_len, page_table, c.batch, c.total_rows,
            c.page_size, c.n_pages, c.max_pages};
  a.q = static_cast<const uint16_t*>(q);
  a.k = static_cast<const uint16_t*>(k);
  a.v = static_cast<const uint16_t*>(v);
  a.q_weight = static_cast<const uint16_t*>(q_weight);
  a.k_weight = static_cast<const uint16_t*>(k_weight);
  a.inv_freq = inv_freq;
  a.positions = positions;
  a.k_cache = static_cast<uint16_t*>(k_cache);
  a.v_cache = static_cast<uint16_t*>(v_cache);
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
  a.scale = c.rope_scale;
  // runs of heads: all that the SMs' warps take at once while rows are few (512
  // rows of 56 heads: 7.1 us in four runs a row, 8.8 in five, which need a second
  // round), whole rows (one set of sines and cosines) once there are enough
  const int heads = c.Hq + 2 * c.Hkv, groups = 512 / c.D;
  const long long warps = static_cast<long long>(num_sms) * kAppendWarps * kAppendCtas;
  long long parts = warps > c.total_rows ? warps / c.total_rows : 1;
  const int most = (heads + groups - 1) / groups;
  if (parts > most) parts = most;
  a.heads_per_part = (heads + static_cast<int>(parts) - 1) / static_cast<int>(parts);
  a.heads_per_part = (a.heads_per_part + groups - 1) / groups * groups;
  a.parts = (heads + a.heads_per_part - 1) / a.heads_per_part;
  const long long items = static_cast<long long>(c.total_rows) * a.parts;
  long long blocks = (items + kAppendWarps - 1) / kAppendWarps;
  if (blocks > num_sms * kAppendCtas) blocks = num_sms * kAppendCtas;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cudaLaunchConfig_t lc = {};
  lc.gridDim = dim3(static_cast<unsigned>(blocks));
  lc.blockDim = dim3(kAppendThreads);
  lc.stream = static_cast<cudaStream_t>(stream);
  lc.attrs = attr;
  lc.numAttrs = 1;
  const void* fn = c.dtype == PCTREE_F16 ? append_kernel<true>(c.D) : append_kernel<false>(c.D);
  void* params[] = {&a};
  return cudaLaunchKernelExC(&lc, fn, params) == cudaSuccess ? PCTREE_OK : PCTREE_ERR_CUDA;
}

}  // extern "C"
