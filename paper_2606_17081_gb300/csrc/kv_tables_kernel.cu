// A step's block tables, positions and slot maps from its requests' lengths
// (kv_tables), and its K and V into the blocks (kv_append).
#include <algorithm>
#include <climits>

#include "rs_internal.h"

namespace rs {

namespace {

constexpr int NT_TAB = 512;          // threads of a k_kv_tables CTA
constexpr int TAB_GROUPS = 2048;     // groups whose starts are kept in shared memory

// Last index i in [0, n) with a[i] <= x, given a[0] <= x (a non-decreasing).
template <class T>
__device__ __forceinline__ int last_le(const T* a, int n, T x) {
  int lo = 0, hi = n;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (a[mid] <= x) lo = mid; else hi = mid;
  }
  return lo;
}

__device__ __forceinline__ int32_t clip32(int64_t x) { return x > INT_MAX ? INT_MAX : (int32_t)x; }

struct Lens {
  int32_t q, prev, kv;
};

// The request's lengths, negative ones as 0, ending at 2^31 - 17.
__device__ __forceinline__ Lens req_lens(const int32_t* q_len, const int32_t* prev_len, int i) {
  Lens l;
  const int top = INT_MAX - 16;
  l.prev = min(max(prev_len[i], 0), top);
  l.q = min(max(q_len[i], 0), top - l.prev);
  l.kv = l.prev + l.q;
  return l;
}

// Per request i: s_i = sum of the q before it, f_i = sum of the new blocks
// before it.  Both sums are over all requests, so every CTA scans all lengths
// by itself (8 bytes a request, from L2) and keeps both starts in shared
// memory: the call is one launch, with no counter or second pass.  Then the
// grid shares the rows of positions and slots (a binary search in shared
// memory finds a row's request) and the table rows (warps, several to a request
// when there are fewer requests than warps).  A slot's block comes from where
// the table entry comes from (prefix list, kept entry, free list), so that no
// thread waits for another's table write.
// Bound: launch and latency.  64 requests of single tokens (26 KB): 4.7 us; 1024
// prompts with 262 000 tokens (3.8 MB, 0.6 us at the copy rate): 11.6 us, of which
// a row's search and lengths are most.
// The inputs are not __restrict__, here and below: such reads may go by the read-only path, which asks for data that
// nobody writes while the kernel runs, and it runs already (behind_stream) while the kernel before it writes.
__global__ void __launch_bounds__(NT_TAB) k_kv_tables(rs_kv_batch b, const int32_t* q_len, const int32_t* prev_len,
                                                      const int32_t* prefix_blocks, int64_t prefix_stride,
                                                      const int32_t* free_ids, int64_t n_free,
                                                      int32_t* __restrict__ positions,
                                                      int64_t* __restrict__ slots,
                                                      int64_t* __restrict__ counts) {
  extern __shared__ int32_t sm[];
  const int n = b.n_req, G = b.n_groups;
  int32_t* s_tok = sm;              // [n] first row, ends at INT_MAX
  int32_t* s_new = sm + n;          // [n] rank of the first new block, likewise
  int32_t* s_grp = sm + 2 * n;      // [G + 1] when G <= TAB_GROUPS
  __shared__ int64_t w_tok[NT_TAB / 32], w_new[NT_TAB / 32];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int32_t* grp = b.group_start;
  behind_stream();
  if (G > 0 && G <= TAB_GROUPS) {
    for (int g = tid; g <= G; g += NT_TAB) s_grp[g] = b.group_start[g];
    grp = s_grp;
  }
  __syncthreads();
  // blocks of the prefix that request i shares, and its group
  auto prefix_of = [&](int i, int& g) -> int {
    g = -1;
    if (G == 0 || i < grp[0] || i >= grp[G]) return 0;
    g = last_le(grp, G, i);
    const int64_t p = max(b.prefix_len[g], 0) >> 4;
    return (int)min(min(p, prefix_stride), (int64_t)b.max_blocks);
  };
  // its first new block, and the end of its blocks, within the table's row
  auto new_blocks = [&](const Lens& l, int pb, int& end) -> int {
    const int first = min(max((l.prev + 15) >> 4, pb), b.max_blocks);
    end = max(first, min((l.kv + 15) >> 4, b.max_blocks));
    return first;
  };
  int64_t tok0 = 0, new0 = 0;   // of the requests of earlier passes
  for (int base = 0; base < n; base += NT_TAB) {
    const int i = base + tid;
    int64_t t = 0, f = 0;
    if (i < n) {
      const Lens l = req_lens(q_len, prev_len, i);
      int g, end;
      const int pb = prefix_of(i, g);
      const int first = new_blocks(l, pb, end);
      t = l.q;
      f = end - first;
    }
    int64_t st = t, sf = f;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int64_t x = __shfl_up_sync(~0u, st, o), y = __shfl_up_sync(~0u, sf, o);
      if (lane >= o) { st += x; sf += y; }
    }
    if (lane == 31) { w_tok[warp] = st; w_new[warp] = sf; }
    __syncthreads();
    int64_t at = tok0 + st - t, af = new0 + sf - f;
    for (int w = 0; w < NT_TAB / 32; w++) {
      if (w < warp) { at += w_tok[w]; af += w_new[w]; }
      tok0 += w_tok[w];
      new0 += w_new[w];
    }
    if (i < n) {
      s_tok[i] = clip32(at);
      s_new[i] = clip32(af);
    }
    __syncthreads();
  }
  const int32_t total = clip32(tok0);
  const int gt = blockIdx.x * NT_TAB + tid, gn = gridDim.x * NT_TAB;
  if (gt == 0) {
    counts[0] = new0;
    counts[1] = tok0;
    b.q_start[n] = total;
  }
  for (int i = gt; i < n; i += gn) {
    b.q_start[i] = s_tok[i];
    b.kv_len[i] = req_lens(q_len, prev_len, i).kv;
  }
  // rows
  for (int r = gt; r < b.n_tokens; r += gn) {
    int32_t pos = -1;
    int64_t slot = -1;
    if (r < total) {
      const int i = last_le(s_tok, n, r);   // (requests without tokens share their start with the next)
      const Lens l = req_lens(q_len, prev_len, i);
      int g, end;
      const int pb = prefix_of(i, g);
      const int first = new_blocks(l, pb, end);
      pos = l.prev + (r - s_tok[i]);
      const int k = pos >> 4;
      int32_t id = -1;
      if (k < pb) {
        id = prefix_blocks[(int64_t)g * prefix_stride + k];
      } else if (k < first) {
        id = b.table[(int64_t)i * b.table_stride + k];
      } else if (k < end) {
        const int64_t rank = (int64_t)s_new[i] + (k - first);
        if (rank < n_free) id = free_ids[rank];
      }
      if (id >= 0) slot = (int64_t)id * 16 + (pos & 15);
    }
    positions[r] = pos;
    slots[r] = slot;
  }
  // table rows
  const int nw = gn >> 5, gw = gt >> 5;
  const int per = max(1, nw / max(n, 1));   // warps to a request
  for (int u = gw; u < n * per; u += nw) {
    const int i = u / per, part = u - i * per;
    const Lens l = req_lens(q_len, prev_len, i);
    int g, end;
    const int pb = prefix_of(i, g);
    const int first = new_blocks(l, pb, end);
    int32_t* row = b.table + (int64_t)i * b.table_stride;
    const int32_t* src = prefix_blocks + (int64_t)max(g, 0) * prefix_stride;
    for (int k = part * 32 + lane; k < pb; k += per * 32) row[k] = src[k];
    for (int k = first + part * 32 + lane; k < end; k += per * 32) {
      const int64_t rank = (int64_t)s_new[i] + (k - first);
      row[k] = rank < n_free ? free_ids[rank] : -1;
    }
  }
}

// Rows of K and V into their slots: per row the heads' elements of K, then of
// V, in pieces of V elements (16 bytes each when the source is aligned so).
// A thread moves UNR pieces whose loads are all in flight together; the rows
// are read past L1 (they are read once).
// Bound: HBM, each byte read once and written once.  131 MB (16 001 rows of 8
// heads of 128): 18.4 us, 7.1 TB/s; 20.2 us with loads through L1, 22.0 us
// with 64-bit places too, 24.5 us with UNR = 8.
template <class T, int UNR>
__global__ void __launch_bounds__(256) k_kv_append(rs_kv_cache c, const uint16_t* k, const uint16_t* v,
                                                   int64_t ts, int64_t hs, uint32_t total, const int64_t* slots,
                                                   uint32_t row_pieces, uint32_t head_pieces) {
  constexpr int V = sizeof(T) / 2;
  const int64_t end = c.n_blocks * 16;
  const uint32_t base = blockIdx.x * (256 * UNR) + threadIdx.x;
  T val[UNR];
  uint16_t* dst[UNR];
  behind_stream();
#pragma unroll
  for (int u = 0; u < UNR; u++) {
    const uint32_t x = base + u * 256;
    dst[u] = nullptr;
    if (x >= total) continue;
    const uint32_t r = x / row_pieces;
    uint32_t p = x - r * row_pieces;
    const bool second = p >= (row_pieces >> 1);
    if (second) p -= row_pieces >> 1;
    const uint32_t h = p / head_pieces, e = (p - h * head_pieces) * V;
    const int64_t slot = slots[r];
    if (slot < 0 || slot >= end) continue;
    val[u] = __ldcs(reinterpret_cast<const T*>((second ? v : k) + r * ts + h * hs + e));
    dst[u] = reinterpret_cast<uint16_t*>(second ? c.v : c.k) + (slot >> 4) * c.stride_block +
             h * c.stride_head + (slot & 15) * c.stride_token + e;
  }
#pragma unroll
  for (int u = 0; u < UNR; u++)
    if (dst[u]) *reinterpret_cast<T*>(dst[u]) = val[u];
}

}  // namespace

cudaError_t launch_kv_tables(const rs_kv_batch& b, const int32_t* q_len, const int32_t* prev_len,
                             const int32_t* prefix_blocks, int64_t prefix_stride,
                             const int32_t* free_ids, int64_t n_free, int32_t* positions,
                             int64_t* slots, int64_t* counts, int sms, cudaStream_t st) {
  const size_t smem = ((size_t)2 * b.n_req + (b.n_groups <= TAB_GROUPS ? b.n_groups + 1 : 0)) * 4;
  // (the limit belongs to the kernel, not to the call: every call sets the most that any needs, or another thread's call
  // could lower it before this one's launch)
  cudaError_t e = cudaFuncSetAttribute(k_kv_tables, cudaFuncAttributeMaxDynamicSharedMemorySize, (2 * KV_MAX_REQ + TAB_GROUPS + 1) * 4);
  if (e != cudaSuccess) return e;
  // rows in threads and requests in warps
  const int64_t want = std::max<int64_t>((b.n_tokens + NT_TAB - 1) / NT_TAB, (b.n_req + 15) / 16);
  const int grid = (int)std::min<int64_t>(std::max<int64_t>(want, 1), sms);
  return launch_behind(k_kv_tables, grid, NT_TAB, smem, st, b, q_len, prev_len, prefix_blocks, prefix_stride, free_ids,
                       n_free, positions, slots, counts);
}

cudaError_t launch_kv_append(const rs_kv_cache& c, const void* k, const void* v, int64_t ts, int64_t hs,
                             int n_tokens, const int64_t* slots, int sms, cudaStream_t st) {
  const bool wide = ((reinterpret_cast<uintptr_t>(k) | reinterpret_cast<uintptr_t>(v)) & 15) == 0 &&
                    ts % 8 == 0 && hs % 8 == 0;
  const int hp = c.head_dim / (wide ? 8 : 1), rp = 2 * c.n_kv_heads * hp;
  const uint16_t *kp = static_cast<const uint16_t*>(k), *vp = static_cast<const uint16_t*>(v);
  // places are 32 bits: rows in runs of up to 2^31 pieces (at least 2^13 rows)
  const int most = (1 << 30) / rp * 2;
  for (int r0 = 0; r0 < n_tokens; r0 += most) {
    const uint32_t total = (uint32_t)std::min(most, n_tokens - r0) * rp;
    const uint16_t *kr = kp + r0 * ts, *vr = vp + r0 * ts;
    // one piece a thread while that leaves an SM no more than two CTAs (64 rows of 8 heads of 128: 2.2 us against 3.1 us)
    const bool small = total <= (uint32_t)sms * 512;
    const unsigned grid = (total + (small ? 255 : 1023)) / (small ? 256 : 1024);
    auto kernel = wide ? small ? k_kv_append<uint4, 1> : k_kv_append<uint4, 4>
                       : small ? k_kv_append<uint16_t, 1> : k_kv_append<uint16_t, 4>;
    const cudaError_t e = launch_behind(kernel, grid, 256, 0, st, c, kr, vr, ts, hs, total, slots + r0, (uint32_t)rp, (uint32_t)hp);
    if (e != cudaSuccess) return e;
  }
  return cudaSuccess;
}

}  // namespace rs
