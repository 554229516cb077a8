// Causal attention over a paged KV cache in 4 bits (kv_attend4): k_kv4_plan cuts the step
// into jobs (kv4_plan.cuh), k_kv4_tiles runs those of many rows on the tensor cores
// (kv4_tiles_kernel.cu), k_kv4_rows those of few, k_kv4_join joins parts.
//
// Mathematics.  A row (token, head) needs o = sum_j p_j v_j / sum_j p_j over the keys j
// below its limit, p_j = exp(scale s_j), s = q K^T.  Over any part of the keys the triple
// (m, l, o), m a reference for the scores, l = sum exp(s - m), o = sum exp(s - m) v, is
// enough: parts join with weights exp(m_part - m).
//
// What is held, code times scale, has at most 6 significant bits in 2^-10 .. 2688, so it is
// an fp16 number: both products are fp16 products with 32-bit sums for q of either type.
// The units of K and V are factors of the scores and of the result.  A q in fp16 enters as
// it is; one in bf16 is first multiplied by a power of two that brings its row's largest
// element to 2^13 .. 2^14 (an element below 2^-30 of that is rounded, to 2^-38 of it; the
// power is divided out of the scores).  A weight is exp2(3 + sl (s - m)), m one of the row's
// scores and at most 12 / sl below the others so far: it is at most 2^15 or so, and half of
// fp16's smallest step is 2^-28 of the weight at m.  (With 7 in place of 3 more references
// moved: 2048 tokens behind 14 336 took 510 us against 459 us.)  s - m before the product
// with sl: two scores of any size keep their difference.
#include <algorithm>
#include <climits>
#include <type_traits>

#include "kv4_plan.cuh"
#include "kv_mma.cuh"

namespace rs {

using namespace kv4;

namespace {

constexpr int NT_PLAN = 1024, PLAN_GROUPS = 1024;   // groups that the plan keeps in shared memory
constexpr int FEW_MAX = 32;        // requests and groups of up to so many rows are warps' jobs
constexpr int WARPS = 16;          // of a k_kv4_rows CTA

// ------------------------------------------------------------------ the plan

__device__ __forceinline__ int clampi(int64_t x, int lo, int hi) { return (int)(x < lo ? lo : x > hi ? hi : x); }

struct Sum {
  int n0, n1;          // jobs of warps, of CTAs (capped: more than there is room for stays that)
  int64_t c0, c1;      // their costs
  __device__ int n(int kind) const { return kind ? n1 : n0; }
  __device__ int64_t c(int kind) const { return kind ? c1 : c0; }
};
__device__ __forceinline__ Sum operator+(const Sum& a, const Sum& b) {
  return Sum{(int)min((unsigned)a.n0 + (unsigned)b.n0, (unsigned)INT_MAX), (int)min((unsigned)a.n1 + (unsigned)b.n1, (unsigned)INT_MAX), a.c0 + b.c0,
             a.c1 + b.c1};
}
__device__ __forceinline__ Sum sum_of(int kind, int n, int64_t c) { return kind ? Sum{0, n, 0, c} : Sum{n, 0, c, 0}; }
// Inclusive sums over a warp.
__device__ __forceinline__ Sum scan_warp(Sum s, int lane) {
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const Sum x{__shfl_up_sync(~0u, s.n0, o), __shfl_up_sync(~0u, s.n1, o), __shfl_up_sync(~0u, s.c0, o), __shfl_up_sync(~0u, s.c1, o)};
    if (lane >= o) s = s + x;
  }
  return s;
}
// Exclusive sum over the CTA's threads, of which only the first `width` have something, added to `before`, which moves on
// by the total.
__device__ __forceinline__ Sum scan_block(const Sum& x, Sum* sm, int width, Sum& before) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const Sum s = warp * 32 < width ? scan_warp(x, lane) : Sum{};
  auto less = [&](const Sum& y) { return Sum{y.n0 - x.n0, y.n1 - x.n1, y.c0 - x.c0, y.c1 - x.c1}; };
  if (lane == 31) sm[warp] = s;
  __syncthreads();
  Sum r;
  if (width <= 32) {
    r = before + less(s);
    before = before + sm[0];
  } else {
    const Sum w = scan_warp(sm[lane], lane);
    const int from = max(warp - 1, 0);
    const Sum ahead{__shfl_sync(~0u, w.n0, from), __shfl_sync(~0u, w.n1, from), __shfl_sync(~0u, w.c0, from), __shfl_sync(~0u, w.c1, from)};
    r = before + (warp ? ahead + less(s) : less(s));
    before = before + Sum{__shfl_sync(~0u, w.n0, 31), __shfl_sync(~0u, w.n1, 31), __shfl_sync(~0u, w.c0, 31), __shfl_sync(~0u, w.c1, 31)};
  }
  __syncthreads();
  return r;
}

struct Lens {
  int q0, q, kv;   // first row, rows, context up to the last of them (below 0: none of them sees anything)
};
__device__ __forceinline__ Lens lens_of(const rs_kv_batch& b, int i) {
  Lens r;
  const int from = b.q_start[i], end = b.q_start[i + 1], kv = b.kv_len[i];
  r.q0 = clampi(from, 0, b.n_tokens);
  r.q = max(clampi(end, 0, b.n_tokens) - r.q0, 0);
  // (past the step's rows where they end inside the request: those tokens are not there)
  r.kv = clampi((int64_t)max(kv, 0) - end + r.q0 + r.q, -(1 << 24), INT_MAX - 1);
  return r;
}
__device__ __forceinline__ int units_of(int kind, int keys) { return keys > 0 ? (keys - 1) / keys_of(kind) + 1 : 0; }
__device__ __forceinline__ int max_keys_of(const rs_kv_batch& b) { return (int)min((int64_t)b.max_blocks * 16, (int64_t)INT_MAX - 256); }

// Job k of request i (its cost's sum left out).
__device__ __forceinline__ Job own_job(int k, int i, int kind, const Lens& r, int key0, int alone, int ratio, int max_keys) {
  Job j;
  const int64_t rows = (int64_t)r.q * ratio;
  j.tok0 = r.q0;
  j.row0 = k * rows_of(kind);
  j.nrows = (int)max(min((int64_t)rows_of(kind), rows - j.row0), (int64_t)0);
  j.trow = i;
  j.key0 = key0;
  // up to what its last token sees
  j.kend = clampi((int64_t)r.kv - r.q + (int)(((unsigned)j.row0 + j.nrows + ratio - 1) / (unsigned)ratio), 0, max_keys);
  j.lim0 = r.kv - r.q + 1;
  j.flags = alone;
  // (one unit at least, of which they see nothing, for rows that no other job has or that the join looks for here)
  j.nt = max(units_of(kind, j.kend - key0), alone || r.kv > key0 ? 1 : 0);
  j.reserved0 = 0;
  j.cost = 0;
  return j;
}

// Shares of two units, or two tiles, at least.
__device__ __forceinline__ int64_t share_of(int64_t total, int workers, int kind) {
  return max(quotient(total + workers - 1, workers), (int64_t)(kind ? 30 : 24));
}

// How the two kinds share the SMs, and the shares.  CTAs of the tiles' kernel beside CTAs of the rows', as many of
// each as lets both end at one time T: x / (T - TILES_START) + y / (T - ROWS_START) = SMs, x and y what each kind takes
// of an SM.  (With both kinds on all SMs, one after the other, and so, us: a prompt's 509 tokens beside 32 single ones
// 51.2 and 44.4; 48 requests of 1 to 5 tokens in 2 groups 40.5 and 35.6; 192 in 8 groups 101 and 91; 64 on a prefix of
// 32 768 107 and 97.  With what follows now: 33.5, 36, 88, 93.)  Times in us, fitted to steps of both head sizes; a third
// more or less for one kind costs up to 20%, and rows that get too few SMs more than that: the tiles' number is rounded down.
constexpr float TILE_128 = 0.45f, TILE_64 = 0.34f;   // of an SM, by cost: of tiles with heads of 128, of 64
constexpr float UNIT_8 = 0.122f;                     // of rows' units, of an SM with 8 heads of 128 a chunk: their throughput
constexpr float UNIT_ALONE = 0.125f, JOB = 6.0f;     // of a worker, by cost, and a job: their latency
constexpr float TILES_START = 8.0f, ROWS_START = 8.0f;
__device__ __forceinline__ void split(const Plan& p, Head& h, int few_jobs, int64_t items, int longest, bool d128) {   // few_jobs: of warps, with units
  const int n = p.workers[1], teams = p.workers[0] / n;
  int tiles = n;
  h.ctas = n;
  h.whole = 0;
  if (h.total[1] > 0) {
    const float N = (float)n, jobs = (float)few_jobs * (float)p.chunks;
    const float x = (d128 ? TILE_128 : TILE_64) * (float)h.total[1];
    const float unit = fmaxf(UNIT_8 * (float)p.chunk * (d128 ? 0.125f : 0.0625f), UNIT_ALONE / (float)teams);
    const float y = unit * ((float)h.total[0] - (float)own_cost(0) * jobs) + JOB / (float)teams * jobs;
    if (h.total[0] > 0) {
      const float b = (TILES_START + ROWS_START) * N + x + y, c = TILES_START * ROWS_START * N + ROWS_START * x + TILES_START * y;
      const float T = (b + sqrtf(fmaxf(b * b - 4.0f * N * c, 0.0f))) / (2.0f * N);
      tiles = max(1, min(n - 2, (int)(x / (T - TILES_START))));
    }
    h.whole = whole_items(items, tiles, longest);
    if (h.whole) tiles = (int)items;
    if (h.total[0] > 0 && tiles < n) h.ctas = n - tiles;
  }
  h.per[0] = share_of(h.total[0], h.ctas * teams, 0);
  h.per[1] = share_of(h.total[1], tiles, 1);
}

// What rows over keys cost as a warp's jobs: 8 for a unit of up to 8 rows, by what a unit takes (0.12 us of an SM with heads
// of 128, 0.06 with 64).
__device__ __forceinline__ int64_t few_take(int64_t rows, int keys) {
  const int64_t full = rows / FEW, rest = rows - full * FEW;
  return units_of(0, keys) * (full * 13 + (rest > 8 ? 13 : rest > 0 ? 8 : 0)) + 8 * (full + 1);
}

// Whether sharing prefixes is worth another job's way through memory for each row, as it saves `saved` (of few_take) a kv
// head: from 7 hundred an SM on.  The limit is of work by these costs, not of a time: with heads of 128 it is some 10 us, with 64
// 5 to 6, as starts and joins are quicker there too.  Hundreds saved an SM, and us a call with and without, for heads of 128 and
// of 64: 8 requests of 4 rows on 1 024 keys 0.6: 18.6 and 16.5; 15.4 and 14.4.  98 of 5 on 1 040, one kv head, 1.5: 30.3 and 22.5; 26.3 and
// 19.4.  40 of 4 on 1 024 4.7: 29.9 and 29.5; 26.0 and 24.0.  4 of 4 on 16 384 5.1: 30.5 and 27.5; 19.9 and 21.2.  64 of 8 on 1 024 7.1: 35.3 and
// 41.7; 30.9 and 31.6.  2 of 4 on 65 536 8.6: 34.9 and 41.8; 23.0 and 27.3.  40 of 4 on 2 048 9.6: 31.3 and 36.2; 26.3 and 28.2.
#ifndef KV4_WORTH   // (a test builds with 0: every prefix is shared that costs less so)
#define KV4_WORTH 700
#endif
__device__ __forceinline__ bool worth(const Plan& p, int64_t saved) { return saved * p.heads >= (int64_t)KV4_WORTH * p.workers[1]; }

// The plan of a step of at most TINY requests, all of few rows, by one warp of every CTA for
// itself: a lane a request, of at most two jobs, then a group.
constexpr int TINY = 32;
__device__ __forceinline__ void tiny_plan(const rs_kv_batch& b, const Plan& p, Head* head, Job* jobs, int lane) {
  const int n = b.n_req, G = b.n_groups, max_keys = max_keys_of(b);
  Lens r{0, 0, 0};
  if (lane < n) r = lens_of(b, lane);
  const int q_begin = n > 0 ? clampi(b.q_start[0], 0, b.n_tokens) : 0, q_end = n > 0 ? clampi(b.q_start[n], 0, b.n_tokens) : 0;
  // lane g: the group's requests, its rows, and its prefix
  int g0 = 0, g1 = 0, T0 = 0, T1 = 0, P = 0;
  if (lane < G) {
    g0 = clampi(b.group_start[lane], 0, n);
    g1 = clampi(b.group_start[lane + 1], 0, n);
    T0 = clampi(b.q_start[g0], 0, b.n_tokens);
    T1 = clampi(b.q_start[max(g0, g1)], 0, b.n_tokens);
    P = min(max(b.prefix_len[lane], 0) & ~15, max_keys & ~15);
  }
  Job pre[2];
  int pre_cost[2] = {0, 0}, pre_count = 0, key0 = 0, alone = JOB_ALONE;
  unsigned shared = 0;
  int64_t saved = 0;
  int least = 0, keys = 0, rows = 0;   // lane g: of the group
  for (int g = 0; g < G; g++) {
    const int first = __shfl_sync(~0u, g0, g), last = __shfl_sync(~0u, g1, g), prefix = __shfl_sync(~0u, P, g);
    const bool has = lane >= first && lane < last && r.q > 0;
    const int seen = r.kv - r.q / 2, top = 1 << 25;
    const int apart = __reduce_add_sync(~0u, has ? (int)min(few_take(r.q * p.ratio, seen), (int64_t)top) : 0);
    const int own = __reduce_add_sync(~0u, has ? (int)min(few_take(r.q * p.ratio, seen - prefix), (int64_t)top) : 0);
    const int low = __reduce_min_sync(~0u, has ? r.kv - r.q + 1 : INT_MAX), most = __reduce_max_sync(~0u, has ? r.kv : 0);
    const int all = max(__shfl_sync(~0u, T1, g) - __shfl_sync(~0u, T0, g), 0) * p.ratio, upto = min(prefix, most);
    // two units a row for the parts' way through memory
    const int64_t saves = apart - (own + few_take(all, upto) + 2 * all);
    if (__popc(__ballot_sync(~0u, has)) > 1 && upto > 0 && all > 0 && all <= 2 * FEW && saves > 0) {
      shared |= 1u << g;
      saved += saves;
    }
    if (lane == g) {
      least = low;
      keys = upto;
      rows = all;
    }
  }
  if (!worth(p, saved)) shared = 0;
  for (unsigned todo = shared; todo; todo &= todo - 1) {
    const int g = __ffs(todo) - 1;
    const int first = __shfl_sync(~0u, g0, g), last = __shfl_sync(~0u, g1, g), prefix = __shfl_sync(~0u, P, g);
    if (lane >= first && lane < last) {
      alone = 0;
      key0 = prefix;
    }
  }
  if (shared >> lane & 1) {
    pre_count = (rows + FEW - 1) / FEW;
#pragma unroll
    for (int k = 0; k < 2; k++) {
      Job j = {};
      j.tok0 = T0;
      j.trow = g0;
      j.kend = j.lim0 = keys;
      j.flags = JOB_PREFIX | (least >= keys ? JOB_EVEN : 0);
      j.nt = units_of(0, keys);
      j.row0 = k * FEW;
      j.nrows = min(FEW, rows - k * FEW);
      pre[k] = j;
      pre_cost[k] = k < pre_count ? job_cost(0, j.nt, j.nrows) : 0;
    }
  }
  const int count = min((r.q * p.ratio + FEW - 1) / FEW, 2);   // (more than two only where starts decrease)
  int cost[2] = {0, 0};
  Job j[2];
#pragma unroll
  for (int k = 0; k < 2; k++)
    if (k < count) {
      j[k] = own_job(k, lane, 0, r, key0, alone, p.ratio, max_keys);
      cost[k] = job_cost(0, j[k].nt, j[k].nrows);
    }
  // all prefix jobs, then the requests' own
  auto place = [&](const Job* job, const int* c, int cnt, int64_t& all, int& jobs_all) {
    int64_t upto = c[0] + c[1];
    int jobs_upto = cnt;
#pragma unroll
    for (int z = 1; z < 32; z <<= 1) {
      const int64_t x = __shfl_up_sync(~0u, upto, z);
      const int y = __shfl_up_sync(~0u, jobs_upto, z);
      if (lane >= z) { upto += x; jobs_upto += y; }
    }
#pragma unroll
    for (int k = 0; k < 2; k++)
      if (k < cnt) {
        Job x = job[k];
        x.cost = all + upto - c[0] - c[1] + (k ? c[0] : 0);
        jobs[jobs_all + jobs_upto - cnt + k] = x;
      }
    all += __shfl_sync(~0u, upto, 31);
    jobs_all += __shfl_sync(~0u, jobs_upto, 31);
  };
  int64_t all = 0;
  int jobs_all = 0;
  if (G > 0) place(pre, pre_cost, pre_count, all, jobs_all);
  place(j, cost, count, all, jobs_all);
  if (blockIdx.x == 0 && G > 0) {   // what the join finds of the tokens
    const int what = alone ? TOK_ALONE : r.kv > key0 ? TOK_BOTH : TOK_PREFIX;
    for (int t = 0; t < r.q; t++) p.tok[r.q0 + t] = what;
  }
  if (lane == 0) {
    Head h = {};
    h.jobs[0] = jobs_all;
    h.total[0] = all * p.chunks;
    h.per[0] = share_of(h.total[0], p.workers[0], 0);
    h.ctas = p.workers[1];
    h.q_begin = q_begin;
    h.q_end = q_end;
    h.room = 1;
    *head = h;
    if (blockIdx.x == 0) *p.head = h;
  }
}

// One CTA: whether each group's prefix pays as jobs of its own, the jobs and their costs'
// sums.  Starts that decrease can ask for more jobs than there is room for: then there is
// no work at all.
// Bound: latency (a few dependent reads and sums over the CTA): 3 to 5 us, with groups 5 to 8.
__global__ void __launch_bounds__(NT_PLAN) k_kv4_plan(rs_kv_batch b, Plan p, int heads, bool d128) {
  __shared__ Sum s_scan[32];
  __shared__ int s_start[PLAN_GROUPS + 1], s_prefix[PLAN_GROUPS];   // of groups: first request; prefix in keys, below 0 where it is not shared
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, n = b.n_req, G = b.n_groups;
  __shared__ int s_longest;   // tiles of a CTA's job
  __shared__ int s_empty;     // warps' jobs without units (of members that end inside a prefix)
  __shared__ unsigned long long s_saved;   // by prefixes as jobs of their own
  const bool staged = G <= PLAN_GROUPS;
  if (warp == 0) s_scan[lane] = Sum{};
  if (tid == 0) {
    s_longest = 0;
    s_empty = 0;
    s_saved = 0;
  }
  __syncthreads();
  behind_stream();
  const int max_keys = max_keys_of(b);
  auto rows_at = [&](int i) { return clampi(b.q_start[i], 0, b.n_tokens); };
  auto lens = [&](int i) { return lens_of(b, i); };
  auto kind_of = [&](int64_t rows) { return rows > p.few_max ? 1 : 0; };
  auto prefix_of = [&](int g) { return min(max(b.prefix_len[g], 0) & ~15, max_keys & ~15); };
  // what rows over keys cost, in the units of few_take
  auto takes = [&](int64_t rows, int keys) -> int64_t {
    if (rows > p.few_max) {
      const int64_t full = rows / MANY, rest = rows - full * MANY;
      return units_of(1, keys) * (full * 120 + (rest > 128 ? 120 : rest > 0 ? 68 : 0));
    }
    return few_take(rows, keys);
  };
  Sum before{};
  bool share = false;
  // what every later step goes by, on its way at once
  Lens mine{0, 0, 0};
  if (tid < n) mine = lens(tid);
  const int q_begin = n > 0 ? rows_at(0) : 0, q_end = n > 0 ? rows_at(n) : 0;
  const int g_lo = G > 0 ? b.group_start[0] : 0, g_hi = G > 0 ? b.group_start[G] : 0;
  if (G > 0) {
    if (staged)
      for (int g = tid; g <= G; g += NT_PLAN) s_start[g] = b.group_start[g];
    // groups, a warp each: (shared: whether all rows see the prefix; else -1), first token, keys, end of tokens
    for (int g = warp; g < G; g += NT_PLAN / 32) {
      const int first = clampi(b.group_start[g], 0, n), last = clampi(b.group_start[g + 1], 0, n), P = prefix_of(g);
      const int t0 = rows_at(first), t1 = rows_at(max(first, last));
      int64_t apart = 0, own = 0;
      int least = INT_MAX, most = 0, members = 0;
      for (int i = first + lane; i < last; i += 32) {
        const Lens r = lens(i);
        if (r.q == 0) continue;
        const int seen = r.kv - r.q / 2;
        apart += takes((int64_t)r.q * p.ratio, seen);
        own += takes((int64_t)r.q * p.ratio, seen - P);
        least = min(least, r.kv - r.q + 1);
        most = max(most, r.kv);
        members++;
      }
#pragma unroll
      for (int o = 16; o; o >>= 1) {
        apart += __shfl_xor_sync(~0u, apart, o);
        own += __shfl_xor_sync(~0u, own, o);
      }
      least = __reduce_min_sync(~0u, least);
      most = __reduce_max_sync(~0u, most);
      members = __reduce_add_sync(~0u, members);
      if (lane == 0) {
        const int64_t rows = (int64_t)max(t1 - t0, 0) * p.ratio;
        const int keys = min(P, most);   // (what nobody has written yet is not read)
        // two units a row for the parts' way through memory
        const int64_t saves = apart - (own + takes(rows, keys) + 2 * rows);
        const bool pays = members > 1 && keys > 0 && rows > 0 && saves > 0;
        if (pays) atomicAdd(&s_saved, (unsigned long long)min(saves, (int64_t)1 << 40));
        p.group[g] = make_int4(pays ? least >= keys : -1, t0, keys, t1);
        if (staged) s_prefix[g] = pays ? P : -1;
      }
    }
    __syncthreads();
    share = worth(p, (int64_t)s_saved);
    for (int base = 0; share && base < G; base += NT_PLAN) {
      const int g = base + tid;
      int4 v = make_int4(-1, 0, 0, 0);
      Sum x{};
      int kind = 0, count = 0, nt = 0;
      int64_t rows = 0;
      if (g < G) v = __ldcg(p.group + g);
      if (v.x >= 0) {
        rows = (int64_t)(v.w - v.y) * p.ratio;
        kind = kind_of(rows);
        count = (int)((rows + rows_of(kind) - 1) / rows_of(kind));
        nt = units_of(kind, v.z);
        x = sum_of(kind, count, (int64_t)(count - 1) * job_cost(kind, nt, rows_of(kind)) +
                                    job_cost(kind, nt, (int)(rows - (int64_t)(count - 1) * rows_of(kind))));
      }
      if (v.x >= 0 && kind) atomicMax(&s_longest, nt);
      const Sum at = scan_block(x, s_scan, min(NT_PLAN, G - base), before);
      if (v.x >= 0) {
        const int f = at.n(kind);
        int64_t cost = at.c(kind);
        Job j = {};
        j.tok0 = v.y;
        j.trow = clampi(b.group_start[g], 0, n - 1);
        j.kend = j.lim0 = v.z;
        j.flags = JOB_PREFIX | (v.x ? JOB_EVEN : 0);
        j.nt = nt;
        for (int k = 0; k < count && (int64_t)f + k < p.cap[kind]; k++) {
          j.row0 = k * rows_of(kind);
          j.nrows = (int)min((int64_t)rows_of(kind), rows - j.row0);
          j.cost = cost;
          (kind ? p.jobs[1] : p.jobs[0])[f + k] = j;
          cost += job_cost(kind, nt, j.nrows);
        }
      }
    }
  }
  // the requests' own jobs
  for (int base = 0; base < n; base += NT_PLAN) {
    const int i = base + tid;
    Lens r{0, 0, 0};
    int key0 = 0, alone = JOB_ALONE, kind = 0, count = 0;
    if (i < n) {
      r = base == 0 ? mine : lens(i);
      const int64_t rows = (int64_t)r.q * p.ratio;
      kind = kind_of(rows);
      count = (int)((rows + rows_of(kind) - 1) / rows_of(kind));
      if (share && i >= g_lo && i < g_hi) {
        const int* const start = staged ? s_start : b.group_start;
        int lo = 0, hi = G;
        while (hi - lo > 1) {
          const int mid = (lo + hi) >> 1;
          if (start[mid] <= i) lo = mid; else hi = mid;
        }
        const int prefix = staged ? s_prefix[lo] : __ldcg(&p.group[lo].x) >= 0 ? prefix_of(lo) : -1;
        if (prefix >= 0) {
          alone = 0;
          key0 = prefix;
        }
      }
    }
    auto job = [&](int k, int i, int kind, const Lens& r, int key0, int alone) { return own_job(k, i, kind, r, key0, alone, p.ratio, max_keys); };
    // a request of few jobs is its thread's; a longer one is its warp's
    const bool longer = count > 4;
    int64_t own = 0;
    int empty = 0;
    if (!longer)
      for (int k = 0; k < count; k++) {
        const Job j = job(k, i, kind, r, key0, alone);
        own += job_cost(kind, j.nt, j.nrows);
        empty += !kind && j.nt == 0;
      }
    if (empty) atomicAdd(&s_empty, empty);
    const unsigned many = __ballot_sync(~0u, longer);
    auto others = [&](int src, Lens& o, int& kd, int& k0, int& al) {
      o = Lens{__shfl_sync(~0u, r.q0, src), __shfl_sync(~0u, r.q, src), __shfl_sync(~0u, r.kv, src)};
      kd = __shfl_sync(~0u, kind, src);
      k0 = __shfl_sync(~0u, key0, src);
      al = __shfl_sync(~0u, alone, src);
      return __shfl_sync(~0u, count, src);
    };
    for (unsigned todo = many; todo; todo &= todo - 1) {
      const int src = __ffs(todo) - 1;
      Lens o;
      int kd, k0, al;
      const int cnt = others(src, o, kd, k0, al);
      int64_t c = 0;
      for (int k = lane; k < cnt; k += 32) {
        const Job j = job(k, 0, kd, o, k0, al);
        c += job_cost(kd, j.nt, j.nrows);
      }
#pragma unroll
      for (int z = 16; z; z >>= 1) c += __shfl_xor_sync(~0u, c, z);
      if (lane == src) own = c;
    }
    // (the last of a request's jobs sees the most keys)
    if (kind) atomicMax(&s_longest, units_of(1, clampi(r.kv, 0, max_keys) - key0));
    const Sum at = scan_block(sum_of(kind, count, own), s_scan, min(NT_PLAN, n - base), before);
    const int first = at.n(kind);
    int64_t cost = at.c(kind);
    const bool room = (int64_t)first + count <= p.cap[kind];
    if (!longer && room)
      for (int k = 0; k < count; k++) {
        Job j = job(k, i, kind, r, key0, alone);
        j.cost = cost;
        (kind ? p.jobs[1] : p.jobs[0])[first + k] = j;
        cost += job_cost(kind, j.nt, j.nrows);
      }
    for (unsigned todo = many; todo; todo &= todo - 1) {
      const int src = __ffs(todo) - 1;
      Lens o;
      int kd, k0, al;
      const int cnt = others(src, o, kd, k0, al), row = __shfl_sync(~0u, i, src), f = __shfl_sync(~0u, first, src);
      int64_t c = __shfl_sync(~0u, cost, src);
      if (!__shfl_sync(~0u, (int)room, src)) continue;
      Job* const jobs = kd ? p.jobs[1] : p.jobs[0];
      for (int kb = 0; kb < cnt; kb += 32) {
        const int k = kb + lane;
        Job j = job(min(k, cnt - 1), row, kd, o, k0, al);
        const int64_t mine = k < cnt ? job_cost(kd, j.nt, j.nrows) : 0;
        int64_t upto = mine;
#pragma unroll
        for (int z = 1; z < 32; z <<= 1) {
          const int64_t y = __shfl_up_sync(~0u, upto, z);
          if (lane >= z) upto += y;
        }
        if (k < cnt) {
          j.cost = c + upto - mine;
          jobs[f + k] = j;
        }
        c += __shfl_sync(~0u, upto, 31);
      }
    }
    if (G > 0) {   // what the join finds of the request's tokens
      const int what = alone ? TOK_ALONE : r.kv > key0 ? TOK_BOTH : TOK_PREFIX;
      if (r.q <= 4)
        for (int t = 0; t < r.q; t++) p.tok[r.q0 + t] = what;
      for (unsigned todo = __ballot_sync(~0u, r.q > 4); todo; todo &= todo - 1) {
        const int src = __ffs(todo) - 1;
        const int q0 = __shfl_sync(~0u, r.q0, src), q = __shfl_sync(~0u, r.q, src), x = __shfl_sync(~0u, what, src);
        for (int t = lane; t < q; t += 32) p.tok[q0 + t] = x;
      }
    }
  }
  if (tid == 0) {
    Head h = {};
    const bool room = before.n0 <= p.cap[0] && before.n1 <= p.cap[1];
    if (room) {
      h.jobs[0] = before.n0;
      h.jobs[1] = before.n1;
      h.total[0] = before.c0 * p.chunks;
      h.total[1] = before.c1 * heads;
    }
    split(p, h, h.jobs[0] - s_empty, (int64_t)h.jobs[1] * heads, s_longest, d128);
    h.q_begin = q_begin;
    h.q_end = q_end;
    h.room = room;
    *p.head = h;
  }
}

// ------------------------------------------------------------------ PTX

__device__ __forceinline__ void mma(float* c, const uint32_t* a, uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t turn(uint32_t x) {   // an 8 x 8 matrix of 16 bits, transposed
  uint32_t y;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}
// ------------------------------------------------------------------ a warp's jobs

// A warp's walk and the piece it is at, in shared memory (its first lane moves on): the registers are the products'.
struct Turn {
  Walk walk;
  int item, t0, t1, more;
};
static_assert(sizeof(Walk) % 16 == 0, "aligned");

template <int D>
struct RowsLay {
  static constexpr int V = 8 * D, KS = 16 * D, VS = 17 * D;   // of a page: codes of K at 0, of V, scales
  static constexpr int PAGE_BYTES = 18 * D;
  static constexpr int STAGES = D == 128 ? 3 : 4;             // of two pages
  static constexpr int WARP_BYTES = STAGES * 2 * PAGE_BYTES;
  static constexpr int WALKS = WARPS * WARP_BYTES;            // Turn [WARPS]
  static constexpr int PLAN = WALKS + WARPS * (int)sizeof(Turn);   // of a tiny step: Head, Job [4 TINY]
  static constexpr int SMEM = PLAN + (int)sizeof(Head) + 4 * TINY * (int)sizeof(Job);
  static_assert(sizeof(Head) % 16 == 0 && sizeof(Turn) % 16 == 0, "aligned");
  static_assert(SMEM <= 227 * 1024, "shared memory");
};

// Units t0 .. t1 - 1 (two pages each) of a job of up to 8 N rows, for kv head `head`.
//
// Scores come as S^T = K q^T (m16n8k16: 16 keys, 8 rows), the result as O^T = V^T p^T (16
// elements, 8 rows): the rows are the 8 columns, so few rows waste little.  Lane (g, t) =
// (lane / 4, lane % 4) has as its part of K's fragments the D / 4 elements from t D / 4 on
// of keys g and g + 8 of a page (any order of the elements will do that q has too), one
// read of 16 bytes each; as its part of V's the D / 8 elements from g D / 8 on of keys 2t,
// 2t + 1, 2t + 8, 2t + 9, whose nibbles are put in pairs of keys before they are converted.
// So codes go from shared memory to the products' registers, and nothing is written back.
// Weights are turned from S^T's fragment to p^T's by movmatrix.
// (tcgen05 would want K and V as tiles in shared memory: at these sizes writing and reading them would take longer than
// HBM takes for the codes.)
// Bound: HBM with up to 8 rows: 128 contexts of 2 048 to 24 576, 8 kv heads of 128, 1.33 GB in 231 us, 5.76 TB/s; a page
// takes an SM 119 clocks, 101 at the copy rate, and 292 instructions (73 clocks of issue), of which the conversions,
// 64, and the scales' products, 64, go through pipes of half rate.  With 9 to 16 rows the same contexts take 370 us, 191
// clocks a page: a page at a time, a stage less, q from shared memory, and at 128 registers 72 bytes of spills; mma.sync
// (1 024 multiply-adds a clock and SM) is a third of it.
// Measured and not kept: a page at a time (247 against 237 us a call); this function out of line (259 us).
template <int D, bool HALF, int N>
__device__ __forceinline__ void rows_segment(const KvAttend4Args& a, const Plan& p, const Job& job, int head, int t0, int t1, int worker,
                                             uint32_t ring) {
  using L = RowsLay<D>;
  constexpr int KS = D / 16, MT = D / 16;   // steps of 16 elements, tiles of 16 elements
  // (q of 16 rows would not leave the registers to the result's fragments: it lies in the last stage's place)
  constexpr int STAGES = N == 1 ? L::STAGES : L::STAGES - 1, U = N == 1 ? 2 : 1;
  const uint32_t qs = ring + STAGES * 2 * L::PAGE_BYTES;
  const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const rs_kv_cache4& c = a.c;
  const int k0 = job.key0 + t0 * UNIT, kend = min(job.kend, job.key0 + t1 * UNIT);   // the segment's keys
  const int cnt = t1 - t0, p0 = k0 / PAGE, pages = (kend - k0 + PAGE - 1) / PAGE;
  // ---- pages: a lane holds the ids of page `lane` of 32
  const int32_t* row = a.b.table + (int64_t)job.trow * a.b.table_stride + p0;
  auto fetch = [&](int i) { return i < pages ? row[i] : -1; };
  int ids = fetch(lane), ids_next = fetch(32 + lane);
  const unsigned char* const sc = static_cast<const unsigned char*>(lane < 16 ? c.k_scale : c.v_scale) + head * c.scale_head + (lane & 15) * c.scale_token;
  // the lane's 16 bytes of a page's codes (at D = 128 and those eight tokens on)
  const int64_t mine = head * c.stride_head + (D == 128 ? (lane >> 2) * c.stride_token + (lane & 3) * 16 : (lane >> 1) * c.stride_token + (lane & 1) * 16);
  const unsigned char* const kc = static_cast<const unsigned char*>(c.k) + mine;
  const unsigned char* const vc = static_cast<const unsigned char*>(c.v) + mine;
  const int64_t half = 8 * c.stride_token;
  auto load = [&](int i, int slot) {   // unit i of the segment, in order
    if ((i & 15) == 0 && i > 0) {
      ids = ids_next;
      ids_next = fetch(2 * i + 32 + lane);
    }
#pragma unroll
    for (int u = 0; u < 2; u++) {
      const int id = __shfl_sync(~0u, ids, (2 * i + u) & 31);
      const bool there = (unsigned)id < (unsigned)c.n_blocks;
      const int64_t at = there ? id : 0, block = at * c.stride_block;
      const uint32_t dst = ring + (slot * 2 + u) * L::PAGE_BYTES;
      if constexpr (D == 128) {
        const int r = lane >> 2, ch = lane & 3;
        copy_async<16>(dst + lane * 16, kc + block, there);
        copy_async<16>(dst + 512 + lane * 16, kc + block + half, there);
        copy_async<16>(dst + L::V + r * 64 + (ch ^ ((r >> 1) & 3)) * 16, vc + block, there);
        copy_async<16>(dst + L::V + 512 + r * 64 + (ch ^ ((r >> 1) & 3)) * 16, vc + block + half, there);
        copy_async<8>(dst + L::KS + lane * 8, sc + at * c.scale_block, there);
      } else {
        const int r = lane >> 1, ch = lane & 1;
        copy_async<16>(dst + lane * 16, kc + block, there);
        copy_async<16>(dst + L::V + (r ^ ((r >> 2) & 1)) * 32 + ch * 16, vc + block, there);
        copy_async<4>(dst + L::KS + lane * 4, sc + at * c.scale_block, there);
      }
    }
  };
#pragma unroll
  for (int s = 0; s < STAGES - 1; s++) {
    if (s < cnt) load(s, s);
    copies_commit();
  }
  // ---- rows: fragments of q, what each of the lane's rows sees, its scores' factor
  uint32_t q[N == 1 ? KS : 1][2];
  float sl[N][2];
  int lim[N][2], low = INT_MAX;
#pragma unroll
  for (int n = 0; n < N; n++) {
    const int r = n * 8 + g;   // as a column of q^T
    const bool live = r < job.nrows;
    int hl;
    const int in = token_of(p, job.row0 + min(r, job.nrows - 1), hl), tok = job.tok0 + in;
    const uint16_t* src = static_cast<const uint16_t*>(a.q) + (int64_t)tok * a.q_ts + (int64_t)(head * p.ratio + hl) * a.q_hs + t * (D / 4);
    uint32_t x[KS * 2];
#pragma unroll
    for (int i = 0; i < D / 32; i++) {
      const uint4 v = live ? *reinterpret_cast<const uint4*>(src + i * 8) : make_uint4(0, 0, 0, 0);
      x[4 * i] = v.x; x[4 * i + 1] = v.y; x[4 * i + 2] = v.z; x[4 * i + 3] = v.w;
    }
    float inverse = 1.0f;
    if (!HALF) {
      float most = 0.0f;
#pragma unroll
      for (int i = 0; i < KS * 2; i++) {
        const float2 f = unpack2<false>(x[i]);
        most = fmaxf(most, fmaxf(fabsf(f.x), fabsf(f.y)));
      }
      most = fmaxf(most, __shfl_xor_sync(~0u, most, 1));
      most = fmaxf(most, __shfl_xor_sync(~0u, most, 2));
      const float power = row_power(most, inverse);
#pragma unroll
      for (int i = 0; i < KS * 2; i++) {
        const float2 f = unpack2<false>(x[i]);
        x[i] = pack2<true>(__fmul_rn(f.x, power), __fmul_rn(f.y, power));
      }
    }
#pragma unroll
    for (int j = 0; j < KS; j++) {
      if constexpr (N == 1) { q[j][0] = x[2 * j]; q[j][1] = x[2 * j + 1]; }
      else asm volatile("st.shared.v2.u32 [%0], {%1, %2};" ::"r"(qs + (j * 32 + lane) * 16 + n * 8), "r"(x[2 * j]), "r"(x[2 * j + 1]) : "memory");
    }
    const float f = row_factor(a, inverse);
    const int see = min(live ? limit_of(a.b, job, tok, in) : kend, kend) - k0;   // keys of the segment
#pragma unroll
    for (int e = 0; e < 2; e++) {   // of rows 2 t + e
      sl[n][e] = __shfl_sync(~0u, f, (2 * t + e) * 4);
      lim[n][e] = __shfl_sync(~0u, see, (2 * t + e) * 4) - g;
    }
    low = min(low, __reduce_min_sync(~0u, see));
  }
  // (ref: what is subtracted from a row's scores, m but where the row has seen nothing yet)
  float o[N][MT][4], ref[N][2], l[N][2];
#pragma unroll
  for (int n = 0; n < N; n++) {
#pragma unroll
    for (int j = 0; j < MT; j++)
#pragma unroll
      for (int e = 0; e < 4; e++) o[n][j][e] = 0.0f;
    ref[n][0] = ref[n][1] = 0.0f;
    l[n][0] = l[n][1] = 0.0f;
  }
  // ---- the keys, 32 at a time
  int slot = 0, into = STAGES - 1;
#pragma unroll 1
  for (int i = 0; i < cnt; i++) {
    copies_wait<STAGES - 2>();
    __syncwarp();
    if (i + STAGES - 1 < cnt) load(i + STAGES - 1, into);
    copies_commit();
    const uint32_t pg0 = ring + slot * 2 * L::PAGE_BYTES;
    const int key = i * UNIT;
    if (++slot == STAGES) slot = 0;
    if (++into == STAGES) into = 0;
#pragma unroll 1
    for (int v = 0; v < 2; v += U) {   // (16 rows a page at a time, for the registers)
      // scores
      float s[U][N][4];
#pragma unroll
      for (int u = 0; u < U; u++) {
        const uint32_t pg = pg0 + (v + u) * L::PAGE_BYTES;
#pragma unroll
        for (int n = 0; n < N; n++) s[u][n][0] = s[u][n][1] = s[u][n][2] = s[u][n][3] = 0.0f;
        uint32_t w[2][D / 32], sp[2];   // codes and scales of keys g, g + 8
#pragma unroll
        for (int h = 0; h < 2; h++) {
          const uint32_t at = pg + h * (4 * D) + lane * (D / 8);
          if constexpr (D == 128) {
            asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(w[h][0]), "=r"(w[h][1]), "=r"(w[h][2]), "=r"(w[h][3]) : "r"(at));
            uint16_t two;
            asm volatile("ld.shared.u16 %0, [%1];" : "=h"(two) : "r"(pg + L::KS + h * 64 + lane * 2));
            sp[h] = scales_f16(two);
          } else {
            asm volatile("ld.shared.v2.u32 {%0, %1}, [%2];" : "=r"(w[h][0]), "=r"(w[h][1]) : "r"(at));
            uint16_t one;
            asm volatile("ld.shared.u8 %0, [%1];" : "=h"(one) : "r"(pg + L::KS + h * 32 + lane));
            sp[h] = scales_f16(one);
          }
        }
#pragma unroll
        for (int i4 = 0; i4 < D / 32; i4++) {
          uint32_t y[2][4];
#pragma unroll
          for (int h = 0; h < 2; h++) {
            codes_f16(w[h][i4], y[h]);
            const uint32_t f = both(sp[h], D == 128 && i4 >= 2);
#pragma unroll
            for (int z = 0; z < 4; z++) y[h][z] = mul_f16x2(y[h][z], f);
          }
#pragma unroll
          for (int z = 0; z < 2; z++) {
            const uint32_t fa[4] = {y[0][2 * z], y[1][2 * z], y[0][2 * z + 1], y[1][2 * z + 1]};
            if constexpr (N == 1) {
              mma(s[u][0], fa, q[2 * i4 + z][0], q[2 * i4 + z][1]);
            } else {
              uint32_t f[4];
              asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];"
                           : "=r"(f[0]), "=r"(f[1]), "=r"(f[2]), "=r"(f[3]) : "r"(qs + ((2 * i4 + z) * 32 + lane) * 16));
              mma(s[u][0], fa, f[0], f[1]);
              mma(s[u][N - 1], fa, f[2], f[3]);
            }
          }
        }
      }
      if (key + (v + U) * PAGE > low) {
#pragma unroll
        for (int u = 0; u < U; u++)
#pragma unroll
          for (int n = 0; n < N; n++)
#pragma unroll
            for (int e = 0; e < 4; e++)
              if (key + PAGE * (v + u) + 8 * (e >> 1) >= lim[n][e & 1]) s[u][n][e] = -INFINITY;
      }
      // weights; a row's reference moves where one is too large
      float w[U][N][4], most = 0.0f;
      auto weigh = [&] {
#pragma unroll
        for (int u = 0; u < U; u++)
#pragma unroll
          for (int n = 0; n < N; n++) {
#pragma unroll
            for (int e = 0; e < 4; e++) w[u][n][e] = ex2(fmaf(__fsub_rn(s[u][n][e], ref[n][e & 1]), sl[n][e & 1], BIAS));
            most = fmaxf(fmaxf(most, fmaxf(w[u][n][0], w[u][n][1])), fmaxf(w[u][n][2], w[u][n][3]));
          }
      };
      const bool first = i == 0 && v == 0;
      if (!first) weigh();
      if (first || __any_sync(~0u, most > HEAVY)) {
#pragma unroll
        for (int n = 0; n < N; n++)
#pragma unroll
          for (int e = 0; e < 2; e++) {
            float x = fmaxf(fmaxf(s[0][n][e], s[0][n][e + 2]), fmaxf(s[U - 1][n][e], s[U - 1][n][e + 2]));
            x = fmaxf(x, __shfl_xor_sync(~0u, x, 4));
            x = fmaxf(x, __shfl_xor_sync(~0u, x, 8));
            x = fmaxf(x, __shfl_xor_sync(~0u, x, 16));
            // (a row that sees nothing of the segment's first keys sees none of it)
            const float r2 = first ? (x == -INFINITY ? 0.0f : x) : fmaxf(ref[n][e], x);
            const float f = first ? 0.0f : ex2(__fmul_rn(__fsub_rn(ref[n][e], r2), sl[n][e]));
            ref[n][e] = r2;
            if (!first) {
              l[n][e] = __fmul_rn(l[n][e], f);
#pragma unroll
              for (int j = 0; j < MT; j++) {
                o[n][j][e] = __fmul_rn(o[n][j][e], f);
                o[n][j][e + 2] = __fmul_rn(o[n][j][e + 2], f);
              }
            }
          }
        weigh();
      }
      uint32_t pb[U][N][2];
#pragma unroll
      for (int u = 0; u < U; u++)
#pragma unroll
        for (int n = 0; n < N; n++) {
#pragma unroll
          for (int e = 0; e < 4; e++) l[n][e & 1] = __fadd_rn(l[n][e & 1], w[u][n][e]);
          pb[u][n][0] = turn(pack2<true>(w[u][n][0], w[u][n][1]));
          pb[u][n][1] = turn(pack2<true>(w[u][n][2], w[u][n][3]));
        }
      // the result
      const bool ends = k0 + key + (v + U) * PAGE > kend;
#pragma unroll
      for (int u = 0; u < U; u++) {
        const uint32_t pg = pg0 + (v + u) * L::PAGE_BYTES;
        uint32_t w[4][D / 64], sv[2];   // codes of keys 2t, 2t + 1, 2t + 8, 2t + 9; their scales in pairs
        uint32_t x[4];
#pragma unroll
        for (int h = 0; h < 4; h++) {
          const int r = 2 * t + (h & 1) + 8 * (h >> 1);
          if constexpr (D == 128) {
            asm volatile("ld.shared.v2.u32 {%0, %1}, [%2];"
                         : "=r"(w[h][0]), "=r"(w[h][1]) : "r"(pg + L::V + r * 64 + (((g >> 1) ^ t) * 16) + (g & 1) * 8));
            asm volatile("ld.shared.u8 %0, [%1];" : "=r"(x[h]) : "r"(pg + L::VS + r * 8 + g));
          } else {
            asm volatile("ld.shared.u32 %0, [%1];" : "=r"(w[h][0]) : "r"(pg + L::V + (r ^ ((r >> 2) & 1)) * 32 + g * 4));
            asm volatile("ld.shared.u8 %0, [%1];" : "=r"(x[h]) : "r"(pg + L::VS + r * 4 + (g >> 1)));
          }
        }
        if (ends) {   // (0 times what lies past the end may be NaN)
#pragma unroll
          for (int h = 0; h < 4; h++)
            if (k0 + key + PAGE * (v + u) + 2 * t + (h & 1) + 8 * (h >> 1) >= kend) x[h] = 0;
        }
        sv[0] = scales_f16(x[0] | x[1] << 8);
        sv[1] = scales_f16(x[2] | x[3] << 8);
#pragma unroll
        for (int i8 = 0; i8 < D / 64; i8++) {
          uint32_t y[4][4];   // elements 2 k (0, 2) and 2 k + 1 (1, 3), of the first pair of keys and of the second
#pragma unroll
          for (int h = 0; h < 2; h++) {
            const uint32_t wa = w[2 * h][i8], wb = w[2 * h + 1][i8];
            codes_f16((wa & 0x0F0F0F0Fu) | ((wb << 4) & 0xF0F0F0F0u), y[2 * h]);
            codes_f16(((wa >> 4) & 0x0F0F0F0Fu) | (wb & 0xF0F0F0F0u), y[2 * h + 1]);
#pragma unroll
            for (int k = 0; k < 4; k++) {
              y[2 * h][k] = mul_f16x2(y[2 * h][k], sv[h]);
              y[2 * h + 1][k] = mul_f16x2(y[2 * h + 1][k], sv[h]);
            }
          }
#pragma unroll
          for (int k = 0; k < 4; k++) {
            const uint32_t fa[4] = {y[0][k], y[1][k], y[2][k], y[3][k]};
#pragma unroll
            for (int n = 0; n < N; n++) mma(o[n][4 * i8 + k], fa, pb[u][n][0], pb[u][n][1]);
          }
        }
      }
    }
  }
  copies_wait<0>();
  __syncwarp();
  // ---- the rows' results; a lane has D / 8 elements of its rows
  const bool whole = t0 == 0 && t1 == job.nt, direct = whole && (job.flags & JOB_ALONE);
#pragma unroll
  for (int n = 0; n < N; n++)
#pragma unroll
    for (int e = 0; e < 2; e++) {
      float sum = l[n][e];
      sum = __fadd_rn(sum, __shfl_xor_sync(~0u, sum, 4));
      sum = __fadd_rn(sum, __shfl_xor_sync(~0u, sum, 8));
      sum = __fadd_rn(sum, __shfl_xor_sync(~0u, sum, 16));
      const int r = n * 8 + 2 * t + e;
      if (r >= job.nrows) continue;
      int hl;
      const int in = token_of(p, job.row0 + r, hl), hq = head * p.ratio + hl;
      const int64_t tok = job.tok0 + in, home = tok * a.n_heads + hq;
      if (direct) {
        const float inv = inverse_of(c.v_unit, sum);
        uint4* out = reinterpret_cast<uint4*>(static_cast<uint16_t*>(a.out) + tok * a.o_ts + hq * a.o_hs + g * (D / 8));
#pragma unroll
        for (int i = 0; i < D / 64; i++) {
          uint32_t w[4];
#pragma unroll
          for (int k = 0; k < 4; k++)
            w[k] = pack2<HALF>(__fmul_rn(o[n][4 * i + k][e], inv), __fmul_rn(o[n][4 * i + k][e + 2], inv));
          out[i] = make_uint4(w[0], w[1], w[2], w[3]);
        }
        if (a.lse && g == 0) a.lse[home] = log_sum(ref[n][e], sum, sl[n][e]);
      } else {
        const int64_t at = whole ? ((job.flags & JOB_PREFIX) ? 0 : (int64_t)a.b.n_tokens * a.n_heads) + home
                                 : part_row(p, 0, worker, head, t0 > 0) + r;
        float4* part = reinterpret_cast<float4*>((whole ? p.home : p.part[0]) + at * D + g * (D / 8));
#pragma unroll
        for (int i = 0; i < D / 32; i++)
          part[i] = make_float4(o[n][2 * i][e], o[n][2 * i][e + 2], o[n][2 * i + 1][e], o[n][2 * i + 1][e + 2]);
        if (g == 0) (whole ? p.home_sum : p.part_sum[0])[at] = make_float4(ref[n][e], sum, sl[n][e], 0.0f);
      }
    }
}

// As many warps as a chunk has heads are a worker and run the same keys, each for its head:
// with token-major blocks the heads of a token lie beside each other, and what one head reads of a DRAM
// access the others use at the same time (on their own, 128 long contexts took 508 us that way, against
// 243 us with head-major blocks; now 240 and 237).  Workers that are neighbours in the numbering are on different SMs.
template <int D, bool HALF>
__global__ void __launch_bounds__(WARPS * 32, 1) k_kv4_rows(const __grid_constant__ KvAttend4Args a, const __grid_constant__ Plan p) {
  using L = RowsLay<D>;
  extern __shared__ __align__(16) unsigned char sm[];
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  // Beside the tiles' kernel: its CTAs are all past their wait for the plan and for what came before that; this
  // kernel's take the SMs as they leave them, and it ends when that has ended.
  if (p.beside) {
    asm volatile("griddepcontrol.launch_dependents;");
    __threadfence();   // (nothing that this SM had read before the plan)
  } else {
    behind_stream();
  }
  const Head* head = p.head;
  const Job* jobs = p.jobs[0];
  if (p.tiny) {
    Head* const h = reinterpret_cast<Head*>(sm + L::PLAN);
    Job* const j = reinterpret_cast<Job*>(h + 1);
    if (warp == 0) tiny_plan(a.b, p, h, j, lane);
    __syncthreads();
    head = h;
    jobs = j;
  }
  const Head hd = *head;
  const int team = warp / p.chunk, place = warp - team * p.chunk;
  if (team < WARPS / p.chunk && blockIdx.x < hd.ctas) {
    const int w = team * hd.ctas + blockIdx.x;
    const uint32_t ring = smem_u32(sm) + warp * L::WARP_BYTES;
    Turn& turn = *reinterpret_cast<Turn*>(sm + L::WALKS + warp * sizeof(Turn));
    const Walk start(jobs, hd, 0, p.chunks, w, lane);
    if (lane == 0) turn.walk = start;
    for (;;) {
      if (lane == 0) turn.more = turn.walk.next(turn.item, turn.t0, turn.t1);
      __syncwarp();
      if (!turn.more) break;
      const int kh = turn.item * p.chunk + place, t0 = turn.t0, t1 = turn.t1;
      if (kh < a.c.n_kv_heads) {
        if (t0 == 0) tell(a, p, turn.walk, head->per[0], w, kh, t1, lane, 32);
        if (turn.walk.job.nrows > 8) rows_segment<D, HALF, 2>(a, p, turn.walk.job, kh, t0, t1, w, ring);
        else rows_segment<D, HALF, 1>(a, p, turn.walk.job, kh, t0, t1, w, ring);
      }
      __syncwarp();
    }
  }
  // rows of no request
  const int q_begin = head->q_begin, q_end = head->q_end;
  const int64_t per = (int64_t)a.n_heads * (D / 8), pads = (int64_t)(q_begin + a.b.n_tokens - q_end) * per;
  for (int64_t x = (int64_t)blockIdx.x * (WARPS * 32) + tid; x < pads; x += (int64_t)gridDim.x * (WARPS * 32)) {
    const int64_t y = x % per, h = y / (D / 8), e = y % (D / 8);
    int64_t r = x / per;
    if (r >= q_begin) r += q_end - q_begin;
    reinterpret_cast<uint4*>(static_cast<uint16_t*>(a.out) + r * a.o_ts + h * a.o_hs)[e] = make_uint4(0, 0, 0, 0);
    if (a.lse && e == 0) a.lse[r * a.n_heads + h] = -INFINITY;
  }
  if (p.beside) asm volatile("griddepcontrol.wait;" ::: "memory");
}

// ------------------------------------------------------------------ joining

constexpr int JOINS = 3;   // CTAs of an SM

// A row's parts, in the order of the keys: of its prefix item, of its own.
struct Parts {
  int count[2];         // of either item
  int kind[2], first[2], row[2];   // of one that is cut: its kind, the worker with its first unit, the row in its job
  bool whole[2];
  int head;             // kv head
  bool any;             // it has parts to join (else it is in out already)

  __device__ Parts(const KvAttend4Args& a, const Plan& p, int64_t home) {
    const int64_t tok = quotient(home, a.n_heads);
    const bool groups = a.b.n_groups > 0;
    const int what = groups ? __ldcg(p.tok + tok) : TOK_ALONE;
    const int places[2] = {groups ? __ldcg(p.where[0] + home) : -1, __ldcg(p.where[1] + home)};   // (on their way at once)
    const bool parts = what == TOK_ALONE ? places[1] >= 0 : what > TOK_ALONE && what <= TOK_PREFIX;
    int hl;
    head = token_of(p, (int)(home - tok * a.n_heads), hl);
#pragma unroll
    for (int s = 0; s < 2; s++) {
      const bool has = parts && (s ? what != TOK_PREFIX : what != TOK_ALONE);
      const int w = has ? places[s] : -1;
      count[s] = has ? 1 : 0;
      whole[s] = w < 0;
      kind[s] = w >= KIND ? 1 : 0;
      first[s] = row[s] = 0;
      if (w >= 0) {
        const int at = w & (KIND - 1), workers = kind[s] ? p.workers[1] : p.workers[0];
        const int4 v = at < workers ? __ldcg(reinterpret_cast<const int4*>((kind[s] ? p.cut[1] : p.cut[0]) + at)) : make_int4(0, -1, 0, 0);
        const int64_t r = (tok - v.w) * p.ratio + hl - v.z;
        // (starts that decrease leave rows of which nothing was written: they may find anything, also a CTA's part in a
        // step that has no room for any)
        const bool sound = (!kind[s] || p.cap[1] > 0) && v.x >= 0 && v.x <= v.y && v.y < workers && r >= 0 && r < rows_of(kind[s]);
        count[s] = sound ? v.y - v.x + 1 : 0;
        first[s] = v.x;
        row[s] = sound ? (int)r : 0;
      }
    }
    any = parts;
  }
  __device__ int n() const { return count[0] + count[1]; }
  // Lane src's, for the whole warp.
  __device__ void take(int src) {
    head = __shfl_sync(~0u, head, src);
#pragma unroll
    for (int s = 0; s < 2; s++) {
      count[s] = __shfl_sync(~0u, count[s], src);
      kind[s] = __shfl_sync(~0u, kind[s], src);
      first[s] = __shfl_sync(~0u, first[s], src);
      row[s] = __shfl_sync(~0u, row[s], src);
      whole[s] = __shfl_sync(~0u, (int)whole[s], src);
    }
  }
  // Part k's sums, and its row.
  __device__ float4 at(const KvAttend4Args& a, const Plan& p, int D, int64_t home, int k, const float4*& r) const {
    const bool own = k >= count[0];
    const int i = own ? k - count[0] : k, kd = own ? kind[1] : kind[0];
    const bool w = own ? whole[1] : whole[0];
    const int64_t to = w ? (own ? (int64_t)a.b.n_tokens * a.n_heads : 0) + home
                         : part_row(p, kd, (own ? first[1] : first[0]) + i, head, i > 0) + (own ? row[1] : row[0]);
    r = reinterpret_cast<const float4*>((w ? p.home : kd ? p.part[1] : p.part[0]) + to * D);
    return __ldcg((w ? p.home_sum : kd ? p.part_sum[1] : p.part_sum[0]) + to);
  }
};

// What is joined so far: o relative to the reference m.  (A part without weights has no reference.)
template <int E>
struct Joined {
  float m, l, sl, o[E];
  __device__ Joined() {
    m = -INFINITY;
    l = sl = 0.0f;
#pragma unroll
    for (int e = 0; e < E; e++) o[e] = 0.0f;
  }
  __device__ __forceinline__ void add(const float4& s, const float* v) {
    if (s.y == 0.0f) return;
    sl = s.z;   // (the same in every part)
    const float m2 = fmaxf(m, s.x);
    const float f = m == -INFINITY ? 0.0f : ex2(__fmul_rn(__fsub_rn(m, m2), sl)), w = ex2(__fmul_rn(__fsub_rn(s.x, m2), sl));
    m = m2;
    l = fmaf(s.y, w, __fmul_rn(l, f));
#pragma unroll
    for (int e = 0; e < E; e++) o[e] = fmaf(v[e], w, __fmul_rn(o[e], f));
  }
};

template <bool HALF>
__device__ __forceinline__ void store4(const KvAttend4Args& a, int64_t tok, int hq, int chunk, const float* o, float inv) {
  *reinterpret_cast<uint2*>(static_cast<uint16_t*>(a.out) + tok * a.o_ts + hq * a.o_hs + chunk * 4) =
      make_uint2(pack2<HALF>(__fmul_rn(o[0], inv), __fmul_rn(o[1], inv)), pack2<HALF>(__fmul_rn(o[2], inv), __fmul_rn(o[3], inv)));
}
// By an eight of lanes (j its lane): every `step`th of a row's parts from part `from` on, joined to x.  Eight parts at a
// time: a lane a part's sums, the eight their weights; then the rows.
template <int D>
__device__ __forceinline__ void join_parts(const KvAttend4Args& a, const Plan& p, const Parts& q, int64_t home, int from, int step, int j,
                                           Joined<D / 8>& x) {
  constexpr int C = D / 32;   // chunks of four elements of a lane: j, j + 8, ...
  const unsigned us = 0xFFu << (threadIdx.x & 24);
  const int n = q.n();
  for (int base = from; base < n; base += 8 * step) {
    const int k = base + j * step, here = min(8, (n - base + step - 1) / step);
    const float4* mine = nullptr;
    float4 t = make_float4(-INFINITY, 0.0f, 0.0f, 0.0f);
    if (k < n) t = q.at(a, p, D, home, k, mine);
    const bool some = t.y != 0.0f;   // (a part without weights has no reference)
    float big = some ? t.x : -INFINITY, unit = some ? t.z : 0.0f;
#pragma unroll
    for (int z = 4; z; z >>= 1) {
      big = fmaxf(big, __shfl_xor_sync(us, big, z));
      unit = fmaxf(unit, __shfl_xor_sync(us, unit, z));   // (the same in every part)
    }
    const float m2 = fmaxf(x.m, big);
    x.sl = fmaxf(x.sl, unit);
    const float f = x.m == -INFINITY ? 0.0f : ex2(__fmul_rn(__fsub_rn(x.m, m2), x.sl)), w = some ? ex2(__fmul_rn(__fsub_rn(t.x, m2), x.sl)) : 0.0f;
    float sum = some ? __fmul_rn(t.y, w) : 0.0f;
#pragma unroll
    for (int z = 4; z; z >>= 1) sum = __fadd_rn(sum, __shfl_xor_sync(us, sum, z));
    x.m = m2;
    x.l = fmaf(x.l, f, sum);
#pragma unroll
    for (int e = 0; e < 4 * C; e++) x.o[e] = __fmul_rn(x.o[e], f);
    for (int i = 0; i < here; i++) {
      const float4* r = reinterpret_cast<const float4*>(__shfl_sync(us, reinterpret_cast<unsigned long long>(mine), i, 8));
      const float y = __shfl_sync(us, w, i, 8);
#pragma unroll
      for (int c = 0; c < C; c++) {
        const float4 v = __ldcg(r + j + 8 * c);
        if (y != 0.0f) {
          x.o[4 * c] = fmaf(y, v.x, x.o[4 * c]);
          x.o[4 * c + 1] = fmaf(y, v.y, x.o[4 * c + 1]);
          x.o[4 * c + 2] = fmaf(y, v.z, x.o[4 * c + 2]);
          x.o[4 * c + 3] = fmaf(y, v.w, x.o[4 * c + 3]);
        }
      }
    }
  }
}

// Rows that have parts: of the items that a share's end cuts and, with groups, of the rows
// that have a prefix job.  Where a CTA has one row at most (each may have hundreds of parts), its 32 eights of lanes take
// every 32nd part of it.  Else a warp looks for 32 rows where their parts are and joins one after another; neighbouring
// rows, which have like numbers of parts, are far apart in the grid.  (An eight of lanes a row, neighbours beside each
// other: 16 us of a step's 44 with 900 rows of up to 40 parts.)  By CTAs and by warps, us a call: one token of 64 heads on 2
// over 16 160 keys 24 and 60; three rows an SM, 57 tokens of 8 heads on one over 8 000, 32 and 38; four, 76 such, 45 and 44, or
// over 600, 24 and 22; sixteen, 76 tokens over 600, 38 and 25, a prompt's 304 tokens of 8 heads behind 3 000, 41 and 29.  The
// order in which parts are joined is fixed, so the result does not depend on when they came.  (ONE: all rows of the
// arrays are so few, and less code has a shorter way to the SM.)
// Bound: latency, of reads that depend on one another (head, place, cut, sums, rows): 3 to 6 us.  Three CTAs an SM and four
// rows on their way (four CTAs: 0 to 2 us more, six to eight: up to 8 us more; eight rows: up to 4 us more).
template <int D, bool HALF>
__device__ __forceinline__ void join_by_cta(const KvAttend4Args& a, const Plan& p, int64_t from, int64_t rows, float (*sm)[D + 4]) {
  constexpr int C = D / 32;
  const int j = threadIdx.x & 7, eight = threadIdx.x >> 3;
  for (int64_t home = from + blockIdx.x; home < rows; home += gridDim.x) {
    const Parts q(a, p, home);
    if (!q.any) continue;
    const int64_t tok = quotient(home, a.n_heads);
    const int hq = (int)(home - tok * a.n_heads);
    Joined<4 * C> x;
    join_parts<D>(a, p, q, home, eight, 32, j, x);
#pragma unroll
    for (int c = 0; c < C; c++)
#pragma unroll
      for (int e = 0; e < 4; e++) sm[eight][(j + 8 * c) * 4 + e] = x.o[4 * c + e];
    if (j == 0) { sm[eight][D] = x.m; sm[eight][D + 1] = x.l; sm[eight][D + 2] = x.sl; }
    __syncthreads();
    if (threadIdx.x < D / 4) {
      const int used = min(q.n(), 32);
      Joined<4> y;
      for (int k = 0; k < used; k++) y.add(make_float4(sm[k][D], sm[k][D + 1], sm[k][D + 2], 0.0f), &sm[k][threadIdx.x * 4]);
      store4<HALF>(a, tok, hq, threadIdx.x, y.o, inverse_of(a.c.v_unit, y.l));
      if (a.lse && threadIdx.x == 0) a.lse[home] = log_sum(y.m, y.l, y.sl);
    }
    __syncthreads();
  }
}

// A lane has D / 32 elements of the row; a lane a part's sums, up to 32 parts at once, the rows four at a time.
template <int D, bool HALF>
__device__ __forceinline__ void join_by_warp(const KvAttend4Args& a, const Plan& p, int64_t from, int64_t rows) {
  constexpr int E = D / 32, Z = 4;
  using Vec = std::conditional_t<E == 4, float4, float2>;
  const int lane = threadIdx.x & 31;
  const int64_t warps = (int64_t)gridDim.x * 8, me = (int64_t)(threadIdx.x >> 5) * gridDim.x + blockIdx.x;
  for (int64_t base = from + me; base < rows; base += 32 * warps) {
    const int64_t mine = base + lane * warps;
    const Parts own(a, p, min(mine, rows - 1));
    for (unsigned todo = __ballot_sync(~0u, own.any && mine < rows); todo; todo &= todo - 1) {
      const int src = __ffs(todo) - 1;
      const int64_t home = base + src * warps;
      Parts q = own;
      q.take(src);
      const int n = q.n();
      float m = -INFINITY, l = 0.0f, sl = 0.0f, o[E];
#pragma unroll
      for (int e = 0; e < E; e++) o[e] = 0.0f;
#pragma unroll 1
      for (int k0 = 0; k0 < n; k0 += 32) {
        const float4* at = nullptr;
        float4 t = make_float4(-INFINITY, 0.0f, 0.0f, 0.0f);
        if (k0 + lane < n) t = q.at(a, p, D, home, k0 + lane, at);
        const bool some = t.y != 0.0f;   // (a part without weights has no reference)
        float big = some ? t.x : -INFINITY;
        sl = some ? t.z : sl;            // (the same in every part)
#pragma unroll
        for (int z = 16; z; z >>= 1) {
          big = fmaxf(big, __shfl_xor_sync(~0u, big, z));
          sl = fmaxf(sl, __shfl_xor_sync(~0u, sl, z));
        }
        const float m2 = fmaxf(m, big);
        const float f = m == -INFINITY ? 0.0f : ex2(__fmul_rn(__fsub_rn(m, m2), sl)), w = some ? ex2(__fmul_rn(__fsub_rn(t.x, m2), sl)) : 0.0f;
        float sum = some ? __fmul_rn(t.y, w) : 0.0f;
#pragma unroll
        for (int z = 16; z; z >>= 1) sum = __fadd_rn(sum, __shfl_xor_sync(~0u, sum, z));
        m = m2;
        l = fmaf(l, f, sum);
#pragma unroll
        for (int e = 0; e < E; e++) o[e] = __fmul_rn(o[e], f);
        const int here = min(32, n - k0);
#pragma unroll 1
        for (int i = 0; i < here; i += Z) {
          Vec v[Z];
#pragma unroll
          for (int z = 0; z < Z; z++) {
            const Vec* r = reinterpret_cast<const Vec*>(__shfl_sync(~0u, reinterpret_cast<unsigned long long>(at), min(i + z, here - 1)));
            if (i + z < here) v[z] = __ldcg(r + lane);
          }
#pragma unroll
          for (int z = 0; z < Z; z++) {
            const float y = __shfl_sync(~0u, w, min(i + z, here - 1));
            if (i + z < here && y != 0.0f) {
              o[0] = fmaf(y, v[z].x, o[0]);
              o[1] = fmaf(y, v[z].y, o[1]);
              if constexpr (E == 4) {
                o[2] = fmaf(y, v[z].z, o[2]);
                o[3] = fmaf(y, v[z].w, o[3]);
              }
            }
          }
        }
      }
      const int64_t tok = quotient(home, a.n_heads);
      const int hq = (int)(home - tok * a.n_heads);
      const float inv = inverse_of(a.c.v_unit, l);
      uint16_t* const out = static_cast<uint16_t*>(a.out) + tok * a.o_ts + hq * a.o_hs + lane * E;
      const uint32_t first = pack2<HALF>(__fmul_rn(o[0], inv), __fmul_rn(o[1], inv));
      if constexpr (E == 4) *reinterpret_cast<uint2*>(out) = make_uint2(first, pack2<HALF>(__fmul_rn(o[2], inv), __fmul_rn(o[3], inv)));
      else *reinterpret_cast<uint32_t*>(out) = first;
      if (a.lse && lane == 0) a.lse[home] = log_sum(m, l, sl);
    }
  }
}

template <int D, bool HALF, bool ONE>
__global__ void __launch_bounds__(256, JOINS) k_kv4_join(const __grid_constant__ KvAttend4Args a, const __grid_constant__ Plan p) {
  __shared__ float sm[32][D + 4];
  behind_stream();
  const int q_end = p.head->room ? p.head->q_end : 0;
  const int64_t from = (int64_t)p.head->q_begin * a.n_heads, rows = (int64_t)q_end * a.n_heads;   // the first, the end
  if (ONE || rows - from <= (int64_t)gridDim.x) join_by_cta<D, HALF>(a, p, from, rows, sm);
  else join_by_warp<D, HALF>(a, p, from, rows);
}

// ------------------------------------------------------------------ host

size_t up(size_t x) { return (x + 255) & ~(size_t)255; }

// The workspace; with ws NULL only its size.
size_t carve(const KvAttend4Args& a, int sms, unsigned char* ws, Plan& p) {
  const size_t n = a.b.n_req, G = a.b.n_groups, D = a.c.head_dim, T = a.b.n_tokens, rows = T * a.n_heads;
  p.ratio = a.n_heads / a.c.n_kv_heads;
  p.ratio_inv = p.ratio == 1 ? UINT32_MAX : (uint32_t)((1ull << 32) / p.ratio);
  p.few_max = FEW_MAX;
  p.heads = a.c.n_kv_heads;
  // the most heads a chunk that leave few of the CTA's warps without one
  const int heads = a.c.n_kv_heads;
  p.chunk = 1;
  for (int h = std::min(heads, WARPS); h > 1; h--)
    if (32 * (WARPS / h) * heads >= 29 * WARPS * ((heads + h - 1) / h)) {   // (of all warp-times, nine tenths)
      p.chunk = h;
      break;
    }
  p.chunks = (heads + p.chunk - 1) / p.chunk;
  p.workers[0] = sms * (WARPS / p.chunk);
  p.workers[1] = sms;
  // each request and each group at most one job more than its share of the rows
  const size_t flat = T * p.ratio * (G ? 2 : 1);
  p.cap[0] = (int32_t)(std::min(flat / FEW + n + G, (n + G) * ((FEW_MAX + FEW - 1) / FEW)) + 1);
  p.cap[1] = T * p.ratio > FEW_MAX ? (int32_t)(flat / MANY + std::min(n + G, flat / FEW_MAX) + 1) : 0;
  size_t o = 0;
  auto take = [&](auto*& ptr, size_t count) {
    if (ws) ptr = reinterpret_cast<std::remove_reference_t<decltype(ptr)>>(ws + o);
    o = up(o + count * sizeof(*ptr));
  };
  take(p.head, 1);
  take(p.jobs[0], p.cap[0] + 1);
  take(p.jobs[1], p.cap[1] + 1);
  take(p.tok, G ? T : 0);
  take(p.group, G);
  take(p.where[0], G ? rows : 0);
  take(p.where[1], rows);
  take(p.cut[0], p.workers[0]);
  take(p.cut[1], p.workers[1]);
  const size_t w0 = (size_t)p.workers[0] * p.chunk * 2 * FEW;
  const size_t w1 = p.cap[1] ? (size_t)p.workers[1] * 2 * MANY : 0;
  take(p.part[0], w0 * D);
  take(p.part_sum[0], w0);
  take(p.part[1], w1 * D);
  take(p.part_sum[1], w1);
  take(p.home, G ? 2 * rows * D : 0);
  take(p.home_sum, G ? 2 * rows : 0);
  return o;
}

template <int D, bool HALF>
cudaError_t run(const KvAttend4Args& a, const Plan& p, int sms, cudaStream_t st) {
  cudaError_t e = p.cap[1] ? launch_tiles(a, p, sms, st) : cudaSuccess;
  if (e != cudaSuccess) return e;
  auto k = k_kv4_rows<D, HALF>;
  e = cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, RowsLay<D>::SMEM);
  if (e != cudaSuccess) return e;
  e = launch_behind(k, sms, WARPS * 32, RowsLay<D>::SMEM, st, a, p);
  if (e != cudaSuccess) return e;
  const int64_t rows = (int64_t)a.b.n_tokens * a.n_heads;
  const bool one = rows <= (int64_t)sms * JOINS;
  return launch_behind(one ? k_kv4_join<D, HALF, true> : k_kv4_join<D, HALF, false>, (unsigned)(one ? rows : sms * JOINS), 256, 0, st, a, p);
}

}  // namespace

size_t kv_attend4_bytes(const KvAttend4Args& a, int sms) {
  Plan p = {};
  return carve(a, sms, nullptr, p);
}

cudaError_t launch_kv_attend4(const KvAttend4Args& a, void* ws, int32_t* err, int sms, cudaStream_t st) {
  Plan p = {};
  carve(a, sms, static_cast<unsigned char*>(ws), p);
  p.err = err;
  p.beside = p.cap[1] > 0;
  // a step so small that no request can have many rows: no plan ahead (a launch and 3 us less)
  p.tiny = p.cap[1] == 0 && a.b.n_req <= TINY;
  if (!p.tiny) {
    const cudaError_t e = launch_behind(k_kv4_plan, 1, NT_PLAN, 0, st, a.b, p, (int)a.c.n_kv_heads, a.c.head_dim == 128);
    if (e != cudaSuccess) return e;
  }
  if (a.c.head_dim == 128) return a.half ? run<128, true>(a, p, sms, st) : run<128, false>(a, p, sms, st);
  return a.half ? run<64, true>(a, p, sms, st) : run<64, false>(a, p, sms, st);
}

}  // namespace rs
