// Causal attention over a paged KV cache (kv_attend): a plan cuts the step into
// jobs, k_kv_attend runs them on the tensor cores, k_kv_join joins parts.
//
// Mathematics.  A row (token, head) needs o = sum_j p_j v_j / sum_j p_j over
// the keys j below its limit, p_j = exp(scale s_j), s = q K^T.  Over any part
// of the keys the triple (m, l, o), m a reference for the scores, l = sum
// exp(s - m), o = sum exp(s - m) v, is enough: parts join with weights
// exp(m_part - m).  So a job walks its keys once, 128 at a time, and the keys of
// a row may be cut anywhere: between a prefix shared by a group (a job whose rows
// are all the group's tokens) and the requests' own keys, and between CTAs.
//
// A job is up to 2 * 128 rows x one kv head x a range of keys.  Rows are
// tokens x the heads of the kv head (so the K and V of a head are read once for
// all of them).  The jobs' tiles are numbered through, and CTA c takes an equal
// share of the numbers (one CTA an SM): whole jobs write out directly, jobs
// cut by a share's end leave parts in 32 bits.
//
// What bounds it (one GB300): single tokens over long contexts, HBM (256 requests
// in 8 groups, 256 to 8192 own tokens each, 8 kv heads of 128: 2.6 GB in 418 us, 6.3
// TB/s); prompts and prefixes that many rows share, the tensor cores (4096 tokens
// behind 12 288, 32 heads: 645 us, 1.49 PFLOP/s; 128 keys for 256 rows take 2048
// clocks of the products and, with all that is between tiles and jobs, 2955 of the
// kernel's); short steps, the chain plan - loads - product - softmax - product -
// stores - join (one token over 701 keys: 14 us).
#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <algorithm>
#include <climits>
#include <type_traits>

#include "rs_internal.h"

namespace rs {

namespace {

constexpr int TK = 128;        // keys of a tile
// Costs, in quarters of a microsecond or so: a tile of a job of at most 128 rows,
// one of a larger job, and a job's own (its rows' loads and stores).  They share the
// work out and are fitted to that, not measured one by one.  When they were chosen
// 64 requests on a prefix of 32 768, 8 groups of 256 in all, 6 prompts of 100 to
// 2047 on a prefix took 83, 427, 259 us; with 4, 6, 3, 10: 86, 427, 273 us; with
// equal tiles and OV 2 for all, on an earlier kernel: 142, 524, 299 us (now 84, 418,
// 254).
constexpr int W_NARROW = 4, W_WIDE = 5, OV_NARROW = 3, OV_WIDE = 10;
constexpr int NT_PLAN = 1024;
constexpr int NT_ATT = 384;
constexpr int PLAN_GROUPS = 1024;   // groups whose sums are kept in shared memory
constexpr int PLAN_JOBS = 1024;     // jobs that are

constexpr int JOB_ALONE = 1;   // no other job has its rows
constexpr int JOB_EVEN = 2;    // every row sees all the job's keys
constexpr int JOB_PREFIX = 4;  // a group's prefix
constexpr int JOB_WIDE = 8;    // more than 128 rows

}  // namespace

// One job, for each kv head alike.
struct __align__(16) KvJob {
  int32_t tok0, ntok;   // rows of tokens
  int32_t row;          // table row
  int32_t key0, kend;   // keys (key0 a multiple of 16)
  int32_t nt;           // tiles of them
  int32_t lim0;         // keys that the first token sees; the next see one more each
  int32_t flags;
  int64_t cost;         // of the jobs before, for one kv head
  int64_t rows;         // of a prefix job: tokens of the prefix jobs before
};

// A job and head that a share's end cuts, at the share's end that cuts it first.
struct __align__(16) KvCut {
  int32_t tok0, ntok;
  int32_t head;
  int32_t c0;           // the CTA in which it begins
  int32_t first, last;  // CTAs that have tiles of it
  int32_t reserved0, reserved1;
};

struct KvHead {
  int64_t total, per;   // cost of all jobs and heads, of one CTA
  int32_t jobs, prefix_jobs;
  int32_t shared;       // tokens of the prefix jobs
  int32_t cuts, cut_rows;   // cut jobs, and the most rows of one
  int32_t reserved0;
};

struct __align__(16) KvStart {
  int32_t job, head, off, reserved0;   // where a CTA's share begins
  int64_t rem, reserved1;              // its cost
  KvJob j;                             // that job
};

struct KvPlan {
  KvHead* head;
  KvJob* jobs;          // [cap + 1]
  int4* shared;         // [n_tokens] of the shared groups' tokens, in order: row, prefix job, own job
  int32_t* gjob;        // [n_groups] first prefix job, -1: not shared (more than PLAN_GROUPS groups)
  unsigned long long* gsum;   // [4 n_groups] (more than PLAN_GROUPS groups)
  KvStart* start;       // [ctas]
  KvCut* cut;           // [ctas] the cut jobs, in any order
  float* part;          // [ctas][2][256][D] cut jobs' rows: of the first cut job (0), of the last (1)
  float2* part_sum;     // [ctas][2][256] of each its reference (a power of two's exponent) and its weights' sum
  float* home;          // [2][rows][D] rows with a prefix job and an own one, each whole
  float2* home_sum;     // [2][rows]
  int32_t* err;         // host memory: set when a wait ran out
  int32_t cap;          // jobs at most
  int32_t ctas;
  int32_t tpt;          // tokens of 128 rows
  int32_t ratio;        // heads of a kv head
  int32_t planned;      // the plan is there before the attention kernel begins
  int32_t whole;        // no job is cut
};

namespace {

// ------------------------------------------------------------------ the plan

__device__ __forceinline__ int clampi(int64_t x, int lo, int hi) {
  return (int)(x < lo ? lo : x > hi ? hi : x);
}

template <class Int>
struct JobSum {
  Int count, cost, rows;   // jobs, their cost, tokens of prefix jobs
};

// Exclusive sum of x over the CTA's first `width` threads (the others have 0), and
// its total; sm: one entry a warp, not the one of the sum before.
template <class Int>
__device__ JobSum<Int> block_scan(JobSum<Int> x, JobSum<Int>* sm, int width, JobSum<Int>& total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  auto scan = [&](JobSum<Int> s) {
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const Int x = __shfl_up_sync(~0u, s.count, o), y = __shfl_up_sync(~0u, s.cost, o), z = __shfl_up_sync(~0u, s.rows, o);
      if (lane >= o) { s.count += x; s.cost += y; s.rows += z; }
    }
    return s;
  };
  JobSum<Int> s{0, 0, 0};
  if (warp * 32 < width) {
    s = scan(x);
    if (lane == 31) sm[warp] = s;
  }
  __syncthreads();
  if (width <= 32) {
    total = sm[0];
    return JobSum<Int>{s.count - x.count, s.cost - x.cost, s.rows - x.rows};
  }
  const JobSum<Int> w = lane * 32 < width ? sm[lane] : JobSum<Int>{0, 0, 0}, ws = scan(w);
  total.count = __shfl_sync(~0u, ws.count, 31);
  total.cost = __shfl_sync(~0u, ws.cost, 31);
  total.rows = __shfl_sync(~0u, ws.rows, 31);
  return JobSum<Int>{__shfl_sync(~0u, ws.count - w.count, warp) + s.count - x.count,
                     __shfl_sync(~0u, ws.cost - w.cost, warp) + s.cost - x.cost,
                     __shfl_sync(~0u, ws.rows - w.rows, warp) + s.rows - x.rows};
}

struct ReqLens {
  int q0, q, kv;   // first row, rows, context up to the last of them (below 0: none of them sees anything)
  int g;           // group, or -1
};

__device__ __forceinline__ int tiles(int keys) { return keys > 0 ? (keys + TK - 1) / TK : 0; }

__device__ __forceinline__ int tile_cost(int flags) { return (flags & JOB_WIDE) ? W_WIDE : W_NARROW; }
__device__ __forceinline__ int own_cost(int flags) { return (flags & JOB_WIDE) ? OV_WIDE : OV_NARROW; }
// (a job without keys whose rows nobody else has writes their zeros)
__device__ __forceinline__ int job_cost(int nt, int flags) {
  return nt > 0 ? nt * tile_cost(flags) + own_cost(flags) : (flags & JOB_ALONE) ? OV_NARROW : 0;
}
// The first tile that starts at cost `off` of a job or after it.
__device__ __forceinline__ int tile_at(int off, int flags) {
  off -= own_cost(flags);
  return off <= 0 ? 0 : (flags & JOB_WIDE) ? (off + W_WIDE - 1) / W_WIDE : (off + W_NARROW - 1) / W_NARROW;
}

// The tiles that CTA c has of a job and head of `cost` from u0 on.
__device__ __forceinline__ bool segment(int64_t u0, int cost, int flags, int nt, int64_t per, int64_t c, int& t0, int& t1) {
  const int64_t lo = max(c * per, u0) - u0, hi = min((c + 1) * per, u0 + cost) - u0;
  if (lo >= hi) return false;
  t0 = min(tile_at((int)lo, flags), nt);
  t1 = min(tile_at((int)hi, flags), nt);
  return t1 > t0;
}

__device__ __forceinline__ int64_t quotient(int64_t a, int64_t b) {
  return ((a | b) >> 32) == 0 ? (int64_t)((uint32_t)a / (uint32_t)b) : a / b;
}

// A plan's working memory.
struct PlanSmem {
  KvJob job[PLAN_JOBS];
  uint64_t sum[4 * PLAN_GROUPS];
  int32_t start[PLAN_GROUPS + 1], prefix[PLAN_GROUPS], gjob[PLAN_GROUPS];
  JobSum<int64_t> scan[2][32];
  int32_t cuts, cut_rows;
};

// By a whole CTA: whether each group's prefix pays as one job for all its rows,
// the jobs, their costs' sums, every CTA's start and what its end cuts.  Latency is
// all that counts here (a few dependent reads and block sums): lengths are read
// once at up to a request a thread, group sums and jobs live in shared memory at
// ordinary sizes.  Starts that decrease can ask for more jobs than there is room
// for: then there is no work at all.
//   all_ctas: one CTA for everybody, starts into p.start.
//   else (at most PLAN_JOBS jobs and PLAN_GROUPS groups): every CTA for itself, its
//     start into *own_start and the jobs of its share into p.jobs; what the joining
//     needs is written by the last one.  3 us for one request, 5 us for 64 in groups; as a
//     kernel of its own before the attention kernel's start it cost 4 us more.
// Int: wide enough for all jobs' cost (64-bit sums made the plan 1 us longer).
template <class Int>
__device__ __forceinline__ void make_plan(const rs_kv_batch& b, const KvPlan& p, int n_kv_heads, PlanSmem& ps, bool all_ctas,
                                          KvStart* own_start) {
  using Sum = JobSum<Int>;
  Sum(*scan)[32] = reinterpret_cast<Sum(*)[32]>(ps.scan);
  const bool writer = all_ctas || blockIdx.x == gridDim.x - 1;   // (of a short step the last CTA has no share)
  KvJob* s_job = ps.job;
  using Acc = std::conditional_t<sizeof(Int) == 4, unsigned, unsigned long long>;
  Acc* s_sum = reinterpret_cast<Acc*>(ps.sum);
  int32_t *s_start = ps.start, *s_prefix = ps.prefix, *s_gjob = ps.gjob;
  const int tid = threadIdx.x, lane = tid & 31, nth = blockDim.x, n = b.n_req, G = b.n_groups;
  const int w2 = 2 * p.tpt;
  const bool few = G <= PLAN_GROUPS;
  Acc* sum = few ? s_sum : reinterpret_cast<Acc*>(p.gsum);
  const int32_t* gstart = few ? s_start : b.group_start;
  const int32_t* glen = few ? s_prefix : b.prefix_len;
  int32_t* gjob = few ? s_gjob : p.gjob;

  auto of = [&](int x) { return few ? s_sum[x] : __ldcg(sum + x); };
  auto prefix_keys = [&](int g) { return (int)min((int64_t)(max(glen[g], 0) & ~15), (int64_t)b.max_blocks * 16); };
  auto rows_at = [&](int i) { return clampi(b.q_start[i], 0, b.n_tokens); };
  auto lens = [&](int i) {
    ReqLens r;
    const int end = b.q_start[i + 1];   // (past the step's rows where they end inside the request: those tokens are not there)
    r.q0 = rows_at(i);
    r.q = max(clampi(end, 0, b.n_tokens) - r.q0, 0);
    r.kv = clampi((int64_t)max(b.kv_len[i], 0) - end + r.q0 + r.q, -(1 << 24), INT_MAX - 1);
    return r;
  };
  auto group = [&](int i) {
    if (G == 0 || i < gstart[0] || i >= gstart[G]) return -1;
    int lo = 0, hi = G;
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (gstart[mid] <= i) lo = mid; else hi = mid;
    }
    return lo;
  };
  // what every later step goes by, all on its way at once
  const int g0 = few && tid <= G && G > 0 ? b.group_start[tid] : 0, p0 = few && tid < G ? b.prefix_len[tid] : 0;
  ReqLens mine{0, 0, 0, -1};   // of request tid
  if (tid < n) mine = lens(tid);
  const int q_end = n > 0 ? rows_at(n) : 0;
  if (tid == 0) ps.cuts = ps.cut_rows = 0;
  Sum jobs{0, 0, 0}, total;
  int turn = 0;
  if (G > 0) {
    if (few) {
      if (tid <= G) s_start[tid] = g0;
      if (tid < G) s_prefix[tid] = p0;
      for (int g = tid + nth; g <= G; g += nth) s_start[g] = b.group_start[g];
      for (int g = tid + nth; g < G; g += nth) s_prefix[g] = b.prefix_len[g];
    }
    // of each group: its requests' costs without and with a shared prefix, whether
    // some row sees less than the prefix, the longest context
    for (int x = tid; x < 4 * G; x += nth) sum[x] = 0;
    __syncthreads();
    if (tid < n) mine.g = group(tid);
  }
  auto request = [&](int i) {
    if (i == tid) return mine;
    ReqLens r = lens(i);
    r.g = group(i);
    return r;
  };
  auto put = [&](Sum at, KvJob j) {
    if (at.count >= p.cap) return;
    j.cost = at.cost;
    j.rows = at.rows;
    if (writer) p.jobs[at.count] = j;
    if (at.count < PLAN_JOBS) s_job[at.count] = j;
  };
  if (G > 0) {
    for (int i = tid; i < n; i += nth) {
      const ReqLens r = request(i);
      const int g = r.g;
      if (g < 0 || r.q == 0) continue;
      const int P = prefix_keys(g), rt = (r.q + w2 - 1) / w2, seen = r.kv - (r.q >> 1);
      const int fl = r.q > p.tpt ? JOB_WIDE : 0;
      // (a warp's requests of one group together; 2^26 a request is more than any step holds)
      const unsigned top = 1u << 26, peers = __match_any_sync(__activemask(), g);
      const unsigned apart = __reduce_add_sync(peers, (unsigned)min((int64_t)rt * job_cost(tiles(seen), fl), (int64_t)top));
      const unsigned with = __reduce_add_sync(peers, (unsigned)min((int64_t)rt * job_cost(tiles(seen - P), fl), (int64_t)top));
      const unsigned less = __reduce_or_sync(peers, r.kv - r.q + 1 < P), most = __reduce_max_sync(peers, (unsigned)max(r.kv, 0));
      if (lane == __ffs(peers) - 1) {
        atomicAdd(&sum[4 * g], (Acc)apart);
        atomicAdd(&sum[4 * g + 1], (Acc)with);
        if (less) sum[4 * g + 2] = 1;
        atomicMax(&sum[4 * g + 3], (Acc)most);
      }
    }
    __syncthreads();
    // prefix jobs.  Shared when that costs less: the group's prefix once for every
    // w2 of its tokens, and a quarter of a tile a token for the parts' way
    // through memory (2 parts written and read, 4 D bytes each a row, against
    // 512 D bytes a tile).
    for (int base = 0; base < G; base += nth) {
      const int g = base + tid;
      int cnt = 0, t0 = 0, t1 = 0, P = 0, first = 0, last_flags = 0;
      Sum x{0, 0, 0};
      if (g < G) {
        first = clampi(gstart[g], 0, n);
        const int last = clampi(gstart[g + 1], 0, n);
        t0 = rows_at(first);
        t1 = rows_at(max(first, last));
        const int rt = t1 > t0 ? (t1 - t0 + w2 - 1) / w2 : 0;
        P = (int)min((Acc)prefix_keys(g), of(4 * g + 3));   // (what nobody has written yet is not read)
        last_flags = t1 - t0 - (rt - 1) * w2 > p.tpt ? JOB_WIDE : 0;
        x.cost = (Int)(rt - 1) * job_cost(tiles(P), JOB_WIDE) + job_cost(tiles(P), last_flags);
        if (P > 0 && first < last && rt > 0 && (int64_t)of(4 * g + 1) + x.cost + W_NARROW / 4 * (t1 - t0) < (int64_t)of(4 * g)) cnt = rt;
        if (cnt == 0) x.cost = 0;
        x.count = cnt;
        x.rows = cnt > 0 ? t1 - t0 : 0;
      }
      Sum at = block_scan(x, scan[turn ^= 1], min(nth, G - base), total);
      at.count += jobs.count;
      at.cost += jobs.cost;
      at.rows += jobs.rows;
      jobs.count += total.count;
      jobs.cost += total.cost;
      jobs.rows += total.rows;
      if (g < G) {
        gjob[g] = cnt > 0 && at.count + cnt <= p.cap ? (int32_t)at.count : -1;
        KvJob j = {};
        j.row = first;
        j.kend = j.lim0 = P;
        j.nt = tiles(P);
        for (int k = 0; k < cnt; k++) {
          j.tok0 = t0 + k * w2;
          j.ntok = min(w2, t1 - j.tok0);
          j.flags = JOB_PREFIX | (of(4 * g + 2) == 0 ? JOB_EVEN : 0) | (k + 1 < cnt ? JOB_WIDE : last_flags);
          put(at, j);
          at.count++;
          at.cost += job_cost(j.nt, j.flags);
          at.rows += j.ntok;
        }
      }
    }
    __syncthreads();   // gjob
  }
  const int prefix_jobs = (int)min((int64_t)jobs.count, (int64_t)p.cap);
  // the requests' own jobs
  for (int base = 0; base < n; base += nth) {
    const int i = base + tid;
    ReqLens r{0, 0, 0, -1};
    int key0 = 0, alone = 1;
    Sum x{0, 0, 0};
    if (i < n) {
      r = request(i);
      if (r.g >= 0 && gjob[r.g] >= 0) {
        alone = 0;
        key0 = prefix_keys(r.g);
      }
      x.count = (r.q + w2 - 1) / w2;
    }
    auto job = [&](int k, int i, int q0, int q, int kv, int key0, int alone) {
      KvJob j;
      const int a = k * w2, e = min(a + w2, q);
      j.tok0 = q0 + a;
      j.ntok = e - a;
      j.row = i;
      j.key0 = key0;
      j.kend = clampi((int64_t)kv - q + e, 0, (int)min((int64_t)b.max_blocks * 16, (int64_t)INT_MAX - 256));
      j.nt = tiles(j.kend - key0);
      j.lim0 = kv - q + a + 1;
      j.flags = (alone ? JOB_ALONE : 0) | (j.ntok > p.tpt ? JOB_WIDE : 0);
      return j;
    };
    // a request of one job is its thread's; a longer one is its warp's
    const KvJob one = job(0, i, r.q0, r.q, r.kv, key0, alone);
    if (x.count == 1) x.cost = job_cost(one.nt, one.flags);
    const unsigned longer = __ballot_sync(~0u, x.count > 1);
    for (unsigned todo = longer; todo; todo &= todo - 1) {
      const int src = __ffs(todo) - 1;
      const int sc = __shfl_sync(~0u, (int)x.count, src), sq = __shfl_sync(~0u, r.q, src), sk = __shfl_sync(~0u, r.kv, src);
      const int s1 = __shfl_sync(~0u, key0, src), sa = __shfl_sync(~0u, alone, src);
      Int c = 0;
      for (int k = lane; k < sc; k += 32) {
        const KvJob j = job(k, 0, 0, sq, sk, s1, sa);
        c += job_cost(j.nt, j.flags);
      }
#pragma unroll
      for (int o = 16; o; o >>= 1) c += __shfl_xor_sync(~0u, c, o);
      if (lane == src) x.cost = c;
    }
    Sum at = block_scan(x, scan[turn ^= 1], min(nth, n - base), total);
    at.count += jobs.count;
    at.cost += jobs.cost;
    jobs.count += total.count;
    jobs.cost += total.cost;
    // where its tokens' parts will be, for the join
    auto share = [&](int t, int q0, int g, int job0) {
      const int pj = gjob[g];
      const KvJob& j = pj < PLAN_JOBS ? s_job[pj] : p.jobs[pj];
      const int64_t in = q0 + t - j.tok0, to = j.rows + in;
      if (in >= 0 && to < b.n_tokens) p.shared[to] = make_int4(q0 + t, pj + (int)(in / w2), job0 + t / w2, 0);
    };
    if (writer && x.count == 1 && !alone)
      for (int t = 0; t < r.q; t++) share(t, r.q0, r.g, (int)at.count);
    if (x.count == 1) put(at, one);
    for (unsigned todo = longer; todo; todo &= todo - 1) {
      const int src = __ffs(todo) - 1;
      const int sc = __shfl_sync(~0u, (int)x.count, src), si = __shfl_sync(~0u, i, src);
      const int s0 = __shfl_sync(~0u, r.q0, src), sq = __shfl_sync(~0u, r.q, src), sk = __shfl_sync(~0u, r.kv, src);
      const int s1 = __shfl_sync(~0u, key0, src), sa = __shfl_sync(~0u, alone, src);
      Sum sat{__shfl_sync(~0u, at.count, src), __shfl_sync(~0u, at.cost, src), 0};
      const int sg = __shfl_sync(~0u, r.g, src);
      if (writer && !sa)
        for (int t = lane; t < sq; t += 32) share(t, s0, sg, (int)sat.count);
      for (int k0 = 0; k0 < sc; k0 += 32) {
        const int k = k0 + lane;
        const KvJob j = job(min(k, sc - 1), si, s0, sq, sk, s1, sa);
        const Int c = k < sc ? job_cost(j.nt, j.flags) : 0;
        Int before = c;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
          const Int y = __shfl_up_sync(~0u, before, o);
          if (lane >= o) before += y;
        }
        if (k < sc) put(Sum{sat.count + k, sat.cost + before - c, 0}, j);
        sat.cost += __shfl_sync(~0u, before, 31);
      }
    }
  }
  // rows of no request: jobs without keys
  const int pads = (b.n_tokens - q_end + w2 - 1) / w2;
  for (int k = tid; k < pads; k += nth) {
    KvJob j = {};
    j.tok0 = q_end + k * w2;
    j.ntok = min(w2, b.n_tokens - j.tok0);
    j.flags = JOB_ALONE | (j.ntok > p.tpt ? JOB_WIDE : 0);
    put(Sum{(Int)(jobs.count + k), jobs.cost + (Int)k * OV_NARROW, 0}, j);
  }
  __syncthreads();   // the jobs
  const bool room = (int64_t)jobs.count + pads <= p.cap;
  const int J = room ? (int)jobs.count + pads : 0;
  auto job_at = [&](int j) { return j < PLAN_JOBS ? s_job[j] : p.jobs[j]; };
  auto cost_at = [&](int j) { return j < PLAN_JOBS ? s_job[j].cost : p.jobs[j].cost; };
  int64_t all = 0;
  if (J > 0) {
    const KvJob j = job_at(J - 1);
    all = (j.cost + job_cost(j.nt, j.flags)) * n_kv_heads;
  }
  // two tiles at least, one for each stream of a CTA
  const int64_t per = max((all + p.ctas - 1) / p.ctas, (int64_t)(2 * W_NARROW + OV_NARROW));
  // the job and head that has cost u < all, and how far in
  auto locate = [&](int64_t u, KvStart& s) {
    int lo = 0, hi = J;   // the last job that starts at or before u
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (cost_at(mid) * n_kv_heads <= u) lo = mid; else hi = mid;
    }
    s.job = lo;
    s.j = job_at(lo);
    const int64_t in = u - s.j.cost * n_kv_heads;
    const int cj = job_cost(s.j.nt, s.j.flags);
    s.head = (int)quotient(in, cj);
    s.off = (int)(in - (int64_t)s.head * cj);
  };
  // the end of the job and head that has cost u - 1 (u <= all): shares begin and end there when none is to be cut
  auto whole_end = [&](int64_t u) {
    if (u <= 0) return (int64_t)0;
    KvStart s;
    locate(u - 1, s);
    return u - 1 - s.off + job_cost(s.j.nt, s.j.flags);
  };
  for (int c = tid; c < p.ctas; c += nth) {
    int64_t u = c * per, end = min(u + per, all);
    KvStart s = {};
    if (p.whole && u < all) {
      u = whole_end(u);
      end = whole_end(end);
    }
    if (u < end) {
      locate(u, s);
      s.rem = end - u;
      const KvJob j = s.j;
      const int cj = job_cost(j.nt, j.flags);
      const int64_t u0 = u - s.off;
      if (writer && s.off > 0 && j.nt > 0 && (j.flags & JOB_ALONE) && u0 >= u - per) {   // not cut before
        int t0, t1, e = (int)quotient(u0 + cj - 1, per);
        KvCut cut = {};
        cut.c0 = c - 1;
        cut.first = segment(u0, cj, j.flags, j.nt, per, c - 1, t0, t1) ? c - 1 : c;
        cut.last = segment(u0, cj, j.flags, j.nt, per, e, t0, t1) ? e : e - 1;
        cut.tok0 = j.tok0;
        cut.head = s.head;
        cut.ntok = j.ntok;
        if (cut.first < cut.last) {   // (else whole in one CTA)
          atomicMax(&ps.cut_rows, j.ntok * p.ratio);
          p.cut[atomicAdd(&ps.cuts, 1)] = cut;
        }
      }
    }
    if (all_ctas) p.start[c] = s;
    else if (c == (int)blockIdx.x) *own_start = s;
  }
  if (!all_ctas) {
    const int64_t u = blockIdx.x * per;
    for (int j = tid; j < J; j += nth) {
      const KvJob x = s_job[j];   // (a share without cuts begins later and ends in its last job)
      const int64_t at = x.cost * n_kv_heads;
      if (at < u + per && at + (int64_t)job_cost(x.nt, x.flags) * n_kv_heads > u) p.jobs[j] = x;
    }
  }
  __syncthreads();
  if (writer && tid == 0) *p.head = KvHead{all, per, J, room ? prefix_jobs : 0, room ? (int)jobs.rows : 0, ps.cuts, ps.cut_rows, 0};
}

__global__ void __launch_bounds__(NT_PLAN) k_kv_plan(rs_kv_batch b, KvPlan p, int n_kv_heads) {
  extern __shared__ __align__(16) unsigned char psm[];
  behind_stream();
  make_plan<int64_t>(b, p, n_kv_heads, *reinterpret_cast<PlanSmem*>(psm), true, nullptr);
}

// ------------------------------------------------------------------ PTX

__device__ __forceinline__ uint32_t smem_u32(const void* x) { return (uint32_t)__cvta_generic_to_shared(x); }

__device__ __forceinline__ void mbar_init(uint32_t bar, uint32_t count) {
  asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory");
}
__device__ __forceinline__ void mbar_arrive(uint32_t bar) {
  asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void mbar_expect(uint32_t bar, uint32_t bytes) {
  asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
#ifndef KV_WAIT_CLOCKS
#define KV_WAIT_CLOCKS (1ll << 32)
#define KV_TRY "try_wait"
#else   // (a test builds with less, and a try may take longer than that)
#define KV_TRY "test_wait"
#endif
__device__ __forceinline__ bool mbar_try(uint32_t bar, uint32_t parity) {
  uint32_t ok;
  asm volatile(
      "{\n\t.reg .pred p;\n\tmbarrier." KV_TRY ".parity.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
  return ok != 0;
}
// A wait ends after 2^32 clocks (two seconds) at the latest: then the CTA gives
// up.  Every later wait returns at once, so what is left of a run passes with
// whatever the tiles hold (every address in it comes from the run, which stays).
// No role takes another run, whose slot may hold none, and no load is issued for a
// stage that was not given back, whose barrier may still count a load.
__device__ __noinline__ void mbar_lost(volatile int* lost, int32_t* err) {
  *lost = 1;
  *reinterpret_cast<volatile int32_t*>(err) = 1;
}
__device__ __forceinline__ void mbar_wait(uint32_t bar, uint32_t parity, volatile int* lost, int32_t* err) {
  if (mbar_try(bar, parity)) return;
  const long long from = clock64();
  while (!*lost) {
    if (clock64() - from >= KV_WAIT_CLOCKS) {
      mbar_lost(lost, err);
      return;
    }
    if (mbar_try(bar, parity)) return;
  }
}
// By a whole warp: whether the CTA has given up, the same for all lanes.
__device__ __forceinline__ bool gave_up(volatile int* lost) { return __any_sync(~0u, *lost); }

__device__ __forceinline__ bool elect_one() {
  uint32_t r;
  asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(r));
  return r != 0;
}

__device__ __forceinline__ void tma_3d(uint32_t dst, const CUtensorMap* m, int x, int y, int z, uint32_t bar) {
  asm volatile(
      "cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
      ::"r"(dst), "l"(m), "r"(x), "r"(y), "r"(z), "r"(bar) : "memory");
}
__device__ __forceinline__ void tma_4d(uint32_t dst, const CUtensorMap* m, int x, int y, int z, int w, uint32_t bar) {
  asm volatile(
      "cp.async.bulk.tensor.4d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];"
      ::"r"(dst), "l"(m), "r"(x), "r"(y), "r"(z), "r"(w), "r"(bar) : "memory");
}

// Shared memory descriptors of 128-byte rows swizzled over 8 of them.  Rows are
// MMA rows (K-major): 8-row groups 1024 bytes apart.  Rows are MMA depth
// (MN-major): the same groups along the depth, 64-element columns `lead` apart.
__device__ __forceinline__ uint64_t smem_desc(uint32_t addr, uint32_t lead) {
  return (uint64_t)((addr & 0x3FFFF) >> 4) | ((uint64_t)(lead >> 4) << 16) | ((uint64_t)(1024 >> 4) << 32) |
         (1ull << 46) | (2ull << 61);
}

__device__ __forceinline__ void mma_ss(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t acc) {
  asm volatile(
      "{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}"
      ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(acc) : "memory");
}
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, uint32_t acc) {
  asm volatile(
      "{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
      ::"r"(d), "r"(a), "l"(b), "r"(idesc), "r"(acc) : "memory");
}
__device__ __forceinline__ void mma_commit(uint32_t bar) {
  asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void tc_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }

#define R8(v, o) "r"(v[o]), "r"(v[o + 1]), "r"(v[o + 2]), "r"(v[o + 3]), "r"(v[o + 4]), "r"(v[o + 5]), "r"(v[o + 6]), "r"(v[o + 7])
#define W8(v, o) "=r"(v[o]), "=r"(v[o + 1]), "=r"(v[o + 2]), "=r"(v[o + 3]), "=r"(v[o + 4]), "=r"(v[o + 5]), "=r"(v[o + 6]), "=r"(v[o + 7])
#define N32 \
  "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}"
// 32 columns of the thread's lane
__device__ __forceinline__ void tm_ld32(uint32_t* v, uint32_t addr) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 " N32 ", [%32];"
               : W8(v, 0), W8(v, 8), W8(v, 16), W8(v, 24) : "r"(addr));
}
__device__ __forceinline__ void tm_st32(uint32_t addr, const uint32_t* v) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x32.b32 [%32], " N32 ";"
               ::R8(v, 0), R8(v, 8), R8(v, 16), R8(v, 24), "r"(addr) : "memory");
}
// Until the loads so far have come; v (one of them) is not touched before.
#define U8(v, o) "+r"(v[o]), "+r"(v[o + 1]), "+r"(v[o + 2]), "+r"(v[o + 3]), "+r"(v[o + 4]), "+r"(v[o + 5]), "+r"(v[o + 6]), "+r"(v[o + 7])
__device__ __forceinline__ void tm_wait_ld(uint32_t* v) {
  asm volatile("tcgen05.wait::ld.sync.aligned;" : U8(v, 0), U8(v, 8), U8(v, 16), U8(v, 24)::"memory");
}
// 16 lanes by 32 columns, 8 columns a group of four registers: thread t has columns
// 2 (t % 4) and the next of rows t / 4 (registers 0, 1) and t / 4 + 8 (2, 3).
__device__ __forceinline__ void tm_ld16(uint32_t* v, uint32_t addr) {
  asm volatile(
      "tcgen05.ld.sync.aligned.16x256b.x4.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
      : W8(v, 0), W8(v, 8) : "r"(addr));
}
__device__ __forceinline__ void tm_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ void fma2(float& x, float& y, float a, float b) {   // (x, y) a + b
  asm("{\n\t.reg .b64 s, t, u;\n\tmov.b64 s, {%0, %1};\n\tmov.b64 t, {%2, %2};\n\tmov.b64 u, {%3, %3};\n\t"
      "fma.rn.f32x2 s, s, t, u;\n\tmov.b64 {%0, %1}, s;\n\t}" : "+f"(x), "+f"(y) : "f"(a), "f"(b));
}
__device__ __forceinline__ void mul2(float& x, float& y, float a) {
  asm("{\n\t.reg .b64 s, t;\n\tmov.b64 s, {%0, %1};\n\tmov.b64 t, {%2, %2};\n\t"
      "mul.rn.f32x2 s, s, t;\n\tmov.b64 {%0, %1}, s;\n\t}" : "+f"(x), "+f"(y) : "f"(a));
}
__device__ __forceinline__ void add2(float& x, float& y, float a, float b) {
  asm("{\n\t.reg .b64 s, t;\n\tmov.b64 s, {%0, %1};\n\tmov.b64 t, {%2, %3};\n\t"
      "add.rn.f32x2 s, s, t;\n\tmov.b64 {%0, %1}, s;\n\t}" : "+f"(x), "+f"(y) : "f"(a), "f"(b));
}
template <bool HALF>
__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
  uint32_t r;
  if (HALF) asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  else asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}

// ------------------------------------------------------------------ a row's tile of scores

// Keys from `left` on are out of the row's sight.
__device__ __forceinline__ void cut32(uint32_t* v, int left) {
#pragma unroll
  for (int k = 0; k < 32; k++)
    if (k >= left) v[k] = 0xFF800000u;
}
__device__ __forceinline__ float max3(float a, uint32_t b, uint32_t c) {
  float r;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(__uint_as_float(b)), "f"(__uint_as_float(c)));
  return r;
}

// The largest score of a row's tile, of which the warp's rows see `seen` keys at
// most and this one `left`.
__device__ __noinline__ float row_max(uint32_t ts, int seen, int left) {
  float m = -INFINITY, n = -INFINITY;
#pragma unroll 1
  for (int c = 0; c < min(seen, TK); c += 32) {
    uint32_t x[32];
    tm_ld32(x, ts + c);
    tm_wait_ld(x);
    cut32(x, left - c);
#pragma unroll
    for (int k = 0; k < 32; k += 4) {
      m = max3(m, x[k], x[k + 1]);
      n = max3(n, x[k + 2], x[k + 3]);
    }
  }
  return fmaxf(m, n);
}

__device__ __forceinline__ float max_of32(const uint32_t* v) {
  float m = __uint_as_float(v[0]), n = __uint_as_float(v[31]);
#pragma unroll
  for (int k = 1; k < 29; k += 4) {
    m = max3(m, v[k], v[k + 1]);
    n = max3(n, v[k + 2], v[k + 3]);
  }
  return fmaxf(max3(m, v[29], v[30]), n);
}

// Weights exp2(sl s + nm) of 4 N scores, packed in pairs into v's first half, and
// added to the sums of even and odd keys.
template <bool HALF, int N>
__device__ __forceinline__ void row_exp(float sl, float nm, uint32_t* v, float& a0, float& a1) {
  float b0 = 0.0f, b1 = 0.0f;
#pragma unroll
  for (int k = 0; k < 4 * N; k += 4) {
    float e0 = __uint_as_float(v[k]), e1 = __uint_as_float(v[k + 1]), e2 = __uint_as_float(v[k + 2]),
          e3 = __uint_as_float(v[k + 3]);
    fma2(e0, e1, sl, nm);
    fma2(e2, e3, sl, nm);
    e0 = ex2(e0); e1 = ex2(e1); e2 = ex2(e2); e3 = ex2(e3);
    add2(a0, a1, e0, e1);
    add2(b0, b1, e2, e3);
    v[k / 2] = pack2<HALF>(e0, e1);
    v[k / 2 + 1] = pack2<HALF>(e2, e3);
  }
  add2(a0, a1, b0, b1);
}

__device__ __forceinline__ float minus(float m, float sl) { return m == -INFINITY ? 0.0f : -__fmul_rn(m, sl); }

// References so large that m sl rounds by more than a half: a weight exp2(sl s + nm) then carries that rounding, which
// may be more than a type's range.
constexpr float FAR = 16777216.0f;

// A tile's weights where some row of the warp is that far (m of each row at its tile's maximum): exp2(sl (s - m)),
// which the largest score makes 1 whatever its size.  The other rows' weights are the same as elsewhere.
template <bool HALF>
__device__ __noinline__ float2 far_weights(uint32_t ts, int seen, int left, float sl, float m) {
  const float nm = minus(m, sl);
  const bool far = fabsf(nm) > FAR;
  float a0 = 0.0f, a1 = 0.0f;
#pragma unroll 1
  for (int c = 0; c < TK; c += 64) {   // (the weights' columns have been read before they are written)
    uint32_t w[32];
#pragma unroll
    for (int h = 0; h < 64; h += 32) {
      uint32_t v[32];
#pragma unroll
      for (int k = 0; k < 32; k++) v[k] = 0;
      if (c + h < seen) {
        tm_ld32(v, ts + c + h);
        tm_wait_ld(v);
        cut32(v, left - c - h);
#pragma unroll
        for (int k = 0; k < 32; k++)
          if (far) v[k] = __float_as_uint(__fsub_rn(__uint_as_float(v[k]), m));
        row_exp<HALF, 8>(sl, far ? 0.0f : nm, v, a0, a1);
      }
#pragma unroll
      for (int k = 0; k < 16; k++) w[h / 2 + k] = v[k];
    }
    tm_st32(ts + c / 2, w);
  }
  return make_float2(a0, a1);
}

// ------------------------------------------------------------------ joining

// Where the parts of a job and head are: whole in its place among all rows (one
// part, last < first), or in CTAs first .. last.
struct Parts {
  int c0, first, last, count;
};

// By a warp: of job j in lanes 0..15 and of job j in lanes 16..31, with a share of the
// arithmetic a lane (a job's first CTA in lanes 0 and 16, its last one in 8 and 24).
__device__ __forceinline__ void parts_of(const KvJob& j, int head, int n_kv_heads, const KvHead& hd, int lane, Parts& x, Parts& y) {
  const bool end = lane & 8;
  const int cost = job_cost(j.nt, j.flags);
  const int64_t u0 = j.cost * n_kv_heads + (int64_t)head * cost;
  const int64_t c = quotient(end ? u0 + cost - 1 : u0, hd.per);
  int t0, t1;
  const int in = (int)(segment(u0, cost, j.flags, j.nt, hd.per, c, t0, t1) ? c : end ? c - 1 : c + 1);
  auto gather = [&](int from) {
    Parts r;
    r.c0 = (int)__shfl_sync(~0u, (int)c, from);
    r.first = __shfl_sync(~0u, in, from);
    r.last = __shfl_sync(~0u, in, from + 8);
    r.count = max(r.last - r.first + 1, 1);
    if (r.count == 1) r.last = r.first - 1;
    return __shfl_sync(~0u, j.nt, from) > 0 ? r : Parts{0, 0, 0, 0};
  };
  x = gather(0);
  y = gather(16);
}

// One row (token, head) from its parts: x's (row rx of the 256 if cut, else at
// home), then y's.  A lane takes the reference and sum of a part, the warp the
// largest reference and the weights, and the rows of Z parts are on their way at
// once.  (Log sums in their place would lose the sums where scores are large: at
// 2^24 a log sum has steps of 2.)
template <int D, bool HALF, int Z>
__device__ __forceinline__ void join_row(const KvAttendArgs& a, const KvPlan& p, const Parts& x, int rx, const Parts& y, int ry,
                                         int64_t row, int hq, int lane) {
  constexpr int E = D / 32;
  const int64_t home = row * a.n_heads + hq, all = (int64_t)a.b.n_tokens * a.n_heads;
  const int count = x.count + y.count;
  float m = -INFINITY, l = 0.0f, o[E];
#pragma unroll
  for (int e = 0; e < E; e++) o[e] = 0.0f;
  for (int base = 0; base < count; base += 32) {
    const int k = base + lane, here = min(32, count - base);
    const float* src = nullptr;
    float2 s = make_float2(-INFINITY, 0.0f);
    if (k < count) {
      const Parts& q = k < x.count ? x : y;
      const int c = q.first + (k < x.count ? k : k - x.count);
      const bool whole = q.last < q.first;
      const int64_t at = whole ? (k < x.count ? 0 : all) + home
                               : ((int64_t)c * 2 + (c == q.c0 ? 1 : 0)) * 256 + (k < x.count ? rx : ry);
      s = (whole ? p.home_sum : p.part_sum)[at];
      src = (whole ? p.home : p.part) + at * D;
    }
    float wt = 0.0f;
    for (int q = 0; q < here; q += Z) {
      float v[Z][E];
#pragma unroll
      for (int z = 0; z < Z; z++) {   // (past the last part: weight 0, the last one's row)
        const int from = min(q + z, here - 1);
        const float* r = reinterpret_cast<const float*>(__shfl_sync(~0u, reinterpret_cast<unsigned long long>(src), from)) + lane * E;
        if constexpr (E == 4) {
          const float4 t = *reinterpret_cast<const float4*>(r);
          v[z][0] = t.x; v[z][1] = t.y; v[z][2] = t.z; v[z][3] = t.w;
        } else {
          const float2 t = *reinterpret_cast<const float2*>(r);
          v[z][0] = t.x; v[z][1] = t.y;
        }
      }
      if (q == 0) {   // the weights, with the first rows on their way
        float big = s.x;
#pragma unroll
        for (int z = 16; z; z >>= 1) big = fmaxf(big, __shfl_xor_sync(~0u, big, z));
        const float m2 = fmaxf(m, big);
        const float f = m == -INFINITY ? 0.0f : ex2(__fsub_rn(m, m2));
        wt = s.y == 0.0f ? 0.0f : __fmul_rn(s.y, ex2(__fsub_rn(s.x, m2)));
        float sum = wt;
#pragma unroll
        for (int z = 16; z; z >>= 1) sum = __fadd_rn(sum, __shfl_xor_sync(~0u, sum, z));
        l = fmaf(l, f, sum);
#pragma unroll
        for (int e = 0; e < E; e++) o[e] = __fmul_rn(o[e], f);
        m = m2;
      }
#pragma unroll
      for (int z = 0; z < Z; z++) {
        const float w = __shfl_sync(~0u, wt, min(q + z, here - 1));
        if (q + z < here && w != 0.0f) {
#pragma unroll
          for (int e = 0; e < E; e++) o[e] = fmaf(w, v[z][e], o[e]);
        }
      }
    }
  }
  const float inv = l == 0.0f ? 0.0f : __fdiv_rn(1.0f, l);
  uint16_t* out = static_cast<uint16_t*>(a.out) + row * a.o_ts + hq * a.o_hs + lane * E;
  uint32_t z[E / 2];
#pragma unroll
  for (int e = 0; e < E; e += 2) z[e / 2] = pack2<HALF>(__fmul_rn(o[e], inv), __fmul_rn(o[e + 1], inv));
  if constexpr (E == 4) *reinterpret_cast<uint2*>(out) = make_uint2(z[0], z[1]);
  else *reinterpret_cast<uint32_t*>(out) = z[0];
  if (a.lse && lane == 0)
    a.lse[home] = l == 0.0f ? -INFINITY : __fmul_rn(__fadd_rn(m, __log2f(l)), 0.6931471805599453f);
}

// Rows that have parts, a warp a row: of the jobs that a share's end cut, and of
// shared groups, whose rows have a prefix job and an own one.  The parts' order
// is the keys', so the result does not depend on when they came.
// Bound: latency (head, list, jobs and parts depend on each other) and, past a few
// rows a warp, arithmetic: 2 us for the rows of one token, 3 to 6 us for the shared rows
// of 8 to 64 tokens (1 to 2 us more when every lane found all parts' places itself).  Joining in the
// attention kernel, behind a barrier of all CTAs, took as long and left fewer warps
// to it (16 rows a group on a prefix of 32 768: 49 us in all against 44 us).
template <int D, bool HALF, int Z>
__global__ void __launch_bounds__(256) k_kv_join(const __grid_constant__ KvAttendArgs a,
                                                 const __grid_constant__ KvPlan p) {
  behind_stream();
  const int lane = threadIdx.x & 31, first = blockIdx.x * 8 + (threadIdx.x >> 5), step = gridDim.x * 8;
  const int hk = a.c.n_kv_heads;
  const KvHead hd = *p.head;
  auto part_row = [&](int tok, int hl) {   // a token's and head's of a job's 256
    return (tok >= p.tpt ? 128 + (tok - p.tpt) * p.ratio : tok * p.ratio) + hl;
  };
  const int64_t cuts = (int64_t)hd.cuts * hd.cut_rows, rows = cuts + (int64_t)hd.shared * a.n_heads;
  for (int64_t x = first; x < rows; x += step) {
    Parts pre{0, 0, 0, 0}, own{0, 0, 0, 0};
    int row, hq, rp, ro = 0;
    if (x < cuts) {
      const int u = (int)quotient(x, hd.cut_rows), r = (int)(x - (int64_t)u * hd.cut_rows), tok = r / p.ratio, hl = r - tok * p.ratio;
      const KvCut c = p.cut[u];
      if (tok >= c.ntok) continue;
      pre = Parts{c.c0, c.first, c.last, c.last - c.first + 1};
      row = c.tok0 + tok;
      hq = c.head * p.ratio + hl;
      rp = part_row(tok, hl);
    } else {
      const int64_t t = quotient(x - cuts, a.n_heads);
      hq = (int)(x - cuts - t * a.n_heads);
      const int4 e = p.shared[t];
      // (starts that decrease leave entries unwritten)
      if (e.y < 0 || e.y >= hd.prefix_jobs || e.z < 0 || e.z >= hd.jobs) continue;
      const KvJob j = p.jobs[lane < 16 ? e.y : e.z];
      const int kh = hq / p.ratio, hl = hq - kh * p.ratio, tok = e.x - j.tok0, at = part_row(tok, hl);
      if (__any_sync(~0u, tok < 0 || tok >= j.ntok)) continue;
      row = e.x;
      rp = __shfl_sync(~0u, at, 0);
      ro = __shfl_sync(~0u, at, 16);
      parts_of(j, kh, hk, hd, lane, pre, own);
    }
    join_row<D, HALF, Z>(a, p, pre, rp, own, ro, row, hq, lane);
  }
}

// ------------------------------------------------------------------ the kernel

// Tiles t0 .. t1 - 1 of a job and head.
struct Seg {
  KvJob job;
  int head, t0, t1;
  int cut_front;        // the CTA's share began inside the job
  __device__ bool wide() const { return job.flags & JOB_WIDE; }
  __device__ int nt() const { return t1 - t0; }
};

// What a CTA's two streams do together, in shared memory for its warps:
//   RUN_WIDE   one job of more than 128 rows, half of them each
//   RUN_SPLIT  one job of fewer rows, every other tile each, joined at the end
//   RUN_PAIR   two such jobs, one each (short ones: no join, and one stream's stores
//              run under the other's products)
//   RUN_NONE   rows without keys
//   RUN_END    no more
enum { RUN_WIDE, RUN_SPLIT, RUN_PAIR, RUN_NONE, RUN_END };

struct Run {
  Seg seg[2];           // of stream 0 (or both), of stream 1 in a RUN_PAIR
  int kind, n[2];       // tiles of each stream
  int reserved0;
  int32_t page[32];     // blocks of each stream's first two tiles
};

// A CTA's share of the jobs, as runs.
struct Walk {
  const KvJob* jobs;
  int64_t rem;
  int j, h, off, heads;
  KvJob ahead;          // job j
  bool held;            // b waits for its turn
  int kind;
  Seg a, b;

  __device__ Walk(const KvPlan& p, const KvStart& s, int n_kv_heads) {
    jobs = p.jobs;
    heads = n_kv_heads;
    rem = s.rem;
    j = s.job; h = s.head; off = s.off;
    ahead = s.j;
    held = false;
  }
  __device__ bool pull(Seg& s) {
    while (rem > 0) {
      const int cost = job_cost(ahead.nt, ahead.flags);
      if (cost == 0) {
        ahead = jobs[++j];
        continue;
      }
      const int take = (int)min((int64_t)(cost - off), rem);
      const bool empty = ahead.nt == 0 && off == 0;
      s.t0 = min(tile_at(off, ahead.flags), ahead.nt);
      s.t1 = min(tile_at(off + take, ahead.flags), ahead.nt);
      s.cut_front = off > 0;
      s.head = h;
      s.job = ahead;
      rem -= take;
      off += take;
      if (off == cost) {
        off = 0;
        if (++h == heads) {
          h = 0;
          j++;
          if (rem > 0) ahead = jobs[j];
        }
      }
      if (s.t1 > s.t0 || empty) return true;
    }
    return false;
  }
  __device__ void next() {
    if (held) {
      a = b;
    } else if (!pull(a)) {
      kind = RUN_END;
      return;
    }
    held = false;
    if (a.nt() == 0) {
      kind = RUN_NONE;
    } else if (a.wide()) {
      kind = RUN_WIDE;
    } else {
      kind = RUN_SPLIT;
      held = pull(b);
      // streams of much the same length
      if (held && !b.wide() && b.nt() > 0 && 2 * b.nt() >= a.nt() && 2 * a.nt() >= b.nt()) {
        kind = RUN_PAIR;
        held = false;
      }
    }
  }
};

constexpr int NR = 4;   // runs ahead

template <int D>
struct Lay {
  static constexpr int QSLOT = 128 * D * 2;       // bytes of 128 rows
  static constexpr int STAGE = TK * D * 2;        // bytes of a tile of K or V
  static constexpr int NST = D == 128 ? 5 : 12;   // stages: what 227 KB leave beside the rows
  static constexpr int RING = 2 * QSLOT;
  static constexpr int MISC = RING + NST * STAGE;
  // barriers: full[NST], empty[NST], qfull[2], qempty[2], sfull[2], pfull[2], ofull[2], oempty[2], meet, rfull[NR], rempty[NR]
  static constexpr int NBAR = 2 * NST + 13 + 2 * NR;
  static constexpr int ML = MISC + 384;           // float2 [128]
  static constexpr int RUNS = ML + 1024;          // Run [NR]
  static constexpr int START = RUNS + NR * (int)sizeof(Run);   // KvStart
  static constexpr int SMEM = START + (int)sizeof(KvStart);
  static_assert((int)sizeof(PlanSmem) <= MISC, "the plan's memory is the tiles'");
};

// The loads' order is that of first use: K of each stream's first tile, then for
// i = 0, 1, ... and each stream the V of its tile i and the K of its tile i + 1
// (a RUN_WIDE job's streams share the tiles: those of stream 0).  The loads before
// the V of stream s's tile i:
__device__ __forceinline__ int vplace(int s, int i, int n0, int n1) {
  auto upto = [&](int n) { return min(i, n) + min(i, max(n - 1, 0)); };
  return (n0 > 0) + (n1 > 0) + upto(n0) + upto(n1) + (s ? (i < n0) + (i + 1 < n0) : 0);
}

// Two streams of 128 rows share the tensor cores, so that one's softmax runs
// under the other's products.  Warps 0-3 and 4-7 are the streams' softmax, a
// thread a row (so no reduction crosses threads); warp 8 issues the products, warp
// 9 the loads, warp 10 finds the runs.  Warps 8 and 9 run as one and let one
// elected thread issue: from a divergent branch the same products took 900 us
// instead of 650 us (4096 tokens behind 12 288).
// Shared memory: two slots of 128 rows, the rest a ring of K and V tiles (160 KB:
// at 43 bytes a nanosecond and SM and 1.5 us of latency HBM asks for 65 KB), each
// loaded page by page from its block (swizzled 128-byte rows, 2 copies of 2 KB a
// page at D = 128).
// TMEM: S of each stream 128 columns (P, 64 columns, overwrites it), O D each:
// full at D = 128, so a stream's next scores wait for its last weights' product.
// The m of a row is the largest score of its first 32 keys and moves only when a
// tile's weights sum to more than 2^15 (up to there each is in range of fp16, and
// bf16 weights are as exact at any size), which hardly happens: O and l are
// scaled then.  Scores, m, l and O are 32 bits; the weights are rounded once to
// the cache's type, l sums them unrounded.
// Measured and not kept: 32 columns of scores loaded while 32 are worked on
// (1016 us against 900 us); the running maximum in every tile; rows written with
// O kept in registers past its release (spills).
template <int D, bool HALF>
__global__ void __launch_bounds__(NT_ATT, 1)
k_kv_attend(const __grid_constant__ CUtensorMap mk, const __grid_constant__ CUtensorMap mv,
            const __grid_constant__ CUtensorMap mq, const __grid_constant__ CUtensorMap mq1,
            const __grid_constant__ KvAttendArgs a, const __grid_constant__ KvPlan p) {
  using L = Lay<D>;
  extern __shared__ __align__(1024) unsigned char sm[];
  const uint32_t base = smem_u32(sm);
  const int tid = threadIdx.x, warp = __shfl_sync(~0u, tid >> 5, 0), lane = tid & 31;
  const uint32_t bars = base + L::MISC;
  const uint32_t FULL = bars, EMPTY = bars + 8 * L::NST, QFULL = bars + 16 * L::NST, QEMPTY = QFULL + 16,
                 SFULL = QFULL + 32, PFULL = QFULL + 48, OFULL = QFULL + 64, OEMPTY = QFULL + 80,
                 MEET = QFULL + 96, RFULL = QFULL + 104, REMPTY = RFULL + 8 * NR;
  Run* const runs = reinterpret_cast<Run*>(sm + L::RUNS);
  KvStart* const start = reinterpret_cast<KvStart*>(sm + L::START);
  uint32_t* s_tmem = reinterpret_cast<uint32_t*>(sm + L::MISC + 8 * L::NBAR);
  volatile int* lost = reinterpret_cast<volatile int*>(sm + L::MISC + 8 * L::NBAR + 4);
  static_assert(8 * L::NBAR + 8 <= 384, "barriers");
  static_assert(L::SMEM <= 227 * 1024, "shared memory");
  if (base & 1023) {   // (swizzled tiles lie on 1024-byte boundaries)
    if (tid == 0) *reinterpret_cast<volatile int32_t*>(p.err) = 1;
    return;
  }
  if (tid == 0) {
    for (int s = 0; s < L::NST; s++) { mbar_init(FULL + 8 * s, 1); mbar_init(EMPTY + 8 * s, 1); }
    for (int s = 0; s < 2; s++) {
      mbar_init(QFULL + 8 * s, 1);
      mbar_init(QEMPTY + 8 * s, 1);
      mbar_init(SFULL + 8 * s, 1);
      mbar_init(PFULL + 8 * s, 4);
      mbar_init(OFULL + 8 * s, 1);
      mbar_init(OEMPTY + 8 * s, 4);
    }
    for (int s = 0; s < NR; s++) { mbar_init(RFULL + 8 * s, 1); mbar_init(REMPTY + 8 * s, 10); }
    mbar_init(MEET, 4);
    *lost = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  if (warp == 8) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_u32(s_tmem)) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    tc_before();
  }
  __syncthreads();
  tc_after();
  const uint32_t tmem = *s_tmem;
  behind_stream();
  if (p.planned) {
    if (tid == 0) *start = p.start[blockIdx.x];
  } else {
    make_plan<int32_t>(a.b, p, a.c.n_kv_heads, *reinterpret_cast<PlanSmem*>(sm), false, start);
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");   // (copies into the same memory follow)
  }
  __syncthreads();

  auto drain = [] {   // copies in flight end before the CTA's memory is another's
    const long long t = clock64();
    while (clock64() - t < 20000000ll) {}
  };
  if (warp >= 8) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 88;");
    if (warp == 10) {
      // ---------------- runs
      Walk w(p, *start, a.c.n_kv_heads);
      for (uint32_t k = 0;; k++) {
        w.next();
        // the lane's page: stream lane / 16, its tile (lane / 8) % 2
        const int s = lane >> 4, i = (lane >> 3) & 1;
        const Seg& g = w.kind == RUN_PAIR && s ? w.b : w.a;
        const int t = g.t0 + (w.kind == RUN_SPLIT ? 2 * i + s : i), pg = g.job.key0 / 16 + t * (TK / 16) + (lane & 7);
        int id = 0;
        if (w.kind <= RUN_PAIR && t < g.t1 && pg < (g.job.kend + 15) / 16)
          id = a.b.table[(int64_t)g.job.row * a.b.table_stride + pg];
        if (id < 0 || id >= a.c.n_blocks) id = (int)a.c.n_blocks;   // reads as zeros
        if (k >= NR) mbar_wait(REMPTY + 8 * (k % NR), (k / NR - 1) & 1, lost, p.err);
        if (gave_up(lost)) break;
        Run* const r = runs + k % NR;
        r->page[lane] = id;
        if (lane == 0) {
          const int n = w.a.nt();
          r->seg[0] = w.a;
          r->seg[1] = w.b;
          r->kind = w.kind;
          r->n[0] = w.kind == RUN_SPLIT ? (n + 1) >> 1 : n;
          r->n[1] = w.kind == RUN_SPLIT ? n >> 1 : w.kind == RUN_PAIR ? w.b.nt() : n;
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(RFULL + 8 * (k % NR));
        if (w.kind == RUN_END) break;
      }
    } else if (warp == 9) {
      // ---------------- loads (the warp as one; one thread issues)
      uint32_t qn = 0, x = 0;   // Q slots used, tiles loaded
      bool stop = false;
      for (uint32_t k = 0;; k++) {
        mbar_wait(RFULL + 8 * (k % NR), (k / NR) & 1, lost, p.err);
        const Run& r = runs[k % NR];
        const int kind = r.kind, n0 = r.n[0], n1 = kind == RUN_WIDE ? 0 : r.n[1];
        if (gave_up(lost) || kind == RUN_END) break;
        if (kind != RUN_NONE) {
          const bool split = kind == RUN_SPLIT;
          // the lane's page of two tiles of its stream (lanes 16 to 31: stream 1), now, next and before
          const Seg& g = r.seg[kind == RUN_PAIR ? lane >> 4 : 0];
          const int32_t* pages = a.b.table + (int64_t)g.job.row * a.b.table_stride;
          const int p0 = g.job.key0 / 16 + (lane & 7), pend = (g.job.kend + 15) / 16;
          auto fetch = [&](int pair) {
            const int i = 2 * pair + ((lane >> 3) & 1), t = g.t0 + (split ? 2 * i + (lane >> 4) : i);
            const int pg = p0 + t * (TK / 16);
            return t < g.t1 && pg < pend ? pages[pg] : 0;   // (as it is: nothing waits for it here)
          };
          int now = r.page[lane], ahead = fetch(1), old = 0, at = 0;
          for (int u = 1; u < 4 * (max(n0, n1) + 1); u++) {
            // V of tile u / 4 - 1, K of the tile after it
            const int s = (u >> 1) & 1, i = (u >> 2) - 1 + (u & 1);
            const bool v = !(u & 1);
            if (i < 0 || i >= (s ? n1 : n0)) continue;
            if ((i >> 1) > at) {
              at++;
              old = now;
              now = ahead < 0 || ahead >= a.c.n_blocks ? (int)a.c.n_blocks : ahead;   // (reads as zeros)
              ahead = fetch(at + 1);
            }
            const int from = (i >> 1) == at ? now : old;
            const Seg& gs = r.seg[kind == RUN_PAIR ? s : 0];
            const int t = gs.t0 + (split ? 2 * i + s : i);
            const int cnt = min(TK / 16, (gs.job.kend + 15 - gs.job.key0) / 16 - t * (TK / 16));
            const uint32_t st = x % L::NST, use = x / L::NST;
            const uint32_t bar = FULL + 8 * st, dst = base + L::RING + st * L::STAGE;
            int id[TK / 16];
#pragma unroll
            for (int q = 0; q < TK / 16; q++) id[q] = __shfl_sync(~0u, from, s * 16 + (i & 1) * 8 + q);
            if (use > 0) {
              mbar_wait(EMPTY + 8 * st, (use - 1) & 1, lost, p.err);
              if ((stop = gave_up(lost))) break;
            }
            const int head = gs.head;
            if (elect_one()) {
              const CUtensorMap* m = v ? &mv : &mk;
              mbar_expect(bar, cnt * 16 * D * 2);
#pragma unroll
              for (int q = 0; q < TK / 16; q++)
                if (q < cnt)
#pragma unroll
                  for (int hf = 0; hf < D / 64; hf++)
                    tma_4d(dst + hf * (TK * 128) + q * 2048, m, hf * 64, 0, head, id[q], bar);
            }
            __syncwarp();
            x++;
            if (u == 1 || (u == 3 && kind == RUN_PAIR)) {   // the rows, after the first K
              for (int o = 0; o < (kind == RUN_WIDE ? 2 : 1); o++) {
                const uint32_t slot = qn & 1, quse = qn >> 1;
                if (quse > 0) {
                  mbar_wait(QEMPTY + 8 * slot, (quse - 1) & 1, lost, p.err);
                  if ((stop = gave_up(lost))) break;
                }
                const bool one = gs.job.ntok == 1;
                const int tok = gs.job.tok0 + o * p.tpt;
                if (elect_one()) {
                  const uint32_t qbar = QFULL + 8 * slot;
                  mbar_expect(qbar, (one ? 1 : p.tpt) * p.ratio * D * 2);
#pragma unroll
                  for (int hf = 0; hf < D / 64; hf++)
                    tma_3d(base + slot * L::QSLOT + hf * (128 * 128), one ? &mq1 : &mq, hf * 64, head * p.ratio, tok, qbar);
                }
                __syncwarp();
                qn++;
              }
              if (stop) break;
            }
          }
        }
        if (stop) break;
        __syncwarp();
        if (lane == 0) mbar_arrive(REMPTY + 8 * (k % NR));
      }
    } else if (warp == 8) {
      // ---------------- products (the warp as one; one thread issues)
      constexpr uint32_t FMT = HALF ? 0u : 1u;
      constexpr uint32_t IQK = (1u << 4) | (FMT << 7) | (FMT << 10) | ((TK / 8) << 17) | ((128 / 16) << 24);
      constexpr uint32_t IPV = (1u << 4) | (FMT << 7) | (FMT << 10) | (1u << 16) | ((D / 8) << 17) | ((128 / 16) << 24);
      const uint64_t dq = smem_desc(base, 16), dk = smem_desc(base + L::RING, 16),
                     dv = smem_desc(base + L::RING, TK * 128);
      uint32_t x = 0, qn = 0, np0 = 0, np1 = 0, done = 0;
      uint32_t kst = 0, vst = 0;   // stages of the last K and V tile
      auto take = [&]() {   // the next load's stage
        const uint32_t st = x % L::NST;
        mbar_wait(FULL + 8 * st, (x / L::NST) & 1, lost, p.err);
        x++;
        return st;
      };
      for (uint32_t k = 0;; k++) {
        mbar_wait(RFULL + 8 * (k % NR), (k / NR) & 1, lost, p.err);
        const int kind = runs[k % NR].kind, n0 = runs[k % NR].n[0], n1 = runs[k % NR].n[1];
        if (gave_up(lost)) break;
        if (lane == 0) mbar_arrive(REMPTY + 8 * (k % NR));
        if (kind == RUN_END) break;
        if (kind == RUN_NONE) continue;
        const bool wide = kind == RUN_WIDE, split = kind == RUN_SPLIT;
        for (int u = 0; u < 2 * (max(n0, n1) + 1); u++) {
          const uint32_t s = u & 1;
          const int i = (u >> 1) - 1, n = s ? n1 : n0;
          if (i >= 0 && i < n) {   // O += P V of tile i
            if (!wide || s == 0) vst = take();
            if (i == 0 && done > 0) mbar_wait(OEMPTY + 8 * s, (done - 1) & 1, lost, p.err);
            mbar_wait(PFULL + 8 * s, (s ? np1 : np0) & 1, lost, p.err);
            np0 += s == 0;
            np1 += s == 1;
            tc_after();
            const uint64_t va = dv + vst * (L::STAGE >> 4);
            const uint32_t more = i > 0;   // O holds something
            if (elect_one()) {
#pragma unroll
              for (int q = 0; q < TK / 16; q++)
                mma_ts(tmem + 256 + s * D, tmem + s * 128 + q * 8, va + q * (2048 >> 4), IPV, q > 0 ? 1u : more);
              if (!wide || s == 1) mma_commit(EMPTY + 8 * vst);
              if (i + 1 == n) mma_commit(OFULL + 8 * s);
            }
            __syncwarp();
          }
          if (i + 1 < n) {   // S = Q K^T of tile i + 1
            if (!wide || s == 0) kst = take();
            const uint32_t qi = qn + (split ? 0 : s), slot = qi & 1;
            if (i < 0 && !(split && s)) mbar_wait(QFULL + 8 * slot, (qi >> 1) & 1, lost, p.err);
            tc_after();
            const uint64_t qa = dq + slot * (L::QSLOT >> 4), ka = dk + kst * (L::STAGE >> 4);
            const bool end = split ? 2 * (i + 1) + (int)s + 1 == n0 + n1 : i + 2 == n;
            if (elect_one()) {
#pragma unroll
              for (int q = 0; q < D / 16; q++) {
                const uint32_t o = ((q >> 2) * (128 * 128) + (q & 3) * 32) >> 4;
                mma_ss(tmem + s * 128, qa + o, ka + o, IQK, q > 0);
              }
              mma_commit(SFULL + 8 * s);
              if (!wide || s == 1) mma_commit(EMPTY + 8 * kst);
              if (end) mma_commit(QEMPTY + 8 * slot);
            }
            __syncwarp();
          }
        }
        qn += split ? 1 : 2;
        done++;
      }
    }
    __syncthreads();   // the streams are done
    if (*lost) drain();
    if (warp == 8) {
      tc_after();
      asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem));
    }
  } else {
    // ---------------- softmax, a thread a row
    asm volatile("setmaxnreg.inc.sync.aligned.u32 208;");
    const int s = warp >> 2, r = tid & 127;
    const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
    const uint32_t ts = tmem + lanes + s * 128;
    const float sl = __fmul_rn(a.scale, 1.4426950408889634f);
    float2* ml = reinterpret_cast<float2*>(sm + L::ML);
    uint32_t ns = 0, nm = 0, no0 = 0, no1 = 0, loads = 0;
    const int tl = r / p.ratio, hl = r - tl * p.ratio;   // the row's token and head in its 128
    const int64_t all = (int64_t)a.b.n_tokens * a.n_heads;
    for (uint32_t k = 0;; k++) {
      mbar_wait(RFULL + 8 * (k % NR), (k / NR) & 1, lost, p.err);
      const Run& run = runs[k % NR];
      const int kind = run.kind;
      if (gave_up(lost) || kind == RUN_END) break;
      const bool wide = kind == RUN_WIDE, split = kind == RUN_SPLIT;
      const Seg& g = run.seg[kind == RUN_PAIR ? s : 0];
      const KvJob& job = g.job;
      const int tok = ((job.flags & JOB_WIDE) && s ? p.tpt : 0) + tl;
      const bool live = tl < p.tpt && tok < job.ntok;
      const int row = job.tok0 + tok, hq = g.head * p.ratio + hl;
      if (kind == RUN_NONE) {
        if (live && (s == 0 || (job.flags & JOB_WIDE))) {
          uint16_t* out = static_cast<uint16_t*>(a.out) + row * a.o_ts + hq * a.o_hs;
          for (int c = 0; c < D; c += 8) *reinterpret_cast<uint4*>(out + c) = make_uint4(0, 0, 0, 0);
          if (a.lse) a.lse[(int64_t)row * a.n_heads + hq] = -INFINITY;
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(REMPTY + 8 * (k % NR));
        continue;
      }
      const int n0 = run.n[0], n1 = run.n[1], n = s ? n1 : n0;
      const bool any = __any_sync(~0u, live);
      int lim = 0;   // keys from key0 on that the row sees
      if (live) {
        if (job.flags & JOB_EVEN) {
          lim = job.kend;
        } else if (job.flags & JOB_PREFIX) {
          int lo = job.row, hi = a.b.n_req;
          while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (a.b.q_start[mid] <= row) lo = mid; else hi = mid;
          }
          const int64_t x = (int64_t)max(a.b.kv_len[lo], 0) - a.b.q_start[lo + 1] + row + 1;
          lim = (int)min((int64_t)job.kend, max(x, (int64_t)0));
        } else {
          lim = (int)min((int64_t)job.kend, (int64_t)job.lim0 + tok);
        }
        lim -= job.key0;
      }
      // keys of a last tile that the job's end cuts
      const int ends = g.t1 == job.nt ? (job.kend - job.key0) & (TK - 1) : 0;
      const int low = __reduce_min_sync(~0u, live ? lim : INT_MAX), high = __reduce_max_sync(~0u, live ? lim : 0);
      float m = live ? -INFINITY : 0.0f, l0 = 0.0f, l1 = 0.0f;
      for (int i = 0; i < n; i++) {
        const int t = split ? 2 * i + s : i;
        mbar_wait(SFULL + 8 * s, ns & 1, lost, p.err);
        ns++;
        tc_after();
        if (any) {
          const int k0 = (g.t0 + t) * TK, left = lim - k0, seen = high - k0;
          const bool first = i == 0;   // O holds nothing yet
          float a0, a1;
          // Twice at most: where some row's weights sum to too much, or it has no m yet, its m moves to the tile's maximum
          // and all weights are taken again (the other rows' come out as they were).  No m would do better than the
          // maximum, so the second pass is not looked at: infinities and NaN in a row end here as in any other.
#pragma unroll 1
          for (int pass = 0; pass < 2; pass++) {
            a0 = a1 = 0.0f;
            // (m from a row's first keys will do)
            if (low >= k0 + TK) {
              uint32_t v[128];
#pragma unroll
              for (int c = 0; c < TK; c += 32) tm_ld32(v + c, ts + c);
#pragma unroll
              for (int c = 0; c < TK; c += 32) tm_wait_ld(v + c);
              if (first && m == -INFINITY) m = max_of32(v);
              const float nm = minus(m, sl);
              row_exp<HALF, 32>(sl, nm, v, a0, a1);
              const bool over = live && (__fadd_rn(a0, a1) > 32768.0f || fabsf(nm) > FAR);
              if (pass || !__any_sync(~0u, over || m == -INFINITY)) {
                tm_st32(ts, v);
                tm_st32(ts + 32, v + 32);
                break;
              }
            } else {
              // the warp's rows see different ends: 32 keys at a time, up to the last that one sees
              uint32_t w[64];
#pragma unroll
              for (int c = 0; c < 64; c++) w[c] = 0;
#pragma unroll
              for (int c = 0; c < TK; c += 32) {
                if (c < seen) {
                  uint32_t v[32];
                  tm_ld32(v, ts + c);
                  tm_wait_ld(v);
                  cut32(v, left - c);
                  if (c == 0 && first && m == -INFINITY) m = max_of32(v);
                  row_exp<HALF, 8>(sl, minus(m, sl), v, a0, a1);
#pragma unroll
                  for (int k = 0; k < 16; k++) w[c / 2 + k] = v[k];
                }
              }
              const bool over = live && (__fadd_rn(a0, a1) > 32768.0f || fabsf(minus(m, sl)) > FAR);
              if (pass || !__any_sync(~0u, over || (m == -INFINITY && left > 0))) {
                tm_st32(ts, w);
                tm_st32(ts + 32, w + 32);
                break;
              }
            }
            // a row's m moves: O and l are scaled
            const bool over = live && (__fadd_rn(a0, a1) > 32768.0f || fabsf(minus(m, sl)) > FAR), none = m == -INFINITY && left > 0;
            const float x = row_max(ts, seen, left);
            const float m2 = over || none ? fmaxf(m, x) : m;
            const bool moved = __any_sync(~0u, m2 > m);
            const float f = m2 > m ? ex2(__fmul_rn(__fsub_rn(m, m2), sl)) : 1.0f;
            if (!first && moved) {
              l0 = __fmul_rn(l0, f);
              l1 = __fmul_rn(l1, f);
#pragma unroll 1
              for (int c = 0; c < D; c += 32) {
                uint32_t o[32];
                tm_ld32(o, tmem + lanes + 256 + s * D + c);
                tm_wait_ld(o);
#pragma unroll
                for (int k = 0; k < 32; k++) o[k] = __float_as_uint(__fmul_rn(__uint_as_float(o[k]), f));
                tm_st32(tmem + lanes + 256 + s * D + c, o);
              }
            }
            m = m2;
            if (__any_sync(~0u, live && fabsf(minus(m, sl)) > FAR)) {
              const float2 y = far_weights<HALF>(ts, seen, left, sl, m);
              a0 = y.x;
              a1 = y.y;
              break;
            }
          }
          l0 = __fadd_rn(l0, a0);
          l1 = __fadd_rn(l1, a1);
          tm_wait_st();
        }
        if (ends && t == g.nt() - 1 && !(wide && s)) {
          // V rows past the keys' end: their weights are 0, but 0 times what lies there may be NaN.
          // (Of a wide job stream 0's product with this tile comes first.)
          const uint32_t x = loads + vplace(s, i, n0, wide ? 0 : n1);
          mbar_wait(FULL + 8 * (x % L::NST), (x / L::NST) & 1, lost, p.err);
          uint4* vt = reinterpret_cast<uint4*>(sm + L::RING + (x % L::NST) * L::STAGE);
#pragma unroll
          for (int hf = 0; hf < D / 64; hf++)
            for (int c = ends * 8 + r; c < TK * 8; c += 128) vt[hf * (TK * 8) + c] = make_uint4(0, 0, 0, 0);
          asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        }
        tc_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(PFULL + 8 * s);
      }
      loads += 2 * (n0 + (wide ? 0 : n1));
      // ---- the rows' results: each stream's own; of a split job both streams', by stream 0's warps
      const bool mine = !split || s == 0;
      float l = __fadd_rn(l0, l1), f1 = 0.0f;
      if (n > 0) mbar_wait(OFULL + 8 * s, (s ? no1 : no0) & 1, lost, p.err);
      if (split && n1 > 0) {
        if (s) {   // (stream 0 is done with the row before, or this product could not have begun)
          ml[r] = make_float2(m, l);
          __syncwarp();
          if (lane == 0) mbar_arrive(MEET);
        } else {
          mbar_wait(MEET, nm++ & 1, lost, p.err);
          mbar_wait(OFULL + 8, no1 & 1, lost, p.err);
          const float2 y = ml[r];
          const float mm = fmaxf(m, y.x);
          const float wx = m == -INFINITY ? 0.0f : ex2(__fmul_rn(__fsub_rn(m, mm), sl));
          f1 = y.x == -INFINITY ? 0.0f : ex2(__fmul_rn(__fsub_rn(y.x, mm), sl));
          l = fmaf(l, wx, __fmul_rn(y.y, f1));
          l0 = wx;
          m = mm;
        }
      }
      no0 += n0 > 0;
      no1 += n1 > 0;
      tc_after();
      if (any && mine) {
        const float inv = l > 0.0f ? __fdiv_rn(1.0f, l) : l == l ? 0.0f : l;
        const float f0 = split && n1 > 0 ? __fmul_rn(l0, inv) : inv;
        const float lse2 = l > 0.0f ? __fadd_rn(__fmul_rn(m, sl), __log2f(l)) : l == l ? -INFINITY : l;
        f1 = __fmul_rn(f1, inv);
        const bool whole = g.t0 == 0 && g.t1 == job.nt;
        const bool direct = whole && (job.flags & JOB_ALONE);
        // a part's row: with the other whole parts of all rows, or with the CTA's cut ones
        uint16_t* out = static_cast<uint16_t*>(a.out) + row * a.o_ts + hq * a.o_hs;
        const int64_t at = whole ? ((job.flags & JOB_PREFIX) ? 0 : all) + (int64_t)row * a.n_heads + hq
                                 : ((int64_t)blockIdx.x * 2 + (g.cut_front ? 0 : 1)) * 256 + (wide ? s * 128 : 0) + r;
        float* part = (whole ? p.home : p.part) + at * D;
        if (live) {
          if (!direct) (whole ? p.home_sum : p.part_sum)[at] = make_float2(l == 0.0f ? -INFINITY : __fmul_rn(m, sl), l);
          else if (a.lse) a.lse[(int64_t)row * a.n_heads + hq] = __fmul_rn(lse2, 0.6931471805599453f);
        }
        const unsigned lives = __ballot_sync(~0u, live);
        if (!split && __popc(lives) > 8) {
          // many rows: 16 at a time, four threads to a row, 64 bytes a store (a thread a row would touch as many
          // lines as there are rows with every store)
          char* const dst = direct ? reinterpret_cast<char*>(out) : reinterpret_cast<char*>(part);
          const int q = lane & 3;
#pragma unroll 1
          for (int h = 0; h < 32; h += 16) {
            const int ra = h + (lane >> 2), rb = ra + 8;
            uint32_t v[D / 2];
#pragma unroll
            for (int c = 0; c < D; c += 32) tm_ld16(v + c / 2, tmem + lanes + ((uint32_t)h << 16) + 256 + s * D + c);
            const float fa = __shfl_sync(~0u, f0, ra), fb = __shfl_sync(~0u, f0, rb);
            char* const da = reinterpret_cast<char*>(__shfl_sync(~0u, reinterpret_cast<unsigned long long>(dst), ra));
            char* const db = reinterpret_cast<char*>(__shfl_sync(~0u, reinterpret_cast<unsigned long long>(dst), rb));
            const bool la = (lives >> ra) & 1, lb = (lives >> rb) & 1;
#pragma unroll
            for (int c = 0; c < D / 2; c += 32) tm_wait_ld(v + c);
#pragma unroll
            for (int c = 0; c < D; c += 32) {
              uint32_t* o = v + c / 2;
#pragma unroll
              for (int k = 0; k < 16; k++) o[k] = __float_as_uint(__fmul_rn(__uint_as_float(o[k]), k & 2 ? fb : fa));
              if (direct) {
                // of each row a thread has two columns of each group; it gets the eight of group q
#pragma unroll
                for (int z = 0; z < 4; z += 2) {
                  uint32_t w[4];
#pragma unroll
                  for (int k = 0; k < 4; k++) w[k] = pack2<HALF>(__uint_as_float(o[4 * k + z]), __uint_as_float(o[4 * k + z + 1]));
#pragma unroll
                  for (int k = 0; k < 4; k += 2) {   // threads 1 apart
                    const uint32_t y = __shfl_xor_sync(~0u, q & 1 ? w[k] : w[k + 1], 1);
                    if (q & 1) w[k] = y; else w[k + 1] = y;
                  }
#pragma unroll
                  for (int k = 0; k < 2; k++) {      // and 2 apart
                    const uint32_t y = __shfl_xor_sync(~0u, q & 2 ? w[k] : w[k + 2], 2);
                    if (q & 2) w[k] = y; else w[k + 2] = y;
                  }
                  if (z ? lb : la) *reinterpret_cast<uint4*>((z ? db : da) + (c + 8 * q) * 2) = make_uint4(w[0], w[1], w[2], w[3]);
                }
              } else {
                // it gets four columns of group k or, the odd ones, of the next
#pragma unroll
                for (int z = 0; z < 4; z += 2)
#pragma unroll
                  for (int k = 0; k < 4; k += 2) {
                    uint32_t* u = o + 4 * k + z;   // u[0], u[1]: group k, u[4], u[5]: the next
                    const uint32_t y0 = __shfl_xor_sync(~0u, q & 1 ? u[0] : u[4], 1), y1 = __shfl_xor_sync(~0u, q & 1 ? u[1] : u[5], 1);
                    const uint4 w = q & 1 ? make_uint4(y0, y1, u[4], u[5]) : make_uint4(u[0], u[1], y0, y1);
                    if (z ? lb : la) *reinterpret_cast<uint4*>((z ? db : da) + (c + 8 * (k + (q & 1)) + 4 * (q >> 1)) * 4) = w;
                  }
              }
            }
          }
        } else {
#pragma unroll 1
        for (int c = 0; c < D; c += 64) {
          uint32_t o[64];
          float y[64];
          const uint32_t to = tmem + lanes + 256 + c;
          tm_ld32(o, to + (split ? 0 : s * D));
          tm_ld32(o + 32, to + (split ? 0 : s * D) + 32);
          tm_wait_ld(o);
          tm_wait_ld(o + 32);
#pragma unroll
          for (int k = 0; k < 64; k += 2) {
            y[k] = __uint_as_float(o[k]);
            y[k + 1] = __uint_as_float(o[k + 1]);
            mul2(y[k], y[k + 1], f0);
          }
          if (split && n1 > 0) {
            tm_ld32(o, to + D);
            tm_ld32(o + 32, to + D + 32);
            tm_wait_ld(o);
            tm_wait_ld(o + 32);
#pragma unroll
            for (int k = 0; k < 64; k++) y[k] = fmaf(__uint_as_float(o[k]), f1, y[k]);
          }
          if (live) {
            if (direct) {
#pragma unroll
              for (int k = 0; k < 64; k += 8)
                *reinterpret_cast<uint4*>(out + c + k) =
                    make_uint4(pack2<HALF>(y[k], y[k + 1]), pack2<HALF>(y[k + 2], y[k + 3]),
                               pack2<HALF>(y[k + 4], y[k + 5]), pack2<HALF>(y[k + 6], y[k + 7]));
            } else {
#pragma unroll
              for (int k = 0; k < 64; k += 4)
                *reinterpret_cast<float4*>(part + c + k) = make_float4(y[k], y[k + 1], y[k + 2], y[k + 3]);
            }
          }
        }
        }
      }
      tc_before();
      __syncwarp();
      if (lane == 0) {
        // (a split job's O of stream 1 is stream 0's to give back)
        if (mine) mbar_arrive(OEMPTY + 8 * s);
        if (split && mine) mbar_arrive(OEMPTY + 8);
        mbar_arrive(REMPTY + 8 * (k % NR));
      }
    }
    __syncthreads();
    if (*lost) drain();
  }
}

// ------------------------------------------------------------------ host

using EncodeFn = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*,
                              const cuuint64_t*, const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave,
                              CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

EncodeFn encode_fn() {
  static const EncodeFn fn = [] {
    void* f = nullptr;
    cudaDriverEntryPointQueryResult q;
    if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &f, 12000, cudaEnableDefault, &q) != cudaSuccess ||
        q != cudaDriverEntryPointSuccess)
      f = nullptr;
    return reinterpret_cast<EncodeFn>(f);
  }();
  return fn;
}

// A map of `rank` axes (sizes, strides of the axes after the first in bytes,
// box) whose boxes are 128-byte rows, swizzled.
bool encode(CUtensorMap* m, bool half, const void* p, int rank, const cuuint64_t* size, const cuuint64_t* stride,
            const cuuint32_t* box) {
  const cuuint32_t one[5] = {1, 1, 1, 1, 1};
  return encode_fn()(m, half ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, rank,
                     const_cast<void*>(p), size, stride, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE,
                     CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                     CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

size_t up(size_t x) { return (x + 255) & ~(size_t)255; }

// The workspace; with ws NULL only its size.
size_t carve(const KvAttendArgs& a, int ctas, unsigned char* ws, KvPlan& p) {
  const size_t n = a.b.n_req, G = a.b.n_groups, D = a.c.head_dim, rows = (size_t)a.b.n_tokens * a.n_heads;
  p.ratio = a.n_heads / a.c.n_kv_heads;
  p.tpt = 128 / p.ratio;
  p.ctas = ctas;
  // each request and each group at most one job more than its share of the rows
  p.cap = (int32_t)(n + G + (G ? 2 : 1) * ((size_t)a.b.n_tokens / (2 * p.tpt)) + 1);
  size_t o = 0;
  auto take = [&](auto*& ptr, size_t count) {
    if (ws) ptr = reinterpret_cast<std::remove_reference_t<decltype(ptr)>>(ws + o);
    o = up(o + count * sizeof(*ptr));
  };
  take(p.head, 1);
  take(p.jobs, (size_t)p.cap + 1);
  take(p.shared, G ? (size_t)a.b.n_tokens : 0);
  take(p.gjob, G > PLAN_GROUPS ? G : 0);
  take(p.gsum, G > PLAN_GROUPS ? 4 * G : 0);
  take(p.start, ctas);
  take(p.cut, ctas);
  take(p.part, (size_t)ctas * 2 * 256 * D);
  take(p.part_sum, (size_t)ctas * 2 * 256);
  take(p.home, G ? 2 * rows * D : 0);
  take(p.home_sum, G ? 2 * rows : 0);
  return o;
}

template <int D, bool HALF>
cudaError_t run(const KvAttendArgs& a, const KvPlan& p, const CUtensorMap* m, cudaStream_t st) {
  using L = Lay<D>;
  static_assert(D == 64 || D == 128, "two head sizes");
  auto k = k_kv_attend<D, HALF>;
  cudaError_t e = cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, L::SMEM);
  if (e != cudaSuccess) return e;
  // the kernel's register split (2 x 208 + 88 a thread of each four warps) has to be within what a CTA starts with
  static const int regs = [] {
    cudaFuncAttributes f;
    return cudaFuncGetAttributes(&f, k_kv_attend<D, HALF>) == cudaSuccess ? f.numRegs : 0;
  }();
  if (regs * 3 < 2 * 208 + 88) return cudaErrorInvalidKernelImage;
  e = launch_behind(k, p.ctas, NT_ATT, L::SMEM, st, m[0], m[1], m[2], m[3], a, p);
  if (e != cudaSuccess || p.whole) return e;
  // a warp a row, no more than the GPU holds at once
  const int64_t rows = std::min<int64_t>((int64_t)p.ctas * 256, (int64_t)a.b.n_tokens * a.n_heads) +
                       (a.b.n_groups ? (int64_t)a.b.n_tokens * a.n_heads : 0);
  // Few rows: eight parts of each on their way at once (111 registers, 16 rows an SM); many: four (75 registers, 24 rows).
  // Eight and four, us a call in a replayed graph, when it was chosen: 256 tokens x heads behind a prefix 17.9 and 18.2, 924 23.6 and 24.1,
  // 4096 85.1 and 84.4, 8192 411 and 408, 6 prompts' 200 000 263 and 256
  auto join = rows < (int64_t)p.ctas * 48 ? k_kv_join<D, HALF, 8> : k_kv_join<D, HALF, 4>;
  return launch_behind(join, (unsigned)std::min<int64_t>((rows + 7) / 8, (int64_t)p.ctas * 8), 256, 0, st, a, p);
}

}  // namespace

size_t kv_attend_bytes(const KvAttendArgs& a, int sms) {
  KvPlan p = {};
  return carve(a, sms, nullptr, p);
}

cudaError_t launch_kv_attend(const KvAttendArgs& a, void* ws, int32_t* err, int sms, cudaStream_t st) {
  if (!encode_fn()) return cudaErrorNotSupported;
  KvPlan p = {};
  carve(a, sms, static_cast<unsigned char*>(ws), p);
  p.err = err;
  const bool half = a.c.dtype == RS_FP16;
  const cuuint64_t D = a.c.head_dim;
  CUtensorMap m[4];
  const cuuint64_t ks[4] = {D, 16, (cuuint64_t)a.c.n_kv_heads, (cuuint64_t)a.c.n_blocks};
  const cuuint64_t kst[3] = {(cuuint64_t)a.c.stride_token * 2, (cuuint64_t)a.c.stride_head * 2, (cuuint64_t)a.c.stride_block * 2};
  const cuuint32_t kbox[4] = {64, 16, 1, 1};
  const cuuint64_t qs[3] = {D, (cuuint64_t)a.n_heads, (cuuint64_t)a.b.n_tokens};
  const cuuint64_t qst[2] = {(cuuint64_t)a.q_hs * 2, (cuuint64_t)a.q_ts * 2};
  const cuuint32_t qbox[3] = {64, (cuuint32_t)p.ratio, (cuuint32_t)p.tpt}, qbox1[3] = {64, (cuuint32_t)p.ratio, 1};
  if (!encode(&m[0], half, a.c.k, 4, ks, kst, kbox) || !encode(&m[1], half, a.c.v, 4, ks, kst, kbox) ||
      !encode(&m[2], half, a.q, 3, qs, qst, qbox) || !encode(&m[3], half, a.q, 3, qs, qst, qbox1))
    return cudaErrorInvalidValue;
  // Without prefixes to join and with tables of at most 64 blocks (eight tiles, four a stream of a CTA) no job is cut and
  // nothing is left to join.  Whole and cut, us a call in a replayed graph, 32 heads on 8: one token over 255 keys 9.1 and
  // 10.3, over 1023 12.5 and 14.2, over 1535 14.7 and 14.4; 64 tokens over 511 27.1 and 33.4, over 1023 43.3 and 46.7
  p.whole = a.b.n_groups == 0 && a.b.max_blocks <= 64;
  // up to PLAN_JOBS jobs every CTA finds its share by itself, in the time that a kernel before it and its start would
  // take; more are one CTA's work for all
  p.planned = p.cap > PLAN_JOBS || a.b.n_groups > PLAN_GROUPS ||
              (int64_t)p.cap * ((a.b.max_blocks / (TK / 16) + 1) * W_WIDE + OV_WIDE) > INT_MAX;   // (costs in 32 bits)
  if (p.planned) {
    cudaError_t e = cudaFuncSetAttribute(k_kv_plan, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)sizeof(PlanSmem));
    if (e != cudaSuccess) return e;
    e = launch_behind(k_kv_plan, 1, NT_PLAN, sizeof(PlanSmem), st, a.b, p, (int)a.c.n_kv_heads);
    if (e != cudaSuccess) return e;
  }
  if (D == 128) return half ? run<128, true>(a, p, m, st) : run<128, false>(a, p, m, st);
  return half ? run<64, true>(a, p, m, st) : run<64, false>(a, p, m, st);
}

}  // namespace rs
