// The plan of a kv_attend4 step: jobs, and how workers share them.
//
// A job is some rows (a request's tokens x the heads of a kv head, numbered token by
// token) by a range of its keys, for each kv head alike: a job and a head are an item.
// Rows that share a group's prefix may have two: the group's prefix for all the group's
// rows, and each request's own keys behind it.  Jobs of few rows are warps' work, jobs of
// many rows CTAs' (two lists, "kinds").  A warp's item is a job and a chunk of kv heads, each
// the work of a warp of its own.  Of each kind the items' costs are numbered
// through, and worker w takes the numbers from w * per to (w + 1) * per: whole items, and
// pieces of those that a share's end cuts, which leave parts.
#pragma once

#include <climits>
#include <cstdint>

#include "kv4_device.cuh"
#include "rs_internal.h"

namespace rs {
namespace kv4 {

constexpr int PAGE = 16;        // keys of a block
constexpr int UNIT = 32;        // keys of a unit of a warp's job
constexpr int FEW = 16;         // rows of a warp's job
constexpr int MANY = 256;       // rows of a CTA's job
constexpr int TILE = 128;       // keys of a CTA's tile

constexpr int JOB_ALONE = 1;    // no other job has its rows
constexpr int JOB_EVEN = 2;     // every row sees all its keys
constexpr int JOB_PREFIX = 4;   // a group's prefix

struct __align__(16) Job {
  int32_t tok0;         // token of row 0 of the request or group
  int32_t row0, nrows;  // its rows, from there
  int32_t trow;         // table row
  int32_t key0, kend;   // keys (key0 a multiple of 16)
  int32_t lim0;         // keys that the first token of the request sees; the next see one more each
  int32_t flags;
  int32_t nt;           // units, or tiles, of its keys
  int32_t reserved0;
  int64_t cost;         // of the jobs before, for one kv head
};

// Whether CTAs have an item each and no more, where there are no more items than CTAs: cutting would shorten the longest
// from `longest` tiles to items / workers of them, and cost about WHOLE tiles (a run's own time, and the join).  Whole and
// cut, us a call: 40 items of 4 tiles 25.4 and 30.7, 56 of up to 6 52.6 and 54.3, 112 of up to 15 52.7 and 58.4; but 40
// of 11 tiles 40.2 and 35.7, 64 of 16 107.4 and 100.7.
constexpr int WHOLE = 5;
__device__ __forceinline__ bool whole_items(int64_t items, int workers, int longest) {
  return items <= workers && longest * (workers - items) <= (int64_t)WHOLE * workers;
}

struct Head {
  int64_t total[2];     // cost of all items of a kind
  int64_t per[2];       // of a worker's share
  int32_t jobs[2];
  int32_t q_begin;      // rows before this belong to no request,
  int32_t q_end;        // and rows from here on
  int32_t room;         // the jobs had room
  int32_t whole;        // a CTA has an item and no more (short ones: no cuts, nothing to join)
  int32_t ctas;         // of the warps' kernel that have work
  int32_t reserved0;
};

constexpr int TOK_ALONE = 0, TOK_BOTH = 1, TOK_PREFIX = 2;   // a token's rows have an own job, both, a prefix job
constexpr int KIND = 1 << 30;

struct __align__(16) Cut {
  int32_t first, last;  // workers that have units of it, in order
  int32_t ratio0;       // its row 0's place in its token (row0 % ratio)
  int32_t tok0;         // its row 0's token
};

struct Plan {
  Head* head;
  Job* jobs[2];         // [cap]: of warps, of CTAs
  int32_t* tok;         // [n_tokens], with groups: TOK_*
  // Where the parts of a row's (token, head) prefix job (0) and own job (1) are: -1 in one
  // place (of a row without a prefix job: in out already), else the worker that has its
  // item's first unit, a CTA plus KIND.  Written by that worker, of rows that have such a job.
  int32_t* where[2];    // [tokens x heads]
  Cut* cut[2];          // [workers]: the item whose first unit the worker has and that its share's end cuts
  int4* group;          // [n_groups]: first prefix job (or -1), first token, prefix in keys
  float* part[2];       // [workers][heads of a chunk][2][rows][D]: rows of pieces of items that are cut: with the first unit (0), without (1)
  float4* part_sum[2];  // [workers][heads of a chunk][2][rows]: m, l, log2(e) * scale in the row's units
  float* home;          // [2][tokens x heads][D]: whole items of rows that have two
  float4* home_sum;
  int32_t* err;         // host memory: set when a wait ran out
  int32_t cap[2];
  int32_t workers[2];
  int32_t ratio;        // heads of a kv head
  uint32_t ratio_inv;   // 2^32 / ratio, rounded down (2^32 - 1 for 1)
  int32_t tiny;         // a step whose CTAs make the plan for themselves
  int32_t beside;       // the warps' kernel runs beside the tiles' kernel and ends behind it
  int32_t few_max;      // requests or groups of up to so many rows are warps' work
  int32_t heads;        // kv heads
  int32_t chunk, chunks;   // kv heads that a worker of warps takes together, and how often
};

__device__ __forceinline__ int64_t quotient(int64_t a, int64_t b) {
  return ((a | b) >> 32) == 0 ? (int64_t)((uint32_t)a / (uint32_t)b) : a / b;
}
// Row x of a request: its token, and its head of the kv head's.  (The product is too small by at most one.)
__device__ __forceinline__ int token_of(const Plan& p, int x, int& hl) {
  int q = (int)__umulhi((uint32_t)x, p.ratio_inv);
  hl = x - q * p.ratio;
  if (hl >= p.ratio) {
    hl -= p.ratio;
    q++;
  }
  return q;
}

// The first row of a piece's part: of a worker's piece with (later: without) the item's first unit.
__device__ __forceinline__ int64_t part_row(const Plan& p, int kind, int worker, int head, bool later) {
  const int64_t at = kind ? worker : (int64_t)worker * p.chunk + head % p.chunk;
  return (at * 2 + later) * (kind ? MANY : FEW);
}

// Costs.  A unit of a warp's job takes 8 with up to 8 rows, 13 with up to 16; a job as much
// as a unit more.  A tile of a CTA's job takes 3 with up to 128 rows, 5 with more; a job
// as much as four tiles more.
__host__ __device__ __forceinline__ int unit_cost(int kind, int nrows) { return kind ? nrows > 128 ? 5 : 3 : nrows > 8 ? 13 : 8; }
__host__ __device__ __forceinline__ int own_cost(int kind) { return kind ? 20 : 8; }
__host__ __device__ __forceinline__ int job_cost(int kind, int nt, int nrows) {
  return nt > 0 ? nt * unit_cost(kind, nrows) + own_cost(kind) : 0;
}
__host__ __device__ __forceinline__ int rows_of(int kind) { return kind ? MANY : FEW; }
__host__ __device__ __forceinline__ int keys_of(int kind) { return kind ? TILE : UNIT; }

// The first unit that starts at cost `off` of an item or after it.
__device__ __forceinline__ int unit_at(int kind, int off, int nt, int nrows) {
  off = max(off - own_cost(kind), 0);
  const int u = kind ? nrows > 128 ? (off + 4) / 5 : (off + 2) / 3 : nrows > 8 ? (off + 12) / 13 : (off + 7) / 8;
  return min(u, nt);
}

// Units of an item (from u0 on, of `cost`) that worker w has; none: false.
__device__ __forceinline__ bool segment(int kind, int64_t u0, int cost, int nt, int nrows, int64_t per, int64_t w, int& t0, int& t1) {
  const int64_t lo = max(w * per, u0) - u0, hi = min((w + 1) * per, u0 + cost) - u0;
  if (lo >= hi) return false;
  t0 = unit_at(kind, (int)lo, nt, nrows);
  t1 = unit_at(kind, (int)hi, nt, nrows);
  return t1 > t0;
}

static_assert(sizeof(int) == 4, "an item's cost is below 2^31: at most 2^23 units of 13, or 2^21 of 5");

// By a whole warp: the last of n jobs whose items start at or before u (jobs[0].cost is 0; 32 of them a step).
__device__ __forceinline__ int job_at(const Job* jobs, int n, int heads, int64_t u, int lane) {
  int lo = 0, len = n;   // in [lo, lo + len)
  while (len > 1) {
    const int step = (len + 31) / 32, at = lo + lane * step;
    const bool before = lane * step < len && jobs[min(at, n - 1)].cost * heads <= u;
    const int last = 31 - __clz(__ballot_sync(~0u, before) | 1u);
    lo += last * step;
    len = min(step, len - last * step);
  }
  return lo;
}

__device__ __forceinline__ Job load_job(const Job* p) {
  Job j;
  const int4 *s = reinterpret_cast<const int4*>(p);
  int4* d = reinterpret_cast<int4*>(&j);
#pragma unroll
  for (int i = 0; i < 3; i++) d[i] = s[i];
  return j;
}
static_assert(sizeof(Job) == 48, "three loads");

// A worker's walk over its items.
struct Walk {
  const Job* jobs;
  int kind, heads;
  int64_t at, end;      // numbers left
  int j, h;             // the item that has number `at`
  int64_t u0;           // its first number
  Job job;              // job j
  int cost;             // of one item of it
  int whole;            // the numbers are the items'

  __device__ Walk(const Job* jobs_, const Head& hd, int kind_, int heads_, int64_t w, int lane) {
    kind = kind_;
    heads = heads_;
    jobs = jobs_;
    whole = kind && hd.whole;
    if (whole) {
      at = w;
      end = w < (int64_t)hd.jobs[kind] * heads ? w + 1 : w;
      if (at >= end) return;
      j = (int)w / heads;
      h = (int)w - j * heads;
      job = load_job(jobs + j);
      return;
    }
    at = w * hd.per[kind];
    end = min(at + hd.per[kind], hd.total[kind]);
    if (at >= end) return;
    j = job_at(jobs, hd.jobs[kind], heads, at, lane);
    job = load_job(jobs + j);
    cost = job_cost(kind, job.nt, job.nrows);
    h = cost > 0 ? (int)quotient(at - job.cost * heads, cost) : 0;
    u0 = job.cost * heads + (int64_t)h * cost;
  }
  // The last worker that has units of the last next()'s item.
  __device__ int last_worker(int64_t per) const {
    const int64_t b = quotient(u0 + cost - 1, per);
    int x, y;
    return (int)(segment(kind, u0, cost, job.nt, job.nrows, per, b, x, y) ? b : b - 1);
  }
  // The next item's units t0 .. t1 - 1 (of `job`, head or chunk `head`).
  __device__ bool next(int& head, int& t0, int& t1) {
    if (whole) {
      const bool more = at < end;
      at = end;
      head = h;
      t0 = 0;
      t1 = job.nt;
      return more && t1 > 0;
    }
    while (at < end) {
      while (u0 + cost <= at) {   // (jobs without cost are passed over)
        if (cost > 0 && ++h < heads) {
          u0 += cost;
          continue;
        }
        u0 += cost;
        h = 0;
        job = load_job(jobs + ++j);
        cost = job_cost(kind, job.nt, job.nrows);
      }
      const int64_t to = min(end, u0 + cost);
      t0 = unit_at(kind, (int)(at - u0), job.nt, job.nrows);
      t1 = unit_at(kind, (int)(to - u0), job.nt, job.nrows);
      head = h;
      at = to;
      if (t1 > t0) return true;
    }
    return false;
  }
};

// ------------------------------------------------------------------ what the kernels that run jobs share

constexpr float BIAS = 3.0f;           // of a weight's exponent
constexpr float HEAVY = 32768.0f;      // a weight past which a row's reference moves
constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;

// The power of two that brings a bf16 row's largest magnitude to 2^13 .. 2^14 (1 for a row of zeros), and its inverse.
__device__ __forceinline__ float row_power(float most, float& inverse) {
  const int e = most > 0.0f ? min(max(13 - ((int)(__float_as_uint(most) >> 23) - 127), -126), 126) : 0;
  inverse = __uint_as_float((uint32_t)(127 - e) << 23);
  return __uint_as_float((uint32_t)(127 + e) << 23);
}

// A result's factor, and the log of a row's weights' sum.
__device__ __forceinline__ float inverse_of(float v_unit, float l) { return l > 0.0f ? __fdiv_rn(v_unit, l) : l == l ? 0.0f : l; }
__device__ __forceinline__ float log_sum(float m, float l, float sl) {
  return l > 0.0f ? __fmul_rn(__fadd_rn(__fmul_rn(m, sl), __fsub_rn(__log2f(l), BIAS)), LN2) : l == l ? -INFINITY : l;
}

// What a row's scores are multiplied by, in powers of two (never 0: a hidden score is -inf).  The row's power comes first:
// a small scale and a large q, or the other way round, meet before bits can be lost.  Past the largest number it ends
// there: scores are 2^-34 apart or equal, so any two that differ are as far apart as weights tell, and equal ones stay equal.
__device__ __forceinline__ float row_factor(const KvAttend4Args& a, float inverse) {
  constexpr float MOST = 3.402823466e38f;
  const float f = fminf(__fmul_rn(__fmul_rn(a.scale, inverse), LOG2E), MOST);
  return fminf(fmaxf(__fmul_rn(f, a.c.k_unit), 1.17549435e-38f), MOST);
}

// Keys that token `tok` (of the step) with row's place `in` in its job's request sees of a job, from key 0 on.
__device__ __forceinline__ int limit_of(const rs_kv_batch& b, const Job& j, int tok, int in) {
  if (j.flags & JOB_EVEN) return j.kend;
  if (j.flags & JOB_PREFIX) {
    int lo = j.trow, hi = b.n_req;   // the token's request
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (b.q_start[mid] <= tok) lo = mid; else hi = mid;
    }
    const int64_t x = (int64_t)max(b.kv_len[lo], 0) - b.q_start[lo + 1] + tok + 1;
    return (int)min((int64_t)j.kend, max(x, (int64_t)0));
  }
  return (int)min((int64_t)j.kend, max((int64_t)j.lim0 + in, (int64_t)0));
}

// Leaves for the join where the parts of the walk's item are, of which worker w has the units up to t1; by `count` threads.
__device__ __forceinline__ void tell(const KvAttend4Args& a, const Plan& p, const Walk& walk, int64_t per, int w, int head, int t1, int thread, int count) {
  const Job& j = walk.job;
  const int kind = walk.kind;
  const bool cut = t1 < j.nt;
  int hl0;
  const int in = token_of(p, j.row0, hl0);
  if (cut && thread == 0) (kind ? p.cut[1] : p.cut[0])[w] = Cut{w, walk.last_worker(per), hl0, j.tok0 + in};
  int32_t* const to = (j.flags & JOB_PREFIX) ? p.where[0] : p.where[1];
  for (int r = thread; r < j.nrows; r += count) {
    int hl;
    const int tok = j.tok0 + token_of(p, j.row0 + r, hl);
    to[(int64_t)tok * a.n_heads + head * p.ratio + hl] = cut ? w | (kind ? KIND : 0) : -1;
  }
}

template <int BYTES>
__device__ __forceinline__ void copy_async(uint32_t dst, const void* src, bool there) {   // (else zeros)
  const uint32_t n = there ? BYTES : 0;
  if constexpr (BYTES == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(n) : "memory");
  else asm volatile("cp.async.ca.shared.global [%0], [%1], %3, %2;" ::"r"(dst), "l"(src), "r"(n), "n"(BYTES) : "memory");
}
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

// The tiles' kernel, for the jobs of CTAs.
cudaError_t launch_tiles(const KvAttend4Args& a, const Plan& p, int sms, cudaStream_t st);

}  // namespace kv4
}  // namespace rs
