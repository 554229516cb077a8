// Causal attention over a paged KV cache (kv_attend): k_kv_plan cuts the step
// into jobs, k_kv_attend runs them on the tensor cores, k_kv_join joins parts.
//
// Mathematics.  A row (token, head) needs o = sum_j p_j v_j / sum_j p_j over
// the keys j below its limit, p_j = exp(scale s_j), s = q K^T.  Over any part
// of the keys the triple (m, l, o), m a bound of the scores, l = sum exp(s - m),
// o = sum exp(s - m) v, is enough: parts join with weights exp(m_part - m).  So
// a job walks its keys once, 128 at a time, and the keys of a row may be cut
// anywhere: between a prefix shared by a group (a job whose rows are all the
// group's tokens) and the requests' own keys, and between CTAs.
//
// A job is up to 2 * 128 rows x one kv head x a range of keys.  Rows are
// tokens x the heads of the kv head (so the K and V of a head are read once for
// all of them).  The jobs' tiles are numbered through, and CTA c takes an equal
// share of the numbers (one CTA an SM): whole jobs write out directly, jobs
// cut by a share's end leave parts.
#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <algorithm>
#include <climits>

#include "rs_internal.h"

namespace rs {

namespace {

constexpr int TK = 128;        // keys of a tile
// Costs: a tile of a job of at most 128 rows, one of a larger job, and a job's
// own (its rows' loads and stores).
constexpr int W_NARROW = 2, W_WIDE = 3, OV = 2;
constexpr int NT_PLAN = 1024;
constexpr int NT_ATT = 384;
constexpr int PLAN_GROUPS = 1024;   // groups whose sums are kept in shared memory
constexpr int PLAN_JOBS = 4096;     // jobs whose costs are

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
};

struct KvHead {
  int64_t total, per;   // cost of all jobs and heads, of one CTA
  int32_t jobs, prefix_jobs;
};

struct KvStart {
  int32_t job, head, off, reserved0;   // where a CTA's share begins
};

// Jobs of a request's rows.
struct KvReq {
  int32_t job0;    // its first own job
};

struct KvPlan {
  KvHead* head;
  KvJob* jobs;          // [cap + 1]
  int64_t* cost;        // [cap + 1] cost of the jobs before, for one kv head
  KvReq* req;           // [n_req]
  int32_t* gjob;        // [n_groups] first prefix job, -1: not shared
  unsigned long long* gsum;   // [4 n_groups] (more than PLAN_GROUPS groups)
  KvStart* start;       // [ctas]
  float* part;          // [ctas][2][256][D] cut jobs' rows: of the first cut job (0), of the last (1)
  float* part_lse;      // [ctas][2][256]
  float* home;          // [2][rows][D] rows with a prefix job and an own one, each whole
  float* home_lse;      // [2][rows]
  int32_t* err;         // host memory: set when a wait ran out
  int32_t cap;          // jobs at most
  int32_t ctas;
  int32_t tpt;          // tokens of 128 rows
  int32_t ratio;        // heads of a kv head
};

namespace {

// ------------------------------------------------------------------ the plan

__device__ __forceinline__ int clampi(int64_t x, int lo, int hi) {
  return (int)(x < lo ? lo : x > hi ? hi : x);
}

// Exclusive block sum of x; *total = the sum over the block.
__device__ int64_t block_scan(int64_t x, int64_t* sm, int64_t* total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int64_t s = x;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int64_t y = __shfl_up_sync(~0u, s, o);
    if (lane >= o) s += y;
  }
  __syncthreads();   // (sm may still be read from the scan before)
  if (lane == 31) sm[warp] = s;
  __syncthreads();
  int64_t w = lane < NT_PLAN / 32 ? sm[lane] : 0, ws = w;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int64_t y = __shfl_up_sync(~0u, ws, o);
    if (lane >= o) ws += y;
  }
  const int64_t before = __shfl_sync(~0u, ws - w, warp);
  *total = __shfl_sync(~0u, ws, 31);
  return before + s - x;
}

struct ReqLens {
  int q0, q, kv;   // first row, rows, context with them
};

__device__ __forceinline__ ReqLens kv_req(const rs_kv_batch& b, int i) {
  ReqLens r;
  r.q0 = clampi(b.q_start[i], 0, b.n_tokens);
  r.q = max(clampi(b.q_start[i + 1], 0, b.n_tokens) - r.q0, 0);
  r.kv = clampi(b.kv_len[i], 0, INT_MAX - 1);
  return r;
}

__device__ __forceinline__ int group_of(const rs_kv_batch& b, int i) {
  if (b.n_groups == 0 || i < b.group_start[0] || i >= b.group_start[b.n_groups]) return -1;
  int lo = 0, hi = b.n_groups;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (b.group_start[mid] <= i) lo = mid; else hi = mid;
  }
  return lo;
}

__device__ __forceinline__ int prefix_keys(const rs_kv_batch& b, int g) {
  return (int)min((int64_t)(max(b.prefix_len[g], 0) & ~15), (int64_t)b.max_blocks * 16);
}

__device__ __forceinline__ int tiles(int keys) { return keys > 0 ? (keys + TK - 1) / TK : 0; }

__device__ __forceinline__ int tile_cost(int flags) { return (flags & JOB_WIDE) ? W_WIDE : W_NARROW; }
// (a job without keys whose rows nobody else has writes their zeros)
__device__ __forceinline__ int job_cost(int nt, int flags) {
  return nt > 0 ? nt * tile_cost(flags) + OV : (flags & JOB_ALONE) ? OV : 0;
}
// The first tile that starts at cost `off` of a job or after it.
__device__ __forceinline__ int tile_at(int off, int w) { return off <= OV ? 0 : (off - OV + w - 1) / w; }

// One CTA: whether each group's prefix pays as one job for all its rows, the
// jobs, their costs' sums, and every CTA's start.  Latency is all that counts
// here (a few dependent reads and block sums); sums live in shared memory at
// ordinary sizes.
__global__ void __launch_bounds__(NT_PLAN) k_kv_plan(rs_kv_batch b, KvPlan p, int n_kv_heads) {
  extern __shared__ unsigned long long psm[];
  int64_t* s_cost = reinterpret_cast<int64_t*>(psm);            // [PLAN_JOBS + 1]
  unsigned long long* s_sum = psm + PLAN_JOBS + 1;               // [4 PLAN_GROUPS]
  __shared__ int64_t s_scan[NT_PLAN / 32];
  const int tid = threadIdx.x, n = b.n_req, G = b.n_groups;
  const int w2 = 2 * p.tpt;
  unsigned long long* sum = G <= PLAN_GROUPS ? s_sum : p.gsum;
  asm volatile("griddepcontrol.launch_dependents;");

  // of each group: its requests' costs without and with a shared prefix, whether
  // some row sees less than the prefix, the longest context
  auto of = [&](int x) { return G <= PLAN_GROUPS ? s_sum[x] : __ldcg(p.gsum + x); };
  for (int x = tid; x < 4 * G; x += NT_PLAN) sum[x] = 0;
  __syncthreads();
  if (G > 0) {
    for (int i = tid; i < n; i += NT_PLAN) {
      const int g = group_of(b, i);
      const ReqLens r = kv_req(b, i);
      if (g < 0 || r.q == 0) continue;
      const int P = prefix_keys(b, g), rt = (r.q + w2 - 1) / w2, seen = r.kv - (r.q >> 1);
      const int t = tiles(seen), ts = tiles(seen - P);
      const int fl = r.q > p.tpt ? JOB_WIDE : 0;
      atomicAdd(&sum[4 * g], (unsigned long long)rt * job_cost(t, fl));
      atomicAdd(&sum[4 * g + 1], (unsigned long long)rt * job_cost(ts, fl));
      if (r.kv - r.q + 1 < P) sum[4 * g + 2] = 1;
      atomicMax(&sum[4 * g + 3], (unsigned long long)r.kv);
    }
    __syncthreads();
  }
  // prefix jobs.  Shared when that costs less: the group's prefix once for every
  // w2 of its tokens, and a quarter of a tile a token for the parts' way
  // through memory (2 parts written and read, 4 D bytes each a row, against
  // 512 D bytes a tile).
  int64_t jobs = 0, total;
  for (int base = 0; base < G; base += NT_PLAN) {
    const int g = base + tid;
    int cnt = 0, t0 = 0, t1 = 0, P = 0, first = 0;
    if (g < G) {
      first = clampi(b.group_start[g], 0, n);
      const int last = clampi(b.group_start[g + 1], 0, n);
      P = prefix_keys(b, g);
      t0 = clampi(b.q_start[first], 0, b.n_tokens);
      t1 = clampi(b.q_start[max(first, last)], 0, b.n_tokens);
      const int rt = t1 > t0 ? (t1 - t0 + w2 - 1) / w2 : 0;
      P = (int)min((unsigned long long)P, of(4 * g + 3));   // (a prefix that nobody has written yet is not read)
      const unsigned long long with = of(4 * g + 1) + (unsigned long long)rt * job_cost(tiles(P), t1 - t0 > p.tpt ? JOB_WIDE : 0) +
                                      (unsigned long long)(max(t1 - t0, 0) >> 1);
      if (P > 0 && first < last && with < of(4 * g)) cnt = rt;
    }
    const int64_t at = jobs + block_scan(cnt, s_scan, &total);
    jobs += total;
    if (g < G) {
      const bool fits = cnt > 0 && at + cnt <= p.cap;
      p.gjob[g] = fits ? (int32_t)at : -1;
      const bool even = of(4 * g + 2) == 0;
      for (int k = 0; k < cnt && at + k < p.cap; k++) {
        KvJob j = {};
        if (!fits) {   // (starts that decrease: no work)
          p.jobs[at + k] = j;
          continue;
        }
        j.tok0 = t0 + k * w2;
        j.ntok = min(w2, t1 - j.tok0);
        j.row = first;
        j.key0 = 0;
        j.kend = P;
        j.nt = tiles(P);
        j.lim0 = P;
        j.flags = JOB_PREFIX | (even ? JOB_EVEN : 0) | (j.ntok > p.tpt ? JOB_WIDE : 0);
        p.jobs[at + k] = j;
      }
    }
  }
  jobs = min(jobs, (int64_t)p.cap);
  const int prefix_jobs = (int)jobs;
  __syncthreads();   // gjob
  // the requests' own jobs
  for (int base = 0; base < n; base += NT_PLAN) {
    const int i = base + tid;
    ReqLens r{0, 0, 0};
    int key0 = 0, cnt = 0, pj = -1;
    if (i < n) {
      r = kv_req(b, i);
      const int g = group_of(b, i);
      if (g >= 0 && p.gjob[g] >= 0) {
        pj = p.gjob[g];
        key0 = prefix_keys(b, g);
      }
      cnt = (r.q + w2 - 1) / w2;
    }
    const int64_t at = jobs + block_scan(cnt, s_scan, &total);
    jobs += total;
    const bool fits = cnt > 0 && at + cnt <= p.cap;
    if (i < n) p.req[i] = KvReq{fits ? (int32_t)at : -1};
    // a request of one job is its thread's; a longer one is its warp's
    for (int k = 0; !fits && k < cnt && at + k < p.cap; k++) p.jobs[at + k] = KvJob{};   // (as above)
    unsigned todo = __ballot_sync(~0u, fits);
    const unsigned mine = 1u << (tid & 31);
    const unsigned lone = __ballot_sync(~0u, fits && cnt == 1);
    auto put = [&](int64_t at, int k, int i, int q0, int q, int kv, int key0, int pj) {
      KvJob j;
      const int a = k * w2, e = min(a + w2, q);
      j.tok0 = q0 + a;
      j.ntok = e - a;
      j.row = i;
      j.key0 = key0;
      j.kend = clampi((int64_t)kv - q + e, 0, (int)min((int64_t)b.max_blocks * 16, (int64_t)INT_MAX - 256));
      j.nt = tiles(j.kend - key0);
      j.lim0 = kv - q + a + 1;
      j.flags = (pj < 0 ? JOB_ALONE : 0) | (j.ntok > p.tpt ? JOB_WIDE : 0);
      p.jobs[at + k] = j;
    };
    if (lone & mine) put(at, 0, i, r.q0, r.q, r.kv, key0, pj);
    todo &= ~lone;
    while (todo) {
      const int src = __ffs(todo) - 1;
      todo &= todo - 1;
      const int64_t sat = __shfl_sync(~0u, at, src);
      const int sc = __shfl_sync(~0u, cnt, src), si = __shfl_sync(~0u, i, src);
      const int s0 = __shfl_sync(~0u, r.q0, src), sq = __shfl_sync(~0u, r.q, src);
      const int sk = __shfl_sync(~0u, r.kv, src), s1 = __shfl_sync(~0u, key0, src);
      const int sp = __shfl_sync(~0u, pj, src);
      for (int k = tid & 31; k < sc; k += 32) put(sat, k, si, s0, sq, sk, s1, sp);
    }
  }
  // rows of no request: jobs without keys
  const int q_end = n > 0 ? clampi(b.q_start[n], 0, b.n_tokens) : 0;
  const int pads = (b.n_tokens - q_end + w2 - 1) / w2;
  for (int k = tid; k < pads && jobs + k < p.cap; k += NT_PLAN) {
    KvJob j = {};
    j.tok0 = q_end + k * w2;
    j.ntok = min(w2, b.n_tokens - j.tok0);
    j.flags = JOB_ALONE | (j.ntok > p.tpt ? JOB_WIDE : 0);
    p.jobs[jobs + k] = j;
  }
  const int J = (int)min(jobs + pads, (int64_t)p.cap);
  __syncthreads();   // the jobs
  int64_t cost = 0;
  for (int base = 0; base <= J; base += NT_PLAN) {
    const int j = base + tid;
    int64_t c = 0;
    if (j < J) c = job_cost(p.jobs[j].nt, p.jobs[j].flags);
    const int64_t at = cost + block_scan(c, s_scan, &total);
    cost += total;
    if (j <= J) {
      p.cost[j] = at;
      if (j <= PLAN_JOBS) s_cost[j] = at;
    }
  }
  __syncthreads();
  const int64_t all = cost * n_kv_heads;
  // two tiles at least, one for each stream of a CTA
  const int64_t per = max((all + p.ctas - 1) / p.ctas, (int64_t)(2 * W_NARROW + OV));
  if (tid == 0) *p.head = KvHead{all, per, J, prefix_jobs};
  const int64_t* cs = J <= PLAN_JOBS ? s_cost : p.cost;
  for (int c = tid; c < p.ctas; c += NT_PLAN) {
    const int64_t u = c * per;
    KvStart s{0, 0, 0, 0};
    if (u < all) {
      int lo = 0, hi = J;   // the last job that starts at or before u
      while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (cs[mid] * n_kv_heads <= u) lo = mid; else hi = mid;
      }
      const int64_t cj = cs[lo + 1] - cs[lo], in = u - cs[lo] * n_kv_heads;
      s.job = lo;
      s.head = (int)(in / cj);
      s.off = (int)(in - s.head * cj);
    }
    p.start[c] = s;
  }
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
__device__ __forceinline__ bool mbar_try(uint32_t bar, uint32_t parity) {
  uint32_t ok;
  asm volatile(
      "{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
  return ok != 0;
}
// A wait ends after 2^32 clocks (two seconds) at the latest: then the CTA gives
// up, and every later wait returns at once.
__device__ __noinline__ void mbar_lost(volatile int* lost, int32_t* err) {
  *lost = 1;
  *reinterpret_cast<volatile int32_t*>(err) = 1;
}
__device__ __forceinline__ void mbar_wait(uint32_t bar, uint32_t parity, volatile int* lost, int32_t* err) {
  if (mbar_try(bar, parity)) return;
  const long long from = clock64();
  while (clock64() - from < (1ll << 32)) {
    if (mbar_try(bar, parity)) return;
    if (*lost) return;
  }
  mbar_lost(lost, err);
}

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

// The largest score of a row's tile.
__device__ __forceinline__ float row_max(uint32_t ts, bool cut, int left) {
  uint32_t v[2][32];
  float m = -INFINITY, n = -INFINITY;
  tm_ld32(v[0], ts);
#pragma unroll
  for (int c = 0; c < 4; c++) {
    uint32_t* x = v[c & 1];
    tm_wait_ld(x);
    if (c < 3) tm_ld32(v[(c + 1) & 1], ts + 32 * (c + 1));
    if (cut) cut32(x, left - 32 * c);
#pragma unroll
    for (int k = 0; k < 32; k += 4) {
      m = max3(m, x[k], x[k + 1]);
      n = max3(n, x[k + 2], x[k + 3]);
    }
  }
  return fmaxf(m, n);
}

// The row's weights exp2(sl s + nm), packed into v's first half, and their sums
// (of even and odd keys).
template <bool HALF>
__device__ __forceinline__ void row_exp(uint32_t ts, bool cut, int left, float sl, float nm, uint32_t* v,
                                        float& a0, float& a1) {
  float b0 = 0.0f, b1 = 0.0f;
  a0 = a1 = 0.0f;
#pragma unroll
  for (int c = 0; c < 128; c += 32) tm_ld32(v + c, ts + c);
#pragma unroll
  for (int c = 0; c < 128; c += 32) tm_wait_ld(v + c);
  if (cut) {
#pragma unroll
    for (int c = 0; c < 128; c += 32) cut32(v + c, left - c);
  }
#pragma unroll
  for (int k = 0; k < 128; k += 4) {
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

  __device__ Walk(const KvPlan& p, int n_kv_heads) {
    const KvHead hd = *p.head;
    const int64_t u = (int64_t)blockIdx.x * hd.per;
    jobs = p.jobs;
    heads = n_kv_heads;
    rem = min(hd.per, hd.total - u);
    const KvStart s = p.start[blockIdx.x];
    j = s.job; h = s.head; off = s.off;
    held = false;
    if (rem > 0) ahead = jobs[j];
  }
  __device__ bool pull(Seg& s) {
    while (rem > 0) {
      const int cost = job_cost(ahead.nt, ahead.flags);
      if (cost == 0) {
        ahead = jobs[++j];
        continue;
      }
      const int take = (int)min((int64_t)(cost - off), rem), w = tile_cost(ahead.flags);
      const bool empty = ahead.nt == 0 && off == 0;
      s.t0 = min(tile_at(off, w), ahead.nt);
      s.t1 = min(tile_at(off + take, w), ahead.nt);
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

template <int D>
struct Lay {
  static constexpr int QSLOT = 128 * D * 2;       // bytes of 128 rows
  static constexpr int STAGE = TK * D * 2;        // bytes of a tile of K or V
  static constexpr int NST = D == 128 ? 5 : 12;   // stages: what 227 KB leave beside the rows
  static constexpr int RING = 2 * QSLOT;
  static constexpr int MISC = RING + NST * STAGE;
  // barriers: full[NST], empty[NST], qfull[2], qempty[2], sfull[2], pfull[2], ofull[2], oempty[2], rfull[2], rempty[2], meet
  static constexpr int NBAR = 2 * NST + 17;
  static constexpr int ML = MISC + 384;           // float2 [2][128]
  static constexpr int RUNS = ML + 2048;          // Run [2]
  static constexpr int SMEM = RUNS + 2 * (int)sizeof(Run);
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
// under the other's products.  Warps 0-3 and 4-7 are the streams' softmax, a thread a row; warp 8 issues the products and
// warp 9 the loads.
// TMEM: S of each stream 128 columns (P, 64 columns, overwrites it), O D each.
// The m of a row is the largest score of its first tile and moves only when a
// tile's weights sum to more than 2^15 (each is then below it, in range of
// fp16), which hardly happens: O and l are scaled then.
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
                 RFULL = QFULL + 96, REMPTY = QFULL + 112, MEET = QFULL + 128;
  Run* const runs = reinterpret_cast<Run*>(sm + L::RUNS);
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
      mbar_init(RFULL + 8 * s, 1);
      mbar_init(REMPTY + 8 * s, 10);
    }
    mbar_init(MEET, 8);
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
  asm volatile("griddepcontrol.launch_dependents;");
  asm volatile("griddepcontrol.wait;" ::: "memory");   // the plan

  if (warp >= 8) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 88;");
    if (warp == 10) {
      // ---------------- runs
      Walk w(p, a.c.n_kv_heads);
      for (uint32_t k = 0; !*lost; k++) {
        w.next();
        // the lane's page: stream lane / 16, its tile (lane / 8) % 2
        const int s = lane >> 4, i = (lane >> 3) & 1;
        const Seg& g = w.kind == RUN_PAIR && s ? w.b : w.a;
        const int t = g.t0 + (w.kind == RUN_SPLIT ? 2 * i + s : i), pg = g.job.key0 / 16 + t * (TK / 16) + (lane & 7);
        int id = 0;
        if (w.kind <= RUN_PAIR && t < g.t1 && pg < (g.job.kend + 15) / 16)
          id = a.b.table[(int64_t)g.job.row * a.b.table_stride + pg];
        if (id < 0 || id >= a.c.n_blocks) id = (int)a.c.n_blocks;   // reads as zeros
        if (k >= 2) mbar_wait(REMPTY + 8 * (k & 1), ((k >> 1) - 1) & 1, lost, p.err);
        Run* const r = runs + (k & 1);
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
        if (lane == 0) mbar_arrive(RFULL + 8 * (k & 1));
        if (w.kind == RUN_END) break;
      }
    } else if (warp == 9) {
      // ---------------- loads (the warp as one; one thread issues)
      uint32_t qn = 0, x = 0;   // Q slots used, tiles loaded
      for (uint32_t k = 0; !*lost; k++) {
        mbar_wait(RFULL + 8 * (k & 1), (k >> 1) & 1, lost, p.err);
        const Run& r = runs[k & 1];
        const int kind = r.kind;
        if (kind == RUN_END) break;
        if (kind != RUN_NONE) {
          const int n0 = r.n[0], n1 = kind == RUN_WIDE ? 0 : r.n[1];
          const bool split = kind == RUN_SPLIT;
          // the lane's page of two tiles of its stream (lanes 16 to 31: stream 1), now, next and before
          const Seg& g = r.seg[kind == RUN_PAIR ? lane >> 4 : 0];
          const int32_t* pages = a.b.table + (int64_t)g.job.row * a.b.table_stride;
          const int p0 = g.job.key0 / 16 + (lane & 7), pend = (g.job.kend + 15) / 16;
          auto fetch = [&](int pair) {
            const int i = 2 * pair + ((lane >> 3) & 1), t = g.t0 + (split ? 2 * i + (lane >> 4) : i);
            const int pg = p0 + t * (TK / 16);
            int id = t < g.t1 && pg < pend ? pages[pg] : 0;
            return id < 0 || id >= a.c.n_blocks ? (int)a.c.n_blocks : id;
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
              now = ahead;
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
            if (use > 0) mbar_wait(EMPTY + 8 * st, (use - 1) & 1, lost, p.err);
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
                if (quse > 0) mbar_wait(QEMPTY + 8 * slot, (quse - 1) & 1, lost, p.err);
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
            }
          }
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(REMPTY + 8 * (k & 1));
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
      for (uint32_t k = 0; !*lost; k++) {
        mbar_wait(RFULL + 8 * (k & 1), (k >> 1) & 1, lost, p.err);
        const int kind = runs[k & 1].kind, n0 = runs[k & 1].n[0], n1 = runs[k & 1].n[1];
        __syncwarp();
        if (lane == 0) mbar_arrive(REMPTY + 8 * (k & 1));
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
  } else {
    // ---------------- softmax, a thread a row
    asm volatile("setmaxnreg.inc.sync.aligned.u32 208;");
    const int s = warp >> 2, r = tid & 127;
    const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
    const uint32_t ts = tmem + lanes + s * 128;
    const float sl = __fmul_rn(a.scale, 1.4426950408889634f);
    float2* ml = reinterpret_cast<float2*>(sm + L::ML);
    uint32_t ns = 0, no0 = 0, no1 = 0, loads = 0;
    const int tl = r / p.ratio, hl = r - tl * p.ratio;   // the row's token and head in its 128
    const int64_t all = (int64_t)a.b.n_tokens * a.n_heads;
    uint32_t nm = 0;
    auto meet = [&]() {   // of both streams' warps
      __syncwarp();
      if (lane == 0) mbar_arrive(MEET);
      mbar_wait(MEET, nm++ & 1, lost, p.err);
    };
    for (uint32_t k = 0;; k++) {
      mbar_wait(RFULL + 8 * (k & 1), (k >> 1) & 1, lost, p.err);
      const Run& run = runs[k & 1];
      const int kind = run.kind;
      if (kind == RUN_END || *lost) break;
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
        if (lane == 0) mbar_arrive(REMPTY + 8 * (k & 1));
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
      const int low = __reduce_min_sync(~0u, live ? lim : INT_MAX);
      float m = live ? -INFINITY : 0.0f, l0 = 0.0f, l1 = 0.0f;
      for (int i = 0; i < n; i++) {
        const int t = split ? 2 * i + s : i;
        mbar_wait(SFULL + 8 * s, ns & 1, lost, p.err);
        ns++;
        tc_after();
        if (any) {
          const int k0 = (g.t0 + t) * TK;
          const bool cut = low < k0 + TK;   // (the warp's rows see different ends)
          const int left = lim - k0;
          const bool first = i == 0;   // O holds nothing yet
          if (first) {
            const float x = row_max(ts, cut, left);
            if (live) m = x;
          }
          uint32_t pk[128];
          float a0, a1;
          for (;;) {
            row_exp<HALF>(ts, cut, left, sl, m == -INFINITY ? 0.0f : -__fmul_rn(m, sl), pk, a0, a1);
            const bool over = live && __fadd_rn(a0, a1) > 32768.0f, none = m == -INFINITY && left > 0;
            if (!__any_sync(~0u, over || none)) break;
            const float x = row_max(ts, cut, left);
            const float m2 = over || none ? fmaxf(m, x) : m;
            if (!__any_sync(~0u, m2 != m)) break;   // (an infinity: no larger m)
            const float f = m == m2 ? 1.0f : ex2(__fmul_rn(__fsub_rn(m, m2), sl));
            if (!first) {
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
          }
          tm_st32(ts, pk);
          tm_st32(ts + 32, pk + 32);
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
      // ---- the rows' results: the stream's own, or both streams' joined, half the columns each
      float l = __fadd_rn(l0, l1);
      float f0, f1 = 0.0f, lse2;
      int c0 = 0, c1 = D;
      if (!split) {
        f0 = l > 0.0f ? __fdiv_rn(1.0f, l) : l == l ? 0.0f : l;
        lse2 = l > 0.0f ? __fadd_rn(__fmul_rn(m, sl), __log2f(l)) : l == l ? -INFINITY : l;
        mbar_wait(OFULL + 8 * s, (s ? no1 : no0) & 1, lost, p.err);
      } else {
        ml[s * 128 + r] = make_float2(m, l);
        meet();
        const float2 x = ml[r], y = ml[128 + r];
        const float mm = n1 > 0 ? fmaxf(x.x, y.x) : x.x;
        const float wx = x.x == -INFINITY ? 0.0f : ex2(__fmul_rn(__fsub_rn(x.x, mm), sl));
        const float wy = n1 == 0 || y.x == -INFINITY ? 0.0f : ex2(__fmul_rn(__fsub_rn(y.x, mm), sl));
        l = fmaf(x.y, wx, __fmul_rn(y.y, wy));
        const float inv = l > 0.0f ? __fdiv_rn(1.0f, l) : l == l ? 0.0f : l;
        f0 = __fmul_rn(wx, inv);
        f1 = __fmul_rn(wy, inv);
        lse2 = l > 0.0f ? __fadd_rn(__fmul_rn(mm, sl), __log2f(l)) : l == l ? -INFINITY : l;
        c0 = s * (D / 2);
        c1 = c0 + D / 2;
        mbar_wait(OFULL, no0 & 1, lost, p.err);
        if (n1 > 0) mbar_wait(OFULL + 8, no1 & 1, lost, p.err);
      }
      no0 += n0 > 0;
      no1 += n1 > 0;
      tc_after();
      const bool whole = g.t0 == 0 && g.t1 == job.nt;
      const bool direct = whole && (job.flags & JOB_ALONE);
      if (any) {
        // a part's row: with the other whole parts of all rows, or with the CTA's cut ones
        uint16_t* out = static_cast<uint16_t*>(a.out) + row * a.o_ts + hq * a.o_hs;
        const int64_t at = whole ? ((job.flags & JOB_PREFIX) ? 0 : all) + (int64_t)row * a.n_heads + hq
                                 : ((int64_t)blockIdx.x * 2 + (g.cut_front ? 0 : 1)) * 256 + (wide ? s * 128 : 0) + r;
        float* part = (whole ? p.home : p.part) + at * D;
        if (live && c0 == 0) {
          if (!direct) (whole ? p.home_lse : p.part_lse)[at] = lse2;
          else if (a.lse) a.lse[(int64_t)row * a.n_heads + hq] = __fmul_rn(lse2, 0.6931471805599453f);
        }
#pragma unroll 1
        for (int c = c0; c < c1; c += 32) {
          uint32_t o[32];
          float y[32];
          tm_ld32(o, tmem + lanes + 256 + (split ? 0 : s * D) + c);
          tm_wait_ld(o);
#pragma unroll
          for (int k = 0; k < 32; k++) y[k] = f0 == 0.0f ? 0.0f : __fmul_rn(__uint_as_float(o[k]), f0);
          if (split && n1 > 0) {
            tm_ld32(o, tmem + lanes + 256 + D + c);
            tm_wait_ld(o);
#pragma unroll
            for (int k = 0; k < 32; k++) y[k] = f1 == 0.0f ? y[k] : fmaf(__uint_as_float(o[k]), f1, y[k]);
          }
          if (live) {
            if (direct) {
#pragma unroll
              for (int k = 0; k < 32; k += 8)
                *reinterpret_cast<uint4*>(out + c + k) =
                    make_uint4(pack2<HALF>(y[k], y[k + 1]), pack2<HALF>(y[k + 2], y[k + 3]),
                               pack2<HALF>(y[k + 4], y[k + 5]), pack2<HALF>(y[k + 6], y[k + 7]));
            } else {
#pragma unroll
              for (int k = 0; k < 32; k += 4)
                *reinterpret_cast<float4*>(part + c + k) = make_float4(y[k], y[k + 1], y[k + 2], y[k + 3]);
            }
          }
        }
      }
      tc_before();
      if (split) meet();   // ml and both O are free again
      __syncwarp();
      if (lane == 0) {
        mbar_arrive(OEMPTY + 8 * s);
        mbar_arrive(REMPTY + 8 * (k & 1));
      }
    }
  }
  __syncthreads();
  if (*lost) {   // copies in flight end before the CTA's memory is another's
    const long long t = clock64();
    while (clock64() - t < 20000000ll) {}
  }
  if (warp == 8) {
    tc_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem));
  }
}

// ------------------------------------------------------------------ joining

// The tiles that CTA c has of a job and head of `cost` from u0 on.
__device__ __forceinline__ bool segment(int64_t u0, int cost, int w, int nt, int64_t per, int64_t c, int& t0, int& t1) {
  const int64_t lo = max(c * per, u0) - u0, hi = min((c + 1) * per, u0 + cost) - u0;
  if (lo >= hi) return false;
  t0 = min(tile_at((int)lo, w), nt);
  t1 = min(tile_at((int)hi, w), nt);
  return t1 > t0;
}

// Parts of one row (token, head).
template <int D>
struct Join {
  static constexpr int E = D / 32;
  float m, l, o[E];
  __device__ Join() : m(-INFINITY), l(0.0f) {
#pragma unroll
    for (int e = 0; e < E; e++) o[e] = 0.0f;
  }
  // those of row rr of 256 of job j, head kh
  __device__ void add(const KvPlan& p, const KvHead& hd, int j, const KvJob& job, int kh, int n_kv_heads,
                      int64_t home, int rr, int lane) {
    if (job.nt <= 0) return;
    const int w = tile_cost(job.flags), cost = job_cost(job.nt, job.flags);
    const int64_t u0 = p.cost[j] * n_kv_heads + (int64_t)kh * cost;
    const int c0 = (int)(u0 / hd.per), c1 = min((int)((u0 + cost - 1) / hd.per), p.ctas - 1);
    for (int c = c0; c <= c1; c++) {
      int t0, t1;
      if (!segment(u0, cost, w, job.nt, hd.per, c, t0, t1)) continue;
      const bool whole = t0 == 0 && t1 == job.nt;
      const int64_t at = whole ? home : ((int64_t)c * 2 + (c == c0 ? 1 : 0)) * 256 + rr;
      const float s = (whole ? p.home_lse : p.part_lse)[at];
      const float* src = (whole ? p.home : p.part) + at * D + lane * E;
      float y[E];
#pragma unroll
      for (int e = 0; e < E; e++) y[e] = src[e];
      if (s == -INFINITY) continue;
      const float m2 = fmaxf(m, s), f = m == -INFINITY ? 0.0f : ex2(__fsub_rn(m, m2)), g = ex2(__fsub_rn(s, m2));
      l = fmaf(l, f, g);
#pragma unroll
      for (int e = 0; e < E; e++) o[e] = fmaf(o[e], f, __fmul_rn(g, y[e]));
      m = m2;
    }
  }
  template <bool HALF>
  __device__ void put(const KvAttendArgs& a, int64_t row, int hq, int lane) const {
    const float inv = l == 0.0f ? 0.0f : __fdiv_rn(1.0f, l);
    uint16_t* out = static_cast<uint16_t*>(a.out) + row * a.o_ts + hq * a.o_hs + lane * E;
#pragma unroll
    for (int e = 0; e < E; e += 2)
      *reinterpret_cast<uint32_t*>(out + e) = pack2<HALF>(__fmul_rn(o[e], inv), __fmul_rn(o[e + 1], inv));
    if (a.lse && lane == 0)
      a.lse[row * a.n_heads + hq] = l == 0.0f ? -INFINITY : __fmul_rn(__fadd_rn(m, __log2f(l)), 0.6931471805599453f);
  }
};

// Rows that have parts, a warp a row: those of the jobs that a share's end cut
// (first looked for at each CTA's start), and those of shared groups, which
// have a prefix job and an own one.  The order of the parts is the keys'.
template <int D, bool HALF>
__global__ void __launch_bounds__(128) k_kv_join(const __grid_constant__ KvAttendArgs a,
                                                 const __grid_constant__ KvPlan p) {
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const int lane = threadIdx.x & 31;
  const int w0 = blockIdx.x * 4 + (threadIdx.x >> 5), nw = gridDim.x * 4;
  const KvHead hd = *p.head;
  const int hk = a.c.n_kv_heads, w2 = 2 * p.tpt, n = a.b.n_req;
  for (int x = w0; x < p.ctas * 256; x += nw) {
    const int c = x >> 8, rr = x & 255;   // CTA c's start, a row of the job there
    if (c * hd.per >= hd.total) break;
    const KvStart s = p.start[c];
    if (s.off == 0) continue;
    const KvJob job = p.jobs[s.job];
    if (!(job.flags & JOB_ALONE) || job.nt == 0) continue;
    const int cost = job_cost(job.nt, job.flags), w = tile_cost(job.flags);
    const int64_t u0 = p.cost[s.job] * hk + (int64_t)s.head * cost;
    if (u0 / hd.per != c - 1) continue;   // (cut before: the first cut's)
    int t0, t1;   // whole in the CTA before, or here?
    if (segment(u0, cost, w, job.nt, hd.per, c - 1, t0, t1) ? t1 == job.nt
        : segment(u0, cost, w, job.nt, hd.per, c, t0, t1) && t0 == 0 && t1 == job.nt)
      continue;
    const int half = rr >> 7, r = rr & 127, tl = r / p.ratio, tok = half * p.tpt + tl;
    if (tl >= p.tpt || tok >= job.ntok) continue;
    Join<D> v;
    v.add(p, hd, s.job, job, s.head, hk, 0, rr, lane);
    v.template put<HALF>(a, (int64_t)job.tok0 + tok, s.head * p.ratio + r - tl * p.ratio, lane);
  }
  const int64_t all = (int64_t)a.b.n_tokens * a.n_heads, units = (int64_t)hd.prefix_jobs * w2 * a.n_heads;
  for (int64_t x = w0; x < units; x += nw) {
    const int slot = (int)(x / a.n_heads), hq = (int)(x - (int64_t)slot * a.n_heads);
    const int pj = slot / w2, pt = slot - pj * w2, kh = hq / p.ratio, hl = hq - kh * p.ratio;
    const KvJob pre = p.jobs[pj];
    if (pt >= pre.ntok) continue;
    const int row = pre.tok0 + pt;
    int i = row;   // single tokens: request i has row i
    if (!(row < n && a.b.q_start[row] == row && a.b.q_start[row + 1] == row + 1)) {
      int lo = 0, hi = n;
      while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (a.b.q_start[mid] <= row) lo = mid; else hi = mid;
      }
      i = lo;
    }
    const KvReq r = p.req[i];
    const int q0 = a.b.q_start[i];
    const int64_t home = (int64_t)row * a.n_heads + hq;
    auto at = [&](int tok) { return (tok >= p.tpt ? 128 + (tok - p.tpt) * p.ratio : tok * p.ratio) + hl; };
    Join<D> v;
    v.add(p, hd, pj, pre, kh, hk, home, at(pt), lane);
    if (r.job0 >= 0 && q0 >= 0 && row >= q0) {
      const int j = min(r.job0 + (row - q0) / w2, hd.jobs - 1);
      const KvJob own = p.jobs[j];
      if (row >= own.tok0 && row - own.tok0 < own.ntok) v.add(p, hd, j, own, kh, hk, all + home, at(row - own.tok0), lane);
    }
    v.template put<HALF>(a, row, hq, lane);
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

template <class... P, class... A>
cudaError_t launch_after(void (*k)(P...), unsigned grid, int threads, size_t smem, cudaStream_t st, A&&... args) {
  cudaLaunchConfig_t c = {};
  c.gridDim = dim3(grid);
  c.blockDim = dim3(threads);
  c.dynamicSmemBytes = smem;
  c.stream = st;
  cudaLaunchAttribute at;
  at.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at.val.programmaticStreamSerializationAllowed = 1;
  c.attrs = &at;
  c.numAttrs = 1;
  return cudaLaunchKernelEx(&c, k, std::forward<A>(args)...);
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
  take(p.cost, (size_t)p.cap + 1);
  take(p.req, n);
  take(p.gjob, G);
  take(p.gsum, G > PLAN_GROUPS ? 4 * G : 0);
  take(p.start, ctas);
  take(p.part, (size_t)ctas * 2 * 256 * D);
  take(p.part_lse, (size_t)ctas * 2 * 256);
  take(p.home, G ? 2 * rows * D : 0);
  take(p.home_lse, G ? 2 * rows : 0);
  return o;
}

template <int D, bool HALF>
cudaError_t run(const KvAttendArgs& a, const KvPlan& p, const CUtensorMap* m, cudaStream_t st) {
  using L = Lay<D>;
  static_assert(D == 64 || D == 128, "two head sizes");
  cudaError_t e = cudaFuncSetAttribute(k_kv_attend<D, HALF>, cudaFuncAttributeMaxDynamicSharedMemorySize, L::SMEM);
  if (e != cudaSuccess) return e;
  // the register split below (2 x 208 + 88 a thread of each four warps) has to be within what the CTA starts with
  static const int regs = [] {
    cudaFuncAttributes f;
    return cudaFuncGetAttributes(&f, k_kv_attend<D, HALF>) == cudaSuccess ? f.numRegs : 0;
  }();
  if (regs * 3 < 2 * 208 + 88) return cudaErrorInvalidKernelImage;
  e = launch_after(k_kv_attend<D, HALF>, p.ctas, NT_ATT, L::SMEM, st, m[0], m[1], m[2], m[3], a, p);
  if (e != cudaSuccess) return e;
  // a warp a row; no more than the GPU holds at once
  const int64_t rows = std::max<int64_t>((int64_t)p.ctas * 256, a.b.n_groups ? (int64_t)a.b.n_tokens * a.n_heads : 0);
  return launch_after(k_kv_join<D, HALF>, (unsigned)std::min<int64_t>((rows + 3) / 4, (int64_t)p.ctas * 8), 128, 0, st, a, p);
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
  const size_t psm = (size_t)(PLAN_JOBS + 1 + 4 * PLAN_GROUPS) * 8;
  cudaError_t e = cudaFuncSetAttribute(k_kv_plan, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)psm);
  if (e != cudaSuccess) return e;
  k_kv_plan<<<1, NT_PLAN, psm, st>>>(a.b, p, a.c.n_kv_heads);
  e = cudaGetLastError();
  if (e != cudaSuccess) return e;
  if (D == 128) return half ? run<128, true>(a, p, m, st) : run<128, false>(a, p, m, st);
  return half ? run<64, true>(a, p, m, st) : run<64, false>(a, p, m, st);
}

}  // namespace rs
