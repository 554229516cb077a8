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
constexpr int OV = 1;          // a job's own cost in tiles: its rows' loads and stores
constexpr int NT_PLAN = 1024;
constexpr int NT_ATT = 384;
constexpr int PLAN_GROUPS = 1024;   // groups whose sums are kept in shared memory
constexpr int PLAN_JOBS = 4096;     // jobs whose costs are

constexpr int JOB_ALONE = 1;   // no other job has its rows
constexpr int JOB_EVEN = 2;    // every row sees all the job's keys
constexpr int JOB_PREFIX = 4;  // a group's prefix

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
  int32_t jobs, reserved0;
};

struct KvStart {
  int32_t job, head, off, reserved0;   // where a CTA's share begins
};

// Jobs of a request's rows.
struct KvReq {
  int32_t job0;    // its first own job
  int32_t pjob0;   // first job of its group's prefix, or -1
  int32_t ptok0;   // first row of the group
  int32_t reserved0;
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
      atomicAdd(&sum[4 * g], (unsigned long long)rt * (t ? t + OV : 0));
      atomicAdd(&sum[4 * g + 1], (unsigned long long)rt * (ts ? ts + OV : 0));
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
      const unsigned long long with = of(4 * g + 1) + (unsigned long long)rt * (tiles(P) + OV) +
                                      (unsigned long long)(max(t1 - t0, 0) >> 2);
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
        j.flags = JOB_PREFIX | (even ? JOB_EVEN : 0);
        p.jobs[at + k] = j;
      }
    }
  }
  jobs = min(jobs, (int64_t)p.cap);
  __syncthreads();   // gjob
  // the requests' own jobs
  for (int base = 0; base < n; base += NT_PLAN) {
    const int i = base + tid;
    ReqLens r{0, 0, 0};
    int key0 = 0, cnt = 0, pj = -1, pt = 0;
    if (i < n) {
      r = kv_req(b, i);
      const int g = group_of(b, i);
      if (g >= 0 && p.gjob[g] >= 0) {
        pj = p.gjob[g];
        pt = clampi(b.q_start[clampi(b.group_start[g], 0, n)], 0, b.n_tokens);
        key0 = prefix_keys(b, g);
      }
      cnt = (r.q + w2 - 1) / w2;
    }
    const int64_t at = jobs + block_scan(cnt, s_scan, &total);
    jobs += total;
    const bool fits = cnt > 0 && at + cnt <= p.cap;
    if (i < n) p.req[i] = KvReq{fits ? (int32_t)at : -1, pj, pt, 0};
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
      j.flags = pj < 0 ? JOB_ALONE : 0;
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
  const int J = (int)min(jobs, (int64_t)p.cap);
  __syncthreads();   // the jobs
  int64_t cost = 0;
  for (int base = 0; base <= J; base += NT_PLAN) {
    const int j = base + tid;
    int64_t c = 0;
    if (j < J) {
      const int nt = p.jobs[j].nt;
      c = nt > 0 ? nt + OV : 0;
    }
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
  const int64_t per = max((all + p.ctas - 1) / p.ctas, (int64_t)(2 + OV));
  if (tid == 0) *p.head = KvHead{all, per, J, 0};
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

// A CTA's share of the jobs: next() gives the segments (a job and head's tiles
// t0 .. t1 - 1) in order.  Every role of the CTA walks it by itself.
struct Walk {
  const KvJob* jobs;
  int64_t rem;
  int j, h, off, heads;
  KvJob job;            // of the segment given last
  int head, t0, t1;
  bool cut_front;       // the share began inside the job
  KvJob ahead;          // job j

  __device__ Walk(const KvPlan& p, int n_kv_heads) {
    const KvHead hd = *p.head;
    const int64_t u = (int64_t)blockIdx.x * hd.per;
    jobs = p.jobs;
    heads = n_kv_heads;
    rem = min(hd.per, hd.total - u);
    const KvStart s = p.start[blockIdx.x];
    j = s.job; h = s.head; off = s.off;
    if (rem > 0) ahead = jobs[j];
  }
  __device__ bool next() {
    while (rem > 0) {
      const int cost = ahead.nt > 0 ? ahead.nt + OV : 0;
      if (cost == 0) {
        ahead = jobs[++j];
        continue;
      }
      const int take = (int)min((int64_t)(cost - off), rem);
      t0 = max(off - OV, 0);
      t1 = max(off + take - OV, 0);
      cut_front = off > 0;
      head = h;
      job = ahead;
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
      if (t1 > t0) return true;
    }
    return false;
  }
};

template <int D>
struct Lay {
  static constexpr int QSLOT = 128 * D * 2;       // bytes of 128 rows
  static constexpr int STAGE = TK * D * 2;        // bytes of a tile of K or V
  static constexpr int NST = D == 128 ? 5 : 12;   // stages: what 227 KB leave beside the rows
  static constexpr int RING = 2 * QSLOT;
  static constexpr int MISC = RING + NST * STAGE;
  // barriers: full[NST], empty[NST], qfull[2], qempty[2], sfull[2], pfull[2], ofull[2], oempty
  static constexpr int NBAR = 2 * NST + 11;
  static constexpr int ML = MISC + 512;           // float2 [2][128]
  static constexpr int SMEM = ML + 2048;
};

// Place of K tile t and V tile t of a segment of n tiles in its loads' order
// K0 K1 V0 K2 V1 ... (the order in which they are first used)
__device__ __forceinline__ int kplace(int t) { return t == 0 ? 0 : 2 * t - 1; }
__device__ __forceinline__ int vplace(int t, int n) { return min(2 * t + 2, 2 * n - 1); }

// Two streams of 128 rows share the tensor cores, so that one's softmax runs
// under the other's products.  Of a job of more than 128 rows each stream has
// half, both over every tile; a job of fewer rows is one Q for both streams,
// which take every other tile each and are joined at the end.  Warps 0-3
// and 4-7 are the streams' softmax, a thread a row; warp 8 issues the products and
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
                 SFULL = QFULL + 32, PFULL = QFULL + 48, OFULL = QFULL + 64, OEMPTY = QFULL + 80;
  uint32_t* s_tmem = reinterpret_cast<uint32_t*>(sm + L::MISC + 8 * L::NBAR);
  volatile int* lost = reinterpret_cast<volatile int*>(sm + L::MISC + 8 * L::NBAR + 4);
  static_assert(8 * L::NBAR + 8 <= 512, "barriers");
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
    }
    mbar_init(OEMPTY, 8);
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
    Walk w(p, a.c.n_kv_heads);
    uint32_t loads = 0;   // tiles loaded before this segment
    if (warp == 9) {
      // ---------------- loads
      uint32_t qn = 0;    // Q slots used before this segment
      auto stage_wait = [&](uint32_t x) {   // until load x's stage is free
        const uint32_t use = x / L::NST;
        if (use > 0) mbar_wait(EMPTY + 8 * (x % L::NST), (use - 1) & 1, lost, p.err);
      };
      while (w.next() && !*lost) {
        const bool wide = w.job.ntok > p.tpt;
        const int nt = w.t1 - w.t0;
        const int32_t* table = a.b.table + (int64_t)w.job.row * a.b.table_stride;
        const int page0 = w.job.key0 / 16 + w.t0 * (TK / 16), pend = (w.job.kend + 15) / 16;
        // a lane's entry of the next 32 pages (four tiles), for K and, one tile behind, V
        int kb = 0, ids = 0, prev_ids = 0;
        auto fetch = [&](int t) {
          if (t >= nt) return;
          prev_ids = ids;
          kb = t;
          const int pg = page0 + t * (TK / 16) + lane;
          int id = pg < pend ? table[pg] : 0;
          if (id < 0 || id >= a.c.n_blocks) id = (int)a.c.n_blocks;   // reads as zeros
          ids = id;
        };
        auto tile = [&](int t, bool v, uint32_t x) {
          const int from = (t & ~3) == kb ? ids : prev_ids;
          const int id = __shfl_sync(~0u, from, (t & 3) * 8 + (lane & 7));
          const int pages = min(TK / 16, pend - page0 - t * (TK / 16));
          const uint32_t bar = FULL + 8 * (x % L::NST);
          const uint32_t dst = base + L::RING + (x % L::NST) * L::STAGE;
          stage_wait(x);
          if (lane == 0) mbar_expect(bar, pages * 16 * D * 2);
          __syncwarp();
          if (lane < pages) {
#pragma unroll
            for (int hf = 0; hf < D / 64; hf++)
              tma_4d(dst + hf * (TK * 128) + lane * 2048, v ? &mv : &mk, hf * 64, 0, w.head, id, bar);
          }
          __syncwarp();
        };
        fetch(0);
        tile(0, false, loads);
        // the rows, into one slot or two
        for (int s = 0; s < (wide ? 2 : 1); s++) {
          const uint32_t slot = (qn + s) & 1, use = (qn + s) >> 1;
          if (use > 0) mbar_wait(QEMPTY + 8 * slot, (use - 1) & 1, lost, p.err);
          if (lane == 0) {
            const bool one = w.job.ntok == 1;
            const uint32_t bar = QFULL + 8 * slot;
            mbar_expect(bar, (one ? 1 : p.tpt) * p.ratio * D * 2);
            for (int hf = 0; hf < D / 64; hf++)
              tma_3d(base + slot * L::QSLOT + hf * (128 * 128), one ? &mq1 : &mq, hf * 64, w.head * p.ratio,
                     w.job.tok0 + s * p.tpt, bar);
          }
          __syncwarp();
        }
        qn += wide ? 2 : 1;
        if (nt > 1) tile(1, false, loads + 1);
        for (int t = 0; t < nt; t++) {
          tile(t, true, loads + vplace(t, nt));
          if (t + 2 < nt) {
            if (((t + 2) & 3) == 0) fetch(t + 2);
            tile(t + 2, false, loads + kplace(t + 2));
          }
        }
        loads += 2 * nt;
      }
    } else if (warp == 8) {
      // ---------------- products (the warp as one; one thread issues)
      constexpr uint32_t FMT = HALF ? 0u : 1u;
      constexpr uint32_t IQK = (1u << 4) | (FMT << 7) | (FMT << 10) | ((TK / 8) << 17) | ((128 / 16) << 24);
      constexpr uint32_t IPV = (1u << 4) | (FMT << 7) | (FMT << 10) | (1u << 16) | ((D / 8) << 17) | ((128 / 16) << 24);
      const uint64_t dq = smem_desc(base, 16), dk = smem_desc(base + L::RING, 16),
                     dv = smem_desc(base + L::RING, TK * 128);
      uint32_t qn = 0, np[2] = {0, 0}, segs = 0;
      while (w.next() && !*lost) {
        const bool wide = w.job.ntok > p.tpt;
        const int nt = w.t1 - w.t0, E = wide ? 2 * nt : nt;
        auto qk = [&](int e) {
          const uint32_t s = e & 1, t = wide ? e >> 1 : e;
          const uint32_t x = loads + kplace(t), slot = (qn + (wide ? s : 0)) & 1, st = x % L::NST;
          if (!wide || s == 0) mbar_wait(FULL + 8 * st, (x / L::NST) & 1, lost, p.err);
          if (t == 0) mbar_wait(QFULL + 8 * slot, ((qn + (wide ? s : 0)) >> 1) & 1, lost, p.err);
          tc_after();
          const uint64_t qa = dq + slot * (L::QSLOT >> 4), ka = dk + st * (L::STAGE >> 4);
          if (elect_one()) {
#pragma unroll
            for (int k = 0; k < D / 16; k++) {
              const uint32_t o = ((k >> 2) * (128 * 128) + (k & 3) * 32) >> 4;
              mma_ss(tmem + s * 128, qa + o, ka + o, IQK, k > 0);
            }
            mma_commit(SFULL + 8 * s);
            if (!wide || s == 1) mma_commit(EMPTY + 8 * st);
            if (t == nt - 1) mma_commit(QEMPTY + 8 * slot);
          }
          __syncwarp();
        };
        qk(0);
        if (E > 1) qk(1);
        for (int e = 0; e < E; e++) {
          const uint32_t s = e & 1, t = wide ? e >> 1 : e;
          const uint32_t x = loads + vplace(t, nt), st = x % L::NST;
          if (!wide || s == 0) mbar_wait(FULL + 8 * st, (x / L::NST) & 1, lost, p.err);
          if (e == 0 && segs > 0) mbar_wait(OEMPTY, (segs - 1) & 1, lost, p.err);
          mbar_wait(PFULL + 8 * s, (s ? np[1] : np[0]) & 1, lost, p.err);
          if (s) np[1]++; else np[0]++;
          tc_after();
          const uint64_t va = dv + st * (L::STAGE >> 4);
          const uint32_t more = wide ? t > 0 : e >= 2;   // O holds something
          if (elect_one()) {
#pragma unroll
            for (int k = 0; k < TK / 16; k++)
              mma_ts(tmem + 256 + s * D, tmem + s * 128 + k * 8, va + k * (2048 >> 4), IPV, k > 0 ? 1u : more);
            if (!wide || s == 1) mma_commit(EMPTY + 8 * st);
            if (e + 2 >= E) mma_commit(OFULL + 8 * s);
          }
          __syncwarp();
          if (e + 2 < E) qk(e + 2);
        }
        qn += wide ? 2 : 1;
        segs++;
        loads += 2 * nt;
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
    uint32_t ns = 0, no[2] = {0, 0}, loads = 0;
    Walk w(p, a.c.n_kv_heads);
    const int tl = r / p.ratio, hl = r - tl * p.ratio;   // the row's token and head in its 128
    while (w.next()) {   // (both streams meet in here: neither leaves early)
      const bool wide = w.job.ntok > p.tpt;
      const int nt = w.t1 - w.t0;
      const int tok = (wide ? s * p.tpt : 0) + tl;
      const bool live = tl < p.tpt && tok < w.job.ntok;
      const bool any = __any_sync(~0u, live);
      int lim = 0;   // keys from key0 on that the row sees
      if (live) {
        if (w.job.flags & JOB_EVEN) {
          lim = w.job.kend;
        } else if (w.job.flags & JOB_PREFIX) {
          const int row = w.job.tok0 + tok;
          int lo = w.job.row, hi = a.b.n_req;
          while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (a.b.q_start[mid] <= row) lo = mid; else hi = mid;
          }
          const int64_t x = (int64_t)max(a.b.kv_len[lo], 0) - a.b.q_start[lo + 1] + row + 1;
          lim = (int)min((int64_t)w.job.kend, max(x, (int64_t)0));
        } else {
          lim = (int)min((int64_t)w.job.kend, (int64_t)w.job.lim0 + tok);
        }
        lim -= w.job.key0;
      }
      // keys of a last tile that the job's end cuts
      const int ends = w.t1 == w.job.nt ? (w.job.kend - w.job.key0) & (TK - 1) : 0;
      const int low = __reduce_min_sync(~0u, live ? lim : INT_MAX);
      float m = live ? -INFINITY : 0.0f, l0 = 0.0f, l1 = 0.0f;
      for (int t = wide ? 0 : s; t < nt; t += wide ? 1 : 2) {
        mbar_wait(SFULL + 8 * s, ns & 1, lost, p.err);
        ns++;
        tc_after();
        if (any) {
          const int k0 = (w.t0 + t) * TK;
          const bool cut = low < k0 + TK;   // (the warp's rows see different ends)
          const int left = lim - k0;
          const bool first = wide ? t == 0 : t < 2;   // O holds nothing yet
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
        if (t == nt - 1 && (!wide || s == 0) && ends) {
          // V rows past the keys' end: their weights are 0, but 0 times what lies there may be NaN.
          // (Of a wide job stream 0's product with this tile comes first.)
          const uint32_t x = loads + vplace(t, nt);
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
      loads += 2 * nt;
      // ---- the rows' results: the stream's own, or both streams' joined, half the columns each
      float l = __fadd_rn(l0, l1);
      float f0, f1 = 0.0f, lse2;
      int c0 = 0, c1 = D;
      if (wide) {
        f0 = l > 0.0f ? __fdiv_rn(1.0f, l) : 0.0f;
        lse2 = l > 0.0f ? __fadd_rn(__fmul_rn(m, sl), __log2f(l)) : -INFINITY;
        if (!(l == l)) f0 = lse2 = l;
        mbar_wait(OFULL + 8 * s, no[s] & 1, lost, p.err);
        no[0]++;   // (the other stream's has its turn too)
        no[1]++;
      } else {
        ml[s * 128 + r] = make_float2(m, l);
        asm volatile("bar.sync 1, 256;" ::: "memory");
        const float2 x = ml[r], y = ml[128 + r];
        const float mm = fmaxf(x.x, y.x);
        const float wx = x.x == -INFINITY ? 0.0f : ex2(__fmul_rn(__fsub_rn(x.x, mm), sl));
        const float wy = y.x == -INFINITY ? 0.0f : ex2(__fmul_rn(__fsub_rn(y.x, mm), sl));
        l = fmaf(x.y, wx, __fmul_rn(y.y, wy));
        const float inv = l > 0.0f ? __fdiv_rn(1.0f, l) : l == l ? 0.0f : l;
        f0 = __fmul_rn(wx, inv);
        f1 = __fmul_rn(wy, inv);
        lse2 = l > 0.0f ? __fadd_rn(__fmul_rn(mm, sl), __log2f(l)) : l == l ? -INFINITY : l;
        c0 = s * (D / 2);
        c1 = c0 + D / 2;
        mbar_wait(OFULL, no[0] & 1, lost, p.err);
        no[0]++;
        if (nt > 1) {
          mbar_wait(OFULL + 8, no[1] & 1, lost, p.err);
          no[1]++;
        }
      }
      tc_after();
      const bool whole = w.t0 == 0 && w.t1 == w.job.nt;
      const bool direct = whole && (w.job.flags & JOB_ALONE);
      if (any) {
        const int64_t row = (int64_t)w.job.tok0 + tok;
        const int hq = w.head * p.ratio + hl;
        // a part's row: with the other whole parts of all rows, or with the CTA's cut ones
        const int64_t all = (int64_t)a.b.n_tokens * a.n_heads;
        const int64_t at = whole ? ((w.job.flags & JOB_PREFIX) ? 0 : all) + row * a.n_heads + hq
                                 : ((int64_t)blockIdx.x * 2 + (w.cut_front ? 0 : 1)) * 256 + (wide ? s * 128 : 0) + r;
        float* part = (whole ? p.home : p.part) + at * D;
        uint16_t* out = static_cast<uint16_t*>(a.out) + row * a.o_ts + hq * a.o_hs;
        if (live && c0 == 0) {
          if (!direct) (whole ? p.home_lse : p.part_lse)[at] = lse2;
          else if (a.lse) a.lse[row * a.n_heads + hq] = __fmul_rn(lse2, 0.6931471805599453f);
        }
#pragma unroll 1
        for (int c = c0; c < c1; c += 32) {
          uint32_t o[32];
          float y[32];
          tm_ld32(o, tmem + lanes + 256 + (wide ? s * D : 0) + c);
          tm_wait_ld(o);
#pragma unroll
          for (int k = 0; k < 32; k++) y[k] = f0 == 0.0f ? 0.0f : __fmul_rn(__uint_as_float(o[k]), f0);
          if (!wide && nt > 1) {
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
      __syncwarp();
      if (lane == 0) mbar_arrive(OEMPTY);
      if (!wide) asm volatile("bar.sync 1, 256;" ::: "memory");   // ml is free again
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

// The tiles of job j, head h that CTA c has.
__device__ __forceinline__ bool segment(int64_t u0, int cost, int64_t per, int64_t c, int& t0, int& t1) {
  const int64_t lo = max(c * per, u0) - u0, hi = min((c + 1) * per, u0 + cost) - u0;
  t0 = max((int)lo - OV, 0);
  t1 = max((int)hi - OV, 0);
  return t1 > t0;
}

// A row (token, head) from the parts its jobs left, a warp for `rpw` heads of a
// token's kv head; rows that no job covers become 0 and -inf.  Rows whose one
// job was whole are done already.
template <int D, bool HALF>
__global__ void __launch_bounds__(128) k_kv_join(const __grid_constant__ KvAttendArgs a,
                                                 const __grid_constant__ KvPlan p, int rpw) {
  asm volatile("griddepcontrol.wait;" ::: "memory");
  constexpr int E = D / 32;
  const int lane = threadIdx.x & 31;
  const int units = a.n_heads / rpw;
  const int64_t w = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 5);
  if (w >= (int64_t)a.b.n_tokens * units) return;
  const int row = (int)(w / units), hq0 = (int)(w - (int64_t)row * units) * rpw;
  const int kh = hq0 / p.ratio, w2 = 2 * p.tpt, n = a.b.n_req;
  const KvHead hd = *p.head;
  int job[2] = {-1, -1};   // the prefix's and the request's own
  if (n > 0 && row < a.b.q_start[n]) {
    int i;
    if (row < n && a.b.q_start[row] == row && a.b.q_start[row + 1] == row + 1) {
      i = row;   // single tokens
    } else {
      int lo = 0, hi = n;
      while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (a.b.q_start[mid] <= row) lo = mid; else hi = mid;
      }
      i = lo;
    }
    const KvReq r = p.req[i];
    const int q0 = a.b.q_start[i];
    if (r.job0 >= 0 && q0 >= 0 && row >= q0) job[1] = min(r.job0 + (row - q0) / w2, hd.jobs - 1);
    if (r.pjob0 >= 0 && row >= r.ptok0) job[0] = min(r.pjob0 + (row - r.ptok0) / w2, hd.jobs - 1);
  }
  int64_t u0[2] = {0, 0};
  int cost[2] = {0, 0}, nt[2] = {0, 0}, rr[2] = {0, 0};
  int c0[2] = {0, 0}, c1[2] = {-1, -1};   // CTAs
  bool done = false;
#pragma unroll
  for (int k = 0; k < 2; k++) {
    if (job[k] < 0) continue;
    const KvJob& j = p.jobs[job[k]];
    if (j.nt <= 0 || row < j.tok0 || row - j.tok0 >= j.ntok) continue;
    nt[k] = j.nt;
    const int64_t at = p.cost[job[k]];
    cost[k] = j.nt + OV;
    u0[k] = at * a.c.n_kv_heads + (int64_t)kh * cost[k];
    c0[k] = (int)(u0[k] / hd.per);
    c1[k] = min((int)((u0[k] + cost[k] - 1) / hd.per), p.ctas - 1);
    const int tok = row - j.tok0, second = j.ntok > p.tpt && tok >= p.tpt;
    rr[k] = second * 128 + (tok - second * p.tpt) * p.ratio;   // the token's first row in the job's 256
    int t0, t1;
    if (k == 1 && (j.flags & JOB_ALONE)) {
      // whole in its first CTA, or in the next when the first has only the job's own cost
      if (segment(u0[k], cost[k], hd.per, c0[k], t0, t1)) done = t1 == j.nt;
      else if (segment(u0[k], cost[k], hd.per, c0[k] + 1, t0, t1)) done = t0 == 0 && t1 == j.nt;
    }
  }
  if (done) return;
  const int64_t all = (int64_t)a.b.n_tokens * a.n_heads;
  for (int x = 0; x < rpw; x++) {
    const int hq = hq0 + x, hl = hq - kh * p.ratio;
    float m = -INFINITY, l = 0.0f, o[E];
#pragma unroll
    for (int e = 0; e < E; e++) o[e] = 0.0f;
#pragma unroll
    for (int k = 0; k < 2; k++) {
      for (int c = c0[k]; c <= c1[k]; c++) {
        int t0, t1;
        if (!segment(u0[k], cost[k], hd.per, c, t0, t1)) continue;
        const bool whole = t0 == 0 && t1 == nt[k];
        const int64_t at = whole ? (k ? all : 0) + (int64_t)row * a.n_heads + hq
                                 : ((int64_t)c * 2 + (c == c0[k] ? 1 : 0)) * 256 + rr[k] + hl;
        const float s = (whole ? p.home_lse : p.part_lse)[at];
        if (s == -INFINITY) continue;
        const float* src = (whole ? p.home : p.part) + at * D + lane * E;
        float y[E];
#pragma unroll
        for (int e = 0; e < E; e++) y[e] = src[e];
        const float m2 = fmaxf(m, s), f = m == -INFINITY ? 0.0f : ex2(__fsub_rn(m, m2)), g = ex2(__fsub_rn(s, m2));
        l = fmaf(l, f, g);
#pragma unroll
        for (int e = 0; e < E; e++) o[e] = fmaf(o[e], f, __fmul_rn(g, y[e]));
        m = m2;
      }
    }
    const float inv = l == 0.0f ? 0.0f : __fdiv_rn(1.0f, l);
    uint16_t* out = static_cast<uint16_t*>(a.out) + (int64_t)row * a.o_ts + hq * a.o_hs + lane * E;
#pragma unroll
    for (int e = 0; e < E; e += 2)
      *reinterpret_cast<uint32_t*>(out + e) = pack2<HALF>(__fmul_rn(o[e], inv), __fmul_rn(o[e + 1], inv));
    if (a.lse && lane == 0)
      a.lse[(int64_t)row * a.n_heads + hq] = l == 0.0f ? -INFINITY : __fmul_rn(__fadd_rn(m, __log2f(l)), 0.6931471805599453f);
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
  // a warp a row while that many warps fit on the GPU at once, else a warp a token and kv head
  const int64_t rows = (int64_t)a.b.n_tokens * a.n_heads;
  const int rpw = rows <= (int64_t)p.ctas * 64 ? 1 : p.ratio;
  return launch_after(k_kv_join<D, HALF>, (unsigned)((rows / rpw + 3) / 4), 128, 0, st, a, p, rpw);
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
