// kv_attend4's jobs of many rows (up to 256 by 128-key tiles) on the tensor cores.
#include <algorithm>
#include <climits>
#include <type_traits>

#include "kv4_plan.cuh"
#include "kv_mma.cuh"

namespace rs {

using namespace kv4;

namespace {

constexpr int NT = 512;
constexpr int NR = 2;      // runs ahead
// registers a thread of the two softmax warpgroups, of the third (products, runs), of the fourth (conversion)
constexpr int R_SOFT = 184, R_MMA = 64, R_CONV = 80;
static_assert(2 * R_SOFT + R_MMA + R_CONV <= 512, "the split is within what a CTA starts with");

struct Run {
  Job job;
  int head, t0, t1;      // t1 = t0: no more
  int reserved0;
};

// References (in powers of two) past which a score's product with the row's factor is not subtracted from them.
constexpr float FAR = 1024.0f;

__device__ __forceinline__ float largest(const uint32_t* v) {   // of 32
  float x = __uint_as_float(v[0]), y = __uint_as_float(v[1]);
#pragma unroll
  for (int c = 2; c < 32; c += 2) {
    x = fmaxf(x, __uint_as_float(v[c]));
    y = fmaxf(y, __uint_as_float(v[c + 1]));
  }
  return fmaxf(x, y);
}

template <int D>
struct Lay {
  static constexpr int QSLOT = 128 * D * 2;             // bytes of 128 rows
  static constexpr int STAGE = TILE * D * 2;            // bytes of a tile of K or V
  static constexpr int NST = 4;
  static constexpr int AHEAD = 3;                       // tiles of codes on their way
  static constexpr int CROW = D / 2 + 16;               // bytes of a key's codes and scales
  static constexpr int RING = 2 * QSLOT;
  static constexpr int CODES = RING + NST * STAGE;
  static constexpr int RUNS = CODES + AHEAD * TILE * CROW;
  static constexpr int BARS = RUNS + NR * (int)sizeof(Run);
  // full[NST], empty[NST], qfull[2], sfull[2], pfull[2][2], hfull[2], ofull[2], rfull[NR], rempty[NR]
  static constexpr int NBAR = 2 * NST + 12 + 2 * NR;
  static constexpr int SMEM = BARS + 8 * NBAR + 16;
  static_assert(SMEM <= 227 * 1024, "shared memory");
};

// Two streams of 128 rows (of one job) share the tensor cores, so that one's softmax runs
// under the other's products.  Warps 0-3 and 4-7 are the streams' softmax, a thread a row;
// warp 8 issues the products; warp 9 finds the runs; warps 12-15 convert, a thread a key:
// codes and scales come by copies of their own two tiles ahead, and leave as fp16 in the
// swizzled rows that the products read.
// Shared memory: two slots of 128 rows of q, a ring of four tiles of K and V in turn.
// TMEM: S of each stream 128 columns (P, 64 columns, overwrites it), O D each.
// The m of a row is the largest score of its first 64 keys and moves only when 64 weights
// sum to more than fp16 allows.
// Bound: 2048 tokens behind 14 336, 32 heads on 8 of 128: 408 us, 1.26 PFLOP/s.  256 rows by 128 keys are 2048
// clocks of the products and take some 3600: a stream's softmax takes 1900 to 2100 clocks after its
// scores are there (two halves; exponentials alone are 512 of the SM's, the other stream's and the
// conversion's instructions lie between), its next weights' and scores' products 1100 after that.
// A job of up to 128 rows is one stream: nothing runs under its softmax, and its tile takes as long as one of 256 (64
// requests of 40 rows over 2 048 to 24 576 keys, 8 kv heads of 128: 440 us, where the codes alone take 98).
// Measured and not kept (us a call, 430 as it is): products of 64 keys, with two sets of scores a stream (466: a
// product of 128 x 64 takes as long as one of 128 x 128, whose rows of q are read as often) or with q in TMEM (543);
// four softmax warpgroups, a thread half a row's tile (456).
template <int D, bool HALF>
__global__ void __launch_bounds__(NT, 1) k_kv4_tiles(const __grid_constant__ KvAttend4Args a, const __grid_constant__ Plan p) {
  using L = Lay<D>;
  extern __shared__ __align__(1024) unsigned char sm[];
  const uint32_t base = smem_u32(sm);
  const int tid = threadIdx.x, warp = __shfl_sync(~0u, tid >> 5, 0), lane = tid & 31;
  const uint32_t FULL = base + L::BARS, EMPTY = FULL + 8 * L::NST, QFULL = EMPTY + 8 * L::NST, SFULL = QFULL + 16, PFULL = QFULL + 32,
                 HFULL = QFULL + 64, OFULL = QFULL + 80, RFULL = QFULL + 96, REMPTY = RFULL + 8 * NR;
  Run* const runs = reinterpret_cast<Run*>(sm + L::RUNS);
  uint32_t* s_tmem = reinterpret_cast<uint32_t*>(sm + L::BARS + 8 * L::NBAR);
  volatile int* lost = reinterpret_cast<volatile int*>(s_tmem + 1);
  if (base & 1023) {   // (swizzled tiles lie on 1024-byte boundaries)
    asm volatile("griddepcontrol.wait;" ::: "memory");
    if (tid == 0) *reinterpret_cast<volatile int32_t*>(p.err) = 1;
    return;
  }
  if (tid == 0) {
    for (int s = 0; s < L::NST; s++) { mbar_init(FULL + 8 * s, 4); mbar_init(EMPTY + 8 * s, 1); }
    for (int s = 0; s < 2; s++) {
      mbar_init(QFULL + 8 * s, 4);
      mbar_init(SFULL + 8 * s, 1);
      mbar_init(PFULL + 16 * s, 4);
      mbar_init(PFULL + 16 * s + 8, 4);
      mbar_init(HFULL + 8 * s, 1);
      mbar_init(OFULL + 8 * s, 1);
    }
    for (int s = 0; s < NR; s++) { mbar_init(RFULL + 8 * s, 1); mbar_init(REMPTY + 8 * s, 13); }
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
  // (What is above does not wait for the plan.  The rows' kernel may begin once all CTAs are past this: the plan is there.)
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;");
  const Head hd = *p.head;
  if (hd.whole ? (int64_t)blockIdx.x >= (int64_t)hd.jobs[1] * a.c.n_kv_heads : hd.total[1] <= (int64_t)blockIdx.x * hd.per[1]) {   // nothing for this CTA
    if (warp == 8) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem));
    return;
  }

  if (warp >= 12) {
    // ---------------- conversion
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(R_CONV));
    const int r = tid & 127;
    const uint32_t mine = base + L::CODES + r * L::CROW;
    const uint32_t dst = base + L::RING + r * 128;
    uint32_t x = 0;   // tiles converted
    for (uint32_t k = 0;; k++) {
      mbar_wait(RFULL + 8 * (k % NR), (k / NR) & 1, lost, p.err);
      const Run& run = runs[k % NR];
      const int t0 = run.t0, n = run.t1 - t0, head = run.head, key0 = run.job.key0 + t0 * TILE + r, kend = run.job.kend;
      if (gave_up(lost) || n == 0) break;
      const int32_t* row = a.b.table + (int64_t)run.job.trow * a.b.table_stride;
      __syncwarp();
      if (lane == 0) mbar_arrive(REMPTY + 8 * (k % NR));
      const unsigned char* const kc = static_cast<const unsigned char*>(a.c.k) + head * a.c.stride_head + (r & 15) * a.c.stride_token;
      const unsigned char* const vc = static_cast<const unsigned char*>(a.c.v) + head * a.c.stride_head + (r & 15) * a.c.stride_token;
      const unsigned char* const ks = static_cast<const unsigned char*>(a.c.k_scale) + head * a.c.scale_head + (r & 15) * a.c.scale_token;
      const unsigned char* const vs = static_cast<const unsigned char*>(a.c.v_scale) + head * a.c.scale_head + (r & 15) * a.c.scale_token;
      // copies of load u: K of tile u / 2, or V; ids of a tile ahead
      auto page = [&](int t) { return t < n && key0 + t * TILE < kend ? row[(key0 + t * TILE) >> 4] : -1; };
      int id = page(0), id_next = page(1);
      auto copy = [&](int u, uint32_t slot) {
        if (u > 0 && !(u & 1)) {
          id = id_next;
          id_next = page((u >> 1) + 1);
        }
        const bool there = id >= 0 && id < a.c.n_blocks;
        const int64_t at = there ? id : 0;
        const unsigned char* const c = ((u & 1) ? vc : kc) + at * a.c.stride_block;
        const uint32_t to = mine + slot * (TILE * L::CROW);
#pragma unroll
        for (int i = 0; i < D / 32; i++) copy_async<16>(to + 16 * i, c + 16 * i, there);
        copy_async<D / 16>(to + D / 2, ((u & 1) ? vs : ks) + at * a.c.scale_block, there);
      };
      uint32_t slot = 0, into = L::AHEAD - 1;
      for (int u = 0; u < L::AHEAD - 1; u++) {
        if (u < 2 * n) copy(u, u);
        copies_commit();
      }
      for (int u = 0; u < 2 * n; u++) {
        copies_wait<L::AHEAD - 2>();
        if (u + L::AHEAD - 1 < 2 * n) copy(u + L::AHEAD - 1, into);
        copies_commit();
        const uint32_t from = mine + slot * (TILE * L::CROW);
        if (++slot == L::AHEAD) slot = 0;
        if (++into == L::AHEAD) into = 0;
        const uint32_t st = x % L::NST, use = x / L::NST;
        x++;
        uint32_t sc[D / 64];
        if constexpr (D == 128) asm volatile("ld.shared.v2.u32 {%0, %1}, [%2];" : "=r"(sc[0]), "=r"(sc[1]) : "r"(from + D / 2));
        else asm volatile("ld.shared.u32 %0, [%1];" : "=r"(sc[0]) : "r"(from + D / 2));
        if (key0 + (u >> 1) * TILE >= kend) {   // (what lies past the end may be NaN)
#pragma unroll
          for (int i = 0; i < D / 64; i++) sc[i] = 0;
        }
        if (use > 0) mbar_wait(EMPTY + 8 * st, (use - 1) & 1, lost, p.err);
        const uint32_t to = dst + st * L::STAGE;
#pragma unroll
        for (int i = 0; i < D / 32; i++) {   // 32 elements
          uint32_t w[4];
          asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "r"(from + 16 * i));
          const uint32_t two = scales_f16(sc[i >> 1] >> (16 * (i & 1)));
#pragma unroll
          for (int q = 0; q < 4; q++) {
            uint32_t y[4];
            codes_f16(w[q], y);
            const uint32_t f = both(two, q >= 2);
#pragma unroll
            for (int z = 0; z < 4; z++) y[z] = mul_f16x2(y[z], f);
            const int c = 4 * i + q;   // chunk of 8 elements
            asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};"
                         ::"r"(to + (c >> 3) * (TILE * 128) + (((c & 7) ^ (r & 7)) * 16)), "r"(y[0]), "r"(y[1]), "r"(y[2]), "r"(y[3]) : "memory");
          }
        }
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        __syncwarp();
        if (lane == 0) mbar_arrive(FULL + 8 * st);
      }
    }
    copies_wait<0>();
  } else if (warp >= 8) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(R_MMA));
    if (warp == 9) {
      // ---------------- runs
      Walk w(p.jobs[1], hd, 1, a.c.n_kv_heads, blockIdx.x, lane);
      for (uint32_t k = 0;; k++) {
        int head = 0, t0 = 0, t1 = 0;
        const bool more = w.next(head, t0, t1);
        if (k >= NR) mbar_wait(REMPTY + 8 * (k % NR), (k / NR - 1) & 1, lost, p.err);
        if (gave_up(lost)) break;
        if (lane == 0) {
          Run* const r = runs + k % NR;
          if (more) r->job = w.job;
          r->head = head;
          r->t0 = t0;
          r->t1 = more ? t1 : t0;
          mbar_arrive(RFULL + 8 * (k % NR));
        }
        __syncwarp();
        if (!more) break;
        if (t0 == 0) tell(a, p, w, hd.per[1], blockIdx.x, head, t1, lane, 32);
      }
    } else if (warp == 8) {
      // ---------------- products (the warp as one; one thread issues)
      constexpr uint32_t IQK = (1u << 4) | ((TILE / 8) << 17) | ((128 / 16) << 24);
      constexpr uint32_t IPV = (1u << 4) | (1u << 16) | ((D / 8) << 17) | ((128 / 16) << 24);
      const uint64_t dq = smem_desc(base, 16), dk = smem_desc(base + L::RING, 16), dv = smem_desc(base + L::RING, TILE * 128);
      uint32_t x = 0, qn0 = 0, qn1 = 0, np0 = 0, np1 = 0;
      auto take = [&]() {   // the next tile's stage
        const uint32_t st = x % L::NST;
        mbar_wait(FULL + 8 * st, (x / L::NST) & 1, lost, p.err);
        x++;
        return st;
      };
      auto scores = [&](uint32_t s, uint32_t st) {
        const uint64_t qa = dq + s * (L::QSLOT >> 4), ka = dk + st * (L::STAGE >> 4);
        if (elect_one()) {
#pragma unroll
          for (int q = 0; q < D / 16; q++) {
            const uint32_t o = ((q >> 2) * (128 * 128) + (q & 3) * 32) >> 4;
            mma_ss(tmem + s * 128, qa + o, ka + o, IQK, q > 0);
          }
          mma_commit(SFULL + 8 * s);
        }
        __syncwarp();
      };
      for (uint32_t k = 0;; k++) {
        mbar_wait(RFULL + 8 * (k % NR), (k / NR) & 1, lost, p.err);
        const int n = runs[k % NR].t1 - runs[k % NR].t0, streams = runs[k % NR].job.nrows > 128 ? 2 : 1;
        if (gave_up(lost) || n == 0) break;
        __syncwarp();
        if (lane == 0) mbar_arrive(REMPTY + 8 * (k % NR));
        uint32_t kst = take(), vst = 0;
        for (int s = 0; s < streams; s++) {
          mbar_wait(QFULL + 8 * s, (s ? qn1 : qn0) & 1, lost, p.err);
          tc_after();
          scores(s, kst);
        }
        if (elect_one()) mma_commit(EMPTY + 8 * kst);
        __syncwarp();
        qn0++;
        qn1 += streams > 1;
        for (int i = 0; i < n; i++) {
          for (int s = 0; s < streams; s++) {
            if (s == 0) vst = take();
            const uint64_t va = dv + vst * (L::STAGE >> 4);
#pragma unroll
            for (int h = 0; h < 2; h++) {   // of either half of the tile's keys
              mbar_wait(PFULL + 16 * s + 8 * h, (s ? np1 : np0) & 1, lost, p.err);
              tc_after();
              const uint32_t more = i > 0;   // O holds something
              if (elect_one()) {
#pragma unroll
                for (int q = h * (TILE / 32); q < (h + 1) * (TILE / 32); q++)
                  mma_ts(tmem + 256 + s * D, tmem + s * 128 + q * 8, va + q * (2048 >> 4), IPV, q > 0 ? 1u : more);
                if (h == 0) mma_commit(HFULL + 8 * s);
                else if (s + 1 == streams) mma_commit(EMPTY + 8 * vst);
                if (h == 1 && i + 1 == n) mma_commit(OFULL + 8 * s);
              }
              __syncwarp();
            }
            np0 += s == 0;
            np1 += s == 1;
            if (i + 1 < n) {
              if (s == 0) kst = take();
              tc_after();
              scores(s, kst);
              if (s + 1 == streams) {
                if (elect_one()) mma_commit(EMPTY + 8 * kst);
                __syncwarp();
              }
            }
          }
        }
      }
    }
  } else {
    // ---------------- softmax, a thread a row
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(R_SOFT));
    const int s = warp >> 2, r = tid & 127;
    const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
    const uint32_t ts = tmem + lanes + s * 128, to = tmem + lanes + 256 + s * D;
    uint32_t ns = 0, no = 0;
    for (uint32_t k = 0;; k++) {
      mbar_wait(RFULL + 8 * (k % NR), (k / NR) & 1, lost, p.err);
      const Run& run = runs[k % NR];
      const Job job = run.job;
      const int head = run.head, t0 = run.t0, t1 = run.t1, n = t1 - t0;
      if (gave_up(lost) || n == 0) break;
      __syncwarp();
      if (lane == 0) mbar_arrive(REMPTY + 8 * (k % NR));
      if (job.nrows <= 128 * s) continue;
      // ---- the rows of q, as fp16, into their places: a row's 16-byte pieces by neighbouring lanes, a few rows at a time
      // (a thread a row would touch 32 lines with every load and store)
      const bool live = s * 128 + r < job.nrows;
      const int flat = job.row0 + min(s * 128 + r, job.nrows - 1);
      int hl;
      const int in = token_of(p, flat, hl);
      const int tok = job.tok0 + in, hq = head * p.ratio + hl;
      const unsigned lives = __ballot_sync(~0u, live);
      constexpr int CH = D / 8, RS = 32 / CH;   // pieces of a row, rows at a time
      const int ch = lane % CH;
      // piece ch of row rr of the warp's 32, of q or of staged results
      auto piece = [&](int rr, int c) {
        const int row = (r & 96) + rr;
        return reinterpret_cast<uint4*>(sm + s * L::QSLOT + (c >> 3) * (128 * 128) + row * 128 + (((c & 7) ^ (row & 7)) * 16));
      };
      float inverse = 1.0f;
      {
        const unsigned long long src = reinterpret_cast<unsigned long long>(static_cast<const uint16_t*>(a.q) + (int64_t)tok * a.q_ts + (int64_t)hq * a.q_hs);
#pragma unroll 8
        for (int rr = 0; rr < 32; rr += RS) {
          const int row = rr + lane / CH;
          copy_async<16>(smem_u32(piece(row, ch)), reinterpret_cast<const uint4*>(__shfl_sync(~0u, src, row)) + ch, (lives >> row) & 1);
        }
        copies_commit();
        copies_wait<0>();
        if (!HALF) {   // a thread a row: no thread waits for another's maximum
          __syncwarp();
          __nv_bfloat162 most2 = __nv_bfloat162{0.0f, 0.0f};
#pragma unroll 8
          for (int c = 0; c < CH; c++) {
            const uint4 v = *piece(lane, c);
            const uint32_t y[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
            for (int z = 0; z < 4; z++) most2 = __hmax2(most2, __habs2(*reinterpret_cast<const __nv_bfloat162*>(&y[z])));
          }
          const float power = row_power(fmaxf(__low2float(most2), __high2float(most2)), inverse);
#pragma unroll 8
          for (int c = 0; c < CH; c++) {
            uint4* const at = piece(lane, c);
            const uint4 v = *at;
            uint32_t y[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
            for (int z = 0; z < 4; z++) {
              const float2 f = unpack2<false>(y[z]);
              y[z] = pack2<true>(__fmul_rn(f.x, power), __fmul_rn(f.y, power));
            }
            *at = make_uint4(y[0], y[1], y[2], y[3]);
          }
        }
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        tc_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(QFULL + 8 * s);
      }
      const float sl = row_factor(a, inverse);
      const int lim = live ? limit_of(a.b, job, tok, in) - job.key0 : 0;   // keys from key0 on that the row sees
      const int low = __reduce_min_sync(~0u, live ? lim : INT_MAX), high = __reduce_max_sync(~0u, lim);
      // The row's reference: m, as a score, and big = m sl (a weight is exp2(BIAS + sl s - big)); past FAR, where the
      // product's rounding would show, exp2(BIAS + sl (s - m)) is taken.
      float m = live ? -INFINITY : 0.0f, shift = BIAS, l0 = 0.0f, l1 = 0.0f;
      bool far = false;
      auto refer = [&](float to) {
        m = to;
        const float big = __fmul_rn(m, sl);
        shift = m == -INFINITY ? BIAS : __fsub_rn(BIAS, big);
        far = live && fabsf(big) > FAR && m != -INFINITY;
      };
      for (int i = 0; i < n; i++) {
        mbar_wait(SFULL + 8 * s, ns & 1, lost, p.err);
        tc_after();
#pragma unroll 1
        for (int h = 0; h < 2; h++) {   // half of the tile's keys, so that their product begins under the other's weights
          const int k0 = (t0 + i) * TILE + h * 64, left = lim - k0, seen = high - k0;
          const uint32_t th = ts + 64 * h;
          float a0, a1;
          uint32_t v[64];
          // Twice at most: where some row's weights sum to too much, its m moves to the keys' maximum and all weights are
          // taken again (the other rows' come out as they were).  The second pass is not looked at: infinities and NaN in a
          // row end here as in any other.
#pragma unroll 1
          for (int pass = 0; pass < 2; pass++) {
            float b0 = 0.0f, b1 = 0.0f;
            a0 = a1 = 0.0f;
            if (seen > 0) {
              tm_ld32(v, th);
              tm_ld32(v + 32, th + 32);
              tm_wait_ld(v);
              tm_wait_ld(v + 32);
              if (low < k0 + 64) {   // some row's sight ends here
#pragma unroll
                for (int c = 0; c < 64; c++)
                  if (c >= left) v[c] = 0xFF800000u;
              }
              if (i == 0 && pass == 0 && live && m == -INFINITY) refer(fmaxf(largest(v), largest(v + 32)));
              if (__any_sync(~0u, far)) {
                const float nm = m == -INFINITY ? 0.0f : -m;
#pragma unroll
                for (int c = 0; c < 64; c++)
                  if (far) v[c] = __float_as_uint(__fadd_rn(__uint_as_float(v[c]), nm));
              }
              const float by = far ? BIAS : shift;
#pragma unroll
              for (int c = 0; c < 64; c += 4) {   // in pairs into v's first half
                float e0 = __uint_as_float(v[c]), e1 = __uint_as_float(v[c + 1]), e2 = __uint_as_float(v[c + 2]), e3 = __uint_as_float(v[c + 3]);
                fma2(e0, e1, sl, by);
                fma2(e2, e3, sl, by);
                e0 = ex2(e0); e1 = ex2(e1); e2 = ex2(e2); e3 = ex2(e3);
                add2(a0, a1, e0, e1);
                add2(b0, b1, e2, e3);
                v[c / 2] = pack2<true>(e0, e1);
                v[c / 2 + 1] = pack2<true>(e2, e3);
              }
              add2(a0, a1, b0, b1);
            } else {
#pragma unroll
              for (int c = 0; c < 32; c++) v[c] = 0;
            }
            const bool over = live && !(__fadd_rn(a0, a1) <= 60000.0f);
            if (pass || !__any_sync(~0u, over)) break;
            // a row's m moves: O and l are scaled
            float top = -INFINITY;
#pragma unroll 1
            for (int c = 0; c < 64; c += 32) {
              uint32_t x[32];
              tm_ld32(x, th + c);
              tm_wait_ld(x);
#pragma unroll
              for (int z = 0; z < 32; z++)
                if (z >= left - c) x[z] = 0xFF800000u;
              top = fmaxf(top, largest(x));
            }
            const float m2 = over ? fmaxf(m, top) : m;
            const float f = m2 > m ? ex2(__fmul_rn(__fsub_rn(m, m2), sl)) : 1.0f;
            if (__any_sync(~0u, m2 > m)) {
              if (h) {   // (the product with the first half's weights is done)
                mbar_wait(HFULL + 8 * s, ns & 1, lost, p.err);
                tc_after();
              }
              if (i > 0 || h) {
                l0 = __fmul_rn(l0, f);
                l1 = __fmul_rn(l1, f);
#pragma unroll 1
                for (int c = 0; c < D; c += 32) {
                  uint32_t o[32];
                  tm_ld32(o, to + c);
                  tm_wait_ld(o);
#pragma unroll
                  for (int z = 0; z < 32; z++) o[z] = __float_as_uint(__fmul_rn(__uint_as_float(o[z]), f));
                  tm_st32(to + c, o);
                }
              }
            }
            refer(m2);
          }
          l0 = __fadd_rn(l0, a0);
          l1 = __fadd_rn(l1, a1);
          tm_st32(ts + 32 * h, v);
          tm_wait_st();
          tc_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(PFULL + 16 * s + 8 * h);
        }
        ns++;
      }
      // ---- the row's result
      mbar_wait(OFULL + 8 * s, no & 1, lost, p.err);
      no++;
      tc_after();
      const float l = __fadd_rn(l0, l1);
      const bool whole = t0 == 0 && t1 == job.nt, direct = whole && (job.flags & JOB_ALONE);
      const int64_t home = (int64_t)tok * a.n_heads + hq;
      const int64_t at = whole ? ((job.flags & JOB_PREFIX) ? 0 : (int64_t)a.b.n_tokens * a.n_heads) + home
                               : part_row(p, 1, blockIdx.x, head, t0 > 0) + s * 128 + r;
      if (live) {
        if (!direct) (whole ? p.home_sum : p.part_sum[1])[at] = make_float4(m, l, sl, 0.0f);
        else if (a.lse) a.lse[home] = log_sum(m, l, sl);
      }
      const float inv = inverse_of(a.c.v_unit, l);
      // through the rows' places in shared memory: results in 16 bits at once, parts in two halves
      const unsigned long long dst = direct ? reinterpret_cast<unsigned long long>(static_cast<uint16_t*>(a.out) + (int64_t)tok * a.o_ts + (int64_t)hq * a.o_hs)
                                            : reinterpret_cast<unsigned long long>((whole ? p.home : p.part[1]) + at * D);
      const int cols = direct ? D : D / 2;   // of a turn
      for (int c0 = 0; c0 < D; c0 += cols) {
#pragma unroll 1
        for (int c = 0; c < cols; c += 32) {
          uint32_t o[32];
          tm_ld32(o, to + c0 + c);
          tm_wait_ld(o);
          if (direct) {
#pragma unroll
            for (int z = 0; z < 32; z += 8) {
              uint32_t y[4];
#pragma unroll
              for (int q = 0; q < 4; q++)
                y[q] = pack2<HALF>(__fmul_rn(__uint_as_float(o[z + 2 * q]), inv), __fmul_rn(__uint_as_float(o[z + 2 * q + 1]), inv));
              *piece(lane, (c + z) / 8) = make_uint4(y[0], y[1], y[2], y[3]);
            }
          } else {
#pragma unroll
            for (int z = 0; z < 32; z += 4) *piece(lane, (c + z) / 4) = make_uint4(o[z], o[z + 1], o[z + 2], o[z + 3]);
          }
        }
        __syncwarp();
#pragma unroll 4
        for (int rr = 0; rr < 32; rr += RS) {
          const int row = rr + lane / CH;
          uint4* to_row = reinterpret_cast<uint4*>(__shfl_sync(~0u, dst, row) + (direct ? 0 : c0 * 4));
          if ((lives >> row) & 1) to_row[ch] = *piece(row, ch);
        }
        __syncwarp();
      }
      tc_before();
    }
  }
  __syncthreads();
  if (*lost) {   // products in flight end before the CTA's memory is another's
    const long long t = clock64();
    while (clock64() - t < 20000000ll) {}
  }
  if (warp == 8) {
    tc_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem));
  }
}

template <int D, bool HALF>
cudaError_t run(const KvAttend4Args& a, const Plan& p, int sms, cudaStream_t st) {
  auto k = k_kv4_tiles<D, HALF>;
  cudaError_t e = cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, Lay<D>::SMEM);
  if (e != cudaSuccess) return e;
  // the kernel's register split has to be within what a CTA starts with
  static const int regs = [] {
    cudaFuncAttributes f;
    return cudaFuncGetAttributes(&f, k_kv4_tiles<D, HALF>) == cudaSuccess ? f.numRegs : 0;
  }();
  if (regs * 4 < 2 * R_SOFT + R_MMA + R_CONV) return cudaErrorInvalidKernelImage;
  return launch_behind(k, sms, NT, Lay<D>::SMEM, st, a, p);
}

}  // namespace

cudaError_t kv4::launch_tiles(const KvAttend4Args& a, const Plan& p, int sms, cudaStream_t st) {
  if (a.c.head_dim == 128) return a.half ? run<128, true>(a, p, sms, st) : run<128, false>(a, p, sms, st);
  return a.half ? run<64, true>(a, p, sms, st) : run<64, false>(a, p, sms, st);
}

}  // namespace rs
