// q4kv_shared_prefix_decode_attention: one query per agent over its whole cache, where groups of agents share a prefix whose keys
// are read and expanded once for the group (Section 3.4 decode; forked agents, q4kv_allocator_fork).
//
//   With the keys of an agent cut into parts i (pieces of the prefix, pieces of its own tokens), part i leaves
//   m_i = a reference for its scores, l_i = sum 2^(s - m_i), o_i = sum 2^(s - m_i) v, and
//   out = sum_i 2^(m_i - M) o_i / sum_i 2^(m_i - M) l_i with M = max m_i.
//
// The work is a list of segments: (group, tile of agents, KV head) over the prefix with up to kMaxRows score rows, then (agent, KV
// head) over its own tokens with n_rep rows.  The list is cut into equal contiguous ranges of 128-key steps, one per CTA and one CTA
// per SM; every CTA leaves a record per segment it touched and a second kernel combines an agent's records.
//
// One step is two products on the fifth-generation tensor cores with the KEYS as the 128 rows, so that the number of query rows is
// the free dimension N (16 .. 64) and few rows cost little:
//   S^T [128 keys][N] = K^ [128][d_qk] Q^T      K^ (binary16, expanded from the codes) in tensor memory, Q in shared memory
//   O^T [d_v][N]     += V^T [d_v][128] P^T      V^ and P^T (binary16) in shared memory
// A lane of tensor memory is a key: a warp that expands keys writes its own lanes (no shared-memory tile, no bank conflicts), and a
// softmax thread has one key and all rows; masks are a matter of whole lanes.  The sums l stay in the threads' registers until the
// segment ends.  What a step costs an SM: HBM 790 clocks at d = 128 (18.4 KB), tensor pipe 512 at N = 64.
//   * A warp streams raw steps into a ring by bulk copies; two warps stage the query rows of the next segment (bf16 times a power of
//     two per row into binary16, exact).
//   * Four warps expand keys, four expand values (dequant8: one binary16 fma per pair, each value rounded once).
//   * Two sets of four softmax warps share the rows, eight at a time.  The reference m of a row is the maximum over the segment's
//     first step; it moves when a probability would exceed 2^kGrow, which is found by all keys of a set together at the barrier
//     that also ends the set's stores of P.
// All waits are bounded; one that runs out raises Q4KV_FLAG_INTERNAL, lets the copies and the tensor pipe drain and gives the
// tensor memory back.
#include "prefill_common.cuh"

namespace q4kv {

namespace {

using namespace tc;
using namespace prefill;

constexpr int kMaxAgents = 512;
constexpr int kSoftmaxWarps = 8, kKeyWarp = 8, kValueWarp = 12, kLoadWarp = 16, kMmaWarp = 17, kQueryWarp = 18;
constexpr int kThreads = 20 * 32;
constexpr int kRegsSoftmax = 144, kRegsOther = 64;       // of the 96 each thread is launched with
static_assert(kSoftmaxWarps * 32 * kRegsSoftmax + (kThreads - kSoftmaxWarps * 32) * kRegsOther <= kThreads * 96, "");
constexpr float kGrow = 14.f;                            // probabilities up to 2^14 (binary16 ends at 65504)
constexpr int kInfo = 8;                                 // segments that the loader may be ahead of the softmax
constexpr int kSegmentCost = 1;                          // of a segment beside its steps, in steps
constexpr uint32_t kColS = 0;                            // tensor-memory columns: S^T 2 x kRows, O^T, K^

template <int G, int Gv>
struct Shape {
  static constexpr int D = 64 * G, Dv = 64 * Gv;
  static constexpr int kRows = G == 2 ? 64 : 32;         // score rows of a segment at most
  static constexpr int kOffKsb = 16 * D, kOffVc = kOffKsb + 128 * G, kOffVsb = kOffVc + 16 * Dv;
  static constexpr int kChunkBytes = kOffVsb + 128 * Gv, kRawBytes = 4 * kChunkBytes;      // a step: 128 keys
  static constexpr int kRaw = G == 4 ? 2 : 4;            // raw steps in flight
  static constexpr int kStagesV = G == 4 ? 1 : 2;
  static constexpr int kTileV = Dv * 128;                // 64 keys of V^, bytes
  static constexpr int kQueryBytes = kRows * D * 2, kProbBytes = kRows * 128 * 2;
  static constexpr int kSboQ = (D / 8) * 128;
  static constexpr uint32_t kColO = 2 * kRows, kColK = kColO + kRows * (Dv / 128);         // K^: two stages of D / 2 columns
  static_assert(kColK + D <= 512, "");
  static constexpr int kRecord = kRows * Dv;             // floats of a prefix record's o
};

// What the work list looks like; the merge reads the copy that the first CTA leaves in the workspace.
struct Plan {
  int total, n_cta, suffix_base;                         // cost of the whole list, CTAs it is cut for, where the agents' own parts begin
  int pre_start[kMaxAgents + 1], prefix[kMaxAgents], lead[kMaxAgents], offs[kMaxAgents + 1], tile0[kMaxAgents];   // per group
  int suf_start[kMaxAgents + 1], kv_len[kMaxAgents];     // per agent; 0: nothing to attend
  short group[kMaxAgents];
};

struct Params {
  Layout y;
  const uint8_t* pool;
  int n_blocks, layer, n_agents, max_blocks;
  const int32_t* tables;
  const int32_t* kv_lens;
  int max_kv_len;
  const int32_t* group_offs;
  const int32_t* prefix_lens;
  int n_groups;
  const uint16_t* q;
  float scale_log2;
  void* out;
  int out_dtype;
  float* lse;
  int32_t* flags;
  Plan* plan;
  float* pre_o;               // [record][row][d_v]
  float2* pre_ml;             // [record][row]
  float* suf_o;               // [record][n_rep][d_v]
  float2* suf_ml;
  CodeMasks masks;
};

__host__ __device__ inline int steps_of(int prefix) { return (prefix + 127) >> 7; }
__host__ __device__ inline int own_steps(int kv_len, int prefix) { return kv_len > prefix ? ((kv_len + 127) >> 7) - (prefix >> 7) : 0; }
__device__ inline int cost_of(int steps) { return steps > 0 ? steps + kSegmentCost : 0; }
// agents of a tile: at most `most`, the tiles of a group as equal as can be
__host__ __device__ inline int tiles_of(int agents, int most) { return (agents + most - 1) / most; }
__device__ inline int cut(const Plan& p, int c) { return (int)((long long)p.total * c / p.n_cta); }
// the CTA whose range holds position u of the list
__device__ inline int cta_of(const Plan& p, int u) { return (int)(((long long)(u + 1) * p.n_cta - 1) / p.total); }

// One CTA's part of a segment.
struct Segment {
  int prefix;                                            // 1: a group's prefix, 0: an agent's own tokens
  int agent0, n_agents, lead, head;                      // rows: agents agent0 .. x n_rep heads of KV head `head`; keys: of agent `lead`
  int key0, key1;                                        // the segment's keys
  int step0, steps;                                      // 128-key steps of this CTA; steps == 0: there is no more
  int record;
};

// Walks the segments of the range [u0, u1) in order.  The loader does, and hands them to the other roles.
struct Walker {
  const Plan* p;
  int n_groups, n_agents, heads, most, cta, u0, u1;
  int which, tile_head;                                  // group or agent, and (tile, head) or head in it
  bool in_prefix;
  __device__ void begin(const Plan* plan, const Params& P, int max_rows, int c) {
    p = plan;
    n_groups = P.n_groups; n_agents = P.n_agents; heads = P.y.Hkv; most = max_rows / P.y.n_rep;
    cta = c;
    u0 = c < p->n_cta ? cut(*p, c) : 0;
    u1 = c < p->n_cta ? cut(*p, c + 1) : 0;
    in_prefix = u0 < p->suffix_base;
    const int* start = in_prefix ? p->pre_start : p->suf_start;
    const int at = in_prefix ? u0 : u0 - p->suffix_base;
    int lo = 0, hi = in_prefix ? n_groups : n_agents;    // the last entry that begins at or before the position
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (start[mid] <= at) lo = mid; else hi = mid;
    }
    which = lo;
    const int len = length();
    tile_head = len > 0 ? (at - start[which]) / len - 1 : -1;              // next() begins with a step forward
  }
  __device__ int length() const {
    return in_prefix ? (p->pre_start[which + 1] > p->pre_start[which] ? cost_of(steps_of(p->prefix[which])) : 0)
                     : (p->suf_start[which + 1] - p->suf_start[which]) / heads;
  }
  __device__ bool next(Segment& s) {
    if (u0 >= u1) return false;
    for (;;) {
      ++tile_head;
      int start;
      if (in_prefix) {
        while (which < n_groups && p->pre_start[which] + tile_head * length() >= p->pre_start[which + 1]) { ++which; tile_head = 0; }
        if (which == n_groups) { in_prefix = false; which = 0; tile_head = -1; continue; }
        start = p->pre_start[which] + tile_head * length();
        s.prefix = 1;
        s.key0 = 0;
        s.key1 = p->prefix[which];
        s.lead = p->lead[which];
        s.head = tile_head % heads;
        const int n = p->offs[which + 1] - p->offs[which], t = tile_head / heads, tiles = tiles_of(n, most);
        const int a = n * t / tiles;
        s.agent0 = p->offs[which] + a;
        s.n_agents = n * (t + 1) / tiles - a;
        s.step0 = 0;
        s.record = p->tile0[which] * heads + tile_head + cta;
      } else {
        while (which < n_agents && p->suf_start[which] + tile_head * length() >= p->suf_start[which + 1]) { ++which; tile_head = 0; }
        if (which == n_agents) return false;
        start = p->suffix_base + p->suf_start[which] + tile_head * length();
        s.prefix = 0;
        s.key0 = p->prefix[p->group[which]];
        s.key1 = p->kv_len[which];
        s.lead = s.agent0 = which;
        s.n_agents = 1;
        s.head = tile_head;
        s.step0 = s.key0 >> 7;
        s.record = which * heads + tile_head + cta;
      }
      if (start >= u1) return false;
      const int all = s.prefix ? steps_of(s.key1) : own_steps(s.key1, s.key0);
      const int first = max(0, u0 - start), last = min(all, u1 - start);
      if (first >= last) continue;                       // this CTA's part is the segment's fixed cost
      s.step0 += first;
      s.steps = last - first;
      return true;
    }
  }
};

// The plan in shared memory, by the whole CTA.
__device__ void make_plan(const Params& P, Plan& p, int max_rows) {
  const int G = P.n_groups, A = P.n_agents, heads = P.y.Hkv, most = max_rows / P.y.n_rep, tid = threadIdx.x;
  bool ok = true;
  for (int g = tid; g <= G; g += blockDim.x) {
    const int lo = P.group_offs[g];
    p.offs[g] = lo;
    ok = ok && lo >= 0 && lo <= A && (g == G || P.group_offs[g + 1] >= lo);
    if (g < G) {
      p.prefix[g] = P.prefix_lens[g];
      p.lead[g] = INT32_MAX;
    }
  }
  ok = __syncthreads_and(ok) != 0;
  bool bad = false;
  for (int a = tid; a < A; a += blockDim.x) {
    int lo = 0, hi = G;
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (p.offs[mid] <= a) lo = mid; else hi = mid;
    }
    const int kv = P.kv_lens[a], prefix = p.prefix[lo];
    const bool fine = ok && G > 0 && p.offs[lo] <= a && a < p.offs[lo + 1] && prefix >= 0 && prefix <= P.max_kv_len && kv >= 0 &&
                      kv <= P.max_kv_len && (kv == 0 || kv >= prefix);
    const bool live = fine && kv > 0;
    bad |= !fine;
    p.group[a] = (short)(live ? lo : -1);
    p.kv_len[a] = live ? kv : 0;
    if (live) atomicMin(&p.lead[lo], a);
  }
  if (bad && blockIdx.x == 0) raise_flag(P.flags, Q4KV_FLAG_BAD_LENGTH);
  __syncthreads();
  const int warp = tid >> 5, lane = tid & 31;
  if (warp < 2) {                                        // running sums: of the groups' cost and tiles, of the agents' cost
    const int n = warp == 0 ? G : A;
    int sum = 0, tiles_sum = 0;
    for (int base = 0; base < n; base += 32) {
      const int i = base + lane;
      int cost = 0, tiles = 0;
      if (i < n) {
        if (warp == 0) {
          const int agents = ok ? p.offs[i + 1] - p.offs[i] : 0;
          tiles = tiles_of(agents, most);
          cost = p.lead[i] == INT32_MAX ? 0 : tiles * heads * cost_of(steps_of(p.prefix[i]));
        } else {
          cost = p.kv_len[i] > 0 ? heads * cost_of(own_steps(p.kv_len[i], p.prefix[p.group[i]])) : 0;
        }
      }
      int c = cost, t = tiles;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int cu = __shfl_up_sync(0xffffffffu, c, o), tu = __shfl_up_sync(0xffffffffu, t, o);
        if (lane >= o) { c += cu; t += tu; }
      }
      if (i < n) {
        if (warp == 0) { p.pre_start[i] = sum + c - cost; p.tile0[i] = tiles_sum + t - tiles; }
        else p.suf_start[i] = sum + c - cost;
      }
      sum += __shfl_sync(0xffffffffu, c, 31);
      tiles_sum += __shfl_sync(0xffffffffu, t, 31);
    }
    if (lane == 0) {
      if (warp == 0) p.pre_start[G] = sum; else p.suf_start[A] = sum;
    }
  }
  __syncthreads();
  if (tid == 0) {
    p.suffix_base = p.pre_start[G];
    p.total = p.suffix_base + p.suf_start[A];
    p.n_cta = min((int)gridDim.x, max(1, p.total));
  }
  __syncthreads();
}

template <int G, int Gv>
struct Smem {
  using Sh = Shape<G, Gv>;
  alignas(128) uint8_t vhat[Sh::kStagesV][2 * Sh::kTileV];     // [half][dim][key 64]: (n%8)*16 + (n/8)*1024 + (k/8)*128
  alignas(128) uint8_t raw[Sh::kRaw][Sh::kRawBytes];
  alignas(128) uint8_t qs[2][Sh::kQueryBytes];                 // [row][dim]: (r%8)*16 + (r/8)*kSboQ + (k/8)*128
  alignas(128) uint8_t prob[2][Sh::kProbBytes];                // [key][row]: (k%8)*16 + (k/8)*128 + (r/8)*2048 + (r%8)*2
  alignas(16) float kappa[2][Sh::kRows];                       // score in log2 units = S * kappa
  // of the two softmax sets: minus the reference of each row, what to scale by when it moves, partial maxima and sums
  alignas(16) float neg_ref[2][Sh::kRows / 2], factor[2][Sh::kRows / 2], red_max[2][4][Sh::kRows / 2], red_sum[2][4][Sh::kRows / 2];
  alignas(8) uint64_t raw_full[Sh::kRaw], raw_free[Sh::kRaw];
  uint64_t k_full[2], s_full[2], p_full[2], o_done[2], q_full[2], q_free[2], info_full[kInfo], info_free[kInfo], drain;
  Segment info[kInfo];
  uint32_t tmem_base;
  int bad[Sh::kRaw], poisoned[kInfo];                          // poisoned: a bad block in the segment
  int abort_flag;
  Plan plan;
};

__device__ inline bool set_any(int set, bool v) {        // over the 128 threads of a softmax set; orders their stores
  uint32_t r;
  asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %1, 0;\n\tbarrier.cta.red.or.pred q, %2, 128, p;\n\tselp.u32 %0, 1, 0, q;\n\t}"
               : "=r"(r) : "r"((uint32_t)v), "r"(1 + set) : "memory");
  return r != 0;
}
__device__ inline void set_sync(int set) { asm volatile("barrier.cta.sync %0, 128;" ::"r"(1 + set) : "memory"); }
__device__ inline float warp_max(float v) {             // (a NaN does not count)
  float r;
  asm volatile("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(r) : "f"(v));
  return r;
}
__device__ inline float warp_sum(float v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}
// The sums over a warp of kCount columns, lane c (mod kCount) getting column c's: halves change hands, then quarters, ...
template <int kCount>
__device__ inline float column_sums(float (&v)[kCount]) {
  const int lane = threadIdx.x & 31;
  if (kCount == 16) {
#pragma unroll
    for (int c = 0; c < kCount; ++c) v[c] += __shfl_xor_sync(0xffffffffu, v[c], 16);
  }
#pragma unroll
  for (int o = kCount / 2; o > 0; o >>= 1) {
    const bool high = lane & o;
#pragma unroll
    for (int c = 0; c < o; ++c) v[c] = (high ? v[c + o] : v[c]) + __shfl_xor_sync(0xffffffffu, high ? v[c] : v[c + o], o);
  }
  return v[0];
}

template <int G, int Gv, bool kBf>
__global__ void __launch_bounds__(kThreads, 1) shared_prefix_kernel(const __grid_constant__ Params P) {
  using Sh = Shape<G, Gv>;
  constexpr int D = Sh::D, Dv = Sh::Dv, kRows = Sh::kRows, kRaw = Sh::kRaw, kStagesV = Sh::kStagesV;
  constexpr int kGroups = kRows / 16;                    // groups of eight rows of a softmax set
  extern __shared__ __align__(128) uint8_t smem_raw[];
  Smem<G, Gv>& sm = *reinterpret_cast<Smem<G, Gv>*>(smem_raw);
  const Layout& y = P.y;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  if (threadIdx.x == 0) {
    for (int s = 0; s < kRaw; ++s) { mbar_init(&sm.raw_full[s], 1); mbar_init(&sm.raw_free[s], 8); sm.bad[s] = 0; }
    for (int s = 0; s < 2; ++s) {
      mbar_init(&sm.k_full[s], 4); mbar_init(&sm.s_full[s], 1); mbar_init(&sm.p_full[s], 6); mbar_init(&sm.o_done[s], 1);
      mbar_init(&sm.q_full[s], 64); mbar_init(&sm.q_free[s], 3);
    }
    for (int s = 0; s < kInfo; ++s) { mbar_init(&sm.info_full[s], 1); mbar_init(&sm.info_free[s], 2); }
    mbar_init(&sm.drain, 1);
    sm.abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    fence_async_smem();
  }
  if (warp == kMmaWarp) { tmem_alloc(&sm.tmem_base, 512); tmem_relinquish(); }
  make_plan(P, sm.plan, kRows);
  fence_before_sync();
  __syncthreads();
  fence_after_sync();
  const uint32_t tb = sm.tmem_base;
  asm volatile("griddepcontrol.wait;" ::: "memory");     // the pool, the queries and the workspace are the preceding kernels' until here
  if (blockIdx.x == 0) {
    const int* from = reinterpret_cast<const int*>(&sm.plan);
    for (int i = threadIdx.x; i < (int)(sizeof(Plan) / 4); i += kThreads) reinterpret_cast<int*>(P.plan)[i] = from[i];
  }
  volatile int* abort_flag = &sm.abort_flag;
  int g = 0;                                             // steps so far

  if (warp >= kLoadWarp) {
    fewer_registers<kRegsOther>();
    if (warp == kLoadWarp) {
      // =============================== segments and raw steps =====================================
      if (lane == 0) {
        Walker w;
        w.begin(&sm.plan, P, kRows, blockIdx.x);
        bool more = true;
        for (int n = 0; more; ++n) {
          Segment s;
          more = w.next(s);
          if (!more) s.steps = 0;
          if (n >= kInfo && !mbar_wait(&sm.info_free[n % kInfo], (uint32_t)(n / kInfo - 1), abort_flag)) break;
          sm.info[n % kInfo] = s;
          sm.poisoned[n % kInfo] = 0;
          mbar_arrive(&sm.info_full[n % kInfo]);
          const uint8_t* row = head_block(P.pool, y, P.layer, 0, s.head);
          for (int j = 0; j < s.steps; ++j, ++g) {
            const int r = g % kRaw, step = s.step0 + j;
            if (g >= kRaw && !mbar_wait(&sm.raw_free[r], (uint32_t)(g / kRaw - 1), abort_flag)) { more = false; break; }
            const int blk = P.tables[(size_t)s.lead * P.max_blocks + (step >> 1)];
            sm.bad[r] = blk < 0 || blk >= P.n_blocks;
            if (sm.bad[r]) {
              sm.poisoned[n % kInfo] = 1;
              raise_flag(P.flags, Q4KV_FLAG_BAD_BLOCK);
              mbar_arrive(&sm.raw_full[r]);
            } else {
              mbar_arrive_expect_tx(&sm.raw_full[r], Sh::kRawBytes);
              bulk_load(sm.raw[r], row + (uint64_t)blk * y.block_bytes + (size_t)(step & 1) * Sh::kRawBytes, Sh::kRawBytes, &sm.raw_full[r]);
            }
          }
        }
        // a CTA that is giving up still lets its own copies land before shared memory is released
        if (*abort_flag)
          for (int j = max(0, g - kRaw); j < g; ++j)
            for (uint32_t i = 0; i < kSpinLimit && !mbar_try_wait(&sm.raw_full[j % kRaw], (uint32_t)(j / kRaw) & 1u); ++i) {}
      }
    } else if (warp == kMmaWarp) {
      // =============================== products ===================================================
      // A product's commit also covers what was issued before it: S^T of a step implies O^T of the step two before, so neither the
      // buffers of P^T nor those of S^T and K^ need barriers of their own.  The value tile's warps arrive where the softmax does.
      auto wait = [&](uint64_t* bar, int use) {
        const bool ok = mbar_spin(bar, (uint32_t)use, abort_flag);
        if (ok) fence_after_sync();
        return ok;
      };
      const uint64_t vd0 = smem_desc(smem_u32(sm.vhat[0]), 128, 1024), pd0 = smem_desc(smem_u32(sm.prob[0]), 128, 2048);
      const uint64_t qd0 = smem_desc(smem_u32(sm.qs[0]), 128, Sh::kSboQ);
      bool first = true;
      uint32_t idesc_pv = 0;                             // of the step whose value product is due
      auto issue_pv = [&](int h) {                       // O^T (+)= V^T P^T of step h
        const uint64_t vd = vd0 + (uint64_t)((h % kStagesV) * (2 * Sh::kTileV >> 4)), pd = pd0 + (uint64_t)((h & 1) * (Sh::kProbBytes >> 4));
        if (elect_one()) {
#pragma unroll
          for (int m = 0; m < Dv / 128; ++m)
#pragma unroll
            for (int k = 0; k < 8; ++k)
              mma_f16_ss(tb + Sh::kColO + kRows * m, vd + (uint64_t)((k >> 2) * (Sh::kTileV >> 4) + m * 1024 + (k & 3) * 16), pd + 16 * k, idesc_pv,
                         (!first || k > 0) ? 1u : 0u);
          commit(&sm.o_done[h & 1]);
        }
        __syncwarp();
      };
      bool ok = true;
      for (int n = 0; ok; ++n) {
        const int slot = n & 1;
        ok = wait(&sm.q_full[slot], n >> 1);
        const int steps = ok ? sm.info[n % kInfo].steps : 0, columns = ok ? (sm.info[n % kInfo].n_agents * y.n_rep + 15) & ~15 : 0;
        const uint32_t size = (uint32_t)(columns >> 3) << 17;
        const uint64_t qd = qd0 + (uint64_t)(slot * (Sh::kQueryBytes >> 4));
        for (int j = 0; ok && (j < steps || (steps == 0 && j == 0)); ++j) {
          if (steps > 0) {
            ok = wait(&sm.k_full[g & 1], g >> 1);
            if (!ok) break;
            if (elect_one()) {
#pragma unroll
              for (int k = 0; k < D / 16; ++k)
                mma_f16_ts(tb + kColS + kRows * (g & 1), tb + Sh::kColK + (D / 2) * (g & 1) + 8 * k, qd + 16 * k, idesc_f16(128, 0) | size, k > 0);
              commit(&sm.s_full[g & 1]);
              if (j == steps - 1) commit(&sm.q_free[slot]);
            }
            __syncwarp();
          }
          if (g > 0) {                                   // the step before, also behind the last segment
            ok = wait(&sm.p_full[(g - 1) & 1], (g - 1) >> 1);
            if (ok) issue_pv(g - 1);
          }
          first = j == 0;
          idesc_pv = idesc_f16(128, 0, 0, 1) | size;
          ++g;
        }
        if (steps == 0) break;
      }
    } else {
      // =============================== query rows =================================================
      constexpr int kLanes = D == 128 ? 16 : 32, kAtOnce = 8, kStride = 2 * (32 / kLanes);     // lanes of a row, rows in flight, rows of both warps
      const int piece = lane % kLanes, sub = (warp - kQueryWarp) * (32 / kLanes) + lane / kLanes;
      for (int n = 0;; ++n) {
        const int slot = n & 1;
        if (!mbar_wait(&sm.info_full[n % kInfo], (uint32_t)(n / kInfo), abort_flag)) break;
        const Segment& s = sm.info[n % kInfo];
        const int steps = s.steps, rows = s.n_agents * y.n_rep, padded = steps > 0 ? (rows + 15) & ~15 : 0;
        const uint16_t* q = P.q + ((size_t)s.agent0 * y.Hq + (size_t)s.head * y.n_rep) * D + 8 * piece;
        if (n >= 2 && !mbar_wait(&sm.q_free[slot], (uint32_t)((n >> 1) - 1), abort_flag)) break;
        for (int base = sub; base < padded; base += kStride * kAtOnce) {
          uint4 v[kAtOnce];
#pragma unroll
          for (int u = 0; u < kAtOnce; ++u) {
            const int r = base + kStride * u, a = r / y.n_rep;
            v[u] = make_uint4(0u, 0u, 0u, 0u);
            if (r < rows && piece < D / 8) v[u] = *reinterpret_cast<const uint4*>(q + ((size_t)a * y.Hq + (r - a * y.n_rep)) * D);
          }
#pragma unroll
          for (int u = 0; u < kAtOnce; ++u) {
            const int r = base + kStride * u;
            float mx = max_abs8(v[u]);
#pragma unroll
            for (int o = kLanes / 2; o > 0; o >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, o, kLanes));
            int ex = (int)((__float_as_uint(mx) >> 23) & 255u) - 127;
            if (mx == 0.f) ex = 0;
            ex = min(max(ex, -100), 100);
            const float sf = __uint_as_float((uint32_t)(127 + 8 - ex) << 23);          // 256 <= max |q| * sf < 512
            if (r < padded) {
              if (piece == 0) sm.kappa[slot][r] = P.scale_log2 * __uint_as_float((uint32_t)(127 - 8 + ex) << 23);
              if (piece < D / 8) *reinterpret_cast<uint4*>(sm.qs[slot] + (r & 7) * 16 + (r >> 3) * Sh::kSboQ + piece * 128) = query8(v[u], sf);
            }
          }
        }
        fence_async_smem();
        mbar_arrive(&sm.q_full[slot]);
        if (steps == 0) break;
      }
    }
  } else if (warp >= kValueWarp) {
    fewer_registers<kRegsOther>();
    // =============================== values into shared memory ==================================
    const int x7 = threadIdx.x - kValueWarp * 32;
    // one 16-byte piece (dims 32 vq + 8 k + vr, k = 0..3) of token octet vo of a chunk; at d_v = 256 vq + 4 as well
    const int vr = x7 & 7, vq = (x7 >> 3) & 3, vo = ((vr >> 1) + (x7 >> 5)) & 3;
    const int v_read = Sh::kOffVc + ((vq * 8 + vr) * 4 + vo) * 16, v_write = vr * 16 + (4 * vq) * 1024 + vo * 128;
    const int v_sb = Sh::kOffVsb + (vo * 2 * Gv + (vq >> 1)) * 4;           // + (i * 8 + e) * Gv * 4: token 8 vo + 4 e + i
    for (int n = 0; mbar_wait(&sm.info_full[n % kInfo], (uint32_t)(n / kInfo), abort_flag); ++n) {
      const int key0 = sm.info[n % kInfo].key0, key1 = sm.info[n % kInfo].key1, step0 = sm.info[n % kInfo].step0, steps = sm.info[n % kInfo].steps;
      bool go = steps > 0;
      for (int j = 0; go && j < steps; ++j, ++g) {
        const int r = g % kRaw, sv = g % kStagesV;
        go = mbar_wait(&sm.raw_full[r], (uint32_t)(g / kRaw), abort_flag) &&
             (g < kStagesV || mbar_wait(&sm.o_done[(g - kStagesV) & 1], (uint32_t)((g - kStagesV) >> 1), abort_flag));
        if (!go) break;
        const bool bad = sm.bad[r] != 0;
        bool over = false;
#pragma unroll 1
        for (int c = 0; c < 4; ++c) {
          const uint8_t* chunk = sm.raw[r] + c * Sh::kChunkBytes;
          const int at = (step0 + j) * 128 + c * 32, pos = at + 8 * vo;
          const bool edge = bad || at < key0 || at + 32 > key1;              // some of its bytes are none of the segment's
#pragma unroll
          for (int half = 0; half < Gv / 2; ++half) {
            const uint4 vw = *reinterpret_cast<const uint4*>(chunk + v_read + half * (4 * 8 * 4 * 16));
            uint32_t e[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) e[i] = *reinterpret_cast<const uint32_t*>(chunk + v_sb + half * 8 + ((i & 3) * 8 + (i >> 2)) * Gv * 4);
            if (edge) {
#pragma unroll
              for (int i = 0; i < 8; ++i)
                if (bad || pos + i < key0 || pos + i >= key1) e[i] = 0u;
            }
            uint32_t sp[4], bp[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              if (kBf) { e[i] = bf16_pair_to_h2(e[i], over); e[i + 4] = bf16_pair_to_h2(e[i + 4], over); }
              sp[i] = __byte_perm(e[i], e[i + 4], 0x5410);
              bp[i] = __byte_perm(e[i], e[i + 4], 0x7632);
            }
            uint8_t* dst = sm.vhat[sv] + v_write + (c >> 1) * Sh::kTileV + (c & 1) * 512 + half * 16384;
            *reinterpret_cast<uint4*>(dst + 0 * 1024) = dequant8(vw.x, sp[0], bp[0], sp[1], bp[1], sp[2], bp[2], sp[3], bp[3], P.masks);
            *reinterpret_cast<uint4*>(dst + 1 * 1024) = dequant8(vw.y, sp[0], bp[0], sp[1], bp[1], sp[2], bp[2], sp[3], bp[3], P.masks);
            *reinterpret_cast<uint4*>(dst + 2 * 1024) = dequant8(vw.z, sp[0], bp[0], sp[1], bp[1], sp[2], bp[2], sp[3], bp[3], P.masks);
            *reinterpret_cast<uint4*>(dst + 3 * 1024) = dequant8(vw.w, sp[0], bp[0], sp[1], bp[1], sp[2], bp[2], sp[3], bp[3], P.masks);
          }
        }
        if (kBf && over) raise_flag(P.flags, Q4KV_FLAG_SB_RANGE);
        fence_async_smem();
        __syncwarp();
        if (lane == 0) { mbar_arrive(&sm.p_full[g & 1]); mbar_arrive(&sm.raw_free[r]); }
      }
      if (!go) break;
    }
  } else if (warp >= kKeyWarp) {
    fewer_registers<kRegsOther>();
    // =============================== keys into tensor memory ====================================
    // Lane l of warp c holds token tau = 8 (l / 8) + elem_of(l % 8) of chunk c, so that lanes follow the order of V^'s keys.  A token's
    // words 16 j + 4 m + t lie in four 16-byte pieces t; lane l begins with piece l / 2 % 4 (no bank conflicts) and turns them back.
    const int c = warp - kKeyWarp, tau = 8 * (lane >> 3) + elem_of(lane & 7), ti = tau & 3, tg = tau >> 2, rot = (lane >> 1) & 3;
    const int k_read = c * Sh::kChunkBytes + ti * (256 * G) + tg * 64;      // + j * 512 + piece * 16
    const int k_sb = c * Sh::kChunkBytes + Sh::kOffKsb + ((ti * 4 + (tau >> 3)) * 2 + ((tau >> 2) & 1)) * G * 4;
    const uint32_t lane_addr = tb + ((uint32_t)(c * 32) << 16) + Sh::kColK;
    auto turned = [&](uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t* out) {      // out[t] = what came as number (t - rot) & 3
      const bool one = rot & 1, two = rot & 2;
      const uint32_t b0 = one ? a3 : a0, b1 = one ? a0 : a1, b2 = one ? a1 : a2, b3 = one ? a2 : a3;
      out[0] = two ? b2 : b0; out[1] = two ? b3 : b1; out[2] = two ? b0 : b2; out[3] = two ? b1 : b3;
    };
    for (int n = 0; mbar_wait(&sm.info_full[n % kInfo], (uint32_t)(n / kInfo), abort_flag); ++n) {
      const int key0 = sm.info[n % kInfo].key0, key1 = sm.info[n % kInfo].key1, step0 = sm.info[n % kInfo].step0, steps = sm.info[n % kInfo].steps;
      bool go = steps > 0;
      for (int j = 0; go && j < steps; ++j, ++g) {
        const int r = g % kRaw;
        go = mbar_wait(&sm.raw_full[r], (uint32_t)(g / kRaw), abort_flag) &&
             (g < 2 || mbar_wait(&sm.s_full[g & 1], (uint32_t)((g >> 1) - 1), abort_flag));
        if (!go) break;
        fence_after_sync();
        const int pos = (step0 + j) * 128 + c * 32 + tau;
        const bool none = sm.bad[r] != 0 || pos < key0 || pos >= key1;
        const uint8_t* raw = sm.raw[r];
        uint32_t sb[G];
        bool over = false;
#pragma unroll
        for (int i = 0; i < G; ++i) {
          sb[i] = none ? 0u : *reinterpret_cast<const uint32_t*>(raw + k_sb + 4 * i);
          if (kBf) sb[i] = bf16_pair_to_h2(sb[i], over);
        }
        if (kBf && over) raise_flag(P.flags, Q4KV_FLAG_SB_RANGE);
        const uint32_t to = lane_addr + (D / 2) * (g & 1);
        auto expand = [&](const uint32_t* words, uint32_t e, uint32_t at) {          // four words of one group: 16 columns
          const uint32_t s2 = __byte_perm(e, e, 0x1010), b2 = __byte_perm(e, e, 0x3232);
          uint32_t col[16];
#pragma unroll
          for (int t = 0; t < 4; ++t) {
            const uint4 v = dequant8(words[t], s2, b2, P.masks);
            col[4 * t] = v.x; col[4 * t + 1] = v.y; col[4 * t + 2] = v.z; col[4 * t + 3] = v.w;
          }
          tmem_st16(to + at, col);
        };
#pragma unroll
        for (int jj = 0; jj < G / 2; ++jj) {
          uint4 p[4];
#pragma unroll
          for (int t = 0; t < 4; ++t) p[t] = *reinterpret_cast<const uint4*>(raw + k_read + jj * 512 + ((t + rot) & 3) * 16);
          uint32_t wd[4];
          turned(p[0].x, p[1].x, p[2].x, p[3].x, wd); expand(wd, sb[2 * jj], 64 * jj);
          turned(p[0].y, p[1].y, p[2].y, p[3].y, wd); expand(wd, sb[2 * jj], 64 * jj + 16);
          turned(p[0].z, p[1].z, p[2].z, p[3].z, wd); expand(wd, sb[2 * jj + 1], 64 * jj + 32);
          turned(p[0].w, p[1].w, p[2].w, p[3].w, wd); expand(wd, sb[2 * jj + 1], 64 * jj + 48);
        }
        if (G & 1) {                                     // the last group: 8-byte pieces, words 16 + 4 m + t, m = 0, 1
          uint2 p[4];
          const int at = c * Sh::kChunkBytes + ti * (256 * G) + (G / 2) * 512 + tg * 32;
#pragma unroll
          for (int t = 0; t < 4; ++t) p[t] = *reinterpret_cast<const uint2*>(raw + at + ((t + rot) & 3) * 8);
          uint32_t wd[4];
          turned(p[0].x, p[1].x, p[2].x, p[3].x, wd); expand(wd, sb[G - 1], 32 * (G - 1));
          turned(p[0].y, p[1].y, p[2].y, p[3].y, wd); expand(wd, sb[G - 1], 32 * (G - 1) + 16);
        }
        wait_st();
        fence_before_sync();
        __syncwarp();
        if (lane == 0) { mbar_arrive(&sm.k_full[g & 1]); mbar_arrive(&sm.raw_free[r]); }
      }
      if (!go) break;
    }
  } else {
    more_registers<kRegsSoftmax>();
    // =============================== softmax: a thread has one key and half of the segment's rows ==============
    // (inside a segment no thread leaves early: after an abort every wait returns at once, and the barriers stay even)
    const int set = warp >> 2, quad = warp & 3;
    const uint32_t lane_addr = tb + ((uint32_t)(quad * 32) << 16);
    const int key = quad * 32 + 8 * (lane >> 3) + elem_of(lane & 7);       // of the step
    const int tid = threadIdx.x & 127;
    float* const neg_ref = sm.neg_ref[set];
    float* const factor = sm.factor[set];
    for (int n = 0;; ++n) {
      const int slot = n & 1;
      bool lost = false;
      if (quad == set) lost = !mbar_spin(&sm.q_full[slot], (uint32_t)(n >> 1), abort_flag);
      if (set_any(set, lost)) break;
      const Segment s = sm.info[n % kInfo];
      if (s.steps == 0) break;
      const int rows = s.n_agents * y.n_rep, first = set * (((rows + 15) & ~15) >> 1);
      const int mine = min(max((rows - first + 7) >> 3, 0), ((rows + 15) & ~15) >> 4);       // groups of eight rows, from row `first` on
      const float* kap = sm.kappa[slot] + first;
      uint64_t l[4 * kGroups];
#pragma unroll
      for (int c = 0; c < 4 * kGroups; ++c) l[c] = 0ull;
      bool started = false;
#pragma unroll 1
      for (int j = 0; j < s.steps; ++j, ++g) {
        const int b = g & 1;
        if (quad == set) mbar_spin(&sm.s_full[b], (uint32_t)(g >> 1), abort_flag);
        set_sync(set);
        fence_after_sync();
        const int pos = (s.step0 + j) * 128 + key;
        const bool valid = pos >= s.key0 && pos < s.key1;
        const bool edge = (s.step0 + j) * 128 < s.key0 || (s.step0 + j) * 128 + 128 > s.key1;
        const uint32_t s_addr = lane_addr + kColS + kRows * b + first;
        uint8_t* const p_at = sm.prob[b] + (quad * 32 + lane) * 16 + (first >> 3) * 2048;
        uint64_t p[4 * kGroups];
        bool grown = false;
#pragma unroll 1
        for (;;) {
          if (started) {
            uint32_t x[8 * kGroups];
            float most = -INFINITY;
#pragma unroll
            for (int i = 0; i < kGroups; ++i)
              if (i < mine) tmem_ld8(s_addr + 8 * i, x + 8 * i);
            if (kGroups == 4) wait_ld32(x); else wait_ld16(x);
            if (edge && !valid) {
#pragma unroll
              for (int c = 0; c < 8 * kGroups; ++c) x[c] = 0xff800000u;
            }
#pragma unroll
            for (int i = 0; i < kGroups; ++i) {
              if (i < mine) {
                uint32_t h[4];
#pragma unroll
                for (int c = 0; c < 4; c += 2) {
                  const ulonglong2 kk = *reinterpret_cast<const ulonglong2*>(kap + 8 * i + 2 * c), rr = *reinterpret_cast<const ulonglong2*>(neg_ref + 8 * i + 2 * c);
                  const float2 t0 = unpair64(fma2(pair64(__uint_as_float(x[8 * i + 2 * c]), __uint_as_float(x[8 * i + 2 * c + 1])), kk.x, rr.x));
                  const float2 t1 = unpair64(fma2(pair64(__uint_as_float(x[8 * i + 2 * c + 2]), __uint_as_float(x[8 * i + 2 * c + 3])), kk.y, rr.y));
                  most = fmaxf(fmaxf(most, t0.x), t0.y);
                  most = fmaxf(fmaxf(most, t1.x), t1.y);
                  const float a0 = fast_exp2(t0.x), a1 = fast_exp2(t0.y), b0 = fast_exp2(t1.x), b1 = fast_exp2(t1.y);
                  p[4 * i + c] = pair64(a0, a1);
                  p[4 * i + c + 1] = pair64(b0, b1);
                  h[c] = f32x2_to_h2(a0, a1);
                  h[c + 1] = f32x2_to_h2(b0, b1);
                }
                *reinterpret_cast<uint4*>(p_at + i * 2048) = make_uint4(h[0], h[1], h[2], h[3]);
              }
            }
            fence_async_smem();
            fence_before_sync();
            if (!set_any(set, most > kGrow) || grown) break;
          } else if (mine == 0) {
            break;
          }
          // the references of the rows that outgrow theirs (of all, in the first step) move to the maximum of this step's scores; the
          // others' stay, so that no row's numbers depend on another's
#pragma unroll 1
          for (int i = 0; i < mine; ++i) {
            uint32_t x[8];
            tmem_ld8(s_addr + 8 * i, x);
            wait_ld8(x);
#pragma unroll
            for (int c = 0; c < 8; ++c) {
              const float m = warp_max(valid ? __uint_as_float(x[c]) * kap[8 * i + c] : -INFINITY);
              if (lane == 0) sm.red_max[set][quad][8 * i + c] = m;
            }
          }
          if (started && quad == set) mbar_spin(&sm.o_done[b ^ 1], (uint32_t)((g - 1) >> 1), abort_flag);     // O^T so far is complete
          set_sync(set);
          if (quad == 0 && lane < 8 * mine) {
            const float m = fmaxf(fmaxf(sm.red_max[set][0][lane], sm.red_max[set][1][lane]), fmaxf(sm.red_max[set][2][lane], sm.red_max[set][3][lane]));
            const float old = started ? -neg_ref[lane] : 0.f;
            const float to = started && !(m - old > kGrow) ? old : m > -INFINITY ? m : 0.f;
            neg_ref[lane] = -to;
            factor[lane] = fast_exp2(old - to);
          }
          set_sync(set);
          if (started) {
            fence_after_sync();
#pragma unroll
            for (int i = 0; i < 4 * kGroups; ++i)
              if (i < 4 * mine) l[i] = mul2(l[i], *reinterpret_cast<const uint64_t*>(factor + 2 * i));
#pragma unroll 1
            for (int i = 0; i < mine * (Dv / 128); ++i) {
              const uint32_t at = lane_addr + Sh::kColO + first + 8 * (i % mine) + kRows * (i / mine);
              uint32_t o[8];
              tmem_ld8(at, o);
              wait_ld8(o);
#pragma unroll
              for (int c = 0; c < 8; ++c) o[c] = __float_as_uint(__uint_as_float(o[c]) * factor[8 * (i % mine) + c]);
              tmem_st8(at, o);
            }
            wait_st();
            fence_before_sync();
          }
          started = grown = true;
        }
        if (tid == 0) mbar_arrive(&sm.p_full[b]);
#pragma unroll
        for (int i = 0; i < 4 * kGroups; ++i)
          if (i < 4 * mine) l[i] = add2(l[i], p[i]);
      }
      // ---- the segment's record ----
      if (quad == set) mbar_spin(&sm.o_done[(g - 1) & 1], (uint32_t)((g - 1) >> 1), abort_flag);
      {
        float v[8 * kGroups];
#pragma unroll
        for (int i = 0; i < 4 * kGroups; ++i) { const float2 u = unpair64(l[i]); v[2 * i] = u.x; v[2 * i + 1] = u.y; }
        const float sum = column_sums(v);
        if (lane < 8 * kGroups) sm.red_sum[set][quad][lane] = sum;
      }
      if (tid == 0) mbar_arrive(&sm.q_free[slot]);       // the set has passed a barrier since it last read kappa
      set_sync(set);
      fence_after_sync();
      const bool bad = *abort_flag || sm.poisoned[n % kInfo];
      float* o_out = s.prefix ? P.pre_o + (size_t)s.record * Sh::kRecord : P.suf_o + (size_t)s.record * y.n_rep * Dv;
      float2* ml = s.prefix ? P.pre_ml + (size_t)s.record * kRows : P.suf_ml + (size_t)s.record * y.n_rep;
      if (tid < 8 * mine && first + tid < rows)
        ml[first + tid] = make_float2(-neg_ref[tid], bad ? -1.f : sm.red_sum[set][0][tid] + sm.red_sum[set][1][tid] + sm.red_sum[set][2][tid] + sm.red_sum[set][3][tid]);
#pragma unroll 1
      for (int i = 0; i < mine * (Dv / 128); ++i) {
        const int row = first + 8 * (i % mine), m = i / mine;
        uint32_t o[8];
        tmem_ld8(lane_addr + Sh::kColO + row + kRows * m, o);
        wait_ld8(o);
        float* at = o_out + (size_t)row * Dv + 128 * m + quad * 32 + lane;
#pragma unroll
        for (int c = 0; c < 8; ++c)
          if (row + c < rows) at[c * Dv] = __uint_as_float(o[c]);
      }
      fence_before_sync();
      set_sync(set);
      if (tid == 0) mbar_arrive(&sm.info_free[n % kInfo]);
    }
  }

  // ---- teardown: nothing may be in flight in the tensor pipe when the columns are given back ----
  fence_before_sync();
  __syncthreads();
  if (warp == kMmaWarp) {
    if (sm.abort_flag) {
      if (elect_one()) {                                 // the lane that issued the MMAs
        commit(&sm.drain);
        for (uint32_t k = 0; k < kSpinLimit && !mbar_try_wait(&sm.drain, 0); ++k) {}
        raise_flag(P.flags, Q4KV_FLAG_INTERNAL);
      }
      __syncwarp();
    }
    fence_after_sync();
    tmem_dealloc(tb, 512);
  }
}

// One warp per (agent, query head): the records of the prefix's parts and of the agent's own, weighted by 2^(m - M).  Bound by the
// latency of the plan and of the records in L2.
template <int Dv>
__global__ void __launch_bounds__(128) shared_prefix_merge_kernel(const __grid_constant__ Params P, int max_rows, int record) {
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  const int lane = threadIdx.x & 31, Hq = P.y.Hq, heads = P.y.Hkv, n_rep = P.y.n_rep;
  const int at = blockIdx.x * 4 + (threadIdx.x >> 5), a = at / Hq, head = at % Hq / n_rep, rep = at % n_rep;
  asm volatile("griddepcontrol.wait;" ::: "memory");
  if (a >= P.n_agents) return;
  const Plan& p = *P.plan;
  const int kv = p.kv_len[a], g = p.group[a];
  int n_pre = 0, n_own = 0, pre = 0, own = 0, row = 0;   // parts, the first one's record, the row in a prefix record
  if (kv > 0) {
    const int prefix = p.prefix[g], steps = steps_of(prefix), mine = own_steps(kv, prefix);
    if (steps > 0) {
      const int n = p.offs[g + 1] - p.offs[g], tiles = tiles_of(n, max_rows / n_rep), i = a - p.offs[g];
      const int t = ((i + 1) * tiles - 1) / n, segment = t * heads + head;
      const int start = p.pre_start[g] + segment * cost_of(steps), c0 = cta_of(p, start);
      n_pre = cta_of(p, start + steps - 1) - c0 + 1;
      pre = p.tile0[g] * heads + segment + c0;
      row = (i - n * t / tiles) * n_rep + rep;
    }
    if (mine > 0) {
      const int start = p.suffix_base + p.suf_start[a] + head * cost_of(mine), c0 = cta_of(p, start);
      n_own = cta_of(p, start + mine - 1) - c0 + 1;
      own = a * heads + head + c0;
    }
  }
  constexpr int kQuads = Dv / 128;
  float4 acc[kQuads];
#pragma unroll
  for (int k = 0; k < kQuads; ++k) acc[k] = make_float4(0.f, 0.f, 0.f, 0.f);
  float M = -INFINITY, L = 0.f;
  bool bad = false;
  for (int base = 0; base < n_pre + n_own; base += 32) {
    const int i = base + lane, n = min(32, n_pre + n_own - base);
    float2 ml = make_float2(-INFINITY, 0.f);
    const float* o = nullptr;
    if (lane < n) {
      if (i < n_pre) {
        ml = __ldcg(P.pre_ml + (size_t)(pre + i) * max_rows + row);
        o = P.pre_o + (size_t)(pre + i) * record + (size_t)row * Dv;
      } else {
        ml = __ldcg(P.suf_ml + (size_t)(own + i - n_pre) * n_rep + rep);
        o = P.suf_o + ((size_t)(own + i - n_pre) * n_rep + rep) * Dv;
      }
    }
    bad |= __any_sync(0xffffffffu, ml.y < 0.f) != 0;
    if (!(ml.y > 0.f) && ml.y == ml.y) ml.x = -INFINITY; // nothing in it
    const float m = fmaxf(M, warp_max(ml.x));
    const float keep = M == -INFINITY ? 0.f : fast_exp2(M - m), e = ml.x == -INFINITY ? 0.f : fast_exp2(ml.x - m);
    L = L * keep + warp_sum(e * ml.y);
    M = m;
#pragma unroll
    for (int k = 0; k < kQuads; ++k) { acc[k].x *= keep; acc[k].y *= keep; acc[k].z *= keep; acc[k].w *= keep; }
#pragma unroll 8
    for (int j = 0; j < n; ++j) {
      const float f = __shfl_sync(0xffffffffu, e, j);
      const float* from = reinterpret_cast<const float*>(__shfl_sync(0xffffffffu, reinterpret_cast<unsigned long long>(o), j));
#pragma unroll
      for (int k = 0; k < kQuads; ++k) {
        const float4 v = __ldcg(reinterpret_cast<const float4*>(from + 128 * k + 4 * lane));
        if (f != 0.f) { acc[k].x = fmaf(f, v.x, acc[k].x); acc[k].y = fmaf(f, v.y, acc[k].y); acc[k].z = fmaf(f, v.z, acc[k].z); acc[k].w = fmaf(f, v.w, acc[k].w); }
      }
    }
  }
  const bool zero = bad || L == 0.f;                     // (a NaN stays one)
  const float inv = zero ? 0.f : 1.f / L;
#pragma unroll
  for (int k = 0; k < kQuads; ++k) {
    const size_t to = (size_t)at * Dv + 128 * k + 4 * lane;
    const float4 v = zero ? make_float4(0.f, 0.f, 0.f, 0.f) : make_float4(acc[k].x * inv, acc[k].y * inv, acc[k].z * inv, acc[k].w * inv);
    if (P.out_dtype == Q4KV_OUT_BF16) {
      const __nv_bfloat162 lo = __floats2bfloat162_rn(v.x, v.y), hi = __floats2bfloat162_rn(v.z, v.w);
      *reinterpret_cast<uint2*>(reinterpret_cast<__nv_bfloat16*>(P.out) + to) =
          make_uint2(*reinterpret_cast<const uint32_t*>(&lo), *reinterpret_cast<const uint32_t*>(&hi));
    } else {
      *reinterpret_cast<float4*>(reinterpret_cast<float*>(P.out) + to) = v;
    }
  }
  if (lane == 0 && P.lse) P.lse[at] = zero ? -INFINITY : (M + log2f(L)) / kLog2e;
}

int max_rows_of(const Layout& y) { return y.D == 128 ? Shape<2, 2>::kRows : Shape<4, 4>::kRows; }
static_assert(Shape<3, 2>::kRows == Shape<4, 4>::kRows, "");

size_t align256(size_t n) { return (n + 255) & ~(size_t)255; }

// The workspace behind the header: the plan, then the records.  A CTA leaves one per segment it touches, and segments and CTAs
// are both in order, so segment + CTA names a record; tiles: sum over groups of ceil(agents / agents of a tile) at most.
struct Sections { size_t pre_ml, suf_ml, pre_o, suf_o, end; };
Sections sections_of(const Layout& y, int n_agents, int n_groups) {
  const int rows = max_rows_of(y), most = rows / y.n_rep;
  const size_t tiles = (size_t)n_agents / most + n_groups, n_pre = tiles * y.Hkv + sm_count(), n_suf = (size_t)n_agents * y.Hkv + sm_count();
  Sections s;
  s.pre_ml = align256(sizeof(Plan));
  s.suf_ml = s.pre_ml + align256(n_pre * rows * sizeof(float2));
  s.pre_o = s.suf_ml + align256(n_suf * y.n_rep * sizeof(float2));
  s.suf_o = s.pre_o + align256(n_pre * rows * y.Dv * sizeof(float));
  s.end = s.suf_o + align256(n_suf * y.n_rep * y.Dv * sizeof(float));
  return s;
}

template <int G, int Gv, bool kBf>
cudaError_t launch(const Params& P, int grid, cudaStream_t st) {
  static bool configured[64] = {};
  const size_t smem = sizeof(Smem<G, Gv>);
  static_assert(sizeof(Smem<G, Gv>) <= 227 * 1024, "");
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  if (dev < 0 || dev >= 64 || !configured[dev]) {
    e = cudaFuncSetAttribute(shared_prefix_kernel<G, Gv, kBf>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
    if (e != cudaSuccess) return e;
    if (dev >= 0 && dev < 64) configured[dev] = true;
  }
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(grid);
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  e = cudaLaunchKernelEx(&cfg, shared_prefix_kernel<G, Gv, kBf>, P);
  if (e != cudaSuccess) return e;
  cfg.gridDim = dim3((P.n_agents * P.y.Hq + 3) / 4);
  cfg.blockDim = dim3(128);
  cfg.dynamicSmemBytes = 0;
  return cudaLaunchKernelEx(&cfg, shared_prefix_merge_kernel<64 * Gv>, P, (int)Shape<G, Gv>::kRows, (int)Shape<G, Gv>::kRecord);
}

}  // namespace

bool shared_prefix_supported(const Layout& y, int n_agents, int max_kv_len) {
  const bool shape = !y.alias && ((y.D == 128 && y.Dv == 128) || (y.D == 256 && y.Dv == 256) || (y.D == 192 && y.Dv == 128));
  // the list's positions are 32-bit numbers
  return shape && y.n_rep <= max_rows_of(y) && n_agents <= kMaxAgents &&
         2ll * n_agents * y.Hkv * (max_kv_len / 128 + 3 + kSegmentCost) < (1ll << 30);
}

size_t shared_prefix_workspace_bytes(const Layout& y, int n_agents, int n_groups) { return sections_of(y, n_agents, n_groups).end; }

cudaError_t launch_shared_prefix(const Layout& y, const void* pool, int n_blocks, int layer, const q4kv_batch& b, const int32_t* kv_lens,
                                 int max_kv_len, const int32_t* group_offs, const int32_t* prefix_lens, int n_groups, const void* q,
                                 float scale, void* out, int out_dtype, float* lse, void* ws, int32_t* flags, cudaStream_t st) {
  const Sections s = sections_of(y, b.n_agents, n_groups);
  uint8_t* at = (uint8_t*)ws;
  Params P;
  P.y = y; P.pool = (const uint8_t*)pool; P.n_blocks = n_blocks; P.layer = layer; P.n_agents = b.n_agents; P.max_blocks = b.max_blocks;
  P.tables = b.block_tables; P.kv_lens = kv_lens; P.max_kv_len = max_kv_len; P.group_offs = group_offs; P.prefix_lens = prefix_lens;
  P.n_groups = n_groups; P.q = (const uint16_t*)q; P.scale_log2 = scale * kLog2e; P.out = out; P.out_dtype = out_dtype; P.lse = lse;
  P.flags = flags; P.plan = (Plan*)at; P.pre_ml = (float2*)(at + s.pre_ml); P.suf_ml = (float2*)(at + s.suf_ml);
  P.pre_o = (float*)(at + s.pre_o); P.suf_o = (float*)(at + s.suf_o);
  const int grid = sm_count();
  if (y.D == 128) return y.sb_bf16 ? launch<2, 2, true>(P, grid, st) : launch<2, 2, false>(P, grid, st);
  if (y.D == 256) return y.sb_bf16 ? launch<4, 4, true>(P, grid, st) : launch<4, 4, false>(P, grid, st);
  return y.sb_bf16 ? launch<3, 2, true>(P, grid, st) : launch<3, 2, false>(P, grid, st);
}

}  // namespace q4kv
