// q4kv_shared_prefix_decode_attention: one query per agent over its whole cache, where groups of agents share a prefix whose keys
// are read and expanded once for the group (Section 3.4 decode; forked agents, q4kv_allocator_fork).
//
//   With the keys of an agent cut into parts i (pieces of the prefix, its own tokens), part i leaves
//   m_i = a reference for its scores, l_i = sum 2^(s - m_i), o_i = sum 2^(s - m_i) v, and
//   out = sum_i 2^(m_i - M) o_i / sum_i 2^(m_i - M) l_i with M = max m_i.
//
// Three launches: the prefixes (here, or on the prefill kernels where many rows share one), the agents' own tokens (decode_mma, its
// range beginning behind the prefix), the sum of the parts (here).  Where that takes longer than every agent reading its own keys, one
// launch of decode_mma does (route_of).
//
// The prefixes' work is a list of segments (group, tile of score rows, KV head) with up to kRows rows each, cut into equal contiguous
// ranges of 128-key steps, one per CTA and one CTA per SM; every CTA leaves a record per segment that it touched.  One step is two
// products on the fifth-generation tensor cores with the KEYS as the 128 rows, so that the number of query rows is the free
// dimension N and few rows cost little.  Both multiply the codes themselves: with x^ = c s + b, one (s, b) per key and 64 elements,
//   S_g^T [128 keys][N]     = C_g [128][64] Q_g^T         C in tensor memory, Q in shared memory; one accumulator per group g,
//   score                   = sum_g s_g S_g + b_g (sum of q over the group),
//   O_g^T [d_v][N]         += C_V^T [d_v][128] (P s_g)^T  C_V and P s_g in shared memory: N columns for each of a tile's two groups,
//   o                       = O_g of the element's group + sum of p b_g.
// A nibble masked in place in the low bits of a 16-bit lane is the binary16 subnormal c 2^-24, one nibble up it is 16 c 2^-24 (the 16 is
// divided out of the other operand): five instructions per eight codes, where the expansion to c s + b takes thirteen.  Scores are
// exact products with binary32 sums; the probabilities times a scale are rounded once to binary16.  (Expanded keys and values, up to
// 64 rows a segment: 1400 instructions a scheduler and step at N = 16, 2200 clocks, whatever the rows.)
// Where a key's p s falls below binary16's range its codes are lost while its bias stays, and it counts as its group's minimum: a sink ten
// nats above the rest and values of 0.01 left a tenth of the output wrong.  So all references of a segment lie lower by as many binary
// orders as its value scales allow (lift_of): p s has its full 11 bits down to 2^-24 of the largest, 2^-20 for odd tokens.
// A lane of tensor memory is a key: a softmax thread has one key, its scales and biases in registers, and half of the rows; the mask is
// a matter of whole lanes.  The sums of p and p b_g stay in the threads' registers until the segment ends.  What a step costs an SM
// at d = 128: HBM 790 clocks (18.4 KB), tensor pipe 512.
//   * A warp walks the list and streams raw steps into a ring by bulk copies; two warps stage the query rows of the next segment
//     (bf16 times a power of two per row into binary16, exact).
//   * Two sets of four warps unpack keys, two values, a set every second step.
//   * Two sets of four softmax warps share the rows.  The reference m of a row is kMargin above the maximum over the segment's first
//     step, less the segment's lift; it moves when a probability would exceed 2^kGrow times the lift, or a value scale what the lift
//     allows, which is found by all keys of a set together at the barrier that also ends the set's stores of P.
// All waits are bounded; one that runs out raises Q4KV_FLAG_INTERNAL, lets the copies and the tensor pipe drain and gives the
// tensor memory back.
#include <cmath>

#include "prefill_common.cuh"

namespace q4kv {

namespace {

using namespace tc;
using namespace prefill;

constexpr int kSoftmaxWarps = 8, kKeyWarp = 8, kValueWarp = 16, kLoadWarp = 24, kMmaWarp = 25, kQueryWarp = 26;
constexpr int kThreads = 28 * 32;
constexpr int kRegsSoftmax = 112, kRegsOther = 56;       // of the 72 each thread is launched with
static_assert(kSoftmaxWarps * 32 * kRegsSoftmax + (kThreads - kSoftmaxWarps * 32) * kRegsOther <= kThreads * 72, "");
constexpr float kGrow = 2.5f;                            // p <= 2^(2.5 + lift), s <= 2^(13 - lift): p s stays below 65504
constexpr float kMargin = 1.f;
constexpr int kSmallest = -40;                           // smaller scales count as 2^-40, so that p stays far from binary32's limits
constexpr int kInfo = 8;                                 // segments that the loader may be ahead of the softmax
constexpr int kSegmentCost = 1;                          // of a segment beside its steps, in steps

template <int G, int Gv>
struct Shape {
  static constexpr int D = 64 * G, Dv = 64 * Gv;
  static constexpr int kRows = G == 4 ? 16 : 32;         // score rows of a segment at most
  static constexpr int kOffKsb = 16 * D, kOffVc = kOffKsb + 128 * G, kOffVsb = kOffVc + 16 * Dv;
  static constexpr int kChunkBytes = kOffVsb + 128 * Gv, kRawBytes = 4 * kChunkBytes;      // a step: 128 keys
  static constexpr int kRaw = G == 4 ? 3 : 4;            // raw steps in flight
  static constexpr int kStagesV = G == 4 ? 1 : 2;
  static constexpr int kTileV = Dv * 128;                // the value codes of 64 keys, bytes
  static constexpr int kQueryBytes = kRows * D * 2, kProbBytes = Gv * kRows * 128 * 2;
  static constexpr int kSboQ = (D / 8) * 128;
  // tensor-memory columns: S^T (two steps of G accumulators), O^T (two groups for each 128 elements), codes of the keys (two steps)
  static constexpr uint32_t kColS = 0, kColO = 2 * G * kRows, kColK = kColO + Gv * kRows;
  static_assert(kColK + D <= 512, "");
  static constexpr int kRecord = kRows * Dv;             // floats of a record's o
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
  int grid;                   // of the launch over the prefixes
  const uint16_t* q;
  float scale_log2;
  void* out;
  int out_dtype;
  float* lse;
  int32_t* flags;
  float* rec_o;               // [record][row][d_v]
  float2* rec_ml;             // [record][row]: m, l
  const float* tile_records;  // instead, where the prefill kernel takes the prefixes: [agent][query head][splits][o, m, l, pad]
  int splits;
  const float* own_o;         // [agent][query head][d_v]: of the agents' own tokens, normalised
  const float* own_lse;       // [agent][query head]
  CodeMasks masks;
};

// Waits in as few instructions as can be: every role's loop holds several, and the kernel's instructions have to be fetched.
__device__ __forceinline__ bool wait_for(uint64_t* bar, int use, volatile int* abort_flag) {
  const uint32_t parity = (uint32_t)use & 1u;
  if (mbar_test_wait(bar, parity)) return true;
#pragma unroll 1
  for (uint32_t i = 0; i < kSpinLimit; ++i) {
    if (mbar_try_wait(bar, parity)) return true;
    if (*abort_flag) return false;
  }
  *abort_flag = 1;
  return false;
}
__device__ __forceinline__ bool spin_for(uint64_t* bar, int use, volatile int* abort_flag) {      // without suspending
  const uint32_t parity = (uint32_t)use & 1u;
#pragma unroll 1
  for (uint32_t i = 0; i < (1u << 26); ++i) {
    if (mbar_test_wait(bar, parity)) return true;
    if ((i & 255u) == 255u && *abort_flag) return false;
  }
  *abort_flag = 1;
  return false;
}

// ---- the work list: positions count steps, and kSegmentCost for each segment ----
struct Group { int agent0, n, prefix, steps, tiles, cost; };   // n: agents; tiles: of score rows; cost: of one segment
template <int kRows>
__device__ inline Group group_of(const Params& P, int g, bool* fine = nullptr) {
  Group q = {0, 0, 0, 0, 0, 0};
  if (g < P.n_groups) {
    const int lo = P.group_offs[g], hi = P.group_offs[g + 1], prefix = P.prefix_lens[g];
    const bool ok = lo >= 0 && lo <= hi && hi <= P.n_agents;
    if (fine) *fine = ok;
    if (ok && prefix >= 0 && prefix <= P.max_kv_len) {
      q.agent0 = lo;
      q.n = hi - lo;
      q.prefix = prefix;
      q.steps = (prefix + 127) >> 7;
      q.tiles = (q.n * P.y.n_rep + kRows - 1) / kRows;   // as equal as can be: see tile_begin
      q.cost = q.tiles > 0 && q.steps > 0 ? q.steps + kSegmentCost : 0;
    }
  }
  return q;
}
// Score row r of a group and KV head is of the group's agent r / n_rep and that agent's query head r % n_rep; tile t of them begins at
__device__ inline int tile_begin(int rows, int tiles, int t) { return (int)((long long)rows * t / tiles); }
__device__ inline int inclusive_sum(int v) {
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int u = __shfl_up_sync(0xffffffffu, v, o);
    if (lane >= o) v += u;
  }
  return v;
}
// The list is cut for n CTAs, the first total % n of them with a position more; a CTA's range begins at begin(), cta_of() is the CTA
// whose range holds position u.
struct Cut {
  int n, each, more;
  __device__ Cut(int total, int grid) : n(min(grid, max(1, total))) {
    each = (int)((unsigned)total / (unsigned)n);
    more = total - each * n;
  }
  __device__ int begin(int c) const { return c * each + min(c, more); }
  __device__ int cta_of(int u) const {
    const int big = more * (each + 1);
    return u < big ? (int)((unsigned)u / (unsigned)(each + 1)) : more + (int)((unsigned)(u - big) / (unsigned)each);
  }
};

// One CTA's part of a segment.  Records are named segment + CTA: both are in order, so no two parts share one.
struct Segment {
  int agent0, row0, rows, lead, head;                    // rows row0 .. of the group that begins with agent0; keys: of agent `lead`
  int prefix, step0, steps;                              // keys of the prefix; 128-key steps of this CTA (0: there is no more)
  int record;
};

template <int G, int Gv>
struct Smem {
  using Sh = Shape<G, Gv>;
  alignas(128) uint8_t vhat[Sh::kStagesV][2 * Sh::kTileV];     // [half][dim][key 64]: (n%8)*16 + (n/8)*1024 + (k/8)*128
  alignas(128) uint8_t raw[Sh::kRaw][Sh::kRawBytes];
  alignas(128) uint8_t qs[2][Sh::kQueryBytes];                 // [row][dim]: (r%8)*16 + (r/8)*kSboQ + (k/8)*128
  alignas(128) uint8_t prob[2][Sh::kProbBytes];                // [key][value group x rows, row]: (k%8)*16 + (k/8)*128 + (r/8)*2048 + (r%8)*2
  // of a row: what S_g times the scale is multiplied by for a score in log2 units, and the sums of q over the groups in those
  alignas(16) float kappa[2][Sh::kRows], q_sum[2][G][Sh::kRows];
  // of the two softmax sets: minus the reference of each row, what to scale by when it moves, partial maxima, sums of p and p b_g
  alignas(16) float neg_ref[2][Sh::kRows / 2], factor[2][Sh::kRows / 2], red_max[2][4][Sh::kRows / 2], red_sum[2][4][Gv + 1][Sh::kRows / 2];
  float red_scale[2][4];                                       // the largest value scale of a warp's keys
  alignas(8) uint64_t raw_full[Sh::kRaw], raw_free[Sh::kRaw];
  uint64_t k_full[2], s_full[2], p_full[2], o_done[2], q_full[2], q_free[2], info_full[kInfo], info_free[kInfo], drain;
  Segment info[kInfo];
  uint32_t tmem_base;
  int bad[Sh::kRaw], poisoned[kInfo];                          // poisoned: a bad block in the segment
  int abort_flag;
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
#pragma unroll
  for (int o = 16; o >= kCount; o >>= 1) {
#pragma unroll
    for (int c = 0; c < kCount; ++c) v[c] += __shfl_xor_sync(0xffffffffu, v[c], o);
  }
#pragma unroll
  for (int o = kCount / 2; o > 0; o >>= 1) {
    const bool high = lane & o;
#pragma unroll
    for (int c = 0; c < o; ++c) v[c] = (high ? v[c + o] : v[c]) + __shfl_xor_sync(0xffffffffu, high ? v[c] : v[c + o], o);
  }
  return v[0];
}

// query8 with the elements that meet a nibble's second place divided by 16
__device__ inline uint4 query_codes8(uint4 v, float sf) {
  const float sh = sf * 0.0625f;
  auto lo = [](uint32_t u) { return __uint_as_float(u << 16); };
  auto hi = [](uint32_t u) { return __uint_as_float(u & 0xffff0000u); };
  return make_uint4(f32x2_to_h2(lo(v.x) * sf, lo(v.z) * sf), f32x2_to_h2(hi(v.x) * sh, hi(v.z) * sh), f32x2_to_h2(lo(v.y) * sf, lo(v.w) * sf),
                    f32x2_to_h2(hi(v.y) * sh, hi(v.w) * sh));
}
__device__ inline float sum_of8(uint4 v) {
  auto two = [](uint32_t u) { return __uint_as_float(u << 16) + __uint_as_float(u & 0xffff0000u); };
  return (two(v.x) + two(v.y)) + (two(v.z) + two(v.w));
}
// Eight codes as binary16 subnormals, in the order 0,4,1,5,2,6,3,7: c 2^-24 and (1,5,3,7) 16 c 2^-24
__device__ inline uint4 codes8(uint32_t w, const CodeMasks& m) {
  const uint32_t wh = w >> 8;
  return make_uint4(w & m.lo, w & m.hi, wh & m.lo, wh & m.hi);
}
// The binary orders that p may lie above 1, and the largest value scale that allows it, by a segment's largest so far: two to four times
// that one, so that it seldom has to move.  Powers of two: nothing is rounded by it.
struct Lift { float orders, limit; };
__device__ inline Lift lift_of(float scale) {
  const int e = max((int)(__float_as_uint(scale) >> 23) - 127, kSmallest) + 2;     // scale < 2^(e - 1)
  return {(float)(13 - e), e < 128 ? __uint_as_float((uint32_t)(127 + e) << 23) : INFINITY};
}
template <bool kBf>
__device__ inline float2 scale_bias(uint32_t u) {
  if (kBf) return make_float2(__uint_as_float(u << 16), __uint_as_float(u & 0xffff0000u));
  return __half22float2(*reinterpret_cast<const __half2*>(&u));
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
    for (int s = 0; s < kRaw; ++s) { mbar_init(&sm.raw_full[s], 1); mbar_init(&sm.raw_free[s], 16); sm.bad[s] = 0; }
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
  fence_before_sync();
  __syncthreads();
  fence_after_sync();
  const uint32_t tb = sm.tmem_base;
  volatile int* abort_flag = &sm.abort_flag;
  int g = 0;                                             // steps so far

  if (warp >= kLoadWarp) {
    fewer_registers<kRegsOther>();
    if (warp == kLoadWarp) {
      // =============================== segments and raw steps =====================================
      // (lengths, offsets and block tables are inputs that no kernel writes)
      int total = 0;
      bool ascending = true;                             // else groups can overlap: more tiles than there are records, or positions
#pragma unroll 1
      for (int base = 0; base < P.n_groups && ascending; base += 32) {
        bool fine = true;
        const Group q = group_of<kRows>(P, base + lane, &fine);
        ascending = __all_sync(0xffffffffu, fine);
        total += __reduce_add_sync(0xffffffffu, q.tiles * y.Hkv * q.cost);
      }
      if (!ascending) total = 0;                         // no work; the merge reports it
      const Cut cut(total, gridDim.x);
      const bool any = (int)blockIdx.x < cut.n && total > 0;
      const int u0 = any ? cut.begin(blockIdx.x) : 0, u1 = any ? cut.begin(blockIdx.x + 1) : 0;
      int first = 0, start = 0, tile0 = 0;               // the group that the range begins in, where that group begins, tiles before it
      if (any) {
        int tiles = 0;
#pragma unroll 1
        for (int base = 0, before = 0;; base += 32) {
          const Group q = group_of<kRows>(P, base + lane);
          const int cost = q.tiles * y.Hkv * q.cost, upto = before + inclusive_sum(cost), t = tiles + inclusive_sum(q.tiles);
          const unsigned past = __ballot_sync(0xffffffffu, upto > u0);
          if (past) {
            const int l = __ffs(past) - 1;
            first = base + l;
            start = __shfl_sync(0xffffffffu, upto - cost, l);
            tile0 = __shfl_sync(0xffffffffu, t - q.tiles, l);
            break;
          }
          before = __shfl_sync(0xffffffffu, upto, 31);
          tiles = __shfl_sync(0xffffffffu, t, 31);
        }
      }
      int n = 0;                                         // segments handed out
      bool ok = true;
      auto hand_out = [&](const Segment& s) {
        if (n >= kInfo && !wait_for(&sm.info_free[n % kInfo], n / kInfo - 1, abort_flag)) ok = false;
        if (ok && lane == 0) {
          sm.info[n % kInfo] = s;
          sm.poisoned[n % kInfo] = 0;
          mbar_arrive(&sm.info_full[n % kInfo]);
        }
      };
      bool waited = false;
#pragma unroll 1
      for (int gr = first; ok && any && start < u1; ++gr) {
        const Group q = group_of<kRows>(P, gr);
        const int lead = first_holder(P.kv_lens, q.agent0, q.n, q.prefix, P.max_kv_len);             // the agent that the prefix is read through
        const int segments = q.tiles * y.Hkv;
        int k = q.cost > 0 && u0 > start ? (u0 - start) / q.cost : 0;
        if (lead < 0 || q.cost == 0) k = segments;
#pragma unroll 1
        for (; ok && k < segments; ++k) {
          const int at = start + k * q.cost;
          if (at >= u1) break;
          const int from = max(0, u0 - at), to = min(q.steps, u1 - at);
          if (from >= to) continue;                      // this CTA's part is the segment's fixed cost
          const int t = k / y.Hkv, all = q.n * y.n_rep;
          Segment s;
          s.agent0 = q.agent0; s.row0 = tile_begin(all, q.tiles, t); s.rows = tile_begin(all, q.tiles, t + 1) - s.row0;
          s.lead = lead; s.head = k - t * y.Hkv;
          s.prefix = q.prefix; s.step0 = from; s.steps = to - from; s.record = tile0 * y.Hkv + k + (int)blockIdx.x;
          hand_out(s);
          if (!waited) asm volatile("griddepcontrol.wait;" ::: "memory");
          waited = true;
          if (lane == 0) {
            const uint8_t* row = head_block(P.pool, y, P.layer, 0, s.head);
#pragma unroll 1
            for (int j = 0; ok && j < s.steps; ++j, ++g) {
              const int r = g % kRaw, step = s.step0 + j;
              if (g >= kRaw && !wait_for(&sm.raw_free[r], g / kRaw - 1, abort_flag)) { ok = false; break; }
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
          ok = __all_sync(0xffffffffu, ok);
          ++n;
        }
        start += segments * q.cost;
        tile0 += q.tiles;
      }
      Segment last = {};
      hand_out(last);
      if (!waited) asm volatile("griddepcontrol.wait;" ::: "memory");        // or this grid could complete before the one it follows
      // a CTA that is giving up still lets its own copies land before shared memory is released
      if (lane == 0 && *abort_flag)
#pragma unroll 1
        for (int j = max(0, g - kRaw); j < g; ++j)
#pragma unroll 1
          for (uint32_t i = 0; i < kSpinLimit && !mbar_try_wait(&sm.raw_full[j % kRaw], (uint32_t)(j / kRaw) & 1u); ++i) {}
    } else if (warp == kMmaWarp) {
      // =============================== products ===================================================
      // A product's commit also covers what was issued before it: S^T of a step implies O^T of the step two before, so neither the
      // buffers of P^T nor those of S^T and K^ need barriers of their own.  The value tile's warps arrive where the softmax does.
      auto wait = [&](uint64_t* bar, int use) {
        const bool ok = spin_for(bar, use, abort_flag);
        if (ok) fence_after_sync();
        return ok;
      };
      const uint64_t vd0 = smem_desc(smem_u32(sm.vhat[0]), 128, 1024), pd0 = smem_desc(smem_u32(sm.prob[0]), 128, 2048);
      const uint64_t qd0 = smem_desc(smem_u32(sm.qs[0]), 128, Sh::kSboQ);
      bool first = true;
      uint32_t idesc_pv = 0;                             // of the step whose value product is due, and its two groups of P s_g
      int p_tile = 0;
      auto issue_pv = [&](int h) {                       // O^T (+)= V^T P^T of step h
        const uint64_t vd = vd0 + (uint64_t)((h % kStagesV) * (2 * Sh::kTileV >> 4)), pd = pd0 + (uint64_t)((h & 1) * (Sh::kProbBytes >> 4));
        if (elect_one()) {
#pragma unroll
          for (int m = 0; m < Dv / 128; ++m)
#pragma unroll
            for (int k = 0; k < 8; ++k)
              mma_f16_ss(tb + Sh::kColO + 2 * kRows * m, vd + (uint64_t)((k >> 2) * (Sh::kTileV >> 4) + m * 1024 + (k & 3) * 16),
                         pd + (uint64_t)(m * p_tile + 16 * k), idesc_pv, (!first || k > 0) ? 1u : 0u);
          commit(&sm.o_done[h & 1]);
        }
        __syncwarp();
      };
      bool ok = true;
#pragma unroll 1
      for (int n = 0; ok; ++n) {
        const int slot = n & 1;
        ok = wait(&sm.q_full[slot], n >> 1);
        const int steps = ok ? sm.info[n % kInfo].steps : 0, columns = ok ? (sm.info[n % kInfo].rows + 15) & ~15 : 0;
        const uint32_t size = (uint32_t)(columns >> 3) << 17;
        const uint64_t qd = qd0 + (uint64_t)(slot * (Sh::kQueryBytes >> 4));
#pragma unroll 1
        for (int j = 0; ok && (j < steps || (steps == 0 && j == 0)); ++j) {
          if (steps > 0) {
            ok = wait(&sm.k_full[g & 1], g >> 1);
            if (!ok) break;
            if (elect_one()) {
#pragma unroll
              for (int k = 0; k < D / 16; ++k)           // four products for each group's accumulator
                mma_f16_ts(tb + Sh::kColS + kRows * (G * (g & 1) + (k >> 2)), tb + Sh::kColK + (D / 2) * (g & 1) + 8 * k, qd + 16 * k,
                           idesc_f16(128, 0) | size, (k & 3) > 0);
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
          idesc_pv = idesc_f16(128, 0, 0, 1) | (size << 1);
          p_tile = (columns >> 3) * (2 * 2048 >> 4);
          ++g;
        }
        if (steps == 0) break;
      }
    } else {
      // =============================== query rows =================================================
      constexpr int kLanes = D == 128 ? 16 : 32, kAtOnce = 4, kStride = 2 * (32 / kLanes);     // lanes of a row, rows in flight, rows of both warps
      asm volatile("griddepcontrol.wait;" ::: "memory");
      const float per_rep = 1.f / (float)y.n_rep;
      const int piece = lane % kLanes, sub = (warp - kQueryWarp) * (32 / kLanes) + lane / kLanes;
#pragma unroll 1
      for (int n = 0;; ++n) {
        const int slot = n & 1;
        if (!wait_for(&sm.info_full[n % kInfo], n / kInfo, abort_flag)) break;
        const Segment& s = sm.info[n % kInfo];
        const int steps = s.steps, rows = s.rows, padded = steps > 0 ? (rows + 15) & ~15 : 0;
        const int row0 = s.row0;
        const uint16_t* q = P.q + ((size_t)s.agent0 * y.Hq + (size_t)s.head * y.n_rep) * D + 8 * piece;
        if (n >= 2 && !wait_for(&sm.q_free[slot], (n >> 1) - 1, abort_flag)) break;
#pragma unroll 1
        for (int base = sub; base < padded; base += kStride * kAtOnce) {
          uint4 v[kAtOnce];
#pragma unroll
          for (int u = 0; u < kAtOnce; ++u) {
            const int r = base + kStride * u, row = row0 + r;
            int a = (int)((float)row * per_rep);         // row / n_rep: the quotient of floats may be off by one
            a -= a * y.n_rep > row;
            a += (a + 1) * y.n_rep <= row;
            v[u] = make_uint4(0u, 0u, 0u, 0u);
            if (r < rows && piece < D / 8) v[u] = *reinterpret_cast<const uint4*>(q + ((size_t)a * y.Hq + (row - a * y.n_rep)) * D);
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
            float sum = sum_of8(v[u]);
#pragma unroll
            for (int o = 4; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o, kLanes);       // over the eight pieces of a group
            if (r < padded) {
              if (piece == 0) sm.kappa[slot][r] = P.scale_log2 * __uint_as_float((uint32_t)(127 - 8 + 24 + ex) << 23);
              if ((piece & 7) == 0 && piece < D / 8) sm.q_sum[slot][piece >> 3][r] = P.scale_log2 * sum;
              if (piece < D / 8) *reinterpret_cast<uint4*>(sm.qs[slot] + (r & 7) * 16 + (r >> 3) * Sh::kSboQ + piece * 128) = query_codes8(v[u], sf);
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
    const int x7 = threadIdx.x & 127, mine = (warp - kValueWarp) >> 2;       // this set's steps: g % 2 == mine
    // one 16-byte piece (dims 32 vq + 8 k + vr, k = 0..3) of token octet vo of a chunk; at d_v = 256 vq + 4 as well
    const int vr = x7 & 7, vq = (x7 >> 3) & 3, vo = ((vr >> 1) + (x7 >> 5)) & 3;
    const int v_read = Sh::kOffVc + ((vq * 8 + vr) * 4 + vo) * 16, v_write = vr * 16 + (4 * vq) * 1024 + vo * 128;
#pragma unroll 1
    for (int n = 0; wait_for(&sm.info_full[n % kInfo], n / kInfo, abort_flag); ++n) {
      const int steps = sm.info[n % kInfo].steps;
      bool go = steps > 0;
#pragma unroll 1
      for (int j = 0; go && j < steps; ++j, ++g) {
        if ((g & 1) != mine) continue;
        const int r = g % kRaw, sv = g % kStagesV;
        go = wait_for(&sm.raw_full[r], g / kRaw, abort_flag) &&
             (g < kStagesV || wait_for(&sm.o_done[(g - kStagesV) & 1], (g - kStagesV) >> 1, abort_flag));
        if (!go) break;
#pragma unroll
        for (int half = 0; half < Gv / 2; ++half) {
          const uint8_t* from = sm.raw[r] + v_read + half * (4 * 8 * 4 * 16);
          uint8_t* dst = sm.vhat[sv] + v_write + half * 16384;
          uint4 w[4];
#pragma unroll
          for (int c = 0; c < 4; ++c) w[c] = *reinterpret_cast<const uint4*>(from + c * Sh::kChunkBytes);
#pragma unroll
          for (int c = 0; c < 4; ++c) {
            uint8_t* to = dst + (c >> 1) * Sh::kTileV + (c & 1) * 512;
            *reinterpret_cast<uint4*>(to + 0 * 1024) = codes8(w[c].x, P.masks);
            *reinterpret_cast<uint4*>(to + 1 * 1024) = codes8(w[c].y, P.masks);
            *reinterpret_cast<uint4*>(to + 2 * 1024) = codes8(w[c].z, P.masks);
            *reinterpret_cast<uint4*>(to + 3 * 1024) = codes8(w[c].w, P.masks);
          }
        }
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
    const int c = warp & 3, mine = (warp - kKeyWarp) >> 2, tau = 8 * (lane >> 3) + elem_of(lane & 7), ti = tau & 3, tg = tau >> 2, rot = (lane >> 1) & 3;
    const int k_read = c * Sh::kChunkBytes + ti * (256 * G) + tg * 64;      // + j * 512 + piece * 16
    const uint32_t lane_addr = tb + ((uint32_t)(c * 32) << 16) + Sh::kColK;
    auto turned = [&](uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t* out) {      // out[t] = what came as number (t - rot) & 3
      const bool one = rot & 1, two = rot & 2;
      const uint32_t b0 = one ? a3 : a0, b1 = one ? a0 : a1, b2 = one ? a1 : a2, b3 = one ? a2 : a3;
      out[0] = two ? b2 : b0; out[1] = two ? b3 : b1; out[2] = two ? b0 : b2; out[3] = two ? b1 : b3;
    };
#pragma unroll 1
    for (int n = 0; wait_for(&sm.info_full[n % kInfo], n / kInfo, abort_flag); ++n) {
      const int steps = sm.info[n % kInfo].steps;
      bool go = steps > 0;
#pragma unroll 1
      for (int j = 0; go && j < steps; ++j, ++g) {
        if ((g & 1) != mine) continue;
        const int r = g % kRaw;
        go = wait_for(&sm.raw_full[r], g / kRaw, abort_flag) &&
             (g < 2 || wait_for(&sm.s_full[g & 1], (g >> 1) - 1, abort_flag));
        if (!go) break;
        fence_after_sync();
        const uint8_t* raw = sm.raw[r];
        const uint32_t to = lane_addr + (D / 2) * (g & 1);
        auto expand = [&](const uint32_t* words, uint32_t at) {              // four words: 16 columns
          uint32_t col[16];
#pragma unroll
          for (int t = 0; t < 4; ++t) {
            const uint4 v = codes8(words[t], P.masks);
            col[4 * t] = v.x; col[4 * t + 1] = v.y; col[4 * t + 2] = v.z; col[4 * t + 3] = v.w;
          }
          tmem_st16(to + at, col);
        };
#pragma unroll
        for (int jj = 0; jj < G; ++jj) {                 // words 4 (2 jj), 4 (2 jj + 1) + t: half of a piece at a time
          if (jj < (G & ~1)) {
            uint2 p[4];
#pragma unroll
            for (int t = 0; t < 4; ++t) p[t] = *reinterpret_cast<const uint2*>(raw + k_read + (jj >> 1) * 512 + (jj & 1) * 8 + ((t + rot) & 3) * 16);
            uint32_t wd[4];
            turned(p[0].x, p[1].x, p[2].x, p[3].x, wd); expand(wd, 32 * jj);
            turned(p[0].y, p[1].y, p[2].y, p[3].y, wd); expand(wd, 32 * jj + 16);
          }
        }
        if (G & 1) {                                     // the last group: 8-byte pieces, words 16 + 4 m + t, m = 0, 1
          uint2 p[4];
          const int at = c * Sh::kChunkBytes + ti * (256 * G) + (G / 2) * 512 + tg * 32;
#pragma unroll
          for (int t = 0; t < 4; ++t) p[t] = *reinterpret_cast<const uint2*>(raw + at + ((t + rot) & 3) * 8);
          uint32_t wd[4];
          turned(p[0].x, p[1].x, p[2].x, p[3].x, wd); expand(wd, 32 * (G - 1));
          turned(p[0].y, p[1].y, p[2].y, p[3].y, wd); expand(wd, 32 * (G - 1) + 16);
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
    const int tau = 8 * (lane >> 3) + elem_of(lane & 7), key = quad * 32 + tau;            // in the chunk, of the step
    const int at_sb = (((tau & 3) * 4 + (tau >> 3)) * 2 + ((tau >> 2) & 1)) * 4;             // of a token's (scale, bias) words, times groups
    const float place = tau & 1 ? 0.0625f : 1.f;                             // its value codes' place in their 16-bit lanes
    const int tid = threadIdx.x & 127;
    float* const neg_ref = sm.neg_ref[set];
    float* const factor = sm.factor[set];
#pragma unroll 1
    for (int n = 0;; ++n) {
      const int slot = n & 1;
      bool lost = false;
      if (quad == set) lost = !spin_for(&sm.q_full[slot], n >> 1, abort_flag);
      if (set_any(set, lost)) break;
      const Segment s = sm.info[n % kInfo];
      if (s.steps == 0) break;
      const int half = ((s.rows + 15) & ~15) >> 1, first = set * half;
      const int mine = min(max((s.rows - first + 7) >> 3, 0), half >> 3);    // groups of eight rows, from row `first` on
      uint64_t l[4 * kGroups], pb[Gv][4 * kGroups];      // sums of p and p b_g
#pragma unroll
      for (int c = 0; c < 4 * kGroups; ++c) {
        l[c] = 0ull;
#pragma unroll
        for (int v = 0; v < Gv; ++v) pb[v][c] = 0ull;
      }
      bool started = false;
      Lift lift = {0.f, 0.f};
#pragma unroll 1
      for (int j = 0; j < s.steps; ++j, ++g) {
        const int b = g & 1, r = g % kRaw;
        wait_for(&sm.s_full[b], g >> 1, abort_flag);
        fence_after_sync();
        const bool edge = (s.step0 + j) * 128 + 128 > s.prefix, valid = (s.step0 + j) * 128 + key < s.prefix;
        wait_for(&sm.raw_full[r], g / kRaw, abort_flag);
        // the key's scales and biases
        uint64_t ks[G], kb[G], vs[Gv], vb[Gv];
        float largest = 0.f;                             // of its value scales
        {
          const uint8_t* chunk = sm.raw[r] + quad * Sh::kChunkBytes;
#pragma unroll
          for (int i = 0; i < G; ++i) {
            const float2 e = scale_bias<kBf>(*reinterpret_cast<const uint32_t*>(chunk + Sh::kOffKsb + at_sb * G + 4 * i));
            ks[i] = pair64(e.x, e.x);
            kb[i] = pair64(e.y, e.y);
          }
#pragma unroll
          for (int i = 0; i < Gv; ++i) {
            float2 e = scale_bias<kBf>(*reinterpret_cast<const uint32_t*>(chunk + Sh::kOffVsb + at_sb * Gv + 4 * i));
            if (edge && !valid) e = make_float2(0.f, 0.f);
            largest = fmaxf(largest, fabsf(e.x));
            vs[i] = pair64(e.x * place, e.x * place);
            vb[i] = pair64(e.y, e.y);
          }
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(&sm.raw_free[r]);
        const uint32_t s_addr = lane_addr + Sh::kColS + kRows * G * b + first;
        uint64_t p[4 * kGroups];
        // scores of eight rows, in log2 units above their references
        auto scores = [&](int i, uint64_t (&t)[4], bool relative) {
          uint32_t x[G][8];
#pragma unroll
          for (int v = 0; v < G; ++v) tmem_ld8(s_addr + kRows * v + 8 * i, x[v]);
#pragma unroll
          for (int v = 0; v < G; ++v) wait_ld8(x[v]);
#pragma unroll
          for (int c = 0; c < 4; ++c) {
            const int row = first + 8 * i + 2 * c;
            uint64_t w = relative ? *reinterpret_cast<const uint64_t*>(neg_ref + 8 * i + 2 * c) : 0ull;
            uint64_t u = mul2(pair64(__uint_as_float(x[0][2 * c]), __uint_as_float(x[0][2 * c + 1])), ks[0]);
#pragma unroll
            for (int v = 1; v < G; ++v) u = fma2(pair64(__uint_as_float(x[v][2 * c]), __uint_as_float(x[v][2 * c + 1])), ks[v], u);
#pragma unroll
            for (int v = 0; v < G; ++v) w = fma2(*reinterpret_cast<const uint64_t*>(&sm.q_sum[slot][v][row]), kb[v], w);
            t[c] = fma2(u, *reinterpret_cast<const uint64_t*>(&sm.kappa[slot][row]), w);
          }
        };
        bool grown = false;
#pragma unroll 1
        for (;;) {
          if (started) {
            float most = -INFINITY;
            uint8_t* const p_at = sm.prob[b] + (quad * 32 + lane) * 16 + (first >> 3) * 2048;
#pragma unroll
            for (int i = 0; i < kGroups; ++i) {
              if (i < mine) {
                uint64_t t[4];
                scores(i, t, true);
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                  const float2 e = unpair64(t[c]);
                  if (!edge || valid) most = fmaxf(fmaxf(most, e.x), e.y);
                  p[4 * i + c] = edge && !valid ? 0ull : pair64(fast_exp2(e.x), fast_exp2(e.y));
                }
#pragma unroll
                for (int v = 0; v < Gv; ++v) {
                  uint32_t h[4];
#pragma unroll
                  for (int c = 0; c < 4; ++c) { const float2 e = unpair64(mul2(p[4 * i + c], vs[v])); h[c] = f32x2_to_h2(e.x, e.y); }
                  *reinterpret_cast<uint4*>(p_at + i * 2048 + v * (half >> 2) * 2048) = make_uint4(h[0], h[1], h[2], h[3]);
                }
              }
            }
            fence_async_smem();
            fence_before_sync();
            if (!set_any(set, most > kGrow + lift.orders || largest > lift.limit) || grown) break;
            fence_after_sync();
          } else if (mine == 0) {
            // a set without rows: all of its warps have seen this step's scores before one arrives for the set, or a warp that is behind
            // could find that barrier two phases on and wait for good
            set_sync(set);
            break;
          }
          // the references of the rows that outgrow theirs (of all, in the first step) move above the maximum of this step's scores; the
          // others' stay, so that no row's numbers depend on another's.  A smaller lift moves all of them
#pragma unroll 1
          for (int i = 0; i < mine; ++i) {
            uint64_t t[4];
            scores(i, t, false);
#pragma unroll
            for (int c = 0; c < 4; ++c) {
              const float2 e = unpair64(t[c]);
              const float m0 = warp_max(valid ? e.x : -INFINITY), m1 = warp_max(valid ? e.y : -INFINITY);
              if (lane == 0) *reinterpret_cast<float2*>(&sm.red_max[set][quad][8 * i + 2 * c]) = make_float2(m0, m1);
            }
          }
          largest = warp_max(largest);
          if (lane == 0) sm.red_scale[set][quad] = largest;
          if (j > 0 && quad == set) spin_for(&sm.o_done[b ^ 1], (g - 1) >> 1, abort_flag);                // O^T so far is complete
          set_sync(set);
          largest = fmaxf(fmaxf(sm.red_scale[set][0], sm.red_scale[set][1]), fmaxf(sm.red_scale[set][2], sm.red_scale[set][3]));
          const Lift now = started && largest <= lift.limit ? lift : lift_of(largest);
          if (quad == 0 && lane < 8 * mine) {
            const float m = fmaxf(fmaxf(sm.red_max[set][0][lane], sm.red_max[set][1][lane]), fmaxf(sm.red_max[set][2][lane], sm.red_max[set][3][lane]));
            const float old = started ? neg_ref[lane] : 0.f;
            float to = now.orders - (m > -INFINITY ? m + kMargin : 0.f);
            if (started && !(m + old - lift.orders > kGrow)) to = old + (now.orders - lift.orders);
            neg_ref[lane] = to;
            factor[lane] = to == old ? 1.f : fast_exp2(to - old);
          }
          lift = now;
          set_sync(set);
          if (started) {
            fence_after_sync();
#pragma unroll
            for (int i = 0; i < 4 * kGroups; ++i) {
              if (i < 4 * mine) {
                const uint64_t f = *reinterpret_cast<const uint64_t*>(factor + 2 * i);
                l[i] = mul2(l[i], f);
#pragma unroll
                for (int v = 0; v < Gv; ++v) pb[v][i] = mul2(pb[v][i], f);
              }
            }
#pragma unroll 1
            for (int i = 0; j > 0 && i < mine * (Dv / 128); ++i) {
              const uint32_t at = lane_addr + Sh::kColO + 2 * kRows * (i / mine) + 2 * half * (quad >> 1) + first + 8 * (i % mine);
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
        for (int i = 0; i < 4 * kGroups; ++i) {
          if (i < 4 * mine) {
            l[i] = add2(l[i], p[i]);
#pragma unroll
            for (int v = 0; v < Gv; ++v) pb[v][i] = fma2(p[i], vb[v], pb[v][i]);
          }
        }
      }
      // ---- the segment's record ----
      if (quad == set) spin_for(&sm.o_done[(g - 1) & 1], (g - 1) >> 1, abort_flag);
#pragma unroll
      for (int k = 0; k <= Gv; ++k) {
        float v[8 * kGroups];
#pragma unroll
        for (int i = 0; i < 4 * kGroups; ++i) { const float2 u = unpair64(k == 0 ? l[i] : pb[k - 1][i]); v[2 * i] = u.x; v[2 * i + 1] = u.y; }
        const float sum = column_sums(v);
        if (lane < 8 * kGroups) sm.red_sum[set][quad][k][lane] = sum;
      }
      if (tid == 0) mbar_arrive(&sm.q_free[slot]);       // the set has passed a barrier since it last read kappa
      set_sync(set);
      fence_after_sync();
      const bool bad = *abort_flag || sm.poisoned[n % kInfo];
      float* o_out = P.rec_o + (size_t)s.record * Sh::kRecord;
      float2* ml = P.rec_ml + (size_t)s.record * kRows;
      auto total = [&](int k, int c) { return (sm.red_sum[set][0][k][c] + sm.red_sum[set][1][k][c]) + (sm.red_sum[set][2][k][c] + sm.red_sum[set][3][k][c]); };
      if (tid < 8 * mine && first + tid < s.rows) ml[first + tid] = make_float2(-neg_ref[tid], bad ? -1.f : total(0, tid));
#pragma unroll 1
      for (int i = 0; i < mine * (Dv / 128); ++i) {
        const int m = i / mine, c0 = 8 * (i % mine);
        uint32_t o[8];
        tmem_ld8(lane_addr + Sh::kColO + 2 * kRows * m + 2 * half * (quad >> 1) + first + c0, o);
        wait_ld8(o);
        float* at = o_out + (size_t)(first + c0) * Dv + 128 * m + quad * 32 + lane;
#pragma unroll
        for (int c = 0; c < 8; ++c)
          if (first + c0 + c < s.rows) at[c * Dv] = fmaf(__uint_as_float(o[c]), 16777216.f, total(1 + 2 * m + (quad >> 1), c0 + c));
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
#pragma unroll 1
        for (uint32_t k = 0; k < kSpinLimit && !mbar_try_wait(&sm.drain, 0); ++k) {}
        raise_flag(P.flags, Q4KV_FLAG_INTERNAL);
      }
      __syncwarp();
    }
    fence_after_sync();
    tmem_dealloc(tb, 512);
  }
}

// One warp per (agent, query head): the records of the prefix's parts and the agent's own tokens, weighted by 2^(m - M).  Bound by
// the latency of the lengths and of the records in L2.
template <int Dv, int kRows>
__global__ void __launch_bounds__(128) shared_prefix_merge_kernel(const __grid_constant__ Params P) {
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  const int lane = threadIdx.x & 31, Hq = P.y.Hq, heads = P.y.Hkv, n_rep = P.y.n_rep;
  const int at = blockIdx.x * 4 + (threadIdx.x >> 5), a = at / Hq, head = at % Hq / n_rep, rep = at % n_rep;
  if (a >= P.n_agents) {                                 // (or the grid could complete before the one it follows)
    asm volatile("griddepcontrol.wait;" ::: "memory");
    return;
  }
  // the agent's group, where it begins in the list, and how the list was cut
  int total = 0, start = 0, tile0 = 0, tiles = 0;
  bool ascending = true, found = false;
  Group mine = {0, 0, 0, 0, 0, 0};
#pragma unroll 1
  for (int base = 0; base < P.n_groups; base += 32) {
    bool fine = true;
    const Group q = group_of<kRows>(P, base + lane, &fine);
    ascending = ascending && __all_sync(0xffffffffu, fine);
    const int cost = q.tiles * heads * q.cost, upto = total + inclusive_sum(cost), t = tiles + inclusive_sum(q.tiles);
    const unsigned here = __ballot_sync(0xffffffffu, q.n > 0 && q.agent0 <= a && a < q.agent0 + q.n);
    if (here && !found) {
      const int l = __ffs(here) - 1;
      found = true;
      mine.agent0 = __shfl_sync(0xffffffffu, q.agent0, l); mine.n = __shfl_sync(0xffffffffu, q.n, l);
      mine.prefix = __shfl_sync(0xffffffffu, q.prefix, l); mine.steps = __shfl_sync(0xffffffffu, q.steps, l);
      mine.tiles = __shfl_sync(0xffffffffu, q.tiles, l); mine.cost = __shfl_sync(0xffffffffu, q.cost, l);
      start = __shfl_sync(0xffffffffu, upto - cost, l);
      tile0 = __shfl_sync(0xffffffffu, t - q.tiles, l);
    }
    total = __shfl_sync(0xffffffffu, upto, 31);
    tiles = __shfl_sync(0xffffffffu, t, 31);
  }
  const int kv = P.kv_lens[a];
  const bool fine = ascending && found && kv >= 0 && kv <= P.max_kv_len && (kv == 0 || kv >= mine.prefix);
  if (!fine && lane == 0) raise_flag(P.flags, Q4KV_FLAG_BAD_LENGTH);
  int parts = 0;                                         // of the prefix
  const float *rec = P.rec_o, *rec_ml = (const float*)P.rec_ml;             // of the first part, then `stride` / `ml_stride` floats further
  size_t stride = (size_t)kRows * Dv, ml_stride = 2 * kRows;
  if (fine && kv > 0 && mine.steps > 0 && P.splits > 0) {
    parts = P.splits;
    stride = ml_stride = prefill_record(Dv);
    rec = P.tile_records + (size_t)at * parts * stride;
    rec_ml = rec + Dv;
  } else if (fine && kv > 0 && mine.steps > 0) {
    const Cut cut(total, P.grid);
    const int all = mine.n * n_rep, r = (a - mine.agent0) * n_rep + rep;
    const int t = (int)(((long long)(r + 1) * mine.tiles - 1) / all), segment = t * heads + head;      // the tile that holds row r
    const int u = start + segment * mine.cost, c = cut.cta_of(u);
    parts = cut.cta_of(u + mine.steps - 1) - c + 1;
    const int record = tile0 * heads + segment + c;
    const int row = r - tile_begin(all, mine.tiles, t);
    rec += (size_t)record * stride + (size_t)row * Dv;
    rec_ml += (size_t)record * ml_stride + 2 * row;
  }
  asm volatile("griddepcontrol.wait;" ::: "memory");
  constexpr int kQuads = Dv / 128, kAtOnce = 16 / kQuads;                  // parts whose numbers are asked for together with their weights
  float4 acc[kQuads];
  float M = -INFINITY, L = 0.f;
  bool bad = !fine || kv == 0;
#pragma unroll
  for (int k = 0; k < kQuads; ++k) acc[k] = make_float4(0.f, 0.f, 0.f, 0.f);
  if (!bad && kv > mine.prefix) {                        // the agent's own tokens: a sum that is missing had a bad block in it
    const float lse = __ldcg(P.own_lse + at);
#pragma unroll
    for (int k = 0; k < kQuads; ++k) acc[k] = __ldcg(reinterpret_cast<const float4*>(P.own_o + (size_t)at * Dv + 128 * k + 4 * lane));
    M = lse * kLog2e;
    L = 1.f;
    bad = lse == -INFINITY;
  }
#pragma unroll 1
  for (int base = 0; base < parts; base += kAtOnce) {
    const int n = min(kAtOnce, parts - base);
    const float2 ml = lane < n ? __ldcg(reinterpret_cast<const float2*>(rec_ml + (base + lane) * ml_stride)) : make_float2(-INFINITY, 0.f);
    float4 v[kAtOnce][kQuads];
#pragma unroll
    for (int j = 0; j < kAtOnce; ++j)
      if (j < n) {
#pragma unroll
        for (int k = 0; k < kQuads; ++k) v[j][k] = __ldcg(reinterpret_cast<const float4*>(rec + (base + j) * stride + 128 * k + 4 * lane));
      }
    bad |= __any_sync(0xffffffffu, ml.y < 0.f) != 0;
    const float m = fmaxf(M, warp_max(ml.x));
    const float keep = M == -INFINITY ? 0.f : fast_exp2(M - m), e = ml.x == -INFINITY ? 0.f : fast_exp2(ml.x - m);
    L = L * keep + warp_sum(e * ml.y);
    M = m;
#pragma unroll
    for (int k = 0; k < kQuads; ++k) { acc[k].x *= keep; acc[k].y *= keep; acc[k].z *= keep; acc[k].w *= keep; }
#pragma unroll
    for (int j = 0; j < kAtOnce; ++j) {
      const float f = __shfl_sync(0xffffffffu, e, j);
      if (j < n) {
#pragma unroll
        for (int k = 0; k < kQuads; ++k) {
          acc[k].x = fmaf(f, v[j][k].x, acc[k].x); acc[k].y = fmaf(f, v[j][k].y, acc[k].y);
          acc[k].z = fmaf(f, v[j][k].z, acc[k].z); acc[k].w = fmaf(f, v[j][k].w, acc[k].w);
        }
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

int max_rows_of(const Layout& y) { return y.D == 256 ? Shape<4, 4>::kRows : Shape<2, 2>::kRows; }
static_assert(Shape<3, 2>::kRows == Shape<2, 2>::kRows, "");

size_t align256(size_t n) { return (n + 255) & ~(size_t)255; }

// How a call is computed, by what the host knows of it.
//   kAlone: every agent by itself, one launch of the decode kernel.  kList: the prefixes by the kernel above.  kTiles: by the prefill
//   kernel, which expands a block once for 256 score rows (128 at d = 256 and 192 / 128) instead of unpacking it for 32.
enum class Route { kAlone, kList, kTiles };
// The launch of the prefill kernel: groups take the agents' place.  Its keys are cut into parts; the unit of time is a 64-key block of
// a tile, 1.3 us.  A CTA's start and end take four of them, and every part adds its records to what the merge reads, at 4 TB/s.
// 64 agents of 32 / 8 heads on 32768 tokens: 18 parts, 144 CTAs (with the 9 of an ordinary prefill call's plan, which allows for ragged
// tiles and stops at 16, 115 us a call instead of 88); 32 of 64 / 1 heads on 32000: 41.8 us instead of 56.4.
constexpr int kMaxTileSplits = 128;
struct TilePlan { int splits; double units; };
bool may_tile(const Layout& y) { return prefill_umma_supported(y) || prefill_umma_1tile_supported(y); }
// d = 128: two tiles of 128 rows to a CTA, or one where the average group has no more rows (8 KV heads of 4, 8 agents on 32000 tokens: 40.5 us
// a call, with two tiles 49.4; 8 in each of 3 groups on 8000 34.0 and 42.0)
bool two_tiles(const Layout& y, int n_agents, int n_groups) { return prefill_umma_supported(y) && (long long)n_agents * y.n_rep > 128ll * n_groups; }
TilePlan plan_tiles(const Layout& y, int n_agents, int n_groups, int max_kv_len, size_t bytes) {
  const long long sms = sm_count();
  const int queries = (two_tiles(y, n_agents, n_groups) ? 2 : 1) * (128 / y.n_rep);
  const long long ctas = (n_groups + (long long)(n_agents - n_groups) / queries) * y.Hkv;     // at most, however groups are cut
  const double blocks = max_kv_len / 64 + 1, merge = 1e-6 * prefill_record_bytes(y, n_agents, 1) / (4. * 1.3);
  TilePlan best = {1, 1e30};
  for (int s = 1; s <= kMaxTileSplits; ++s) {
    // the kernel numbers blocks times parts in 32 bits, a grid's second dimension in 16
    if (s > 1 && (s * 4 > blocks || (long long)y.Hkv * s > 65535 || (s + 1) * blocks > 2147483647. || prefill_record_bytes(y, n_agents, s) > bytes)) break;
    const double t = (double)((ctas * s + sms - 1) / sms) * (blocks / s + 4.) + s * merge;
    if (t < 0.97 * best.units) best = {s, t};
  }
  return best;
}

// The way with the least estimated time, in us.  m: megabytes of keys and values at the longest length, which is all that is known here,
// of one agent.  alone: a fixed part, m for every agent and every 8 (d = 128) or 4 query heads to a KV head, and the merge by output rows.
// list: m for every group and every 32 score rows (16 at d = 256; 16 or fewer at the other dimensions cost three quarters).  tiles: the
// plan's units.  Fitted to 330 measured cases of 2 to 96 agents in 1 or 3 groups on 2000 to 32000 shared tokens with 200 of their own, 1
// to 64 query heads to a KV head: the choice costs 0.6 % over the best of the three on average, 26 % at most.  It sees one average
// group and the longest length only: one group beside agents that share nothing (32 on 32000 tokens and 32 others: all alone, where
// the 32 on tiles would save 180 us by these estimates) and bounds far above the lengths are not its cases.  Measured alone / list /
// tiles, one group unless said otherwise:
//   8 KV heads of 4 query heads, d = 128, 4 agents on 8000     14.1 /  21.1 /  23.7      32 agents on 32000         206.4 / 99.4 / 43.7
//   8 KV heads of 1, d = 128, 8 agents on 8000 tokens          21.2 /  20.8 /  23.8      on 32000                    58.0 / 32.1 / 40.2
//   8 KV heads of 8, d = 128, 16 agents in each of 3 on 8000  107.3 / 100.2 /  71.3      2 agents on 2000: alone in every shape
//   8 KV heads of 2, d = 256, 16 agents on 32000              220.5 /  76.4 /  64.6      on 2000                     24.8 / 27.3 / 28.0
//   16 KV heads of 1, d = 192 and 128, 32 agents on 8000      132.6 /  53.6 /  42.3      on 2000                     46.3 / 39.5 / 34.7
struct RouteCost {
  double alone[3], list[3], tiles[3];      // fixed, a megabyte (tiles: a unit), a thousand output rows
};
Route route_of(const Layout& y, int n_agents, int n_groups, int max_kv_len, bool tiles_allowed) {
  if (n_groups >= n_agents) return Route::kAlone;        // nothing is shared
  constexpr RouteCost k128 = {{7., .185, 3.}, {18., .54, 5.}, {12., 1.13, 4.}}, k192 = {{7., .165, 3.}, {20., .5, 12.}, {12., .96, 7.}},
                      k256 = {{9., .18, 5.}, {23., .3, 9.}, {17.4, 1.25, 8.3}};
  constexpr double kOneTile = 0.89;                      // a unit of the one-tile kernel at d = 128
  const RouteCost& k = y.D == 128 ? k128 : y.D == 192 ? k192 : k256;
  const double m = 1e-6 * y.chunk_bytes / kChunkTokens * y.Hkv * max_kv_len, all = 1e-3 * n_agents * y.Hq;
  const double rows = (double)n_agents * y.n_rep / n_groups;             // of an average group and KV head
  const double passes = y.D == 256 ? ceil(rows / 16.) : rows <= 16. ? 0.75 : ceil(rows / 32.);
  const double alone = k.alone[0] + k.alone[1] * m * n_agents * ceil(y.n_rep / (y.D == 128 ? 8. : 4.)) + k.alone[2] * all;
  const double list = k.list[0] + k.list[1] * m * n_groups * passes + k.list[2] * all;
  double tiles = 1e30;
  if (tiles_allowed && may_tile(y)) {
    const double unit = y.D == 128 && !two_tiles(y, n_agents, n_groups) ? kOneTile : k.tiles[1];
    tiles = k.tiles[0] + unit * plan_tiles(y, n_agents, n_groups, max_kv_len, (size_t)-1).units + k.tiles[2] * all;
  }
  return alone <= list && alone <= tiles ? Route::kAlone : tiles < list ? Route::kTiles : Route::kList;
}

// The workspace behind the header: the decode launch's records, what it leaves for the agents' own tokens, the prefixes' records (a CTA
// of the list leaves one per segment it touches).  Tiles: sum over groups of ceil(rows / rows of a tile) at most.
struct Sections { size_t own_lse, own_o, rec_ml, rec_o, end; };
Sections sections_of(const Layout& y, int n_agents, int n_groups, int max_kv_len, Route route) {
  const size_t q_rows = (size_t)n_agents * y.Hq;
  Sections s;
  s.own_lse = align256(decode_mma_workspace_bytes(y, n_agents));
  s.own_o = s.own_lse + align256(q_rows * sizeof(float));
  s.rec_ml = s.own_o + align256(q_rows * y.Dv * sizeof(float));
  if (route == Route::kTiles) {
    s.rec_o = s.rec_ml;
    s.end = s.rec_o + align256(prefill_record_bytes(y, n_agents, plan_tiles(y, n_agents, n_groups, max_kv_len, (size_t)-1).splits));
  } else {
    const int rows = max_rows_of(y);
    const size_t tiles = q_rows / y.Hkv / rows + n_groups, records = tiles * y.Hkv + sm_count();
    s.rec_o = s.rec_ml + align256(records * rows * sizeof(float2));
    s.end = s.rec_o + align256(records * rows * y.Dv * sizeof(float));
  }
  return s;
}

template <class K, class... A>
cudaError_t launch_pdl(K kernel, int grid, int threads, size_t smem, cudaStream_t st, const A&... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(grid);
  cfg.blockDim = dim3(threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kernel, args...);
}

template <int G, int Gv, bool kBf>
cudaError_t launch_prefixes(const Params& P, cudaStream_t st) {
  static bool configured[64] = {};
  constexpr size_t smem = sizeof(Smem<G, Gv>);
  static_assert(smem <= 227 * 1024, "");
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  if (dev < 0 || dev >= 64 || !configured[dev]) {
    e = cudaFuncSetAttribute(shared_prefix_kernel<G, Gv, kBf>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
    if (e != cudaSuccess) return e;
    if (dev >= 0 && dev < 64) configured[dev] = true;
  }
  return launch_pdl(shared_prefix_kernel<G, Gv, kBf>, P.grid, kThreads, smem, st, P);
}
template <int G, int Gv>
cudaError_t launch_list(const Params& P, cudaStream_t st) {
  return P.y.sb_bf16 ? launch_prefixes<G, Gv, true>(P, st) : launch_prefixes<G, Gv, false>(P, st);
}
template <int Dv, int kRows>
cudaError_t launch_merge(const Params& P, cudaStream_t st) {
  return launch_pdl(shared_prefix_merge_kernel<Dv, kRows>, (P.n_agents * P.y.Hq + 3) / 4, 128, 0, st, P);
}

}  // namespace

bool shared_prefix_supported(const Layout& y, int n_agents, int max_blocks, int max_kv_len) {
  // the list's positions are 32-bit numbers
  return decode_mma_supported(y) && decode_mma_fits(y, n_agents, max_blocks) &&
         (2ll * n_agents * y.Hq / max_rows_of(y) + n_agents * y.Hkv) * (max_kv_len / 128 + 2 + kSegmentCost) < (1ll << 30);
}

// Whatever way a call takes, with as many parts of the tiles' keys as are planned.  least: with one part, which is what a call has to
// have; it grows with the agents and groups and does not depend on the lengths, so that one workspace serves smaller calls too.
size_t shared_prefix_workspace_bytes(const Layout& y, int n_agents, int n_groups, int max_kv_len, bool least) {
  const size_t list = sections_of(y, n_agents, n_groups, max_kv_len, Route::kList).end;
  if (!may_tile(y)) return list;
  const Sections tiles = sections_of(y, n_agents, n_groups, max_kv_len, Route::kTiles);
  const size_t end = least ? tiles.rec_o + prefill_record_bytes(y, n_agents, 1) : tiles.end;
  return end > list ? end : list;
}

// workspace: with its header (the decode launch's arrival counters)
cudaError_t launch_shared_prefix(const Layout& y, const void* pool, int n_blocks, int layer, const q4kv_batch& b, const int32_t* kv_lens,
                                 int max_kv_len, const int32_t* group_offs, const int32_t* prefix_lens, int n_groups, const void* q,
                                 float scale, bool tiles_allowed, void* out, int out_dtype, float* lse, void* workspace,
                                 size_t workspace_bytes, int32_t* flags, cudaStream_t st) {
  const Route route = route_of(y, b.n_agents, n_groups, max_kv_len, tiles_allowed);
  const int no_window = 0;
  if (route == Route::kAlone) {
    const DecodeGroups whole = {group_offs, prefix_lens, n_groups, true};
    return launch_decode_mma(y, pool, n_blocks, layer, b, kv_lens, max_kv_len, &no_window, 1, q, scale, out, out_dtype, lse, workspace,
                             flags, st, nullptr, nullptr, nullptr, nullptr, &whole);
  }
  const Sections s = sections_of(y, b.n_agents, n_groups, max_kv_len, route);
  uint8_t* at = (uint8_t*)workspace + kWorkspaceHeaderBytes;
  Params P;
  P.y = y; P.pool = (const uint8_t*)pool; P.n_blocks = n_blocks; P.layer = layer; P.n_agents = b.n_agents; P.max_blocks = b.max_blocks;
  P.tables = b.block_tables; P.kv_lens = kv_lens; P.max_kv_len = max_kv_len; P.group_offs = group_offs; P.prefix_lens = prefix_lens;
  P.n_groups = n_groups; P.grid = sm_count(); P.q = (const uint16_t*)q; P.scale_log2 = scale * kLog2e; P.out = out;
  P.out_dtype = out_dtype; P.lse = lse; P.flags = flags; P.own_lse = (float*)(at + s.own_lse); P.own_o = (float*)(at + s.own_o);
  P.rec_ml = (float2*)(at + s.rec_ml); P.rec_o = (float*)(at + s.rec_o); P.tile_records = P.rec_o; P.splits = 0;
  cudaError_t e;
  if (route == Route::kTiles) {
    PrefillExtra x = {};
    P.splits = x.n_splits = plan_tiles(y, b.n_agents, n_groups, max_kv_len, workspace_bytes - kWorkspaceHeaderBytes - s.rec_o).splits;
    x.records = P.rec_o; x.agent_lens = kv_lens; x.n_agents = b.n_agents; x.max_kv_len = max_kv_len;
    const q4kv_batch groups = {n_groups, b.max_blocks, b.block_tables};
    const auto launch = two_tiles(y, b.n_agents, n_groups) ? launch_prefill_umma : launch_prefill_umma_1tile;
    e = launch(y, pool, n_blocks, layer, groups, prefix_lens, group_offs, b.n_agents, 0, q, scale, nullptr, Q4KV_OUT_F32, nullptr, flags, st, x);
  } else {
    e = y.D == 128 ? launch_list<2, 2>(P, st) : y.D == 256 ? launch_list<4, 4>(P, st) : launch_list<3, 2>(P, st);
  }
  if (e != cudaSuccess) return e;
  const DecodeGroups own = {group_offs, prefix_lens, n_groups, false};
  e = launch_decode_mma(y, pool, n_blocks, layer, b, kv_lens, max_kv_len, &no_window, 1, q, scale, (void*)P.own_o, Q4KV_OUT_F32,
                        (float*)P.own_lse, workspace, flags, st, nullptr, nullptr, nullptr, nullptr, &own);
  if (e != cudaSuccess) return e;
  return y.D == 256 ? launch_merge<256, Shape<4, 4>::kRows>(P, st) : launch_merge<128, Shape<2, 2>::kRows>(P, st);
}

}  // namespace q4kv
