// q4kv_norm_rope: the norm of every query and key head and the rotation by position, in one pass over the new rows -- what
// stands between a layer's projection and q4kv_quantize_append / q4kv_append_decode_attention / q4kv_prefill_attention.
//
//   y_e = x_e * rsqrt(mean of x^2 over the first norm_dim elements + eps) * (w_e + offset)      e < norm_dim
//   (y_a, y_b) -> scale * (y_a cos t - y_b sin t, y_b cos t + y_a sin t),  t = position * inv_freq[j]
//
// Every element is read once and written once (bound: HBM), a handful of binary32 operations each, rounded once to bfloat16
// (between the norm and the rotation nothing is rounded).  The angles are the expensive part: they are taken, in half turns, and
// reduced in binary64 (position / pi and its product with inv_freq are each rounded once, less than 2^-51 of the angle together), because in
// binary32 an angle of 10^5 is off by 4e-3.  All heads of a token share its angles, and what norm weights and angles make of an
// element's two factors: a warp takes one token, or, when there are few tokens, a part of its heads, whose angles it then turns again
// (twice a token at 4900 tokens, five or six times at 600 to 2000).  It turns rot_dim / 2 angles into cosines and sines in its part of
// shared memory and keeps the factors of its elements in registers for all of its heads.  Warps never wait for one another.
//
// A head belongs to kLanes lanes with kVecs 16-byte pieces each, neighbouring lanes next to each other.  Where the whole head turns in
// pairs half a head apart, a lane holds both halves of its pairs.  Else the other half lies rot_dim / 16 pieces away: a shuffle when a
// lane holds one piece, else a second read (from L1).
//
// 4900 tokens of 24 heads, d = 256, norm and rotation: 27 us (4.4 TB/s; 59 with a block to a token, whose lanes read their angles for
// every head); 32768 of 40 heads, d = 128, rotation: 105 us (6.4 TB/s); 32768 of 32 heads, d = 192, 64 elements in adjacent pairs: 123 us
// (6.6 TB/s).  Five tokens of 40 heads: 5 us, a launch and a chain of three reads.
#include <climits>

#include "f32x2.cuh"
#include "q4kv_layout.cuh"

namespace q4kv {

namespace {

constexpr int kThreads = 128;
constexpr int ctas_of(int vecs) { return vecs > 2 ? 5 : 6; }       // on an SM: the registers' limit

struct Params {
  q4kv_norm_rotation how;
  float inv_norm_dim;
  int d, hq, hk;              // hq or hk is 0 when that side is not asked for
  int rows, n_agents;
  int part_heads;             // heads of a warp: query heads first, then key heads
  const int32_t* pos;
  const int32_t* offs;
  const uint16_t* q;
  const uint16_t* k;
  long long q_stride, k_stride;
  uint16_t* q_out;
  uint16_t* k_out;
  int32_t* flags;
};

// eight elements as four pairs of binary32 numbers
struct Eight { uint64_t v[4]; };
__device__ __forceinline__ uint64_t pair(float a, float b) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ float2 parts_of(uint64_t v) {
  float2 r;
  asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(v));
  return r;
}
__device__ __forceinline__ Eight unpack8(uint4 v) {
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
  Eight x;
#pragma unroll
  for (int i = 0; i < 4; ++i) x.v[i] = pair(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xffff0000u));
  return x;
}
__device__ __forceinline__ uint4 pack8(const Eight& x) {
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 f = parts_of(x.v[i]);
    const __nv_bfloat162 b = __floats2bfloat162_rn(f.x, f.y);
    w[i] = *reinterpret_cast<const uint32_t*>(&b);
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}
__device__ __forceinline__ Eight load8(const float* p) {
  const float4 a = *reinterpret_cast<const float4*>(p), b = *reinterpret_cast<const float4*>(p + 4);
  return {pair(a.x, a.y), pair(a.z, a.w), pair(b.x, b.y), pair(b.z, b.w)};
}
__device__ __forceinline__ Eight times(const Eight& a, const Eight& b) {
  return {mul2(a.v[0], b.v[0]), mul2(a.v[1], b.v[1]), mul2(a.v[2], b.v[2]), mul2(a.v[3], b.v[3])};
}
__device__ __forceinline__ Eight times(const Eight& a, float f) {
  const uint64_t b = pair(f, f);
  return {mul2(a.v[0], b), mul2(a.v[1], b), mul2(a.v[2], b), mul2(a.v[3], b)};
}
__device__ __forceinline__ Eight times_plus(const Eight& a, const Eight& b, const Eight& c) {
  return {fma2(a.v[0], b.v[0], c.v[0]), fma2(a.v[1], b.v[1], c.v[1]), fma2(a.v[2], b.v[2], c.v[2]), fma2(a.v[3], b.v[3], c.v[3])};
}
__device__ __forceinline__ uint32_t halves_swapped(uint32_t w) { return __funnelshift_l(w, w, 16); }

// A warp's work: heads [h_begin, h_end) of one token, counted over the query heads and then the key heads; kHeads: heads a lane works
// on at once (their loads are in flight together).  kFew: a launch of few tokens, whose angles are ready before the wait for the
// preceding kernel; else the first heads' loads are in flight while the angles are computed.  kWhole: the whole head turns in pairs half
// a head apart, and a lane holds both (kVecs == 2).
template <int kLanes, int kVecs, int kHeads, bool kWhole, bool kFew>
__global__ void __launch_bounds__(kThreads, kFew ? 1 : ctas_of(kVecs)) norm_rope_kernel(const __grid_constant__ Params P) {
  static_assert(!kWhole || kVecs == 2, "");
  extern __shared__ __align__(16) float turns[];         // a warp's cosines * rot_scale, then its sines * rot_scale
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  constexpr int kGroups = 32 / kLanes, kStep = kGroups * kHeads, kEarly = 4;
  const int lane = threadIdx.x & 31, warp = threadIdx.x / 32, group = lane / kLanes, l = lane % kLanes;
  const int row = blockIdx.x * (kThreads / 32) + warp, part = blockIdx.y, d = kWhole ? 16 * kLanes : P.d, pieces = d / 8;
  if (row >= P.rows) {                                   // whole warps; no barrier of the block follows
    asm volatile("griddepcontrol.wait;" ::: "memory");   // or this grid could complete before the one it follows
    return;
  }
  const int h_begin = part * P.part_heads, h_last = min(h_begin + P.part_heads, P.hq + P.hk);
  // one side at a time: its heads [h, h_end) of in and out
  const uint16_t* in;
  uint16_t* out;
  int h, h_end;
  auto side = [&](bool is_q) {
    in = is_q ? P.q + row * P.q_stride : P.k + row * P.k_stride;
    out = is_q ? P.q_out + (size_t)row * P.hq * d : P.k_out + (size_t)row * P.hk * d;
    h = is_q ? h_begin : max(h_begin - P.hq, 0);
    h_end = is_q ? min(h_last, P.hq) : h_last - P.hq;
  };
  uint4 v[kHeads][kVecs];
  auto load = [&] {
#pragma unroll
    for (int u = 0; u < kHeads; ++u) {
      const int at = h + u * kGroups + group;
#pragma unroll
      for (int i = 0; i < kVecs; ++i) {
        const int p = i * kLanes + l;
        v[u][i] = at < h_end && p < pieces ? *reinterpret_cast<const uint4*>(in + at * d + 8 * p) : make_uint4(0u, 0u, 0u, 0u);
      }
    }
  };
  bool is_q = h_begin < P.hq;
  side(is_q);
  if (!kFew) {
    asm volatile("griddepcontrol.wait;" ::: "memory");
    load();
  }
  const int half = P.how.rot_dim / 2;
  float freq[kEarly];                                    // of a head of up to 256 elements
#pragma unroll
  for (int i = 0; i < kEarly; ++i) freq[i] = lane + 32 * i < half ? P.how.inv_freq[lane + 32 * i] : 0.f;
  if (kFew) {                                            // the rows, on their way to L2 before the wait
    for (int p = 4 * lane; p < (h_end - h) * pieces; p += 128)
      asm volatile("prefetch.global.L2 [%0];" ::"l"(in + h * d + 8 * p) : "memory");
  }
  // the agent of the row: offsets at or below it
  int before = 0, first = 0, start = 0;
  for (int i = 0; i <= P.n_agents; i += 32) {
    const int a = i + lane, off = a <= P.n_agents ? P.offs[a] : INT_MAX, pos = a < P.n_agents ? P.pos[a] : 0;
    const int n = __popc(__ballot_sync(0xffffffffu, a <= P.n_agents && off <= row));
    before += n;
    if (n > 0) {
      first = __shfl_sync(0xffffffffu, pos, n - 1);
      start = __shfl_sync(0xffffffffu, off, n - 1);
    }
    if (n < 32) break;
  }
  if (before == 0 || before > P.n_agents) {              // rows of no agent are left as they are
    if (kFew) asm volatile("griddepcontrol.wait;" ::: "memory");
    return;
  }
  const int ahead = row - start;
  const bool bad = first < 0;
  if (bad && lane == 0) raise_flag(P.flags, Q4KV_FLAG_BAD_LENGTH);
  float* cosine = turns + warp * P.how.rot_dim;
  float* sine = cosine + half;
  const double position = ((double)first + (double)ahead) * 0.31830988618379067154;     // in half turns for an angle of one
  auto turn = [&](int j, float f) {
    const double t = position * (double)f;
    float s, c;
    sincospif((float)(t - 2.0 * rint(0.5 * t)), &s, &c);
    cosine[j] = c * P.how.rot_scale;
    sine[j] = s * P.how.rot_scale;
  };
#pragma unroll
  for (int i = 0; i < kEarly; ++i)
    if (lane + 32 * i < half) turn(lane + 32 * i, freq[i]);
  for (int j = lane + 32 * kEarly; j < half; j += 32) turn(j, P.how.inv_freq[j]);
  if (kFew) {
    asm volatile("griddepcontrol.wait;" ::: "memory");
    load();
  }
  __syncwarp();
  const int rb = P.how.rot_begin / 8, re = rb + P.how.rot_dim / 8, apart = P.how.rot_dim / 16;     // in pieces
  const bool neighbours = !kWhole && P.how.interleaved;
  auto turned = [&](int p) { return kWhole || (p >= rb && p < re); };
  auto mate = [&](int p) { return neighbours || !turned(p) ? p : p < rb + apart ? p + apart : p - apart; };

  for (;;) {                                             // a side
    const uint16_t* w = P.how.norm_dim > 0 ? (const uint16_t*)(is_q ? P.how.q_weight : P.how.k_weight) : nullptr;
    auto normed = [&](int p) { return w && 8 * p < P.how.norm_dim; };
    auto weight = [&](int p) {
      if (!normed(p)) return Eight{pair(1.f, 1.f), pair(1.f, 1.f), pair(1.f, 1.f), pair(1.f, 1.f)};
      Eight g = unpack8(*reinterpret_cast<const uint4*>(w + 8 * p));
      const uint64_t o = pair(P.how.weight_offset, P.how.weight_offset);
#pragma unroll
      for (int e = 0; e < 4; ++e) g.v[e] = add2(g.v[e], o);
      return g;
    };
    // piece p of a normed and turned head is own * x + other * z, z being the other elements of its pairs
    auto factors = [&](int p, Eight& own, Eight& other) {
      own = weight(p);
      if (!turned(p)) {
        other = {};
      } else if (neighbours) {
        const float4 c = *reinterpret_cast<const float4*>(cosine + 4 * (p - rb)), s = *reinterpret_cast<const float4*>(sine + 4 * (p - rb));
        const float cs[4] = {c.x, c.y, c.z, c.w}, sn[4] = {s.x, s.y, s.z, s.w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float2 g = parts_of(own.v[e]);
          other.v[e] = pair(-sn[e] * g.y, sn[e] * g.x);
          own.v[e] = pair(cs[e] * g.x, cs[e] * g.y);
        }
      } else {
        const bool low = p < rb + apart;
        const int j = 8 * ((low ? p : p - apart) - rb);
        other = times(times(weight(mate(p)), load8(sine + j)), low ? -1.f : 1.f);
        own = times(own, load8(cosine + j));
      }
    };
    constexpr int kKept = kWhole ? 2 : 1;
    Eight own[kKept], other[kKept];                      // the same for all of the token's heads on this side
    if (kVecs == kKept) {
#pragma unroll
      for (int i = 0; i < kKept; ++i) factors(i * kLanes + l, own[i], other[i]);
    }
    for (;;) {                                           // kStep heads
      float norm[kHeads];
#pragma unroll
      for (int u = 0; u < kHeads; ++u) norm[u] = 1.f;
      if (w) {
#pragma unroll
        for (int u = 0; u < kHeads; ++u) {
          uint64_t sums = 0;
#pragma unroll
          for (int i = 0; i < kVecs; ++i) {
            if (normed(i * kLanes + l)) {
              const Eight x = unpack8(v[u][i]);
#pragma unroll
              for (int e = 0; e < 4; ++e) sums = fma2(x.v[e], x.v[e], sums);
            }
          }
          const float2 s = parts_of(sums);
          float sum = s.x + s.y;
#pragma unroll
          for (int o = kLanes / 2; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o, kLanes);
          norm[u] = rsqrtf(fmaf(sum, P.inv_norm_dim, P.how.eps));
        }
      }
      if (kWhole) {
        const bool n0 = normed(l), n1 = normed(kLanes + l);
#pragma unroll
        for (int u = 0; u < kHeads; ++u) {
          Eight a = unpack8(v[u][0]), b = unpack8(v[u][kVecs - 1]);
          if (w) {
            a = times(a, n0 ? norm[u] : 1.f);
            b = times(b, n1 ? norm[u] : 1.f);
          }
          v[u][0] = pack8(times_plus(b, other[0], times(a, own[0])));
          v[u][kVecs - 1] = pack8(times_plus(a, other[kKept - 1], times(b, own[kKept - 1])));
        }
      } else {
#pragma unroll
        for (int i = 0; i < kVecs; ++i) {
          const int p = i * kLanes + l, q = mate(p);
          if (kVecs > 1) {
            if (p >= pieces || (!turned(p) && !normed(p))) continue;
            factors(p, own[0], other[0]);
          }
#pragma unroll
          for (int u = 0; u < kHeads; ++u) {
            uint4 z = v[u][i];
            if (neighbours) {
              z = make_uint4(halves_swapped(z.x), halves_swapped(z.y), halves_swapped(z.z), halves_swapped(z.w));
            } else if (kVecs == 1) {                     // every lane takes part
              z = make_uint4(__shfl_sync(0xffffffffu, z.x, q, kLanes), __shfl_sync(0xffffffffu, z.y, q, kLanes),
                             __shfl_sync(0xffffffffu, z.z, q, kLanes), __shfl_sync(0xffffffffu, z.w, q, kLanes));
            } else if (h + u * kGroups + group < h_end) {
              z = *reinterpret_cast<const uint4*>(in + (h + u * kGroups + group) * d + 8 * q);
            }
            if (!turned(p)) z = make_uint4(0u, 0u, 0u, 0u);        // what it is not paired with, it does not see
            const Eight x = times(unpack8(v[u][i]), normed(p) ? norm[u] : 1.f);
            v[u][i] = pack8(times_plus(times(unpack8(z), normed(q) ? norm[u] : 1.f), other[0], times(x, own[0])));
          }
        }
        if (kVecs > 1) __syncwarp();                     // rows that go back where they came from: all reads come first
      }
#pragma unroll
      for (int u = 0; u < kHeads; ++u) {
        const int at = h + u * kGroups + group;
#pragma unroll
        for (int i = 0; i < kVecs; ++i) {
          const int p = i * kLanes + l;
          if (at < h_end && p < pieces) *reinterpret_cast<uint4*>(out + at * d + 8 * p) = bad ? make_uint4(0u, 0u, 0u, 0u) : v[u][i];
        }
      }
      h += kStep;
      if (h >= h_end) break;
      load();
    }
    if (!is_q || h_last <= P.hq) break;
    side(is_q = false);
    load();
  }
}

// part_heads: heads of a warp
template <int kLanes, int kVecs, int kHeads, bool kWhole, bool kFew>
cudaError_t launch(Params P, int part_heads, cudaStream_t st) {
  P.part_heads = part_heads;
  constexpr int warps = kThreads / 32;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((P.rows - 1) / warps + 1, (P.hq + P.hk - 1) / part_heads + 1);
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = sizeof(float) * (size_t)P.how.rot_dim * warps;
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, norm_rope_kernel<kLanes, kVecs, kHeads, kWhole, kFew>, P);
}
template <int kLanes, int kVecs, int kHeads, bool kWhole>
cudaError_t launch(const Params& P, cudaStream_t st) {
  constexpr int at_once = 32 / kLanes;
  // few tokens: a warp to each group of heads, the angles before the wait
  if (P.rows < 4 * sm_count()) return launch<kLanes, kVecs, 1, kWhole, true>(P, at_once, st);
  // One warp to a token computes its angles once; parts of a token balance the load.  At least twice as many warps as fit the GPU:
  // 4900 tokens of 24 heads, d = 256, 27.2 us; once 28.5, four times 28.5; 4096 of 40 at d = 128 20.4, 22.4, 24.1 us; for 32768 all the same.
  const int steps = (P.hq + P.hk - 1) / (at_once * kHeads) + 1;
  const long long fit = 2ll * sm_count() * ctas_of(kVecs) * (kThreads / 32), each = (long long)P.rows * steps / fit;
  const int parts = each < 2 ? steps : each >= steps ? 1 : (steps - 1) / (int)each + 1;
  return launch<kLanes, kVecs, kHeads, kWhole, false>(P, at_once * kHeads * ((steps - 1) / parts + 1), st);
}

}  // namespace

cudaError_t launch_norm_rope(const Layout& y, const q4kv_norm_rotation& how, int n_agents, const int32_t* pos, const int32_t* offs,
                             int rows, const void* q, long long q_stride, const void* k, long long k_stride, void* q_out, void* k_out,
                             int32_t* flags, cudaStream_t st) {
  Params P;
  P.how = how;
  P.inv_norm_dim = how.norm_dim > 0 ? 1.f / (float)how.norm_dim : 0.f;
  P.d = y.D; P.hq = q ? y.Hq : 0; P.hk = k ? y.Hkv : 0; P.rows = rows; P.n_agents = n_agents; P.pos = pos; P.offs = offs;
  P.q = (const uint16_t*)q; P.k = (const uint16_t*)k; P.q_stride = q_stride; P.k_stride = k_stride;
  P.q_out = (uint16_t*)q_out; P.k_out = (uint16_t*)k_out; P.flags = flags;
  if (!how.interleaved && how.rot_dim == y.D) {
    if (y.D == 64) return launch<4, 2, 2, true>(P, st);
    if (y.D == 128) return launch<8, 2, 2, true>(P, st);
    if (y.D == 256) return launch<16, 2, 2, true>(P, st);
  }
  if (y.D == 64) return launch<8, 1, 4, false>(P, st);
  if (y.D == 128) return launch<16, 1, 4, false>(P, st);
  if (y.D == 192) return launch<8, 3, 2, false>(P, st);
  if (y.D <= 256) return launch<32, 1, 4, false>(P, st);
  if (y.D <= 512) return launch<32, 2, 2, false>(P, st);
  if (y.D <= 768) return launch<32, 3, 1, false>(P, st);
  return launch<32, 4, 1, false>(P, st);
}

}  // namespace q4kv
