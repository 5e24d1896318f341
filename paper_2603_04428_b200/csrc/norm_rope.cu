// q4kv_norm_rope: the norm of every query and key head and the rotation by position, in one pass over the new rows -- what
// stands between a layer's projection and q4kv_quantize_append / q4kv_append_decode_attention / q4kv_prefill_attention.
//
//   y_e = x_e * rsqrt(mean of x^2 over the first norm_dim elements + eps) * (w_e + offset)      e < norm_dim
//   (y_a, y_b) -> scale * (y_a cos t - y_b sin t, y_b cos t + y_a sin t),  t = position * inv_freq[j]
//
// Every element is read once and written once (bound: HBM), a handful of binary32 operations each, rounded once to bfloat16
// (between the norm and the rotation nothing is rounded).  The angles are the expensive part: position * inv_freq is exact in
// binary64 (31 + 24 bits at most, rounded at 53), and reduced there, because in binary32 an angle of 10^5 is off by 4e-3.  All
// heads of a token share its angles, so a CTA takes one token (or a part of its heads, when there are few tokens), and its first
// threads turn rot_dim / 2 angles into cosines and sines in shared memory, before the wait for the preceding kernel.
//
// A head belongs to kLanes lanes with kVecs 16-byte pieces each, neighbouring lanes next to each other.  The other half of a
// rotated pair lies rot_dim / 16 pieces away: a shuffle when a lane holds one piece, else a second read (from L1).
#include "q4kv_layout.cuh"

namespace q4kv {

namespace {

constexpr int kThreads = 256;

struct Params {
  q4kv_norm_rotation how;
  int d, hq, hk;              // hq or hk is 0 when that side is not asked for
  int rows, n_agents;
  int parts, q_parts, part_heads;      // warps of a token, those of its query heads, heads of a warp
  const int32_t* pos;
  const int32_t* offs;
  const uint16_t* q;
  const uint16_t* k;
  long long q_stride, k_stride;
  uint16_t* q_out;
  uint16_t* k_out;
  int32_t* flags;
};

__device__ inline void unpack8(uint4 v, float (&x)[8]) {
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[2 * i] = __uint_as_float(w[i] << 16);
    x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
  }
}
__device__ inline uint4 pack8(const float (&x)[8]) {
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const __nv_bfloat162 b = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
    w[i] = *reinterpret_cast<const uint32_t*>(&b);
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}

__device__ inline void load8(const float* p, float (&x)[8]) {
  const float4 a = *reinterpret_cast<const float4*>(p), b = *reinterpret_cast<const float4*>(p + 4);
  x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w; x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
}

// A warp's work: heads [h_begin, h_end) of one token; kHeads: heads a lane works on at once (their loads are in flight together).
// kFew: a launch of few tokens, whose angles are ready before the wait for the preceding kernel; else the first heads' loads are in
// flight while the angles are computed.
template <int kLanes, int kVecs, int kHeads, bool kFew>
__global__ void __launch_bounds__(kThreads) norm_rope_kernel(const __grid_constant__ Params P) {
  extern __shared__ __align__(16) float turns[];         // a warp's cosines * rot_scale, then its sines * rot_scale
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  constexpr int kGroups = 32 / kLanes;
  const int lane = threadIdx.x & 31, warp = threadIdx.x / 32, group = lane / kLanes, l = lane % kLanes;
  const long long unit = (long long)blockIdx.x * (kThreads / 32) + warp;
  const int row = (int)(unit / P.parts), part = (int)(unit % P.parts), pieces = P.d / 8;
  if (row >= P.rows) return;                             // whole warps; no barrier of the block follows
  const bool is_q = part < P.q_parts;
  const int h_begin = (is_q ? part : part - P.q_parts) * P.part_heads, heads = is_q ? P.hq : P.hk, h_end = min(h_begin + P.part_heads, heads);
  const uint16_t* in = is_q ? P.q + row * P.q_stride : P.k + row * P.k_stride;
  uint16_t* out = is_q ? P.q_out + (size_t)row * heads * P.d : P.k_out + (size_t)row * heads * P.d;
  const uint16_t* w = P.how.norm_dim > 0 ? (const uint16_t*)(is_q ? P.how.q_weight : P.how.k_weight) : nullptr;
  uint4 v[kHeads][kVecs];
  auto load = [&](int h0) {
#pragma unroll
    for (int u = 0; u < kHeads; ++u) {
      const int h = h0 + u * kGroups + group;
#pragma unroll
      for (int i = 0; i < kVecs; ++i) {
        const int p = i * kLanes + l;
        v[u][i] = h < h_end && p < pieces ? *reinterpret_cast<const uint4*>(in + h * P.d + 8 * p) : make_uint4(0u, 0u, 0u, 0u);
      }
    }
  };
  if (!kFew) {
    asm volatile("griddepcontrol.wait;" ::: "memory");
    load(h_begin);
  }
  // the agent of the row: offsets at or below it
  int before = 0;
  for (int i = 0; i <= P.n_agents; i += 32) {
    const bool below = i + lane <= P.n_agents && P.offs[i + lane] <= row;
    const int n = __popc(__ballot_sync(0xffffffffu, below));
    before += n;
    if (n < 32) break;
  }
  if (before == 0 || before > P.n_agents) return;        // rows of no agent are left as they are
  const int first = P.pos[before - 1], ahead = row - P.offs[before - 1];
  const bool bad = first < 0;
  if (bad && lane == 0) raise_flag(P.flags, Q4KV_FLAG_BAD_LENGTH);
  const int half = P.how.rot_dim / 2;
  float* cosine = turns + warp * P.how.rot_dim;
  float* sine = cosine + half;
  const double position = (double)first + (double)ahead;
  for (int j = lane; j < half; j += 32) {
    const double t = position * (double)P.how.inv_freq[j] * 0.31830988618379067154;     // in half turns
    float s, c;
    sincospif((float)(t - 2.0 * rint(0.5 * t)), &s, &c);
    cosine[j] = c * P.how.rot_scale;
    sine[j] = s * P.how.rot_scale;
  }
  if (kFew) {
    asm volatile("griddepcontrol.wait;" ::: "memory");
    load(h_begin);
  }
  __syncwarp();
  const int rb = P.how.rot_begin / 8, re = rb + P.how.rot_dim / 8, apart = P.how.rot_dim / 16;     // in pieces
  auto turned = [&](int p) { return p >= rb && p < re; };
  auto mate = [&](int p) { return P.how.interleaved || !turned(p) ? p : p < rb + apart ? p + apart : p - apart; };
  auto weight = [&](int p, float (&g)[8]) {
    if (w && 8 * p < P.how.norm_dim) {
      unpack8(*reinterpret_cast<const uint4*>(w + 8 * p), g);
#pragma unroll
      for (int e = 0; e < 8; ++e) g[e] += P.how.weight_offset;
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) g[e] = 1.f;
    }
  };
  // piece p of a normed and turned head is own * x + other * z, z being the other elements of its pairs
  auto factors = [&](int p, float (&own)[8], float (&other)[8]) {
    weight(p, own);
    if (!turned(p)) {
#pragma unroll
      for (int e = 0; e < 8; ++e) other[e] = 0.f;
    } else if (P.how.interleaved) {
      const float4 c = *reinterpret_cast<const float4*>(cosine + 4 * (p - rb)), s = *reinterpret_cast<const float4*>(sine + 4 * (p - rb));
      const float cs[4] = {c.x, c.y, c.z, c.w}, sn[4] = {s.x, s.y, s.z, s.w};
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        other[2 * e] = -sn[e] * own[2 * e + 1];
        other[2 * e + 1] = sn[e] * own[2 * e];
        own[2 * e] *= cs[e];
        own[2 * e + 1] *= cs[e];
      }
    } else {
      const bool low = p < rb + apart;
      float c[8], s[8];
      load8(cosine + 8 * ((low ? p : p - apart) - rb), c);
      load8(sine + 8 * ((low ? p : p - apart) - rb), s);
      weight(mate(p), other);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        own[e] *= c[e];
        other[e] *= low ? -s[e] : s[e];
      }
    }
  };
  auto is_normed = [&](int p) { return w && 8 * p < P.how.norm_dim; };
  float own[8], other[8];
  if (kVecs == 1) factors(l, own, other);                // the same for all of the token's heads on this side
  for (int h0 = h_begin;;) {
    float norm[kHeads];
#pragma unroll
    for (int u = 0; u < kHeads; ++u) {
      norm[u] = 1.f;
      if (w) {
        float sum = 0.f;
#pragma unroll
        for (int i = 0; i < kVecs; ++i) {
          float x[8];
          unpack8(v[u][i], x);
          if (8 * (i * kLanes + l) < P.how.norm_dim) {
#pragma unroll
            for (int e = 0; e < 8; ++e) sum = fmaf(x[e], x[e], sum);
          }
        }
#pragma unroll
        for (int o = kLanes / 2; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o, kLanes);
        norm[u] = rsqrtf(sum / (float)P.how.norm_dim + P.how.eps);
      }
    }
#pragma unroll
    for (int i = 0; i < kVecs; ++i) {
      const int p = i * kLanes + l, q = mate(p);
      if (kVecs > 1) {
        if (p >= pieces || (!turned(p) && !is_normed(p))) continue;
        factors(p, own, other);
      }
#pragma unroll
      for (int u = 0; u < kHeads; ++u) {
        uint4 mates = v[u][i];
        if (!P.how.interleaved) {
          if (kVecs == 1) {                              // every lane takes part
            mates.x = __shfl_sync(0xffffffffu, mates.x, q, kLanes);
            mates.y = __shfl_sync(0xffffffffu, mates.y, q, kLanes);
            mates.z = __shfl_sync(0xffffffffu, mates.z, q, kLanes);
            mates.w = __shfl_sync(0xffffffffu, mates.w, q, kLanes);
          } else if (h0 + u * kGroups + group < h_end) {
            mates = *reinterpret_cast<const uint4*>(in + (h0 + u * kGroups + group) * P.d + 8 * q);
          }
        }
        float x[8], z[8];
        unpack8(v[u][i], x);
        unpack8(mates, z);
        const float nx = is_normed(p) ? norm[u] : 1.f, nz = is_normed(q) ? norm[u] : 1.f;
        const bool t = turned(p);
        float y[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float m = t ? (P.how.interleaved ? z[e ^ 1] : z[e]) : 0.f;       // what it is not paired with, it does not see
          y[e] = fmaf(m * nz, other[e], x[e] * nx * own[e]);
        }
        v[u][i] = pack8(y);
      }
    }
    if (kVecs > 1) __syncwarp();                         // rows that go back where they came from: all reads come first
#pragma unroll
    for (int u = 0; u < kHeads; ++u) {
      const int h = h0 + u * kGroups + group;
#pragma unroll
      for (int i = 0; i < kVecs; ++i) {
        const int p = i * kLanes + l;
        if (h < h_end && p < pieces) *reinterpret_cast<uint4*>(out + h * P.d + 8 * p) = bad ? make_uint4(0u, 0u, 0u, 0u) : v[u][i];
      }
    }
    h0 += kHeads * kGroups;
    if (h0 >= h_end) break;
    load(h0);
  }
}

// part_heads: heads of a warp
template <int kLanes, int kVecs, int kHeads, bool kFew>
cudaError_t launch(Params P, int part_heads, cudaStream_t st) {
  P.part_heads = part_heads;
  P.q_parts = (P.hq + part_heads - 1) / part_heads;
  P.parts = P.q_parts + (P.hk + part_heads - 1) / part_heads;
  constexpr int warps = kThreads / 32;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(((long long)P.rows * P.parts + warps - 1) / warps));
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = sizeof(float) * (size_t)P.how.rot_dim * warps;
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, norm_rope_kernel<kLanes, kVecs, kHeads, kFew>, P);
}
template <int kLanes, int kVecs, int kHeads>
cudaError_t launch(const Params& P, cudaStream_t st) {
  constexpr int at_once = 32 / kLanes;
  if (P.rows < 4 * sm_count()) return launch<kLanes, kVecs, 1, true>(P, at_once, st);
  return launch<kLanes, kVecs, kHeads, false>(P, at_once * kHeads * 2, st);
}

}  // namespace

cudaError_t launch_norm_rope(const Layout& y, const q4kv_norm_rotation& how, int n_agents, const int32_t* pos, const int32_t* offs,
                             int rows, const void* q, long long q_stride, const void* k, long long k_stride, void* q_out, void* k_out,
                             int32_t* flags, cudaStream_t st) {
  Params P;
  P.how = how;
  P.d = y.D; P.hq = q ? y.Hq : 0; P.hk = k ? y.Hkv : 0; P.rows = rows; P.n_agents = n_agents; P.pos = pos; P.offs = offs;
  P.q = (const uint16_t*)q; P.k = (const uint16_t*)k; P.q_stride = q_stride; P.k_stride = k_stride;
  P.q_out = (uint16_t*)q_out; P.k_out = (uint16_t*)k_out; P.flags = flags;
  if (y.D == 64) return launch<8, 1, 4>(P, st);
  if (y.D == 128) return launch<16, 1, 4>(P, st);
  if (y.D == 192) return launch<8, 3, 2>(P, st);
  if (y.D <= 256) return launch<32, 1, 4>(P, st);
  if (y.D <= 512) return launch<32, 2, 2>(P, st);
  if (y.D <= 768) return launch<32, 3, 1>(P, st);
  return launch<32, 4, 1>(P, st);
}

}  // namespace q4kv
