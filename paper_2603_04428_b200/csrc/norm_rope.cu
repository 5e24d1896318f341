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
  int n_agents;
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

// kHeads: heads a thread works on at once (their loads are in flight together)
template <int kLanes, int kVecs, int kHeads>
__global__ void __launch_bounds__(kThreads) norm_rope_kernel(const __grid_constant__ Params P) {
  extern __shared__ float2 turn[];                       // (cos, sin) * rot_scale
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  const int row = blockIdx.x, lane = threadIdx.x & 31;
  // the agent of the row: offsets at or below it
  int before = 0;
  for (int i = 0; i <= P.n_agents; i += 32) {
    const bool below = i + lane <= P.n_agents && P.offs[i + lane] <= row;
    const int n = __popc(__ballot_sync(0xffffffffu, below));
    before += n;
    if (n < 32) break;
  }
  if (before == 0 || before > P.n_agents) return;        // rows of no agent are left as they are (uniform in the CTA)
  const int a = before - 1;
  const int first = P.pos[a];
  const bool bad = first < 0;
  if (bad && threadIdx.x == 0) raise_flag(P.flags, Q4KV_FLAG_BAD_LENGTH);
  const int half = P.how.rot_dim / 2;
  const double position = (double)first + (double)(row - P.offs[a]);
  for (int j = threadIdx.x; j < half; j += kThreads) {
    const double t = position * (double)P.how.inv_freq[j] * 0.31830988618379067154;     // in half turns
    float s, c;
    sincospif((float)(t - 2.0 * rint(0.5 * t)), &s, &c);
    turn[j] = make_float2(c * P.how.rot_scale, s * P.how.rot_scale);
  }
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const int group = threadIdx.x / kLanes, l = threadIdx.x % kLanes, pieces = P.d / 8;
  const uint16_t* in[kHeads];
  uint4 v[kHeads][kVecs];
#pragma unroll
  for (int u = 0; u < kHeads; ++u) {
    const int h = (blockIdx.y * kHeads + u) * (kThreads / kLanes) + group;
    in[u] = h < P.hq ? P.q + row * P.q_stride + (size_t)h * P.d
                     : h < P.hq + P.hk ? P.k + row * P.k_stride + (size_t)(h - P.hq) * P.d : nullptr;
#pragma unroll
    for (int i = 0; i < kVecs; ++i) {
      const int p = i * kLanes + l;
      v[u][i] = in[u] && p < pieces && !bad ? *reinterpret_cast<const uint4*>(in[u] + 8 * p) : make_uint4(0u, 0u, 0u, 0u);
    }
  }
  __syncthreads();                                       // the angles
  const int rb = P.how.rot_begin / 8, re = rb + P.how.rot_dim / 8, apart = P.how.rot_dim / 16;     // in pieces
#pragma unroll
  for (int u = 0; u < kHeads; ++u) {
    const int h = (blockIdx.y * kHeads + u) * (kThreads / kLanes) + group;
    const uint16_t* w = reinterpret_cast<const uint16_t*>(h < P.hq ? P.how.q_weight : P.how.k_weight);
    float norm = 1.f;
    if (P.how.norm_dim > 0) {                            // for every lane of a warp, whichever of its heads have a weight
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
      norm = rsqrtf(sum / (float)P.how.norm_dim + P.how.eps);
    }
    auto normed = [&](uint4 piece, int p, float (&x)[8]) {
      unpack8(piece, x);
      if (w && 8 * p < P.how.norm_dim) {
        float g[8];
        unpack8(*reinterpret_cast<const uint4*>(w + 8 * p), g);
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = x[e] * norm * (g[e] + P.how.weight_offset);
      }
    };
    uint4 y[kVecs];
#pragma unroll
    for (int i = 0; i < kVecs; ++i) {
      const int p = i * kLanes + l;
      float x[8];
      normed(v[u][i], p, x);
      const bool turned = p >= rb && p < re;
      if (P.how.interleaved) {
        if (turned) {
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float2 t = turn[4 * (p - rb) + e];
            const float x0 = x[2 * e], x1 = x[2 * e + 1];
            x[2 * e] = x0 * t.x - x1 * t.y;
            x[2 * e + 1] = x1 * t.x + x0 * t.y;
          }
        }
      } else {
        const bool low = p < rb + apart;
        const int q = turned ? (low ? p + apart : p - apart) : p;
        float z[8];
        if (kVecs == 1) {                                // every lane takes part
#pragma unroll
          for (int e = 0; e < 8; ++e) z[e] = __shfl_sync(0xffffffffu, x[e], q, kLanes);
        } else if (turned && in[u] && !bad) {
          normed(*reinterpret_cast<const uint4*>(in[u] + 8 * q), q, z);
        } else {
#pragma unroll
          for (int e = 0; e < 8; ++e) z[e] = 0.f;
        }
        if (turned) {
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const float2 t = turn[8 * ((low ? p : q) - rb) + e];
            x[e] = low ? x[e] * t.x - z[e] * t.y : x[e] * t.x + z[e] * t.y;
          }
        }
      }
      y[i] = pack8(x);
    }
    if (kVecs > 1) __syncwarp();                         // rows that go back where they came from: all reads come first
    uint16_t* out = h < P.hq ? P.q_out + ((size_t)row * P.hq + h) * P.d : P.k_out + ((size_t)row * P.hk + (h - P.hq)) * P.d;
#pragma unroll
    for (int i = 0; i < kVecs; ++i) {
      const int p = i * kLanes + l;
      if (in[u] && p < pieces) *reinterpret_cast<uint4*>(out + 8 * p) = bad ? make_uint4(0u, 0u, 0u, 0u) : y[i];
    }
  }
}

template <int kLanes, int kVecs, int kHeads>
cudaError_t launch(const Params& P, int rows, cudaStream_t st) {
  const int per_cta = kThreads / kLanes * kHeads;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(rows, (P.hq + P.hk + per_cta - 1) / per_cta);
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = sizeof(float2) * (size_t)(P.how.rot_dim / 2);
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, norm_rope_kernel<kLanes, kVecs, kHeads>, P);
}

}  // namespace

cudaError_t launch_norm_rope(const Layout& y, const q4kv_norm_rotation& how, int n_agents, const int32_t* pos, const int32_t* offs,
                             int rows, const void* q, long long q_stride, const void* k, long long k_stride, void* q_out, void* k_out,
                             int32_t* flags, cudaStream_t st) {
  Params P;
  P.how = how;
  P.d = y.D; P.hq = q ? y.Hq : 0; P.hk = k ? y.Hkv : 0; P.n_agents = n_agents; P.pos = pos; P.offs = offs;
  P.q = (const uint16_t*)q; P.k = (const uint16_t*)k; P.q_stride = q_stride; P.k_stride = k_stride;
  P.q_out = (uint16_t*)q_out; P.k_out = (uint16_t*)k_out; P.flags = flags;
  const bool few = rows < 4 * sm_count();                // few tokens: more CTAs, each with fewer heads
  if (y.D == 64) return few ? launch<8, 1, 1>(P, rows, st) : launch<8, 1, 4>(P, rows, st);
  if (y.D == 128) return few ? launch<16, 1, 1>(P, rows, st) : launch<16, 1, 4>(P, rows, st);
  if (y.D == 192) return few ? launch<8, 3, 1>(P, rows, st) : launch<8, 3, 2>(P, rows, st);
  if (y.D <= 256) return few ? launch<32, 1, 1>(P, rows, st) : launch<32, 1, 4>(P, rows, st);
  if (y.D <= 512) return launch<32, 2, 1>(P, rows, st);
  if (y.D <= 768) return launch<32, 3, 1>(P, rows, st);
  return launch<32, 4, 1>(P, rows, st);
}

}  // namespace q4kv
