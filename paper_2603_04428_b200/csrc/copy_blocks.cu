// q4kv_copy_blocks: blocks of one pool into blocks of the same or another pool, all layers in one launch (forks, truncation
// into a shared block, compaction; Section 3.1 block pool).
//
// Nothing is computed: the floor is every copied byte read once and written once.  A block of one layer and KV head is one
// contiguous range of eight chunks (32 tokens each), and only the chunks that hold tokens are copied.  One CTA per (copy,
// layer, KV head), one warp per chunk: its lanes ask for a whole batch of 16-byte pieces before they store the first, so that
// what an SM has in flight (64 warps x 4.6 KB at d = 128) covers the latency of HBM several times over.
#include "q4kv_layout.cuh"

namespace q4kv {

namespace {

constexpr int kThreads = 32 * kChunksPerBlock;
constexpr int kBatch = 9;                                // 9 x 32 x 16 bytes: a chunk at d = 128, half of one at d = 256

__global__ void __launch_bounds__(kThreads)
copy_blocks_kernel(uint32_t chunk_bytes, int heads, const uint8_t* src, int src_blocks, uint8_t* dst, int dst_blocks, int layer0,
                   const int32_t* __restrict__ copies, int32_t* flags) {
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int i = blockIdx.x / heads, hk = blockIdx.x % heads, layer = layer0 + blockIdx.y;
  const int32_t* const mine = copies + 3 * (size_t)i;    // a long list passes 32 bits
  const int from = mine[0], to = mine[1], n = mine[2];
  const bool bad_block = from < 0 || from >= src_blocks || to < 0 || to >= dst_blocks, bad_length = n < 0 || n > kBlockTokens;
  if (bad_block || bad_length) {
    if (threadIdx.x == 0) raise_flag(flags, (bad_block ? Q4KV_FLAG_BAD_BLOCK : 0) | (bad_length ? Q4KV_FLAG_BAD_LENGTH : 0));
  }
  if (bad_block || bad_length || warp * kChunkTokens >= n || (from == to && src == dst)) {
    asm volatile("griddepcontrol.wait;" ::: "memory");   // or a grid without copies could complete before the one it follows
    return;
  }
  const size_t chunk = (size_t)hk * kChunksPerBlock + warp, per_block = (size_t)heads * kChunksPerBlock;
  const uint4* a = reinterpret_cast<const uint4*>(src + (((size_t)layer * src_blocks + from) * per_block + chunk) * chunk_bytes);
  uint4* b = reinterpret_cast<uint4*>(dst + (((size_t)layer * dst_blocks + to) * per_block + chunk) * chunk_bytes);
  const int pieces = chunk_bytes / 16;
  asm volatile("griddepcontrol.wait;" ::: "memory");
  for (int p = lane; p < pieces; p += 32 * kBatch) {
    uint4 v[kBatch];
#pragma unroll
    for (int k = 0; k < kBatch; ++k)
      if (p + 32 * k < pieces) v[k] = __ldcs(a + p + 32 * k);
#pragma unroll
    for (int k = 0; k < kBatch; ++k)
      if (p + 32 * k < pieces) __stcs(b + p + 32 * k, v[k]);
  }
}

}  // namespace

cudaError_t launch_copy_blocks(const Layout& y, const void* src, int src_blocks, void* dst, int dst_blocks, int layer0, int layers,
                               const int32_t* copies, int n_copies, int32_t* flags, cudaStream_t st) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)n_copies * y.Hkv, layers);
  cfg.blockDim = dim3(kThreads);
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, copy_blocks_kernel, y.chunk_bytes, y.Hkv, (const uint8_t*)src, src_blocks, (uint8_t*)dst, dst_blocks,
                            layer0, copies, flags);
}

}  // namespace q4kv
