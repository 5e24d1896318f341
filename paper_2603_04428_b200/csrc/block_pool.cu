// Block pool bookkeeping and the dense-batch shim (Section 3.1 "Block Pool with Per-Agent Isolation"; Section 3.4
// BatchQuantizedKVCache.merge / extract).
//
// The allocator is host-side policy: it hands out the pool's 256-token blocks to agents (each block belongs to one agent
// at a time, so no agent can read another's cache, unless the caller forks an agent: parent and child then share whole
// blocks, which are counted and become free with their last holder), keeps a least-recently-used order of the agents, and
// names the agent to evict when the pool is full.  It never touches device memory; persisting a victim before its blocks are
// reused is the caller's step (q4kv_save), which is why eviction is a two-call affair: pick, then release.
//
// merge / extract exist in the paper because its framework attends over dense tensors: caches of different lengths
// are left-padded to a common length and stacked.  This library attends through block tables and needs neither, but
// code written against the dense form can move a layer's batch into the pool (merge) and out of it (extract).
#include <algorithm>
#include <cstdlib>
#include <cstring>
#include <list>
#include <new>
#include <unordered_map>
#include <vector>

#include "q4kv_layout.cuh"

using namespace q4kv;

struct q4kv_allocator {
  struct Agent {
    std::vector<int32_t> blocks;
    bool pinned = false;
    std::list<int64_t>::iterator lru_pos;
  };
  int32_t n_blocks = 0;
  std::vector<int32_t> free_list;                    // a stack: the most recently freed block is reused first
  std::unordered_map<int64_t, Agent> agents;
  std::list<int64_t> lru;                            // front: least recently used
  std::vector<int32_t> holders;                      // per block: the agents whose lists hold it
};

namespace {

void touch(q4kv_allocator* al, q4kv_allocator::Agent& ag) { al->lru.splice(al->lru.end(), al->lru, ag.lru_pos); }   // moves the node

// A block's use by one agent begins or ends.  Neither allocates: free_list was given room for every block.
int32_t take_block(q4kv_allocator* al) {
  const int32_t b = al->free_list.back();
  al->free_list.pop_back();
  al->holders[b] = 1;
  return b;
}
void drop_block(q4kv_allocator* al, int32_t b) {
  if (--al->holders[b] == 0) al->free_list.push_back(b);
}

void write_row(const q4kv_allocator::Agent& ag, int32_t* table_row, int32_t max_blocks) {
  for (int32_t i = 0; i < max_blocks; ++i) table_row[i] = i < (int32_t)ag.blocks.size() ? ag.blocks[i] : -1;
}

void set_copy(int32_t* copy, int32_t from, int32_t to, int32_t tokens) { copy[0] = from; copy[1] = to; copy[2] = tokens; }

size_t dense_need(const q4kv_spec* spec, int32_t n_agents, int32_t T) {
  const Layout y = make_layout(*spec, 1);
  const size_t rows = (size_t)n_agents * y.Hkv * T;
  return rows * ((size_t)y.D / 2 + 4 * y.G + (y.alias ? 0 : (size_t)y.Dv / 2 + 4 * y.Gv));
}

int dense_call(const q4kv_spec* spec, void* pool, int32_t n_blocks, int32_t layer, const q4kv_batch* batch,
               const int32_t* kv_lens, int32_t T, void* dense, size_t dense_bytes, bool to_pool, int32_t* flags,
               void* stream) {
  if (!spec || !batch || !pool || n_blocks <= 0 || T <= 0 || batch->n_agents < 0 || batch->max_blocks <= 0) return Q4KV_EINVAL;
  if (q4kv_pool_bytes(spec, n_blocks) == 0) return Q4KV_EUNSUPPORTED;
  if (layer < 0 || layer >= spec->n_layers) return Q4KV_EINVAL;
  if (batch->n_agents == 0) return Q4KV_OK;
  if (!kv_lens || !dense || !batch->block_tables) return Q4KV_EINVAL;
  if ((reinterpret_cast<uintptr_t>(pool) | reinterpret_cast<uintptr_t>(dense)) & 15u) return Q4KV_EINVAL;
  const size_t need = dense_need(spec, batch->n_agents, T);
  if (dense_bytes < need) return Q4KV_EWORKSPACE;
  const Layout y = make_layout(*spec, n_blocks);
  cudaStream_t st = (cudaStream_t)stream;
  if (!to_pool && cudaMemsetAsync(dense, 0, need, st) != cudaSuccess) return Q4KV_ECUDA;   // the left padding is zero bytes
  const cudaError_t e = launch_dense_exchange(y, pool, n_blocks, layer, *batch, kv_lens, T, dense, to_pool, flags, st);
  return e == cudaSuccess ? Q4KV_OK : Q4KV_ECUDA;
}

}  // namespace

extern "C" {

q4kv_allocator* q4kv_allocator_create(int32_t n_blocks) {
  if (n_blocks <= 0) return nullptr;
  q4kv_allocator* al = new (std::nothrow) q4kv_allocator;
  if (!al) return nullptr;
  al->n_blocks = n_blocks;
  try {
    al->free_list.reserve(n_blocks);
    al->holders.assign(n_blocks, 0);
  } catch (...) {                                      // no host memory
    delete al;
    return nullptr;
  }
  for (int32_t b = n_blocks - 1; b >= 0; --b) al->free_list.push_back(b);   // block 0 is handed out first
  return al;
}

void q4kv_allocator_destroy(q4kv_allocator* al) { delete al; }

int32_t q4kv_allocator_free_blocks(const q4kv_allocator* al) { return al ? (int32_t)al->free_list.size() : -1; }

int32_t q4kv_allocator_agent_blocks(const q4kv_allocator* al, int64_t agent_id) {
  if (!al) return -1;
  const auto it = al->agents.find(agent_id);
  return it == al->agents.end() ? 0 : (int32_t)it->second.blocks.size();
}

int q4kv_allocator_reserve(q4kv_allocator* al, int64_t agent_id, int32_t n_tokens, int32_t* table_row, int32_t max_blocks) {
  if (!al || n_tokens < 0 || !table_row || max_blocks <= 0) return Q4KV_EINVAL;
  const int32_t want = n_tokens / kBlockTokens + (n_tokens % kBlockTokens ? 1 : 0);
  if (want > max_blocks) return Q4KV_EINVAL;
  auto it = al->agents.find(agent_id);
  const int32_t have = it == al->agents.end() ? 0 : (int32_t)it->second.blocks.size();
  if (want > have && (size_t)(want - have) > al->free_list.size()) return Q4KV_EWORKSPACE;   // evict first (pick a victim)
  try {                                                // everything that can fail comes before the first change
    if (it == al->agents.end()) {
      q4kv_allocator::Agent fresh;
      fresh.blocks.reserve(want);
      std::list<int64_t> node(1, agent_id);
      it = al->agents.emplace(agent_id, std::move(fresh)).first;
      al->lru.splice(al->lru.end(), node);
      it->second.lru_pos = std::prev(al->lru.end());
    } else {
      std::vector<int32_t>& blocks = it->second.blocks;
      if ((size_t)want > blocks.capacity()) blocks.reserve(std::max((size_t)want, std::min(2 * blocks.capacity(), (size_t)al->n_blocks)));
      touch(al, it->second);
    }
  } catch (...) {                                      // no host memory
    return Q4KV_EWORKSPACE;
  }
  q4kv_allocator::Agent& ag = it->second;
  while ((int32_t)ag.blocks.size() < want) ag.blocks.push_back(take_block(al));
  write_row(ag, table_row, max_blocks);
  return Q4KV_OK;
}

int q4kv_allocator_touch(q4kv_allocator* al, int64_t agent_id) {
  if (!al) return Q4KV_EINVAL;
  const auto it = al->agents.find(agent_id);
  if (it == al->agents.end()) return Q4KV_EINVAL;
  touch(al, it->second);
  return Q4KV_OK;
}

int q4kv_allocator_pin(q4kv_allocator* al, int64_t agent_id, int32_t pinned) {
  if (!al) return Q4KV_EINVAL;
  const auto it = al->agents.find(agent_id);
  if (it == al->agents.end()) return Q4KV_EINVAL;
  it->second.pinned = pinned != 0;
  return Q4KV_OK;
}

int q4kv_allocator_pick_victim(const q4kv_allocator* al, int64_t* agent_id) {
  if (!al || !agent_id) return Q4KV_EINVAL;
  for (const int64_t id : al->lru) {
    const auto it = al->agents.find(id);
    if (it != al->agents.end() && !it->second.pinned && !it->second.blocks.empty()) { *agent_id = id; return Q4KV_OK; }
  }
  return Q4KV_EWORKSPACE;                              // every agent that holds blocks is pinned
}

int q4kv_allocator_release(q4kv_allocator* al, int64_t agent_id) {
  if (!al) return Q4KV_EINVAL;
  const auto it = al->agents.find(agent_id);
  if (it == al->agents.end()) return Q4KV_EINVAL;
  for (auto b = it->second.blocks.rbegin(); b != it->second.blocks.rend(); ++b) drop_block(al, *b);
  al->lru.erase(it->second.lru_pos);
  al->agents.erase(it);
  return Q4KV_OK;
}

int q4kv_allocator_table(const q4kv_allocator* al, int64_t agent_id, int32_t* table_row, int32_t max_blocks) {
  if (!al || !table_row || max_blocks <= 0) return Q4KV_EINVAL;
  const auto it = al->agents.find(agent_id);
  if (it == al->agents.end() || (int32_t)it->second.blocks.size() > max_blocks) return Q4KV_EINVAL;
  write_row(it->second, table_row, max_blocks);
  return Q4KV_OK;
}

int32_t q4kv_allocator_block_holders(const q4kv_allocator* al, int32_t block) {
  return !al || block < 0 || block >= al->n_blocks ? -1 : al->holders[block];
}

int q4kv_allocator_fork(q4kv_allocator* al, int64_t parent_id, int64_t child_id, int32_t n_tokens, int32_t* table_row,
                        int32_t max_blocks, int32_t* copy) {
  if (!al || n_tokens < 0 || !table_row || max_blocks <= 0 || !copy) return Q4KV_EINVAL;
  const auto parent = al->agents.find(parent_id);
  if (parent == al->agents.end() || al->agents.count(child_id)) return Q4KV_EINVAL;
  const int32_t whole = n_tokens / kBlockTokens, part = n_tokens % kBlockTokens, want = whole + (part ? 1 : 0);
  if (want > max_blocks || want > (int32_t)parent->second.blocks.size()) return Q4KV_EINVAL;
  if (part && al->free_list.empty()) return Q4KV_EWORKSPACE;
  try {                                                // everything that can fail comes before the first change
    q4kv_allocator::Agent child;
    child.blocks.reserve(want);
    child.blocks.assign(parent->second.blocks.begin(), parent->second.blocks.begin() + whole);
    std::list<int64_t> node(1, child_id);
    const auto it = al->agents.emplace(child_id, std::move(child)).first;
    touch(al, al->agents.find(parent_id)->second);
    al->lru.splice(al->lru.end(), node);
    it->second.lru_pos = std::prev(al->lru.end());
  } catch (...) {
    return Q4KV_EWORKSPACE;
  }
  q4kv_allocator::Agent& child = al->agents.find(child_id)->second;
  for (const int32_t b : child.blocks) ++al->holders[b];
  set_copy(copy, -1, -1, 0);
  if (part) {
    child.blocks.push_back(take_block(al));
    set_copy(copy, al->agents.find(parent_id)->second.blocks[whole], child.blocks.back(), part);
  }
  write_row(child, table_row, max_blocks);
  return Q4KV_OK;
}

int q4kv_allocator_truncate(q4kv_allocator* al, int64_t agent_id, int32_t n_tokens, int32_t* table_row, int32_t max_blocks,
                            int32_t* copy) {
  if (!al || n_tokens < 0 || !table_row || max_blocks <= 0 || !copy) return Q4KV_EINVAL;
  const auto it = al->agents.find(agent_id);
  if (it == al->agents.end()) return Q4KV_EINVAL;
  q4kv_allocator::Agent& ag = it->second;
  const int32_t part = n_tokens % kBlockTokens, keep = n_tokens / kBlockTokens + (part ? 1 : 0);
  if (keep > max_blocks || keep > (int32_t)ag.blocks.size()) return Q4KV_EINVAL;
  const bool shared = part && al->holders[ag.blocks[keep - 1]] > 1;      // what follows would be written into others' block
  if (shared && al->free_list.empty()) {
    const bool frees = std::any_of(ag.blocks.begin() + keep, ag.blocks.end(), [&](int32_t b) { return al->holders[b] == 1; });
    if (!frees) return Q4KV_EWORKSPACE;
  }
  while ((int32_t)ag.blocks.size() > keep) { drop_block(al, ag.blocks.back()); ag.blocks.pop_back(); }
  set_copy(copy, -1, -1, 0);
  if (shared) {
    const int32_t from = ag.blocks.back(), to = take_block(al);
    drop_block(al, from);
    ag.blocks.back() = to;
    set_copy(copy, from, to, part);
  }
  touch(al, ag);
  write_row(ag, table_row, max_blocks);
  return Q4KV_OK;
}

int q4kv_allocator_compact(q4kv_allocator* al, int32_t* copies, int32_t max_copies, int32_t* n_copies) {
  if (!al || !n_copies || max_copies < 0 || (max_copies > 0 && !copies)) return Q4KV_EINVAL;
  *n_copies = 0;
  try {
    std::vector<int32_t> to(al->n_blocks);
    for (int32_t b = 0; b < al->n_blocks; ++b) to[b] = b;
    int32_t low = 0, high = al->n_blocks - 1, n = 0;
    while (n < max_copies) {                           // the highest block in use into the lowest free one
      while (low < high && al->holders[low] > 0) ++low;
      while (high > low && al->holders[high] == 0) --high;
      if (low >= high) break;
      to[high] = low;
      set_copy(copies + 3 * (size_t)n++, high, low, kBlockTokens);
      ++low;
      --high;
    }
    *n_copies = n;
    for (int32_t b = 0; b < al->n_blocks; ++b)
      if (to[b] != b) { al->holders[to[b]] = al->holders[b]; al->holders[b] = 0; }
    for (auto& entry : al->agents)
      for (int32_t& b : entry.second.blocks) b = to[b];
    al->free_list.clear();
    for (int32_t b = al->n_blocks - 1; b >= 0; --b)
      if (al->holders[b] == 0) al->free_list.push_back(b);               // the lowest is handed out first
  } catch (...) {                                      // before any change: `to` is all that is allocated
    return Q4KV_EWORKSPACE;
  }
  return Q4KV_OK;
}

size_t q4kv_dense_bytes(const q4kv_spec* spec, int32_t n_agents, int32_t T) {
  if (!spec || n_agents < 0 || T < 0 || q4kv_pool_bytes(spec, 1) == 0) return 0;
  return dense_need(spec, n_agents, T);
}

int q4kv_merge_dense(const q4kv_spec* spec, void* pool, int32_t n_blocks, int32_t layer, const q4kv_batch* batch,
                     const int32_t* kv_lens, int32_t T, const void* dense, size_t dense_bytes, int32_t* status_flags,
                     void* stream) {
  return dense_call(spec, pool, n_blocks, layer, batch, kv_lens, T, const_cast<void*>(dense), dense_bytes, true, status_flags,
                    stream);
}

int q4kv_extract_dense(const q4kv_spec* spec, const void* pool, int32_t n_blocks, int32_t layer, const q4kv_batch* batch,
                       const int32_t* kv_lens, int32_t T, void* dense, size_t dense_bytes, int32_t* status_flags,
                       void* stream) {
  return dense_call(spec, const_cast<void*>(pool), n_blocks, layer, batch, kv_lens, T, dense, dense_bytes, false, status_flags,
                    stream);
}

}  // extern "C"
