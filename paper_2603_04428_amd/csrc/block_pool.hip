// Host-side block pool (Sec. 3.1 "Block Pool with Per-Agent Isolation"): which 256-token block of the device pools
// belongs to which agent, in which order, and which agent has been idle longest.  Pure bookkeeping in host memory:
// no device call, no kernel.  The device side of the same component is the block table the attention kernels read
// (one row per agent, written from q4kv_block_pool_table_row) and the block images of persist.hip (an evicted
// agent's blocks leave through q4kv_export_blocks and come back, into whatever blocks are free then, through
// q4kv_import_blocks).
//
// Isolation is structural: a block id is either on the free list or in an agent's list, and in several only where
// q4kv_block_pool_fork put it there: blocks that are full of tokens all of those agents have, so that no append
// writes into them.  Every entry point keeps that invariant and none hands out a block twice.  All entry points lock
// one mutex per pool.
#include <cstdint>
#include <functional>
#include <mutex>
#include <new>
#include <queue>
#include <unordered_map>
#include <utility>
#include <vector>

#include "../../include/q4kv.h"

struct q4kv_block_pool {
    struct Agent {
        std::vector<int32_t> blocks; // token order: entry i holds tokens 256 i .. 256 i + 255
        uint64_t stamp = 0;          // larger = used more recently
        bool pinned = false;         // part of a running batch: never a victim
    };
    std::mutex mu;
    std::vector<int64_t> owner;                                                     // per block: agent id (the smallest that lists it), or -1 when free
    std::vector<int32_t> refs;                                                      // per block: agents that list it
    std::vector<uint8_t> is_free;
    std::priority_queue<int32_t, std::vector<int32_t>, std::greater<int32_t>> free_ids; // lowest id first
    std::unordered_map<int64_t, Agent> agents;
    uint64_t clock = 0;
    int32_t free_count = 0;

    int32_t take(int64_t agent_id) // the lowest free block; there is one
    {
        const int32_t id = free_ids.top();
        free_ids.pop();
        is_free[(size_t)id] = 0;
        owner[(size_t)id] = agent_id;
        refs[(size_t)id] = 1;
        --free_count;
        return id;
    }
    // One agent fewer lists the block (its list no longer holds it); 1 when that freed it.  settle() follows the last one.
    int32_t drop(int32_t id, int64_t agent_id)
    {
        if (--refs[(size_t)id] > 0) {
            if (owner[(size_t)id] == agent_id) {
                owner[(size_t)id] = INT64_MAX;
                unsettled = true;
            }
            return 0;
        }
        owner[(size_t)id] = -1;
        is_free[(size_t)id] = 1;
        free_ids.push(id);
        ++free_count;
        return 1;
    }
    // The smallest lister of every block whose own has left it: one pass over all lists, however many blocks these are.
    void settle()
    {
        if (!unsettled) return;
        unsettled = false;
        for (const auto &kv : agents)
            for (int32_t id : kv.second.blocks)
                if (kv.first < owner[(size_t)id]) owner[(size_t)id] = kv.first;
    }
    bool unsettled = false;
};

namespace {
constexpr int64_t kBlock = 256;
}

extern "C" {

q4kv_block_pool *q4kv_block_pool_create(int32_t num_blocks)
{
    if (num_blocks <= 0) return nullptr;
    q4kv_block_pool *p = new (std::nothrow) q4kv_block_pool;
    if (!p) return nullptr;
    try {
        p->owner.assign((size_t)num_blocks, -1);
        p->refs.assign((size_t)num_blocks, 0);
        p->is_free.assign((size_t)num_blocks, 1);
        for (int32_t i = 0; i < num_blocks; ++i) p->free_ids.push(i);
    } catch (...) {
        delete p;
        return nullptr;
    }
    p->free_count = num_blocks;
    return p;
}

void q4kv_block_pool_destroy(q4kv_block_pool *pool) { delete pool; }

int32_t q4kv_block_pool_reserve(q4kv_block_pool *pool, int64_t agent_id, int64_t tokens)
{
    if (!pool || agent_id < 0 || tokens < 0) return Q4KV_EINVAL;
    const int64_t need64 = (tokens + kBlock - 1) / kBlock;
    std::lock_guard<std::mutex> lock(pool->mu);
    if (need64 > (int64_t)pool->owner.size()) return Q4KV_ENOSPACE;
    const int32_t need = (int32_t)need64;
    auto it = pool->agents.find(agent_id);
    const int32_t have = it == pool->agents.end() ? 0 : (int32_t)it->second.blocks.size();
    if (need - have > pool->free_count) return Q4KV_ENOSPACE; // nothing has changed
    try {
        q4kv_block_pool::Agent &a = pool->agents[agent_id];
        a.blocks.reserve((size_t)(need > have ? need : have));
        for (int32_t i = have; i < need; ++i) a.blocks.push_back(pool->take(agent_id));
        a.stamp = ++pool->clock;
        return (int32_t)a.blocks.size();
    } catch (...) {
        return Q4KV_ENOSPACE;
    }
}

int32_t q4kv_block_pool_release(q4kv_block_pool *pool, int64_t agent_id)
{
    if (!pool) return Q4KV_EINVAL;
    std::lock_guard<std::mutex> lock(pool->mu);
    auto it = pool->agents.find(agent_id);
    if (it == pool->agents.end()) return Q4KV_EINVAL;
    try {
        const std::vector<int32_t> blocks = std::move(it->second.blocks);
        pool->agents.erase(it);
        int32_t n = 0;
        for (int32_t id : blocks) n += pool->drop(id, agent_id);
        pool->settle();
        return n;
    } catch (...) { // the free list had no room to grow: it never holds more than it did at the start
        return Q4KV_ENOSPACE;
    }
}

int32_t q4kv_block_pool_blocks(q4kv_block_pool *pool, int64_t agent_id, int32_t *ids, int32_t cap)
{
    if (!pool || cap < 0 || (cap > 0 && !ids)) return Q4KV_EINVAL;
    std::lock_guard<std::mutex> lock(pool->mu);
    auto it = pool->agents.find(agent_id);
    if (it == pool->agents.end()) return Q4KV_EINVAL;
    const int32_t n = (int32_t)it->second.blocks.size();
    for (int32_t i = 0; i < n && i < cap; ++i) ids[i] = it->second.blocks[(size_t)i];
    return n;
}

int32_t q4kv_block_pool_table_row(q4kv_block_pool *pool, int64_t agent_id, int32_t *row, int32_t max_blocks, int32_t fill)
{
    if (!pool || !row || max_blocks <= 0) return Q4KV_EINVAL;
    std::lock_guard<std::mutex> lock(pool->mu);
    auto it = pool->agents.find(agent_id);
    if (it == pool->agents.end()) return Q4KV_EINVAL;
    const int32_t n = (int32_t)it->second.blocks.size();
    if (n > max_blocks) return Q4KV_ERANGE;
    for (int32_t i = 0; i < max_blocks; ++i) row[i] = i < n ? it->second.blocks[(size_t)i] : fill;
    return n;
}

int32_t q4kv_block_pool_touch(q4kv_block_pool *pool, int64_t agent_id)
{
    if (!pool) return Q4KV_EINVAL;
    std::lock_guard<std::mutex> lock(pool->mu);
    auto it = pool->agents.find(agent_id);
    if (it == pool->agents.end()) return Q4KV_EINVAL;
    it->second.stamp = ++pool->clock;
    return Q4KV_OK;
}

int32_t q4kv_block_pool_pin(q4kv_block_pool *pool, int64_t agent_id, int32_t pinned)
{
    if (!pool) return Q4KV_EINVAL;
    std::lock_guard<std::mutex> lock(pool->mu);
    auto it = pool->agents.find(agent_id);
    if (it == pool->agents.end()) return Q4KV_EINVAL;
    it->second.pinned = pinned != 0;
    return Q4KV_OK;
}

int64_t q4kv_block_pool_lru_victim(q4kv_block_pool *pool)
{
    if (!pool) return -1;
    std::lock_guard<std::mutex> lock(pool->mu);
    int64_t victim = -1;
    uint64_t oldest = 0;
    for (const auto &kv : pool->agents) {
        const q4kv_block_pool::Agent &a = kv.second;
        if (a.pinned || a.blocks.empty()) continue;
        if (victim < 0 || a.stamp < oldest) {
            victim = kv.first;
            oldest = a.stamp;
        }
    }
    return victim;
}

int32_t q4kv_block_pool_free_blocks(q4kv_block_pool *pool)
{
    if (!pool) return Q4KV_EINVAL;
    std::lock_guard<std::mutex> lock(pool->mu);
    return pool->free_count;
}

int64_t q4kv_block_pool_owner(q4kv_block_pool *pool, int32_t block_id)
{
    if (!pool) return -1;
    std::lock_guard<std::mutex> lock(pool->mu);
    if (block_id < 0 || (size_t)block_id >= pool->owner.size()) return -1;
    return pool->owner[(size_t)block_id];
}

int32_t q4kv_block_pool_fork(q4kv_block_pool *pool, int64_t parent_id, int64_t child_id, int64_t tokens, int32_t *copy_from,
                             int32_t *copy_to)
{
    if (!pool || child_id < 0 || parent_id == child_id || tokens < 0 || !copy_from || !copy_to) return Q4KV_EINVAL;
    std::lock_guard<std::mutex> lock(pool->mu);
    auto it = pool->agents.find(parent_id);
    if (it == pool->agents.end() || pool->agents.count(child_id)) return Q4KV_EINVAL;
    if (tokens > (int64_t)it->second.blocks.size() * kBlock) return Q4KV_ERANGE;
    const size_t full = (size_t)(tokens / kBlock);
    const bool partial = tokens % kBlock != 0;
    if (partial && pool->free_count < 1) return Q4KV_ENOSPACE;
    try {
        std::vector<int32_t> blocks(it->second.blocks.begin(), it->second.blocks.begin() + (ptrdiff_t)full);
        const int32_t last = partial ? it->second.blocks[full] : -1;
        blocks.reserve(full + 1);
        q4kv_block_pool::Agent &child = pool->agents[child_id]; // the last step that can fail
        for (int32_t id : blocks) {
            ++pool->refs[(size_t)id];
            if (child_id < pool->owner[(size_t)id]) pool->owner[(size_t)id] = child_id;
        }
        *copy_from = last;
        *copy_to = -1;
        if (partial) blocks.push_back(*copy_to = pool->take(child_id));
        child.blocks = std::move(blocks);
        pool->agents.find(parent_id)->second.stamp = ++pool->clock;
        child.stamp = ++pool->clock;
        return (int32_t)child.blocks.size();
    } catch (...) {
        return Q4KV_ENOSPACE;
    }
}

int32_t q4kv_block_pool_truncate(q4kv_block_pool *pool, int64_t agent_id, int64_t tokens, int32_t *copy_from, int32_t *copy_to)
{
    if (!pool || tokens < 0 || !copy_from || !copy_to) return Q4KV_EINVAL;
    std::lock_guard<std::mutex> lock(pool->mu);
    auto it = pool->agents.find(agent_id);
    if (it == pool->agents.end()) return Q4KV_EINVAL;
    std::vector<int32_t> &blocks = it->second.blocks;
    if (tokens > (int64_t)blocks.size() * kBlock) return Q4KV_ERANGE;
    const size_t keep = (size_t)((tokens + kBlock - 1) / kBlock);
    // a block that stays with unused slots is the agent's own from here on: the next append writes into it
    const bool copy = tokens % kBlock != 0 && pool->refs[(size_t)blocks[keep - 1]] > 1;
    if (copy) {
        int32_t freed = 0;
        for (size_t i = keep; i < blocks.size(); ++i) freed += pool->refs[(size_t)blocks[i]] == 1;
        if (pool->free_count + freed < 1) return Q4KV_ENOSPACE;
    }
    try {
        while (blocks.size() > keep) {
            const int32_t id = blocks.back();
            blocks.pop_back();
            pool->drop(id, agent_id);
        }
        *copy_from = *copy_to = -1;
        if (copy) {
            *copy_from = blocks.back();
            blocks.back() = *copy_to = pool->take(agent_id);
            pool->drop(*copy_from, agent_id);
        }
        pool->settle();
        it->second.stamp = ++pool->clock;
        return (int32_t)blocks.size();
    } catch (...) {
        return Q4KV_ENOSPACE;
    }
}

int32_t q4kv_block_pool_compact(q4kv_block_pool *pool, int32_t *copy_from, int32_t *copy_to, int32_t cap)
{
    if (!pool || cap < 0 || (cap > 0 && (!copy_from || !copy_to))) return Q4KV_EINVAL;
    std::lock_guard<std::mutex> lock(pool->mu);
    try {
        const int32_t blocks = (int32_t)pool->owner.size();
        std::vector<uint8_t> stays((size_t)blocks, 0); // listed by an agent of a running batch
        for (const auto &kv : pool->agents)
            if (kv.second.pinned)
                for (int32_t id : kv.second.blocks) stays[(size_t)id] = 1;
        std::vector<int32_t> new_id((size_t)blocks, -1);
        std::vector<std::pair<int32_t, int32_t>> moves;
        for (int32_t to = 0, from = blocks - 1;; ++to, --from) { // lowest free block, highest used one that may move
            while (to < from && !pool->is_free[(size_t)to]) ++to;
            while (to < from && (pool->is_free[(size_t)from] || stays[(size_t)from])) --from;
            if (to >= from) break;
            moves.emplace_back(from, to);
            new_id[(size_t)from] = to;
        }
        if (cap == 0) return (int32_t)moves.size();
        if ((int32_t)moves.size() > cap) return Q4KV_ERANGE;
        std::vector<int32_t> free_now;
        free_now.reserve((size_t)blocks);
        std::vector<uint8_t> is_free = pool->is_free;
        for (const auto &m : moves) {
            is_free[(size_t)m.first] = 1;
            is_free[(size_t)m.second] = 0;
        }
        for (int32_t i = 0; i < blocks; ++i)
            if (is_free[(size_t)i]) free_now.push_back(i);
        decltype(pool->free_ids) heap(std::greater<int32_t>(), std::move(free_now)); // the last step that can fail
        pool->free_ids.swap(heap);
        pool->is_free.swap(is_free);
        for (size_t i = 0; i < moves.size(); ++i) {
            const size_t from = (size_t)moves[i].first, to = (size_t)moves[i].second;
            copy_from[i] = moves[i].first;
            copy_to[i] = moves[i].second;
            pool->owner[to] = pool->owner[from];
            pool->refs[to] = pool->refs[from];
            pool->owner[from] = -1;
            pool->refs[from] = 0;
        }
        for (auto &kv : pool->agents)
            for (int32_t &id : kv.second.blocks)
                if (new_id[(size_t)id] >= 0) id = new_id[(size_t)id];
        return (int32_t)moves.size();
    } catch (...) {
        return Q4KV_ENOSPACE;
    }
}

int32_t q4kv_block_pool_shares(q4kv_block_pool *pool, int32_t block_id)
{
    if (!pool) return Q4KV_EINVAL;
    std::lock_guard<std::mutex> lock(pool->mu);
    if (block_id < 0 || (size_t)block_id >= pool->refs.size()) return Q4KV_EINVAL;
    return pool->refs[(size_t)block_id];
}

} // extern "C"
