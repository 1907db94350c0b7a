// batch.hip -- a worker's batch: prefix groups, block tables and slot maps, cache writes.
#include <hip/hip_runtime.h>

#include "rk_internal.h"

namespace rk {

constexpr int kBatchMax = RK_MAX_BATCH;
constexpr int kBatchThreads = 1024;
constexpr int kPer = kBatchMax / kBatchThreads;      // requests per thread
constexpr int kMasks = kBatchMax / 64;

// Inclusive sum over the workgroup's threads (kBatchThreads of them); tmp: 16 words.
__device__ __forceinline__ int64_t group_incl_sum(int64_t v, int64_t* tmp)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const int64_t o = __shfl_up(v, d);
        if (lane >= d) v += o;
    }
    __syncthreads();                       // tmp's last readers
    if (lane == 63) tmp[wave] = v;
    __syncthreads();
    int64_t before = 0;
    for (int w = 0; w < wave; ++w) before += tmp[w];
    return v + before;
}

// --------------------------------------------------------------- prefix groups
//
// One workgroup: a batch is small (4,096 requests at most) and its keys fit an
// LDS hash table, so grouping is a matter of latency, not of bandwidth.  Each
// request's key (its hash at block min_blocks - 1) is entered with the lowest
// request number that has it; the requests that are their key's lowest number
// the groups, by a population count over 64-request masks; a counting sort by
// group number, 6 bits a pass, gives the stable order.  32 requests: 10 us, 4,096 of 256 groups: 18.8 us and
// 5.3 us for their common blocks; some ten waits for loads, LDS and the other wavefronts one after the other.
constexpr int kGroupSlots = 2 * kBatchMax;
// Batches up to this are done in one launch, their common blocks by this workgroup, 64 requests at a time: calls of 64 and 128
// requests 11.4 and 12.4 us (14.0 and 13.7 by two launches), of 192 and 512 14.1 and 20.9 us (13.8 and 14.8).
constexpr int kFewGroups = 128;

struct GroupLds {
    uint64_t key[kGroupSlots];
    int32_t first[kGroupSlots];
    uint64_t lead[kMasks];
    int32_t lead_before[kMasks];
    int64_t tmp[16];
    int32_t off[kBatchMax + 1];              // group sizes, then offsets
};

// A pass of the stable counting sort: bits [shift, shift + 6) of the key, thread-order elements el[]
// (wave w, round u, lane l holds element 64 (kPer w + u) + l).  hist: 64 * 16 words.
__device__ __forceinline__ void sort_pass(const int32_t* el, const int32_t* key, int32_t B, int shift, int32_t* hist,
                                          int64_t* tmp, int32_t* out)
{
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    hist[tid] = 0;                           // hist[digit * 16 + wave]
    __syncthreads();
    int32_t rank[kPer], digit[kPer];
#pragma unroll
    for (int u = 0; u < kPer; ++u) {
        const bool in = 64 * (kPer * wave + u) + lane < B;
        digit[u] = (key[u] >> shift) & 63;
        uint64_t same = __ballot(in);
#pragma unroll
        for (int b = 0; b < 6; ++b) {
            const uint64_t m = __ballot((digit[u] >> b) & 1);
            same &= (digit[u] >> b) & 1 ? m : ~m;
        }
        const uint64_t below = same & ((1ull << lane) - 1);
        int32_t base = 0;
        if (in) base = hist[digit[u] * 16 + wave];
        rank[u] = base + __popcll(below);
        // (a wavefront's LDS accesses are done in order)
        if (in && (same >> lane) == 1ull) hist[digit[u] * 16 + wave] = rank[u] + 1;
        __builtin_amdgcn_wave_barrier();
    }
    __syncthreads();
    const int64_t mine = hist[tid], incl = group_incl_sum(mine, tmp);
    __syncthreads();
    hist[tid] = (int32_t)(incl - mine);
    __syncthreads();
#pragma unroll
    for (int u = 0; u < kPer; ++u)
        if (64 * (kPer * wave + u) + lane < B) out[hist[digit[u] * 16 + wave] + rank[u]] = el[u];
    __syncthreads();
}

// Leading blocks that request i's chain has in common with request f's, by a team of Team lanes; 0 for teams with
// pair = false, which take part all the same.  Chained hashes agree up to the first block that
// differs and nowhere after it, so each round tests Team positions and keeps a Team-th of the interval.  A hash of 0 is one that
// is missing (from there on to the chain's end) and agrees with none.
template <int Team>
__device__ __forceinline__ int32_t common_blocks(const uint64_t* __restrict__ chains, const int64_t* __restrict__ chain_off,
                                                 int32_t i, int32_t f, bool pair)
{
    const int sub = threadIdx.x & (Team - 1), shift = threadIdx.x & 63 & ~(Team - 1);
    int64_t a = 0, b = 0;
    int32_t have = 0, most = 0;              // `have` blocks agree; at most `most` do
    if (pair) {
        a = chain_off[i];
        b = chain_off[f];
        const int64_t la = chain_off[i + 1] - a, lb = chain_off[f + 1] - b, l = la < lb ? la : lb;
        most = l > 0 ? (int32_t)(l < 0x7ffffffe ? l : 0x7ffffffe) : 0;
    }
    while (__any(have < most)) {
        const int64_t w = most - have;
        const int32_t x = have + (int32_t)((int64_t)(sub + 1) * w / Team);     // a count of blocks, <= most
        bool same = false;
        if (have < most) {
            same = x == have;
            if (!same) {
                const uint64_t h = chains[a + x - 1];
                same = h != 0ull && h == chains[b + x - 1];
            }
        }
        const uint32_t m = (uint32_t)(__ballot(same) >> shift) & ((1u << Team) - 1);
        if (have < most) {
            const int k = __ffs(~m) - 1;     // the first k samples agree (bit Team of m is 0)
            const int32_t agreed = have + (int32_t)((int64_t)k * w / Team);
            if (k < Team) most = have + (int32_t)((int64_t)(k + 1) * w / Team) - 1;
            have = agreed;
        }
    }
    return have;
}

__global__ __launch_bounds__(kBatchThreads) void group_kernel(int32_t B, const uint64_t* __restrict__ chains,
                                                              const int64_t* __restrict__ chain_off, int32_t min_blocks,
                                                              int32_t* __restrict__ order, int64_t* __restrict__ group_off,
                                                              int32_t* __restrict__ shared, int32_t* __restrict__ n_groups,
                                                              int32_t* status)
{
    __shared__ GroupLds s;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    int32_t slot[kPer], first[kPer];
    uint64_t key[kPer];
    int64_t c0[kPer], c1[kPer];
#pragma unroll
    for (int u = 0; u < kPer; ++u) {
        const int32_t i = 64 * (kPer * wave + u) + lane;
        c0[u] = c1[u] = 0;
        if (i < B) {
            c0[u] = chain_off[i];
            c1[u] = chain_off[i + 1];
        }
    }
    for (int x = tid; x < kGroupSlots; x += kBatchThreads) {       // (while the offsets come)
        s.key[x] = 0ull;
        s.first[x] = 0x7fffffff;
    }
    for (int x = tid; x <= kBatchMax; x += kBatchThreads) s.off[x] = 0;
#pragma unroll
    for (int u = 0; u < kPer; ++u) {
        const int32_t i = 64 * (kPer * wave + u) + lane;
        key[u] = 0ull;
        if (i < B) {
            if (c1[u] < c0[u] || c0[u] < 0) atomicOr(status, RK_DEV_BAD_OFFSETS);
            else if (c1[u] - c0[u] >= min_blocks) {
                key[u] = chains[c0[u] + min_blocks - 1];
                if (key[u] == 0ull) atomicOr(status, RK_DEV_ZERO_KEY);
            }
        }
    }
    __syncthreads();
#pragma unroll
    for (int u = 0; u < kPer; ++u) {
        const int32_t i = 64 * (kPer * wave + u) + lane;
        slot[u] = -1;
        if (key[u] == 0ull) continue;
        uint32_t p = (uint32_t)key[u] & (kGroupSlots - 1);
        for (;;) {                           // the table is at most half full
            const unsigned long long prev = atomicCAS((unsigned long long*)&s.key[p], 0ull, (unsigned long long)key[u]);
            if (prev == 0ull || prev == key[u]) break;
            p = (p + 1) & (kGroupSlots - 1);
        }
        slot[u] = (int32_t)p;
        atomicMin(&s.first[p], i);
    }
    __syncthreads();
#pragma unroll
    for (int u = 0; u < kPer; ++u) {
        const int32_t i = 64 * (kPer * wave + u) + lane;
        first[u] = slot[u] >= 0 ? s.first[slot[u]] : i;
        const uint64_t m = __ballot(i < B && first[u] == i);
        if (lane == 0) s.lead[kPer * wave + u] = m;
    }
    __syncthreads();
    {
        const int64_t c = tid < kMasks ? __popcll(s.lead[tid]) : 0, incl = group_incl_sum(c, s.tmp);
        if (tid < kMasks) s.lead_before[tid] = (int32_t)(incl - c);
    }
    __syncthreads();
    const int32_t G = s.lead_before[kMasks - 1] + __popcll(s.lead[kMasks - 1]);
    int32_t group[kPer];
#pragma unroll
    for (int u = 0; u < kPer; ++u) {
        const int32_t i = 64 * (kPer * wave + u) + lane, f = first[u];
        group[u] = 0;
        if (i >= B) continue;
        group[u] = s.lead_before[f >> 6] + __popcll(s.lead[f >> 6] & ((1ull << (f & 63)) - 1));
        atomicAdd(&s.off[group[u]], 1);
    }
    __syncthreads();
    {
        int32_t n[kPer];
        int64_t sum = 0;
#pragma unroll
        for (int u = 0; u < kPer; ++u) sum += n[u] = s.off[kPer * tid + u];
        int64_t at = group_incl_sum(sum, s.tmp) - sum;
#pragma unroll
        for (int u = 0; u < kPer; ++u) {
            const int32_t g = kPer * tid + u;
            if (g < B) {
                group_off[g] = at;
                const int32_t least = n[u] > 1 ? 0x7fffffff : 0;
                if (B <= kFewGroups) s.off[g] = least;       // (a thread's own places are read)
                else shared[g] = least;                      // the next kernel's minimum
            }
            at += n[u];
        }
    }
    if (tid == 0) {
        group_off[B] = B;
        *n_groups = G;
    }
    if (B <= kFewGroups) {
        // the groups' common blocks, by the teams of this workgroup
        int32_t* first_of = reinterpret_cast<int32_t*>(s.key) + 2 * kBatchThreads;
        int32_t* group_of = first_of + kFewGroups;
        __syncthreads();
#pragma unroll
        for (int u = 0; u < kPer; ++u) {
            const int32_t i = 64 * (kPer * wave + u) + lane;
            if (i < B) {
                first_of[i] = first[u];
                group_of[i] = group[u];
            }
        }
        __syncthreads();
        for (int32_t i0 = 0; i0 < B; i0 += kBatchThreads / 16) {
            const int32_t i = i0 + (tid >> 4), f = i < B ? first_of[i] : i;
            const int32_t n = common_blocks<16>(chains, chain_off, i, f, f != i);
            if (f != i && (tid & 15) == 0) atomicMin(&s.off[group_of[i]], n);
        }
        __syncthreads();
        if (tid < B) shared[tid] = s.off[tid];
    }
    // the order; the hash table's memory is free by now
    int32_t* hist = reinterpret_cast<int32_t*>(s.key);
    int32_t* sorted = s.first;
    int32_t el[kPer];
#pragma unroll
    for (int u = 0; u < kPer; ++u) el[u] = 64 * (kPer * wave + u) + lane;
    __syncthreads();
    sort_pass(el, group, B, 0, hist, s.tmp, G <= 64 ? order : sorted);
    if (G > 64) {
        int32_t* number = reinterpret_cast<int32_t*>(s.key) + kBatchThreads;         // request -> group
#pragma unroll
        for (int u = 0; u < kPer; ++u)
            if (el[u] < B) number[el[u]] = group[u];
        __syncthreads();
#pragma unroll
        for (int u = 0; u < kPer; ++u) {
            const int32_t x = 64 * (kPer * wave + u) + lane;
            el[u] = x < B ? sorted[x] : 0;
            group[u] = x < B ? number[el[u]] : 0;
        }
        __syncthreads();
        sort_pass(el, group, B, 6, hist, s.tmp, order);
    }
}

// shared_g: the least number of leading blocks that a member has in common with its group's first request; a team of
// 4 lanes per place in the order.  A workgroup's 64 places are those of at most 64 groups, one after the other, so it
// makes one global minimum a group: a popular group's members would wait for each other there (one a member:
// 20 us for 4,096 requests of 256 groups).
__global__ __launch_bounds__(256) void common_kernel(int32_t B, const uint64_t* __restrict__ chains,
                                                     const int64_t* __restrict__ chain_off,
                                                     const int32_t* __restrict__ order,
                                                     const int64_t* __restrict__ group_off, int32_t* __restrict__ shared)
{
    __shared__ int32_t s_least[64], s_group;
    const int tid = threadIdx.x, lane = tid & 63;
    if (tid < 64) s_least[tid] = 0x7fffffff;
    // the group that holds the wavefront's first place: the last g with group_off[g] <= r0
    const int32_t r0 = (int32_t)(blockIdx.x * 64 + (tid >> 6) * 16), r = r0 + (lane >> 2);
    int32_t lo = 0, hi = B;                  // group_off[lo] <= r0 < group_off[hi], if r0 is a place
    while (r0 < B && hi - lo > 1) {
        const int32_t w = hi - lo, x = lo + (int32_t)((int64_t)(lane + 1) * w / 65);
        const int k = __popcll(__ballot(group_off[x] <= r0));      // the first k samples are <= r0
        if (k < 64) hi = lo + (int32_t)((int64_t)(k + 1) * w / 65);
        if (k > 0) lo = lo + (int32_t)((int64_t)k * w / 65);
    }
    if (tid == 0) s_group = lo;
    // the 16 places' groups are among the next 16
    const int32_t next = lo + 1 + (lane & 15);
    const int64_t start = group_off[next < B ? next : B];
    int32_t g = lo;
#pragma unroll
    for (int u = 0; u < 16; ++u)
        if (__shfl(start, u) <= r && r < B) g = lo + 1 + u;
    const bool in = r < B;
    const int32_t f = in ? order[group_off[g]] : 0, i = in ? order[r] : 0;
    const bool pair = in && f != i;
    const int32_t n = common_blocks<4>(chains, chain_off, i, f, pair);
    __syncthreads();
    if (pair && (lane & 3) == 0) atomicMin(&s_least[(g - s_group) & 63], n);
    __syncthreads();
    if (tid < 64 && s_least[tid] != 0x7fffffff) atomicMin(&shared[s_group + tid], s_least[tid]);
}

// --------------------------------------------------------------- block tables
//
// Every workgroup sums the whole batch's blocks and tokens for itself (4,096
// requests at most, four a thread) and then fills its share of the table
// entries and of the slots, so a step takes one launch.  An entry that is lent
// by the group's first row is computed as that row's entry is, never read from
// what another workgroup writes.  64 decoding requests 6.4 us, 9.3 MB of tables
// and slots of a million tokens 14.7 us (0.63 TB/s): the sums take 5 us of it,
// the search for each entry's row, 12 steps in LDS, most of the rest.
struct TableLds {
    int32_t goff[kBatchMax + 1];
    int32_t kv[kBatchMax], have[kBatchMax], lead[kBatchMax], first[kBatchMax];
    uint32_t base[kBatchMax];                // first of the request's blocks in the free list
    int64_t tok[kBatchMax + 1];              // tokens before the request's
    uint32_t fill[kBatchMax + 1];            // entries to write before the request's
    int64_t tmp[48];
    int32_t bad;
};

// the last x in [0, n) with off[x] <= v (off[0] <= v)
template <class T, class V>
__device__ __forceinline__ int32_t last_le(const T* off, int32_t n, V v)
{
    int32_t lo = 0, hi = n;
    while (hi - lo > 1) {
        const int32_t mid = (lo + hi) >> 1;
        if (off[mid] <= (T)v) lo = mid;
        else hi = mid;
    }
    return lo;
}

__global__ __launch_bounds__(kBatchThreads) void tables_kernel(
    int32_t B, const int32_t* __restrict__ kv_len, const int32_t* __restrict__ new_len, const int32_t* __restrict__ have,
    const int64_t* __restrict__ group_off, const int32_t* __restrict__ shared, const int32_t* __restrict__ free_blocks,
    int32_t n_free, int32_t* tables, int32_t stride, int64_t* __restrict__ slots, int64_t n_slots,
    int64_t* __restrict__ q_off, int32_t* __restrict__ taken, int32_t* status)
{
    __shared__ TableLds s;
    const int tid = threadIdx.x;
    const bool tell = blockIdx.x == 0;       // one workgroup reports
    const int32_t per = (B + kBatchThreads - 1) / kBatchThreads;             // requests of a thread, side by side
    if (tid == 0) s.bad = 0;
    __syncthreads();
    int32_t kv[kPer], nw[kPer], hv[kPer];
#pragma unroll
    for (int u = 0; u < kPer; ++u) {
        const int32_t i = per * tid + u;
        kv[u] = nw[u] = hv[u] = 0;
        if (u >= per || i >= B) continue;
        kv[u] = kv_len[i];
        nw[u] = new_len[i];
        hv[u] = have[i];
        const bool large = (int64_t)kv[u] > (int64_t)stride * RK_BLOCK_TOKENS;
        if (nw[u] < 0 || nw[u] > kv[u] || hv[u] < 0 || hv[u] > stride || large) {
            if (tell) atomicOr(status, large ? RK_DEV_TOO_LARGE : RK_DEV_BAD_OFFSETS);
            kv[u] = nw[u] = hv[u] = 0;
        }
        s.kv[i] = kv[u];
        s.have[i] = hv[u];
        if (group_off) {
            const int64_t a = group_off[i], b = group_off[i + 1];
            if (a > b || a < 0 || b > B || (i == 0 && a != 0) || (i == B - 1 && b != B)) s.bad = 1;
            s.goff[i] = (int32_t)a;
            if (i == B - 1) s.goff[B] = (int32_t)b;
        }
    }
    __syncthreads();
    const bool groups = group_off && !s.bad;
    if (tell && tid == 0 && s.bad) atomicOr(status, RK_DEV_BAD_OFFSETS);
    int64_t count[kPer], blocks = 0, tokens = 0, fills = 0;
#pragma unroll
    for (int u = 0; u < kPer; ++u) {
        const int32_t i = per * tid + u;
        count[u] = 0;
        if (u >= per || i >= B) continue;
        int32_t f = i, lead = 0;
        if (groups) {
            const int32_t g = last_le(s.goff, B, i);
            f = s.goff[g];
            if (f != i) {
                const int32_t sh = shared[g], most = s.kv[f] / RK_BLOCK_TOKENS;
                lead = sh < most ? sh : most;
                if (lead < 0) lead = 0;
            }
        }
        const int32_t need = (int32_t)(((int64_t)kv[u] + RK_BLOCK_TOKENS - 1) / RK_BLOCK_TOKENS);
        const int32_t start = hv[u] > lead ? hv[u] : lead;
        s.first[i] = f;
        s.lead[i] = lead;
        count[u] = need > start ? need - start : 0;
        blocks += count[u];
        tokens += nw[u];
        fills += need > hv[u] ? need - hv[u] : 0;
    }
    int64_t blocks_at = blocks, tokens_at = tokens, fills_at = fills;
    {
        const int lane = tid & 63, wave = tid >> 6;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const int64_t x = __shfl_up(blocks_at, d), y = __shfl_up(tokens_at, d), z = __shfl_up(fills_at, d);
            if (lane >= d) {
                blocks_at += x;
                tokens_at += y;
                fills_at += z;
            }
        }
        if (lane == 63) {
            s.tmp[wave] = blocks_at;
            s.tmp[16 + wave] = tokens_at;
            s.tmp[32 + wave] = fills_at;
        }
        __syncthreads();
        blocks_at -= blocks;
        tokens_at -= tokens;
        fills_at -= fills;
        for (int w = 0; w < wave; ++w) {
            blocks_at += s.tmp[w];
            tokens_at += s.tmp[16 + w];
            fills_at += s.tmp[32 + w];
        }
    }
#pragma unroll
    for (int u = 0; u < kPer; ++u) {
        const int32_t i = per * tid + u;
        if (u >= per || i >= B) continue;
        s.base[i] = blocks_at < 0x7fffffff ? (uint32_t)blocks_at : 0x7fffffffu;
        s.tok[i] = tokens_at;
        s.fill[i] = (uint32_t)fills_at;
        if (tell) q_off[i] = tokens_at;
        const int32_t need = (int32_t)(((int64_t)kv[u] + RK_BLOCK_TOKENS - 1) / RK_BLOCK_TOKENS);
        blocks_at += count[u];
        tokens_at += nw[u];
        fills_at += need > hv[u] ? need - hv[u] : 0;
        if (i == B - 1) {
            s.tok[B] = tokens_at;
            s.fill[B] = (uint32_t)fills_at;
            if (tell) {
                q_off[B] = tokens_at;
                *taken = (int32_t)(blocks_at < n_free ? blocks_at : n_free);
                if (blocks_at > n_free) atomicOr(status, RK_DEV_TABLE_FULL);
                if (tokens_at > n_slots) atomicOr(status, RK_DEV_SHORT_INPUT);
            }
        }
    }
    if (B == 0 && tell && tid == 0) {
        q_off[0] = 0;
        *taken = 0;
    }
    __syncthreads();
    auto own_entry = [&](int32_t i, int32_t p) -> int32_t {        // of a row that borrows nothing at p
        const int32_t h = s.have[i];
        if (p < h) return tables[(int64_t)i * stride + p];
        const int32_t start = s.lead[i] > h ? s.lead[i] : h;
        const int64_t x = (int64_t)s.base[i] + (p - start);
        return x < n_free ? free_blocks[x] : -1;
    };
    auto entry = [&](int32_t i, int32_t p) -> int32_t {
        return p >= s.have[i] && p < s.lead[i] ? own_entry(s.first[i], p) : own_entry(i, p);
    };
    const int64_t step = (int64_t)gridDim.x * kBatchThreads, at = (int64_t)blockIdx.x * kBatchThreads + tid;
    const int64_t n_fill = B ? s.fill[B] : 0, n_tok = B ? s.tok[B] : 0;
    for (int64_t x = at; x < n_fill; x += step) {
        const int32_t i = last_le(s.fill, B, x);
        const int32_t p = s.have[i] + (int32_t)(x - s.fill[i]);
        tables[(int64_t)i * stride + p] = entry(i, p);
    }
    for (int64_t t = at; t < n_slots; t += step) {
        int64_t slot = -1;
        if (t < n_tok) {
            const int32_t i = last_le(s.tok, B, t);
            const int32_t x = s.kv[i] - (int32_t)(s.tok[i + 1] - s.tok[i]) + (int32_t)(t - s.tok[i]);
            const int32_t p = x / RK_BLOCK_TOKENS;
            if (p < s.have[i] || p >= s.lead[i]) {
                const int32_t e = own_entry(i, p);
                if (e >= 0) slot = (int64_t)e * RK_BLOCK_TOKENS + x % RK_BLOCK_TOKENS;
            }
        }
        slots[t] = slot;
    }
}

// --------------------------------------------------------------- cache writes

// A thread per 16 bytes, side by side in a head, so that whole rows are read and written; blockIdx.y: keys or values.
// Bound by memory: 16,384 tokens of 8 heads of 128, 134 MB in 21.2 us (6.3 TB/s, as much of it as the caches hold; 27 us, 5.0 TB/s,
// when they hold other things), 64 tokens of 2 heads 2.8 us.
__global__ __launch_bounds__(256) void write_kernel(int64_t T, int32_t Hkv, int32_t D8, const uint16_t* __restrict__ k,
                                                    int64_t k_token, int64_t k_head, const uint16_t* __restrict__ v,
                                                    int64_t v_token, int64_t v_head, uint16_t* __restrict__ kc,
                                                    rk_cache_strides ks, uint16_t* __restrict__ vc, rk_cache_strides vs,
                                                    int32_t n_blocks, const int64_t* __restrict__ slots, int32_t* status)
{
    const bool values = blockIdx.y != 0;
    const uint16_t* __restrict__ src = values ? v : k;
    uint16_t* __restrict__ dst = values ? vc : kc;
    const int64_t s_token = values ? v_token : k_token, s_head = values ? v_head : k_head;
    const rk_cache_strides cs = values ? vs : ks;
    const uint32_t per = (uint32_t)Hkv * (uint32_t)D8;             // chunks of a token
    const int64_t n = T * per;
    for (int64_t x = (int64_t)blockIdx.x * 256 + threadIdx.x; x < n; x += (int64_t)gridDim.x * 256) {
        const int64_t t = x / per;
        const uint32_t r = (uint32_t)(x - t * per), h = r / (uint32_t)D8, c = r - h * (uint32_t)D8;
        const int64_t slot = slots[t];
        if (slot < 0) continue;
        const int64_t block = slot / RK_BLOCK_TOKENS, tok = slot % RK_BLOCK_TOKENS;
        if (block >= n_blocks) {
            if (r == 0) atomicOr(status, RK_DEV_BAD_BLOCK);
            continue;
        }
        const u32x4 val = *reinterpret_cast<const u32x4*>(src + t * s_token + h * s_head + 8 * c);
        *reinterpret_cast<u32x4*>(dst + block * cs.block + tok * cs.token + h * cs.head + 8 * c) = val;
    }
}

// Whether no two of an array's rows of D elements share one, as the strides of its dimensions tell: by size, each steps over
// all that the smaller ones span.
bool rows_apart(std::initializer_list<ArrayDim> dims, int32_t D)
{
    ArrayDim d[4];
    int n = 0;
    for (const ArrayDim& x : dims) {
        if (x.n == 0) return true;
        if (x.n == 1) continue;
        int at = n++;
        for (; at > 0 && d[at - 1].stride > x.stride; --at) d[at] = d[at - 1];
        d[at] = x;
    }
    __int128 span = D;
    for (int k = 0; k < n; ++k) {
        if (d[k].stride < span) return false;
        span += (__int128)d[k].stride * (d[k].n - 1);
    }
    return true;
}

}  // namespace rk

using namespace rk;

extern "C" {

int rk_prefix_groups(int32_t B, const uint64_t* chains, const int64_t* chain_off, int32_t min_blocks, int32_t* order,
                     int64_t* group_off, int32_t* shared, int32_t* n_groups, void* stream)
{
    if (B < 0) return fail(RK_EINVAL, "rk_prefix_groups: B < 0");
    if (B > kBatchMax) return fail(RK_EUNSUPPORTED, "rk_prefix_groups: B > %d", kBatchMax);
    if (min_blocks < 1) return fail(RK_EINVAL, "rk_prefix_groups: min_blocks < 1");
    if (!group_off || !n_groups || (B > 0 && (!chains || !chain_off || !order || !shared)))
        return fail(RK_EINVAL, "rk_prefix_groups: NULL array");
    int32_t* st = status_word();
    if (!st) return fail(RK_EHIP, "rk_prefix_groups: no status word");
    hipStream_t s = (hipStream_t)stream;
    hipLaunchKernelGGL(group_kernel, dim3(1), dim3(kBatchThreads), 0, s, B, chains, chain_off, min_blocks, order,
                       group_off, shared, n_groups, st);
    if (B > kFewGroups)
        hipLaunchKernelGGL(common_kernel, dim3((unsigned)((B + 63) / 64)), dim3(256), 0, s, B, chains, chain_off, order,
                           group_off, shared);
    return hip_check(hipGetLastError(), "rk_prefix_groups launch");
}

int rk_block_tables(int32_t B, const int32_t* kv_len, const int32_t* new_len, const int32_t* have,
                    const int64_t* group_off, const int32_t* shared, const int32_t* free_blocks, int32_t n_free,
                    int32_t* tables, int32_t stride, int64_t* slots, int64_t n_slots, int64_t* q_off, int32_t* taken,
                    void* stream)
{
    if (B < 0 || n_free < 0 || n_slots < 0 || stride < 0)
        return fail(RK_EINVAL, "rk_block_tables: a negative size");
    if (B > kBatchMax) return fail(RK_EUNSUPPORTED, "rk_block_tables: B > %d", kBatchMax);
    if (stride >= 1 << 20) return fail(RK_EUNSUPPORTED, "rk_block_tables: stride >= 2^20 blocks");
    if (!q_off || !taken || (B > 0 && (!kv_len || !new_len || !have)) || (B > 0 && stride > 0 && !tables) ||
        (n_free > 0 && !free_blocks) || (n_slots > 0 && !slots))
        return fail(RK_EINVAL, "rk_block_tables: NULL array");
    if (!group_off != !shared) return fail(RK_EINVAL, "rk_block_tables: group_off without shared, or the reverse");
    int32_t* st = status_word();
    if (!st) return fail(RK_EHIP, "rk_block_tables: no status word");
    int64_t blocks = (n_slots + 16 * (int64_t)B + 2 * kBatchThreads - 1) / (2 * kBatchThreads);
    if (blocks < 1) blocks = 1;
    if (blocks > 256) blocks = 256;
    hipLaunchKernelGGL(tables_kernel, dim3((unsigned)blocks), dim3(kBatchThreads), 0, (hipStream_t)stream, B, kv_len,
                       new_len, have, group_off, shared, free_blocks, n_free, tables, stride, slots, n_slots, q_off,
                       taken, st);
    return hip_check(hipGetLastError(), "rk_block_tables launch");
}

int rk_kv_write(int64_t T, int32_t Hkv, int32_t D, const void* k, int64_t k_token, int64_t k_head, const void* v,
                int64_t v_token, int64_t v_head, void* k_cache, rk_cache_strides ks, void* v_cache, rk_cache_strides vs,
                int32_t n_blocks, const int64_t* slots, void* stream)
{
    if (T < 0 || n_blocks < 0) return fail(RK_EINVAL, "rk_kv_write: a negative size");
    if (Hkv < 1 || Hkv > 1024) return fail(RK_EUNSUPPORTED, "rk_kv_write: Hkv outside 1..1024");
    if (D < 8 || D > 256 || D % 8) return fail(RK_EUNSUPPORTED, "rk_kv_write: D is no multiple of 8 in 8..256");
    const int64_t strides[] = {k_token, k_head, v_token, v_head, ks.block, ks.token, ks.head, vs.block, vs.token, vs.head};
    for (int64_t x : strides)
        if (x < 0 || x % 8) return fail(RK_EINVAL, "rk_kv_write: a stride is negative or no multiple of 8");
    for (const rk_cache_strides& c : {ks, vs})
        if (!rows_apart({{n_blocks, c.block}, {RK_BLOCK_TOKENS, c.token}, {Hkv, c.head}}, D))
            return fail(RK_EINVAL, "rk_kv_write: a cache's strides lay heads, tokens or blocks over each other");
    if (T == 0) return RK_OK;
    if (!k || !v || !slots || (n_blocks > 0 && (!k_cache || !v_cache)))
        return fail(RK_EINVAL, "rk_kv_write: NULL array");
    if (((uintptr_t)k | (uintptr_t)v | (uintptr_t)k_cache | (uintptr_t)v_cache) % 16)
        return fail(RK_EINVAL, "rk_kv_write: an array is not aligned to 16 bytes");
    int32_t* st = status_word();
    if (!st) return fail(RK_EHIP, "rk_kv_write: no status word");
    const int64_t chunks = T * Hkv * (D / 8);
    int64_t blocks = (chunks + 255) / 256;
    if (blocks > 16384) blocks = 16384;
    hipLaunchKernelGGL(write_kernel, dim3((unsigned)blocks, 2), dim3(256), 0, (hipStream_t)stream, T, Hkv, D / 8,
                       (const uint16_t*)k, k_token, k_head, (const uint16_t*)v, v_token, v_head, (uint16_t*)k_cache, ks,
                       (uint16_t*)v_cache, vs, n_blocks, slots, st);
    return hip_check(hipGetLastError(), "rk_kv_write launch");
}

}  // extern "C"
