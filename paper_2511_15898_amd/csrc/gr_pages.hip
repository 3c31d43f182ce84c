// Pages of the cache after lengths have changed: block tables, slot maps and the free list, in one launch and without the host.
#include <algorithm>

#include "gr_paths.h"

namespace gr {

namespace {

constexpr int kPageThreads = 1024, kPageWaves = kPageThreads / 64, kRun = 4;
constexpr double kMostTokens = 2147483648.0;

// Division by a fixed block size: a shift where it is a power of two.
struct BlockSize {
    unsigned size; int shift;
    __device__ __forceinline__ unsigned div(unsigned x) const { return shift >= 0 ? x >> shift : x / size; }
    __device__ __forceinline__ unsigned up(unsigned x) const { return div(x + size - 1); }
};

// The first i of [0, n) with sums[i + 1] > x, for x < sums[n].
__device__ __forceinline__ int owner_of(const int* sums, int n, int x) {
    int lo = 0, hi = n - 1;
    while (lo < hi) { const int mid = (lo + hi) >> 1; if (sums[mid + 1] > x) hi = mid; else lo = mid + 1; }
    return lo;
}

// Every workgroup adds up the needs of all requests by itself (at most GR_MAX_REQUESTS of them: 64 KB of lengths, from L2 but for the first) and then takes its share of
// the new table entries, the slots and the blocks that go back; the first workgroup writes what there is one of per request.  The new lengths and the free
// count go to arrays of their own, because other workgroups may still be reading the old ones.
// LDS, by request: exclusive sums of new tokens, new blocks and released blocks; the old length of one that grows, the new one of one that shrinks; OPEN: the block
// that a growing one has not filled, asked for while the sums are formed (of more requests than kOpenRequests LDS has no room for it; then it is read where it is needed).
// Bound: the launch and a chain of two reads, scan, search and stores; with many prompt tokens the stores of the slots.  64 requests, a token each 4.4 us; 4096 requests after a
// verification 13.1 us; a million slots of 512 prompts 8.7 us (1.0 TB/s).
constexpr int kOpenRequests = 4096, kPerThread = GR_MAX_REQUESTS / kPageThreads;
template <bool OPEN>
__global__ __launch_bounds__(kPageThreads) void pages_kernel(const PageParams pp, const BlockSize bs) {
    extern __shared__ int lds[];
    const int R = pp.R;
    int* const starts = lds; int* const fresh = lds + R + 1; int* const freed = lds + 2 * (R + 1); int* const from = lds + 3 * (R + 1); int* const open = lds + 4 * (R + 1);
    __shared__ double wave_tokens[kPageWaves];
    __shared__ int wave_fresh[kPageWaves], wave_freed[kPageWaves];
    __shared__ unsigned got_tokens, got_fresh;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const bool first = blockIdx.x == 0;
    const int per = (R + kPageThreads - 1) / kPageThreads, r0 = min(R, tid * per), mine = min(R, r0 + per) - r0;
    const long long most = static_cast<long long>(pp.width) * pp.block;
    const int count = max(0, min(*pp.free_count, pp.pool));

    // this thread's requests: all of their lengths are on their way at once, then all of their open blocks
    int old[kPerThread], now[kPerThread], part[kPerThread];
#pragma unroll
    for (int i = 0; i < kPerThread; ++i) if (i < mine) { old[i] = pp.lengths[r0 + i]; now[i] = pp.new_lengths[r0 + i]; }
    if (tid == 0) { got_tokens = ~0u; got_fresh = ~0u; }
    double tokens = 0.0;                                  // up to 2^44; blocks are at most R * width, below 2^31
    int need = 0, give = 0;
    unsigned bad = 0u;
#pragma unroll
    for (int i = 0; i < kPerThread; ++i)
        if (i < mine) {
            part[i] = -1;
            if (old[i] < 0 || now[i] < 0 || old[i] > most || now[i] > most) { bad |= 1u << i; continue; }
            const int had = static_cast<int>(bs.up(old[i])), has = static_cast<int>(bs.up(now[i]));
            if (now[i] > old[i]) {
                tokens += static_cast<double>(now[i] - old[i]); need += has - had;
                const int j = static_cast<int>(bs.div(old[i]));
                if (OPEN && j < had) part[i] = pp.table[static_cast<long long>(r0 + i) * pp.width + j];
            } else give += had - has;
        }
    // Sums over the requests of the threads before.  All waves join the waves' sums, a lane to a wave.
    const double tokens_in = wave_scan_d(tokens);
    const int need_in = wave_scan_i(need), give_in = wave_scan_i(give);
    if (lane == 63) { wave_tokens[wave] = tokens_in; wave_fresh[wave] = need_in; wave_freed[wave] = give_in; }
    __syncthreads();
    const bool is_wave = lane < kPageWaves;
    const double tokens_up = wave_scan_d(is_wave ? wave_tokens[lane] : 0.0);
    const int need_up = wave_scan_i(is_wave ? wave_fresh[lane] : 0), give_up = wave_scan_i(is_wave ? wave_freed[lane] : 0), given = __builtin_amdgcn_readlane(give_up, 63);
    const double tokens_to = tokens_in + (wave > 0 ? read_lane(tokens_up, wave - 1) : 0.0);
    const int need_to = need_in + (wave > 0 ? __builtin_amdgcn_readlane(need_up, wave - 1) : 0), give_to = give_in + (wave > 0 ? __builtin_amdgcn_readlane(give_up, wave - 1) : 0);
    // Grants in order: the sums only rise, so from the first request that finds too little on, every growing one does, and what is granted are the
    // sums before that one.
    const unsigned have = static_cast<unsigned>(count) + static_cast<unsigned>(given), capacity = static_cast<unsigned>(pp.slots_capacity);
    // tokens beyond 2^31 are beyond any capacity, and stay there: a request adds 2^31 at most
    unsigned at_tokens = static_cast<unsigned>(fmin(tokens_to - tokens, kMostTokens));
    int at_need = need_to - need, at_give = give_to - give;
#pragma unroll
    for (int i = 0; i < kPerThread; ++i)
        if (i < mine) {
            const int r = r0 + i;
            starts[r] = static_cast<int>(min(at_tokens, 0x7FFFFFFFu)); fresh[r] = at_need; freed[r] = at_give;
            int status = GR_ROW_OK, length = now[i];
            from[r] = old[i];
            if (bad >> i & 1u) { status = GR_ROW_BAD; length = old[i]; }
            else if (now[i] > old[i]) {
                const unsigned before_tokens = at_tokens;
                const int before_need = at_need;
                at_tokens = min(at_tokens, 0x7FFFFFFFu) + static_cast<unsigned>(now[i] - old[i]);
                at_need += static_cast<int>(bs.up(now[i])) - static_cast<int>(bs.up(old[i]));
                if (static_cast<unsigned>(at_need) > have || at_tokens > capacity) {
                    status = GR_ROW_NO_ROOM; length = old[i];
                    atomicMin(&got_tokens, before_tokens); atomicMin(&got_fresh, static_cast<unsigned>(before_need));
                }
            } else { at_give += static_cast<int>(bs.up(old[i])) - static_cast<int>(bs.up(now[i])); from[r] = now[i]; }
            if (OPEN) open[r] = part[i];
            if (first) { pp.out_lengths[r] = length; pp.status[r] = status; }
        }
    if (tid == kPageThreads - 1) {
        starts[R] = static_cast<int>(min(static_cast<unsigned>(fmin(tokens_to, kMostTokens)), 0x7FFFFFFFu)); fresh[R] = need_to; freed[R] = given;
    }
    __syncthreads();
    const bool refused = got_tokens != ~0u;
    if (refused) {                                        // the same for all threads
        const int t = static_cast<int>(got_tokens), f = static_cast<int>(got_fresh);
        for (int r = tid; r <= R; r += kPageThreads) { starts[r] = min(starts[r], t); fresh[r] = min(fresh[r], f); }
        __syncthreads();
    }
    const int T = starts[R], fresh_all = fresh[R], freed_all = given;
    if (first) {
        for (int r = tid; r <= R; r += kPageThreads) pp.starts[r] = starts[r];
        if (tid == 0) *pp.out_free_count = static_cast<int>(min(have - static_cast<unsigned>(fresh_all), static_cast<unsigned>(pp.pool)));
    }

    // the m-th released block, by request and place; the table's rows of shrinking requests are written by nobody
    const auto released = [&](int m) {
        const int r = owner_of(freed, R, m);
        return pp.table[static_cast<long long>(r) * pp.width + bs.up(from[r]) + (m - freed[r])];
    };
    // the i-th block taken off the stack: what was released lies on top of the free ones
    const auto taken = [&](int i) { return i < freed_all ? released(freed_all - 1 - i) : pp.free_blocks[count - 1 - (i - freed_all)]; };
    const int step = gridDim.x * kPageThreads, me = blockIdx.x * kPageThreads + tid;
    for (int i = me; i < fresh_all; i += step) {
        const int r = owner_of(fresh, R, i);
        pp.table[static_cast<long long>(r) * pp.width + bs.up(from[r]) + (i - fresh[r])] = taken(i);
    }
    for (int m = me; m < freed_all - fresh_all; m += step)
        if (count + m < pp.pool) pp.free_blocks[count + m] = released(m);
    // the block of place `at` of a growing request
    const auto block_of = [&](int r, unsigned old_length, int j) {
        const int had = static_cast<int>(bs.up(old_length));
        return j >= had ? taken(fresh[r] + (j - had)) : (OPEN ? open[r] : pp.table[static_cast<long long>(r) * pp.width + j]);
    };
    const auto slot_of = [&](int id, int j, unsigned at) { return id < 0 ? -1ll : static_cast<long long>(id) * bs.size + (at - static_cast<unsigned>(j) * bs.size); };
    if (T <= step) {
        if (me < T) {
            const int r = owner_of(starts, R, me);
            const unsigned at = static_cast<unsigned>(from[r]) + static_cast<unsigned>(me - starts[r]);
            const int j = static_cast<int>(bs.div(at));
            pp.slots[me] = slot_of(block_of(r, from[r], j), j, at);
        }
        return;
    }
    // many: kRun one after the other per thread, one search for all of them
    for (long long t0 = static_cast<long long>(me) * kRun; t0 < T; t0 += static_cast<long long>(step) * kRun) {
        int r = owner_of(starts, R, static_cast<int>(t0)), block = -1, id = -1;
        long long slot[kRun];
#pragma unroll
        for (int u = 0; u < kRun; ++u) {
            const long long t = t0 + u;
            if (t >= T) { slot[u] = 0; continue; }
            if (t >= starts[r + 1]) {
                do ++r; while (t >= starts[r + 1]);
                block = -1;
            }
            const unsigned at = static_cast<unsigned>(from[r]) + static_cast<unsigned>(t - starts[r]);
            const int j = static_cast<int>(bs.div(at));
            if (j != block) { block = j; id = block_of(r, from[r], j); }
            slot[u] = slot_of(id, j, at);
        }
        if (t0 + kRun <= T && (reinterpret_cast<uintptr_t>(pp.slots) & 15) == 0) {
#pragma unroll
            for (int u = 0; u < kRun; u += 2) *reinterpret_cast<longlong2*>(pp.slots + t0 + u) = make_longlong2(slot[u], slot[u + 1]);
        } else {
#pragma unroll
            for (int u = 0; u < kRun; ++u) if (t0 + u < T) pp.slots[t0 + u] = slot[u];
        }
    }
}

}  // namespace

hipError_t launch_pages(const PageParams& pp, hipStream_t stream) {
    BlockSize bs;
    bs.size = static_cast<unsigned>(pp.block);
    bs.shift = (pp.block & (pp.block - 1)) == 0 ? __builtin_ctz(pp.block) : -1;
    // a workgroup to 4096 slots, or to 16384 places of the table, which may all be released; as many as there are compute units at most
    const long long places = static_cast<long long>(pp.R) * pp.width;
    const long long groups = std::min(256ll, std::max((pp.slots_capacity + kPageThreads * kRun - 1) / (kPageThreads * kRun), (places + 16383) / 16384));
    const bool open = pp.R <= kOpenRequests;
    const int lds = (open ? 5 : 4) * (pp.R + 1) * static_cast<int>(sizeof(int));
    const void* const kernel = open ? reinterpret_cast<const void*>(pages_kernel<true>) : reinterpret_cast<const void*>(pages_kernel<false>);
    if (lds > 48 * 1024) {
        const hipError_t e = hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, lds);
        if (e != hipSuccess) return e;
    }
    if (open) hipLaunchKernelGGL(pages_kernel<true>, dim3(static_cast<unsigned>(groups)), dim3(kPageThreads), lds, stream, pp, bs);
    else hipLaunchKernelGGL(pages_kernel<false>, dim3(static_cast<unsigned>(groups)), dim3(kPageThreads), lds, stream, pp, bs);
    return hipGetLastError();
}

}  // namespace gr
