// Pages of the cache after lengths have changed: block tables, slot maps and the free list, in one launch and without the host.
#include <algorithm>

#include "gr_paths.h"

namespace gr {

namespace {

constexpr int kPageThreads = 1024, kPageWaves = kPageThreads / 64, kRun = 4;
constexpr long long kMostInt = 0x7FFFFFFFll, kEndless = 0x7FFFFFFFFFFFFFFFll;

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
// LDS: exclusive sums by request of new tokens, new blocks and released blocks.
// Bound: the launch and a chain of scan, search and stores; with many prompt tokens the stores of the slots.
__global__ __launch_bounds__(kPageThreads) void pages_kernel(const PageParams pp, const BlockSize bs) {
    extern __shared__ int lds[];
    const int R = pp.R;
    int* const starts = lds; int* const fresh = lds + R + 1; int* const freed = lds + 2 * (R + 1);
    __shared__ long long wave_tokens[kPageWaves], wave_fresh[kPageWaves], wave_freed[kPageWaves];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const bool first = blockIdx.x == 0;
    const int per = (R + kPageThreads - 1) / kPageThreads, r0 = min(R, tid * per), r1 = min(R, r0 + per);
    const long long most = static_cast<long long>(pp.width) * pp.block;
    const int count = max(0, min(*pp.free_count, pp.pool));
    const auto bad = [&](int old, int now) { return old < 0 || now < 0 || old > most || now > most; };

    // sums over this thread's requests, then over those of the threads before it
    long long tokens = 0, need = 0, give = 0;
    for (int r = r0; r < r1; ++r) {
        const int old = pp.lengths[r], now = pp.new_lengths[r];
        if (bad(old, now)) continue;
        const int had = static_cast<int>(bs.up(old)), has = static_cast<int>(bs.up(now));
        if (now > old) { tokens += now - old; need += has - had; } else give += had - has;
    }
    const auto scan = [&](long long v) {
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) { const long long w = __shfl_up(v, o); if (lane >= o) v += w; }
        return v;
    };
    long long tokens_to = scan(tokens), need_to = scan(need), give_to = scan(give);
    if (lane == 63) { wave_tokens[wave] = tokens_to; wave_fresh[wave] = need_to; wave_freed[wave] = give_to; }
    __syncthreads();
    long long given = 0;
    for (int w = 0; w < kPageWaves; ++w) {
        if (w < wave) { tokens_to += wave_tokens[w]; need_to += wave_fresh[w]; give_to += wave_freed[w]; }
        given += wave_freed[w];
    }
    // Grants in order: the sums only rise, so from the first request that finds too little on, every growing one does, and what is granted are the
    // sums before that one.
    const long long have = count + given;
    long long at_tokens = tokens_to - tokens, at_need = need_to - need, at_give = give_to - give;
    long long got_tokens = kPageThreads - 1 == tid ? tokens_to : kEndless, got_need = kPageThreads - 1 == tid ? need_to : kEndless;
    for (int r = r0; r < r1; ++r) {
        const int old = pp.lengths[r], now = pp.new_lengths[r];
        starts[r] = static_cast<int>(min(at_tokens, kMostInt)); fresh[r] = static_cast<int>(min(at_need, kMostInt)); freed[r] = static_cast<int>(at_give);
        int status = GR_ROW_OK, length = now;
        if (bad(old, now)) { status = GR_ROW_BAD; length = old; }
        else if (now > old) {
            const long long before_tokens = at_tokens, before_need = at_need;
            at_tokens += now - old;
            at_need += static_cast<int>(bs.up(now)) - static_cast<int>(bs.up(old));
            if (at_need > have || at_tokens > pp.slots_capacity) {
                status = GR_ROW_NO_ROOM; length = old;
                got_tokens = min(got_tokens, before_tokens); got_need = min(got_need, before_need);
            }
        } else at_give += static_cast<int>(bs.up(old)) - static_cast<int>(bs.up(now));
        if (first) { pp.out_lengths[r] = length; pp.status[r] = status; }
    }
    __syncthreads();                                      // the waves' sums have been read
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) { got_tokens = min(got_tokens, __shfl_xor(got_tokens, o)); got_need = min(got_need, __shfl_xor(got_need, o)); }
    if (lane == 0) { wave_tokens[wave] = got_tokens; wave_fresh[wave] = got_need; }
    __syncthreads();
    for (int w = 0; w < kPageWaves; ++w) { got_tokens = min(got_tokens, wave_tokens[w]); got_need = min(got_need, wave_fresh[w]); }
    const int T = static_cast<int>(got_tokens), fresh_all = static_cast<int>(got_need), freed_all = static_cast<int>(given);
    for (int r = r0; r < r1; ++r) {
        starts[r] = min(starts[r], T); fresh[r] = min(fresh[r], fresh_all);
        if (first) pp.starts[r] = starts[r];
    }
    if (tid == 0) {
        starts[R] = T; fresh[R] = fresh_all; freed[R] = freed_all;
        if (first) { pp.starts[R] = T; *pp.out_free_count = static_cast<int>(min(have - fresh_all, static_cast<long long>(pp.pool))); }
    }
    __syncthreads();

    // the m-th released block, by request and place; the table's rows of shrinking requests are written by nobody
    const auto released = [&](int m) {
        const int r = owner_of(freed, R, m);
        return pp.table[static_cast<long long>(r) * pp.width + bs.up(pp.new_lengths[r]) + (m - freed[r])];
    };
    // the i-th block taken off the stack: what was released lies on top of the free ones
    const auto taken = [&](int i) { return i < freed_all ? released(freed_all - 1 - i) : pp.free_blocks[count - 1 - (i - freed_all)]; };
    const int step = gridDim.x * kPageThreads, me = blockIdx.x * kPageThreads + tid;
    for (int i = me; i < fresh_all; i += step) {
        const int r = owner_of(fresh, R, i);
        pp.table[static_cast<long long>(r) * pp.width + bs.up(pp.lengths[r]) + (i - fresh[r])] = taken(i);
    }
    for (int m = me; m < freed_all - fresh_all; m += step)
        if (count + m < pp.pool) pp.free_blocks[count + m] = released(m);
    // slots, kRun one after the other per thread: one search for all of them
    for (long long t0 = static_cast<long long>(me) * kRun; t0 < T; t0 += static_cast<long long>(step) * kRun) {
        int r = owner_of(starts, R, static_cast<int>(t0)), block = -1, id = -1;
        unsigned old = pp.lengths[r];
        long long slot[kRun];
#pragma unroll
        for (int u = 0; u < kRun; ++u) {
            const long long t = t0 + u;
            if (t >= T) { slot[u] = 0; continue; }
            if (t >= starts[r + 1]) {
                do ++r; while (t >= starts[r + 1]);
                old = pp.lengths[r];
                block = -1;
            }
            const unsigned at = old + static_cast<unsigned>(t - starts[r]);
            const int j = static_cast<int>(bs.div(at));
            if (j != block) {
                const int had = static_cast<int>(bs.up(old));
                block = j;
                id = j < had ? pp.table[static_cast<long long>(r) * pp.width + j] : taken(fresh[r] + (j - had));
            }
            slot[u] = id < 0 ? -1ll : static_cast<long long>(id) * bs.size + (at - static_cast<unsigned>(j) * bs.size);
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
    // a workgroup to 4096 slots, as many as there are compute units at most
    const long long groups = std::min(256ll, std::max(1ll, (pp.slots_capacity + kPageThreads * kRun - 1) / (kPageThreads * kRun)));
    const int lds = 3 * (pp.R + 1) * static_cast<int>(sizeof(int));
    if (lds > 48 * 1024) {
        const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(pages_kernel), hipFuncAttributeMaxDynamicSharedMemorySize, lds);
        if (e != hipSuccess) return e;
    }
    hipLaunchKernelGGL(pages_kernel, dim3(static_cast<unsigned>(groups)), dim3(kPageThreads), lds, stream, pp, bs);
    return hipGetLastError();
}

}  // namespace gr
