// One streaming pass over rows of logits or probabilities in float32, bfloat16 or float16: the k largest entries of every row slice and,
// where they are asked for, the sum of the row (probabilities) or of its exponentials (logits); and the sums of a row by pieces.
// It stands behind the drafts' draw (gr_draft.hip) and the beams' selection (gr_beam.hip).
//
// Bound: HBM, one read of the row, where only the largest are asked for (about 5 instructions per element).  With the exponentials, in float64, it is about 20, 12 of them in the
// innermost loop, and a rate of one instruction for 40 million million elements a second, which float64 has here as float32 has unpacked: 16.5 us for the 29.5 million bfloat16 logits
// of 230 rows of 128256, whose 59 MB a copy's rate reads in 12.
// Measured: those 28 us; 640 rows of 128256 in float32 82 us (4.0 TB/s); one row of 32000 8.0 us; without sums 256 rows of 128256 in bfloat16, k = 128, 20.6 us (3.2 TB/s).
#include <algorithm>

#include "gr_draft.h"

namespace gr {

namespace {

// What a scan of NT threads keeps in LDS: candidate keys, chunks with candidates (a share to every wave).
template <int NT> constexpr int kRowCap = NT <= 256 ? 1024 : 2048;
template <int NT> constexpr int kListCap = NT <= 256 ? 1024 : 2048;
template <int NT> constexpr int kWaveList = kListCap<NT> / (NT / 64);

// Of the keys of a stretch of the row one that exactly k of them reach (0, as ruled out entries: fewer than k).  Only slices with more entries at their threshold than LDS holds come
// here (rows of equal entries, rows that rise), so the stretch is read again for every digit, and a digit that a whole wave agrees on is counted once.
template <int NT, typename KeyAt>
__device__ __forceinline__ unsigned long long stretch_kth_largest(KeyAt key_at, int count, int k, int* hist, int* pick) {
    const int tid = threadIdx.x;
    unsigned long long prefix = 0;
    int need = k;
    for (int shift = 56; shift >= 0; shift -= 8) {
        if (tid < 256) hist[tid] = 0;
        __syncthreads();
        const unsigned long long mask = (shift == 56) ? 0ull : (~0ull << (shift + 8));
        for (int i = tid; i < count; i += NT) {
            const unsigned long long key = key_at(i);
            if (key != 0ull && (key & mask) == prefix) {
                const int digit = static_cast<int>((key >> shift) & 255ull);
                const unsigned long long here = __ballot(1);
                if (__all(digit == __builtin_amdgcn_readfirstlane(digit))) {
                    if ((tid & 63) == __ffsll(here) - 1) atomicAdd(&hist[digit], __popcll(here));
                } else atomicAdd(&hist[digit], 1);
            }
        }
        __syncthreads();
        if (tid < 64) {
            // lane l owns digits 255-4l .. 252-4l (largest digits in lane 0)
            int c[4]; int tot = 0;
            for (int j = 0; j < 4; ++j) { c[j] = hist[255 - 4 * tid - j]; tot += c[j]; }
            const int incl = wave_scan_i(tot);
            const int excl = incl - tot;
            if (excl < need && need <= incl) {
                int above = excl;
                for (int j = 0; j < 4; ++j) {
                    if (need <= above + c[j]) { pick[0] = 255 - 4 * tid - j; pick[1] = need - above; pick[2] = c[j]; break; }
                    above += c[j];
                }
            }
            if (tid == 63 && incl < need) { pick[0] = 0; pick[1] = 0; pick[2] = 0; }         // fewer than k: at the first digit only
        }
        __syncthreads();
        prefix |= static_cast<unsigned long long>(pick[0]) << shift;
        need = pick[1];
        const bool whole_bucket = pick[2] == need;
        __syncthreads();
        if (whole_bucket) break;
    }
    return prefix;
}

// A threshold that at least k of the entries reach (-inf: none was found), from the largest entries `top` of the threads' chunks (kLoads each, different entries; -inf: none), of which
// `threads` have some: about the k-th largest of them.  With 8192 entries to a tile 9 reach it for k = 8, 136 for k = 128, 290 for k = 256.  First a bound from below: of k groups of
// adjacent lanes at least the smallest of the groups' largest.  Then 256 linear bins from there to the largest entry.  All threads call it.
template <bool PROBS, int NT>
__device__ __forceinline__ float find_threshold(const float* tops, int threads, int k, int* hist, float* edge) {
    constexpr int kNW = NT / 64;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    float top[kLoads], most = kNone;
#pragma unroll
    for (int l = 0; l < kLoads; ++l) { top[l] = binned<PROBS>(tops[l]); most = fmaxf(most, top[l]); }
    // the largest of 2, 4, 8, 16 lanes; groups as large as leave k of them, where nothing is masked
    const float of2 = fmaxf(most, dpp_move_f<kDppXor1>(most)), of4 = fmaxf(of2, dpp_move_f<kDppXor2>(of2)), of8 = fmaxf(of4, dpp_move_f<kDppHalfMirror>(of4));
    const float of16 = fmaxf(of8, dpp_move_f<kDppMirror>(of8));
    const int size = threads >= 16 * k ? 16 : (threads >= 8 * k ? 8 : (threads >= 4 * k ? 4 : (threads >= 2 * k ? 2 : 1)));
    const float group = size == 16 ? of16 : (size == 8 ? of8 : (size == 4 ? of4 : (size == 2 ? of2 : most)));
    const bool any = group > kNone;
    float hi = wave_max_f(of16), lo = wave_min_f(any ? group : __builtin_inff()), lanes = static_cast<float>(__popcll(__ballot(any)));
    __syncthreads();                                      // whoever reads what an earlier call left is done
    if (tid < 256) hist[tid] = 0;
    if (lane == 0) { edge[wave] = lo; edge[kNW + wave] = hi; edge[2 * kNW + wave] = lanes; }
    __syncthreads();
    join_edges<kNW>(edge, lo, hi);
    lanes = lanes_sum_f<kNW>(edge[2 * kNW + (lane & (kNW - 1))]);
    if (__any(lanes < static_cast<float>(size * k))) return kNone;               // the same for all threads
    const float per = 255.f / (hi - lo);
#pragma unroll
    for (int l = 0; l < kLoads; ++l) if (top[l] >= lo) atomicAdd(&hist[static_cast<int>(fminf(fmaxf((top[l] - lo) * per, 0.f), 255.f))], 1);
    __syncthreads();
    int in[4], tot = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) { in[j] = hist[255 - 4 * lane - j]; tot += in[j]; }
    const int incl = wave_scan_i(tot);
    int above = incl - tot, from = -1;
    const bool mine_is = above < k && k <= incl;
    if (mine_is)
#pragma unroll
        for (int j = 0; j < 4; ++j) { above += in[j]; if (from < 0 && above >= k) from = 255 - 4 * lane - j; }
    from = __builtin_amdgcn_readlane(from, __ffsll(static_cast<unsigned long long>(__ballot(mine_is))) - 1);
    return unbinned<PROBS>(bin_edge(lo, hi, from));
}

// rows_kernel: grid = (splits * rows), 256 threads.  Workgroup s of a row reads chunks [s * per, (s + 1) * per) of its row, tiles of 256 * kLoads chunks, the next
// tile's loads on their way while the present one is worked on, and no barrier between tiles but for the threshold of the first.
// The k largest: a chunk whose largest entry reaches the threshold goes, as it was loaded, to a list in LDS; the few on it are taken apart together at
// the end (in the order of tiles every one would cost all lanes of its wave the test of every entry: 55 us where this takes 21, 256 rows of 128256 in bfloat16).
// Keys are 64 bits (entry, ~id).  After `refresh` tiles the list is worked off and the threshold rises to about the k-th key.
// A slice leaves at least its k largest, up to `limit` candidates.
// SUM: PROBS: the float64 sum of the slice.  Logits: the sum of exp((x - ref) / T) in float64, per wave with its own reference, joined at the end.  (The hardware's float32
// exponential, with the listed chunks in float64, took 22 us for 230 rows and 72 for 640 where this takes 27.5 and 81, but sums are good to 2e-8 only then, and beams closer than that
// change places.)
// Rows of beams that are not in use or finished are not read (Rows::skip).
// Four waves to a SIMD with the exponentials: for a fifth their loop spills (32 us became 37, 89 became 114).
template <bool EXP, int NT>
struct ScanLds {
    unsigned long long keys[kRowCap<NT>];
    uint4 list[kListCap<NT>];
    int list_chunk[kListCap<NT>];
    int hist[256], pick[4], count, listed[NT / 64];
    float edge[3 * (NT / 64)];
    double red[NT / 64], tab[EXP ? kExpEntries : 1];
};
// What a thread has of a slice behind a scan: how many keys lie in LDS (the same for all), whether it met a bad entry, its part of the sum (with its wave's reference).
struct Scanned { int found, bad; double total; ExpSum<> es; };

template <typename T, bool PROBS, bool EXP, int NT>
__device__ __forceinline__ Scanned scan_slice(ScanLds<EXP, NT>& L, const Rows<T>& in, int row, const RowChunks<T, PROBS>& x, int c_first, int c_end, int k) {
    constexpr int N = Packed<T>::N, kTileChunks = NT * kLoads, kNW = NT / 64, kCap = kRowCap<NT>;
    constexpr bool kExp = EXP;
    unsigned long long* const keys = L.keys;
    uint4* const list = L.list; int* const list_chunk = L.list_chunk; int* const hist = L.hist; int* const pick = L.pick; int* const listed = L.listed;
    int& count = L.count;
    float* const edge = L.edge; double* const tab = L.tab;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    uint4 next[kLoads];
    const auto fetch = [&](int c0) {
        if (c0 + kTileChunks <= c_end && x.inside(c0, c0 + kTileChunks)) {
#pragma unroll
            for (int l = 0; l < kLoads; ++l) next[l] = x.load(c0, l * NT + tid);
        } else if (c0 < c_end)
#pragma unroll
            for (int l = 0; l < kLoads; ++l) {
                const int c = c0 + l * NT;
                if (c + NT <= c_end && x.inside(c, c + NT)) next[l] = x.load(c, tid);
                else if (c < c_end) next[l] = x.load_guarded(c + tid < c_end ? c + tid : x.chunks);
            }
    };
    fetch(c_first);
    int bad = 0;
    double scale = 1.0;
    if (kExp) {
        const float temp = in.temperature_of(row);
        if (!good_temperature(temp)) bad = 1; else scale = kPerTemp / static_cast<double>(temp);
        if (tid < kExpEntries) fill_exp_table(tab);
    }
    if (tid == 0) count = 0;
    int mine_listed = 0;                                  // chunks on the wave's own share of the list
    __syncthreads();

    float theta = kNone;                                  // entries below it are no candidates
    bool over = false;                                    // more candidates than LDS holds
    double total = 0.0;
    ExpSum<> es(scale);
    const float least = PROBS ? 0.f : kNone;              // entries must lie above it
    const auto key_of = [](float v, int id) { return PROBS ? make_key(v, id) : make_key_logit(v, id); };
    // the list taken apart: its entries that reach the threshold become keys
    const auto work_off = [&]() {
        if (lane == 0) listed[wave] = mine_listed;
        mine_listed = 0;
        __syncthreads();
        const int n = lane < kNW ? listed[lane] : 0, upto_wave = wave_scan_i(min(n, kWaveList<NT>)), all = __builtin_amdgcn_readlane(upto_wave, 63);
        over = over || __any(n > kWaveList<NT>);
#pragma unroll
        for (int r = 0; r < kListCap<NT> / NT; ++r) {
            // the i-th chunk of the waves' shares one after the other
            const int i0 = tid + r * NT;
            const bool have = i0 < all;
            if (!__any(have)) break;
            int i = i0;
#pragma unroll
            for (int w = 1; w < kNW; ++w) {
                const int before = __builtin_amdgcn_readlane(upto_wave, w - 1);
                if (i0 >= before) i = w * kWaveList<NT> + i0 - before;
            }
            const uint4 raw = have ? list[i] : make_uint4(0u, 0u, 0u, 0u);
            const int chunk = have ? list_chunk[i] : 0;
            unsigned mask = 0u;
#pragma unroll
            for (int j = 0; j < N; ++j) {
                const float v = Packed<T>::get(raw, j);
                if (have && v >= theta && v > least) mask |= 1u << j;
            }
            const int upto = wave_scan_i(__popc(mask));
            int base = 0;
            if (lane == 63) base = atomicAdd(&count, upto);
            int slot = __builtin_amdgcn_readlane(base, 63) + upto - __popc(mask);
#pragma unroll
            for (int j = 0; j < N; ++j)
                if (mask >> j & 1u) { if (slot < kCap) keys[slot] = key_of(Packed<T>::get(raw, j), x.id(chunk, j)); ++slot; }
        }
        __syncthreads();
        over = over || count > kCap;
    };

    // The first tile's threshold lies at about its k-th entry, give or take 1 / sqrt(k) of its rank, and a wave finds its share of them, give or take the root: six times that
    // much has room for so many tiles.  Later ones hold ever fewer candidates, so the stretches double.
    const float wave_k = static_cast<float>(k) / kNW;
    int refresh = max(1, static_cast<int>(kWaveList<NT> / (wave_k + 6.f * sqrtf(wave_k) + 8.f))), tiles = 0;
    const int quarter = (c_end - c_first + 3) / 4;
    for (int c0 = c_first; c0 < c_end; c0 += kTileChunks) {
        if (kExp) {
            // Arithmetic bounds this loop, and of the waves on a SIMD the oldest goes first by itself, so that the last is left with nothing to cover its latencies.  Those that are behind go
            // first: 31.4 us become 28.4 (256 rows of 128256 in bfloat16), 86 become 82 (640 in float32).
            const int gone = c0 - c_first;
            if (gone < quarter) __builtin_amdgcn_s_setprio(3);
            else if (gone < 2 * quarter) __builtin_amdgcn_s_setprio(2);
            else if (gone < 3 * quarter) __builtin_amdgcn_s_setprio(1);
            else __builtin_amdgcn_s_setprio(0);
        }
        uint4 now[kLoads];
#pragma unroll
        for (int l = 0; l < kLoads; ++l) now[l] = next[l];
        fetch(c0 + kTileChunks);
        const int loads = min(kLoads, (c_end - c0 + NT - 1) / NT);     // of the last tile maybe fewer
        // Bad: NaN, logits above kMostLogit, negative entries (probabilities).
        float top[kLoads], most = kNone, probe = 0.f;
#pragma unroll
        for (int l = 0; l < kLoads; ++l) {
            top[l] = kNone;
            if (l >= loads) continue;
#pragma unroll
            for (int j = 0; j < N; ++j) {
                const float v = Packed<T>::get(now[l], j);
                top[l] = fmaxf(top[l], v);
                if (PROBS) {
                    bad |= static_cast<int>(!(v >= 0.f));
                    total += static_cast<double>(v);
                } else if (!kExp) probe += v;
            }
            most = fmaxf(most, top[l]);
            unpack_again(now[l]);
        }
        if (!PROBS && !kExp) bad |= static_cast<int>(probe != probe) | static_cast<int>(most > kMostLogit);          // NaN makes the sum NaN
        if (kExp) {
            bad |= static_cast<int>(most > kMostLogit);
            es.raise(most, tab);
            if (es.ref == kNone) {
                // nothing but masked entries and NaN, which the maximum passes over
#pragma unroll
                for (int l = 0; l < kLoads; ++l)
#pragma unroll
                    for (int j = 0; j < N; ++j) { const float v = Packed<T>::get(now[l], j); bad |= static_cast<int>(l < loads) & static_cast<int>(v != v); }
            } else
#pragma unroll
                for (int l = 0; l < kLoads; l += ExpSum<>::kEight / N) {
                    if (l >= loads) continue;
                    float v[ExpSum<>::kEight];
#pragma unroll
                    for (int j = 0; j < ExpSum<>::kEight; ++j) v[j] = l + j / N < loads ? Packed<T>::get(now[l + j / N], j % N) : kNone;
                    es.add(v, tab);
                }
        }
        if (PROBS && theta == kNone) {
            // chunks behind the slice, zeros, have no part in the threshold
#pragma unroll
            for (int l = 0; l < kLoads; ++l) if (c0 + l * NT + tid >= c_end) top[l] = kNone;
        }
        if (theta == kNone) theta = find_threshold<PROBS, NT>(top, min(NT, c_end - c0), k, hist, edge);
        unsigned long long hit[kLoads];
        int hits = 0;
#pragma unroll
        for (int l = 0; l < kLoads; ++l) { hit[l] = __ballot(top[l] >= theta && top[l] > least); hits += __popcll(hit[l]); }
        if (hits != 0) {
            int slot = mine_listed;
#pragma unroll
            for (int l = 0; l < kLoads; ++l) {
                const int at = slot + __builtin_amdgcn_mbcnt_hi(static_cast<unsigned>(hit[l] >> 32), __builtin_amdgcn_mbcnt_lo(static_cast<unsigned>(hit[l]), 0u));
                if ((hit[l] >> lane & 1ull) && at < kWaveList<NT>) { list[wave * kWaveList<NT> + at] = now[l]; list_chunk[wave * kWaveList<NT> + at] = c0 + l * NT + tid; }
                slot += __popcll(hit[l]);
            }
            mine_listed = slot;
        }
        if (++tiles == refresh && c0 + kTileChunks < c_end) {
            refresh *= 2;
            work_off();
            const int c = count;
            __syncthreads();
            if (!over && c > k) {
                float reach;
                thin_keys<kCap, PROBS, NT>(keys, c, k, kCap / 2, hist, pick, edge, &count, &reach);
                theta = fmaxf(theta, reach);
            }
            __syncthreads();
        }
    }
    work_off();
    int found = count;
    __syncthreads();
    if (over) {
        // the slice's k largest by themselves
        const long long e0 = max(0ll, static_cast<long long>(c_first) * N - x.lead), e1 = min(static_cast<long long>(x.V), static_cast<long long>(c_end) * N - x.lead);
        const auto slice_key = [&](int i) -> unsigned long long {
            const float e = Packed<T>::one(x.row[e0 + i]);
            return e > least ? key_of(e, static_cast<int>(e0 + i)) : 0ull;
        };
        const unsigned long long reach = stretch_kth_largest<NT>(slice_key, static_cast<int>(e1 - e0), k, hist, pick);
        if (tid == 0) count = 0;
        __syncthreads();
        for (int i = tid; i < static_cast<int>(e1 - e0); i += NT) {
            const unsigned long long key = slice_key(i);
            if (key >= reach && key != 0ull) keys[atomicAdd(&count, 1)] = key;
        }
        __syncthreads();
        found = count;                                    // k, or all that there are
        __syncthreads();
    }
    return Scanned{found, bad, total, es};
}

template <typename T, bool PROBS, bool SUM>
__global__ __launch_bounds__(kThreads, SUM && !PROBS ? 4 : 5) void rows_kernel(const Rows<T> in, int k, int limit, int splits, int per, const RowParts out) {
    constexpr bool kExp = SUM && !PROBS;
    __shared__ ScanLds<kExp, kThreads> L;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int row = blockIdx.x / splits, s = blockIdx.x - row * splits;
    if (in.skip(row)) return;
    const RowChunks<T, PROBS> x(in.row(row), in.V);
    Scanned mine = scan_slice<T, PROBS, kExp, kThreads>(L, in, row, x, s * per, min(x.chunks, s * per + per), k);
    int found = mine.found;
    const int room = min(kSelCap / splits, limit);        // k at least
    unsigned long long* const to = out.cand + static_cast<size_t>(row) * kSelCap + s * (kSelCap / splits);
    if (found > room) found = thin_keys<kRowCap<kThreads>, PROBS>(L.keys, found, k, room, L.hist, L.pick, L.edge, &L.count);
    for (int i = tid; i < found; i += kThreads) to[i] = L.keys[i];
    // the waves' sums: of exponentials, to the largest of their references
    __syncthreads();
    if (kExp) mine.bad |= static_cast<int>(!(mine.es.sum == mine.es.sum));
    const double wave_total = SUM ? wave_sum(kExp ? mine.es.sum : mine.total) : 0.0;
    const bool wave_bad = __any(mine.bad != 0);
    if (lane == 0) { L.red[wave] = wave_total; L.edge[wave] = mine.es.ref; L.pick[wave] = wave_bad; }
    __syncthreads();
    if (tid < kWaves) {
        // a lane to a wave's sum
        float ref = mine.es.ref;
        double sum = L.red[tid];
        if (kExp) {
            mine.es.set(L.edge[tid]); mine.es.sum = sum;
            ref = fmaxf(fmaxf(L.edge[0], L.edge[1]), fmaxf(L.edge[2], L.edge[3]));
            sum = mine.es.rebased(ref, L.tab);
        }
        sum += __shfl_xor(sum, 1);
        sum += __shfl_xor(sum, 2);
        if (tid == 0) {
            const int at = row * splits + s;
            out.count[at] = found; out.bad[at] = L.pick[0] | L.pick[1] | L.pick[2] | L.pick[3];
            if (SUM) { out.sum[at] = sum; if (!PROBS) out.ref[at] = ref; }
        }
    }
}

// The drafts of rows that one workgroup each reads: grid = (rows), NT threads.  No slices to join, so one launch does, and the candidates never leave LDS.
// Bound: for one row a chain of dependent steps, 9.5 us for 32000 float32 logits, k = 64, of them 1.5 until the first tile has come, 2.2 for its threshold, 1.0 for the second tile, 1.6
// to take the list apart, 0.8 to put 118 candidates in order, 0.6 to put 64 in order by id, 0.4 for the draws.  For 256 rows of 128256 in bfloat16 22.8 us, of which
// the read takes 10 where the last cache holds the 66 MB (13 at a copy's rate).
// What all waves repeat costs four times its instructions on a SIMD with four of them, so it is kept short.
template <typename T, bool PROBS, int NT>
__global__ __launch_bounds__(NT) void draft_rows_kernel(const Rows<T> in, int k, double tail_mass, const DraftOut out) {
    __shared__ union { ScanLds<false, NT> scan; DraftLds<kRowCap<NT>, NT> draft; } L;       // the keys are the first of both
    static_assert(offsetof(decltype(L.scan), keys) == 0 && offsetof(decltype(L.draft), keys) == 0 && sizeof(L.scan.keys) == sizeof(L.draft.keys));
    __shared__ double q_wave[PROBS ? NT / 64 : 1];
    __shared__ int any_bad;
    const int tid = threadIdx.x, lane = tid & 63, row = blockIdx.x;
    if (tid == 0) any_bad = 0;
    const RowChunks<T, PROBS> x(in.row(row), in.V);
    const Uniforms<NT> uniforms(out, row);
    const float t = PROBS ? 1.f : in.temperature_of(row);
    const Scanned mine = scan_slice<T, PROBS, false, NT>(L.scan, in, row, x, 0, x.chunks, k);
    if (PROBS) {
        const double q_mine = wave_sum(mine.total);
        if (lane == 0) q_wave[tid >> 6] = q_mine;
    }
    if (mine.bad) any_bad = 1;                            // cleared before the scan, which has barriers
    __syncthreads();
    double q_total = 0.0, inv_temp = 1.0;
    if (PROBS) q_total = wave_sum(lane < NT / 64 ? q_wave[lane] : 0.0);
    bool bad = mine.found == 0 || any_bad != 0;
    if (PROBS) bad = bad || !(fabs(q_total - 1.0) <= 1e-3);
    else if (!good_temperature(t)) bad = true;
    else inv_temp = 1.0 / static_cast<double>(t);
    if (bad) {                                            // the same for all threads
        if (tid < out.n) out.drafts[static_cast<size_t>(row) * out.n + tid] = -1;
        if (tid == 0) out.status[row] = GR_ROW_BAD;
        return;
    }
    draw_from<PROBS>(L.draft, mine.found, k, tail_mass, q_total, inv_temp, uniforms, row, out);
}

// The sum of piece `piece` of a row, a wave's 64 * kLoads chunks one after the other; all lanes hold it.  PROBS: of the entries; logits: of exp((x - ref) / T) with the piece's
// largest entry as ref, scale 0 for a bad temperature.  A bad entry makes it NaN, and with it the row's total.  The exponentials are the finer ones: 256 rows of 128256 in bfloat16 take 32.2 us
// where the others took 31.4, 256 of 151936 in float32 35.6 for 33.9.
struct PieceMass { double mass; float ref; };
template <typename T, bool PROBS>
__device__ __forceinline__ PieceMass piece_mass(const RowChunks<T, PROBS>& x, int piece, double scale, const double* tab) {
    constexpr int N = Packed<T>::N;
    const int lane = threadIdx.x & 63;
    int bad = static_cast<int>(!(scale > 0.0));
    const int c0 = piece * 64 * kLoads;
    uint4 r[kLoads];
    if (x.inside(c0, c0 + 64 * kLoads))
#pragma unroll
        for (int l = 0; l < kLoads; ++l) r[l] = x.load(c0 + l * 64 + lane);
    else
#pragma unroll
        for (int l = 0; l < kLoads; ++l) r[l] = x.load_guarded(c0 + l * 64 + lane);
    float top = kNone;
    double sum = 0.0;
#pragma unroll
    for (int l = 0; l < kLoads; ++l) {
#pragma unroll
        for (int j = 0; j < N; ++j) {
            const float v = Packed<T>::get(r[l], j);
            if (PROBS) {
                bad |= static_cast<int>(!(v >= 0.f));
                sum += static_cast<double>(v);
            } else top = fmaxf(top, v);
        }
        unpack_again(r[l]);
    }
    float ref = 0.f;
    if (!PROBS) {
        bad |= static_cast<int>(top > kMostLogit);
        ref = wave_max_f(top);
        if (ref > kNone && scale > 0.0) {
            ExpSum<true> es(scale);                       // the draws' borders stand on these sums
            es.refer(ref);
#pragma unroll
            for (int l = 0; l < kLoads; l += ExpSum<>::kEight / N) {
                float v[ExpSum<>::kEight];
#pragma unroll
                for (int j = 0; j < ExpSum<>::kEight; ++j) v[j] = Packed<T>::get(r[l + j / N], j % N);
                es.add(v, tab);
            }
            sum = es.rebased(ref, tab);                   // NaN if an entry is
        } else {
            // nothing but masked entries and NaN, which the maximum passes over
#pragma unroll
            for (int l = 0; l < kLoads; ++l)
#pragma unroll
                for (int j = 0; j < N; ++j) { const float v = Packed<T>::get(r[l], j); bad |= static_cast<int>(v != v); }
        }
    }
    sum = wave_sum(sum);
    return PieceMass{__any(bad != 0) ? __builtin_nan("") : sum, ref};
}
template <typename T>
__device__ __forceinline__ double scale_of(const Rows<T>& in, int row) {
    const float temp = in.temperature_of(row);
    return good_temperature(temp) ? kPerTemp / static_cast<double>(temp) : 0.0;
}

// The sums of a row by pieces, a wave to a piece.  grid = (pieces / 4 * rows).  Bound: HBM (probabilities) or the exponentials; 203 rows of 50021 probabilities 8.8 us (4.6 TB/s).
template <typename T, bool PROBS>
__global__ __launch_bounds__(kThreads) void masses_kernel(const Rows<T> in, int pieces, int stride, double* __restrict__ mass, float* __restrict__ refs) {
    __shared__ double tab[PROBS ? 1 : kExpEntries];
    const int tid = threadIdx.x, groups = (pieces + kWaves - 1) / kWaves, row = blockIdx.x / groups;
    if (!PROBS) { fill_exp_table(tab); __syncthreads(); }
    const int piece = (blockIdx.x - row * groups) * kWaves + (tid >> 6);
    if (piece >= pieces) return;                          // whole waves
    const PieceMass m = piece_mass<T, PROBS>(RowChunks<T, PROBS>(in.row(row), in.V), piece, PROBS ? 1.0 : scale_of(in, row), tab);
    if ((tid & 63) == 0) {
        const size_t at = static_cast<size_t>(row) * stride + piece;
        mass[at] = m.mass; refs[at] = m.ref;
    }
}

// Sums and draws of rows that one workgroup each reads, in one launch; the sums by pieces stay in LDS.  grid = (rows), NT threads.
// Bound: HBM.  203 rows of 50021 probabilities, 16 draws each: 12.0 us (3.4 TB/s), 10.4 where the rows lie in the last cache.
template <typename T, bool PROBS, int NT>
__global__ __launch_bounds__(NT) void draft_whole_rows_kernel(const Rows<T> in, int pieces, const DraftOut out) {
    __shared__ double tab[PROBS ? 1 : kExpEntries], mass[kLdsPieces];
    __shared__ float refs[kLdsPieces];
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), row = blockIdx.x;
    if (!PROBS) { if (tid < kExpEntries) fill_exp_table(tab); __syncthreads(); }
    const RowChunks<T, PROBS> x(in.row(row), in.V);
    const double scale = PROBS ? 1.0 : scale_of(in, row);
    for (int piece = wave; piece < pieces; piece += NT / 64) {
        const PieceMass m = piece_mass<T, PROBS>(x, piece, scale, tab);
        if ((tid & 63) == 0) { mass[piece] = m.mass; refs[piece] = m.ref; }
    }
    __syncthreads();
    for (int draw = wave; draw < out.n; draw += NT / 64) draw_whole<T, PROBS>(in, row, draw, pieces, mass, refs, out);
}

template <typename T, bool PROBS, bool SUM>
void launch_rows_as(const RowSource& src, int k, int limit, RowSlices cut, const RowParts& out, hipStream_t stream) {
    hipLaunchKernelGGL((rows_kernel<T, PROBS, SUM>), dim3(cut.splits * src.rows), dim3(kThreads), 0, stream, Rows<T>(src), k, limit, cut.splits, cut.per, out);
}
template <typename T, bool PROBS>
void launch_draft_rows_as(const RowSource& src, int k, double tail_mass, const DraftOut& out, hipStream_t stream) {
    const auto run = [&](auto threads) {
        constexpr int NT = decltype(threads)::value;
        hipLaunchKernelGGL((draft_rows_kernel<T, PROBS, NT>), dim3(src.rows), dim3(NT), 0, stream, Rows<T>(src), k, tail_mass, out);
    };
    const bool one_tile = src.V <= 512 * kLoads * chunk_elements(src.dtype);
    if (src.rows <= kComputeUnits && !one_tile) run(std::integral_constant<int, 1024>{});
    else if (src.rows <= 2 * kComputeUnits) run(std::integral_constant<int, 512>{});
    else run(std::integral_constant<int, 256>{});
}
template <typename T, bool PROBS>
void launch_draft_whole_rows_as(const RowSource& src, int pieces, const DraftOut& out, hipStream_t stream) {
    const auto run = [&](auto threads) {
        constexpr int NT = decltype(threads)::value;
        hipLaunchKernelGGL((draft_whole_rows_kernel<T, PROBS, NT>), dim3(src.rows), dim3(NT), 0, stream, Rows<T>(src), pieces, out);
    };
    if (src.rows <= kComputeUnits) run(std::integral_constant<int, 1024>{});
    else run(std::integral_constant<int, 512>{});
}
template <typename T, bool PROBS>
void launch_masses_as(const RowSource& src, int pieces, int stride, double* mass, float* refs, hipStream_t stream) {
    hipLaunchKernelGGL((masses_kernel<T, PROBS>), dim3(static_cast<unsigned>((pieces + kWaves - 1) / kWaves) * src.rows), dim3(kThreads), 0, stream, Rows<T>(src), pieces, stride, mass, refs);
}

}  // namespace

// Slices of a tile at least, whose keys fit the row's candidates together.  How many: the chip holds four workgroups to a compute unit with the exponentials and five without, and
// works them off in rounds; a slice takes its tiles and about one more for its threshold, its list and its sums.
RowSlices choose_row_slices(int rows, int V, int dtype, int k, bool sums) {
    const long long tile = static_cast<long long>(kThreads) * kLoads * chunk_elements(dtype);
    const int tiles = static_cast<int>((static_cast<long long>(V) + chunk_elements(dtype) - 1 + tile - 1) / tile);       // wherever the row begins
    const int groups = tiles * kLoads, most = std::min(std::min(kMaxSplits, kSelCap / k), tiles);     // groups: of 256 chunks
    const long long held = kComputeUnits * (sums ? 4 : 5);
    int best = 1;
    long long least = -1;
    for (int s = 1; s <= most; ++s) {
        const int each = (groups + s - 1) / s;
        const long long rounds = (static_cast<long long>(rows) * ((groups + each - 1) / each) + held - 1) / held, cost = rounds * (each + kLoads);
        if (least < 0 || cost < least) { least = cost; best = s; }
    }
    const int each = (groups + best - 1) / best;
    return RowSlices{(groups + each - 1) / each, each * kThreads};
}

// Whether a workgroup to a row takes less time than slices that a second launch joins: where the row is short (three tiles of 1024 threads), and where there are rows enough to occupy
// half the chip.  Measured, split against whole, us per call: one row of 32000 in float32 14.4, 11.2; 256 of them 17.5, 13.2; one of 128256 in bfloat16 14.1, 15.3, 64 of them 15.0, 15.9,
// 128 of them 18.5, 16.5, 256 of them 24.0, 21.5; of 151936 in float32 one 15.3, 21.3, 128 24.6, 25.6, 256 35.7, 34.0.
// As many threads as let all rows be read at the same time, 1024 to a compute unit, or, past 512 rows, 256, of which five workgroups fit: 1024 rows of 32000 in bfloat16 take 29.5
// in slices, 43.1 with 1024 threads, 27.0 with 512, 21.8 with 256; 320 rows 17.3, 20.4, 13.5, 14.8.
// Rows that 512 threads read in one tile are left to 512, whose barriers and repeated steps cost less: one row of 8192 in float32 takes 6.3 us with 512 and 7.8 with 1024 (kernel), of 16384
// 8.3 and 7.4; 256 rows of 8192 8.0 and 9.2.
bool draft_in_one(int rows, int V, int dtype) {
    return rows >= kComputeUnits / 2 || static_cast<long long>(V) <= 3ll * 1024 * kLoads * chunk_elements(dtype);
}

// The same for draws from whole rows.  Short: 32768 logits (their exponentials take longer than the read) or 65536 probabilities.  Measured, two launches against one, 4 draws a row, us per call: a row of
// 16384 logits in float32 9.8, 8.4, of 32768 10.0, 10.6, of 50021 10.8, 13.5, of 65536 in bfloat16 12.6, 16.1; of 65536 probabilities 9.4, 7.0, of 98304 9.3, 8.8.  192 rows and more: 203 of
// 50021 probabilities, 16 draws each, 13.8, 11.4; 203 of 128256 in bfloat16 28.9, 29.7, 256 of them 32.5, 30.2; 256 of 151936 in float32 41.9, 36.6.  More rows than compute units: with
// 512 threads 1024 rows of 16384 in float32 take 25.8, with 1024 threads 26.8, in two launches 26.5; 4096 of 2048 47.2, 55.5, 42.4.
bool draft_whole_in_one(int rows, int V, int dtype, bool probs) {
    return piece_count(V, dtype) <= kLdsPieces && (4 * rows >= 3 * kComputeUnits || V <= (probs ? 65536 : 32768));
}

void launch_rows(const RowSource& src, bool probs, bool sums, int k, int limit, RowSlices cut, const RowParts& out, hipStream_t stream) {
    if (probs) launch_rows_as<float, true, true>(src, k, limit, cut, out, stream);
    else if (src.dtype == GR_F32) sums ? launch_rows_as<float, false, true>(src, k, limit, cut, out, stream) : launch_rows_as<float, false, false>(src, k, limit, cut, out, stream);
    else if (src.dtype == GR_BF16) sums ? launch_rows_as<Bf16, false, true>(src, k, limit, cut, out, stream) : launch_rows_as<Bf16, false, false>(src, k, limit, cut, out, stream);
    else sums ? launch_rows_as<_Float16, false, true>(src, k, limit, cut, out, stream) : launch_rows_as<_Float16, false, false>(src, k, limit, cut, out, stream);
}

void launch_draft_rows(const RowSource& src, bool probs, int k, double tail_mass, const DraftOut& out, hipStream_t stream) {
    if (probs) launch_draft_rows_as<float, true>(src, k, tail_mass, out, stream);
    else if (src.dtype == GR_F32) launch_draft_rows_as<float, false>(src, k, 0.0, out, stream);
    else if (src.dtype == GR_BF16) launch_draft_rows_as<Bf16, false>(src, k, 0.0, out, stream);
    else launch_draft_rows_as<_Float16, false>(src, k, 0.0, out, stream);
}

void launch_draft_whole_rows(const RowSource& src, bool probs, int pieces, const DraftOut& out, hipStream_t stream) {
    if (probs) launch_draft_whole_rows_as<float, true>(src, pieces, out, stream);
    else if (src.dtype == GR_F32) launch_draft_whole_rows_as<float, false>(src, pieces, out, stream);
    else if (src.dtype == GR_BF16) launch_draft_whole_rows_as<Bf16, false>(src, pieces, out, stream);
    else launch_draft_whole_rows_as<_Float16, false>(src, pieces, out, stream);
}

void launch_masses(const RowSource& src, bool probs, int pieces, int stride, double* mass, float* refs, hipStream_t stream) {
    if (probs) launch_masses_as<float, true>(src, pieces, stride, mass, refs, stream);
    else if (src.dtype == GR_F32) launch_masses_as<float, false>(src, pieces, stride, mass, refs, stream);
    else if (src.dtype == GR_BF16) launch_masses_as<Bf16, false>(src, pieces, stride, mass, refs, stream);
    else launch_masses_as<_Float16, false>(src, pieces, stride, mass, refs, stream);
}

}  // namespace gr
