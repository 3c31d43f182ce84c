// One streaming pass over rows of logits or probabilities in float32, bfloat16 or float16: the k largest entries of every row slice and,
// where they are asked for, the sum of the row (probabilities) or of its exponentials (logits); and the sums of a row by pieces.
// It stands behind the drafts' draw (gr_draft.hip) and the beams' selection (gr_beam.hip).
//
// Bound: HBM, one read of the row.  Arithmetic per element: about 5 instructions for a selection alone, about 20 with a float64 exponential
// (float64 runs at the rate of unpacked float32 here), 0.83 us for a million elements and instruction on 32.8 million elements: for 16-bit
// rows the exponentials and the read take about the same time, so both have to overlap.
#include <algorithm>

#include "gr_paths.h"

namespace gr {

namespace {

constexpr int kRowCap = 1024;                             // candidate keys in LDS
constexpr int kListCap = 1024, kWaveList = kListCap / kWaves;         // chunks with candidates in LDS, a quarter to a wave

// Of the keys of a stretch of the row one that exactly k of them reach (0: no key).  Only slices with more entries at their threshold than LDS holds come
// here (rows of equal entries, rows that rise), so the stretch is read again for every digit, and a digit that a whole wave agrees on is counted once.
template <typename KeyAt>
__device__ __forceinline__ unsigned long long stretch_kth_largest(KeyAt key_at, int count, int k, int* hist, int* pick) {
    const int tid = threadIdx.x;
    unsigned long long prefix = 0;
    int need = k;
    for (int shift = 56; shift >= 0; shift -= 8) {
        hist[tid] = 0;
        __syncthreads();
        const unsigned long long mask = (shift == 56) ? 0ull : (~0ull << (shift + 8));
        for (int i = tid; i < count; i += kThreads) {
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

// A threshold that at least k of the entries reach (-inf: there are too few), from the largest entries `top` of the threads' chunks (kLoads each, different entries): about the k-th
// largest of them.  With 8192 entries to a tile 9 reach it for k = 8, 136 for k = 128, 290 for k = 256.  First a bound from below: of 64 (128, 256) groups of threads, k at
// least, the smallest of the groups' largest.  Then 256 linear bins from there to the largest entry.  All threads call it.
__device__ __forceinline__ float find_threshold(const float* top, int k, int* hist, float* group_max, float* edge) {
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    float most = top[0];
#pragma unroll
    for (int l = 1; l < kLoads; ++l) most = fmaxf(most, top[l]);
    float lo, hi = wave_max_f(most);
    __syncthreads();                                      // whoever reads what an earlier call left is done
    hist[tid] = 0;
    if (lane == 0) edge[kWaves + wave] = hi;
    group_max[tid] = most;
    __syncthreads();
    if (k <= 64) lo = wave_min_f(fmaxf(fmaxf(group_max[lane], group_max[lane + 64]), fmaxf(group_max[lane + 128], group_max[lane + 192])));
    else {
        lo = wave_min_f(k <= 128 ? fmaxf(most, group_max[tid ^ 128]) : most);
        if (lane == 0) edge[wave] = lo;
        __syncthreads();
        lo = fminf(fminf(edge[0], edge[1]), fminf(edge[2], edge[3]));
    }
    hi = fmaxf(fmaxf(edge[4], edge[5]), fmaxf(edge[6], edge[7]));
    if (!(lo > kNone)) return kNone;                      // the same for all threads
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
    return bin_edge(lo, hi, from);
}

// grid = (splits * rows), 256 threads.  Workgroup s of a row reads chunks [s * per, (s + 1) * per) of its row, tiles of 256 * kLoads chunks, the next
// tile's loads on their way while the present one is worked on, and no barrier between tiles but for the threshold of the first.
// The k largest: a chunk whose largest entry reaches the threshold goes, as it was loaded, to a list in LDS; the few on it are taken apart together at
// the end (in the order of tiles every one would cost all lanes of its wave the test of every entry: 81 us where this takes %ROWS%).
// Keys are 64 bits (entry, ~id).  After `refresh` tiles the list is worked off and the threshold rises to about the k-th key.
// A slice leaves at least its k largest, up to `limit` candidates.
// SUM: PROBS: the float64 sum of the slice.  Logits: the sum of exp((x - ref) / T) in float64, per wave with its own reference, joined at the end.  (The hardware's float32
// exponential, with the listed chunks in float64, was measured: %F32%, but sums good to 2e-8 only, which depend on how a row is cut.)
// Rows of beams that are not in use or finished are not read (Rows::skip).
// Four waves to a SIMD with the exponentials: for a fifth their loop spills (32 us become 37, 89 become 114).
template <typename T, bool PROBS, bool SUM>
__global__ __launch_bounds__(kThreads, SUM && !PROBS ? 4 : 5) void rows_kernel(const Rows<T> in, int k, int limit, int splits, int per, const RowParts out) {
    constexpr int N = Packed<T>::N, kTileChunks = kThreads * kLoads;
    constexpr bool kExp = SUM && !PROBS;
    __shared__ unsigned long long keys[kRowCap];
    __shared__ uint4 list[kListCap];
    __shared__ int list_chunk[kListCap];
    __shared__ int hist[256];
    __shared__ int pick[4];
    __shared__ int count, listed[kWaves];
    __shared__ float group_max[kThreads];
    __shared__ double red[kWaves];
    __shared__ float edge[2 * kWaves];
    __shared__ double tab[kExp ? kExpEntries : 1];

    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int row = blockIdx.x / splits, s = blockIdx.x - row * splits;
    if (in.skip(row)) return;
    const RowChunks<T> x(in.row(row), in.V);
    const int c_first = s * per, c_end = min(x.chunks, c_first + per);

    uint4 next[kLoads];
    const auto fetch = [&](int c0) {
        if (c0 + kTileChunks <= c_end && x.inside(c0, c0 + kTileChunks)) {
#pragma unroll
            for (int l = 0; l < kLoads; ++l) next[l] = x.load(c0, l * kThreads + tid);
        } else if (c0 < c_end)
#pragma unroll
            for (int l = 0; l < kLoads; ++l) {
                const int c = c0 + l * kThreads;
                if (c + kThreads <= c_end && x.inside(c, c + kThreads)) next[l] = x.load(c, tid);
                else if (c < c_end) next[l] = x.load_guarded(c + tid < c_end ? c + tid : x.chunks);
            }
    };
    fetch(c_first);
    int bad = 0;
    double scale = 1.0;
    if (kExp) {
        const float temp = in.temperature_of(row);
        if (!(temp > 0.f) || !(temp <= 3.0e38f)) bad = 1; else scale = kPerTemp / static_cast<double>(temp);
        fill_exp_table(tab);
    }
    if (tid == 0) count = 0;
    int mine_listed = 0;                                  // chunks on the wave's own quarter of the list
    __syncthreads();

    float theta = kNone;                                  // entries below it are no candidates
    bool over = false;                                    // more candidates than LDS holds
    double total = 0.0;
    ExpSum es(scale);
    const float least = PROBS ? 0.f : kNone;              // entries must lie above it
    const auto key_of = [](float v, int id) { return PROBS ? make_key(v, id) : make_key_logit(v, id); };
    // the list taken apart: its entries that reach the threshold become keys
    const auto work_off = [&]() {
        if (lane == 0) listed[wave] = mine_listed;
        mine_listed = 0;
        __syncthreads();
        int n[kWaves], upto_wave[kWaves], all = 0;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) { n[w] = listed[w]; over = over || n[w] > kWaveList; all += min(n[w], kWaveList); upto_wave[w] = all; }
#pragma unroll
        for (int r = 0; r < kListCap / kThreads; ++r) {
            // the i-th chunk of the four quarters one after the other
            const int i0 = tid + r * kThreads;
            const bool have = i0 < all;
            if (!__any(have)) break;
            int i = i0;
#pragma unroll
            for (int w = 1; w < kWaves; ++w) if (i0 >= upto_wave[w - 1]) i = w * kWaveList + i0 - upto_wave[w - 1];
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
                if (mask >> j & 1u) { if (slot < kRowCap) keys[slot] = key_of(Packed<T>::get(raw, j), x.id(chunk, j)); ++slot; }
        }
        __syncthreads();
        over = over || count > kRowCap;
    };

    // The first tile's threshold lies at about its k-th entry, give or take 1 / sqrt(k) of its rank, and a wave finds a quarter of them, give or take its root: six times that
    // much has room for so many tiles.  Later ones hold ever fewer candidates, so the stretches double.
    const float wave_k = 0.25f * static_cast<float>(k);
    int refresh = max(1, static_cast<int>(kWaveList / (wave_k + 6.f * sqrtf(wave_k) + 8.f))), tiles = 0;
    for (int c0 = c_first; c0 < c_end; c0 += kTileChunks) {
        uint4 now[kLoads];
#pragma unroll
        for (int l = 0; l < kLoads; ++l) now[l] = next[l];
        fetch(c0 + kTileChunks);
        const int loads = min(kLoads, (c_end - c0 + kThreads - 1) / kThreads);     // of the last tile maybe fewer
        // Entries outside the row are -inf.  Bad: NaN, +inf (logits), negative entries (probabilities).
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
                    bad |= static_cast<int>(!(v >= 0.f)) & static_cast<int>(v != kNone);
                    total += static_cast<double>(v == kNone ? 0.f : v);
                } else if (!kExp) probe += v;
            }
            most = fmaxf(most, top[l]);
            unpack_again(now[l]);
        }
        if (!PROBS && !kExp) bad |= static_cast<int>(!(probe < 3.0e38f));
        if (kExp) {
            bad |= static_cast<int>(most > 3.0e38f);
            es.raise(most, tab);
            if (es.ref == kNone) {
                // nothing but masked entries and NaN, which the maximum passes over
#pragma unroll
                for (int l = 0; l < kLoads; ++l)
#pragma unroll
                    for (int j = 0; j < N; ++j) { const float v = Packed<T>::get(now[l], j); bad |= static_cast<int>(l < loads) & static_cast<int>(v != v); }
            } else
#pragma unroll
                for (int l = 0; l < kLoads; l += ExpSum::kEight / N) {
                    if (l >= loads) continue;
                    float v[ExpSum::kEight];
#pragma unroll
                    for (int j = 0; j < ExpSum::kEight; ++j) v[j] = l + j / N < loads ? Packed<T>::get(now[l + j / N], j % N) : kNone;
                    es.add(v, tab);
                }
        }
        if (theta == kNone) theta = find_threshold(top, k, hist, group_max, edge);
        unsigned long long hit[kLoads];
        int hits = 0;
#pragma unroll
        for (int l = 0; l < kLoads; ++l) { hit[l] = __ballot(top[l] >= theta && top[l] > least); hits += __popcll(hit[l]); }
        if (hits != 0) {
            int slot = mine_listed;
#pragma unroll
            for (int l = 0; l < kLoads; ++l) {
                const int at = slot + __builtin_amdgcn_mbcnt_hi(static_cast<unsigned>(hit[l] >> 32), __builtin_amdgcn_mbcnt_lo(static_cast<unsigned>(hit[l]), 0u));
                if ((hit[l] >> lane & 1ull) && at < kWaveList) { list[wave * kWaveList + at] = now[l]; list_chunk[wave * kWaveList + at] = c0 + l * kThreads + tid; }
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
                thin_keys<kRowCap, PROBS>(keys, c, k, kRowCap / 2, hist, pick, edge, &count, &reach);
                theta = fmaxf(theta, reach);
            }
            __syncthreads();
        }
    }
    work_off();
    const int room = min(kSelCap / splits, limit);        // k at least
    unsigned long long* const to = out.cand + static_cast<size_t>(row) * kSelCap + s * (kSelCap / splits);
    int found = count;
    __syncthreads();
    if (over) {
        // the slice's k largest by themselves
        const long long e0 = max(0ll, static_cast<long long>(c_first) * N - x.lead), e1 = min(static_cast<long long>(x.V), static_cast<long long>(c_end) * N - x.lead);
        const auto slice_key = [&](int i) -> unsigned long long {
            const float e = Packed<T>::one(x.row[e0 + i]);
            return e > least ? key_of(e, static_cast<int>(e0 + i)) : 0ull;
        };
        const unsigned long long reach = stretch_kth_largest(slice_key, static_cast<int>(e1 - e0), k, hist, pick);
        if (tid == 0) count = 0;
        __syncthreads();
        for (int i = tid; i < static_cast<int>(e1 - e0); i += kThreads) {
            const unsigned long long key = slice_key(i);
            if (key >= reach && key != 0ull) keys[atomicAdd(&count, 1)] = key;
        }
        __syncthreads();
        found = k;
    } else if (found > room) found = thin_keys<kRowCap, PROBS>(keys, found, k, room, hist, pick, edge, &count);
    for (int i = tid; i < found; i += kThreads) to[i] = keys[i];
    // the waves' sums: of exponentials, to the largest of their references
    __syncthreads();
    if (kExp) bad |= static_cast<int>(!(es.sum == es.sum));
    const double wave_total = SUM ? wave_sum(kExp ? es.sum : total) : 0.0;
    const bool wave_bad = __any(bad != 0);
    if (lane == 0) { red[wave] = wave_total; edge[wave] = es.ref; pick[wave] = wave_bad; }
    __syncthreads();
    if (tid < kWaves) {
        // a lane to a wave's sum
        float ref = es.ref;
        double sum = red[tid];
        if (kExp) {
            es.ref = edge[tid]; es.sum = sum;
            ref = fmaxf(fmaxf(edge[0], edge[1]), fmaxf(edge[2], edge[3]));
            sum = es.rebased(ref, tab);
        }
        sum += __shfl_xor(sum, 1);
        sum += __shfl_xor(sum, 2);
        if (tid == 0) {
            const int at = row * splits + s;
            out.count[at] = found; out.bad[at] = pick[0] | pick[1] | pick[2] | pick[3];
            if (SUM) { out.sum[at] = sum; if (!PROBS) out.ref[at] = ref; }
        }
    }
}

// The sums of a row by pieces: a wave to 64 * kLoads chunks one after the other.  grid = (pieces / 4 * rows).  PROBS: sums of the entries; logits: sums of
// exp((x - ref) / T) with the piece's largest entry as ref.
template <typename T, bool PROBS>
__global__ __launch_bounds__(kThreads) void masses_kernel(const Rows<T> in, int pieces, int stride, double* __restrict__ mass, float* __restrict__ refs) {
    constexpr int N = Packed<T>::N;
    __shared__ double tab[PROBS ? 1 : kExpEntries];
    const int tid = threadIdx.x, lane = tid & 63, groups = (pieces + kWaves - 1) / kWaves, row = blockIdx.x / groups;
    const RowChunks<T> x(in.row(row), in.V);
    int bad = 0;
    double scale = 0.0;
    if (!PROBS) {
        const float temp = in.temperature_of(row);
        if (!(temp > 0.f) || !(temp <= 3.0e38f)) bad = 1; else scale = kPerTemp / static_cast<double>(temp);
        fill_exp_table(tab);
        __syncthreads();
    }
    const int piece = (blockIdx.x - row * groups) * kWaves + (tid >> 6);
    if (piece >= pieces) return;                          // whole waves
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
                bad |= static_cast<int>(!(v >= 0.f)) & static_cast<int>(v != kNone);
                sum += static_cast<double>(v == kNone ? 0.f : v);
            } else top = fmaxf(top, v);
        }
        unpack_again(r[l]);
    }
    float ref = 0.f;
    if (!PROBS) {
        bad |= static_cast<int>(top > 3.0e38f);
        ref = wave_max_f(top);
        if (ref > kNone && scale > 0.0) {
            ExpSum es(scale);
            es.refer(ref);
#pragma unroll
            for (int l = 0; l < kLoads; l += ExpSum::kEight / N) {
                float v[ExpSum::kEight];
#pragma unroll
                for (int j = 0; j < ExpSum::kEight; ++j) v[j] = Packed<T>::get(r[l + j / N], j % N);
                es.add(v, tab);
            }
            sum = es.sum;                                 // NaN if an entry is
        } else {
            // nothing but masked entries and NaN, which the maximum passes over
#pragma unroll
            for (int l = 0; l < kLoads; ++l)
#pragma unroll
                for (int j = 0; j < N; ++j) { const float v = Packed<T>::get(r[l], j); bad |= static_cast<int>(v != v); }
        }
    }
    sum = wave_sum(sum);
    const unsigned long long any_bad = __ballot(bad != 0);
    if (lane == 0) {
        const size_t at = static_cast<size_t>(row) * stride + piece;
        mass[at] = any_bad ? __builtin_nan("") : sum; refs[at] = ref;          // a bad entry makes the row's total NaN
    }
}

template <typename T, bool PROBS, bool SUM>
void launch_rows_as(const RowSource& src, int k, int limit, RowSlices cut, const RowParts& out, hipStream_t stream) {
    hipLaunchKernelGGL((rows_kernel<T, PROBS, SUM>), dim3(cut.splits * src.rows), dim3(kThreads), 0, stream, Rows<T>(src), k, limit, cut.splits, cut.per, out);
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
    const long long held = 256 * (sums ? 4 : 5);
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

void launch_rows(const RowSource& src, bool probs, bool sums, int k, int limit, RowSlices cut, const RowParts& out, hipStream_t stream) {
    if (probs) launch_rows_as<float, true, true>(src, k, limit, cut, out, stream);
    else if (src.dtype == GR_F32) sums ? launch_rows_as<float, false, true>(src, k, limit, cut, out, stream) : launch_rows_as<float, false, false>(src, k, limit, cut, out, stream);
    else if (src.dtype == GR_BF16) sums ? launch_rows_as<Bf16, false, true>(src, k, limit, cut, out, stream) : launch_rows_as<Bf16, false, false>(src, k, limit, cut, out, stream);
    else sums ? launch_rows_as<_Float16, false, true>(src, k, limit, cut, out, stream) : launch_rows_as<_Float16, false, false>(src, k, limit, cut, out, stream);
}

void launch_masses(const RowSource& src, bool probs, int pieces, int stride, double* mass, float* refs, hipStream_t stream) {
    if (probs) launch_masses_as<float, true>(src, pieces, stride, mass, refs, stream);
    else if (src.dtype == GR_F32) launch_masses_as<float, false>(src, pieces, stride, mass, refs, stream);
    else if (src.dtype == GR_BF16) launch_masses_as<Bf16, false>(src, pieces, stride, mass, refs, stream);
    else launch_masses_as<_Float16, false>(src, pieces, stride, mass, refs, stream);
}

}  // namespace gr
