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

constexpr int kRowCap = 2048;                             // candidate keys in LDS
static_assert(kRowCap >= 2 * kMaxSupport && kRowCap <= kSelCap, "a tile that overflows adds k keys to at most k kept ones");

__device__ __forceinline__ float wave_max_f(float v) {
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) v = fmaxf(v, __shfl_xor(v, o));
    return v;
}
__device__ __forceinline__ float wave_min_f(float v) {
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) v = fminf(v, __shfl_xor(v, o));
    return v;
}

// The keys of a stretch of the row that reach `from`: one that exactly k of them reach.  Only tiles with thousands of entries at their threshold come
// here (rows of equal entries), so the stretch is read again for every digit, and a digit that a whole wave agrees on is counted once.
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

// The keys in LDS cut to the k largest, in place; all threads call it.  Returns the key that they reach.
__device__ __forceinline__ unsigned long long cut_keys(unsigned long long* keys, int* count, int c, int k, int* hist, int* pick) {
    const int tid = threadIdx.x;
    const unsigned long long theta = block_kth_largest(keys, c, k, hist, pick);
    unsigned long long mine[kRowCap / kThreads];
#pragma unroll
    for (int r = 0; r < kRowCap / kThreads; ++r) {
        const int i = tid + r * kThreads;
        mine[r] = i < c ? keys[i] : 0ull;
    }
    __syncthreads();
    if (tid == 0) *count = 0;
    __syncthreads();
#pragma unroll
    for (int r = 0; r < kRowCap / kThreads; ++r)
        if (mine[r] >= theta && mine[r] != 0ull) keys[atomicAdd(count, 1)] = mine[r];
    __syncthreads();
    return theta;
}


// grid = (splits * rows), 256 threads.  Workgroup s of a row reads chunks [s * per, (s + 1) * per) of its row, tiles of 256 * kLoads chunks, the next
// tile's loads on their way while the present one is worked on.
// The k largest: of the first tile every thread knows its largest entry; the threads form G groups, the smallest power of two >= k, and the
// smallest of the groups' largest entries is reached by at least k entries, so nothing below it is a candidate.  With 8192 entries to a tile about 22 reach
// it for k = 8 and 600 for k = 128.  Candidates go to LDS as 64-bit keys (entry, ~id); when there are many they are cut to the k largest by radix
// selection and the threshold rises.
// SUM: PROBS: the float64 sum of the slice.  Logits: the sum of exp((x - ref) / T), per wave with its own reference, joined at the end.
// Rows of beams that are not in use or finished are not read (Rows::skip).
template <typename T, bool PROBS, bool SUM>
__global__ __launch_bounds__(kThreads) void rows_kernel(const Rows<T> in, int k, int splits, int per, const RowParts out) {
    constexpr int N = Packed<T>::N, kTileChunks = kThreads * kLoads;
    __shared__ unsigned long long keys[kRowCap];
    __shared__ int hist[256];
    __shared__ int pick[4];
    __shared__ int count;
    __shared__ float group_max[kThreads];
    __shared__ double red[kWaves];
    __shared__ float wref[kWaves];
    __shared__ double tab[32];

    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int row = blockIdx.x / splits, s = blockIdx.x - row * splits;
    if (in.skip(row)) return;
    const RowChunks<T> x(in.row(row), in.V);
    const int c_first = s * per, c_end = min(x.chunks, c_first + per);
    int bad = 0;
    double scale = 0.0;
    if (SUM && !PROBS) {
        const float temp = in.temperature_of(row);
        if (!(temp > 0.f) || !(temp <= 3.0e38f)) bad = 1; else scale = kPerTemp / static_cast<double>(temp);
        if (tid < 32) tab[tid] = exp2(static_cast<double>(tid) / 32.0);
    }
    if (tid == 0) count = 0;
    __syncthreads();

    float theta = kNone;                                  // entries below it are no candidates, keys below theta_key neither
    unsigned long long theta_key = 0ull;
    ExpSum es;
    double total = 0.0;
    int held = 0;                                         // candidates of the tiles before
    const auto key_of = [](float v, int id) { return PROBS ? make_key(v, id) : make_key_logit(v, id); };

    uint4 now[kLoads], next[kLoads];
    bool whole = false;
    const auto fetch = [&](int c0, uint4* r) {
        whole = c0 + kTileChunks <= c_end && x.inside(c0, c0 + kTileChunks);
        if (whole)
#pragma unroll
            for (int l = 0; l < kLoads; ++l) r[l] = x.load(c0 + l * kThreads + tid);
    };
    fetch(c_first, next);
    for (int c0 = c_first; c0 < c_end; c0 += kTileChunks) {
        float v[kLoads * N];
        if (whole) {
#pragma unroll
            for (int l = 0; l < kLoads; ++l) now[l] = next[l];
            fetch(c0 + kTileChunks, next);                // may leave `whole` false for the next round
#pragma unroll
            for (int l = 0; l < kLoads; ++l)
#pragma unroll
                for (int j = 0; j < N; ++j) v[l * N + j] = Packed<T>::get(now[l], j);
        } else {
#pragma unroll
            for (int l = 0; l < kLoads; ++l) {
                const int c = c0 + l * kThreads + tid;
                if (c < c_end) x.load_guarded(c, v + l * N);
                else
#pragma unroll
                    for (int j = 0; j < N; ++j) v[l * N + j] = kNone;
            }
            fetch(c0 + kTileChunks, next);
        }
        // NaN, +inf (logits), negative entries (probabilities); entries outside the row are -inf
        float most = kNone, probe = 0.f;
#pragma unroll
        for (int i = 0; i < kLoads * N; ++i) {
            most = fmaxf(most, v[i]);
            if (PROBS) bad |= static_cast<int>(!(v[i] >= 0.f)) & static_cast<int>(v[i] != kNone);
            else probe += v[i];
        }
        if (!PROBS) bad |= static_cast<int>(!(probe < 3.0e38f));
        if (SUM && PROBS) {
#pragma unroll
            for (int i = 0; i < kLoads * N; ++i) total += static_cast<double>(v[i] == kNone ? 0.f : v[i]);
        }
        if (SUM && !PROBS) {
            es.raise(wave_max_f(most), scale);
            if (es.ref > kNone) {
                const double r = static_cast<double>(es.ref);
                double part = 0.0;
#pragma unroll
                for (int i = 0; i < kLoads * N; ++i) part += exp_term(v[i], scale, r, tab);
                es.sum += part;
            }
        }
        if (theta == kNone) {
            // the first tile's threshold (and the next ones', while there is none)
            float g;
            if (k <= 64) {
                int groups = 1;
                while (groups < k) groups *= 2;
                g = most;
                for (int o = 32; o >= groups; o >>= 1) g = fmaxf(g, __shfl_xor(g, o));
                group_max[tid] = g;
                __syncthreads();
                g = fmaxf(fmaxf(group_max[lane], group_max[lane + 64]), fmaxf(group_max[lane + 128], group_max[lane + 192]));
                theta = wave_min_f(g);
            } else {
                group_max[tid] = most;
                __syncthreads();
                g = k <= 128 ? fmaxf(most, group_max[tid ^ 128]) : most;
                g = wave_min_f(g);
                if (lane == 0) wref[wave] = g;
                __syncthreads();
                theta = fminf(fminf(wref[0], wref[1]), fminf(wref[2], wref[3]));
            }
            if (!(theta > kNone)) theta = kNone;          // too few entries, or NaN among them
        }
        const float least = PROBS ? 0.f : kNone;
#pragma unroll
        for (int l = 0; l < kLoads; ++l)
#pragma unroll
            for (int j = 0; j < N; ++j) {
                const float e = v[l * N + j];
                if (e >= theta && e > least) {
                    const unsigned long long key = key_of(e, x.id(c0 + l * kThreads + tid, j));
                    if (key >= theta_key) {
                        const int slot = atomicAdd(&count, 1);
                        if (slot < kRowCap) keys[slot] = key;
                    }
                }
            }
        __syncthreads();
        int c = count;
        __syncthreads();
        if (c > kRowCap) {
            // more than there is room for, equal entries for the most part: the tile's k largest by themselves
            const long long e0 = static_cast<long long>(c0) * N - x.lead;
            const int tile_end = min(c_end, c0 + kTileChunks);
            const auto tile_key = [&](int i) -> unsigned long long {
                const long long at = e0 + i;
                if (at < 0 || at >= x.V) return 0ull;
                const float e = Packed<T>::one(x.row[at]);
                if (!(e >= theta && e > least)) return 0ull;
                const unsigned long long key = key_of(e, static_cast<int>(at));
                return key >= theta_key ? key : 0ull;
            };
            const int entries = (tile_end - c0) * N;
            const unsigned long long reach = stretch_kth_largest(tile_key, entries, k, hist, pick);
            if (tid == 0) count = held;                   // its keys lie where they were
            __syncthreads();
            for (int i = tid; i < entries; i += kThreads) {
                const unsigned long long key = tile_key(i);
                if (key >= reach && key != 0ull) keys[atomicAdd(&count, 1)] = key;
            }
            __syncthreads();
            c = count;
            __syncthreads();
        }
        if (c > k && (c > kRowCap / 2 || c0 + kTileChunks >= c_end || c > 4 * k + 64)) {
            theta_key = cut_keys(keys, &count, c, k, hist, pick);
            theta = PROBS ? key_q(theta_key) : key_logit(theta_key);
            c = k;
        }
        held = c;                                         // kRowCap / 2 at most, so that k more have room
    }
    __syncthreads();
    const int room = kSelCap / splits, found = min(min(count, k), room);
    unsigned long long* const to = out.cand + static_cast<size_t>(row) * kSelCap + s * room;
    for (int i = tid; i < found; i += kThreads) to[i] = keys[i];
    double sum = 0.0;
    float ref = 0.f;
    if (SUM && PROBS) sum = block_sum(total, red);
    if (SUM && !PROBS) {
        if (lane == 0) wref[wave] = es.ref;
        __syncthreads();
        ref = fmaxf(fmaxf(wref[0], wref[1]), fmaxf(wref[2], wref[3]));
        const double mine = es.ref > kNone ? es.sum * exp((static_cast<double>(es.ref) - static_cast<double>(ref)) * scale / kPerTemp) : 0.0;
        sum = block_sum(mine, red);
    }
    const int any_bad = block_sum_i(bad, red);
    if (tid == 0) {
        const int at = row * splits + s;
        out.count[at] = found; out.bad[at] = any_bad;
        if (SUM) { out.sum[at] = sum; if (!PROBS) out.ref[at] = ref; }
    }
}

// The sums of a row by pieces: a wave to 64 * kLoads chunks one after the other.  grid = (pieces / 4 * rows).  PROBS: sums of the entries; logits: sums of
// exp((x - ref) / T) with the piece's largest entry as ref.
template <typename T, bool PROBS>
__global__ __launch_bounds__(kThreads) void masses_kernel(const Rows<T> in, int pieces, int stride, double* __restrict__ mass, float* __restrict__ refs) {
    constexpr int N = Packed<T>::N;
    __shared__ double tab[32];
    const int tid = threadIdx.x, lane = tid & 63, groups = (pieces + kWaves - 1) / kWaves, row = blockIdx.x / groups;
    const RowChunks<T> x(in.row(row), in.V);
    int bad = 0;
    double scale = 0.0;
    if (!PROBS) {
        const float temp = in.temperature_of(row);
        if (!(temp > 0.f) || !(temp <= 3.0e38f)) bad = 1; else scale = kPerTemp / static_cast<double>(temp);
        if (tid < 32) tab[tid] = exp2(static_cast<double>(tid) / 32.0);
        __syncthreads();
    }
    const int piece = (blockIdx.x - row * groups) * kWaves + (tid >> 6);
    if (piece >= pieces) return;                          // whole waves
    const int c0 = piece * 64 * kLoads;
    float v[kLoads * N];
    if (x.inside(c0, c0 + 64 * kLoads)) {
        uint4 r[kLoads];
#pragma unroll
        for (int l = 0; l < kLoads; ++l) r[l] = x.load(c0 + l * 64 + lane);
#pragma unroll
        for (int l = 0; l < kLoads; ++l)
#pragma unroll
            for (int j = 0; j < N; ++j) v[l * N + j] = Packed<T>::get(r[l], j);
    } else {
#pragma unroll
        for (int l = 0; l < kLoads; ++l) x.load_guarded(c0 + l * 64 + lane, v + l * N);
    }
    float most = kNone, probe = 0.f;
#pragma unroll
    for (int i = 0; i < kLoads * N; ++i) {
        most = fmaxf(most, v[i]);
        if (PROBS) bad |= static_cast<int>(!(v[i] >= 0.f)) & static_cast<int>(v[i] != kNone);
        else probe += v[i];
    }
    if (!PROBS) bad |= static_cast<int>(!(probe < 3.0e38f));
    double sum = 0.0;
    float ref = 0.f;
    if (PROBS) {
#pragma unroll
        for (int i = 0; i < kLoads * N; ++i) sum += static_cast<double>(v[i] == kNone ? 0.f : v[i]);
    } else {
        ref = wave_max_f(most);
        if (ref > kNone) {
            const double r = static_cast<double>(ref);
#pragma unroll
            for (int i = 0; i < kLoads * N; ++i) sum += exp_term(v[i], scale, r, tab);
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
void launch_rows_as(const RowSource& src, int k, RowSlices cut, const RowParts& out, hipStream_t stream) {
    hipLaunchKernelGGL((rows_kernel<T, PROBS, SUM>), dim3(cut.splits * src.rows), dim3(kThreads), 0, stream, Rows<T>(src), k, cut.splits, cut.per, out);
}
template <typename T, bool PROBS>
void launch_masses_as(const RowSource& src, int pieces, int stride, double* mass, float* refs, hipStream_t stream) {
    hipLaunchKernelGGL((masses_kernel<T, PROBS>), dim3(static_cast<unsigned>((pieces + kWaves - 1) / kWaves) * src.rows), dim3(kThreads), 0, stream, Rows<T>(src), pieces, stride, mass, refs);
}

}  // namespace

// About eight workgroups to a compute unit, slices of whole tiles, and the keys of a row's slices fit its candidates together.
RowSlices choose_row_slices(int rows, int V, int dtype, int k) {
    const long long tile = static_cast<long long>(kThreads) * kLoads * chunk_elements(dtype);
    const int tiles = static_cast<int>((static_cast<long long>(V) + chunk_elements(dtype) - 1 + tile - 1) / tile);       // wherever the row begins
    int s = std::max(1, 2048 / rows);
    s = std::min(std::min(s, kMaxSplits), std::min(kSelCap / k, tiles));
    const int each = (tiles + s - 1) / s;
    return RowSlices{(tiles + each - 1) / each, each * kThreads * kLoads};
}

void launch_rows(const RowSource& src, bool probs, bool sums, int k, RowSlices cut, const RowParts& out, hipStream_t stream) {
    if (probs) launch_rows_as<float, true, true>(src, k, cut, out, stream);
    else if (src.dtype == GR_F32) sums ? launch_rows_as<float, false, true>(src, k, cut, out, stream) : launch_rows_as<float, false, false>(src, k, cut, out, stream);
    else if (src.dtype == GR_BF16) sums ? launch_rows_as<Bf16, false, true>(src, k, cut, out, stream) : launch_rows_as<Bf16, false, false>(src, k, cut, out, stream);
    else sums ? launch_rows_as<_Float16, false, true>(src, k, cut, out, stream) : launch_rows_as<_Float16, false, false>(src, k, cut, out, stream);
}

void launch_masses(const RowSource& src, bool probs, int pieces, int stride, double* mass, float* refs, hipStream_t stream) {
    if (probs) launch_masses_as<float, true>(src, pieces, stride, mass, refs, stream);
    else if (src.dtype == GR_F32) launch_masses_as<float, false>(src, pieces, stride, mass, refs, stream);
    else if (src.dtype == GR_BF16) launch_masses_as<Bf16, false>(src, pieces, stride, mass, refs, stream);
    else launch_masses_as<_Float16, false>(src, pieces, stride, mass, refs, stream);
}

}  // namespace gr
