// The drafts of a row: n independent draws from the draft distribution cut to its k largest entries (App. "Top-k Sampling for the Relaxed OTLP"),
// or from the whole row, by inverse CDF over ascending token ids, one uniform per draw.  Masses and their sums are float64: a draw is a whole
// number, and next to a border of the CDF float32 sums over 128256 tokens would move one in some thousands.
//
// Bound: the streaming pass before these kernels.  What is left here is a chain of dependent steps on one workgroup per row (candidates, cut, order by id, sum,
// search), or, for whole rows, two reads per draw: the sums of the row's pieces, then the 1024 (float32) or 2048 entries of one piece.
#include "gr_paths.h"

namespace gr {

namespace {

constexpr int kDraftThreads = 512, kDraftWaves = kDraftThreads / 64;
constexpr int kPaddedSupport = 2 * kMaxSupport;           // candidates ranked at once, with what pads them to 8 `parts`; the scan's 64 behind a support

struct DraftLds {
    unsigned long long keys[kSelCap];
    double mass[kPaddedSupport], sum[kPaddedSupport + 1];
    int ids[kPaddedSupport], hist[256], pick[4], count;
    float edge[2 * kDraftWaves];
};

// grid = (rows), 512 threads.  The candidates are thinned to 512 at most, ranked by counting and so put in order, best first; a token's CDF is the sum of the
// masses of the tokens up to its id, added in that order whatever the slices' order was.  Sums of more masses in one order are never smaller, so the CDF
// rises with the id, and where nothing is added it stays the same: no sort by id and no scan is needed.
template <bool PROBS>
__global__ __launch_bounds__(kDraftThreads) void draft_topk_kernel(const float* __restrict__ temperature, int k, double tail_mass, int splits, const RowParts in, const DraftOut out) {
    __shared__ DraftLds L;
    const int tid = threadIdx.x, lane = tid & 63, row = blockIdx.x, room = kSelCap / splits;
    // the keys are asked for before it is known how many there are: what lies behind them is the handle's, too, and is not used
    constexpr int kAhead = kSelCap / kDraftThreads;
    const unsigned long long* const cand = in.cand + static_cast<size_t>(row) * kSelCap;
    unsigned long long ahead[kAhead];
#pragma unroll
    for (int r = 0; r < kAhead; ++r) {
        const int i = r * kDraftThreads + tid;
        ahead[r] = i < splits * room ? cand[i] : 0ull;
    }
    const SliceTotals found = slice_totals<false>(in.count, in.bad, in.sum, in.sum, nullptr, row, splits, 0.0);
    bool bad = found.bad != 0 || found.total == 0;
    double inv_temp = 1.0;
    if (PROBS) bad = bad || !(fabs(found.qtot - 1.0) <= 1e-3);
    else {
        const float t = temperature[row];
        if (!(t > 0.f) || !(t <= 3.0e38f)) bad = true; else inv_temp = 1.0 / static_cast<double>(t);
    }
    if (bad) {                                            // the same for all threads
        if (tid < out.n) out.drafts[static_cast<size_t>(row) * out.n + tid] = -1;
        if (tid == 0) out.status[row] = GR_ROW_BAD;
        return;
    }
#pragma unroll
    for (int r = 0; r < kAhead; ++r) {
        const int i = r * kDraftThreads + tid, s = min(i / room, splits - 1), at = i - s * room;
        const int count = __shfl(found.count, s), before = __shfl(found.before, s);
        if (at < count) L.keys[before + at] = ahead[r];   // at < room: i lies in slice s (behind the last one none counts)
    }
    __syncthreads();
    int c = found.total;
    if (c > 2 * k + 32 || c > kPaddedSupport) c = thin_keys<kSelCap, PROBS, kDraftThreads>(L.keys, c, k, kPaddedSupport, L.hist, L.pick, L.edge, &L.count);
    // `parts` threads to a candidate, side by side
    int parts = 1;
    while (parts < 64 && c * parts * 2 <= kDraftThreads) parts *= 2;
    const int me = tid / parts, part = tid % parts;
    const unsigned long long mine = me < c ? L.keys[me] : 0ull;
    // eight reads on their way at once: one after the other they cost 200 cycles each
    const int step = 8 * parts, padded = (c + step - 1) / step * step;
    for (int i = c + tid; i < padded; i += kDraftThreads) L.keys[i] = 0ull;
    __syncthreads();
    int rank = 0;
    for (int j = part; j < padded; j += step) {
        unsigned long long key[8];
#pragma unroll
        for (int u = 0; u < 8; ++u) key[u] = L.keys[j + u * parts];
#pragma unroll
        for (int u = 0; u < 8; ++u) rank += static_cast<int>(key[u] > mine);
    }
    for (int o = 1; o < parts; o <<= 1) rank += __shfl_xor(rank, o);
    __syncthreads();
    int kk = min(c, k);
    if (me < c && part == 0 && rank < kk) L.keys[rank] = mine;
    __syncthreads();
    if (PROBS && tail_mass > 0.0) {
        // the nucleus cut of gr_solve: up to the first token at which the running sum, added one after the other, reaches (1 - tail_mass) of the row's mass
        if (tid < kk) L.mass[tid] = static_cast<double>(key_q(L.keys[tid]));
        if (tid < 64) L.mass[kk + tid] = 0.0;             // the scan reads up to a multiple of 64
        if (tid == 0) L.count = kk;
        __syncthreads();
        if (tid < 64) wave_sequential_scan_padded(L.mass, L.sum, kk, 0.0);
        __syncthreads();
        if (tid < kk && L.sum[tid + 1] >= (1.0 - tail_mass) * found.qtot) atomicMin(&L.count, tid + 1);
        __syncthreads();
        kk = L.count;
    }
    for (int i = kk + tid; i < padded; i += kDraftThreads) { L.ids[i] = 0; L.mass[i] = 0.0; }
    if (tid < kk) {
        const unsigned long long key = L.keys[tid];
        L.ids[tid] = key_id(key);
        L.mass[tid] = PROBS ? static_cast<double>(key_q(key)) : exp((static_cast<double>(key_logit(key)) - static_cast<double>(key_logit(L.keys[0]))) * inv_temp);
    }
    __syncthreads();
    const int id = me < kk ? L.ids[me] : -1;
    double upto = 0.0;
    for (int j = part; j < padded; j += step) {
        int ids[8]; double mass[8];
#pragma unroll
        for (int u = 0; u < 8; ++u) { ids[u] = L.ids[j + u * parts]; mass[u] = L.mass[j + u * parts]; }
#pragma unroll
        for (int u = 0; u < 8; ++u) upto += ids[u] <= id ? mass[u] : 0.0;
    }
    for (int o = 1; o < parts; o <<= 1) upto += __shfl_xor(upto, o);
    if (me < kk && part == 0) L.sum[me] = upto;
    __syncthreads();
    // a wave to a draw: the total is the CDF of the largest id
    double total = 0.0;
    for (int i = lane; i < kk; i += 64) total = fmax(total, L.sum[i]);
    total = wave_max(total);
    for (int d = tid >> 6; d < out.n; d += kDraftWaves) {
        const size_t at = static_cast<size_t>(row) * out.n + d;
        const double t = static_cast<double>(out.uniforms[at]) * total;
        int first = 0x7FFFFFFF, last = -1;
        for (int i = lane; i < kk; i += 64) {
            if (L.sum[i] > t && L.mass[i] > 0.0) first = min(first, L.ids[i]);
            if (L.mass[i] > 0.0) last = max(last, L.ids[i]);
        }
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) { first = min(first, __shfl_xor(first, o)); last = max(last, __shfl_xor(last, o)); }
        if (lane == 0) out.drafts[at] = first == 0x7FFFFFFF ? last : first;
    }
    if (tid == 0) out.status[row] = GR_ROW_OK;
}

__device__ __forceinline__ double wave_scan_d(double v) {  // inclusive, all lanes active
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) { const double w = __shfl_up(v, o); if (lane >= o) v += w; }
    return v;
}

// grid = (rows), a wave to a draw.
template <typename T, bool PROBS>
__global__ __launch_bounds__(64 * GR_MAX_N) void draft_whole_kernel(const Rows<T> in, int pieces, int stride, const double* __restrict__ mass, const float* __restrict__ refs,
                                                                   const DraftOut out) {
    constexpr int N = Packed<T>::N;
    const int lane = threadIdx.x & 63, draw = threadIdx.x >> 6, row = blockIdx.x;
    const double* const m_row = mass + static_cast<size_t>(row) * stride;
    const float* const r_row = refs + static_cast<size_t>(row) * stride;
    const double inv_temp = PROBS ? 1.0 : 1.0 / static_cast<double>(in.temperature_of(row));
    double top = 0.0;
    if (!PROBS) {
        top = -1e300;
        for (int i = lane; i < pieces; i += 64) if (m_row[i] > 0.0) top = fmax(top, static_cast<double>(r_row[i]));
        top = wave_max(top);
    }
    const auto mass_of = [&](int i) -> double {
        if (i >= pieces) return 0.0;
        const double m = m_row[i];
        return PROBS || m == 0.0 ? m : m * exp((static_cast<double>(r_row[i]) - top) * inv_temp);
    };
    double total = 0.0;
    for (int i0 = 0; i0 < pieces; i0 += 64) total += wave_sum(mass_of(i0 + lane));
    const size_t at = static_cast<size_t>(row) * out.n + draw;
    if (!(total > 0.0) || (PROBS && !(fabs(total - 1.0) <= 1e-3))) {                // NaN: a bad entry or temperature
        if (lane == 0) out.drafts[at] = -1;
        if (threadIdx.x == 0) out.status[row] = GR_ROW_BAD;
        return;
    }
    const double target = static_cast<double>(out.uniforms[at]) * total;
    // the piece: the first whose running sum exceeds the target, or, where rounding leaves none, the last that has mass
    double base = 0.0, before = 0.0;
    int piece = -1, last = 0;
    for (int i0 = 0; i0 < pieces && piece < 0; i0 += 64) {
        const double m = mass_of(i0 + lane), upto = base + wave_scan_d(m);
        const unsigned long long over = __ballot(upto > target && m > 0.0), any = __ballot(m > 1e-290);
        if (any) last = i0 + 63 - __clzll(any);
        if (over) {
            const int at_lane = __ffsll(over) - 1;
            piece = i0 + at_lane;
            before = __shfl(upto - m, at_lane);
        }
        base = __shfl(upto, 63);
    }
    const bool found = piece >= 0;
    if (!found) piece = last;
    const double rest = found ? target - before : __builtin_inf();
    const RowChunks<T> x(in.row(row), in.V);
    const int c0 = piece * 64 * kLoads;
    const bool whole = x.inside(c0, c0 + 64 * kLoads);
    double done = 0.0;
    int token = -1, last_id = -1;
#pragma unroll
    for (int l = 0; l < kLoads; ++l) {
        const int c = c0 + l * 64 + lane;
        const uint4 r = whole ? x.load(c) : x.load_guarded(c);
        float v[N];
#pragma unroll
        for (int j = 0; j < N; ++j) v[j] = Packed<T>::get(r, j);
        double e[N], mine = 0.0;
#pragma unroll
        for (int j = 0; j < N; ++j) {
            e[j] = v[j] == kNone ? 0.0 : (PROBS ? static_cast<double>(v[j]) : exp((static_cast<double>(v[j]) - top) * inv_temp));
            mine += e[j];
            if (e[j] > 0.0) last_id = x.id(c, j);
        }
        const double upto = done + wave_scan_d(mine);
        const unsigned long long over = __ballot(upto > rest && mine > 0.0);
        if (over && token < 0) {
            const int at_lane = __ffsll(over) - 1;
            double run = upto - mine;
            int pick = -1;
#pragma unroll
            for (int j = 0; j < N; ++j) {
                run += e[j];
                if (pick < 0 && run > rest && e[j] > 0.0) pick = x.id(c, j);
            }
            token = __shfl(pick < 0 ? last_id : pick, at_lane);
        }
        done = __shfl(upto, 63);
    }
    if (token < 0) {                                      // rounding: the piece's last token of positive mass
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) last_id = max(last_id, __shfl_xor(last_id, o));
        token = last_id;
    }
    if (lane == 0) out.drafts[at] = token;
    if (threadIdx.x == 0) out.status[row] = GR_ROW_OK;
}

template <typename T, bool PROBS>
void launch_whole_as(const RowSource& src, int pieces, int stride, const double* mass, const float* refs, const DraftOut& out, hipStream_t stream) {
    hipLaunchKernelGGL((draft_whole_kernel<T, PROBS>), dim3(src.rows), dim3(64 * out.n), 0, stream, Rows<T>(src), pieces, stride, mass, refs, out);
}

}  // namespace

void launch_draft_topk(const RowSource& src, bool probs, int k, double tail_mass, RowSlices cut, const RowParts& in, const DraftOut& out, hipStream_t stream) {
    if (probs) hipLaunchKernelGGL(draft_topk_kernel<true>, dim3(src.rows), dim3(kDraftThreads), 0, stream, src.temperature, k, tail_mass, cut.splits, in, out);
    else hipLaunchKernelGGL(draft_topk_kernel<false>, dim3(src.rows), dim3(kDraftThreads), 0, stream, src.temperature, k, 0.0, cut.splits, in, out);
}

void launch_draft_whole(const RowSource& src, bool probs, int pieces, int stride, const double* mass, const float* refs, const DraftOut& out, hipStream_t stream) {
    if (probs) launch_whole_as<float, true>(src, pieces, stride, mass, refs, out, stream);
    else if (src.dtype == GR_F32) launch_whole_as<float, false>(src, pieces, stride, mass, refs, out, stream);
    else if (src.dtype == GR_BF16) launch_whole_as<Bf16, false>(src, pieces, stride, mass, refs, out, stream);
    else launch_whole_as<_Float16, false>(src, pieces, stride, mass, refs, out, stream);
}

}  // namespace gr
