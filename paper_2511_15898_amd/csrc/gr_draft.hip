// The drafts of a row: n independent draws from the draft distribution cut to its k largest entries (App. "Top-k Sampling for the Relaxed OTLP"),
// or from the whole row, by inverse CDF over ascending token ids, one uniform per draw.  Masses and their sums are float64: a draw is a whole
// number, and next to a border of the CDF float32 sums over 128256 tokens would move one in some thousands.
//
// Bound: the streaming pass before these kernels.  What is left here is a chain of dependent steps on one workgroup per row (candidates, cut, order by id, sum,
// search), or, for whole rows, two reads per draw: the sums of the row's pieces, then the 1024 (float32) or 2048 entries of one piece.
#include "gr_paths.h"

namespace gr {

namespace {

struct DraftLds {
    unsigned long long keys[kSelCap];
    double mass[kMaxSupport + 64], sum[kMaxSupport + 64 + 1], tmp[kMaxSupport];
    int ids[kMaxSupport], sorted[kMaxSupport], hist[256], pick[4], count, keep;
};

// grid = (rows), 256 threads.
template <bool PROBS>
__global__ __launch_bounds__(kThreads) void draft_topk_kernel(const float* __restrict__ temperature, int k, double tail_mass, int splits, const RowParts in, const DraftOut out) {
    __shared__ DraftLds L;
    const int tid = threadIdx.x, row = blockIdx.x;
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
    gather_keys<kThreads>(L.keys, in.cand + static_cast<size_t>(row) * kSelCap, found, splits);
    if (tid == 0) L.count = 0;
    __syncthreads();
    const int total = found.total;
    unsigned long long theta = 0ull;
    if (total > k) theta = block_kth_largest(L.keys, total, k, L.hist, L.pick);
    int kk = min(total, k);
    for (int i = tid; i < total; i += kThreads) {
        const unsigned long long key = L.keys[i];
        if (key >= theta) {
            const int slot = atomicAdd(&L.count, 1);      // in any order: they are sorted by id below
            if (slot < kMaxSupport) { L.ids[slot] = key_id(key); L.tmp[slot] = static_cast<double>(PROBS ? key_q(key) : key_logit(key)); }
        }
    }
    __syncthreads();
    int id = tid < kk ? L.ids[tid] : 0x7FFFFFFF;
    double value = tid < kk ? L.tmp[tid] : 0.0;
    bool stay = tid < kk;
    if (PROBS && tail_mass > 0.0) {
        // the nucleus cut of gr_solve: by decreasing q (ties by id), up to the first token at which the running sum, added one after the other,
        // reaches (1 - tail_mass) of the row's mass
        int rank = 0;
        if (stay) for (int j = 0; j < kk; ++j) rank += static_cast<int>(L.tmp[j] > value) | (static_cast<int>(L.tmp[j] == value) & static_cast<int>(L.ids[j] < id));
        if (stay) L.mass[rank] = value;
        if (tid < 64) L.mass[kk + tid] = 0.0;
        __syncthreads();
        if (tid < 64) wave_sequential_scan_padded(L.mass, L.sum, kk, 0.0);
        if (tid == 0) L.keep = kk;
        __syncthreads();
        if (stay && L.sum[tid + 1] >= (1.0 - tail_mass) * found.qtot) atomicMin(&L.keep, tid + 1);
        __syncthreads();
        stay = stay && rank < L.keep;
        if (tid < kk && !stay) L.ids[tid] = 0x7FFFFFFF;   // behind every id that stays
        kk = L.keep;
        __syncthreads();
    }
    const int listed = min(total, k);
    if (!PROBS) {
        double most = stay ? value : -1e300;
        most = wave_max(most);
        if ((tid & 63) == 0) L.sum[tid >> 6] = most;
        __syncthreads();
        most = fmax(fmax(L.sum[0], L.sum[1]), fmax(L.sum[2], L.sum[3]));
        value = exp((value - most) * inv_temp);
    }
    if (stay) {
        int rank = 0;
#pragma unroll 8
        for (int j = 0; j < listed; ++j) rank += static_cast<int>(L.ids[j] < id);
        L.sorted[rank] = id; L.mass[rank] = value;
    }
    if (tid < 64) L.mass[kk + tid] = 0.0;                 // behind the last: the scan reads up to a multiple of 64
    __syncthreads();
    if (tid < 64) wave_sequential_scan_padded(L.mass, L.sum, kk, 0.0);
    __syncthreads();
    if (tid < out.n) {
        const size_t at = static_cast<size_t>(row) * out.n + tid;
        const double t = static_cast<double>(out.uniforms[at]) * L.sum[kk];
        int lo = 0, hi = kk;                              // the first i with sum[i + 1] > t
        while (lo < hi) { const int mid = (lo + hi) / 2; if (L.sum[mid + 1] > t) hi = mid; else lo = mid + 1; }
        if (lo >= kk) for (lo = kk - 1; lo > 0 && !(L.mass[lo] > 0.0); --lo) {}
        out.drafts[at] = L.sorted[lo];
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
        float v[N];
        if (whole) {
            const uint4 r = x.load(c);
#pragma unroll
            for (int j = 0; j < N; ++j) v[j] = Packed<T>::get(r, j);
        } else x.load_guarded(c, v);
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
    if (probs) hipLaunchKernelGGL(draft_topk_kernel<true>, dim3(src.rows), dim3(kThreads), 0, stream, src.temperature, k, tail_mass, cut.splits, in, out);
    else hipLaunchKernelGGL(draft_topk_kernel<false>, dim3(src.rows), dim3(kThreads), 0, stream, src.temperature, k, 0.0, cut.splits, in, out);
}

void launch_draft_whole(const RowSource& src, bool probs, int pieces, int stride, const double* mass, const float* refs, const DraftOut& out, hipStream_t stream) {
    if (probs) launch_whole_as<float, true>(src, pieces, stride, mass, refs, out, stream);
    else if (src.dtype == GR_F32) launch_whole_as<float, false>(src, pieces, stride, mass, refs, out, stream);
    else if (src.dtype == GR_BF16) launch_whole_as<Bf16, false>(src, pieces, stride, mass, refs, out, stream);
    else launch_whole_as<_Float16, false>(src, pieces, stride, mass, refs, out, stream);
}

}  // namespace gr
