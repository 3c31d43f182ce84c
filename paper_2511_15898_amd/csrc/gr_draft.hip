// The drafts of a row: n independent draws from the draft distribution cut to its k largest entries (App. "Top-k Sampling for the Relaxed OTLP"),
// or from the whole row, by inverse CDF over ascending token ids, one uniform per draw.  Masses and their sums are float64: a draw is a whole
// number, and next to a border of the CDF float32 sums over 128256 tokens would move one in some thousands.
//
// Few long rows come here, whose slices or pieces one launch reads and a second joins; short rows, and many, are drawn from where they are read (gr_rows.hip).
// Bound: the streaming pass before these kernels.  What is left here is a chain of dependent steps on one workgroup per row (candidates, cut, order by id, sum,
// search), or, for whole rows, two reads per draw: the sums of the row's pieces, then the 1024 (float32) or 2048 entries of one piece.
#include "gr_draft.h"

namespace gr {

namespace {

constexpr int kDraftThreads = 512;

// grid = (rows), 512 threads.  Bound: a chain of steps behind one read; counts, sums and keys of the slices lie in other chips' L2, a microsecond away, and are asked for together.
// 5.3 us for one row, k = 64.
template <bool PROBS>
__global__ __launch_bounds__(kDraftThreads) void draft_topk_kernel(const float* __restrict__ temperature, int k, double tail_mass, int splits, const RowParts in, const DraftOut out) {
    __shared__ DraftLds<kSelCap, kDraftThreads> L;
    const int tid = threadIdx.x, row = blockIdx.x, room = kSelCap / splits;
    // the keys are asked for before it is known how many there are: what lies behind them is the handle's, too, and is not used
    constexpr int kAhead = kSelCap / kDraftThreads;
    const unsigned long long* const cand = in.cand + static_cast<size_t>(row) * kSelCap;
    unsigned long long ahead[kAhead];
#pragma unroll
    for (int r = 0; r < kAhead; ++r) {
        const int i = r * kDraftThreads + tid;
        ahead[r] = i < splits * room ? cand[i] : 0ull;
    }
    const Uniforms<kDraftThreads> uniforms(out, row);
    const float t = PROBS ? 1.f : temperature[row];
    const SliceTotals found = slice_totals<false>(in.count, in.bad, in.sum, in.sum, nullptr, row, splits, 0.0);
    bool bad = found.bad != 0 || found.total == 0;
    double inv_temp = 1.0;
    if (PROBS) bad = bad || !(fabs(found.qtot - 1.0) <= 1e-3);
    else if (!good_temperature(t)) bad = true;
    else inv_temp = 1.0 / static_cast<double>(t);
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
    draw_from<PROBS>(L, found.total, k, tail_mass, found.qtot, inv_temp, uniforms, row, out);
}

// grid = (rows), a wave to a draw.  5.6 us for 203 rows of 50021 probabilities, 16 draws each.
template <typename T, bool PROBS>
__global__ __launch_bounds__(64 * GR_MAX_N) void draft_whole_kernel(const Rows<T> in, int pieces, int stride, const double* __restrict__ mass, const float* __restrict__ refs,
                                                                   const DraftOut out) {
    const int draw = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), row = blockIdx.x;
    draw_whole<T, PROBS>(in, row, draw, pieces, mass + static_cast<size_t>(row) * stride, refs + static_cast<size_t>(row) * stride, out);
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
