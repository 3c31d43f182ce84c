// The drafts of a row from its candidates: put in order, cut, summed up by token id, drawn from.  Shared by the kernel that joins the slices of a row (gr_draft.hip) and the one that
// reads whole rows (gr_rows.hip).
#pragma once
#include "gr_paths.h"

namespace gr {

constexpr int kRanked = 512;                              // candidates put in order at once
constexpr int kSupportRegs = kMaxSupport / 64;

// CAP: candidates, in `keys`.
template <int CAP, int NT>
struct DraftLds {
    unsigned long long keys[CAP];
    unsigned long long best[kMaxSupport];                 // by decreasing key
    double mass[kMaxSupport + 64], sum[kMaxSupport + 64 + 1];
    int ids[kMaxSupport], place[kMaxSupport], hist[256], pick[4], count;       // by id: token, place in `best`
    float edge[2 * (NT / 64)];
};

// The uniforms of a wave's draws: asked for before the row is read, a microsecond that nobody waits for then.
template <int NT>
struct Uniforms {
    static constexpr int kNW = NT / 64, kMost = (GR_MAX_N + kNW - 1) / kNW;
    float of[kMost];
    __device__ __forceinline__ Uniforms(const DraftOut& out, int row) {
        const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
#pragma unroll
        for (int i = 0; i < kMost; ++i) of[i] = out.uniforms[static_cast<size_t>(row) * out.n + min(wave + i * kNW, out.n - 1)];
    }
};

// n independent draws from c candidates, c > 0, of which the k largest count, by inverse CDF over ascending token ids, one uniform per draw.  The candidates are thinned to 512
// at most and put in order, best first; the k best, or what the nucleus cut leaves of them, are put in order by id, and a wave that has their running sums in its lanes looks up a draw.
// In order without moving anything: every wave holds all candidates in its lanes and takes its share of them in turn, whose rank is the number of set bits of the comparison of all with it
// (reading all from LDS for each of them took 22 us for 128 candidates, eight reads at once 10; so 8).
// Masses and their sums are float64: a draw is a whole number, and next to a border of the CDF float32 sums would move some.
template <bool PROBS, int CAP, int NT>
__device__ __forceinline__ void draw_from(DraftLds<CAP, NT>& L, int c, int k, double tail_mass, double q_total, double inv_temp, const Uniforms<NT>& uniforms, int row, const DraftOut& out) {
    constexpr int kNW = NT / 64;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    if (c > 2 * k + 32 || c > kRanked) c = thin_keys<CAP, PROBS, NT>(L.keys, c, k, kRanked, L.hist, L.pick, L.edge, &L.count);
    c = __builtin_amdgcn_readfirstlane(c);                // the same in all lanes, and known to be: branches on it cost nothing
    int kk = min(c, k);
    with_registers<kRanked / 64>(c, [&](auto regs) {
        constexpr int R = decltype(regs)::value;
        unsigned long long key[R];
#pragma unroll
        for (int r = 0; r < R; ++r) key[r] = r * 64 + lane < c ? L.keys[r * 64 + lane] : 0ull;
#pragma unroll
        for (int r = 0; r < R; ++r) {
            int rank = kRanked;                           // of the lane's own candidate, where it is the wave's turn
#pragma unroll
            for (int turn = 0; turn < 64 / kNW; ++turn) {
                const int at = turn * kNW + wave;
                const unsigned long long mine = read_lane64(key[r], at);
                int before = 0;
#pragma unroll
                for (int o = 0; o < R; ++o) before += __popcll(__ballot(key[o] > mine));
                rank = lane == at ? before : rank;
            }
            if (rank < kk && r * 64 + lane < c) L.best[rank] = key[r];
        }
    });
    __syncthreads();
    if (PROBS && tail_mass > 0.0) {
        // the nucleus cut of gr_solve: up to the first token at which the running sum, added one after the other, reaches (1 - tail_mass) of the row's mass
        if (tid < kk) L.mass[tid] = static_cast<double>(key_q(L.best[tid]));
        if (tid < 64) L.mass[kk + tid] = 0.0;             // the scan reads up to a multiple of 64
        if (tid == 0) L.count = kk;
        __syncthreads();
        if (tid < 64) wave_sequential_scan_padded<16>(L.mass, L.sum, kk, 0.0);
        __syncthreads();
        if (tid < kk && L.sum[tid + 1] >= (1.0 - tail_mass) * q_total) atomicMin(&L.count, tid + 1);
        __syncthreads();
        kk = __builtin_amdgcn_readfirstlane(L.count);
        __syncthreads();
    }
    // a thread to a mass: with the order by id, which all waves work on, every wave would work out all exponentials (0.4 us)
    if (tid < kk) {
        const unsigned long long key = L.best[tid];
        L.mass[tid] = PROBS ? static_cast<double>(key_q(key)) : exp((static_cast<double>(key_logit(key)) - static_cast<double>(key_logit(L.best[0]))) * inv_temp);
    }
    with_registers<kSupportRegs>(kk, [&](auto regs) {
        constexpr int R = decltype(regs)::value;
        int id[R];
#pragma unroll
        for (int r = 0; r < R; ++r) id[r] = r * 64 + lane < kk ? key_id(L.best[r * 64 + lane]) : 0x7FFFFFFF;
#pragma unroll
        for (int r = 0; r < R; ++r) {
            int rank = kMaxSupport;
#pragma unroll
            for (int turn = 0; turn < 64 / kNW; ++turn) {
                const int at = turn * kNW + wave, mine = __builtin_amdgcn_readlane(id[r], at);
                int before = 0;
#pragma unroll
                for (int o = 0; o < R; ++o) before += __popcll(__ballot(id[o] < mine));
                rank = lane == at ? before : rank;
            }
            if (rank < kMaxSupport && r * 64 + lane < kk) { L.ids[rank] = id[r]; L.place[rank] = r * 64 + lane; }
        }
    });
    __syncthreads();
    // running sums: a lane has four tokens one after the other, or fewer
    const int per = (kk + 63) / 64, first = lane * per;
    double cdf[kSupportRegs], own = 0.0;
    unsigned any = 0u;
#pragma unroll
    for (int r = 0; r < kSupportRegs; ++r) {
        const double m = r < per && first + r < kk ? L.mass[L.place[first + r]] : 0.0;
        own += m;
        cdf[r] = own;
        any |= m > 0.0 ? 1u << r : 0u;
    }
    const double upto = wave_scan_d(own), before = upto - own;
    const double total = read_lane(upto, 63);
    const unsigned long long massive = __ballot(any != 0u);
#pragma unroll
    for (int i = 0; i < Uniforms<NT>::kMost; ++i) {
        const int d = wave + i * kNW;
        if (d >= out.n) break;
        const size_t at = static_cast<size_t>(row) * out.n + d;
        const double t = static_cast<double>(uniforms.of[i]) * total;
        int mine = -1;                                    // the lane's first token of some mass whose running sum exceeds t
#pragma unroll
        for (int r = kSupportRegs - 1; r >= 0; --r) if ((any >> r & 1u) && before + cdf[r] > t) mine = first + r;
        const unsigned long long over = __ballot(mine >= 0);
        // none: rounding at the end; the last token of some mass
        const int owner = over ? __ffsll(static_cast<unsigned long long>(over)) - 1 : 63 - __clzll(static_cast<long long>(massive));
        if (lane == owner) out.drafts[at] = L.ids[over ? mine : first + 31 - __clz(static_cast<int>(any))];
    }
    if (tid == 0) out.status[row] = GR_ROW_OK;
}

// Draw `draw` of a row from all its tokens, by the calling wave: m_row and r_row hold the sums of its pieces and their references.  The running sums of the pieces give the piece, those of
// its entries, read again, the token.
template <typename T, bool PROBS>
__device__ __forceinline__ void draw_whole(const Rows<T>& in, int row, int draw, int pieces, const double* m_row, const float* r_row, const DraftOut& out) {
    constexpr int N = Packed<T>::N;
    const int lane = threadIdx.x & 63;
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
        if (draw == 0 && lane == 0) out.status[row] = GR_ROW_BAD;
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
    const RowChunks<T, PROBS> x(in.row(row), in.V);
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
            e[j] = PROBS ? static_cast<double>(v[j]) : (v[j] == kNone ? 0.0 : exp((static_cast<double>(v[j]) - top) * inv_temp));
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
    if (draw == 0 && lane == 0) out.status[row] = GR_ROW_OK;
}

}  // namespace gr
