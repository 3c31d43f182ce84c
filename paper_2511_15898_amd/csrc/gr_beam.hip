// Beams: the choice of the best continuations of a sequence's beams, and the states that follow their beams.
#include <algorithm>

#include "gr_paths.h"

namespace gr {

namespace {

constexpr int kMergeThreads = 512, kMergeWaves = kMergeThreads / 64, kMergeCap = 1024;
static_assert(GR_MAX_BEAMS * kMaxSplits <= 2048, "beam_of");
constexpr int kMaxLists = GR_MAX_BEAMS * kMaxSplits;
constexpr int kBatchKeys = kMergeWaves * GR_MAX_BEAMS;    // a wave to a slice's list, at most GR_MAX_BEAMS keys each
static_assert(kMergeCap >= GR_MAX_BEAMS + kBatchKeys, "a batch always has room behind the best ones");
constexpr double kNoScore = -__builtin_inf();

struct MergeLds {
    unsigned long long value[kMergeCap], key[kMergeCap];  // candidates: the score as a rising pattern, (logit, ~id)
    int beam[kMergeCap];
    int lists[kMaxLists];                                 // keys in the list of (beam, slice)
    double top[GR_MAX_BEAMS], log_sum[GR_MAX_BEAMS], score[GR_MAX_BEAMS];
    double best[kMergeThreads];
    double edge[kMergeWaves];
    int hist[256];
    int count, bad;
};

// The candidates in LDS cut to the best M, in order: by score, then the lower beam, then the larger logit, then the lower id.  A wave holds the scores of all in its lanes and
// takes an eighth of them in turn: its rank is the number of set bits of the comparison of all with it; where scores are equal, which 16-bit logits often are, the rest is
// compared the same way (one by one it took 44 us for 24 of 12 beams of 1139 in bfloat16).
__device__ __forceinline__ void keep_best(MergeLds& L, int c, int M) {
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    c = __builtin_amdgcn_readfirstlane(c);                // the same in all lanes, and known to be
    constexpr int kRegs = kMergeCap / 64;
    with_registers<kRegs>(c, [&](auto regs) {
        constexpr int R = decltype(regs)::value;
        unsigned long long v[R], k[R];
        int b[R], rank[R];
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const int i = r * 64 + lane;
            const bool have = i < c;
            v[r] = have ? L.value[i] : 0ull;              // 0: below every score
            k[r] = have ? L.key[i] : 0ull; b[r] = have ? L.beam[i] : 0;
        }
        int ties[R];
#pragma unroll
        for (int r = 0; r < R; ++r) {
            rank[r] = kMergeCap;                          // of the lane's own candidate, where it is the wave's turn
            ties[r] = 0;
#pragma unroll
            for (int turn = 0; turn < 64 / kMergeWaves; ++turn) {
                const int at = turn * kMergeWaves + wave;
                const unsigned long long mine = read_lane64(v[r], at);
                int before = 0, same = 0;
#pragma unroll
                for (int o = 0; o < R; ++o) { before += __popcll(__ballot(v[o] > mine)); same += __popcll(__ballot(v[o] == mine)); }
                rank[r] = lane == at ? before : rank[r];
                ties[r] |= mine != 0ull && same > 1 ? 1 << turn : 0;
            }
        }
#pragma unroll
        for (int r = 0; r < R; ++r)
            for (int left = __builtin_amdgcn_readfirstlane(ties[r]); left != 0; left &= left - 1) {
                const int at = (__ffs(left) - 1) * kMergeWaves + wave, my_beam = __builtin_amdgcn_readlane(b[r], at);
                const unsigned long long mine = read_lane64(v[r], at), my_key = read_lane64(k[r], at);
                int before = 0;
#pragma unroll
                for (int o = 0; o < R; ++o) before += __popcll(__ballot(v[o] == mine && (b[o] < my_beam || (b[o] == my_beam && k[o] > my_key))));
                rank[r] += lane == at ? before : 0;
            }
        __syncthreads();                                  // all have read
#pragma unroll
        for (int r = 0; r < R; ++r) if (rank[r] < M && v[r] != 0ull) { L.value[rank[r]] = v[r]; L.key[rank[r]] = k[r]; L.beam[rank[r]] = b[r]; }
    });
    if (tid == 0) L.count = min(c, M);
    __syncthreads();
}

// grid = (S), 512 threads.  score + (x - top) / T - log sum exp((x' - top) / T), in float64, of every candidate that the slices kept; a lower bound of the
// M-th best, from groups of threads, leaves some dozens, which are put in order by counting.
// Bound: a chain of steps behind one read.  What the slices left lies in other chips' L2, a microsecond away, so counts, sums and keys are all asked for at the
// beginning, keys before it is known how many there are (each list after the other took 25 us for 64 lists).
// 8.0 us for one sequence of 4 beams in 8 slices each, M = 4; 8.8 us for 32 sequences of 8 beams in 4 slices, M = 16, and for 64 of 10 in 3, M = 20.
// HELD: lists of a wave whose keys are on their way at once, and stay in registers if there are no more.
template <int HELD>
__global__ __launch_bounds__(kMergeThreads) void beam_merge_kernel(const Rows<float> in, int K, int M, int eos, int splits, int inverse, const RowParts parts, const BeamOut out) {
    __shared__ MergeLds L;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), seq = blockIdx.x;
    const int row0 = seq * K, lists = K * splits, room = kSelCap / splits, most = min(room, GR_MAX_BEAMS);
    const auto beam_of = [&](int list) { return (list * inverse) >> 16; };        // list / splits: inverse is 2^16 / splits, rounded up; exact below 2^11 lists
    // lanes take turns at being the first of a list, so that every group of lanes meets candidates
    const auto place = [&](int list) { return (lane + list * 13) & 63; };
    const auto load_key = [&](int list) -> unsigned long long {
        const int b = beam_of(list), i = place(list);
        return list < lists && i < most ? parts.cand[static_cast<size_t>(row0 + b) * kSelCap + (list - b * splits) * room + i] : 0ull;
    };
    unsigned long long held[HELD];                  // of lists wave, wave + 8, ..
#pragma unroll
    for (int u = 0; u < HELD; ++u) held[u] = load_key(wave + u * kMergeWaves);
    const float temp = in.temperature ? in.temperature[seq] : 1.f;
    const double inv_temp = 1.0 / static_cast<double>(temp);
    // a wave to a beam, a lane to a slice; of two beams everything is asked for at once
    constexpr int kTwo = 2;
    bool bad_beam = false;
    for (int b0 = wave; b0 < K; b0 += kTwo * kMergeWaves) {
        int n[kTwo], bad[kTwo]; float ref[kTwo], score[kTwo]; double sum[kTwo]; bool skip[kTwo];
#pragma unroll
        for (int u = 0; u < kTwo; ++u) {
            // of a beam that was not read, too: what lies there is the handle's and is not used
            const int b = min(b0 + u * kMergeWaves, K - 1), at = (row0 + b) * splits + min(lane, splits - 1);
            skip[u] = in.skip(row0 + b);
            score[u] = in.scores[row0 + b];
            n[u] = parts.count[at]; bad[u] = parts.bad[at]; ref[u] = parts.ref[at]; sum[u] = parts.sum[at];
        }
#pragma unroll
        for (int u = 0; u < kTwo; ++u) if (lane >= splits || skip[u]) { n[u] = 0; bad[u] = 0; ref[u] = kNone; sum[u] = 0.0; }
#pragma unroll
        for (int u = 0; u < kTwo; ++u) {
            const int b = b0 + u * kMergeWaves;
            if (b >= K) break;
            if (lane < splits) L.lists[b * splits + lane] = n[u];
            const double top = static_cast<double>(wave_max_f(ref[u]));
            const double total = wave_sum(ref[u] > kNone ? sum[u] * exp((static_cast<double>(ref[u]) - top) * inv_temp) : 0.0);
            bad_beam = bad_beam || __any(bad[u] != 0) || !(score[u] <= kMostFloat);
            if (lane == 0) { L.top[b] = top; L.log_sum[b] = log(total); L.score[b] = static_cast<double>(score[u]); }
        }
    }
    if (tid == 0) { L.count = 0; L.bad = 0; }
    __syncthreads();
    if (lane == 0 && (bad_beam || !good_temperature(temp))) L.bad = 1;       // any wave that sets it
    __syncthreads();
    const size_t at0 = static_cast<size_t>(seq) * M;
    if (L.bad) {
        for (int r = tid; r < M; r += kMergeThreads) {
            out.scores[at0 + r] = kNone; out.parent[at0 + r] = -1; out.token[at0 + r] = -1;
            if (out.finished) out.finished[at0 + r] = 0;
        }
        if (tid == 0) out.status[seq] = GR_ROW_BAD;
        return;
    }
    const auto candidate = [&](int list, unsigned long long key, double& value) -> bool {
        if (list >= lists || place(list) >= L.lists[list]) return false;
        const int b = beam_of(list);
        value = L.score[b] + ((static_cast<double>(key_logit(key)) - L.top[b]) * inv_temp - L.log_sum[b]);
        // to a multiple of 2^-35, a seventh of what the sums may be off by: sums of equal rows that were added up in another order meet again, so equal beams tie (but for one in thousands)
        value = rint(value * 0x1p35) * 0x1p-35;
        return true;
    };
    // Calls use(list, key, value) for every candidate.
    double scores_held[HELD];
    const bool all_held = lists <= HELD * kMergeWaves;
    const auto each = [&](bool again, auto&& use) {
        for (int l0 = 0; l0 < lists; l0 += HELD * kMergeWaves) {
            if (!all_held)
#pragma unroll
                for (int u = 0; u < HELD; ++u) held[u] = load_key(l0 + wave + u * kMergeWaves);
            if (!all_held || !again)
#pragma unroll
                for (int u = 0; u < HELD; ++u) if (!candidate(l0 + wave + u * kMergeWaves, held[u], scores_held[u])) scores_held[u] = kNoScore;
#pragma unroll
            for (int u = 0; u < HELD; ++u) if (scores_held[u] > kNoScore) use(l0 + wave + u * kMergeWaves, held[u], scores_held[u]);
        }
    };
    double mine = kNoScore;
    each(false, [&](int, unsigned long long, double value) { mine = fmax(mine, value); });
    // A bound of the M-th best from below, as in find_threshold (gr_rows.hip): of 64 groups of threads the smallest of the groups' best, then 256 linear bins from
    // there to the best of all for the threads' best: about M candidates reach the bin that holds the M-th of them.
    const double top = wave_max(mine);
    L.best[tid] = mine;
    if (lane == 0) L.edge[wave] = top;
    if (tid < 256) L.hist[tid] = 0;
    __syncthreads();
    double group = L.best[lane], hi = L.edge[0];
#pragma unroll
    for (int w = 1; w < kMergeWaves; ++w) { group = fmax(group, L.best[lane + 64 * w]); hi = fmax(hi, L.edge[w]); }
    double theta = wave_min(group);                       // -inf where some group has met none
    const float per = 255.f / static_cast<float>(hi - theta);                    // 0, infinite or NaN where theta is -inf or all are equal: then the bins say nothing
    const auto bin = [&](double value) { return static_cast<int>(fminf(fmaxf(static_cast<float>(value - theta) * per, 0.f), 255.f)); };       // rises with the score; NaN: 0
    if (mine > kNoScore && mine >= theta) atomicAdd(&L.hist[bin(mine)], 1);
    __syncthreads();
    int held_by[4], total = 0;                            // every wave by itself: lane l owns bins 255-4l .. 252-4l
#pragma unroll
    for (int j = 0; j < 4; ++j) { held_by[j] = L.hist[255 - 4 * lane - j]; total += held_by[j]; }
    const int incl = wave_scan_i(total);
    int above = incl - total, from = 0;
    const bool is_mine = above < M && M <= incl;
    if (is_mine)
#pragma unroll
        for (int j = 0; j < 4; ++j) { above += held_by[j]; if (from == 0 && above >= M) from = 255 - 4 * lane - j; }
    const unsigned long long owner = __ballot(is_mine);
    from = owner ? __builtin_amdgcn_readlane(from, __ffsll(owner) - 1) : 0;      // fewer threads than M have met any: all that reach theta
    const auto append = [&](double value, unsigned long long key, int b) {
        const int slot = atomicAdd(&L.count, 1);
        // plus 0.0: a score rounded to -0.0, or given as one, ties with 0.0
        if (slot < kMergeCap) { L.value[slot] = mono64(value + 0.0); L.key[slot] = key; L.beam[slot] = b; }
    };
    // a finished beam's one candidate
    const auto append_finished = [&]() {
        if (tid < K && in.finished && in.finished[row0 + tid] != 0 && L.score[tid] > kNoScore) append(L.score[tid], make_key_logit(0.f, eos), tid);
    };
    append_finished();
    each(true, [&](int list, unsigned long long key, double value) { if (value >= theta && bin(value) >= from) append(value, key, beam_of(list)); });
    __syncthreads();
    int c = L.count;
    if (c > kMergeCap) {
        // more than there is room for, equal scores for the most part: a batch of lists at a time behind the best so far
        __syncthreads();
        if (tid == 0) L.count = 0;
        __syncthreads();
        append_finished();
        for (int first = 0; first < lists; first += kMergeWaves) {
            __syncthreads();
            c = L.count;
            __syncthreads();
            if (c > kMergeCap - kBatchKeys) {
                keep_best(L, c, M);
                c = min(c, M);
                if (c == M) theta = fmax(theta, unmono64(L.value[M - 1]));
                __syncthreads();
            }
            const int list = first + wave;
            const unsigned long long key = load_key(list);
            double value;
            if (candidate(list, key, value) && value >= theta) append(value, key, beam_of(list));
        }
        __syncthreads();
        c = L.count;
    }
    __syncthreads();
    keep_best(L, c, M);
    c = min(c, M);
    for (int r = tid; r < M; r += kMergeThreads) {
        const bool have = r < c;
        const int token = have ? key_id(L.key[r]) : -1;
        out.scores[at0 + r] = have ? static_cast<float>(unmono64(L.value[r])) : kNone;
        out.parent[at0 + r] = have ? L.beam[r] : -1;
        out.token[at0 + r] = token;
        if (out.finished) out.finished[at0 + r] = have && token == eos;
    }
    if (tid == 0) out.status[seq] = GR_ROW_OK;
}

// ---------------------------------------------------------------- states

struct __attribute__((packed, aligned(1))) Any16 { unsigned w[4]; };   // 16 bytes wherever they lie (gfx950 loads and stores them in one instruction)

// The last unit of a stretch, 1 to 15 bytes of it.
struct __attribute__((packed, aligned(1))) Any8 { unsigned w[2]; };
struct __attribute__((packed, aligned(1))) Any4 { unsigned w; };
struct __attribute__((packed, aligned(1))) Any2 { unsigned short w; };
__device__ __forceinline__ Any16 load_part(const unsigned char* p, int bytes) {
    Any16 v = {};
    if (bytes & 8) { const Any8 x = *reinterpret_cast<const Any8*>(p); v.w[0] = x.w[0]; v.w[1] = x.w[1]; p += 8; }
    if (bytes & 4) { v.w[2] = reinterpret_cast<const Any4*>(p)->w; p += 4; }
    if (bytes & 2) { v.w[3] = reinterpret_cast<const Any2*>(p)->w; p += 2; }
    if (bytes & 1) v.w[3] |= static_cast<unsigned>(*p) << 16;
    return v;
}
__device__ __forceinline__ void store_part(unsigned char* p, int bytes, const Any16& v) {
    if (bytes & 8) { Any8 x; x.w[0] = v.w[0]; x.w[1] = v.w[1]; *reinterpret_cast<Any8*>(p) = x; p += 8; }
    if (bytes & 4) { reinterpret_cast<Any4*>(p)->w = v.w[2]; p += 4; }
    if (bytes & 2) { reinterpret_cast<Any2*>(p)->w = static_cast<unsigned short>(v.w[3]); p += 2; }
    if (bytes & 1) *p = static_cast<unsigned char>(v.w[3] >> 16);
}

// grid = (chunks of tokens, sequences, groups of slices), 256 threads; a slice is an (outer index, head).
// In place, so a beam may be read for one and written for another: a thread reads all that its 16 bytes of the beams need before it writes any, and no
// other thread touches them.  W: steps of 256 units that are in flight at once; N W loads per thread, 16 of them, fill the chip's memory pipes.
// Bound: HBM; every row that another beam takes is read from it once (a second taker finds it in L2), every row whose parent is another is written.  24 x 16 sequences of 8 rows of
// 256 KB: 234 us (5.1 TB/s); pages of 4 KB, about 450 MB moved: 96 us (4.7 TB/s); one sequence's 13 MB: 8.4 us, half of it the launch and the look-ups.
template <int N, int W>
__global__ __launch_bounds__(kThreads) void reorder_kernel(const ReorderParams rp, int per_group) {
    __shared__ long long from_row[N], to_row[N];
    __shared__ int moves_shared;
    const int tid = threadIdx.x, chunk = blockIdx.x, seq = blockIdx.y;
    // asked for together with the lengths
    const int row_asked = seq * rp.K + min(tid, rp.K - 1);
    const int parent_asked = rp.parent[row_asked], page_asked = rp.table ? rp.table[static_cast<long long>(row_asked) * rp.width + chunk] : 0;
    const long long t_first = static_cast<long long>(chunk) * rp.block;
    const long long len = rp.length ? rp.length[seq] * rp.scale : rp.tokens, lo = rp.first ? rp.first[seq] * rp.scale : 0;
    const long long t0 = max(max(lo, 0ll), t_first), t1 = min(min(len, rp.tokens), t_first + rp.block);
    if (t0 >= t1) return;
    if (tid < 64) {
        long long from = 0, to = 0;
        bool move = false;
        if (tid < rp.K) {
            const int row = row_asked, parent = parent_asked;
            move = parent >= 0 && parent < rp.K && parent != tid;
            if (move) {
                if (rp.table) {
                    const int a = rp.table[static_cast<long long>(seq * rp.K + parent) * rp.width + chunk], b = page_asked;
                    move = a != b && a >= 0 && a < rp.blocks && b >= 0 && b < rp.blocks;       // a page that the two share stays as it is
                    from = a * rp.row_stride; to = b * rp.row_stride;
                } else {
                    from = static_cast<long long>(seq * rp.K + parent) * rp.row_stride + t_first * rp.token_stride;
                    to = static_cast<long long>(row) * rp.row_stride + t_first * rp.token_stride;
                }
            }
        }
        const unsigned long long all = __ballot(move);
        if (move) { const int at = __popcll(all & ((1ull << tid) - 1ull)); from_row[at] = from; to_row[at] = to; }
        if (tid == 0) moves_shared = __popcll(all);
    }
    __syncthreads();
    const int moves = __builtin_amdgcn_readfirstlane(moves_shared);
    if (moves == 0) return;
    // the stretch of a row: `segments` tokens of seg bytes, one if they lie one after the other
    const bool joined = rp.token_stride == rp.token_bytes;
    const long long skip = (t0 - t_first) * rp.token_stride;
    const long long seg = joined ? (t1 - t0) * rp.token_bytes : rp.token_bytes;
    const int segments = joined ? 1 : static_cast<int>(t1 - t0);
    const int per_seg = static_cast<int>((seg + 15) / 16), units = per_seg * segments, rounds = (units + kThreads - 1) / kThreads;
    const unsigned heads = static_cast<unsigned>(rp.heads), q0 = blockIdx.z * static_cast<unsigned>(per_group);
    const int steps = min(per_group, static_cast<int>(static_cast<unsigned>(rp.outer) * heads - q0)) * rounds;
    for (int step = 0; step < steps; step += W) {
        long long off[W]; int bytes[W];
#pragma unroll
        for (int w = 0; w < W; ++w) {
            const int st = step + w, qi = st / rounds, u = (st - qi * rounds) * kThreads + tid;
            const unsigned q = q0 + qi, o = q / heads, h = q - o * heads;
            const int sg = segments == 1 ? 0 : u / per_seg, i = u - sg * per_seg;
            off[w] = o * rp.outer_stride + h * rp.head_stride + skip + sg * rp.token_stride + static_cast<long long>(i) * 16;
            bytes[w] = st < steps && u < units ? static_cast<int>(min(16ll, seg - static_cast<long long>(i) * 16)) : 0;
        }
        Any16 v[W][N];
#pragma unroll
        for (int m = 0; m < N; ++m)
            if (m < moves) {
                const long long from = from_row[m];
#pragma unroll
                for (int w = 0; w < W; ++w) {
                    const unsigned char* const p = rp.state + from + off[w];
                    if (bytes[w] == 16) v[w][m] = *reinterpret_cast<const Any16*>(p);
                    else if (bytes[w] > 0) v[w][m] = load_part(p, bytes[w]);
                }
            }
#pragma unroll
        for (int m = 0; m < N; ++m)
            if (m < moves) {
                const long long to = to_row[m];
#pragma unroll
                for (int w = 0; w < W; ++w) {
                    unsigned char* const p = rp.state + to + off[w];
                    if (bytes[w] == 16) *reinterpret_cast<Any16*>(p) = v[w][m];
                    else if (bytes[w] > 0) store_part(p, bytes[w], v[w][m]);
                }
            }
    }
}

}  // namespace

void launch_beam_merge(const RowSource& src, int S, int K, int M, int eos, RowSlices cut, const RowParts& in, const BeamOut& out, hipStream_t stream) {
    const auto run = [&](auto held) {
        hipLaunchKernelGGL(beam_merge_kernel<decltype(held)::value>, dim3(S), dim3(kMergeThreads), 0, stream, Rows<float>(src), K, M, eos, cut.splits, (65536 + cut.splits - 1) / cut.splits, in, out);
    };
    // As many as there are: of 12 lists 7.8 us with 2, 8.5 with 8, 9.0 with 16; of 100 11.5 with 16, 15.4 with 8, which asks twice, each time for all.
    const int lists = K * cut.splits;
    if (lists <= 2 * kMergeWaves) run(std::integral_constant<int, 2>{});
    else if (lists <= 4 * kMergeWaves) run(std::integral_constant<int, 4>{});
    else if (lists <= 8 * kMergeWaves) run(std::integral_constant<int, 8>{});
    else run(std::integral_constant<int, 16>{});
}

bool launch_reorder(const ReorderParams& params, hipStream_t stream) {
    // what a grid takes along x with 256 threads, and what the kernel counts in 32 bits: units of a chunk, steps of a workgroup
    constexpr long long kMostChunks = (1 << 24) - 1, kMostUnits = 1 << 30;
    ReorderParams rp = params;
    // heads that lie side by side in a token are part of it
    if (rp.heads > 1 && rp.head_stride == rp.token_bytes && rp.token_stride % rp.heads == 0 && rp.token_stride / rp.heads == rp.token_bytes) { rp.token_bytes = rp.token_stride; rp.heads = 1; rp.head_stride = 0; }
    const long long slices = rp.outer * rp.heads;
    if (rp.tokens == 1) rp.token_stride = rp.token_bytes;
    rp.scale = 1;
    if (!rp.table && rp.token_stride == rp.token_bytes) {
        // a dense row whose tokens lie one after the other is so many bytes
        rp.scale = rp.token_bytes;
        if (__builtin_mul_overflow(rp.tokens, rp.scale, &rp.tokens)) return false;
        rp.token_bytes = rp.token_stride = 1;
    }
    // a chunk of a dense row: 8 KB (of 16 rows of 4 MB: 236 us, with 4, 16 and 32 KB 244, 241 and 258)
    if (!rp.table) rp.block = static_cast<int>(std::min(std::max(1ll, 8192 / rp.token_bytes), rp.tokens));
    const long long chunks = (rp.tokens - 1) / rp.block + 1, segments = rp.token_stride == rp.token_bytes ? 1 : rp.block;      // segments: of a chunk, tokens that lie apart
    long long bytes, chunk_units;
    if (chunks > kMostChunks || __builtin_mul_overflow(rp.token_bytes, rp.block / segments, &bytes) || __builtin_mul_overflow((bytes - 1) / 16 + 1, segments, &chunk_units) ||
        chunk_units > kMostUnits)
        return false;
    // Slices to a workgroup, whose moves and table entries are looked up once: as many as fill the steps in flight (pages of 4 KB: 96 us with 4 slices, 101 with 8, 107 with 16), and the
    // chip wants some thousands of workgroups.
    const long long units = (static_cast<long long>(rp.block) * rp.token_bytes + 16 * kThreads - 1) / (16 * kThreads);
    long long per_group = std::max(1ll, 4 / units);
    per_group = std::min(per_group, std::max(1ll, std::min(slices, 65536ll) * chunks * rp.S / 4096));
    per_group = std::max(per_group, (slices + 65534) / 65535);
    if (per_group * ((chunk_units - 1) / kThreads + 1) > kMostUnits) return false;
    const dim3 grid(static_cast<unsigned>(chunks), rp.S, static_cast<unsigned>((slices + per_group - 1) / per_group));
    const int pg = static_cast<int>(per_group);
    if (rp.K <= 4) hipLaunchKernelGGL((reorder_kernel<4, 4>), grid, dim3(kThreads), 0, stream, rp, pg);
    else if (rp.K <= 8) hipLaunchKernelGGL((reorder_kernel<8, 2>), grid, dim3(kThreads), 0, stream, rp, pg);
    else if (rp.K <= 16) hipLaunchKernelGGL((reorder_kernel<16, 1>), grid, dim3(kThreads), 0, stream, rp, pg);
    else if (rp.K <= 32) hipLaunchKernelGGL((reorder_kernel<32, 1>), grid, dim3(kThreads), 0, stream, rp, pg);
    else hipLaunchKernelGGL((reorder_kernel<64, 1>), grid, dim3(kThreads), 0, stream, rp, pg);
    return true;
}

}  // namespace gr
