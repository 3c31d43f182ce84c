// Declarations shared by the operators beside the verification: drafts drawn from rows, beams selected and moved, pages of the cache.
#pragma once
#include <type_traits>

#include "gr_internal.h"

namespace gr {

struct Bf16 { unsigned short bits; };

// Rows of logits or probabilities as a call gives them: [rows, V] elements of `dtype` (GR_F32, GR_BF16, GR_F16), `stride` elements from one to the
// next.  temperature: one for every `per_temp` rows, or nullptr for 1.  scores, finished: of beams (nullptr: all rows are read).
struct RowSource {
    const void* x; int dtype; long long stride; int rows, V;
    const float* temperature; int per_temp;
    const float* scores; const unsigned char* finished;
};
template <typename T>
struct Rows {
    const T* x; long long stride; int V;
    const float* temperature; int per_temp;
    const float* scores; const unsigned char* finished;
    explicit Rows(const RowSource& s)
        : x(static_cast<const T*>(s.x)), stride(s.stride), V(s.V), temperature(s.temperature), per_temp(s.per_temp), scores(s.scores), finished(s.finished) {}
    __device__ __forceinline__ const T* row(int r) const { return x + static_cast<long long>(r) * stride; }
    __device__ __forceinline__ float temperature_of(int r) const { return temperature ? temperature[r / per_temp] : 1.f; }
    // a beam that has no candidates of its own row: not in use (score -inf), or finished
    __device__ __forceinline__ bool skip(int r) const {
        return (scores && scores[r] == -__builtin_inff()) || (finished && finished[r] != 0);
    }
};
// What the pass leaves of every slice of a row: keys [rows, kSelCap] (kSelCap / splits of each slice), how many, the sum, its reference, whether an entry is no logit (probability).
struct RowParts { unsigned long long* cand; int* count; double* sum; float* ref; int* bad; };
struct RowSlices { int splits, per; };                     // workgroups to a row, 16-byte chunks to a workgroup

// elements of a 16-byte chunk
constexpr int chunk_elements(int dtype) { return dtype == GR_F32 ? 4 : 8; }
RowSlices choose_row_slices(int rows, int V, int dtype, int k, bool sums);
// The k largest (1 <= k <= kMaxSupport) of every slice; or up to `limit` candidates with them; probs: rows of probabilities (float32) and their sums; sums: logits and the sums of their exponentials
void launch_rows(const RowSource& src, bool probs, bool sums, int k, int limit, RowSlices cut, const RowParts& out, hipStream_t stream);
// Sums by pieces, see masses_kernel; pieces of `piece_elements` entries, counted from the 16-byte boundary at or before the row's begin
constexpr int piece_elements(int dtype) { return 64 * 4 * chunk_elements(dtype); }
constexpr int piece_count(int V, int dtype) { return static_cast<int>((static_cast<long long>(V) + chunk_elements(dtype) - 1 + piece_elements(dtype) - 1) / piece_elements(dtype)); }
void launch_masses(const RowSource& src, bool probs, int pieces, int stride, double* mass, float* refs, hipStream_t stream);

// Drafts.  Of rows cut to their k largest: from what launch_rows left; of whole rows: from what launch_masses left.
struct DraftOut { const float* uniforms; int n; int* drafts; int* status; };
constexpr int kComputeUnits = 256;                        // of an MI355X
constexpr int kLdsPieces = 2048;                          // piece sums of a row that one workgroup reads
bool draft_in_one(int rows, int V, int dtype);
void launch_draft_rows(const RowSource& src, bool probs, int k, double tail_mass, const DraftOut& out, hipStream_t stream);
bool draft_whole_in_one(int rows, int V, int dtype, bool probs);
void launch_draft_whole_rows(const RowSource& src, bool probs, int pieces, const DraftOut& out, hipStream_t stream);
void launch_draft_topk(const RowSource& src, bool probs, int k, double tail_mass, RowSlices cut, const RowParts& in, const DraftOut& out, hipStream_t stream);
void launch_draft_whole(const RowSource& src, bool probs, int pieces, int stride, const double* mass, const float* refs, const DraftOut& out, hipStream_t stream);

// Beams.
struct BeamOut { float* scores; int* parent; int* token; unsigned char* finished; int* status; };
void launch_beam_merge(const RowSource& src, int S, int K, int M, int eos, RowSlices cut, const RowParts& in, const BeamOut& out, hipStream_t stream);

// States that follow their beams, in bytes.  A row is a beam's states of one slice (an outer index and a head).
struct ReorderParams {
    unsigned char* state;
    long long outer, outer_stride, heads, head_stride, token_stride, token_bytes;
    long long row_stride;           // dense: from a beam to the next; paged: from a block to the next
    int S, K; long long tokens; int block;   // tokens of a row (paged: width * block); tokens of a block (dense: set by the launch)
    long long scale;                // what a token counts in `tokens` (set by the launch)
    const int* parent; const int* first; const int* length;
    const int* table; int width; int blocks;
};
bool launch_reorder(const ReorderParams& rp, hipStream_t stream);       // false: the kernel's counters do not hold such a row; nothing was launched

// Pages.
struct PageParams {
    const int* lengths; const int* new_lengths; int* table; int* free_blocks; const int* free_count;
    int R, width, block, pool; long long slots_capacity;
    int* out_lengths; int* out_free_count; int* starts; int* status; long long* slots;
};
hipError_t launch_pages(const PageParams& pp, hipStream_t stream);

// ---------------------------------------------------------------- device helpers
constexpr int kLoads = 4;                                 // 16-byte loads in flight per thread
static_assert(kLoads == piece_elements(GR_F32) / (64 * chunk_elements(GR_F32)), "a piece is what a wave reads");

template <typename T> struct Packed;                      // what a 16-byte load holds
template <> struct Packed<float> {
    static constexpr int N = 4;
    static __device__ __forceinline__ float get(const uint4& r, int j) { return __uint_as_float(j == 0 ? r.x : (j == 1 ? r.y : (j == 2 ? r.z : r.w))); }
    static __device__ __forceinline__ float one(float v) { return v; }
    static __device__ __forceinline__ unsigned bits(float v) { return __float_as_uint(v); }
    static constexpr unsigned kNoneBits = 0xFF800000u;    // -inf
};
template <> struct Packed<Bf16> {
    static constexpr int N = 8;
    static __device__ __forceinline__ float get(const uint4& r, int j) {
        const unsigned w = j < 2 ? r.x : (j < 4 ? r.y : (j < 6 ? r.z : r.w));
        return __uint_as_float((j & 1) ? (w & 0xFFFF0000u) : (w << 16));
    }
    static __device__ __forceinline__ float one(Bf16 v) { return __uint_as_float(static_cast<unsigned>(v.bits) << 16); }
    static __device__ __forceinline__ unsigned bits(Bf16 v) { return v.bits; }
    static constexpr unsigned kNoneBits = 0xFF80u;
};
template <> struct Packed<_Float16> {
    static constexpr int N = 8;
    static __device__ __forceinline__ float get(const uint4& r, int j) {
        const unsigned w = j < 2 ? r.x : (j < 4 ? r.y : (j < 6 ? r.z : r.w));
        const unsigned short h = static_cast<unsigned short>((j & 1) ? (w >> 16) : w);
        return static_cast<float>(__builtin_bit_cast(_Float16, h));
    }
    static __device__ __forceinline__ float one(_Float16 v) { return static_cast<float>(v); }
    static __device__ __forceinline__ unsigned bits(_Float16 v) { return __builtin_bit_cast(unsigned short, v); }
    static constexpr unsigned kNoneBits = 0xFC00u;
};
constexpr float kNone = -__builtin_inff();
constexpr float kMostFloat = 3.402823466e38f;
__device__ __forceinline__ bool good_temperature(float t) { return t > 0.f && t <= kMostFloat; }        // NaN: no
constexpr float kMostLogit = 1e37f;                       // a logit above it is a bad entry: so many of a thread's add up below infinity

// From here on the chunk's entries are unpacked again: one instruction each, where keeping them would cost a register each.
__device__ __forceinline__ void unpack_again(uint4& r) { asm volatile("" : "+v"(r.x), "+v"(r.y), "+v"(r.z), "+v"(r.w)); }

template <int CTRL>
__device__ __forceinline__ float dpp_move_f(float v) { return __int_as_float(dpp_move<CTRL>(__float_as_int(v))); }
// The largest (the sum) of N values that lie in N lanes side by side, again and again over the wave; N a power of two, 16 at most.
template <int N>
__device__ __forceinline__ float lanes_max_f(float v) {
    if (N > 1) v = fmaxf(v, dpp_move_f<kDppXor1>(v));
    if (N > 2) v = fmaxf(v, dpp_move_f<kDppXor2>(v));
    if (N > 4) v = fmaxf(v, dpp_move_f<kDppHalfMirror>(v));
    if (N > 8) v = fmaxf(v, dpp_move_f<kDppMirror>(v));
    return v;
}
template <int N>
__device__ __forceinline__ float lanes_sum_f(float v) {
    if (N > 1) v += dpp_move_f<kDppXor1>(v);
    if (N > 2) v += dpp_move_f<kDppXor2>(v);
    if (N > 4) v += dpp_move_f<kDppHalfMirror>(v);
    if (N > 8) v += dpp_move_f<kDppMirror>(v);
    return v;
}
// The largest and the smallest of a wave's values, the same in all lanes (as in gr_internal.h: no LDS round trips, all lanes active).  NaN is passed over.
__device__ __forceinline__ float wave_max_f(float v) {
    const int b = __float_as_int(lanes_max_f<16>(v));
    return fmaxf(fmaxf(__int_as_float(__builtin_amdgcn_readlane(b, 0)), __int_as_float(__builtin_amdgcn_readlane(b, 16))),
                 fmaxf(__int_as_float(__builtin_amdgcn_readlane(b, 32)), __int_as_float(__builtin_amdgcn_readlane(b, 48))));
}
__device__ __forceinline__ float wave_min_f(float v) { return -wave_max_f(-v); }

__device__ __forceinline__ double wave_scan_d(double v) {  // inclusive, all lanes active
    v += dpp_shift<0x111, 0xF>(v, 0.0);
    v += dpp_shift<0x112, 0xF>(v, 0.0);
    v += dpp_shift<0x114, 0xF>(v, 0.0);
    v += dpp_shift<0x118, 0xF>(v, 0.0);
    v += dpp_shift<0x142, 0xA>(v, 0.0);
    v += dpp_shift<0x143, 0xC>(v, 0.0);
    return v;
}


// A row as 16-byte chunks at 16-byte boundaries, wherever it begins: chunk c holds elements [c N - lead, c N - lead + N).  Chunks that reach
// over an end of the row are read element by element; entries outside it are -inf, of probabilities 0 (a -inf among them is a bad entry of the row's own).
template <typename T, bool PROBS>
struct RowChunks {
    static constexpr int N = Packed<T>::N;
    const T* row; int V, lead, chunks;
    __device__ __forceinline__ RowChunks(const T* r, int v) : row(r), V(v) {
        lead = static_cast<int>((reinterpret_cast<uintptr_t>(r) & 15) / sizeof(T));
        chunks = static_cast<int>((static_cast<long long>(v) + lead + N - 1) / N);
    }
    __device__ __forceinline__ bool inside(int c0, int c1) const {           // whether chunks c0 .. c1 - 1 lie in the row whole
        return (c0 > 0 || lead == 0) && static_cast<long long>(c1) * N - lead <= V;
    }
    __device__ __forceinline__ uint4 load(int c) const { return *reinterpret_cast<const uint4*>(row + (static_cast<long long>(c) * N - lead)); }
    // a chunk that may reach over an end of the row, or lie outside it
    __device__ __forceinline__ uint4 load_guarded(int c) const {
        if (inside(c, c + 1)) return load(c);
        unsigned w[4] = {};
#pragma unroll
        for (int j = 0; j < N; ++j) {
            const long long i = static_cast<long long>(c) * N - lead + j;
            w[j * 4 / N] |= ((i >= 0 && i < V) ? Packed<T>::bits(row[i]) : (PROBS ? 0u : Packed<T>::kNoneBits)) << (j * 32 * 4 / N % 32);
        }
        return make_uint4(w[0], w[1], w[2], w[3]);
    }
    // the same with a first chunk that all lanes share
    __device__ __forceinline__ uint4 load(int c0, unsigned at) const {
        const char* const first = reinterpret_cast<const char*>(row) + (static_cast<long long>(c0) * 16 - lead * static_cast<int>(sizeof(T)));
        return *reinterpret_cast<const uint4*>(first + at * 16u);
    }
    __device__ __forceinline__ int id(int c, int j) const { return static_cast<int>(static_cast<unsigned>(c) * N - lead + j); }
};

// 2^(y/256), |y| <= 256 * 700, added to sum: a table of 2^(j/256) in LDS and a polynomial of degree 2 in the rest, the best one for the relative error, 1.04e-10 either
// way; sums of many terms are nearer.  The whole part is read off the low bits of y + 1.5 * 2^52; its multiple of 256 goes into the exponent by one addition, since
// the table's upper words have j 2^12 taken off.  Ten instructions behind the float64 argument and one read of the table.  (A table of 32 entries without bank conflicts
// and degree 3: 15.)  In two steps, so that several reads are on their way before the first is used.
// FINE: degree 3, 1.8e-14 either way with its last rounding, one operation more: for draws, whose borders are held to 1e-12 of the total.
constexpr int kExpEntries = 256;
constexpr double kExpMagic = 6755399441055744.0;         // 1.5 * 2^52
struct ExpPart { double rest, entry; int whole; };
__device__ __forceinline__ ExpPart exp2_256_begin(double y, const double* tab) {
    const double m = y + kExpMagic;
    ExpPart e;
    e.whole = __double2loint(m);
    e.entry = tab[e.whole & (kExpEntries - 1)];
    e.rest = y - (m - kExpMagic);
    return e;
}
// The same for y = x scale + shift with a whole shift, from shift + 1.5 * 2^52, which is exact: one operation less, and the rest is rounded once.
__device__ __forceinline__ ExpPart exp2_256_begin(double x, double scale, double shift_magic, const double* tab) {
    const double m = fma(x, scale, shift_magic);
    ExpPart e;
    e.whole = __double2loint(m);
    e.entry = tab[e.whole & (kExpEntries - 1)];
    e.rest = fma(x, scale, shift_magic - m);
    return e;
}
template <bool FINE = false>
__device__ __forceinline__ double exp2_256_end(const ExpPart& e, double sum) {
    double p;
    if (FINE) {
        p = fma(e.rest, 3.308302377575631e-09, 3.66556615675881e-06);
        p = fma(p, e.rest, 2.7076061740623904e-03);
        p = fma(p, e.rest, 0.9999999999999825);
    } else {
        p = fma(e.rest, 3.6655651770288774e-06, 2.7076067943688897e-03);
        p = fma(p, e.rest, 1.0000000000001048);
    }
    return fma(p, __hiloint2double(__double2hiint(e.entry) + (e.whole << 12), __double2loint(e.entry)), sum);
}
constexpr double kPerTemp = 369.32993046757463;           // 256 / ln 2
constexpr float kLowest = -175200.f, kHighest = 160000.f; // the y that exp2_256 takes, with room for the sums of its results; e^-474 is nothing to a sum
__device__ __forceinline__ void fill_exp_table(double* tab) {        // by 256 threads
    const double v = exp2(static_cast<double>(threadIdx.x) / kExpEntries);
    tab[threadIdx.x] = __hiloint2double(__double2hiint(v) - (threadIdx.x << 12), __double2loint(v));
}

// A wave's sum of exponentials: of exp((x - ref) / T), but for a factor near 1, ref the largest entry of its first tile that has any.  A later entry may lie above ref
// (float64 has room for e^433 of them) until that is used up; then the sum is brought to a new reference.
template <bool FINE = false>
struct ExpSum {
    double sum = 0.0, scale, shift = 0.0;                 // of 2^(place(x) / 256); scale: kPerTemp / T; shift: -ref * scale, rounded to a whole number
    float ref = kNone, floor = kNone, ceiling = kNone;    // floor: entries below it count as if they were e^-474 of the reference; above the ceiling there is no room
    bool plain = false;                                   // ref * scale is small enough for that
    __device__ __forceinline__ explicit ExpSum(double s) : scale(s) {}
    __device__ __forceinline__ void set(float r) {
        ref = r;
        shift = rint(-static_cast<double>(ref) * scale);
        plain = fabs(shift) < 3.0e7;                      // floor and ceiling are then off by 4 at most, as places
    }
    __device__ __forceinline__ double place(double x) const { return plain ? fma(x, scale, shift) : (x - static_cast<double>(ref)) * scale; }
    __device__ __forceinline__ void refer(float most) {
        // the same in all lanes, and known to be
        set(__int_as_float(__builtin_amdgcn_readfirstlane(__float_as_int(most))));
        plain = __builtin_amdgcn_readfirstlane(plain) != 0;
        // not below the lowest float: rounded to -inf, it would let masked entries into the arm for those at or above it
        floor = fmaxf(static_cast<float>(static_cast<double>(ref) + static_cast<double>(kLowest) / scale), -kMostFloat);
        // rounded down: the float above it may lie hundreds of temperatures further
        const double room = static_cast<double>(ref) + static_cast<double>(kHighest) / scale;
        ceiling = static_cast<float>(room);
        if (static_cast<double>(ceiling) > room) ceiling = __int_as_float(__float_as_int(ceiling) + (ceiling > 0.f ? -1 : 1));
    }
    // the sum as one of exp((x - to) / T), `to` not below ref
    __device__ __forceinline__ double rebased(float to, const double* tab) const {
        const double y = fmax(-place(static_cast<double>(to)), static_cast<double>(kLowest));
        return ref > kNone ? sum * exp2_256_end<FINE>(exp2_256_begin(y, tab), 0.0) : 0.0;
    }
    // from here on entries up to `most` (this lane's) come
    __device__ __forceinline__ void raise(float most, const double* tab) {
        if (__any(most > ceiling)) {
            most = wave_max_f(most);
            sum = rebased(most, tab);
            refer(most);
            sum *= exp2_256_end<FINE>(exp2_256_begin(place(static_cast<double>(ref)), tab), 0.0);
        }
    }
    // kEight entries per lane.  A NaN makes the sum NaN.  Where a wave meets an entry below the floor, and at temperatures below some 1e-5 of the largest entry, it takes the second arm, a
    // lane's entries one after the other: with every third logit masked, or at a temperature of 1e-4, 256 rows of 128256 in bfloat16 take 52 us for 35 (beams), 52 for 34 (draws).
    static constexpr int kEight = 8;
    __device__ __forceinline__ void add(const float* x, const double* tab) {
        float least = x[0];
#pragma unroll
        for (int i = 1; i < kEight; ++i) least = fminf(least, x[i]);
        if (plain && !__any(least < floor)) {
            const double shift_magic = shift + kExpMagic;
#pragma unroll
            for (int i0 = 0; i0 < kEight; i0 += 4) {                              // four table entries on their way: eight would spill
                ExpPart e[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) e[i] = exp2_256_begin(static_cast<double>(x[i0 + i]), scale, shift_magic, tab);
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int i = 0; i < 4; ++i) sum = exp2_256_end<FINE>(e[i], sum);
                __builtin_amdgcn_sched_barrier(0);
            }
        } else {
            // masked entries, lowest values, tiny temperatures
#pragma unroll 1
            for (int i = 0; i < kEight; ++i) {
                float v = x[0];
#pragma unroll
                for (int j = 1; j < kEight; ++j) v = i == j ? x[j] : v;
                const double upto = exp2_256_end<FINE>(exp2_256_begin(fmax(place(static_cast<double>(v)), static_cast<double>(kLowest)), tab), sum);
                sum = v == v ? upto : static_cast<double>(v);
            }
        }
    }
};

// The keys in LDS (CAP at most) cut to the k largest, in place; all threads call it.  Returns the key that they reach.
template <int CAP, int NT = kThreads>
__device__ __forceinline__ unsigned long long cut_keys(unsigned long long* keys, int* count, int c, int k, int* hist, int* pick) {
    const int tid = threadIdx.x;
    const unsigned long long theta = block_kth_largest<NT>(keys, c, k, hist, pick);
    unsigned long long mine[CAP / NT];
#pragma unroll
    for (int r = 0; r < CAP / NT; ++r) {
        const int i = tid + r * NT;
        mine[r] = i < c ? keys[i] : 0ull;
    }
    __syncthreads();
    if (tid == 0) *count = 0;
    __syncthreads();
#pragma unroll
    for (int r = 0; r < CAP / NT; ++r)
        if (mine[r] >= theta && mine[r] != 0ull) keys[atomicAdd(count, 1)] = mine[r];
    __syncthreads();
    return theta;
}


// Entries as they are counted in linear bins: logits as they are, probabilities by their bit pattern, about their logarithm (next to one of 0.9 the others would share a bin).  Rises with
// the entry; no entry, a negative one or NaN: -inf.  unbinned: a value not above those whose place is `t` or more.
template <bool PROBS>
__device__ __forceinline__ float binned(float v) { return !PROBS ? v : (v >= 0.f ? static_cast<float>(__float_as_int(v)) : kNone); }
template <bool PROBS>
__device__ __forceinline__ float unbinned(float t) { return !PROBS || t == kNone ? t : __int_as_float(max(0, static_cast<int>(t) - 64)); }   // patterns are rounded to 24 bits

// Not above any entry of bin `from` and those behind it, of 256 linear bins from lo to hi: the bin's lower edge, lowered by more than its roundings (a few 2^-24 of
// either addend); not below lo.
__device__ __forceinline__ float bin_edge(float lo, float hi, int from) {
    const float up = static_cast<float>(from) * ((hi - lo) / 255.f), edge = lo + up - 0x1p-20f * (fabsf(lo) + up);
    return edge > lo ? edge : lo;                         // NaN, too: lo
}

// The smallest and the largest of what the waves left in `edge`.
template <int NW>
__device__ __forceinline__ void join_edges(const float* edge, float& lo, float& hi) {
    const int at = threadIdx.x & (NW - 1);
    lo = -lanes_max_f<NW>(-edge[at]); hi = lanes_max_f<NW>(edge[NW + at]);
}

// Of c > k keys in LDS the largest ones, moved to its begin: at least k, at most `limit`; all threads call it.  Returns how many;
// `reach`: a value that at least k of all keys' entries reach.
// The keys go into 256 bins, linear over their range (entries are spread smoothly there: one round where digits of the bit pattern take three), and the
// bins from the top that hold k stay; where they hold more than `limit`, equal entries mostly, the radix selection finds the k.
template <int CAP, bool PROBS, int NT = kThreads>
__device__ __forceinline__ int thin_keys(unsigned long long* keys, int c, int k, int limit, int* hist, int* pick, float* edge, int* count, float* reach = nullptr) {
    constexpr int kNW = NT / 64;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    constexpr int kEach = CAP / NT;
    unsigned long long mine[kEach];
    const auto value = [](unsigned long long key) { return PROBS ? binned<true>(key_q(key)) : key_logit(key); };
    float lo = __builtin_inff(), hi = kNone;
#pragma unroll
    for (int r = 0; r < kEach; ++r) {
        const int i = tid + r * NT;
        mine[r] = i < c ? keys[i] : 0ull;
        if (i < c) { const float v = value(mine[r]); lo = fminf(lo, v); hi = fmaxf(hi, v); }
    }
    lo = wave_min_f(lo); hi = wave_max_f(hi);
    if (lane == 0) { edge[wave] = lo; edge[kNW + wave] = hi; }
    if (tid < 256) hist[tid] = 0;
    if (tid == 0) *count = 0;
    __syncthreads();
    join_edges<kNW>(edge, lo, hi);
    const float per = 255.f / (hi - lo);                  // infinite or 0 where all are equal, or some lie beyond float32 apart: the bins still rise with the entry
    const auto bin = [&](unsigned long long key) { return static_cast<int>(fminf(fmaxf((value(key) - lo) * per, 0.f), 255.f)); };   // NaN: 0
#pragma unroll
    for (int r = 0; r < kEach; ++r) if (mine[r] != 0ull) atomicAdd(&hist[bin(mine[r])], 1);
    __syncthreads();
    int in[4], tot = 0;                                   // every wave by itself: lane l owns bins 255-4l .. 252-4l
#pragma unroll
    for (int j = 0; j < 4; ++j) { in[j] = hist[255 - 4 * lane - j]; tot += in[j]; }
    const int incl = wave_scan_i(tot);
    int above = incl - tot, from = -1, left = 0;
    const bool mine_is = above < k && k <= incl;
    if (mine_is)
#pragma unroll
        for (int j = 0; j < 4; ++j) { above += in[j]; if (from < 0 && above >= k) { from = 255 - 4 * lane - j; left = above; } }
    const int owner = __ffsll(static_cast<unsigned long long>(__ballot(mine_is))) - 1;
    from = __builtin_amdgcn_readlane(from, owner); left = __builtin_amdgcn_readlane(left, owner);
    if (left > limit) {
        __syncthreads();
        const unsigned long long kth = cut_keys<CAP, NT>(keys, count, c, k, hist, pick);
        if (reach) *reach = unbinned<PROBS>(value(kth));
        return k;
    }
#pragma unroll
    for (int r = 0; r < kEach; ++r) if (mine[r] != 0ull && bin(mine[r]) >= from) keys[atomicAdd(count, 1)] = mine[r];
    __syncthreads();
    if (reach) *reach = unbinned<PROBS>(bin_edge(lo, hi, from));
    return left;
}

__device__ __forceinline__ unsigned long long read_lane64(unsigned long long v, int lane) {
    return static_cast<unsigned long long>(static_cast<unsigned>(__builtin_amdgcn_readlane(static_cast<int>(v >> 32), lane))) << 32 |
           static_cast<unsigned>(__builtin_amdgcn_readlane(static_cast<int>(v), lane));
}
// Calls use(R) with the number of registers, MOST at most, that hold `count` values in a wave's lanes, known at compile time: a branch per register and turn cost 20 cycles each.
template <int MOST, typename Use>
__device__ __forceinline__ void with_registers(int count, Use&& use) {
    if (count <= 64) use(std::integral_constant<int, 1>{});
    else if (count <= 128) use(std::integral_constant<int, 2>{});
    else if (count <= 192) use(std::integral_constant<int, 3>{});
    else if (MOST <= 4 || count <= 256) use(std::integral_constant<int, 4>{});
    else if (MOST <= 6 || count <= 384) use(std::integral_constant<int, MOST < 6 ? 4 : 6>{});
    else use(std::integral_constant<int, MOST < 6 ? 4 : MOST>{});
}

}  // namespace gr
