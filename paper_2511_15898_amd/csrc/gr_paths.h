// Declarations shared by the operators beside the verification: drafts drawn from rows, beams selected and moved, pages of the cache.
#pragma once
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
RowSlices choose_row_slices(int rows, int V, int dtype, int k);
// The k largest (1 <= k <= kMaxSupport) of every slice; probs: rows of probabilities (float32) and their sums; sums: logits and the sums of their exponentials
void launch_rows(const RowSource& src, bool probs, bool sums, int k, RowSlices cut, const RowParts& out, hipStream_t stream);
// Sums by pieces, see masses_kernel; pieces of `piece_elements` entries, counted from the 16-byte boundary at or before the row's begin
constexpr int piece_elements(int dtype) { return 64 * 4 * chunk_elements(dtype); }
constexpr int piece_count(int V, int dtype) { return static_cast<int>((static_cast<long long>(V) + chunk_elements(dtype) - 1 + piece_elements(dtype) - 1) / piece_elements(dtype)); }
void launch_masses(const RowSource& src, bool probs, int pieces, int stride, double* mass, float* refs, hipStream_t stream);

// Drafts.  Of rows cut to their k largest: from what launch_rows left; of whole rows: from what launch_masses left.
struct DraftOut { const float* uniforms; int n; int* drafts; int* status; };
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
void launch_reorder(const ReorderParams& rp, hipStream_t stream);

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
};
template <> struct Packed<Bf16> {
    static constexpr int N = 8;
    static __device__ __forceinline__ float get(const uint4& r, int j) {
        const unsigned w = j < 2 ? r.x : (j < 4 ? r.y : (j < 6 ? r.z : r.w));
        return __uint_as_float((j & 1) ? (w & 0xFFFF0000u) : (w << 16));
    }
    static __device__ __forceinline__ float one(Bf16 v) { return __uint_as_float(static_cast<unsigned>(v.bits) << 16); }
};
template <> struct Packed<_Float16> {
    static constexpr int N = 8;
    static __device__ __forceinline__ float get(const uint4& r, int j) {
        const unsigned w = j < 2 ? r.x : (j < 4 ? r.y : (j < 6 ? r.z : r.w));
        const unsigned short h = static_cast<unsigned short>((j & 1) ? (w >> 16) : w);
        return static_cast<float>(__builtin_bit_cast(_Float16, h));
    }
    static __device__ __forceinline__ float one(_Float16 v) { return static_cast<float>(v); }
};
constexpr float kNone = -__builtin_inff();

// A row as 16-byte chunks at 16-byte boundaries, wherever it begins: chunk c holds elements [c N - lead, c N - lead + N).  Chunks that reach
// over an end of the row are read element by element, entries outside it are -inf.
template <typename T>
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
    __device__ __forceinline__ void load_guarded(int c, float* v) const {
        if (inside(c, c + 1)) {
            const uint4 r = load(c);
#pragma unroll
            for (int j = 0; j < N; ++j) v[j] = Packed<T>::get(r, j);
            return;
        }
#pragma unroll
        for (int j = 0; j < N; ++j) {
            const long long i = static_cast<long long>(c) * N - lead + j;
            v[j] = (i >= 0 && i < V) ? Packed<T>::one(row[i]) : kNone;
        }
    }
    __device__ __forceinline__ int id(int c, int j) const { return static_cast<int>(static_cast<long long>(c) * N - lead + j); }
};

// 2^(y/32) for y <= 32 * 1000 (lower ones than -32 * 1000 count as that: 2^-1000 is nothing to any sum) from a table of 2^(j/32) in LDS and a
// polynomial of degree 4 in the rest, |rest| <= ln2/64: relative error 1.3e-12.  The whole part is read off the bits of y + 1.5 * 2^52.
// 64 lanes that read 32 doubles of LDS meet no bank conflict (64 banks), so the table costs one read.
__device__ __forceinline__ double exp2_32(double y, const double* tab) {
    constexpr double kMagic = 6755399441055744.0, kC = 6.93147180559945309417e-01 / 32.0;
    const double m = y + kMagic;
    const double r = y - (m - kMagic);
    const int whole = __double2loint(m);
    const double tv = tab[whole & 31];
    double p = fma(r, kC * kC * kC * kC / 24.0, kC * kC * kC / 6.0);
    p = fma(p, r, kC * kC / 2.0);
    p = fma(p, r, kC);
    p = fma(p, r, 1.0);
    const double scaled = __hiloint2double(__double2hiint(tv) + ((whole >> 5) << 20), __double2loint(tv));
    return p * scaled;
}
constexpr double kPerTemp = 46.166241308446828;           // 32 / ln 2
constexpr float kLowest = -21900.f, kHighest = 20000.f;   // 32 * log2 of the range that exp2_32 and the sums of its results keep, below 32 * 1000

// What a wave has of a sum of exponentials: exp((x - ref) / T), ref the largest entry of its first tile that has any.  A later entry may lie
// above ref (float64 has room for e^400 of them) until that is used up; then the sum is brought to a new reference.
struct ExpSum {
    double sum = 0.0; float ref = kNone;
    // from here on entries up to `most` (of the whole wave) come
    __device__ __forceinline__ void raise(float most, double scale) {
        if (most > ref && (ref == kNone || (static_cast<double>(most) - static_cast<double>(ref)) * scale > static_cast<double>(kHighest))) {
            sum *= exp((static_cast<double>(ref) - static_cast<double>(most)) * scale / kPerTemp);        // from -inf: 0
            ref = most;
        }
    }
};
// (x - ref first: exact, where a product with the scale would be rounded at the size of the lowest float)
__device__ __forceinline__ double exp_term(float v, double scale, double ref, const double* tab) {
    return exp2_32(fmax((static_cast<double>(v) - ref) * scale, static_cast<double>(kLowest)), tab);
}

}  // namespace gr
