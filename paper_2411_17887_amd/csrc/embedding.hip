// Rows of an embedding table by token number, scaled, and the gradient of the table by sorted tokens.
//
//   lookup   : out[t] = scale * weight[id[t]]
//   gradient : d_weight[r] = scale * (sum of d_out[t] over the t with id[t] = r, in ascending order of t)
//              Few tokens: workgroups list those of their rows.  Many: the (id, t) pairs are sorted by id
//              (tcuscan_split_radix_sort_u32: stable, so t ascends within an id); a row's tokens then are one run of the sorted pairs.
//
// Sums are held in 32 bits, put together from parts in an order that the token numbers alone fix, and rounded once to the table's type.  Both move
// bytes and compute next to nothing.

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/tcuscan.h"
#include "chain_layout.h"
#include "element_types.h"
#include "wave_ops.h"

extern "C" void tcuscan_internal_workspace_reused(void *d_ws);                // tcuscan.hip

namespace {

constexpr int kThreads = 256;

struct LookupArgs {
    const void *ids, *weight;
    void *out, *ws;
    size_t n, vocab, dim, weight_stride, out_stride, slices;
    float scale;
    int wide_ids;
};

__device__ __forceinline__ long long id_at(const void *ids, int wide, size_t i)
{
    return wide ? ((const long long *)ids)[i] : (long long)((const int *)ids)[i];
}

// Columns of a row that one lane holds: a wavefront takes 64 * kLaneCols of them at a time.  ALIGNED: columns next to each other load and store as whole
// granules, eight of 16-bit types; where one of two types is fp32, two times four 256 columns apart, so that the fp32 side, too, moves 1 KiB of consecutive
// bytes an instruction (fp32 rows stored 32 bytes a lane: 45.5 -> 55 us for 65536 bf16 rows of 1024 looked up).  Otherwise a lane's columns are 64 apart,
// so that rows of any length and start load in runs of 64 elements.
template <int DG> constexpr int kLaneCols = DG == kF32 ? 4 : 8;
template <int DG, int DOTHER, bool ALIGNED> struct Lane {
    typedef typename Elem<DG>::T G;
    static constexpr int N = kLaneCols<DG>, kSlice = 64 * N, kGroup = DOTHER == kF32 ? 4 : N;
    template <class X> using VecOf = X __attribute__((ext_vector_type(N)));
    template <class X> using GroupOf = X __attribute__((ext_vector_type(kGroup)));
    typedef VecOf<G> Vec;
    static __device__ __forceinline__ size_t col(int lane, int k) { return ALIGNED ? (size_t)(k / kGroup) * 64 * kGroup + lane * kGroup + k % kGroup : (size_t)k * 64 + lane; }
    // Columns of `row` from c0 on; those from `dim` on are zeros.  (ALIGNED: dim is a multiple of N.)
    template <class X> static __device__ __forceinline__ VecOf<X> load(const X *row, size_t c0, size_t dim, int lane)
    {
        VecOf<X> v{};
        if constexpr (ALIGNED) {
#pragma unroll
            for (int k = 0; k < N; k += kGroup)
                if (c0 + col(lane, k) < dim) {
                    const GroupOf<X> g = *(const GroupOf<X> *)(row + c0 + col(lane, k));
#pragma unroll
                    for (int i = 0; i < kGroup; ++i) v[k + i] = g[i];
                }
        } else {
#pragma unroll
            for (int k = 0; k < N; ++k) v[k] = c0 + col(lane, k) < dim ? row[c0 + col(lane, k)] : (X)0.0f;
        }
        return v;
    }
    static __device__ __forceinline__ void add(float (&sum)[N], Vec v)
    {
#pragma unroll
        for (int k = 0; k < N; ++k) sum[k] += (float)v[k];
    }
    // The finished row: scaled, added to what is there or not, rounded.  AROUND: past the caches, for what is not read again soon.
    template <int DW, bool AROUND = false> static __device__ __forceinline__ void finish(typename Elem<DW>::T *row, size_t c0, size_t dim, int lane, const float (&sum)[N], float scale, bool accumulate)
    {
        typedef typename Elem<DW>::T W;
        if constexpr (ALIGNED) {
#pragma unroll
            for (int k = 0; k < N; k += kGroup) {
                if (c0 + col(lane, k) >= dim) continue;
                GroupOf<W> *p = (GroupOf<W> *)(row + c0 + col(lane, k)), w;
                const GroupOf<W> old = accumulate ? *p : GroupOf<W>{};
#pragma unroll
                for (int i = 0; i < kGroup; ++i) w[i] = (W)(accumulate ? fmaf(sum[k + i], scale, (float)old[i]) : sum[k + i] * scale);
                if constexpr (AROUND) __builtin_nontemporal_store(w, p);
                else *p = w;
            }
        } else {
#pragma unroll
            for (int k = 0; k < N; ++k) {
                const size_t c = c0 + col(lane, k);
                if (c < dim) row[c] = (W)(accumulate ? fmaf(sum[k], scale, (float)row[c]) : sum[k] * scale);
            }
        }
    }
};

// A wavefront takes a slice of the columns of kTokens tokens: their loads are on their way together.  (kTokens = 1: few tokens, whose columns are spread
// over as many wavefronts as there are.)  Bound by memory: 65536 bf16 rows of 1024 from an fp32 table (74 MB of it read, 134 MB written) take 44 us,
// 4.7 TB/s (streaming reaches 6.1 to 6.5); 24 rows of 2048 2.5 us, their loads one after the other: the number, the row.
template <int DW, int DO, bool ALIGNED, int kTokens> __global__ __launch_bounds__(kThreads) void lookup_kernel(LookupArgs A)
{
    typedef Lane<DW == kF32 ? DO : DW, DW == kF32 ? DW : DO, ALIGNED> L;       // (eight columns to a lane unless both types are fp32)
    typedef typename Elem<DW>::T W;
    const int lane = threadIdx.x & 63;
    const size_t item = (size_t)blockIdx.x * (kThreads / 64) + (threadIdx.x >> 6), t0 = item / A.slices * kTokens, c0 = item % A.slices * L::kSlice;
    if (t0 >= A.n) return;
    typename L::template VecOf<W> v[kTokens];
#pragma unroll
    for (int u = 0; u < kTokens; ++u) {
        v[u] = typename L::template VecOf<W>{};
        if (t0 + u >= A.n) break;
        const long long id = id_at(A.ids, A.wide_ids, t0 + u);
        if (id >= (long long)A.vocab) { if (c0 == 0 && lane == 0) raise_fault(A.ws, kFaultBadIndex); }
        else if (id >= 0) v[u] = L::template load<W>((const W *)A.weight + (size_t)id * A.weight_stride, c0, A.dim, lane);
    }
#pragma unroll
    for (int u = 0; u < kTokens; ++u) {
        if (t0 + u >= A.n) break;
        float f[L::N];
#pragma unroll
        for (int k = 0; k < L::N; ++k) f[k] = (float)v[u][k];
        L::template finish<DO, (kTokens > 1)>((typename Elem<DO>::T *)A.out + (t0 + u) * A.out_stride, c0, A.dim, lane, f, A.scale, false);
    }
}

struct GradArgs {
    const void *ids, *d_out;
    void *d_weight, *ws;
    uint32_t *keys, *tokens;
    float *partial;
    size_t n, vocab, dim, out_stride, weight_stride;
    long long padding;
    size_t slices, piece_groups, zero_groups, rows;      // rows: of the table to a workgroup, where there are few tokens
    float scale;
    int wide_ids, accumulate;
};

// The pairs to sort.  What takes no row of the table sorts behind all rows.
__global__ __launch_bounds__(kThreads) void token_keys_kernel(GradArgs A)
{
    const size_t t = (size_t)blockIdx.x * kThreads + threadIdx.x;
    if (t >= A.n) return;
    const long long id = id_at(A.ids, A.wide_ids, t);
    if (id >= (long long)A.vocab) raise_fault(A.ws, kFaultBadIndex);
    A.keys[t] = id < 0 || id >= (long long)A.vocab || id == A.padding ? (uint32_t)A.vocab : (uint32_t)id;
    A.tokens[t] = (uint32_t)t;
}

// Few tokens: no sort.  A workgroup takes `rows` rows of the table and a slice of the columns.  Each of its wavefronts looks an eighth of the token numbers over
// and lists those of its rows in order, then sums them row by row; a row that several eighths have is put together in LDS, in their order.
// One launch, whose time is that of its dependent steps: the numbers, a gradient's rows eight at a time, the table's row: 3001 tokens of 1000 numbers and
// 512 columns take 8 us, into 8000 rows of 515 14.  It grows with the tokens of the most frequent number, the sort and its launches do not: 4096 tokens take 15 us here and 30 there
// where 32000 numbers share them, 63 and 27 where all have the same (fp32, 512 columns); twice as many all the same would take 117 and 31.
constexpr int kFewTokens = 4096, kMaxFewRows = 64, kWaves = 8, kShare = kFewTokens / kWaves;
template <int DG, int DW, bool ALIGNED> __global__ __launch_bounds__(64 * kWaves) void few_tokens_kernel(GradArgs A)
{
    typedef Lane<DG, DW, ALIGNED> L;
    typedef typename L::G G;
    typedef typename Elem<DW>::T W;
    __shared__ uint32_t list[kWaves][kShare];      // (row of the workgroup) << 16 | token
    __shared__ uint64_t rows_of[kWaves];           // rows that a share of the tokens has
    __shared__ float part[kWaves][L::N * 64];
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const unsigned lane = threadIdx.x & 63;
    const size_t first = blockIdx.x / A.slices * A.rows, c0 = blockIdx.x % A.slices * L::kSlice;
    const size_t last = first + A.rows < A.vocab ? first + A.rows : A.vocab;
    int listed = 0;
    uint64_t mine = 0;
    {
        const size_t share = ((A.n + kWaves - 1) / kWaves + 63) & ~(size_t)63, begin = wave * share, end = begin + share < A.n ? begin + share : A.n;
        constexpr int kAhead = 8;
        for (size_t t0 = begin; t0 < end; t0 += 64 * kAhead) {
            long long id[kAhead];
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                const size_t t = t0 + 64 * u + lane;
                id[u] = t < end ? id_at(A.ids, A.wide_ids, t) : -1;
            }
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                if (blockIdx.x == 0 && id[u] >= (long long)A.vocab) raise_fault(A.ws, kFaultBadIndex);
                const bool in = id[u] >= (long long)first && id[u] < (long long)last && id[u] != A.padding;
                const uint64_t votes = __ballot(in);
                if (!votes) continue;
                const uint32_t row = (uint32_t)(id[u] - (long long)first);
                if (in) {
                    list[wave][listed + __popcll(votes & (((uint64_t)1 << lane) - 1))] = row << 16 | (uint32_t)(t0 + 64 * u + lane);
                    mine |= (uint64_t)1 << row;
                }
                listed += __popcll(votes);
            }
        }
    }
    const uint64_t has = (uint64_t)wave_or((uint32_t)(mine >> 32)) << 32 | wave_or((uint32_t)mine);
    if (lane == 0) rows_of[wave] = has;
    __syncthreads();
    uint64_t any = 0, several = 0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
        several |= any & rows_of[w];
        any |= rows_of[w];
    }
    W *const table = (W *)A.d_weight + first * A.weight_stride;
    auto sum_row = [&](int row, float (&sum)[L::N]) {          // of the wavefront's own list
        for (int i0 = 0; i0 < listed; i0 += 64) {
            const uint32_t item = i0 + lane < listed ? list[wave][i0 + lane] : 0xFFFFFFFFu;
            uint64_t votes = __ballot(item >> 16 == (uint32_t)row);
            while (votes) {
                constexpr int kAhead = 8;
                typename L::Vec v[kAhead];
#pragma unroll
                for (int u = 0; u < kAhead; ++u) {
                    v[u] = typename L::Vec{};
                    if (votes) v[u] = L::load((const G *)A.d_out + (size_t)(__builtin_amdgcn_readlane((int)item, __builtin_ctzll(votes)) & 0xFFFF) * A.out_stride, c0, A.dim, lane);
                    votes &= votes - 1;
                }
#pragma unroll
                for (int u = 0; u < kAhead; ++u) L::add(sum, v[u]);
            }
        }
    };
    const int rows = (int)(last - first);
    if (!A.accumulate) {                           // rows of none, all of them together
        const unsigned columns = (unsigned)(A.dim - c0 < L::kSlice ? A.dim - c0 : L::kSlice);
        if constexpr (ALIGNED) {
            typedef W Group __attribute__((ext_vector_type(L::kGroup)));
            const unsigned width = columns / L::kGroup;
            for (unsigned i = threadIdx.x; i < rows * width; i += 64 * kWaves) {
                const unsigned row = i / width;
                if (!(any >> row & 1)) *(Group *)(table + row * A.weight_stride + c0 + (i - row * width) * L::kGroup) = Group{};
            }
        } else {                                   // 16 bytes at a time between a row's first and last boundary of 16
            for (int row = wave; row < rows; row += kWaves) {
                if (any >> row & 1) continue;
                W *const to = table + (size_t)row * A.weight_stride + c0;
                constexpr unsigned kWide = 16 / sizeof(W);
                unsigned lead = (unsigned)(-(uintptr_t)to & 15) / sizeof(W);
                if (lead > columns) lead = columns;
                const unsigned wide = (columns - lead) / kWide, rest = lead + wide * kWide;
                if (lane < lead) to[lane] = W(0);
                for (unsigned i = lane; i < wide; i += 64) *(uint4 *)(to + lead + i * kWide) = uint4{};
                if (rest + lane < columns) to[rest + lane] = W(0);
            }
        }
    }
    for (uint64_t left = has & ~several; left; left &= left - 1) {        // rows of this share alone
        const int row = __builtin_ctzll(left);
        float sum[L::N] = {};
        sum_row(row, sum);
        L::template finish<DW>(table + (size_t)row * A.weight_stride, c0, A.dim, lane, sum, A.scale, A.accumulate);
    }
    for (uint64_t left = several; left; left &= left - 1) {
        const int row = __builtin_ctzll(left);
        float sum[L::N] = {};
        if (has >> row & 1) sum_row(row, sum);
        __syncthreads();                           // (the row before has been read)
#pragma unroll
        for (int k = 0; k < L::N; ++k) part[wave][k * 64 + lane] = sum[k];
        __syncthreads();
        if (row % kWaves != wave) continue;
#pragma unroll
        for (int k = 0; k < L::N; ++k) {
            sum[k] = part[0][k * 64 + lane];
#pragma unroll
            for (int w = 1; w < kWaves; ++w) sum[k] += part[w][k * 64 + lane];
        }
        L::template finish<DW>(table + (size_t)row * A.weight_stride, c0, A.dim, lane, sum, A.scale, A.accumulate);
    }
}

// Many tokens.  The sorted pairs are cut into pieces of 32 pairs, whatever runs they hold, so that a frequent token's run is shared by many
// wavefronts: a wavefront takes a piece and a slice of the columns.  Runs that lie inside a piece are finished there; what a piece has of
// a run that goes on beyond it is kept, in fp32, in one of the piece's two places (0: the run comes from the piece before, 1: it starts here)
// and added up, piece by piece in their order, by join_runs_kernel.  Every second workgroup, as long as both are left, writes zeros into rows that no token took.
// Bound by memory: 65536 bf16 gradients of 1024 columns into 65536 fp32 rows (134 MB read, 268 written) take 95 us, 4.2 TB/s, after a sort of 35.
constexpr int kPiece = 32, kZeroRows = 64;
template <int DG, int DW, bool ALIGNED> __global__ __launch_bounds__(kThreads) void sum_runs_kernel(GradArgs A)
{
    typedef Lane<DG, DW, ALIGNED> L;
    typedef typename L::G G;
    typedef typename Elem<DW>::T W;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    // pieces and rows to clear take turns, so that reading and writing go side by side
    const size_t both = A.piece_groups < A.zero_groups ? A.piece_groups : A.zero_groups, index = blockIdx.x < 2 * both ? blockIdx.x / 2 : blockIdx.x - both;
    if (blockIdx.x < 2 * both ? blockIdx.x & 1 : A.zero_groups > both) {
        __shared__ uint64_t taken;
        const size_t first = index * kZeroRows;
        if (wave == 0) {
            const uint32_t row = (uint32_t)first + lane;
            size_t lo = 0, hi = A.n;               // the first pair whose key is not below the row
            while (lo < hi) {
                const size_t mid = lo + (hi - lo) / 2;
                if (A.keys[mid] < row) lo = mid + 1; else hi = mid;
            }
            const uint64_t votes = __ballot(lo < A.n && A.keys[lo] == row);
            if (lane == 0) taken = votes;
        }
        __syncthreads();
        const float zeros[L::N] = {};
        for (int r = wave; r < kZeroRows && first + r < A.vocab; r += kThreads / 64)
            if (!(taken >> r & 1))
                for (size_t c0 = 0; c0 < A.dim; c0 += L::kSlice) L::template finish<DW>((W *)A.d_weight + (first + r) * A.weight_stride, c0, A.dim, lane, zeros, 0.0f, false);
        return;
    }
    const size_t item = index * (kThreads / 64) + wave, piece = item / A.slices, c0 = item % A.slices * L::kSlice;
    const size_t begin = piece * kPiece;
    if (begin >= A.n) return;
    const int count = (int)(begin + kPiece < A.n ? kPiece : A.n - begin);
    // lane i: the piece's i-th pair; lane 62: the key in front, 63: the one behind (none there: one that no pair has)
    const uint32_t none = 0xFFFFFFFFu;
    uint32_t key = none, token = 0;
    if (lane < count) { key = A.keys[begin + lane]; token = A.tokens[begin + lane]; }
    if (lane == 62 && begin > 0) key = A.keys[begin - 1];
    if (lane == 63 && begin + count < A.n) key = A.keys[begin + count];
    const uint32_t before = (uint32_t)__builtin_amdgcn_readlane((int)key, 62), behind = (uint32_t)__builtin_amdgcn_readlane((int)key, 63);
    float sum[L::N] = {};
    bool from_before = (uint32_t)__builtin_amdgcn_readlane((int)key, 0) == before;
    constexpr int kAhead = 8;
    for (int i0 = 0; i0 < count; i0 += kAhead) {
        typename L::Vec v[kAhead];
#pragma unroll
        for (int u = 0; u < kAhead; ++u)
            if (i0 + u < count) v[u] = L::load((const G *)A.d_out + (size_t)(uint32_t)__builtin_amdgcn_readlane((int)token, i0 + u) * A.out_stride, c0, A.dim, lane);
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            const int i = i0 + u;
            if (i >= count) break;
            const uint32_t row = (uint32_t)__builtin_amdgcn_readlane((int)key, i);
            L::add(sum, v[u]);
            const bool ends = i + 1 == count || (uint32_t)__builtin_amdgcn_readlane((int)key, i + 1) != row;
            if (!ends) continue;
            const bool goes_on = i + 1 == count && behind == row;
            if (row < A.vocab) {
                if (from_before || goes_on) {
                    float *p = A.partial + (2 * piece + (from_before ? 0 : 1)) * A.dim;
#pragma unroll
                    for (int k = 0; k < L::N; ++k)
                        if (c0 + L::col(lane, k) < A.dim) p[c0 + L::col(lane, k)] = sum[k];
                } else {
                    L::template finish<DW>((W *)A.d_weight + (size_t)row * A.weight_stride, c0, A.dim, lane, sum, A.scale, A.accumulate);
                }
            }
            from_before = false;
#pragma unroll
            for (int k = 0; k < L::N; ++k) sum[k] = 0.0f;
        }
    }
}

// The runs that lie in several pieces.  A workgroup looks at one piece and a slice of 64 VEC columns: if a run starts in it and goes on behind it, its wavefronts
// take the pieces that hold it in turns of consecutive ones, and the first of them adds the others' sums.  Most pieces have nothing to do here; the rest of the
// 14 us at 65536 tokens is the most frequent number's run.
constexpr int kJoinWaves = 4;
template <int DW, int VEC> __global__ __launch_bounds__(64 * kJoinWaves) void join_runs_kernel(GradArgs A)
{
    typedef typename Elem<DW>::T W;
    typedef float Vec __attribute__((ext_vector_type(VEC)));
    typedef W WVec __attribute__((ext_vector_type(VEC)));
    const size_t slices = (A.dim + 64 * VEC - 1) / (64 * VEC), piece = blockIdx.x / slices, behind = (piece + 1) * kPiece;
    if (behind >= A.n) return;
    const uint32_t row = A.keys[behind];
    if (A.keys[behind - 1] != row || row >= A.vocab) return;
    if (piece > 0 && A.keys[piece * kPiece] == row && A.keys[piece * kPiece - 1] == row) return;      // (the run started before)
    __shared__ size_t end;
    __shared__ Vec sums[kJoinWaves][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    if (threadIdx.x == 0) {
        size_t lo = behind, hi = A.n;              // the first pair behind the run
        while (lo < hi) {
            const size_t mid = lo + (hi - lo) / 2;
            if (A.keys[mid] <= row) lo = mid + 1; else hi = mid;
        }
        end = (lo - 1) / kPiece + 1;              // the piece behind the run's last
    }
    __syncthreads();
    const size_t count = end - piece, each = (count + kJoinWaves - 1) / kJoinWaves;
    const size_t from = piece + wave * each, to = from + each < end ? from + each : end, c = (blockIdx.x % slices * 64 + lane) * VEC;
    Vec sum = {};
    if (c < A.dim) {
        constexpr size_t kAhead = 8;
        for (size_t p = from; p < to; p += kAhead) {
            Vec v[kAhead];
#pragma unroll
            for (size_t u = 0; u < kAhead; ++u) {
                v[u] = Vec{};
                if (p + u < to) v[u] = *(const Vec *)(A.partial + (2 * (p + u) + (p + u == piece ? 1 : 0)) * A.dim + c);
            }
#pragma unroll
            for (size_t u = 0; u < kAhead; ++u) sum += v[u];
        }
    }
    sums[wave][lane] = sum;
    __syncthreads();
    if (wave != 0 || c >= A.dim) return;
#pragma unroll
    for (int w = 1; w < kJoinWaves; ++w) sum += sums[w][lane];
    WVec *to_row = (WVec *)((W *)A.d_weight + (size_t)row * A.weight_stride + c), x;
    const WVec old = A.accumulate ? *to_row : WVec{};
#pragma unroll
    for (int k = 0; k < VEC; ++k) x[k] = (W)(A.accumulate ? fmaf(sum[k], A.scale, (float)old[k]) : sum[k] * A.scale);
    *to_row = x;
}

// A kernel for two element types (checked before).
template <template <int, int> class Pick, int A> const void *pick_second(int b)
{
    return b == kF16 ? Pick<A, kF16>::fn() : b == kF32 ? Pick<A, kF32>::fn() : Pick<A, kBF16>::fn();
}
template <template <int, int> class Pick> const void *pick(int a, int b)
{
    return a == kF16 ? pick_second<Pick, kF16>(b) : a == kF32 ? pick_second<Pick, kF32>(b) : pick_second<Pick, kBF16>(b);
}
constexpr int kTokensAtOnce = 4;
template <int W, int O> struct Lookup { static const void *fn() { return (const void *)lookup_kernel<W, O, false, 1>; } };
template <int W, int O> struct LookupAligned { static const void *fn() { return (const void *)lookup_kernel<W, O, true, 1>; } };
template <int W, int O> struct LookupMany { static const void *fn() { return (const void *)lookup_kernel<W, O, false, kTokensAtOnce>; } };
template <int W, int O> struct LookupManyAligned { static const void *fn() { return (const void *)lookup_kernel<W, O, true, kTokensAtOnce>; } };
template <int G, int W> struct Few { static const void *fn() { return (const void *)few_tokens_kernel<G, W, false>; } };
template <int G, int W> struct FewAligned { static const void *fn() { return (const void *)few_tokens_kernel<G, W, true>; } };
template <int G, int W> struct Runs { static const void *fn() { return (const void *)sum_runs_kernel<G, W, false>; } };
template <int G, int W> struct RunsAligned { static const void *fn() { return (const void *)sum_runs_kernel<G, W, true>; } };

// What the gradient's workspace holds, in bytes from its start.
struct GradLayout {
    size_t chain, keys, keys_tmp, tokens, tokens_tmp, flags, positions, partial, all;
    GradLayout(size_t n, size_t dim)
    {
        const size_t words = (4 * n + 15) / 16 * 16;
        chain = tcuscan_workspace_bytes(1, n, TCUSCAN_I8_I32);          // what the sort asks for, in each of its forms
        if (chain < chain_layout::kHeaderBytes) chain = chain_layout::kHeaderBytes;
        keys = chain;
        if (n <= kFewTokens) { keys_tmp = tokens = tokens_tmp = flags = positions = partial = all = chain; return; }
        keys_tmp = keys + words;
        tokens = keys_tmp + words;
        tokens_tmp = tokens + words;
        positions = tokens_tmp + words;
        flags = positions + words;
        partial = (flags + n + 255) / 256 * 256;
        all = partial + 2 * ((n + kPiece - 1) / kPiece) * dim * 4;
    }
};

constexpr size_t kMostRows = 0x7FFFFFFFu;
// Wavefronts' items from which on each takes four tokens: 32768 bf16 rows of 512 take 10.0 us, one token at a time 11.7; below, either is as fast but for single
// tokens, which four at a time would give to one wavefront.
constexpr size_t kManyItems = 1 << 14;

}  // namespace

extern "C" {

tcuscan_status_t tcuscan_embedding(const void *d_ids, int id_bytes, size_t n, const void *d_weight, size_t vocab, size_t dim, size_t weight_stride,
                                   tcuscan_dtype_t weight_dt, void *d_out, size_t out_stride, tcuscan_dtype_t out_dt, float scale,
                                   void *d_ws, size_t ws_bytes, tcuscan_stream_t stream)
{
    const size_t we = elem_bytes(weight_dt), oe = elem_bytes(out_dt);
    if (!we || !oe || vocab > kMostRows) return TCUSCAN_ERR_UNSUPPORTED;
    if (id_bytes != 4 && id_bytes != 8) return TCUSCAN_ERR_INVALID_ARG;
    if (n == 0 || dim == 0) return TCUSCAN_OK;
    if (!d_ids || !d_weight || !d_out || vocab == 0 || weight_stride < dim || out_stride < dim) return TCUSCAN_ERR_INVALID_ARG;
    if ((uintptr_t)d_ids % (size_t)id_bytes || (uintptr_t)d_weight % we || (uintptr_t)d_out % oe || d_out == d_weight) return TCUSCAN_ERR_INVALID_ARG;
    if (d_ws && (ws_bytes < chain_layout::kHeaderBytes || (uintptr_t)d_ws % 8)) return TCUSCAN_ERR_WORKSPACE;
    const size_t cols = weight_dt == kF32 && out_dt == kF32 ? kLaneCols<kF32> : kLaneCols<kBF16>, slices = (dim + 64 * cols - 1) / (64 * cols);
    const bool aligned = dim % cols == 0 && weight_stride % cols == 0 && out_stride % cols == 0 && (uintptr_t)d_weight % 16 == 0 && (uintptr_t)d_out % 16 == 0;
    const bool many = n * slices >= kManyItems;
    const size_t at_once = many ? kTokensAtOnce : 1, blocks = ((n + at_once - 1) / at_once * slices + kThreads / 64 - 1) / (kThreads / 64);
    if (blocks > most_groups(kThreads)) return TCUSCAN_ERR_UNSUPPORTED;
    LookupArgs A = {d_ids, d_weight, d_out, d_ws, n, vocab, dim, weight_stride, out_stride, slices, scale, id_bytes == 8};
    void *args[] = {&A};
    const void *fn = many ? aligned ? pick<LookupManyAligned>(weight_dt, out_dt) : pick<LookupMany>(weight_dt, out_dt)
                          : aligned ? pick<LookupAligned>(weight_dt, out_dt) : pick<Lookup>(weight_dt, out_dt);
    return hipLaunchKernel(fn, dim3((unsigned)blocks), dim3(kThreads), args, 0, (hipStream_t)stream) == hipSuccess ? TCUSCAN_OK : TCUSCAN_ERR_HIP;
}

size_t tcuscan_embedding_backward_workspace_bytes(size_t n, size_t vocab, size_t dim)
{
    return n > 0xFFFFFFFFull || vocab == 0 || vocab > kMostRows || dim == 0 ? 0 : GradLayout(n, dim).all;
}

tcuscan_status_t tcuscan_embedding_backward(const void *d_ids, int id_bytes, size_t n, const void *d_out_grad, size_t out_stride, tcuscan_dtype_t out_dt,
                                            void *d_weight_grad, size_t vocab, size_t dim, size_t weight_stride, tcuscan_dtype_t weight_dt, float scale,
                                            long long padding, unsigned flags, void *d_ws, size_t ws_bytes, tcuscan_stream_t stream)
{
    const size_t oe = elem_bytes(out_dt), we = elem_bytes(weight_dt);
    if (!we || !oe || vocab > kMostRows || n > 0xFFFFFFFFull) return TCUSCAN_ERR_UNSUPPORTED;
    if ((id_bytes != 4 && id_bytes != 8) || (flags & ~TCUSCAN_ACCUMULATE)) return TCUSCAN_ERR_INVALID_ARG;
    const int accumulate = (flags & TCUSCAN_ACCUMULATE) != 0;
    if (vocab == 0 || dim == 0 || (n == 0 && accumulate)) return TCUSCAN_OK;
    if (!d_weight_grad || weight_stride < dim || (uintptr_t)d_weight_grad % we) return TCUSCAN_ERR_INVALID_ARG;
    if (n && (!d_ids || !d_out_grad || out_stride < dim || d_out_grad == d_weight_grad)) return TCUSCAN_ERR_INVALID_ARG;
    if ((uintptr_t)d_ids % (size_t)id_bytes || (uintptr_t)d_out_grad % oe) return TCUSCAN_ERR_INVALID_ARG;
    const GradLayout L(n, dim);
    if (!d_ws || ws_bytes < L.all || (uintptr_t)d_ws % 16) return TCUSCAN_ERR_WORKSPACE;
    char *ws = (char *)d_ws;
    hipStream_t s = (hipStream_t)stream;
    GradArgs A = {};
    A.ids = d_ids; A.d_out = d_out_grad; A.d_weight = d_weight_grad; A.ws = d_ws;
    A.keys = (uint32_t *)(ws + L.keys); A.tokens = (uint32_t *)(ws + L.tokens); A.partial = (float *)(ws + L.partial);
    A.n = n; A.vocab = vocab; A.dim = dim; A.out_stride = out_stride; A.weight_stride = weight_stride;
    A.padding = padding; A.scale = scale; A.wide_ids = id_bytes == 8; A.accumulate = accumulate;
    void *args[] = {&A};
    const size_t cols = out_dt == kF32 ? kLaneCols<kF32> : kLaneCols<kBF16>;
    const bool aligned = dim % cols == 0 && out_stride % cols == 0 && weight_stride % cols == 0 && (uintptr_t)d_out_grad % 16 == 0 && (uintptr_t)d_weight_grad % (cols * we) == 0;
    if (n <= kFewTokens) {
        // up to 1024 workgroups, as many as run side by side for fp32 gradients (43 to 46 registers: four to a unit; three for 16-bit ones, which take 74 to 77), and
        // no more: each of them reads all token numbers (3000 tokens, 8000 bf16 rows of 200: 10.9 us, with twice as many 13.5)
        A.slices = (dim + 64 * cols - 1) / (64 * cols);
        A.rows = 4;
        while (A.rows < kMaxFewRows && (vocab + A.rows - 1) / A.rows * A.slices > 1024) A.rows *= 2;
        const size_t groups = (vocab + A.rows - 1) / A.rows * A.slices;
        if (groups > most_groups(64 * kWaves)) return TCUSCAN_ERR_UNSUPPORTED;
        const void *fn = aligned ? pick<FewAligned>(out_dt, weight_dt) : pick<Few>(out_dt, weight_dt);
        return hipLaunchKernel(fn, dim3((unsigned)groups), dim3(64 * kWaves), args, 0, s) == hipSuccess ? TCUSCAN_OK : TCUSCAN_ERR_HIP;
    }
    A.slices = (dim + 64 * cols - 1) / (64 * cols);
    const size_t pieces = (n + kPiece - 1) / kPiece, zero_groups = accumulate ? 0 : (vocab + kZeroRows - 1) / kZeroRows;
    A.zero_groups = zero_groups;
    A.piece_groups = (pieces * A.slices + kThreads / 64 - 1) / (kThreads / 64);
    const size_t by = aligned ? 4 : 1, join_groups = pieces * ((dim + 64 * by - 1) / (64 * by)), key_groups = (n + kThreads - 1) / kThreads;
    if (key_groups > most_groups(kThreads) || A.piece_groups + zero_groups > most_groups(kThreads) || join_groups > most_groups(64 * kJoinWaves)) return TCUSCAN_ERR_UNSUPPORTED;
    tcuscan_internal_workspace_reused(d_ws);       // (keys, tokens and sums, at places that depend on n; the sort's forms with a chain clear its status words)
    if (hipLaunchKernel((const void *)token_keys_kernel, dim3((unsigned)key_groups), dim3(kThreads), args, 0, s) != hipSuccess) return TCUSCAN_ERR_HIP;
    int bits = 0;
    while (((size_t)1 << bits) <= vocab) ++bits;
    const tcuscan_status_t st = tcuscan_split_radix_sort_u32(A.keys, A.tokens, n, bits, ws + L.keys_tmp, ws + L.tokens_tmp, ws + L.flags, ws + L.positions,
                                                             d_ws, L.chain, stream);
    if (st != TCUSCAN_OK) return st;
    const void *fn = aligned ? pick<RunsAligned>(out_dt, weight_dt) : pick<Runs>(out_dt, weight_dt);
    if (hipLaunchKernel(fn, dim3((unsigned)(A.piece_groups + zero_groups)), dim3(kThreads), args, 0, s) != hipSuccess) return TCUSCAN_ERR_HIP;
    fn = weight_dt == kF16 ? aligned ? (const void *)join_runs_kernel<kF16, 4> : (const void *)join_runs_kernel<kF16, 1>
       : weight_dt == kF32 ? aligned ? (const void *)join_runs_kernel<kF32, 4> : (const void *)join_runs_kernel<kF32, 1>
                           : aligned ? (const void *)join_runs_kernel<kBF16, 4> : (const void *)join_runs_kernel<kBF16, 1>;
    return hipLaunchKernel(fn, dim3((unsigned)join_groups), dim3(64 * kJoinWaves), args, 0, s) == hipSuccess ? TCUSCAN_OK : TCUSCAN_ERR_HIP;
}

}  // extern "C"
