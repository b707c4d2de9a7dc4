// Linear attention with one decay per head: the prefix sum with a matrix for an element and a decay between elements.
//
// For one row of tokens and one head, with a = exp(log_decay):
//
//   forward  : S_t = a S_(t-1) + k_t v_t^T,   o_t = scale q_t S_t            (S: dk x dv, S_(-1) = state_in, q_t a row vector)
//   gradients: with R_t = scale q_t^T do_t + a R_(t+1)  (R_(T) = d_state_out / a, so that R_(T-1) = scale q^T do + d_state_out)
//              dq_t = scale do_t S_t^T,  dv_t = k_t R_t,  dk_t = v_t R_t^T,  d_state_in = a R_0
//
// All four are one operator, "walk": a state M (A x E) that takes y_t z_t^T token by token and is read as x_t M, from the front
//   M_t = a M_(t-1) + by_new y_t z_t^T;  out_t = by_read x_t M_t
// or from the end, where the state decays after the token rather than before it
//   M_t = M_(t+1) + by_new y_t z_t^T;  out_t = by_read x_t M_t;  M_t *= a
//   o: (q, k, v) from the front, M = S;    dq: (do, v, k) from the front, M = S^T
//   dv: (k, q, do) from the end, M = R;    dk: (v, do, q) from the end, M = R^T
// Stored heads that several heads share give each of them a walk; gradients of shared heads are summed over them afterwards.

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "../../include/tcuscan.h"
#include "chain_layout.h"
#include "element_types.h"
#include "wave_ops.h"

extern "C" void tcuscan_internal_workspace_reused(void *d_ws);                // tcuscan.hip

namespace {

constexpr int kMaxDim = 256;

// One of the arrays [token][stored head][feature]: head h is the stored head h * heads / all heads.
struct Heads {
    void *data;
    long long token, head;                         // strides in elements
    unsigned heads;
    __device__ __forceinline__ long long at(unsigned h, unsigned all) const { return (long long)(h * (unsigned long long)heads / all) * head; }
};

struct WalkArgs {
    Heads x, y, z, out;                            // out.heads is the number of heads
    const float *log_decay;
    const long long *offsets, *slots;              // slots: null, or the state that each row has
    const float *m_in;                             // null: zeros
    float *m_out;                                  // null: not wanted
    float *between;                                // [piece][head][state]: what segments add, then what they start from, laid out as lanes hold it
    float *between_turned;                         // null, or where what they start from goes transposed, too: for a walk with A and E exchanged
    void *ws;
    long long states;                              // how many states there are
    long long total;
    unsigned rows, heads, A, E;
    unsigned m_a, m_e;                             // strides of a state: M[a][e] is at a * m_a + e * m_e
    unsigned pieces, segment_log2;
    float by_new, by_read;
    int from_end;
    int wide;                                      // the output is fp32 whatever the element type
};

// A log_decay of minus infinity as a number whose product with 0 is 0.  (Not by fmaxf, which would make a number of NaN: a model whose decays have gone wrong
// gets NaN.)
__device__ __forceinline__ float not_infinite(float log_decay) { return log_decay < -1e30f ? -1e30f : log_decay; }
// a^n, for weights.  (An n of 0 gives 1 for a decay of 0, too.)
__device__ __forceinline__ float decay_power(float log_decay, float n) { return __expf(not_infinite(log_decay) * n); }
// Takes a state n tokens on: m becomes a^n m.  Slow decays (a^n from 1/2 on) as m + (a^n - 1) m: multiplied by a rounded a^n, a state
// would be off by up to half a unit in the last place of 1 each time, always to the same side: 1e-5 for 1 - 2^-9 token by token.
struct Decay {
    float by;
    bool slow;
    __device__ __forceinline__ Decay(float log_decay, float n)
    {
        const float x = not_infinite(log_decay) * n;
        slow = x > -0.69f;
        by = slow ? expm1f(x) : __expf(x);
    }
    __device__ __forceinline__ float operator()(float m) const { return fmaf(m, by, slow ? m : 0.0f); }
};

// The same for many steps of n tokens each, one multiplication per element: what rounding takes from a^n, by() adds to a later factor, so that the
// product of all factors stays within an ulp or two of the decay.
struct Decays {
    float factor, less, owed;                      // a^n = factor + less
    __device__ __forceinline__ Decays(float log_decay, float n)
    {
        const Decay d(log_decay, n);
        factor = d.slow ? 1.0f + d.by : d.by;
        less = d.slow ? d.by - (factor - 1.0f) : 0.0f;
        owed = 0.0f;
    }
    __device__ __forceinline__ float by()
    {
        owed += less;
        const float f = factor + owed;
        owed -= f - factor;
        return f;
    }
};

// Row r's tokens, clipped to the arrays.
__device__ __forceinline__ void row_extent(const long long *offsets, unsigned r, long long total, long long &lo, long long &hi)
{
    lo = offsets[r]; hi = offsets[r + 1];
    lo = lo < 0 ? 0 : lo > total ? total : lo;
    hi = hi < lo ? lo : hi > total ? total : hi;
}

// Row r's place among the states, or -1 for none.
__device__ __forceinline__ long long state_of(const long long *slots, unsigned r, long long states)
{
    const long long s = slots ? slots[r] : (long long)r;
    return s >= 0 && s < states ? s : -1;
}

// ---------------------------------------------------------------- the walk in blocks of tokens, on the matrix unit
//
// C tokens i = 0 .. C-1 of a row (from the end: the last token first) with the state M in front of them:
//
//   out_i = by_read (a^(i+1) x_i M + sum over j <= i of by_new a^(i-j) (x_i . y_j) z_j)    (from the end a^i in place of a^(i+1))
//   M    <- a^C M + sum over j of by_new a^(C-1-j) y_j^T z_j                          (from the end a^(C-j))
//
// Every sum over features or tokens is a matrix product: P^T = Y X^T (then weighted and cut to j <= i), out^T = M^T X^T and Z^T P^T,
// M += Y^T (wZ).  A wavefront owns 16 CT columns of Z, out and M and all A rows of M, in MFMA accumulators from the first token to the
// last.  The products are ordered so that operands fall into the lanes that have them: the accumulators of M, two row tiles side by side, are
// the left operand of M^T X^T as they stand (tile rows are dealt so that a lane's eight values are eight consecutive a), and Z's columns are
// read transposed once, for Z^T P^T and, weighted, for the update.  Only X, Y and Z, which all wavefronts of a workgroup share, go through LDS.
//
// What it costs.  A row of many tokens is cut into segments, so Y and Z are read twice: once for what each segment adds to the state, then, with what
// each segment starts from (join_kernel), for the outputs.  65536 bf16 tokens, 16 heads of 128 x 128 (inputs and outputs 1.08 GB, 1.73 GB moved): 125 us for the
// first reading (0.55 GB, 4.4 TB/s where streaming reaches 6.5), 14 for the join, 250 for the outputs (1.1 GB, 4.4 TB/s); with all inputs in L2 97 and 206.  So
// the walk itself is most of it: vector instructions (half of the outputs' cycles, the scores among them, which each of the four wavefronts computes for itself)
// and the matrix unit (busy a third of them), in the order in which one block's products wait for each other.  f16 and fp32 multiply three and six pairs of parts and
// split their inputs on the way: 20011 f16 tokens in 30 ragged rows, 16 heads of 80 x 96, 81 + 9 + 162 us; the units work 60 % of the last and wait for the
// longest rows' ends.  In short rows the time is that of blocks in a row, 2 us each.
//
// Precision.  The matrix unit multiplies bf16 and adds in fp32, so every operand is a sum of bf16 parts: bf16 inputs one, f16 two (exact),
// fp32 three.  What is rounded on the way:
//   * what is added to a state, by_new a^(C-1-j) z_j: three parts (24 bits) where the row's last state is asked for and any of it is left there, so that
//     states come out as exact as fp32 sums make them; two (16 bits) where only 16-bit outputs are read from it
//   * the state, where it is read: two parts (16 bits), three for fp32
//   * the weighted scores P: two parts, three for fp32 (one part would do for bf16 but for its error, as large as that of the rounded output: 0.0024 of the
//     result in place of 0.0017 on rows of a few tokens; the second costs 1 % of 65536 tokens' time, 2 to 3 % of many short rows')
// and products of parts that together lie below what is kept are left out (kOrder).  In all at most 2^-15 (bf16) and 2^-14 (f16) of the sum of the terms' sizes:
// where the terms of an output cancel, that is what is seen of it, and fp32 sums would be closer.

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short  s16x4 __attribute__((ext_vector_type(4)));
typedef short  s16x8 __attribute__((ext_vector_type(8)));
typedef float  f32x4 __attribute__((ext_vector_type(4)));
typedef float  f32x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef unsigned u32x4 __attribute__((ext_vector_type(4)));

constexpr int parts_of(int dt) { return dt == kBF16 ? 1 : dt == kF16 ? 2 : 3; }
// Tokens of a block.  With 64 the state would be read (split, multiplied) half as often, but LDS would hold no more than the next block beside the present
// one: too little on its way to keep the memory busy (65536 tokens 400 us, and 300 with all inputs in L2; with 32 tokens 382 and 286).
constexpr int kBlock = 32;

constexpr int kWalkWaves = 4;
// Workgroups on a compute unit, by what LDS and registers give.  States of 128 x 128 with their products of fp32's six pairs of parts need more than half of a
// lane's registers: 20011 tokens of 8 heads take 285 us with one workgroup, 341 with two whose values are in part kept in memory.
constexpr int groups_at_once(int dt, int ap, int ct, bool reads) { return ap > 128 || (dt == kF32 && ap == 128 && ct == 2 && reads) ? 1 : 2; }
// s_waitcnt: no more than n loads and stores on their way, whatever else is.
constexpr int loads_left(int n) { return (n & 15) | (n >> 4) << 14 | 0x0F70; }

template <int N> struct Parts { bf16x8 p[N]; };

// The first N bf16 parts of eight values: x = part 0 + part 1 + ..., each the rounding of what the ones before leave.
template <int N> __device__ __forceinline__ Parts<N> split(f32x8 x)
{
    Parts<N> parts;
#pragma unroll
    for (int n = 0; n < N; ++n) {
        u32x4 pairs = __builtin_bit_cast(u32x4, __builtin_convertvector(x, bf16x8));
        asm("" : "+v"(pairs));                     // (or every value is converted a second time on its own, to be subtracted)
        parts.p[n] = __builtin_bit_cast(bf16x8, pairs);
        if (n + 1 < N)
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                x[2 * k] -= bits<float>(pairs[k] << 16);
                x[2 * k + 1] -= bits<float>(pairs[k] & 0xFFFF0000u);
            }
    }
    return parts;
}
__device__ __forceinline__ f32x4 mfma(bf16x8 a, bf16x8 b, f32x4 acc) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, acc, 0, 0, 0); }
// A product of sums of parts: step(i, j) for all products a[i] b[j] with i + j < kOrder, small ones first.
template <int kOrder, class Step, int NA, int NB> __device__ __forceinline__ void products(Step step, const Parts<NA> &, const Parts<NB> &)
{
#pragma unroll
    for (int i = NA - 1; i >= 0; --i)
#pragma unroll
        for (int j = NB - 1; j >= 0; --j)
            if (i + j < kOrder) step(i, j);
}

// Tiles in LDS are rows of COLS bf16 whose 16-byte granules are permuted within each row by an exclusive or with a number made of the row.  The
// permutation keeps both kinds of reading free of bank conflicts: the same granule of 16 consecutive rows (row operands), and four
// granules of four consecutive rows (operands read transposed).
template <int COLS> struct Tile {
    static constexpr int kGranules = COLS / 8;
    __device__ __forceinline__ static int swizzle(int row)
    {
        if constexpr (kGranules >= 16) return (row & 3) << 2 | ((row >> 2) & 3);
        else if constexpr (kGranules == 8) return ((row >> 1) & 1) << 2 | ((row >> 2) & 3);
        else return (row >> 2) & 3;
    }
    __device__ __forceinline__ static int at(int row, int col) { return row * COLS + ((((col >> 3) ^ swizzle(row)) << 3) | (col & 7)); }
};

// Where a lane finds operands.  Both kinds of reading go through one number per lane and tile shape; the operand's place in the tile then is an exclusive or
// with a constant (columns) and a constant offset (rows, which the swizzle repeats every 16 of).
//
// Row operand: lane l of group g receives the eight columns k0 + 8 g .. + 7 of row row0 + l (row0 a multiple of 16, k0 of 32).
template <int COLS> __device__ __forceinline__ int row_lane(int lane) { return Tile<COLS>::at(lane & 15, 8 * (lane >> 4)); }
template <int COLS> __device__ __forceinline__ bf16x8 row_operand(const bf16_t *tile, int mine, int row0, int k0) { return *(const bf16x8 *)(tile + row0 * COLS + (mine ^ k0)); }
// Column operand: lane l of group g receives one column of the eight rows 4 g .. 4 g + 3 and 16 + 4 g .. 16 + 4 g + 3 (the order in which P^T's accumulators
// hold its rows, two tiles of them above each other).  The instruction hands lane l of 16 the l-th column of the four rows whose 16 pieces of four columns
// the 16 lanes point at: lane s at row s / 4 and piece s % 4, which starts PIECE columns behind the one before.  `first`: the wavefront's first column, a
// multiple of 32 (of 16, if it is the only one); col0: from there, a multiple of 16 or with PIECE = 8 of 32, and there + 4 for the other halves of the
// pieces' granules.
__device__ __forceinline__ s16x4 read_transposed(const bf16_t *p)
{
    return __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4 *)p);
}
template <int COLS, int PIECE> __device__ __forceinline__ int column_lane(int lane, int first) { return Tile<COLS>::at(4 * (lane >> 4) + ((lane & 15) >> 2), first + PIECE * (lane & 3)); }
template <int COLS> __device__ __forceinline__ bf16x8 column_operand(const bf16_t *tile, int mine, int col0)
{
    const bf16_t *p = tile + (col0 & 4) + (mine ^ (col0 & ~4));
    return __builtin_bit_cast(bf16x8, __builtin_shufflevector(read_transposed(p), read_transposed(p + 16 * COLS), 0, 1, 2, 3, 4, 5, 6, 7));
}
__device__ __forceinline__ int column_row(int g, int k) { return k < 4 ? 4 * g + k : 12 + 4 * g + k; }       // the k-th of these rows
// Keeps the compiler from computing what depends on v ahead of a loop: addresses made of a lane's number and constants would take dozens of registers.
template <class T> __device__ __forceinline__ T here(T v)
{
    asm volatile("" : "+v"(v));
    return v;
}

// A block of tokens on its way from memory to LDS: C rows of COLS elements, a granule of eight to a lane at a time.  Rows from n on and columns from `cols`
// on become zeros.  Three ways:
//   kDirect   bf16, granules aligned and either inside or outside: loads that write LDS themselves, lane after lane, so that it is the lanes' addresses
//             that are permuted; what is outside is beyond the end of the buffer they read from.  They need no registers while they are on
//             their way (the 48 a lane would need at dk = dv = 128 do not fit beside the state and are spilled).
//   kStaged   fp32 and f16, granules as above: through registers, split into parts on the way.
//   kSlow     anything else: element by element.
enum Way { kDirect, kStaged, kSlow };
constexpr Way way_of(int dt, bool whole) { return !whole ? kSlow : dt == kBF16 ? kDirect : kStaged; }
template <int DT, int C, int COLS, int THREADS, bool WHOLE> struct Stage {
    typedef typename Elem<DT>::T T;
    static constexpr Way kWay = way_of(DT, WHOLE);
    static constexpr int kItems = C * COLS / 8, kEach = (kItems + THREADS - 1) / THREADS, kQuads = sizeof(T) / 2, N = parts_of(DT);
    static constexpr int kRowsAtOnce = THREADS / (COLS / 8);
    static_assert(THREADS % (COLS / 8) == 0, "a lane keeps to its columns");
    static constexpr int kOffsets = kRowsAtOnce % 16 == 0 ? 1 : 2;             // the swizzle repeats every 16 rows
    static_assert(kRowsAtOnce % 8 == 0, "or every second time");
    static constexpr int kSure = kItems / THREADS;             // loads that every wavefront makes of a block
    u32x4 v[kWay == kStaged ? kEach : 1][kQuads];
    const T *first;                                // the block's first row (the same for all lanes)
    long long step;                                // from row to row
    int row, col, cols;
    int offset[kOffsets];                          // kDirect: the lane's first granules in a whole block, in bytes from its lowest address

    __device__ __forceinline__ void begin(const T *p, long long row_step, int columns)
    {
        row = (int)threadIdx.x / (COLS / 8); col = (int)threadIdx.x % (COLS / 8) * 8; cols = columns; first = p; step = row_step;
        if constexpr (kWay == kDirect)
#pragma unroll
            for (int i = 0; i < kOffsets; ++i) {
                const int r = row + i * kRowsAtOnce, c = (int)(threadIdx.x % (COLS / 8) ^ Tile<COLS>::swizzle(r)) * 8;
                offset[i] = c < cols ? ((step < 0 ? C - 1 - r : r) * (int)(step < 0 ? -step : step) + c) * (int)sizeof(T) : kOutside;
            }
    }
    static constexpr int kOutside = 1 << 30;       // beyond the end of any block (64 rows less than 2^22 elements apart)
    // kDirect: all the way, to be waited for; kStaged: as far as the registers.
    __device__ __forceinline__ void load(bf16_t *tile, int n)
    {
        if constexpr (kWay == kDirect) {
            const int by_row = (int)(step < 0 ? -step : step) * (int)sizeof(T), shift = step < 0 ? (C - n) * by_row : 0;
            const __amdgpu_buffer_rsrc_t block = __builtin_amdgcn_make_buffer_rsrc((void *)(step < 0 ? first + (n - 1) * step : first), 0, (n - 1) * by_row + cols * (int)sizeof(T), 0x00027000);
            bf16_t *to = tile + __builtin_amdgcn_readfirstlane((int)threadIdx.x / 64) * 512;
#pragma unroll
            for (int i = 0; i < kEach; ++i) {
                const int at = offset[i % kOffsets] + (i - i % kOffsets) * kRowsAtOnce * (step < 0 ? -by_row : by_row) - shift;
                if (kEach * THREADS <= kItems || (int)threadIdx.x < kItems)
                    __builtin_amdgcn_raw_ptr_buffer_load_lds(block, (__attribute__((address_space(3))) void *)(to + i * THREADS * 8), 16, at, 0, 0, 0);
            }
            first += C * step;
        } else if constexpr (kWay == kStaged) {
            const T *p = first + row * step + col;
#pragma unroll
            for (int i = 0; i < kEach; ++i, p += kRowsAtOnce * step) {
#pragma unroll
                for (int q = 0; q < kQuads; ++q) v[i][q] = u32x4{0u, 0u, 0u, 0u};
                if (row + i * kRowsAtOnce < n && col < cols)
#pragma unroll
                    for (int q = 0; q < kQuads; ++q) v[i][q] = ((const u32x4 *)p)[q];
            }
        }
    }
    static __device__ __forceinline__ void put(bf16_t *to, const T (&e)[8])                       // the parts are C * COLS elements apart
    {
        if constexpr (N == 1) {
            __builtin_memcpy(to, e, 16);
        } else {
            f32x8 x;
#pragma unroll
            for (int k = 0; k < 8; ++k) x[k] = (float)e[k];
            const Parts<N> parts = split<N>(x);
#pragma unroll
            for (int n = 0; n < N; ++n) *(bf16x8 *)(to + n * C * COLS) = parts.p[n];
        }
    }
    // kStaged and kSlow: the rest of the way, and on to the next block.
    __device__ __forceinline__ void store(bf16_t *tile, int n)
    {
        if constexpr (kWay == kStaged) {
#pragma unroll
            for (int i = 0; i < kEach; ++i) {
                T e[8];
                __builtin_memcpy(e, &v[i][0], sizeof e);
                if (row + i * kRowsAtOnce < C) put(tile + Tile<COLS>::at(row + i * kRowsAtOnce, col), e);
            }
        } else if constexpr (kWay == kSlow) {
#pragma unroll 1
            for (int r = row; r < C; r += kRowsAtOnce) {
                const T *p = first + r * step + col;
                T e[8];
#pragma unroll
                for (int k = 0; k < 8; ++k) e[k] = r < n && col + k < cols ? p[k] : (T)0.0f;
                put(tile + Tile<COLS>::at(r, col), e);
            }
        }
        first += C * step;
    }
};

// Which piece of which row a workgroup walks over.  Rows are cut into segments of 2^segment_log2 tokens; the segments of row r have the numbers
// from offsets[r] / 2^segment_log2 + r on, which leaves every row room for its own without anything being counted first.
struct Piece {
    unsigned r;
    long long lo, hi;                              // the row's tokens
    long long first, end;                          // the segment's, counted from where the walk starts
    bool last;
};
__device__ __forceinline__ long long uniform(long long v)
{   // (the same in all lanes: into scalar registers)
    return (long long)((unsigned long long)(unsigned)__builtin_amdgcn_readfirstlane((int)(v >> 32)) << 32 | (unsigned)__builtin_amdgcn_readfirstlane((int)v));
}
__device__ __forceinline__ bool find_piece(const WalkArgs &W, unsigned number, Piece &p)
{
    unsigned lo = 0, hi = W.rows;
    const bool one = (W.total >> W.segment_log2) == 0;       // a row is one segment
    if (one) {
        lo = number;
    } else {
        while (hi - lo > 1) {                      // the last row whose segments start at or below `number`
            const unsigned mid = lo + (hi - lo) / 2;
            if ((W.offsets[mid] >> W.segment_log2) + mid <= (long long)number) lo = mid; else hi = mid;
        }
    }
    p.r = lo;
    row_extent(W.offsets, p.r, W.total, p.lo, p.hi);
    p.lo = uniform(p.lo); p.hi = uniform(p.hi);
    const long long length = p.hi - p.lo, s = one ? 0 : (long long)number - (p.lo >> W.segment_log2) - p.r, segment = 1ll << W.segment_log2;
    p.first = s * segment;
    if (s < 0 || (s > 0 && p.first >= length)) return false;
    p.end = p.first + segment < length ? p.first + segment : length;
    p.last = p.end == length;
    return true;
}

// K consecutive columns of the output, `col` the first of them.  WHOLE: they are aligned and all inside or all outside.
template <class T, bool WHOLE, int K> __device__ __forceinline__ void store_columns(T *p, int col, int cols, const f32x4 *v)
{
    typedef T Some __attribute__((ext_vector_type(K)));
    Some x;
#pragma unroll
    for (int k = 0; k < K; ++k) x[k] = (T)v[k / 4][k % 4];
    if constexpr (WHOLE) {
        if (col < cols) *(Some *)p = x;
    } else {
#pragma unroll
        for (int k = 0; k < K; ++k)
            if (col + k < cols) p[k] = x[k];
    }
}

// How a state lies in the registers of a workgroup, and between segments in memory: M[t][c][r] of thread `tid` is M[a][e] with
//   a = 32 (t / 2) + 8 g + 4 (t % 2) + r,  e = 64 CT block + 16 CT wave + 4 CT (l / 4) + 4 c + l % 4,  tid = 64 wave + 16 g + l.
// Four lanes side by side and r make 4 x 4 squares, so the transposed state lies likewise.  In memory: [block][t][c][tid][r].
struct StateShape {
    unsigned AP, CT;                               // A and E are padded to these multiples
    __host__ __device__ unsigned columns() const { return 64 * CT; }
    __host__ __device__ unsigned floats(unsigned E) const { return AP * ((E + columns() - 1) / columns()) * columns(); }
    __device__ __forceinline__ void element(unsigned quad, unsigned &a0, unsigned &e) const        // of the quad-th four elements: (a0 + r, e)
    {
        const unsigned tid = quad % 256, c = quad / 256 % CT, t = quad / 256 / CT % (AP / 16), block = quad / 16 / AP / CT;
        a0 = 32 * (t / 2) + 8 * (tid / 16 % 4) + 4 * (t % 2);
        e = columns() * block + 16 * CT * (tid / 64) + 4 * CT * (tid / 4 % 4) + 4 * c + tid % 4;
    }
    __device__ __forceinline__ unsigned quad(unsigned a0, unsigned e) const
    {
        const unsigned block = e / columns(), x = e % columns(), wave = x / (16 * CT), y = x % (16 * CT), c = y / 4 % CT;
        const unsigned tid = 64 * wave + 16 * (a0 / 8 % 4) + 4 * (y / (4 * CT)) + x % 4, t = 2 * (a0 / 32) + a0 / 4 % 2;
        return ((block * (AP / 16) + t) * CT + c) * 256 + tid;
    }
};
// (a workgroup's share of the registers: 256 rows of a state and 32 columns to a wavefront do not fit them)
__host__ __device__ inline StateShape state_shape(unsigned A, unsigned E) { return {A <= 32 ? 32u : A <= 64 ? 64u : A <= 96 ? 96u : A <= 128 ? 128u : A <= 192 ? 192u : 256u, E <= 64 || A > 128 ? 1u : 2u}; }

// The 4 x 4 square that four lanes side by side hold, transposed.
__device__ __forceinline__ f32x4 turned(f32x4 v, int lane)
{
    auto from = [](float x, auto how) { return bits<float>((uint32_t)__builtin_amdgcn_mov_dpp((int)bits<uint32_t>(x), decltype(how)::value, 0xf, 0xf, true)); };
    typedef std::integral_constant<int, kQuadPerm1032> Next;
    typedef std::integral_constant<int, kQuadPerm2301> Across;
    const bool odd = lane & 1, high = lane & 2;
    const float a = from(odd ? v[0] : v[1], Next()), b = from(odd ? v[2] : v[3], Next());
    v = odd ? f32x4{a, v[1], b, v[3]} : f32x4{v[0], a, v[2], b};
    const float c = from(high ? v[0] : v[2], Across()), d = from(high ? v[1] : v[3], Across());
    return high ? f32x4{c, d, v[2], v[3]} : f32x4{v[0], v[1], c, d};
}
// A caller's state into the registers or out of them: M[a][e] at p[a * m_a + e * m_e].  16 bytes at a time where rows or columns are dense.  The lane's number
// passes through an empty asm statement: otherwise the compiler keeps every address and predicate from the reading of a state to its writing.
template <int AP, int CT, bool OUT, class P> __device__ __forceinline__ void move_state(f32x4 (&M)[AP / 16][CT], P *p, unsigned first_e, unsigned A, unsigned E, size_t m_a, size_t m_e)
{
    const unsigned lane = here(threadIdx.x & 63), a0 = 8 * (lane >> 4), s = lane & 3, e_lane = first_e + 4 * CT * ((lane & 15) >> 2) + s;
    typedef std::conditional_t<OUT, f32x4, const f32x4> Quad;
    const bool rows = m_e == 1 && E % 4 == 0, columns = m_a == 1 && A % 4 == 0;
#pragma unroll
    for (int t = 0; t < AP / 16; ++t)
#pragma unroll
        for (int c = 0; c < CT; ++c) {
            const unsigned a = a0 + 32 * (t / 2) + 4 * (t & 1), e = e_lane + 4 * c;
            if (rows) {
                Quad *q = (Quad *)(p + (size_t)(a + s) * m_a + (e - s));
                f32x4 v = {0.0f, 0.0f, 0.0f, 0.0f};
                const bool there = a + s < A && e < E;
                if constexpr (OUT) {
                    v = turned(M[t][c], lane);
                    if (there) *q = v;
                } else {
                    if (there) v = *q;
                    M[t][c] = turned(v, lane);
                }
            } else if (columns) {
                Quad *q = (Quad *)(p + a + (size_t)e * m_e);
                if (a < A && e < E) {
                    if constexpr (OUT) *q = M[t][c];
                    else M[t][c] = *q;
                }
            } else {
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    if (a + r < A && e < E) {
                        if constexpr (OUT) p[(a + r) * m_a + e * m_e] = M[t][c][r];
                        else M[t][c][r] = p[(a + r) * m_a + e * m_e];
                    }
            }
        }
}

// Columns of a tile of AP features: a power of two, for the permutation of granules.
constexpr int tile_columns(int AP) { return AP <= 32 ? 32 : AP <= 64 ? 64 : AP <= 128 ? 128 : 256; }

// READS: writes outputs and, of a row's last segment, the state.  Otherwise only what each segment but the last adds to the state.
template <int DT, int AP, int CT, bool WHOLE, bool READS> __global__ __launch_bounds__(64 * kWalkWaves, groups_at_once(DT, AP, CT, READS)) void walk_kernel(WalkArgs W)
{
    typedef typename Elem<DT>::T T;
    constexpr int N = parts_of(DT), C = kBlock, LP = tile_columns(AP), EB = 16 * kWalkWaves * CT, kThreads = 64 * kWalkWaves;
    constexpr bool kDirectly = way_of(DT, WHOLE) == kDirect;
    constexpr int kTiles = 2, kOrder = N == 3 ? 3 : 2;         // tiles of 16 tokens
    typedef Stage<DT, C, LP, kThreads, WHOLE> StageA;
    typedef Stage<DT, C, EB, kThreads, WHOLE> StageE;
    // Loads that write LDS themselves go round kRing tiles of each array: while a block is worked on, the kRing - 1 behind it are on their way.
    constexpr int kRing = !kDirectly ? 1 : READS ? 3 : 4, kLoads = (READS ? 2 : 1) * StageA::kSure + StageE::kSure;
    // (Each tile is an array of its own: the compiler has a wavefront wait for loads into an array before it reads from it.)
    constexpr int kX = READS ? N * C * LP : 8, kY = N * C * LP, kZ = N * C * EB, kNone = 8;
    __shared__ __attribute__((aligned(16))) bf16_t sx0[kX], sx1[kRing > 1 ? kX : kNone], sx2[kRing > 2 ? kX : kNone];
    __shared__ __attribute__((aligned(16))) bf16_t sy0[kY], sy1[kRing > 1 ? kY : kNone], sy2[kRing > 2 ? kY : kNone], sy3[kRing > 3 ? kY : kNone];
    __shared__ __attribute__((aligned(16))) bf16_t sz0[kZ], sz1[kRing > 1 ? kZ : kNone], sz2[kRing > 2 ? kZ : kNone], sz3[kRing > 3 ? kZ : kNone];

    const unsigned blocks = (W.E + EB - 1) / EB;
    const unsigned block = blockIdx.x % blocks, h = blockIdx.x / blocks % W.heads, number = blockIdx.x / blocks / W.heads;
    const int lane = threadIdx.x & 63, l = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    if (block == 0 && h == 0)                      // offsets and slots are looked over once
        for (size_t r = (size_t)number * kThreads + threadIdx.x; r < W.rows; r += (size_t)W.pieces * kThreads) {
            const long long a = W.offsets[r], b = W.offsets[r + 1];
            if (a < 0 || b < a || b > W.total || (W.slots && W.slots[r] >= W.states)) raise_fault(W.ws, kFaultBadIndex);
        }
    Piece piece;
    if (!find_piece(W, number, piece)) return;
    if (!READS && piece.last) return;              // (what a row's last segment adds, nobody asks for)

    const float log_decay = W.log_decay[h];
    const int e0 = (int)block * EB, wave_e = 16 * CT * wave;        // the workgroup's first column, and the wavefront's of these
    const long long slot = state_of(W.slots, piece.r, W.states);
    const size_t state = ((size_t)slot * W.heads + h) * W.A * W.E;
    f32x4 *between = (f32x4 *)W.between + (((size_t)number * W.heads + h) * blocks + block) * (AP * EB / 4) + threadIdx.x;
    const bool cut = piece.first > 0 || !piece.last;                // a row of several segments
    f32x4 M[AP / 16][CT] = {};
    if constexpr (READS) {
        // a row of several segments finds what it starts from in the workspace, also for the first of them
        if (cut)
#pragma unroll
            for (int t = 0; t < AP / 16; ++t)
#pragma unroll
                for (int c = 0; c < CT; ++c) M[t][c] = between[(t * CT + c) * 256];
        else if (W.m_in && slot >= 0)
            move_state<AP, CT, false>(M, W.m_in + state, e0 + wave_e, W.A, W.E, W.m_a, W.m_e);
    }
    float reading[kTiles];                         // by_read a^(i+1), from the end a^i, of the lane's token in each tile
    const float by_key = W.by_read * W.by_new;
#pragma unroll
    for (int t = 0; t < kTiles; ++t) reading[t] = W.by_read * decay_power(log_decay, (float)(16 * t + l + (W.from_end ? 0 : 1)));
    // and of P^T's rows j = 4 g + r and columns i = l: tiles on the diagonal (nothing where j is behind i) and below it
    f32x4 on_diagonal, below_diagonal;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        const int apart = l - 4 * g - r;
        on_diagonal[r] = apart >= 0 ? by_key * decay_power(log_decay, (float)apart) : 0.0f;
        below_diagonal[r] = by_key * decay_power(log_decay, (float)(apart + 16));
    }

    const long long sign = W.from_end ? -1 : 1, origin = (W.from_end ? piece.hi - 1 : piece.lo) + sign * piece.first;
    StageA next_x, next_y;
    StageE next_z;
    next_x.begin((const T *)W.x.data + W.x.at(h, W.heads) + origin * W.x.token, sign * W.x.token, (int)W.A);
    next_y.begin((const T *)W.y.data + W.y.at(h, W.heads) + origin * W.y.token, sign * W.y.token, (int)W.A);
    next_z.begin((const T *)W.z.data + W.z.at(h, W.heads) + origin * W.z.token + e0, sign * W.z.token, (int)W.E - e0);
    // the lane's first output: token l of the block, column 4 CT g of the wavefront's
    const int out_size = W.wide ? 4 : (int)sizeof(T), col = e0 + wave_e + 4 * CT * g;
    const long long out_step = sign * W.out.token * out_size;
    char *out = (char *)W.out.data + (W.out.at(h, W.heads) + origin * W.out.token) * out_size + (sign < 0 ? 15 * out_step : 0);
    typedef std::conditional_t<WHOLE, unsigned, long long> Offset;
    const Offset out_lane = (Offset)((sign < 0 ? l - 15 : l) * out_step) + (Offset)(col * out_size);         // (not negative: outputs have positive strides)
    // The third part of what is added to a state counts where the state itself is asked for, not where 16-bit outputs are read from it; and there for the segments
    // of which more than 2^-24 is left at the end of the row (beyond, two parts are off by 2^-40 of what was added.  With the limit at 1/8 65536 tokens take 380 us,
    // with this one 387, without one 405; but a state to which the last tokens add little would have 16 bits where fp32 sums have 24).
    constexpr int kParts = N == 3 ? 3 : 2;
    const bool exact = W.m_out && slot >= 0 && decay_power(log_decay, (float)(piece.hi - piece.lo - piece.end)) > 0x1p-24f;
    const long long length = piece.end - piece.first;
    auto tokens = [&](long long left) { return (int)(left < C ? left : C); };
    // by_new a^(n-1-j), from the end a^(n-j), of the lane's tokens j = column_row(g, k): in whole blocks a power for the lane's group times one for k, which is
    // the same for all lanes
    const float group_power = W.by_new * decay_power(log_decay, (float)(12 - 4 * g + (W.from_end ? 1 : 0)));
    float near_power[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) near_power[k] = __builtin_bit_cast(float, __builtin_amdgcn_readfirstlane(__builtin_bit_cast(int, decay_power(log_decay, (float)(19 - column_row(0, k))))));
    auto weights = [&](int n) {
        f32x8 w;
        if (n == C) {
            const float far = here(group_power);
#pragma unroll
            for (int k = 0; k < 8; ++k) w[k] = far * near_power[k];
        } else {
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const int j = column_row(here(g), k);
                w[k] = j < n ? W.by_new * decay_power(log_decay, (float)(n - 1 - j + (W.from_end ? 1 : 0))) : 0.0f;
            }
        }
        return w;
    };
    long long left = length;                       // tokens that are not on their way yet
    auto load = [&](bf16_t *x_tile, bf16_t *y_tile, bf16_t *z_tile) {
        if (left <= 0) return;
        const int n = tokens(left);
        if constexpr (READS) next_x.load(x_tile, n);
        next_y.load(y_tile, n);
        next_z.load(z_tile, n);
        left -= C;
    };
    load(sx0, sy0, sz0);
    if constexpr (kRing > 2) load(sx1, sy1, sz1);
    if constexpr (kRing > 3) load(sx2, sy2, sz2);
    Decays whole_block(log_decay, (float)C);
    long long at = 0;
    // A block in the tiles `now`; behind the barrier, the tiles of the block before are free to be loaded into.
    auto take_block = [&](bf16_t *x_now, bf16_t *x_free, bf16_t *y_now, bf16_t *y_free, bf16_t *z_now, bf16_t *z_free) __attribute__((always_inline)) {
        const long long behind = length - at - C;
        const int n = tokens(length - at);
        const int row_at = here(row_lane<LP>(lane)), y_at = here(column_lane<LP, 8>(lane, 0)), z_at = here(column_lane<EB, 4 * CT>(lane, wave_e));
        if constexpr (kDirectly) {
            // of the loads behind this block's, as many may be on their way as there surely are (stores are waited for with them)
            if (kRing > 3 && behind > C) __builtin_amdgcn_s_waitcnt(loads_left((kRing > 3 ? 2 : 1) * kLoads));
            else if (behind > 0) __builtin_amdgcn_s_waitcnt(loads_left(kLoads));
            else __builtin_amdgcn_s_waitcnt(loads_left(0));
        } else {
            __syncthreads();                       // everybody has done with the block before
            if constexpr (READS) next_x.store(x_now, n);
            next_y.store(y_now, n);
            next_z.store(z_now, n);
        }
        __syncthreads();
        if constexpr (kDirectly) load(x_free, y_free, z_free);
        if constexpr (AP <= 128)
            if (e0 + wave_e >= (int)W.E) {         // a wavefront of no columns only loads (96 columns: 3 % less; with larger states the branch costs as much)
                if constexpr (!kDirectly) load(x_now, y_now, z_now);
                at += C;
                return;
            }
        Parts<N> zt[CT];                           // 16 columns of Z by 32 tokens
#pragma unroll
        for (int c = 0; c < CT; ++c)
#pragma unroll
            for (int m = 0; m < N; ++m) zt[c].p[m] = column_operand<EB>(z_now + m * C * EB, z_at, 4 * c);
        // what is added to the state
        const f32x8 w = weights(n);
        auto weighted = [&](int c) {
#pragma clang fp contract(off)                     // (a product rounded once: fused with what a split subtracts, its parts would differ between the two places that split it)
            f32x8 v = __builtin_convertvector(zt[c].p[N - 1], f32x8);
#pragma unroll
            for (int m = N - 2; m >= 0; --m) v += __builtin_convertvector(zt[c].p[m], f32x8);
            return v * w;
        };
        if constexpr (READS) {
            // P^T, by every wavefront for itself (through LDS it would cost a barrier), and M^T X^T, from the same rows of X.  P^T[j][i] of keys' and queries' tile 0 |
            // of queries' tile 1 with keys' tile 0 and 1
            constexpr int NM = N == 3 ? 3 : 2;
            f32x4 o[2][CT], p00 = {}, p01 = {}, p11 = {};
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int c = 0; c < CT; ++c) o[t][c] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
            Parts<NM> m[2][CT];                    // this step's parts of M and the next one's
            auto split_m = [&](int s) {
#pragma unroll
                for (int c = 0; c < CT; ++c) m[s & 1][c] = split<NM>(__builtin_shufflevector(M[2 * s][c], M[2 * s + 1][c], 0, 1, 2, 3, 4, 5, 6, 7));
            };
            split_m(0);
#pragma unroll
            for (int s = 0; s < AP / 32; ++s) {
                __builtin_amdgcn_sched_barrier(0);             // (or the parts of all steps take registers at once)
                Parts<N> queries[2], keys[2];
#pragma unroll
                for (int t = 0; t < 2; ++t)
#pragma unroll
                    for (int i = 0; i < N; ++i) {
                        queries[t].p[i] = row_operand<LP>(x_now + i * C * LP, row_at, 16 * t, 32 * s);
                        keys[t].p[i] = row_operand<LP>(y_now + i * C * LP, row_at, 16 * t, 32 * s);
                    }
                if (s + 1 < AP / 32) split_m(s + 1);
                products<kOrder>([&](int i, int j) {           // (independent ones behind each other)
                    p00 = mfma(keys[0].p[i], queries[0].p[j], p00);
                    p01 = mfma(keys[0].p[i], queries[1].p[j], p01);
                    p11 = mfma(keys[1].p[i], queries[1].p[j], p11);
                }, keys[0], queries[0]);
                products<kOrder>([&](int i, int j) {
#pragma unroll
                    for (int c = 0; c < CT; ++c)
#pragma unroll
                        for (int t = 0; t < 2; ++t) o[t][c] = mfma(m[s & 1][c].p[i], queries[t].p[j], o[t][c]);
                }, m[0][0], queries[0]);
            }
            p00 *= on_diagonal;
            p01 *= below_diagonal;
            p11 *= on_diagonal;
            const f32x4 none = {0.0f, 0.0f, 0.0f, 0.0f};
            const Parts<kParts> p[2] = {split<kParts>(__builtin_shufflevector(p00, none, 0, 1, 2, 3, 4, 5, 6, 7)), split<kParts>(__builtin_shufflevector(p01, p11, 0, 1, 2, 3, 4, 5, 6, 7))};
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int c = 0; c < CT; ++c) o[t][c] *= reading[t];
            products<kOrder>([&](int i, int j) {
#pragma unroll
                for (int t = 0; t < 2; ++t)
#pragma unroll
                    for (int c = 0; c < CT; ++c) o[t][c] = mfma(zt[c].p[i], p[t].p[j], o[t][c]);
            }, zt[0], p[0]);
#pragma unroll
            for (int t = 0; t < kTiles; ++t) {
                if (16 * t + l >= n) continue;
                char *to_row = out + 16 * t * out_step + out_lane;
                if (W.wide) store_columns<float, WHOLE, 4 * CT>((float *)to_row, col, (int)W.E, o[t]);
                else store_columns<T, WHOLE, 4 * CT>((T *)to_row, col, (int)W.E, o[t]);
            }
            out += C * out_step;
        }
        if constexpr (!kDirectly) load(x_now, y_now, z_now);   // (as far as the registers)
        // the state
        const float by = n == C ? whole_block.by() : Decays(log_decay, (float)n).by();
        Parts<kParts> wz[CT];
#pragma unroll
        for (int c = 0; c < CT; ++c) wz[c] = split<kParts>(weighted(c));
        Parts<N> yt[2][2];                         // two tiles of M's rows, and the next two
        auto load_y = [&](int t) {
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int m = 0; m < N; ++m) yt[t / 2 & 1][u].p[m] = column_operand<LP>(y_now + m * C * LP, y_at, 16 * t + 4 * u);
        };
        load_y(0);
#pragma unroll
        for (int t = 0; t < AP / 16; t += 2) {
            if (t + 2 < AP / 16) load_y(t + 2);
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int c = 0; c < CT; ++c) M[t + u][c] *= by;
            products<kParts>([&](int i, int j) {
#pragma unroll
                for (int u = 0; u < 2; ++u)
#pragma unroll
                    for (int c = 0; c < CT; ++c) M[t + u][c] = mfma(yt[t / 2 & 1][u].p[i], wz[c].p[j], M[t + u][c]);
            }, yt[0][0], wz[0]);
        }
        if constexpr (kParts == 2)
            if (exact) {                           // the third parts
                Parts<3> third[CT];
#pragma unroll
                for (int c = 0; c < CT; ++c) third[c] = split<3>(weighted(c));
#pragma unroll
                for (int t = 0; t < AP / 16; ++t)
#pragma unroll
                    for (int m = 0; m < N; ++m) {
                        const bf16x8 y_part = column_operand<LP>(y_now + m * C * LP, y_at, 32 * (t / 2) + 4 * (t & 1));
#pragma unroll
                        for (int c = 0; c < CT; ++c) M[t][c] = mfma(y_part, third[c].p[2 - m], M[t][c]);
                    }
            }
        at += C;
    };
    if constexpr (kRing == 4) {
        while (at < length) {
            take_block(sx0, sx0, sy0, sy3, sz0, sz3);
            if (at < length) take_block(sx0, sx0, sy1, sy0, sz1, sz0);
            if (at < length) take_block(sx0, sx0, sy2, sy1, sz2, sz1);
            if (at < length) take_block(sx0, sx0, sy3, sy2, sz3, sz2);
        }
    } else if constexpr (kRing == 3) {
        while (at < length) {
            take_block(sx0, sx2, sy0, sy2, sz0, sz2);
            if (at < length) take_block(sx1, sx0, sy1, sy0, sz1, sz0);
            if (at < length) take_block(sx2, sx1, sy2, sy1, sz2, sz1);
        }
    } else {
        while (at < length) take_block(sx0, sx0, sy0, sy0, sz0, sz0);
    }
    if constexpr (!READS) {
#pragma unroll
        for (int t = 0; t < AP / 16; ++t)
#pragma unroll
            for (int c = 0; c < CT; ++c) between[(t * CT + c) * 256] = M[t][c];
    } else if (piece.last && W.m_out && slot >= 0) {
        move_state<AP, CT, true>(M, W.m_out + state, e0 + wave_e, W.A, W.E, W.m_a, W.m_e);
    }
}

// What each segment of a row starts from, from what the segments in front of it add: a thread takes four elements of the state along the row, four segments'
// loads on their way at a time.  The carry across segments is a sum with one decay, so this is all that has to be done in order.  Bound by memory for many rows
// (8 rows of 4096 tokens, 16 heads of 128 x 128: 16 us, 20 with the transposed states), by the steps in a row for few (65536 tokens in 32 segments: 14 us).
constexpr int kJoinThreads = 256, kJoinAhead = 4;
__global__ __launch_bounds__(kJoinThreads) void join_kernel(WalkArgs W)
{
    const StateShape shape = state_shape(W.A, W.E), turned_shape = state_shape(W.E, W.A);
    const unsigned quads = shape.floats(W.E) / 4, turned_quads = turned_shape.floats(W.A) / 4, blocks = quads / kJoinThreads;
    const unsigned i = blockIdx.x % blocks * kJoinThreads + threadIdx.x, h = blockIdx.x / blocks % W.heads, row = blockIdx.x / blocks / W.heads;
    long long lo, hi;
    row_extent(W.offsets, row, W.total, lo, hi);
    const long long segment = 1ll << W.segment_log2, segments = (hi - lo + segment - 1) >> W.segment_log2, first = (lo >> W.segment_log2) + row;
    if (segments <= 1 || first + segments > (long long)W.pieces) return;
    const long long slot = state_of(W.slots, row, W.states);
    unsigned a0, e;
    shape.element(i, a0, e);
    f32x4 m = {0.0f, 0.0f, 0.0f, 0.0f};
    if (W.m_in && slot >= 0)
#pragma unroll
        for (int r = 0; r < 4; ++r)
            if (a0 + r < W.A && e < W.E) m[r] = W.m_in[((size_t)slot * W.heads + h) * W.A * W.E + (size_t)(a0 + r) * W.m_a + (size_t)e * W.m_e];
    const Decay decay(W.log_decay[h], (float)segment);
    f32x4 *p = (f32x4 *)W.between + ((size_t)first * W.heads + h) * quads + i;
    // of the transposed state, rows e .. and column a0 + r change places
    const bool turn = W.between_turned && (e & ~3u) < turned_shape.AP && a0 < turned_quads * 4 / turned_shape.AP;
    f32x4 *q = (f32x4 *)W.between_turned + ((size_t)first * W.heads + h) * turned_quads + (turn ? turned_shape.quad(e & ~3u, a0 + (threadIdx.x & 3)) : 0);
    const size_t step = (size_t)W.heads * quads, turned_step = (size_t)W.heads * turned_quads;
    for (long long s = 0; s < segments; s += kJoinAhead) {
        f32x4 added[kJoinAhead];                   // (of the last segment nothing is known, nor asked for)
#pragma unroll
        for (int u = 0; u < kJoinAhead; ++u) {
            added[u] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
            if (s + u + 1 < segments) added[u] = p[(s + u) * step];
        }
#pragma unroll
        for (int u = 0; u < kJoinAhead; ++u) {
            if (s + u < segments) {
                p[(s + u) * step] = m;
                const f32x4 across = turned(m, threadIdx.x);
                if (turn) q[(s + u) * turned_step] = across;
            }
#pragma unroll
            for (int r = 0; r < 4; ++r) m[r] = decay(m[r]) + added[u][r];
        }
    }
}

// out[t][stored head][i] = the sum of part[t][head][i] over the heads that share the stored head, in their order, for the tokens that rows hold (others have
// no part, and their outputs are not written).  One pass, bound by reading fp32; four elements a thread where the output allows stores of four (12289 tokens, 4 x 4 heads of 64: 10 us, one element a thread 15).
struct SumArgs {
    const float *part;
    Heads out;
    const long long *offsets;
    long long total;
    unsigned rows, heads, D;
};
constexpr int kSumThreads = 256;
template <int DT, int VEC> __global__ __launch_bounds__(kSumThreads) void sum_heads_kernel(SumArgs S)
{
    typedef typename Elem<DT>::T T;
    typedef float From __attribute__((ext_vector_type(VEC)));
    typedef T To __attribute__((ext_vector_type(VEC)));
    const unsigned groups = S.D / VEC, each = groups * S.out.heads, group = S.heads / S.out.heads;          // (each: at most 2^24)
    const size_t i = (size_t)blockIdx.x * kSumThreads + threadIdx.x;
    const long long t = (long long)(i / each);
    if (t >= S.total || t < S.offsets[0] || t >= S.offsets[S.rows]) return;
    const unsigned at = (unsigned)(i - (size_t)t * each), h = at / groups, d = (at - h * groups) * VEC;
    const float *p = S.part + ((size_t)t * S.heads + (size_t)h * group) * S.D + d;
    From sum = 0.0f;
    for (unsigned g = 0; g < group; ++g) sum += *(const From *)(p + (size_t)g * S.D);
    *(To *)((T *)S.out.data + t * S.out.token + (long long)h * S.out.head + d) = __builtin_convertvector(sum, To);
}

// One token for each of many sequences.  A workgroup takes a block of columns of one state: 2^lanes_log2 lanes to a row, VEC columns each, as many rows at
// a time as the workgroup has lanes for; the state stays in registers between its product with q and its writing.  The state is read and written once and
// nothing else counts: 256 sequences of 16 heads of 128 x 128 (537 MB) take 112 us, 4.8 TB/s (streaming from one array to another 6.5); one sequence, whose columns are spread over
// as many workgroups as there are columns for, the time of a launch.
struct StepArgs {
    Heads q, k, v, out;
    const float *log_decay;
    const long long *slots;
    float *state;
    void *ws;
    long long states;
    unsigned heads, A, E, blocks, lanes_log2;
    float scale;
};
constexpr int kStepThreads = 256;
template <int DT, int VEC> __global__ __launch_bounds__(kStepThreads) void step_kernel(StepArgs S)
{
    typedef typename Elem<DT>::T T;
    typedef float Vec __attribute__((ext_vector_type(VEC)));
    __shared__ float ks[kMaxDim], qs[kMaxDim];
    __shared__ Vec sums[kStepThreads / 64][64];
    const unsigned block = blockIdx.x % S.blocks, h = blockIdx.x / S.blocks % S.heads, i = blockIdx.x / S.blocks / S.heads;
    const unsigned lanes = 1u << S.lanes_log2, e = (block * lanes + (threadIdx.x & (lanes - 1))) * VEC, row0 = threadIdx.x >> S.lanes_log2, rows = kStepThreads >> S.lanes_log2;
    const long long slot = state_of(S.slots, i, S.states);
    if (threadIdx.x == 0 && block == 0 && h == 0 && S.slots && S.slots[i] >= S.states) raise_fault(S.ws, kFaultBadIndex);
    const bool column = e < S.E, there = slot >= 0;
    float *m = S.state + ((size_t)(there ? slot : 0) * S.heads + h) * S.A * S.E + e;
    constexpr unsigned kAhead = 8;
    Vec s[kAhead];
    // the first rows are on their way before anything else is looked at
    auto load = [&](unsigned a0) {
#pragma unroll
        for (unsigned u = 0; u < kAhead; ++u) {
            const unsigned a = a0 + u * rows;
            s[u] = Vec{};
            if (there && column && a < S.A) s[u] = *(const Vec *)(m + (size_t)a * S.E);
        }
    };
    load(row0);
    const T *q = (const T *)S.q.data + S.q.at(h, S.heads) + i * S.q.token, *k = (const T *)S.k.data + S.k.at(h, S.heads) + i * S.k.token,
            *v = (const T *)S.v.data + S.v.at(h, S.heads) + i * S.v.token;
    for (unsigned a = threadIdx.x; a < S.A; a += kStepThreads) {
        ks[a] = (float)k[a];
        qs[a] = (float)q[a];
    }
    Vec ve = {}, sum = {};
#pragma unroll
    for (int c = 0; c < VEC; ++c)
        if (e + c < S.E) ve[c] = (float)v[e + c];
    const Decay decay(S.log_decay[h], 1.0f);
    __syncthreads();
    for (unsigned a0 = row0; a0 < S.A; a0 += kAhead * rows) {
        if (a0 != row0) load(a0);
#pragma unroll
        for (unsigned u = 0; u < kAhead; ++u) {
            const unsigned a = a0 + u * rows;
            if (a >= S.A) break;
#pragma unroll
            for (int c = 0; c < VEC; ++c) {
                s[u][c] = fmaf(ks[a], ve[c], decay(s[u][c]));
                sum[c] = fmaf(qs[a], s[u][c], sum[c]);
            }
            if (there && column) *(Vec *)(m + (size_t)a * S.E) = s[u];
        }
    }
    // over the rows: lanes of a wavefront that have the same columns, then the wavefronts
#pragma unroll
    for (int c = 0; c < VEC; ++c)
        for (unsigned d = lanes; d < 64; d *= 2) sum[c] += __shfl_xor(sum[c], (int)d);
    sums[threadIdx.x >> 6][threadIdx.x & 63] = sum;
    __syncthreads();
    if (threadIdx.x >= lanes || !column) return;
#pragma unroll
    for (int w = 1; w < kStepThreads / 64; ++w) sum += sums[w][threadIdx.x];
    T *out = (T *)S.out.data + S.out.at(h, S.heads) + i * S.out.token;
#pragma unroll
    for (int c = 0; c < VEC; ++c)
        if (e + c < S.E) out[e + c] = (T)(sum[c] * S.scale);
}

bool launch(const void *fn, size_t grid, unsigned block, void *args, hipStream_t s)
{
    void *list[] = {args};
    return hipLaunchKernel(fn, dim3((unsigned)grid), dim3(block), list, 0, s) == hipSuccess;
}

template <template <int> class Pick> const void *pick(int dt) { return dt == kF16 ? Pick<kF16>::fn() : dt == kF32 ? Pick<kF32>::fn() : Pick<kBF16>::fn(); }
template <int DT> struct SumHeads { static const void *fn() { return (const void *)sum_heads_kernel<DT, 1>; } };
template <int DT> struct SumHeadsByFour { static const void *fn() { return (const void *)sum_heads_kernel<DT, 4>; } };
template <int DT> struct Step { static const void *fn() { return (const void *)step_kernel<DT, 1>; } };
template <int DT> struct StepByFour { static const void *fn() { return (const void *)step_kernel<DT, 4>; } };

// What a call can do, by its sizes alone: TCUSCAN_OK, or why not.
tcuscan_status_t check_shape(const tcuscan_attention_shape_t *p, int dt)
{
    if (!p) return TCUSCAN_ERR_INVALID_ARG;
    const tcuscan_attention_shape_t &s = *p;
    if (!elem_bytes(dt)) return TCUSCAN_ERR_UNSUPPORTED;
    if (s.rows < 0 || s.total < 0 || s.heads < 1 || s.dk < 1 || s.dv < 1) return TCUSCAN_ERR_INVALID_ARG;
    for (long long shared : {s.q_heads, s.k_heads, s.v_heads})
        if (shared < 1 || shared > s.heads || s.heads % shared) return TCUSCAN_ERR_INVALID_ARG;
    if (s.dk > kMaxDim || s.dv > kMaxDim) return TCUSCAN_ERR_UNSUPPORTED;
    if (s.total >> 40) return TCUSCAN_ERR_UNSUPPORTED;
    if (s.rows > 0x3FFFFFFF || s.heads > 0xFFFF || (unsigned long long)s.rows * s.heads > 0xFFFFFFF) return TCUSCAN_ERR_UNSUPPORTED;
    return TCUSCAN_OK;
}

// Rows are cut into segments so that a call with few rows and heads still has work for the whole chip.  Each segment costs a state written and read, and a
// step of join_kernel.
//   * Not cut: calls of up to 256 tokens to a row, as far as the host can tell: 256 for each row, 512 in all (256 tokens in one row, 8 heads of 64: 16 us against
//     20 in three launches; 512 tokens 26 against 19, their gradients 71 against 41).
//   * 64 tokens a segment while these are no more workgroups than compute units (gradients of 512 tokens, 8 heads of 64: 41 us, with 128 tokens 47; but
//     5000 tokens in 3 rows 38, with 128 tokens 31).
//   * Then 128 or more, for 512 workgroups (65536 tokens, 16 heads of 128: 382 us, with 256 workgroups 431, with 1024 407), or 1024 where both sides of the
//     state are at most 64, of which more fit a unit (20000 tokens in 60 rows, 16 heads of 64: 82 us, with 512 104), and eight heads or more share the
//     workgroups, or there would be too many segments in a row (30000 tokens of 4 heads of 48: 77, with 512 55).
constexpr size_t kUnits = 256, kWantedGroups = 512;
constexpr unsigned kWholeRows = 62;
constexpr long long kMostUncutRow = 256, kMostUncut = 512;
bool uncut(const tcuscan_attention_shape_t &s) { return s.total <= kMostUncut && s.total <= kMostUncutRow * s.rows; }
size_t groups_of_a_token(const tcuscan_attention_shape_t &s) { return (size_t)s.heads * ((size_t)((s.dk > s.dv ? s.dk : s.dv) + 127) / 128); }
size_t wanted_groups(const tcuscan_attention_shape_t &s) { return s.dk <= 64 && s.dv <= 64 && s.heads >= 8 ? 2 * kWantedGroups : kWantedGroups; }
unsigned segment_log2_for(const tcuscan_attention_shape_t &s)
{
    if (uncut(s)) return kWholeRows;
    const size_t work = (size_t)s.total * groups_of_a_token(s);
    if (work >> 6 <= kUnits) return 6;
    unsigned log2 = 7;
    while (work >> log2 > wanted_groups(s)) ++log2;
    return (size_t)s.total >> log2 ? log2 : kWholeRows;
}
size_t pieces_for(const tcuscan_attention_shape_t &s, unsigned segment_log2) { return (size_t)s.rows + ((size_t)s.total >> segment_log2); }
// The most segments beyond one a row that any call of up to s.total tokens makes: a call's segments double in length where they become too many, so it is not the
// largest one that makes most.  (They hold at least 64 tokens, and their number times the groups of a token is at most what is wanted.)
size_t most_segments(const tcuscan_attention_shape_t &s)
{
    const size_t shortest = (size_t)s.total >> 6, wanted = wanted_groups(s) / groups_of_a_token(s);
    return uncut(s) ? 0 : shortest < wanted ? shortest : wanted;
}

// The workspace: the header, what lies between `pieces` segments (none: rows are not cut), parts of shared heads.
struct Layout {
    size_t between, turned, part, all;
    Layout(const tcuscan_attention_shape_t &s, bool backward, size_t pieces)
    {
        between = chain_layout::kHeaderBytes;
        turned = part = between;
        if (pieces) {
            const size_t state = state_shape((unsigned)s.dk, (unsigned)s.dv).floats((unsigned)s.dv), other = state_shape((unsigned)s.dv, (unsigned)s.dk).floats((unsigned)s.dk);
            const size_t all_states = pieces * s.heads * 4;
            turned = between + all_states * (backward && other > state ? other : state);
            part = turned + (backward ? all_states * other : 0);
        }
        size_t wide = 0;
        if (backward) {
            if (s.q_heads < s.heads || s.k_heads < s.heads) wide = (size_t)s.dk;
            if (s.v_heads < s.heads && (size_t)s.dv > wide) wide = (size_t)s.dv;
        }
        all = part + (size_t)s.total * s.heads * wide * 4;
    }
};
// How a call cuts its rows.  One that is cut although it has no more tokens than calls that are not may be given the workspace of such a call (512 tokens in two
// rows, then in one): it is not cut then, either.
struct Cut {
    unsigned segment_log2;
    size_t pieces;
    Layout layout;
    Cut(const tcuscan_attention_shape_t &s, bool backward, unsigned log2) : segment_log2(log2), pieces(pieces_for(s, log2)), layout(s, backward, log2 == kWholeRows ? 0 : pieces) {}
    static Cut of(const tcuscan_attention_shape_t &s, bool backward, size_t ws_bytes)
    {
        const Cut wanted(s, backward, segment_log2_for(s));
        return ws_bytes < wanted.layout.all && s.total <= kMostUncut ? Cut(s, backward, kWholeRows) : wanted;
    }
};

bool misaligned(const void *p, size_t to) { return (uintptr_t)p % to != 0; }

Heads heads_of(const void *data, long long token, long long head, long long heads) { return {(void *)data, token, head, (unsigned)heads}; }

template <int DT, int CT, bool WHOLE, bool READS> const void *walk_for(unsigned A)
{
    switch (state_shape(A, 1).AP) {
        case 32: return (const void *)walk_kernel<DT, 32, CT, WHOLE, READS>;
        case 64: return (const void *)walk_kernel<DT, 64, CT, WHOLE, READS>;
        case 96: return (const void *)walk_kernel<DT, 96, CT, WHOLE, READS>;
        case 128: return (const void *)walk_kernel<DT, 128, CT, WHOLE, READS>;
        case 192: return (const void *)walk_kernel<DT, 192, 1, WHOLE, READS>;
        default: return (const void *)walk_kernel<DT, 256, 1, WHOLE, READS>;
    }
}
template <int DT, int CT, bool READS> const void *walk_for(unsigned A, bool whole) { return whole ? walk_for<DT, CT, true, READS>(A) : walk_for<DT, CT, false, READS>(A); }
template <int DT, bool READS> const void *walk_for(unsigned A, bool whole, unsigned CT) { return CT == 1 ? walk_for<DT, 1, READS>(A, whole) : walk_for<DT, 2, READS>(A, whole); }
template <bool READS> const void *walk_for(int dt, unsigned A, bool whole, unsigned CT)
{
    return dt == kF16 ? walk_for<kF16, READS>(A, whole, CT) : dt == kF32 ? walk_for<kF32, READS>(A, whole, CT) : walk_for<kBF16, READS>(A, whole, CT);
}

// Whether groups of eight elements of every token's features are aligned and whole, and 64 tokens within reach of a 32-bit offset.
bool whole(const Heads &x, unsigned dims, size_t esz)
{
    return dims % 8 == 0 && (uintptr_t)x.data % 16 == 0 && (size_t)x.token * esz % 16 == 0 && (size_t)x.head * esz % 16 == 0 &&
           (x.token < 0 ? -x.token : x.token) < (1ll << 22);
}

// Gradients of heads that share `out`, added four columns a thread or one: threads, and how many columns.
bool sums_by_four(const Heads &out, unsigned E, size_t esz)
{
    return E % 4 == 0 && out.token % 4 == 0 && out.head % 4 == 0 && !misaligned(out.data, 4 * esz);
}
size_t sum_groups(const Heads &out, long long total, unsigned E, size_t esz)
{
    return ((size_t)total * out.heads * (E / (sums_by_four(out, E, esz) ? 4 : 1)) + kSumThreads - 1) / kSumThreads;
}
size_t walk_groups(const WalkArgs &W, const StateShape &shape) { return (size_t)W.pieces * W.heads * ((W.E + shape.columns() - 1) / shape.columns()); }
size_t join_groups(const WalkArgs &W, const StateShape &shape) { return (size_t)W.rows * W.heads * (shape.floats(W.E) / 4 / kJoinThreads); }
// Whether a walk's launches can be made.
bool launches_fit(const WalkArgs &W, const Heads &out, int dt)
{
    const StateShape shape = state_shape(W.A, W.E);
    return walk_groups(W, shape) <= most_groups(64 * kWalkWaves) && (W.segment_log2 == kWholeRows || join_groups(W, shape) <= most_groups(kJoinThreads)) &&
           (out.heads == W.heads || sum_groups(out, W.total, W.E, elem_bytes(dt)) <= most_groups(kSumThreads));
}

// One walk, into `out`; with heads that share the output, into `part` first.  `states_ready`: what the segments start from is in the workspace.
tcuscan_status_t walk(WalkArgs W, Heads out, float *part, int dt, hipStream_t s, bool states_ready = false)
{
    const size_t esz = elem_bytes(dt);
    const StateShape shape = state_shape(W.A, W.E);
    const size_t groups = walk_groups(W, shape);
    const bool shared = out.heads < W.heads;
    const Heads to = shared ? Heads{part, (long long)W.heads * W.E, W.E, W.heads} : out;
    W.wide = shared;
    const bool new_whole = whole(W.y, W.A, esz) && whole(W.z, W.E, esz), all_whole = new_whole && whole(W.x, W.A, esz) && whole(to, W.E, shared ? 4 : esz) && to.token > 0;
    if (W.segment_log2 != kWholeRows && !states_ready) {
        if (!launch(walk_for<false>(dt, W.A, new_whole, shape.CT), groups, 64 * kWalkWaves, &W, s) || !launch((const void *)join_kernel, join_groups(W, shape), kJoinThreads, &W, s))
            return TCUSCAN_ERR_HIP;
    }
    W.out = to;
    if (!launch(walk_for<true>(dt, W.A, all_whole, shape.CT), groups, 64 * kWalkWaves, &W, s)) return TCUSCAN_ERR_HIP;
    if (!shared || !W.total) return TCUSCAN_OK;
    SumArgs S = {part, out, W.offsets, W.total, W.rows, W.heads, W.E};
    return launch(sums_by_four(out, W.E, esz) ? pick<SumHeadsByFour>(dt) : pick<SumHeads>(dt), sum_groups(out, W.total, W.E, esz), kSumThreads, &S, s) ? TCUSCAN_OK : TCUSCAN_ERR_HIP;
}

}  // namespace

extern "C" {

size_t tcuscan_decay_attention_workspace_bytes(const tcuscan_attention_shape_t *shape, tcuscan_dtype_t dt, int backward)
{
    if (check_shape(shape, dt) != TCUSCAN_OK) return 0;
    const size_t segments = most_segments(*shape);
    return Layout(*shape, backward != 0, segments ? (size_t)shape->rows + segments : 0).all;
}

tcuscan_status_t tcuscan_decay_attention(const tcuscan_attention_shape_t *shape, const void *d_q, const void *d_k, const void *d_v, void *d_out,
                                         const float *d_log_decay, const long long *d_offsets, tcuscan_dtype_t dt, float scale,
                                         const float *d_state_in, float *d_state_out, const long long *d_slots, size_t states,
                                         void *d_ws, size_t ws_bytes, tcuscan_stream_t stream)
{
    const tcuscan_status_t st = check_shape(shape, dt);
    if (st != TCUSCAN_OK) return st;
    const tcuscan_attention_shape_t &p = *shape;
    if (p.rows == 0 || (p.total == 0 && !d_state_out)) return TCUSCAN_OK;
    const size_t esz = elem_bytes(dt);
    if (!d_log_decay || !d_offsets || misaligned(d_log_decay, 4) || misaligned(d_offsets, 8) || misaligned(d_slots, 8)) return TCUSCAN_ERR_INVALID_ARG;
    if (misaligned(d_state_in, 16) || misaligned(d_state_out, 16)) return TCUSCAN_ERR_INVALID_ARG;
    if (p.total && (!d_q || !d_k || !d_v || !d_out || misaligned(d_q, esz) || misaligned(d_k, esz) || misaligned(d_v, esz) || misaligned(d_out, esz)))
        return TCUSCAN_ERR_INVALID_ARG;
    if (p.total && (d_out == d_q || d_out == d_k || d_out == d_v)) return TCUSCAN_ERR_INVALID_ARG;
    if (!d_slots && (d_state_in || d_state_out) && states < (size_t)p.rows) return TCUSCAN_ERR_INVALID_ARG;
    const Cut cut = Cut::of(p, false, ws_bytes);
    const Layout &L = cut.layout;
    if (!d_ws || ws_bytes < L.all || misaligned(d_ws, 16)) return TCUSCAN_ERR_WORKSPACE;
    WalkArgs W = {};
    W.x = heads_of(d_q, p.q_token, p.q_head, p.q_heads);
    W.y = heads_of(d_k, p.k_token, p.k_head, p.k_heads);
    W.z = heads_of(d_v, p.v_token, p.v_head, p.v_heads);
    W.log_decay = d_log_decay; W.offsets = d_offsets; W.slots = d_slots; W.m_in = d_state_in; W.m_out = d_state_out; W.ws = d_ws;
    W.between = (float *)((char *)d_ws + L.between); W.segment_log2 = cut.segment_log2; W.pieces = (unsigned)cut.pieces;
    W.states = (long long)states; W.total = p.total; W.rows = (unsigned)p.rows; W.heads = (unsigned)p.heads;
    W.A = (unsigned)p.dk; W.E = (unsigned)p.dv; W.m_a = W.E; W.m_e = 1;
    W.by_new = 1.0f; W.by_read = scale; W.from_end = 0;
    const Heads out = heads_of(d_out, p.o_token, p.o_head, p.heads);
    if (!launches_fit(W, out, dt)) return TCUSCAN_ERR_UNSUPPORTED;
    if (L.all > chain_layout::kHeaderBytes) tcuscan_internal_workspace_reused(d_ws);
    return walk(W, out, nullptr, dt, (hipStream_t)stream);
}

tcuscan_status_t tcuscan_decay_attention_backward(const tcuscan_attention_shape_t *shape, const void *d_q, const void *d_k, const void *d_v, const void *d_out_grad,
                                                  void *d_q_grad, void *d_k_grad, void *d_v_grad, const float *d_log_decay, const long long *d_offsets,
                                                  tcuscan_dtype_t dt, float scale, const float *d_state_in, const float *d_state_out_grad,
                                                  float *d_state_in_grad, void *d_ws, size_t ws_bytes, tcuscan_stream_t stream)
{
    const tcuscan_status_t st = check_shape(shape, dt);
    if (st != TCUSCAN_OK) return st;
    const tcuscan_attention_shape_t &p = *shape;
    if (p.rows == 0 || (p.total == 0 && !d_state_in_grad)) return TCUSCAN_OK;
    const size_t esz = elem_bytes(dt);
    if (!d_log_decay || !d_offsets || misaligned(d_log_decay, 4) || misaligned(d_offsets, 8)) return TCUSCAN_ERR_INVALID_ARG;
    if (misaligned(d_state_in, 16) || misaligned(d_state_out_grad, 16) || misaligned(d_state_in_grad, 16)) return TCUSCAN_ERR_INVALID_ARG;
    const void *ins[] = {d_q, d_k, d_v, d_out_grad}, *outs[] = {d_q_grad, d_k_grad, d_v_grad};
    if (p.total) {
        for (const void *i : ins)
            if (!i || misaligned(i, esz)) return TCUSCAN_ERR_INVALID_ARG;
        for (const void *o : outs) {
            if (!o || misaligned(o, esz)) return TCUSCAN_ERR_INVALID_ARG;
            for (const void *i : ins)
                if (o == i) return TCUSCAN_ERR_INVALID_ARG;
        }
        if (d_q_grad == d_k_grad || d_q_grad == d_v_grad || d_k_grad == d_v_grad) return TCUSCAN_ERR_INVALID_ARG;
    }
    if (d_state_in_grad && (d_state_in_grad == d_state_in || d_state_in_grad == d_state_out_grad)) return TCUSCAN_ERR_INVALID_ARG;
    const Cut cut = Cut::of(p, true, ws_bytes);
    const Layout &L = cut.layout;
    if (!d_ws || ws_bytes < L.all || misaligned(d_ws, 16)) return TCUSCAN_ERR_WORKSPACE;
    float *part = (float *)((char *)d_ws + L.part);
    hipStream_t s = (hipStream_t)stream;
    const Heads q = heads_of(d_q, p.q_token, p.q_head, p.q_heads), k = heads_of(d_k, p.k_token, p.k_head, p.k_heads),
                v = heads_of(d_v, p.v_token, p.v_head, p.v_heads), o = heads_of(d_out_grad, p.o_token, p.o_head, p.heads);
    const Heads q_grad = heads_of(d_q_grad, p.dq_token, p.dq_head, p.q_heads), k_grad = heads_of(d_k_grad, p.dk_token, p.dk_head, p.k_heads),
                v_grad = heads_of(d_v_grad, p.dv_token, p.dv_head, p.v_heads);
    WalkArgs W = {};
    W.log_decay = d_log_decay; W.offsets = d_offsets; W.ws = d_ws;
    W.between = (float *)((char *)d_ws + L.between); W.segment_log2 = cut.segment_log2; W.pieces = (unsigned)cut.pieces;
    W.states = p.rows; W.total = p.total; W.rows = (unsigned)p.rows; W.heads = (unsigned)p.heads;
    const unsigned dk = (unsigned)p.dk, dv = (unsigned)p.dv;
    W.A = dk; W.E = dv;
    if (!launches_fit(W, v_grad, dt)) return TCUSCAN_ERR_UNSUPPORTED;
    W.A = dv; W.E = dk;
    if (!launches_fit(W, q_grad, dt) || !launches_fit(W, k_grad, dt)) return TCUSCAN_ERR_UNSUPPORTED;
    if (L.all > chain_layout::kHeaderBytes) tcuscan_internal_workspace_reused(d_ws);
    // dq, with the states of the forward pass: S^T
    W.x = o; W.y = v; W.z = k; W.A = dv; W.E = dk; W.m_a = 1; W.m_e = dv; W.m_in = d_state_in;
    W.by_new = 1.0f; W.by_read = scale; W.from_end = 0;
    tcuscan_status_t r = walk(W, q_grad, part, dt, s);
    if (r != TCUSCAN_OK) return r;
    // dv and the gradient by the first states, from the end: R
    W.by_new = scale; W.by_read = 1.0f; W.from_end = 1; W.m_in = d_state_out_grad; W.m_out = d_state_in_grad;
    W.x = k; W.y = q; W.z = o; W.A = dk; W.E = dv; W.m_a = dv; W.m_e = 1;
    W.between_turned = cut.segment_log2 != kWholeRows ? (float *)((char *)d_ws + L.turned) : nullptr;
    r = walk(W, v_grad, part, dt, s);
    if (r != TCUSCAN_OK) return r;
    // dk, with the same states, transposed: R^T.  What its segments start from is there.
    W.m_out = nullptr;
    W.between = W.between_turned;
    W.x = v; W.y = o; W.z = q; W.A = dv; W.E = dk; W.m_a = 1; W.m_e = dv;
    return walk(W, k_grad, part, dt, s, true);
}

tcuscan_status_t tcuscan_decay_attention_step(const tcuscan_attention_shape_t *shape, const void *d_q, const void *d_k, const void *d_v, void *d_out,
                                              const float *d_log_decay, tcuscan_dtype_t dt, float scale, float *d_state, const long long *d_slots,
                                              size_t states, void *d_ws, size_t ws_bytes, tcuscan_stream_t stream)
{
    const tcuscan_status_t st = check_shape(shape, dt);
    if (st != TCUSCAN_OK) return st;
    const tcuscan_attention_shape_t &p = *shape;
    if (p.rows != p.total) return TCUSCAN_ERR_INVALID_ARG;
    if (p.rows == 0) return TCUSCAN_OK;
    const size_t esz = elem_bytes(dt);
    if (!d_log_decay || !d_state || !d_q || !d_k || !d_v || !d_out) return TCUSCAN_ERR_INVALID_ARG;
    if (misaligned(d_log_decay, 4) || misaligned(d_state, 16) || misaligned(d_slots, 8)) return TCUSCAN_ERR_INVALID_ARG;
    if (misaligned(d_q, esz) || misaligned(d_k, esz) || misaligned(d_v, esz) || misaligned(d_out, esz)) return TCUSCAN_ERR_INVALID_ARG;
    if (d_out == d_q || d_out == d_k || d_out == d_v || (!d_slots && states < (size_t)p.rows)) return TCUSCAN_ERR_INVALID_ARG;
    if (d_ws && (ws_bytes < chain_layout::kHeaderBytes || misaligned(d_ws, 8))) return TCUSCAN_ERR_WORKSPACE;
    StepArgs S = {};
    S.q = heads_of(d_q, p.q_token, p.q_head, p.q_heads); S.k = heads_of(d_k, p.k_token, p.k_head, p.k_heads);
    S.v = heads_of(d_v, p.v_token, p.v_head, p.v_heads); S.out = heads_of(d_out, p.o_token, p.o_head, p.heads);
    S.log_decay = d_log_decay; S.slots = d_slots; S.state = d_state; S.ws = d_ws; S.states = (long long)states;
    S.heads = (unsigned)p.heads; S.A = (unsigned)p.dk; S.E = (unsigned)p.dv; S.scale = scale;
    // lanes to a row: all of it, up to a wavefront; 128 bytes where there are few states, for more workgroups
    const unsigned vec = S.E % 4 == 0 ? 4 : 1, row_lanes = (S.E + vec - 1) / vec;
    const size_t all = (size_t)p.rows * p.heads;
    while ((1u << S.lanes_log2) < row_lanes && S.lanes_log2 < 6) ++S.lanes_log2;
    while (S.lanes_log2 > 3 && all * ((row_lanes + (1u << S.lanes_log2) - 1) >> S.lanes_log2) < kWantedGroups) --S.lanes_log2;
    S.blocks = (row_lanes + (1u << S.lanes_log2) - 1) >> S.lanes_log2;
    if (all * S.blocks > most_groups(kStepThreads)) return TCUSCAN_ERR_UNSUPPORTED;
    return launch(vec == 4 ? pick<StepByFour>(dt) : pick<Step>(dt), all * S.blocks, kStepThreads, &S, (hipStream_t)stream) ? TCUSCAN_OK : TCUSCAN_ERR_HIP;
}

}  // extern "C"
