// Rows of an embedding table by token number, scaled, and the gradient of the table by sorted tokens.
//
//   lookup   : out[t] = scale * weight[id[t]]
//   gradient : d_weight[r] = scale * (sum of d_out[t] over the t with id[t] = r, in ascending order of t)
//              The (id, t) pairs are sorted by id (tcuscan_split_radix_sort_u32: stable, so t ascends within an id); a row's
//              tokens then are one run of the sorted pairs.
//
// Sums are held in 32 bits and rounded once to the table's type.  Both move bytes and compute next to nothing.

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/tcuscan.h"
#include "chain_layout.h"
#include "element_types.h"

namespace {

constexpr int kThreads = 256;

struct LookupArgs {
    const void *ids, *weight;
    void *out, *ws;
    size_t n, vocab, dim, weight_stride, out_stride;
    float scale;
    int wide_ids;
};

__device__ __forceinline__ long long id_at(const void *ids, int wide, size_t i)
{
    return wide ? ((const long long *)ids)[i] : (long long)((const int *)ids)[i];
}

// One wavefront per token.
template <int DW, int DO> __global__ __launch_bounds__(kThreads) void lookup_kernel(LookupArgs A)
{
    typedef typename Elem<DW>::T W;
    typedef typename Elem<DO>::T O;
    const size_t t = (size_t)blockIdx.x * (kThreads / 64) + (threadIdx.x >> 6);
    if (t >= A.n) return;
    const int lane = threadIdx.x & 63;
    const long long id = id_at(A.ids, A.wide_ids, t);
    const bool there = id >= 0 && id < (long long)A.vocab;
    if (id >= (long long)A.vocab && lane == 0) raise_fault(A.ws, kFaultBadIndex);
    const W *w = (const W *)A.weight + (there ? (size_t)id * A.weight_stride : 0);
    O *o = (O *)A.out + t * A.out_stride;
    for (size_t i = lane; i < A.dim; i += 64) o[i] = there ? (O)((float)w[i] * A.scale) : (O)0.0f;
}

struct GradArgs {
    const void *ids, *d_out;
    void *d_weight, *ws;
    uint32_t *keys, *tokens;
    size_t n, vocab, dim, out_stride, weight_stride;
    long long padding;
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

// One workgroup per row of the table.
template <int DG, int DW> __global__ __launch_bounds__(kThreads) void row_sums_kernel(GradArgs A)
{
    typedef typename Elem<DG>::T G;
    typedef typename Elem<DW>::T W;
    const uint32_t row = blockIdx.x;
    size_t lo = 0, hi = A.n;                                   // the first pair whose key is not below the row
    while (lo < hi) {
        const size_t mid = lo + (hi - lo) / 2;
        if (A.keys[mid] < row) lo = mid + 1; else hi = mid;
    }
    size_t end = lo;
    while (end < A.n && A.keys[end] == row) ++end;
    if (A.accumulate && lo == end) return;
    W *w = (W *)A.d_weight + (size_t)row * A.weight_stride;
    for (size_t i = threadIdx.x; i < A.dim; i += kThreads) {
        float sum = 0.0f;
        for (size_t p = lo; p < end; ++p) sum += (float)((const G *)A.d_out)[(size_t)A.tokens[p] * A.out_stride + i];
        sum *= A.scale;
        w[i] = (W)(A.accumulate ? (float)w[i] + sum : sum);
    }
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
template <int W, int O> struct Lookup { static const void *fn() { return (const void *)lookup_kernel<W, O>; } };
template <int G, int W> struct RowSums { static const void *fn() { return (const void *)row_sums_kernel<G, W>; } };

// What the gradient's workspace holds, in bytes from its start.
struct GradLayout {
    size_t chain, keys, keys_tmp, tokens, tokens_tmp, flags, positions, all;
    explicit GradLayout(size_t n)
    {
        const size_t words = (4 * n + 15) / 16 * 16;
        chain = tcuscan_workspace_bytes(1, n, TCUSCAN_I8_I32);          // what the sort asks for, in each of its forms
        if (chain < chain_layout::kHeaderBytes) chain = chain_layout::kHeaderBytes;
        keys = chain;
        keys_tmp = keys + words;
        tokens = keys_tmp + words;
        tokens_tmp = tokens + words;
        positions = tokens_tmp + words;
        flags = positions + words;
        all = flags + (n + 15) / 16 * 16;
    }
};

constexpr size_t kMostRows = 0x7FFFFFFFu;

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
    const size_t blocks = (n + kThreads / 64 - 1) / (kThreads / 64);
    if (blocks > kMostRows) return TCUSCAN_ERR_UNSUPPORTED;
    LookupArgs A = {d_ids, d_weight, d_out, d_ws, n, vocab, dim, weight_stride, out_stride, scale, id_bytes == 8};
    void *args[] = {&A};
    return hipLaunchKernel(pick<Lookup>(weight_dt, out_dt), dim3((unsigned)blocks), dim3(kThreads), args, 0, (hipStream_t)stream) == hipSuccess ? TCUSCAN_OK : TCUSCAN_ERR_HIP;
}

size_t tcuscan_embedding_backward_workspace_bytes(size_t n, size_t vocab, size_t dim)
{
    return n > 0xFFFFFFFFull || vocab == 0 || vocab > kMostRows || dim == 0 ? 0 : GradLayout(n).all;
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
    const GradLayout L(n);
    if (!d_ws || ws_bytes < L.all || (uintptr_t)d_ws % 16) return TCUSCAN_ERR_WORKSPACE;
    char *ws = (char *)d_ws;
    hipStream_t s = (hipStream_t)stream;
    GradArgs A = {d_ids, d_out_grad, d_weight_grad, d_ws, (uint32_t *)(ws + L.keys), (uint32_t *)(ws + L.tokens),
                  n, vocab, dim, out_stride, weight_stride, padding, scale, id_bytes == 8, accumulate};
    void *args[] = {&A};
    if (n) {
        if (hipLaunchKernel((const void *)token_keys_kernel, dim3((unsigned)((n + kThreads - 1) / kThreads)), dim3(kThreads), args, 0, s) != hipSuccess) return TCUSCAN_ERR_HIP;
        int bits = 0;
        while (((size_t)1 << bits) <= vocab) ++bits;
        const tcuscan_status_t st = tcuscan_split_radix_sort_u32(A.keys, A.tokens, n, bits, ws + L.keys_tmp, ws + L.tokens_tmp, ws + L.flags, ws + L.positions,
                                                                 d_ws, L.chain, stream);
        if (st != TCUSCAN_OK) return st;
    }
    return hipLaunchKernel(pick<RowSums>(out_dt, weight_dt), dim3((unsigned)vocab), dim3(kThreads), args, 0, s) == hipSuccess ? TCUSCAN_OK : TCUSCAN_ERR_HIP;
}

}  // extern "C"
