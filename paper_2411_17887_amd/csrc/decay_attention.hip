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

#include "../../include/tcuscan.h"
#include "chain_layout.h"
#include "element_types.h"

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
    void *ws;
    long long states;                              // how many states there are
    long long total;
    unsigned rows, heads, A, E;
    unsigned m_a, m_e;                             // strides of a state: M[a][e] is at a * m_a + e * m_e
    float by_new, by_read;
    int from_end;
};

// a^n, for weights.  (An n of 0 gives 1 for a decay of 0, a log_decay of minus infinity, too.)
__device__ __forceinline__ float decay_power(float log_decay, float n) { return __expf(fmaxf(log_decay, -1e30f) * n); }
// Takes a state n tokens on: m becomes a^n m.  Slow decays (a^n from 1/2 on) as m + (a^n - 1) m: multiplied by a rounded a^n, a state
// would be off by up to half a unit in the last place of 1 each time, always to the same side: 1e-5 for 1 - 2^-9 token by token.
struct Decay {
    float by, keep;
    __device__ __forceinline__ Decay(float log_decay, float n)
    {
        const float x = fmaxf(log_decay, -1e30f) * n;
        keep = x > -0.69f ? 1.0f : 0.0f;
        by = x > -0.69f ? expm1f(x) : __expf(x);
    }
    __device__ __forceinline__ float operator()(float m) const { return fmaf(m, by, keep * m); }
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

// The walk token by token: a workgroup of one wavefront per (row, head, 64 columns), the state in LDS.
template <int DT, int DO> __global__ __launch_bounds__(64) void walk_kernel(WalkArgs W)
{
    typedef typename Elem<DT>::T T;
    typedef typename Elem<DO>::T O;
    __shared__ float m[kMaxDim][64];
    const unsigned blocks = (W.E + 63) / 64;
    const unsigned e = blockIdx.x % blocks * 64 + threadIdx.x, h = blockIdx.x / blocks % W.heads, r = blockIdx.x / blocks / W.heads;
    const int col = threadIdx.x;
    long long lo, hi;
    row_extent(W.offsets, r, W.total, lo, hi);
    if (threadIdx.x == 0) {
        const long long a = W.offsets[r], b = W.offsets[r + 1];
        if (a < 0 || b < a || b > W.total) raise_fault(W.ws, kFaultBadIndex);
        if (W.slots && W.slots[r] >= W.states) raise_fault(W.ws, kFaultBadIndex);
    }
    if (e >= W.E) return;                          // (lanes work on columns of their own; nothing is waited for)
    const long long slot = state_of(W.slots, r, W.states);
    const size_t state = ((size_t)slot * W.heads + h) * W.A * W.E;
    for (unsigned a = 0; a < W.A; ++a) m[a][col] = W.m_in && slot >= 0 ? W.m_in[state + (size_t)a * W.m_a + (size_t)e * W.m_e] : 0.0f;
    const Decay decay(W.log_decay[h], 1.0f);
    const T *x = (const T *)W.x.data + W.x.at(h, W.heads), *y = (const T *)W.y.data + W.y.at(h, W.heads), *z = (const T *)W.z.data + W.z.at(h, W.heads);
    O *out = (O *)W.out.data + W.out.at(h, W.heads);
    for (long long i = 0; i < hi - lo; ++i) {
        const long long t = W.from_end ? hi - 1 - i : lo + i;
        const T *xt = x + t * W.x.token, *yt = y + t * W.y.token;
        const float zt = (float)z[t * W.z.token + e] * W.by_new;
        float sum = 0.0f;
        for (unsigned a = 0; a < W.A; ++a) {
            float v = m[a][col];
            if (!W.from_end) v = decay(v);
            v += (float)yt[a] * zt;
            sum += (float)xt[a] * v;
            if (W.from_end) v = decay(v);
            m[a][col] = v;
        }
        out[t * W.out.token + e] = (O)(sum * W.by_read);
    }
    if (W.m_out && slot >= 0)
        for (unsigned a = 0; a < W.A; ++a) W.m_out[state + (size_t)a * W.m_a + (size_t)e * W.m_e] = m[a][col];
}

// out[t][stored head][i] = the sum of part[t][head][i] over the heads that share the stored head.
struct SumArgs {
    const float *part;
    Heads out;
    long long total;
    unsigned heads, D;
};
constexpr int kSumThreads = 256;
template <int DT> __global__ __launch_bounds__(kSumThreads) void sum_heads_kernel(SumArgs S)
{
    typedef typename Elem<DT>::T T;
    const size_t i = (size_t)blockIdx.x * kSumThreads + threadIdx.x;
    if (i >= (size_t)S.total * S.out.heads * S.D) return;
    const unsigned d = (unsigned)(i % S.D), h = (unsigned)(i / S.D % S.out.heads), group = S.heads / S.out.heads;
    const long long t = (long long)(i / S.D / S.out.heads);
    const float *p = S.part + ((size_t)t * S.heads + (size_t)h * group) * S.D + d;
    float sum = 0.0f;
    for (unsigned g = 0; g < group; ++g) sum += p[(size_t)g * S.D];
    ((T *)S.out.data)[t * S.out.token + (long long)h * S.out.head + d] = (T)sum;
}

// One token for each of many sequences: a workgroup per (sequence, head), lanes along the state's rows (dv).
struct StepArgs {
    Heads q, k, v, out;
    const float *log_decay;
    const long long *slots;
    float *state;
    void *ws;
    long long states;
    unsigned n, heads, A, E;
    float scale;
};
template <int DT> __global__ __launch_bounds__(256) void step_kernel(StepArgs S)
{
    typedef typename Elem<DT>::T T;
    const unsigned h = blockIdx.x % S.heads, i = blockIdx.x / S.heads;
    const long long slot = state_of(S.slots, i, S.states);
    if (threadIdx.x == 0 && S.slots && S.slots[i] >= S.states) raise_fault(S.ws, kFaultBadIndex);
    const T *q = (const T *)S.q.data + S.q.at(h, S.heads) + i * S.q.token, *k = (const T *)S.k.data + S.k.at(h, S.heads) + i * S.k.token,
            *v = (const T *)S.v.data + S.v.at(h, S.heads) + i * S.v.token;
    T *out = (T *)S.out.data + S.out.at(h, S.heads) + i * S.out.token;
    const unsigned e = threadIdx.x;
    if (e >= S.E) return;
    const Decay decay(S.log_decay[h], 1.0f);
    const float ve = (float)v[e];
    float sum = 0.0f;
    float *m = S.state + ((size_t)(slot < 0 ? 0 : slot) * S.heads + h) * S.A * S.E + e;
    for (unsigned a = 0; a < S.A; ++a) {
        const float old = slot < 0 ? 0.0f : m[(size_t)a * S.E], s = decay(old) + (float)k[a] * ve;
        if (slot >= 0) m[(size_t)a * S.E] = s;
        sum += (float)q[a] * s;
    }
    out[e] = (T)(sum * S.scale);
}

bool launch(const void *fn, size_t grid, unsigned block, void *args, hipStream_t s)
{
    void *list[] = {args};
    return hipLaunchKernel(fn, dim3((unsigned)grid), dim3(block), list, 0, s) == hipSuccess;
}

template <template <int> class Pick> const void *pick(int dt) { return dt == kF16 ? Pick<kF16>::fn() : dt == kF32 ? Pick<kF32>::fn() : Pick<kBF16>::fn(); }
template <int DT> struct WalkSame { static const void *fn() { return (const void *)walk_kernel<DT, DT>; } };
template <int DT> struct WalkWide { static const void *fn() { return (const void *)walk_kernel<DT, kF32>; } };
template <int DT> struct SumHeads { static const void *fn() { return (const void *)sum_heads_kernel<DT>; } };
template <int DT> struct Step { static const void *fn() { return (const void *)step_kernel<DT>; } };

constexpr size_t kMostBlocks = 0x7FFFFFFFu;

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
    if (s.rows > 0x3FFFFFFF || s.heads > 0xFFFF || (unsigned long long)s.rows * s.heads > kMostBlocks / 8) return TCUSCAN_ERR_UNSUPPORTED;
    return TCUSCAN_OK;
}

struct Layout {
    size_t part, all;
    Layout(const tcuscan_attention_shape_t &s, bool backward)
    {
        part = chain_layout::kHeaderBytes;
        size_t wide = 0;
        if (backward) {
            if (s.q_heads < s.heads || s.k_heads < s.heads) wide = (size_t)s.dk;
            if (s.v_heads < s.heads && (size_t)s.dv > wide) wide = (size_t)s.dv;
        }
        all = part + (size_t)s.total * s.heads * wide * 4;
    }
};

bool misaligned(const void *p, size_t to) { return (uintptr_t)p % to != 0; }

Heads heads_of(const void *data, long long token, long long head, long long heads) { return {(void *)data, token, head, (unsigned)heads}; }

// One walk, into `out`; with heads that share the output, into `part` first.
tcuscan_status_t walk(WalkArgs W, Heads out, float *part, int dt, hipStream_t s)
{
    const size_t grid = (size_t)W.rows * W.heads * ((W.E + 63) / 64);
    const bool shared = out.heads < W.heads;
    W.out = shared ? Heads{part, (long long)W.heads * W.E, W.E, W.heads} : out;
    if (!launch(shared ? pick<WalkWide>(dt) : pick<WalkSame>(dt), grid, 64, &W, s)) return TCUSCAN_ERR_HIP;
    if (!shared) return TCUSCAN_OK;
    SumArgs S = {part, out, W.total, W.heads, W.E};
    const size_t items = (size_t)W.total * out.heads * W.E;
    if (!items) return TCUSCAN_OK;
    return launch(pick<SumHeads>(dt), (items + kSumThreads - 1) / kSumThreads, kSumThreads, &S, s) ? TCUSCAN_OK : TCUSCAN_ERR_HIP;
}

}  // namespace

extern "C" {

size_t tcuscan_decay_attention_workspace_bytes(const tcuscan_attention_shape_t *shape, tcuscan_dtype_t dt, int backward)
{
    return check_shape(shape, dt) != TCUSCAN_OK ? 0 : Layout(*shape, backward != 0).all;
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
    const Layout L(p, false);
    if (!d_ws || ws_bytes < L.all || misaligned(d_ws, 16)) return TCUSCAN_ERR_WORKSPACE;
    WalkArgs W = {};
    W.x = heads_of(d_q, p.q_token, p.q_head, p.q_heads);
    W.y = heads_of(d_k, p.k_token, p.k_head, p.k_heads);
    W.z = heads_of(d_v, p.v_token, p.v_head, p.v_heads);
    W.log_decay = d_log_decay; W.offsets = d_offsets; W.slots = d_slots; W.m_in = d_state_in; W.m_out = d_state_out; W.ws = d_ws;
    W.states = (long long)states; W.total = p.total; W.rows = (unsigned)p.rows; W.heads = (unsigned)p.heads;
    W.A = (unsigned)p.dk; W.E = (unsigned)p.dv; W.m_a = W.E; W.m_e = 1;
    W.by_new = 1.0f; W.by_read = scale; W.from_end = 0;
    return walk(W, heads_of(d_out, p.o_token, p.o_head, p.heads), nullptr, dt, (hipStream_t)stream);
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
    const Layout L(p, true);
    if (!d_ws || ws_bytes < L.all || misaligned(d_ws, 16)) return TCUSCAN_ERR_WORKSPACE;
    float *part = (float *)((char *)d_ws + L.part);
    hipStream_t s = (hipStream_t)stream;
    const Heads q = heads_of(d_q, p.q_token, p.q_head, p.q_heads), k = heads_of(d_k, p.k_token, p.k_head, p.k_heads),
                v = heads_of(d_v, p.v_token, p.v_head, p.v_heads), o = heads_of(d_out_grad, p.o_token, p.o_head, p.heads);
    WalkArgs W = {};
    W.log_decay = d_log_decay; W.offsets = d_offsets; W.ws = d_ws;
    W.states = p.rows; W.total = p.total; W.rows = (unsigned)p.rows; W.heads = (unsigned)p.heads;
    const unsigned dk = (unsigned)p.dk, dv = (unsigned)p.dv;
    // dq, with the states of the forward pass
    W.x = o; W.y = v; W.z = k; W.A = dv; W.E = dk; W.m_a = 1; W.m_e = dv; W.m_in = d_state_in;
    W.by_new = 1.0f; W.by_read = scale; W.from_end = 0;
    tcuscan_status_t r = walk(W, heads_of(d_q_grad, p.dq_token, p.dq_head, p.q_heads), part, dt, s);
    if (r != TCUSCAN_OK) return r;
    // dk, dv and the gradient by the first states, from the end
    W.by_new = scale; W.by_read = 1.0f; W.from_end = 1; W.m_in = d_state_out_grad;
    W.x = v; W.y = o; W.z = q;
    r = walk(W, heads_of(d_k_grad, p.dk_token, p.dk_head, p.k_heads), part, dt, s);
    if (r != TCUSCAN_OK) return r;
    W.x = k; W.y = q; W.z = o; W.A = dk; W.E = dv; W.m_a = dv; W.m_e = 1; W.m_out = d_state_in_grad;
    return walk(W, heads_of(d_v_grad, p.dv_token, p.dv_head, p.v_heads), part, dt, s);
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
    StepArgs S = {heads_of(d_q, p.q_token, p.q_head, p.q_heads), heads_of(d_k, p.k_token, p.k_head, p.k_heads), heads_of(d_v, p.v_token, p.v_head, p.v_heads),
                  heads_of(d_out, p.o_token, p.o_head, p.heads), d_log_decay, d_slots, d_state, d_ws, (long long)states,
                  (unsigned)p.rows, (unsigned)p.heads, (unsigned)p.dk, (unsigned)p.dv, scale};
    return launch(pick<Step>(dt), (size_t)p.rows * p.heads, 256, &S, (hipStream_t)stream) ? TCUSCAN_OK : TCUSCAN_ERR_HIP;
}

}  // extern "C"
