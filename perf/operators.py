"""The operators of language models this library has, as cases that can be timed and checked one by one.

A case is a plain dict.  ``prepare`` makes what a program holds before the call, ``run`` is one pass: where ``own`` is false
in elementary torch operations in 32 bits, where it is true through the public entry points of
``paper_2411_17887_amd.tcuscan``; ``exact`` is the same result from the definition in 64 bits.  Five kinds of work, by ``op``:

  prompt         linear attention with one decay per head over rows of tokens stored back to back, from a state to a state:
                 S_t = a_h S_(t-1) + k_t v_t^T,  o_t = scale q_t S_t,  a_h = exp(log_decay_h)
  backward       its gradients by q, k, v and by the state that a row starts from
  step           one token for each of a batch of sequences whose states lie in a pool
  lookup         rows of an embedding table, scaled
  lookup_grad    the table's gradient: the sum of the gradients of all tokens that took a row, zeros for rows that none took
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

TORCH = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
BYTES = {"f32": 4, "f16": 2, "bf16": 2}
CHUNK = 64                                    # tokens that the plain form takes at a time


def listed():
    return [
        # A short prompt of one user: latency.
        attention("prompt_bf16_1x200", "prompt", "bf16", rows=1, total=200, heads=8, dk=64, dv=64),
        # Ragged prompts of a serving batch, keys and queries shared by two value heads each, head size no power of two.
        attention("prompt_f16_30rows_shared", "prompt", "f16", rows=30, total=20011, heads=16, q_heads=8, k_heads=8, dk=80, dv=96),
        # One long document: few rows, so the work has to be split along the tokens.
        attention("prompt_bf16_1x65536", "prompt", "bf16", rows=1, total=65536, heads=16, dk=128, dv=128),
        # A small training step in 32 bits (a test configuration, a fine-tuning run on one card).
        attention("backward_f32_2rows", "backward", "f32", rows=2, total=1027, heads=4, dk=64, dv=64),
        # Ragged documents packed into one batch, keys and values shared by four query heads each.
        attention("backward_bf16_9rows_shared", "backward", "bf16", rows=9, total=12289, heads=16, k_heads=4, v_heads=4, dk=64, dv=64),
        # A training batch of full rows.
        attention("backward_bf16_8x4096", "backward", "bf16", rows=8, total=32768, heads=16, dk=128, dv=128),
        # One user's next token.
        attention("step_bf16_1", "step", "bf16", rows=1, total=1, heads=16, dk=128, dv=128, pool=4),
        # The next tokens of a full serving batch.
        attention("step_bf16_256", "step", "bf16", rows=256, total=256, heads=16, dk=128, dv=128, pool=320),
        # The tokens of one decoding step.
        embedding("lookup_bf16_24", "lookup", "bf16", "bf16", n=24, vocab=32000, dim=2048),
        # A training batch: 32-bit weights, 16-bit activations.
        embedding("lookup_f32_bf16_65536", "lookup", "f32", "bf16", n=65536, vocab=65536, dim=1024),
        # The gradient of a small batch, rows of odd length.
        embedding("lookup_grad_f32_3001", "lookup_grad", "f32", "f32", n=3001, vocab=8000, dim=515),
        # The gradient of a training batch: frequent tokens take long runs, most of the table takes none or few.
        embedding("lookup_grad_f32_bf16_65536", "lookup_grad", "f32", "bf16", n=65536, vocab=65536, dim=1024),
    ]


def attention(name, op, kind, rows, total, heads, dk, dv, q_heads=0, k_heads=0, v_heads=0, pool=0):
    return dict(name=name, op=op, kind=kind, rows=rows, total=total, heads=heads, q_heads=q_heads or heads, k_heads=k_heads or heads,
                v_heads=v_heads or heads, dk=dk, dv=dv, pool=pool)


def embedding(name, op, weights, kind, n, vocab, dim):
    """`weights`: the type of the table or of its gradient, `kind`: that of the activations or their gradients."""
    return dict(name=name, op=op, weights=weights, kind=kind, n=n, vocab=vocab, dim=dim)


def _log_int(rng, lo, hi):
    """An integer of [lo, hi], its logarithm uniform."""
    return max(lo, min(hi, int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))))


def draw(rng):
    op = rng.choice(["prompt", "prompt", "backward", "backward", "step", "lookup", "lookup_grad"])
    kind = rng.choice(["bf16", "bf16", "f16", "f32"])
    if op in ("lookup", "lookup_grad"):
        vocab = _log_int(rng, 100, 100_000)
        dim = min(_log_int(rng, 16, 4096), (1 << 26) // vocab)
        n = _log_int(rng, 1, min(1 << 17, (1 << 26) // dim))
        case = embedding("", op, rng.choice(["f32", kind]), kind, n, vocab, dim)
    else:
        sizes = (32, 48, 64, 80, 96, 128, 192, 256)
        dk = rng.choice(sizes)
        dv = rng.choice((dk, dk, rng.choice(sizes)))
        heads = rng.choice((1, 2, 4, 6, 8, 12, 16, 32))
        shared = rng.choice([d for d in (1, 1, 2, 4) if heads % d == 0])
        which = rng.choice(["qk", "kv"])
        split = {"q": heads // shared if which == "qk" else heads, "k": heads // shared, "v": heads // shared if which == "kv" else heads}
        # no more bytes than the largest listed case of the kind
        most = {"prompt": 65536 * 16 * 128 * 8, "backward": 32768 * 16 * 128 * 14, "step": 256 * 16 * 128 * 128 * 8}[op]
        if op == "step":
            total = rows = _log_int(rng, 1, min(512, most // (heads * dk * dv * 8)))
        else:
            per_token = {"prompt": 2, "backward": 4}[op] * heads * (dk + dv) * BYTES[kind]
            total = _log_int(rng, 1, min(65536, most // per_token))
            rows = min(total, _log_int(rng, 1, 64))
        case = attention("", op, kind, rows, total, heads, dk, dv, split["q"], split["k"], split["v"], rows + rng.randrange(1, 64) if op == "step" else 0)
    del case["name"]
    return case


# ---------------------------------------------------------------- what a program holds before the call

def _lengths(rows, total, seed):
    """Lengths of `rows` rows, `total` in all: equal for few rows that divide it, a long-tailed mix otherwise, one of more than four then empty."""
    if total % rows == 0 and rows < 16:
        return [total // rows] * rows
    r = np.random.RandomState(seed % (1 << 31))
    share = r.lognormal(0.0, 0.9, rows)
    if rows > 4:
        share[r.randint(rows)] = 0.0
    cut = np.floor(np.cumsum(share) / share.sum() * total + 0.5).astype(np.int64)
    cut[-1] = total
    return np.diff(cut, prepend=0).tolist()


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)

    def normal(*shape, dtype=torch.float32, by=1.0):
        return (torch.randn(*shape, generator=g, device="cuda") * by).to(dtype)

    c = dict(case)
    kind = TORCH[c["kind"]]
    if c["op"] in ("lookup", "lookup_grad"):
        # token numbers as a text has them: the r-th most frequent one in proportion to 1 / (r + 3), numbered at random
        n, vocab, dim = c["n"], c["vocab"], c["dim"]
        weight = 1.0 / (torch.arange(vocab, device="cuda", dtype=torch.float64) + 3.0)
        edge = torch.cumsum(weight, 0)
        rank = torch.searchsorted(edge, torch.rand(n, generator=g, device="cuda", dtype=torch.float64) * edge[-1]).clamp_(max=vocab - 1)
        c["ids"] = torch.randperm(vocab, generator=g, device="cuda")[rank]
        if c["op"] == "lookup":
            c["weight"] = normal(vocab, dim, dtype=TORCH[c["weights"]], by=dim ** -0.5)
            c["out"] = torch.empty(n, dim, dtype=kind, device="cuda")
            c["scale"] = math.sqrt(dim)
        else:
            c["d_out"] = normal(n, dim, dtype=kind)
            c["d_weight"] = torch.empty(vocab, dim, dtype=TORCH[c["weights"]], device="cuda")
            c["scale"] = math.sqrt(dim)
        return c
    total, heads, dk, dv = c["total"], c["heads"], c["dk"], c["dv"]
    # queries, keys and values are slices of one projection's output, a token after the other
    qw, kw, vw = c["q_heads"] * dk, c["k_heads"] * dk, c["v_heads"] * dv
    qkv = normal(total, qw + kw + vw, dtype=kind)
    c["q"] = qkv[:, :qw].view(total, c["q_heads"], dk)
    c["k"] = qkv[:, qw:qw + kw].view(total, c["k_heads"], dk)
    c["v"] = qkv[:, qw + kw:].view(total, c["v_heads"], dv)
    c["scale"] = dk ** -0.5
    # decays from 1 - 2^-2 to 1 - 2^-9, one for each head
    c["log_decay"] = torch.log1p(-torch.pow(2.0, -2.0 - 7.0 * torch.arange(heads, device="cuda", dtype=torch.float32) / max(1, heads - 1)))
    if c["op"] == "step":
        c["state"] = normal(c["pool"], heads, dk, dv)
        c["slots"] = torch.randperm(c["pool"], generator=g, device="cuda")[:c["rows"]].contiguous()
        c["out"] = torch.empty(total, heads, dv, dtype=kind, device="cuda")
        return c
    c["lengths"] = _lengths(c["rows"], total, seed)
    c["offsets"] = torch.from_numpy(np.cumsum([0] + c["lengths"])).cuda()
    c["state_in"] = normal(c["rows"], heads, dk, dv)
    if c["op"] == "prompt":
        c["out"] = torch.empty(total, heads, dv, dtype=kind, device="cuda")
        c["state_out"] = torch.empty(c["rows"], heads, dk, dv, device="cuda")
    else:
        c["d_out"] = normal(total, heads, dv, dtype=kind)
        c["d_state_out"] = normal(c["rows"], heads, dk, dv)
        c["dq"], c["dk_"], c["dv_"] = (torch.empty(total, h, d, dtype=kind, device="cuda")
                                       for h, d in ((c["q_heads"], dk), (c["k_heads"], dk), (c["v_heads"], dv)))
        c["d_state_in"] = torch.empty(c["rows"], heads, dk, dv, device="cuda")
    return c


# ---------------------------------------------------------------- one pass

def run(c):
    return _own(c) if own else _plain(c)


def _own(c):
    from paper_2411_17887_amd import tcuscan
    op = c["op"]
    if op == "lookup":
        tcuscan.embedding(c["ids"], c["weight"], c["out"], scale=c["scale"])
        return [c["out"]]
    if op == "step":
        tcuscan.decay_attention_step(c["q"], c["k"], c["v"], c["out"], c["log_decay"], c["state"], slots=c["slots"], scale=c["scale"])
        return [c["out"], c["state"]]
    if "ws" not in c:                         # a program keeps its workspace
        if op == "lookup_grad":
            c["ws"] = tcuscan.new_embedding_backward_workspace(c["n"], c["vocab"], c["dim"])
        elif op == "prompt":
            c["ws"] = tcuscan.new_decay_attention_workspace(c["rows"], c["total"], c["heads"], c["dk"], c["dv"])
        else:
            c["ws"] = tcuscan.new_decay_attention_backward_workspace(c["rows"], c["total"], c["heads"], c["dk"], c["dv"],
                                                                     c["q_heads"], c["k_heads"], c["v_heads"])
    if op == "lookup_grad":
        tcuscan.embedding_backward(c["ids"], c["d_out"], c["d_weight"], scale=c["scale"], ws=c["ws"])
        return [c["d_weight"]]
    if op == "prompt":
        tcuscan.decay_attention(c["q"], c["k"], c["v"], c["out"], c["log_decay"], c["offsets"], scale=c["scale"],
                                state_in=c["state_in"], state_out=c["state_out"], ws=c["ws"])
        return [c["out"], c["state_out"]]
    tcuscan.decay_attention_backward(c["q"], c["k"], c["v"], c["d_out"], c["dq"], c["dk_"], c["dv_"], c["log_decay"], c["offsets"],
                                     scale=c["scale"], state_in=c["state_in"], d_state_out=c["d_state_out"],
                                     d_state_in=c["d_state_in"], ws=c["ws"])
    return [c["dq"], c["dk_"], c["dv_"], c["d_state_in"]]


def _plain(c):
    op, scale = c["op"], c["scale"]
    kind = TORCH[c["kind"]]
    if op == "lookup":
        return [(c["weight"][c["ids"]].float() * scale).to(kind)]
    if op == "lookup_grad":
        d_weight = torch.zeros(c["vocab"], c["dim"], device="cuda")
        return [d_weight.index_add_(0, c["ids"], c["d_out"].float() * scale).to(TORCH[c["weights"]])]
    heads = c["heads"]
    q, k, v = (x.float().repeat_interleave(heads // x.shape[1], dim=1) for x in (c["q"], c["k"], c["v"]))
    if op == "step":
        a = torch.exp(c["log_decay"])[:, None, None]
        new = a * c["state"][c["slots"]] + k[..., :, None] * v[..., None, :]
        c["state"][c["slots"]] = new
        return [((q[..., :, None] * new).sum(-2) * scale).to(kind), c["state"]]
    chunks = _chunks(c)
    if op == "prompt":
        o, state = _mix(c, chunks, q, k, v, c["state_in"], False)
        return [(o * scale).to(kind), state]
    do = c["d_out"].float() * scale           # o = scale q S: the gradient by q S
    turned = c["state_in"].transpose(-1, -2)
    d_turned = c["d_state_out"].transpose(-1, -2)
    dq, _ = _mix(c, chunks, do, v, k, turned, False)
    dv, d_state = _mix(c, chunks, k, q, do, c["d_state_out"], True)
    dk, _ = _mix(c, chunks, v, do, q, d_turned, True)
    grads = [x.view(x.shape[0], x_heads, heads // x_heads, -1).sum(2).to(kind)
             for x, x_heads in ((dq, c["q_heads"]), (dk, c["k_heads"]), (dv, c["v_heads"]))]
    return grads + [d_state]


def _chunks(c):
    """Where each token goes when every row is cut into chunks of its own: its place, the chunk's row and number in it."""
    lengths = np.array(c["lengths"])
    counts = -(-lengths // CHUNK)
    n = int(counts.sum())
    row = torch.from_numpy(np.repeat(np.arange(len(lengths)), counts)).cuda()
    first = torch.from_numpy(np.cumsum(counts) - counts).cuda()
    number = torch.arange(n, device="cuda") - first[row]
    token_row = torch.from_numpy(np.repeat(np.arange(len(lengths)), lengths)).cuda()
    place = torch.arange(c["total"], device="cuda") - c["offsets"][token_row]
    at = first[token_row] * CHUNK + place
    return dict(n=n, row=row, number=number, at=at, lengths=torch.from_numpy(lengths).cuda())


def _mix(c, chunks, x, y, z, init, reverse):
    """Linear attention with queries x, keys y, values z and the state `init` of each row, from the front or from the end:
    (x_t (sum over s <= t of a^(t-s) y_s z_s^T + a^(t+1) init)), and the state behind the row.  From the end, where nothing
    has decayed before the last token's reading, x_t (sum over s >= t of a^(s-t) y_s z_s^T + a^(T-1-t) init)."""
    n, row, at = chunks["n"], chunks["row"], chunks["at"]
    heads = x.shape[1]
    log_a = c["log_decay"][:, None]

    def padded(t):
        p = torch.zeros(n * CHUNK, heads, t.shape[2], device="cuda")
        p[at] = t
        return p.view(n, CHUNK, heads, -1).transpose(1, 2)                       # chunk, head, token, feature

    def power(exponents):
        """a_h to the given exponents: [heads, ...] or, for an exponent of each chunk, [chunks, heads, ...]."""
        return torch.exp(log_a * exponents[..., None, :].float())

    x, y, z = padded(x), padded(y), padded(z)
    i = torch.arange(CHUNK, device="cuda")
    apart = (i[None, :] - i[:, None] if reverse else i[:, None] - i[None, :])    # query's place against key's
    weight = torch.exp(log_a[..., None] * apart.clamp(min=0).float()) * (apart >= 0)
    o = torch.matmul(torch.matmul(x, y.transpose(-1, -2)) * weight, z)
    to_edge = i if reverse else CHUNK - 1 - i
    added = torch.matmul((y * power(to_edge)[..., None]).transpose(-1, -2), z)   # what a chunk adds, as its edge sees it
    number = chunks["number"]
    between = number[None, :] - number[:, None] if reverse else number[:, None] - number[None, :]
    link = (row[None, :] == row[:, None]) & (between > 0)
    link = torch.exp(log_a[..., None] * ((between - 1) * CHUNK).clamp(min=0).float()) * link
    before = torch.matmul(link, added.transpose(0, 1).reshape(heads, n, -1)).view(heads, n, *added.shape[2:]).transpose(0, 1)
    reading = CHUNK - i if reverse else i + 1
    o += torch.matmul(x, before) * power(reading)[..., None]
    place = number[:, None] * CHUNK + i[None, :]
    to_end = chunks["lengths"][row][:, None] - 1 - place
    o += torch.matmul(x, init[row]) * power((to_end if reverse else place + 1).clamp(min=0))[..., None]
    whole = power((place + 1 if reverse else to_end).clamp(min=0))[..., None]
    state = torch.exp(log_a * chunks["lengths"].float()).T[..., None, None] * init
    state = state.index_add(0, row, torch.matmul((y * whole).transpose(-1, -2), z))
    return o.transpose(1, 2).reshape(n * CHUNK, heads, -1)[at], state


# ---------------------------------------------------------------- what a pass cannot do without

def work(case):
    c = case
    if c["op"] in ("lookup", "lookup_grad"):
        n, dim = c["n"], c["dim"]
        if c["op"] == "lookup":
            often = 1.0 / (np.arange(c["vocab"]) + 3.0)
            taken = float(np.sum(-np.expm1(n * np.log1p(-often / often.sum()))))         # table rows that are read, on average
            return {"bytes": 8 * n + taken * dim * BYTES[c["weights"]] + n * dim * BYTES[c["kind"]], "flops": n * dim}
        return {"bytes": 8 * n + n * dim * BYTES[c["kind"]] + c["vocab"] * dim * BYTES[c["weights"]], "flops": n * dim}
    heads, dk, dv, total = c["heads"], c["dk"], c["dv"], c["total"]
    ins = total * (c["q_heads"] * dk + c["k_heads"] * dk + c["v_heads"] * dv) * BYTES[c["kind"]]
    out = total * heads * dv * BYTES[c["kind"]]
    states = c["rows"] * heads * dk * dv * 4
    if c["op"] == "backward":                 # two states kept up and three readings of them for each token
        return {"bytes": 2 * ins + out + 3 * states, "flops": 10 * total * heads * dk * dv}
    return {"bytes": ins + out + 2 * states, "flops": 4 * total * heads * dk * dv}


# ---------------------------------------------------------------- the definition in 64 bits

def exact(case, seed):
    c = prepare(case, seed)
    op, scale = c["op"], c["scale"]
    if op == "lookup":
        return [c["weight"].double().index_select(0, c["ids"]) * scale]
    if op == "lookup_grad":
        d_out, order = c["d_out"].double(), torch.argsort(c["ids"], stable=True)
        sums = torch.cumsum(d_out[order], 0)
        ids, last = torch.unique_consecutive(c["ids"][order], return_counts=True)
        sums = sums[torch.cumsum(last, 0) - 1]
        sums[1:] = sums[1:] - sums[:-1].clone()
        d_weight = torch.zeros(c["vocab"], c["dim"], dtype=torch.float64, device="cuda")
        d_weight[ids] = sums * scale
        return [d_weight]
    heads, dk, dv = c["heads"], c["dk"], c["dv"]
    decay = c["log_decay"].double()
    q, k, v = ([x[:, h * x.shape[1] // heads].double() for h in range(heads)] for x in (c["q"], c["k"], c["v"]))
    if op == "step":
        state = c["state"].double()
        out = torch.empty(c["total"], heads, dv, dtype=torch.float64, device="cuda")
        for h in range(heads):
            new = math.exp(float(decay[h])) * state[c["slots"], h] + k[h].unsqueeze(2) * v[h].unsqueeze(1)
            state[c["slots"], h] = new
            out[:, h] = (new * q[h].unsqueeze(2)).sum(1) * scale
        return [out, state]
    states = torch.empty(c["rows"], heads, dk, dv, dtype=torch.float64, device="cuda")
    if op == "prompt":
        out = torch.empty(c["total"], heads, dv, dtype=torch.float64, device="cuda")
    else:
        dq, dk_, dv_ = (torch.zeros(c["total"], h, d, dtype=torch.float64, device="cuda")
                        for h, d in ((c["q_heads"], dk), (c["k_heads"], dk), (c["v_heads"], dv)))
    lo = 0
    for r, length in enumerate(c["lengths"]):
        t = torch.arange(length, device="cuda", dtype=torch.float64)
        for h in range(heads):
            qh, kh, vh = q[h][lo:lo + length], k[h][lo:lo + length], v[h][lo:lo + length]
            s0, g = c["state_in"][r, h].double(), decay[h]
            up, down = torch.exp(g * (t + 1))[:, None], torch.exp(g * (length - 1 - t))[:, None]
            if op == "prompt":
                states[r, h] = math.exp(float(g) * length) * s0 + (kh * down).T @ vh
                out[lo:lo + length, h] = up * (qh @ s0) * scale
            else:
                doh, ds = c["d_out"][lo:lo + length, h].double(), c["d_state_out"][r, h].double()
                gq, gk, gv = up * (doh @ s0.T) * scale, down * (vh @ ds.T), down * (kh @ ds)
                states[r, h] = math.exp(float(g) * length) * ds + scale * (qh * up).T @ doh
            for b in range(0, length, 4096):                                     # queries of a block against all keys up to it
                e = min(length, b + 4096)
                apart = t[b:e, None] - t[None, :e]
                w = torch.where(apart >= 0, torch.exp(g * apart.clamp(min=0)), 0.0) * scale
                p = (qh[b:e] @ kh[:e].T) * w
                if op == "prompt":
                    out[lo + b:lo + e, h] += p @ vh[:e]
                else:
                    dp = (doh[b:e] @ vh[:e].T) * w
                    gq[b:e] += dp @ kh[:e]
                    gk[:e] += dp.T @ qh[b:e]
                    gv[:e] += p.T @ doh[b:e]
            if op == "backward":
                for whole, part in ((dq, gq), (dk_, gk), (dv_, gv)):
                    whole[lo:lo + length, h * whole.shape[1] // heads] += part
        lo += length
    return [out, states] if op == "prompt" else [dq, dk_, dv_, states]
