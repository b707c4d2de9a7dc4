"""Linear attention with decays on the GPU (prompt, gradients, single tokens) against the definition in 64 bits: types, shared heads, ragged
rows from no token to many, sizes that are no multiple of anything, strides, states by slot, decays of 0 and 1."""
import numpy as np
import pytest

import attention_reference as ref
from paper_2411_17887_amd import tcuscan

pytestmark = pytest.mark.gpu

NONE = object()


class Case:
    """Inputs on the GPU with their values in 64 bits.  `gap` unused tokens, all NaN, lie in front of the rows and behind them."""

    def __init__(self, kind, lengths, heads=(2, 2, 2), all_heads=None, dk=32, dv=32, decays=None, packed=False, gap=0, seed=1, states=True, scale=0.3):
        import torch
        self.kind, self.dt = kind, {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}[kind]
        g = torch.Generator().manual_seed(seed)
        self.heads = all_heads or max(heads)
        total = sum(lengths) + 2 * gap
        self.offsets = np.cumsum([gap] + list(lengths))
        self.rows, self.total, self.dk, self.dv, self.scale, self.longest = len(lengths), total, dk, dv, scale, max(lengths, default=0)
        widths = [heads[0] * dk, heads[1] * dk, heads[2] * dv]
        if packed:                                             # slices of one array, features offset by 3 elements
            whole = torch.full((total, sum(widths) + 3), float("nan"), dtype=self.dt)
            at = [3, 3 + widths[0], 3 + widths[0] + widths[1]]
            hosts = [whole[:, a:a + w] for a, w in zip(at, widths)]
        else:
            hosts = [torch.full((total, w), float("nan"), dtype=self.dt) for w in widths]
        for x, w in zip(hosts, widths):
            x[gap:total - gap] = torch.randn(total - 2 * gap, w, generator=g).to(self.dt)
        dims = (dk, dk, dv)
        self.host = [x.reshape(total, h, d).double().numpy() for x, h, d in zip(hosts, heads, dims)]
        if packed:
            dev = whole.cuda()
            self.qkv = [dev[:, a:a + w].view(total, h, d) for a, w, h, d in zip(at, widths, heads, dims)]
        else:
            self.qkv = [x.cuda().view(total, h, d) for x, h, d in zip(hosts, heads, dims)]
        decays = list(decays) if decays is not None else [1.0 - 2.0 ** -(2 + 6 * h / max(1, self.heads - 1)) for h in range(self.heads)]
        self.g = torch.tensor(np.log(np.maximum(decays, 0.0), where=np.array(decays) > 0, out=np.full(len(decays), -np.inf)), dtype=torch.float32)
        self.log_decay = self.g.cuda()
        self.offs = torch.from_numpy(self.offsets).cuda()
        shape = (self.rows, self.heads, dk, dv)
        self.s0 = torch.randn(*shape, generator=g) if states else torch.zeros(*shape)
        self.ds = torch.randn(*shape, generator=g) if states else torch.zeros(*shape)
        self.do = torch.full((total, self.heads, dv), float("nan"), dtype=self.dt)
        self.do[gap:total - gap] = torch.randn(total - 2 * gap, self.heads, dv, generator=g).to(self.dt)
        self.states = states
        self.features = max(dk, dv)

    def forward(self, ws=None, stream=None):
        import torch
        out = torch.full((self.total, self.heads, self.dv), -77.0, dtype=self.dt, device="cuda")
        state_out = torch.full((self.rows, self.heads, self.dk, self.dv), -77.0, device="cuda")
        ws = tcuscan.new_decay_attention_workspace(self.rows, self.total, self.heads, self.dk, self.dv, dt=self.kind) if ws is None else ws
        tcuscan.decay_attention(*self.qkv, out, self.log_decay, self.offs, scale=self.scale, state_in=self.s0.cuda() if self.states else None,
                                state_out=state_out, ws=ws, stream=stream)
        torch.cuda.synchronize()
        assert tcuscan.workspace_fault(ws) == 0
        return out, state_out

    def check_forward(self, out, state_out):
        args = (*self.host, self.g.double().numpy(), self.offsets, self.scale, self.s0.numpy())
        (want, want_state), (size, size_state) = ref.forward(*args), ref.forward(*args, absolute=True)
        got = out.float().cpu().numpy()
        lo, hi = self.offsets[0], self.offsets[-1]
        assert (got[:lo] == -77.0).all() and (got[hi:] == -77.0).all()
        ref.close(got, want, size, self.kind, self.longest, self.features)
        ref.close(state_out.cpu().numpy(), want_state, size_state, self.kind, self.longest, self.features, state=True)

    def backward(self, ws=None):
        import torch
        grads = [torch.full(x.shape, -77.0, dtype=self.dt, device="cuda") for x in self.qkv]
        d_in = torch.full((self.rows, self.heads, self.dk, self.dv), -77.0, device="cuda")
        if ws is None:
            ws = tcuscan.new_decay_attention_backward_workspace(self.rows, self.total, self.heads, self.dk, self.dv, *(x.shape[1] for x in self.qkv), dt=self.kind)
        tcuscan.decay_attention_backward(*self.qkv, self.do.cuda(), *grads, self.log_decay, self.offs, scale=self.scale,
                                         state_in=self.s0.cuda() if self.states else None, d_state_out=self.ds.cuda() if self.states else None,
                                         d_state_in=d_in, ws=ws)
        torch.cuda.synchronize()
        assert tcuscan.workspace_fault(ws) == 0
        return *grads, d_in

    def check_backward(self, *got):
        args = (*self.host, self.g.double().numpy(), self.offsets, self.scale, self.s0.numpy(), self.do.double().numpy(), self.ds.numpy())
        want, size = ref.backward(*args), ref.backward(*args, absolute=True)
        lo, hi = self.offsets[0], self.offsets[-1]
        for x, w, s in list(zip(got, want, size))[:3]:
            x = x.float().cpu().numpy()
            assert (x[:lo] == -77.0).all() and (x[hi:] == -77.0).all()
            ref.close(x, w, s, self.kind, self.longest, self.features)
        ref.close(got[3].cpu().numpy(), want[3], size[3], self.kind, self.longest, self.features, state=True)


KINDS = ["bf16", "f16", "f32"]
LENGTHS = [[1], [0], [0, 0, 5, 0], [63, 64, 65], [1, 2, 3, 31, 32, 33, 0, 127, 128, 129], [700], [257, 0, 511]]
DIMS = [(1, 1), (16, 48), (33, 65), (64, 64), (80, 96), (128, 128), (7, 256), (256, 31), (256, 256)]
HEADS = [(1, 1, 1), (4, 4, 4), (2, 2, 4), (4, 2, 2), (6, 3, 2), (1, 6, 1)]


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("lengths", LENGTHS, ids=str)
def test_rows_of_all_lengths(kind, lengths):
    c = Case(kind, lengths, heads=(2, 2, 2), dk=48, dv=40, gap=3, packed=True)
    c.check_forward(*c.forward())
    c.check_backward(*c.backward())


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("dk,dv", DIMS)
def test_features_of_all_sizes(kind, dk, dv):
    c = Case(kind, [70, 1, 130], heads=(2, 2, 2), dk=dk, dv=dv, seed=2)
    c.check_forward(*c.forward())
    c.check_backward(*c.backward())


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("heads", HEADS, ids=str)
def test_shared_heads_and_their_gradients(kind, heads):
    c = Case(kind, [100, 0, 67], heads=heads, all_heads=12 if heads == (6, 3, 2) else None, dk=64, dv=32, packed=True, seed=3)
    c.check_forward(*c.forward())
    c.check_backward(*c.backward())


@pytest.mark.parametrize("kind", KINDS)
def test_a_long_row_and_slow_decays(kind):
    c = Case(kind, [3333], heads=(3, 3, 3), dk=64, dv=64, decays=[1.0, 1.0 - 2.0 ** -12, 0.5], seed=4)
    c.check_forward(*c.forward())
    c.check_backward(*c.backward())


@pytest.mark.parametrize("kind", KINDS)
def test_decays_of_zero_and_one_and_without_states(kind):
    for states in (True, False):
        c = Case(kind, [0, 150, 64], heads=(4, 4, 4), dk=32, dv=64, decays=[0.0, 1.0, 1e-30, 1.001], seed=5, states=states)
        c.check_forward(*c.forward())
        c.check_backward(*c.backward())


def test_many_rows_of_few_tokens():
    rng = np.random.RandomState(6)
    c = Case("bf16", rng.randint(0, 9, 700).tolist(), heads=(2, 2, 2), dk=16, dv=16, seed=6)
    c.check_forward(*c.forward())
    c.check_backward(*c.backward())


@pytest.mark.parametrize("kind", KINDS)
def test_gradients_against_differences(kind):
    """The result is linear in q, in k and in v, so differences are exact but for rounding: (L(x + d) - L(x - d)) / 2 = <dx, d>, with
    L = <do, o> + <ds, S>, the forward pass in 64 bits.  The allowance is the gradients' own rounding, as in close()."""
    c = Case(kind, [90, 37], heads=(4, 2, 2), dk=32, dv=48, seed=7)
    grads = [g.double().cpu().numpy() for g in c.backward()]
    args = (c.g.double().numpy(), c.offsets, c.scale)
    size = ref.backward(*c.host, *args, c.s0.numpy(), c.do.double().numpy(), c.ds.numpy(), absolute=True)
    rng = np.random.RandomState(7)
    inputs = [*c.host, c.s0.double().numpy()]
    for i, grad in enumerate(grads):
        d = rng.standard_normal(inputs[i].shape)
        loss = []
        for sign in (1, -1):
            x = [a + sign * d if j == i else a for j, a in enumerate(inputs)]
            o, s = ref.forward(*x[:3], *args, x[3])
            loss.append((o * c.do.double().numpy()).sum() + (s * c.ds.double().numpy()).sum())
        state = i == 3
        inside = ref.UNIT["f32" if state else kind] + (2.0 ** -21 if state else ref.INNER[kind]) + (c.features + 64 + 90 / 16) * 2.0 ** -24
        assert abs((loss[0] - loss[1]) / 2 - (grad * d).sum()) <= inside * (size[i] * np.abs(d)).sum()


def test_states_by_slot_and_in_place():
    """Row r starts from and ends in state slots[r] of one array; rows without a state start from zeros; other states are not touched."""
    import torch
    c = Case("bf16", [70, 5, 0, 200], heads=(2, 2, 2), dk=32, dv=32, seed=8)
    pool = torch.randn(6, 2, 32, 32, generator=torch.Generator().manual_seed(9))
    slots = [4, -1, 0, 2]
    dev, out = pool.cuda(), torch.empty(c.total, 2, 32, dtype=c.dt, device="cuda")
    ws = tcuscan.new_decay_attention_workspace(c.rows, c.total, 2, 32, 32)
    tcuscan.decay_attention(*c.qkv, out, c.log_decay, c.offs, scale=c.scale, state_in=dev, state_out=dev, slots=torch.tensor(slots).cuda(), ws=ws)
    torch.cuda.synchronize()
    assert tcuscan.workspace_fault(ws) == 0
    for r, s in enumerate(slots):
        c.s0[r] = pool[s] if s >= 0 else 0.0
    got = torch.stack([dev[s] if s >= 0 else torch.zeros_like(dev[0]) for s in slots])
    args = (*c.host, c.g.double().numpy(), c.offsets, c.scale, c.s0.numpy())
    (want, want_state), (size, size_state) = ref.forward(*args), ref.forward(*args, absolute=True)
    ref.close(out.float().cpu().numpy(), want, size, "bf16", c.longest, c.features)
    kept = [r for r, s in enumerate(slots) if s >= 0]
    ref.close(got.cpu().numpy()[kept], want_state[kept], size_state[kept], "bf16", c.longest, c.features, state=True)
    for s in (1, 3, 5):
        assert torch.equal(dev[s].cpu(), pool[s])


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("heads,dk,dv", [((3, 3, 3), 128, 128), ((4, 2, 2), 64, 64), ((2, 2, 4), 33, 65), ((1, 1, 1), 1, 1), ((1, 2, 1), 256, 256), ((2, 2, 2), 7, 130)])
@pytest.mark.parametrize("n", [1, 5, 90])
def test_single_tokens(kind, heads, dk, dv, n):
    """One token for each sequence, three in a row, with states by slot; a sequence without a state reads only its own token."""
    import torch
    c = Case(kind, [1] * n, heads=heads, dk=dk, dv=dv, packed=True, seed=10 + n)
    all_heads = max(heads)
    pool = torch.randn(n + 3, all_heads, dk, dv, generator=torch.Generator().manual_seed(11))
    slots = np.random.RandomState(n).permutation(n + 3)[:n]
    if n > 1:
        slots[n // 2] = -5
    dev, d_slots, states = pool.cuda(), torch.from_numpy(slots).cuda(), pool.double().numpy()
    ws = torch.zeros(32, dtype=torch.int64, device="cuda")
    for _ in range(3):
        out = torch.full((n, all_heads, dv), -77.0, dtype=c.dt, device="cuda")
        tcuscan.decay_attention_step(*c.qkv, out, c.log_decay, dev, slots=d_slots, scale=c.scale, ws=ws)
        torch.cuda.synchronize()
        s0 = np.stack([states[s] if s >= 0 else np.zeros_like(states[0]) for s in slots])
        args = (*c.host, c.g.double().numpy(), c.offsets, c.scale, s0)
        (want, want_state), (size, size_state) = ref.forward(*args), ref.forward(*args, absolute=True)
        ref.close(out.float().cpu().numpy(), want, size, kind, 1, max(dk, dv))
        got = dev.cpu().numpy()
        for i, s in enumerate(slots):
            if s >= 0:
                ref.close(got[s], want_state[i], size_state[i], kind, 1, max(dk, dv), state=True)
                states[s] = got[s]                             # (the next token starts from what is there)
        assert np.array_equal(got[[s for s in range(n + 3) if s not in slots]], pool.numpy()[[s for s in range(n + 3) if s not in slots]])
    assert tcuscan.workspace_fault(ws) == 0


def test_a_prompt_then_single_tokens_is_one_row():
    """40 tokens as a prompt, the rest one by one: the same as all of them as one row."""
    import torch
    c = Case("f32", [75], heads=(2, 2, 2), dk=64, dv=32, seed=12)
    whole, _ = c.forward()
    state = torch.zeros(1, 2, 64, 32, device="cuda")
    out = torch.empty(40, 2, 32, device="cuda")
    ws = tcuscan.new_decay_attention_workspace(1, 40, 2, 64, 32, dt="f32")
    tcuscan.decay_attention(*(x[:40] for x in c.qkv), out, c.log_decay, torch.tensor([0, 40]).cuda(), scale=c.scale, state_in=c.s0.cuda(), state_out=state, ws=ws)
    parts = [out]
    for t in range(40, 75):
        one = torch.empty(1, 2, 32, device="cuda")
        tcuscan.decay_attention_step(*(x[t:t + 1] for x in c.qkv), one, c.log_decay, state, scale=c.scale)
        parts.append(one)
    torch.cuda.synchronize()
    c.check_forward(torch.cat(parts), state)
    assert (whole - torch.cat(parts)).abs().max() <= 1e-4 * whole.abs().max()


def test_workspace_and_streams_and_graphs():
    """One workspace for calls of different sizes, on a stream of its own and in a replayed graph: bit for bit the same as the first time."""
    import torch
    big, small = Case("bf16", [900, 300], heads=(2, 2, 2), dk=64, dv=64, seed=13), Case("bf16", [20, 90], heads=(2, 2, 2), dk=64, dv=64, seed=14)
    ws = tcuscan.new_decay_attention_workspace(2, big.total, 2, 64, 64)
    first = [x.clone() for c in (big, small) for x in c.forward(ws)]
    for c in (big, small):
        c.check_forward(*(first[:2] if c is big else first[2:]))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for _ in range(2):
        again = [x for c in (big, small) for x in c.forward(ws, stream=side)]
        assert all(torch.equal(a, b) for a, b in zip(first, again))
    out, state_out = torch.empty(big.total, 2, 64, dtype=torch.bfloat16, device="cuda"), torch.empty(2, 2, 64, 64, device="cuda")
    s0 = big.s0.cuda()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        tcuscan.decay_attention(*big.qkv, out, big.log_decay, big.offs, scale=big.scale, state_in=s0, state_out=state_out, ws=ws, stream=side)
    for _ in range(3):
        out.fill_(-1.0)
        state_out.fill_(-1.0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, first[0]) and torch.equal(state_out, first[1])
        small.check_forward(*small.forward(ws))


def test_other_rows_do_not_see_what_is_not_finite():
    import torch
    c = Case("bf16", [80, 70, 90], heads=(2, 2, 2), dk=32, dv=32, seed=15)
    want, _ = c.forward()
    for x, bad in zip(c.qkv, (float("nan"), float("inf"), float("-inf"))):
        x[100, 1] = bad
    got, _ = c.forward()
    assert torch.equal(got[:80], want[:80]) and torch.equal(got[150:], want[150:]) and torch.equal(got[80:150, 0], want[80:150, 0])
    assert not torch.isfinite(got[100, 1].float()).all()


def test_offsets_and_slots_out_of_range_are_reported_and_touch_nothing_outside():
    import torch
    c = Case("bf16", [40, 40, 40], heads=(1, 1, 1), dk=32, dv=32, seed=16)
    guard = torch.full((c.total + 64, 1, 32), -77.0, dtype=c.dt, device="cuda")
    out = guard[32:32 + c.total]
    for offsets in ([0, 40, 80, 4000], [-50, 40, 80, 120], [0, 90, 30, 120], [5000, 6000, 7000, 8000]):
        ws = tcuscan.new_decay_attention_workspace(3, c.total, 1, 32, 32)
        tcuscan.decay_attention(*c.qkv, out, c.log_decay, torch.tensor(offsets).cuda(), scale=1.0, ws=ws)
        torch.cuda.synchronize()
        assert tcuscan.workspace_fault(ws) == 2
        assert (guard[:32] == -77.0).all() and (guard[-32:] == -77.0).all()
    ws = torch.zeros(32, dtype=torch.int64, device="cuda")
    state = torch.zeros(5, 1, 32, 32, device="cuda")
    tcuscan.decay_attention_step(*(x[:2] for x in c.qkv), torch.empty(2, 1, 32, dtype=c.dt, device="cuda"), c.log_decay, state[:3], slots=torch.tensor([1, 3]).cuda(), ws=ws)
    torch.cuda.synchronize()
    assert tcuscan.workspace_fault(ws) == 2 and (state[3:] == 0).all() and (state[1] != 0).any()


@pytest.mark.parametrize("kind", KINDS)
def test_long_rows_with_states_in_place(kind):
    """Rows of several segments that start from and end in the same array: no segment may see the states already written."""
    import torch
    c = Case(kind, [900, 0, 1100, 64], heads=(2, 2, 2), dk=64, dv=48, decays=[0.9995, 0.97], seed=17)
    state, out = c.s0.cuda(), torch.empty(c.total, 2, 48, dtype=c.dt, device="cuda")
    ws = tcuscan.new_decay_attention_workspace(c.rows, c.total, 2, 64, 48, dt=kind)
    tcuscan.decay_attention(*c.qkv, out, c.log_decay, c.offs, scale=c.scale, state_in=state, state_out=state, ws=ws)
    torch.cuda.synchronize()
    c.check_forward(out, state)


@pytest.mark.parametrize("stride", [4_000_000, 5_000_000])
def test_tokens_further_apart_than_32_bits_reach(stride):
    """Tokens 4 and 5 million elements apart (within and beyond what offsets of a block take): the last ones lie beyond 2^32 bytes."""
    import torch
    c = Case("bf16", [600], heads=(1, 1, 1), dk=32, dv=32, seed=18)
    far = [torch.empty(stride * 599 + 32, dtype=torch.bfloat16, device="cuda").as_strided((600, 1, 32), (stride, 32, 1)) for _ in range(2)]
    far[0].copy_(c.qkv[1])
    c.qkv[1] = far[0]
    out, state_out = c.forward()
    c.check_forward(out, state_out)
    ws = tcuscan.new_decay_attention_workspace(1, 600, 1, 32, 32)
    tcuscan.decay_attention(*c.qkv, far[1], c.log_decay, c.offs, scale=c.scale, state_in=c.s0.cuda(), state_out=state_out, ws=ws)
    torch.cuda.synchronize()
    c.check_forward(far[1].contiguous(), state_out)


def test_inputs_shared_by_all_tokens_or_heads_without_copies():
    """Strides of 0: one key for all tokens, one query for all heads."""
    import torch
    c = Case("bf16", [200, 30], heads=(3, 3, 3), dk=32, dv=32, seed=19)
    k = c.qkv[1][:1].expand(c.total, 3, 32)
    q = c.qkv[0][:, :1].expand(c.total, 3, 32)
    c.qkv = [q, k, c.qkv[2]]
    c.host = [x.double().cpu().numpy() for x in c.qkv]
    assert k.stride(0) == 0 and q.stride(1) == 0
    c.check_forward(*c.forward())


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("dk,dv", [(96, 192), (192, 90), (70, 96), (130, 160)])
def test_states_between_powers_of_two(kind, dk, dv):
    """In one segment and in several; some wavefronts have no columns."""
    for lengths in ([45, 3], [290, 20]):
        c = Case(kind, lengths, heads=(2, 1, 2), dk=dk, dv=dv, seed=31)
        c.check_forward(*c.forward())
        c.check_backward(*c.backward())


@pytest.mark.parametrize("kind", KINDS)
def test_gradients_of_shared_heads_of_any_size(kind):
    for dk, dv, packed in ((13, 6, False), (12, 20, True), (12, 20, False)):
        c = Case(kind, [90, 0, 7], heads=(2, 1, 2), all_heads=4, dk=dk, dv=dv, packed=packed, seed=32)
        c.check_forward(*c.forward())
        c.check_backward(*c.backward())


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("lengths", [[256], [257], [320], [64, 65, 63, 128], [1023], [2049], [1, 2100]], ids=str)
def test_calls_around_the_choices_of_segments(kind, lengths):
    c = Case(kind, lengths, heads=(8, 8, 8), dk=32, dv=48, seed=33)
    c.check_forward(*c.forward())
    c.check_backward(*c.backward())
