"""A small language model on the library's operators: an embedding, layers of linear attention with decays, a classifier.

Trains on texts of period `PERIOD` (each token is the one `PERIOD` places before), packed ragged into one batch, then continues a prompt token by token
from the state that the prompt leaves.

    python examples/decay_lm.py [--steps 300]
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2411_17887_amd import tcuscan  # noqa: E402

VOCAB, DIM, HEADS, HEAD, LAYERS, PERIOD = 64, 256, 4, 64, 2, 7


class Embedding(torch.autograd.Function):
    """Rows of the table, scaled; the table's gradient by sorted tokens."""

    @staticmethod
    def forward(ctx, ids, weight, scale):
        out = torch.empty(ids.numel(), weight.shape[1], dtype=torch.bfloat16, device=ids.device)
        tcuscan.embedding(ids, weight.detach(), out, scale=scale)
        ctx.save_for_backward(ids)
        ctx.shape, ctx.scale = weight.shape, scale
        return out

    @staticmethod
    def backward(ctx, d_out):
        ids, = ctx.saved_tensors
        d_weight = torch.empty(ctx.shape, device=ids.device)
        ws = tcuscan.new_embedding_backward_workspace(ids.numel(), *ctx.shape)
        tcuscan.embedding_backward(ids, d_out.contiguous(), d_weight, scale=ctx.scale, ws=ws)
        return None, d_weight, None


class DecayAttention(torch.autograd.Function):
    """Linear attention over ragged rows, from states of zeros."""

    @staticmethod
    def forward(ctx, qkv, log_decay, offsets, scale):
        q, k, v = split(qkv)
        out = torch.empty(q.shape[0], HEADS, HEAD, dtype=qkv.dtype, device=qkv.device)
        rows = offsets.numel() - 1
        ws = tcuscan.new_decay_attention_workspace(rows, q.shape[0], HEADS, HEAD, HEAD)
        tcuscan.decay_attention(q, k, v, out, log_decay, offsets, scale=scale, ws=ws)
        ctx.save_for_backward(qkv, log_decay, offsets)
        ctx.scale = scale
        return out

    @staticmethod
    def backward(ctx, d_out):
        qkv, log_decay, offsets = ctx.saved_tensors
        d_qkv = torch.empty_like(qkv)                      # the gradients land where the projection wants them
        ws = tcuscan.new_decay_attention_backward_workspace(offsets.numel() - 1, qkv.shape[0], HEADS, HEAD, HEAD)
        tcuscan.decay_attention_backward(*split(qkv), d_out.contiguous(), *split(d_qkv), log_decay, offsets, scale=ctx.scale, ws=ws)
        return d_qkv, None, None, None


def split(qkv):
    return [x.view(-1, HEADS, HEAD) for x in qkv.split(HEADS * HEAD, dim=1)]


class Model(torch.nn.Module):
    def __init__(self):
        super().__init__()
        self.table = torch.nn.Parameter(torch.randn(VOCAB, DIM) * DIM ** -0.5)
        self.norms = torch.nn.ModuleList(torch.nn.LayerNorm(DIM) for _ in range(LAYERS + 1))
        self.qkv = torch.nn.ModuleList(torch.nn.Linear(DIM, 3 * HEADS * HEAD) for _ in range(LAYERS))
        self.mix = torch.nn.ModuleList(torch.nn.Linear(HEADS * HEAD, DIM) for _ in range(LAYERS))
        self.up = torch.nn.ModuleList(torch.nn.Linear(DIM, 2 * DIM) for _ in range(LAYERS))
        self.down = torch.nn.ModuleList(torch.nn.Linear(2 * DIM, DIM) for _ in range(LAYERS))
        self.head = torch.nn.Linear(DIM, VOCAB)
        self.places = torch.nn.Parameter(torch.randn(PERIOD, DIM) * DIM ** -0.5)
        self.register_buffer("log_decay", torch.log1p(-torch.pow(2.0, -3.0 - torch.arange(HEADS, dtype=torch.float32))))
        self.scale = HEAD ** -0.5

    def layers(self, x, attend):
        """x [tokens, DIM] through all layers; attend(layer, qkv) -> [tokens, HEADS, HEAD]."""
        for i in range(LAYERS):
            qkv = self.qkv[i](self.norms[i](x)).to(torch.bfloat16)
            x = x + self.mix[i](attend(i, qkv).float().view(-1, HEADS * HEAD))
            x = x + self.down[i](torch.nn.functional.gelu(self.up[i](x)))
        return self.head(self.norms[-1](x))

    def embed(self, ids, places):
        return Embedding.apply(ids, self.table, DIM ** 0.5).float() + Embedding.apply(places % PERIOD, self.places, DIM ** 0.5).float()

    def forward(self, ids, places, offsets):
        return self.layers(self.embed(ids, places), lambda i, qkv: DecayAttention.apply(qkv, self.log_decay, offsets, self.scale))

    @torch.no_grad()
    def generate(self, prompt, count):
        """The prompt's states, then `count` tokens one by one from them."""
        n = prompt.numel()
        states = torch.zeros(LAYERS, 1, HEADS, HEAD, HEAD, device=prompt.device)
        offsets = torch.tensor([0, n], device=prompt.device)
        ws = tcuscan.new_decay_attention_workspace(1, n, HEADS, HEAD, HEAD)

        def attend(i, qkv):
            q, k, v = split(qkv)
            out = torch.empty_like(q, memory_format=torch.contiguous_format)
            if q.shape[0] > 1:
                tcuscan.decay_attention(q, k, v, out, self.log_decay, offsets, scale=self.scale, state_in=states[i], state_out=states[i], ws=ws)
            else:
                tcuscan.decay_attention_step(q, k, v, out, self.log_decay, states[i], scale=self.scale)
            return out

        tokens = [self.layers(self.embed(prompt, torch.arange(n, device=prompt.device)), attend)[-1:].argmax(-1)]
        for place in range(n, n + count - 1):
            tokens.append(self.layers(self.embed(tokens[-1], torch.tensor([place], device=prompt.device)), attend).argmax(-1))
        return torch.cat(tokens)


def texts(rows, generator):
    """Periodic texts of different lengths: token numbers, places within a text, offsets."""
    lengths = torch.randint(3 * PERIOD, 8 * PERIOD, (rows,), generator=generator)
    ids = [torch.randint(VOCAB, (PERIOD,), generator=generator).repeat(8)[:n] for n in lengths.tolist()]
    places = [torch.arange(n) for n in lengths.tolist()]
    return torch.cat(ids).cuda(), torch.cat(places).cuda(), torch.cat([torch.zeros(1, dtype=torch.long), lengths.cumsum(0)]).cuda()


def train(steps, rows=48, seed=0, say=print):
    torch.manual_seed(seed)
    generator = torch.Generator().manual_seed(seed)
    model = Model().cuda()
    optimizer = torch.optim.Adam(model.parameters(), lr=2e-3)
    losses = []
    for step in range(steps):
        ids, places, offsets = texts(rows, generator)
        logits = model(ids, places, offsets)
        known = (places >= PERIOD - 1) & (torch.arange(len(ids), device="cuda") + 1 < len(ids))
        known[offsets[1:] - 1] = False                    # what follows a text's last token is another text
        known = known.nonzero().squeeze(1)
        loss = torch.nn.functional.cross_entropy(logits[known], ids[known + 1])
        optimizer.zero_grad()
        loss.backward()
        optimizer.step()
        losses.append(loss.item())
        if step % 50 == 0 or step == steps - 1:
            say(f"step {step}: loss {losses[-1]:.3f}")
    return model, losses


def main():
    parser = argparse.ArgumentParser(description=__doc__)
    parser.add_argument("--steps", type=int, default=300)
    steps = parser.parse_args().steps
    model, _ = train(steps)
    period = torch.randint(VOCAB, (PERIOD,), generator=torch.Generator().manual_seed(1))
    prompt = period.repeat(4).cuda()
    print("prompt   ", prompt.tolist())
    print("continued", model.generate(prompt, 2 * PERIOD).tolist())
    print("expected ", period.repeat(2).tolist())


if __name__ == "__main__":
    main()
