"""A small language model of gated linear attention layers, trained and then run token by token with the library's operators.

    python examples/gated_linear_attention.py [--steps 60]

A layer is  y -> q, k, v, gate, decays;  linear attention;  norm and gate of each head;  projection;  residual and the norm
before the next layer.  heinsen_linear_attention and heinsen_block_norm do all of it but the projections, forward and backward,
in bfloat16 over packed sequences of different lengths.  The text is synthetic: each sequence counts in steps of its own, so that
what comes next follows from a token and from what the states remember of those before it.  Afterwards a sequence is generated one token at a time, with a
state of H x K x V for each layer in place of a cache of all tokens, and compared with the pass over the whole sequence."""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2311_06281_amd import binding as hs

VOCABULARY, WIDTH, LAYERS, HEADS, K, V, EPS = 64, 256, 2, 4, 32, 64, 1e-6
BF16 = torch.bfloat16


class LinearAttention(torch.autograd.Function):
    """q, k: [tokens, HEADS, K], v: [tokens, HEADS, V], which may be slices of one projection; log_a: [tokens, HEADS];
    starts: where the sequences start, or None for sequences of one length; s0: [B, HEADS, K, V] -> out, states at the ends."""

    @staticmethod
    def forward(ctx, q, k, v, log_a, s0, starts, B, n):
        out, sn = torch.empty(v.shape, dtype=v.dtype, device=v.device), torch.empty_like(s0)
        ctx.sizes = (B, n, HEADS, K, V, K**-0.5, hs.HEINSEN_IN_BF16)
        ctx.strides = dict(q_stride=q.stride(0), k_stride=k.stride(0), v_stride=v.stride(0))
        hs.heinsen_linear_attention(q, k, v, log_a, s0, out, sn, *ctx.sizes, torch.cuda.current_stream(), starts=starts, **ctx.strides)
        ctx.save_for_backward(q, k, v, log_a, s0, starts)
        return out, sn

    @staticmethod
    def backward(ctx, grad_out, grad_sn):
        q, k, v, log_a, s0, starts = ctx.saved_tensors
        grads = [torch.empty(t.shape, dtype=t.dtype, device=t.device) for t in (q, k, v, log_a, s0)]
        hs.heinsen_linear_attention_backward(q, k, v, log_a, s0, grad_out.contiguous(), grad_sn.contiguous(), *grads, *ctx.sizes,
                                             torch.cuda.current_stream(), starts=starts, **ctx.strides)
        return *grads, None, None, None


class BlockNorm(torch.autograd.Function):
    """h = residual + scale * silu(gate) * norm(u) w_post and, with w_pre, y = norm(h) w_pre; what is None is left out."""

    @staticmethod
    def forward(ctx, u, gate, residual, scale, w_post, w_pre):
        ctx.given = (u, gate, residual, scale, w_post, w_pre)
        h = torch.empty_like(u)
        y = torch.empty_like(u) if w_pre is not None else None
        hs.heinsen_block_norm(*ctx.given, h, y, u.shape[0], u.shape[1], EPS, hs.HEINSEN_IN_BF16, torch.cuda.current_stream())
        return h, y

    @staticmethod
    def backward(ctx, grad_h, grad_y):
        grads = [None if t is None else torch.empty_like(t) for t in ctx.given]
        u = ctx.given[0]
        hs.heinsen_block_norm_backward(*ctx.given, None if grad_h is None else grad_h.contiguous(),
                                       None if grad_y is None or ctx.given[5] is None else grad_y.contiguous(), *grads, u.shape[0], u.shape[1],
                                       EPS, hs.HEINSEN_IN_BF16, torch.cuda.current_stream())
        return tuple(grads)


class Model(torch.nn.Module):
    def __init__(self):
        super().__init__()
        matrix = lambda rows, cols: torch.nn.Parameter((torch.randn(rows, cols) * rows**-0.5).cuda())
        vector = lambda size, value: torch.nn.Parameter(torch.full((size,), value, device="cuda"))
        self.embedding = torch.nn.Parameter(torch.randn(VOCABULARY, WIDTH).cuda())
        self.first_norm = vector(WIDTH, 1.0)
        joint = HEADS * (2 * K + V)
        self.layers = torch.nn.ModuleList(
            torch.nn.ParameterDict(dict(joint=matrix(WIDTH, joint), gate=matrix(WIDTH, HEADS * V), decay=matrix(WIDTH, HEADS), head_norm=vector(V, 1.0),
                                        out=matrix(HEADS * V, WIDTH), scale=vector(WIDTH, 0.5), norm=vector(WIDTH, 1.0)))
            for _ in range(LAYERS))
        self.head = matrix(WIDTH, VOCABULARY)

    def forward(self, tokens, states, starts, B, n):
        """tokens: [total]; states: one of [B, HEADS, K, V] for each layer -> logits, the layers' new states."""
        h = self.embedding[tokens].to(BF16)
        h, y = BlockNorm.apply(h, None, None, None, None, self.first_norm)
        new_states = []
        for layer, s0 in zip(self.layers, states):
            joint = y @ layer["joint"].to(BF16)  # q, k and v of a token side by side: read where they are
            q, k, v = (t.unflatten(1, (HEADS, -1)) for t in joint.split((HEADS * K, HEADS * K, HEADS * V), 1))
            log_a = torch.nn.functional.logsigmoid((y @ layer["decay"].to(BF16)).float() + 4.0).to(BF16)
            out, sn = LinearAttention.apply(q, k, v, log_a, s0, starts, B, n)
            new_states.append(sn)
            gate = y @ layer["gate"].to(BF16)
            rows = (len(tokens) * HEADS, V)
            out, _ = BlockNorm.apply(out.view(rows), gate.view(rows), None, None, layer["head_norm"], None)
            block = out.view(len(tokens), HEADS * V) @ layer["out"].to(BF16)
            h, y = BlockNorm.apply(block, None, h, layer["scale"], None, layer["norm"])
        return (y @ self.head.to(BF16)).float(), new_states


def no_memory(B):
    return [torch.zeros(B, HEADS, K, V, device="cuda") for _ in range(LAYERS)]


def text(lengths, generator):
    """Sequences that count, from anywhere in steps of 1, 3, 5 or 7, one after the other, and where each starts."""
    draw = lambda most: int(torch.randint(most, (1,), generator=generator))
    parts = [(draw(VOCABULARY) + (2 * draw(4) + 1) * torch.arange(m)) % VOCABULARY for m in lengths]
    return torch.cat(parts).cuda(), torch.tensor([0, *torch.tensor(lengths).cumsum(0)], device="cuda")


def main(steps=60, say=print):
    torch.manual_seed(0)
    generator = torch.Generator().manual_seed(1)
    model = Model()
    optimizer = torch.optim.Adam(model.parameters(), lr=3e-3)
    lengths = [200, 33, 128, 1, 150, 96, 200, 64]
    losses = []
    for step in range(steps):
        tokens, starts = text(lengths, generator)
        logits, _ = model(tokens, no_memory(len(lengths)), starts, len(lengths), max(lengths))
        follows = torch.ones(len(tokens), dtype=torch.bool, device="cuda")
        follows[starts[1:] - 1] = False  # a sequence's last token is followed by none
        losses.append(torch.nn.functional.cross_entropy(logits[follows], tokens[1:][follows[:-1]]))
        optimizer.zero_grad()
        losses[-1].backward()
        optimizer.step()
        if step % 20 == 0 or step == steps - 1:
            say(f"step {step}: loss {float(losses[-1].detach()):.3f}")

    with torch.no_grad():
        tokens, _ = text([48], generator)
        whole, ends = model(tokens, no_memory(1), None, 1, len(tokens))
        states, rows = no_memory(1), []
        for t in range(len(tokens)):
            logits, states = model(tokens[t : t + 1], states, None, 1, 1)
            rows.append(logits)
        apart = float((torch.cat(rows) - whole).norm() / whole.norm())
        states_apart = max(float((a - b).norm() / b.norm()) for a, b in zip(states, ends))
        right = float((whole[16:-1].argmax(1) == tokens[17:]).float().mean())
    say(f"token by token: logits {apart:.2g} and states {states_apart:.2g} from those of the whole sequence; {100 * right:.0f} % of the tokens foretold")
    return [float(x.detach()) for x in losses], apart, states_apart


if __name__ == "__main__":
    parser = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    parser.add_argument("--steps", type=int, default=60)
    main(parser.parse_args().steps)
