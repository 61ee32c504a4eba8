"""A gated cross-attention layer over a boundary, trained for some steps and then decoded from.

A language model's sequence sees the images that came before each position; the images' states are the rows of the
encoder's buffers, packed in image order.  The layer is the library's operators with plain matrix products between
them: rotary positions in queries (their place in the sequence) and keys (their place in the image's grid), attention
over the ranges that the token map gives, and the norms, the gate and the residual stream in one pass.

    python examples/cross_layer.py
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2605_27678_amd as hp  # noqa: E402


class CrossLayer(torch.nn.Module):
    def __init__(self, hidden, enc_hidden, heads_q, heads_k, dim, positions, device, dtype, seed=0):
        super().__init__()
        g = torch.Generator(device=device).manual_seed(seed)
        new = lambda a, b: torch.nn.Parameter((torch.randn(a, b, generator=g, device=device) / a ** 0.5).to(dtype))  # noqa: E731
        one = lambda n: torch.nn.Parameter(torch.ones(n, device=device, dtype=dtype))                                # noqa: E731
        self.heads_q, self.heads_k, self.dim = heads_q, heads_k, dim
        self.wq, self.wo = new(hidden, heads_q * dim), new(heads_q * dim, hidden)
        self.wk, self.wv = new(enc_hidden, heads_k * dim), new(enc_hidden, heads_k * dim)
        self.w_in, self.w_post, self.w_pre = one(hidden), one(hidden), one(hidden)
        self.gate = torch.nn.Parameter(torch.full((1,), 0.5, device=device, dtype=dtype))
        self.table = torch.empty(positions, dim // 2, 2, device=device)
        hp.hp_rotary_table(self.table, stream=torch.cuda.current_stream())

    def states(self, encoded, grid):
        """Keys, turned by their row and column in the image, and values of encoder states [rows, enc_hidden]."""
        k = (encoded @ self.wk).view(-1, self.heads_k, self.dim)
        v = (encoded @ self.wv).view(-1, self.heads_k, self.dim)
        half = self.dim // 2
        return hp.rotary([k], self.table, grid, sections=(half - half // 2, half // 2))[0], v

    def queries(self, x, positions):
        _, z = hp.gated_norm(x, None, w_pre=self.w_in)
        return hp.rotary([(z @ self.wq).view(-1, self.heads_q, self.dim)], self.table, positions)[0]

    def behind(self, x, attended):
        return hp.gated_norm(x, attended.flatten(1) @ self.wo, self.w_post, self.gate, self.w_pre, gate_tanh=True)

    def forward(self, x, positions, k, v, ranges):
        """(residual stream, the next block's input) of rows x [rows, hidden]."""
        return self.behind(x, hp.cross_attention(self.queries(x, positions), k, v, ranges))

    @torch.no_grad()
    def step(self, x, positions, k, v, ranges):
        """The same for single tokens of many sequences against their cached states."""
        q = self.queries(x, positions)
        out = torch.empty_like(q)
        size = hp.hp_cross_attend_workspace(q, k, "step")
        scratch = torch.empty(max(size, 16), dtype=torch.uint8, device=q.device)
        hp.hp_cross_attend_step(q, k, v, ranges, out, workspace=scratch, stream=torch.cuda.current_stream())
        return self.behind(x, out)


def main(batch=2, seq=512, side=24, hidden=1024, enc_hidden=768, heads_q=16, heads_k=4, dim=64, steps=8,
         dtype=torch.bfloat16, say=print):
    dev = torch.device("cuda", torch.cuda.current_device())
    n = side * side                                          # tokens of an image
    starts = [s for b in range(batch) for s in (10 + b, seq // 2)]
    tm = hp.TokenMap(batch, seq, hidden, [b for b in range(batch) for _ in range(2)], starts, [1] * (2 * batch))
    # a position sees the images whose (one-token) mark is behind it; the states are n rows for each mark
    marks = torch.from_numpy(hp.hp_image_ranges(tm, "previous")).to(dev)
    ranges = (marks * n).contiguous()
    g = torch.Generator(device=dev).manual_seed(1)
    x = torch.randn(batch * seq, hidden, generator=g, device=dev).to(dtype)
    encoded = torch.randn(2 * batch * n, enc_hidden, generator=g, device=dev).to(dtype)
    target = torch.randn(batch * seq, hidden, generator=g, device=dev).to(dtype)
    positions = torch.arange(seq, dtype=torch.int32, device=dev).repeat(batch)
    at = torch.arange(n, dtype=torch.int32, device=dev)
    grid = torch.stack([at // side, at % side]).repeat(1, 2 * batch).contiguous()
    layer = CrossLayer(hidden, enc_hidden, heads_q, heads_k, dim, max(seq, side), dev, dtype)
    optim = torch.optim.SGD(layer.parameters(), lr=2.0)
    losses = []
    for _ in range(steps):
        k, v = layer.states(encoded, grid)
        _, z = layer(x, positions, k, v, ranges)
        loss = (z.float() - target.float()).square().mean()
        optim.zero_grad()
        loss.backward()
        optim.step()
        losses.append(float(loss.detach()))
        say(f"step {len(losses)}: loss {losses[-1]:.4f}")
    # decode: the last token of each sample by itself, against the states that its request keeps
    with torch.no_grad():
        k, v = layer.states(encoded, grid)
        last = torch.arange(batch, device=dev) * seq + seq - 1
        _, whole = layer(x, positions, k, v, ranges)
        _, token = layer.step(x[last], positions[last], k, v, ranges[last].contiguous())
    apart = float((token.float() - whole[last].float()).abs().max())
    say(f"last tokens decoded by themselves: at most {apart:.4f} from the whole pass")
    return losses, apart


if __name__ == "__main__":
    main()
