"""A small decoder language model of the framework's parts: token embedding, attention with normed and rotated heads
between sketched projections, a sketched feed-forward layer, dropout with the residual added; training, and generation
from a cache of keys and values.  The same with dense layers and layer norms, as a sketched model's teacher.

    python -m paper_2601_15473_amd.decoder [--steps 200] [--distill]

trains one on sequences that repeat themselves after a random first half, and lets it continue some; with --distill it is first a dense one, and then a
sketched one that learns from the dense one's likeliest tokens.
"""
from __future__ import annotations

import argparse

import torch
import torch.nn.functional as F

from .block import attention, distillation_loss, dropout, embedding, head_norm_rope, layer_norm, linear
from .nn import SKLinear


def rotation_tables(positions: int, rotated: int, base: float = 10000.0, device="cuda"):
    """cos and sin [positions, rotated / 2] of position / base^(2 i / rotated), as head_norm_rope takes them."""
    angle = torch.arange(positions, device=device, dtype=torch.float64)[:, None] * \
        base ** (-torch.arange(0, rotated, 2, device=device, dtype=torch.float64) / rotated)
    return angle.cos().float(), angle.sin().float()


class DecoderLayer(torch.nn.Module):
    """x + attention(norm(x)), then x + feed_forward(norm(x)); the additions are the dropouts' residuals."""

    def __init__(self, width, heads, kv_heads, head_dim, hidden, terms, rank, dtype, seed):
        super().__init__()
        self.heads, self.kv_heads, self.head_dim = heads, kv_heads, head_dim
        make = lambda i, o, s: SKLinear(i, o, terms, rank, bias=False, dtype=dtype, seed=seed * 4 + s)  # noqa: E731
        self.qkv, self.out = make(width, (heads + 2 * kv_heads) * head_dim, 0), make(heads * head_dim, width, 1)
        self.up, self.down = make(width, hidden, 2), make(hidden, width, 3)
        ones = lambda n: torch.nn.Parameter(torch.ones(n, dtype=dtype, device="cuda"))  # noqa: E731
        self.norm_attention, self.norm_hidden, self.q_weight, self.k_weight = ones(width), ones(width), ones(head_dim), ones(head_dim)

    def heads_of(self, x, tables, positions):
        """Queries, keys and values [batch, tokens, heads, head_dim] of x [batch, tokens, width]."""
        qkv = self.qkv(F.rms_norm(x, x.shape[-1:], self.norm_attention, 1e-6)).unflatten(-1, (-1, self.head_dim))
        q, k, v = qkv.split((self.heads, self.kv_heads, self.kv_heads), 2)
        q, k = head_norm_rope(q, k, self.q_weight, self.k_weight, *tables, positions)
        return q, k, v

    def finish(self, x, o, p, seed, offset):
        x = dropout(self.out(o.flatten(2)), p, seed, offset, residual=x)
        h = self.down(F.gelu(self.up(F.rms_norm(x, x.shape[-1:], self.norm_hidden, 1e-6))))
        return dropout(h, p, seed, offset + 1, residual=x)


class DenseDecoderLayer(torch.nn.Module):
    """``DecoderLayer`` with dense projections and layer norms: each norm takes the addition before it along, the activation and (without a dropout between)
    the last addition are the dense layers' own."""

    def __init__(self, width, heads, kv_heads, head_dim, hidden, dtype, seed):
        super().__init__()
        self.heads, self.kv_heads, self.head_dim = heads, kv_heads, head_dim
        g = torch.Generator().manual_seed(seed)
        weight = lambda o, i: torch.nn.Parameter((torch.randn(o, i, generator=g) * i ** -0.5).to(dtype).cuda())  # noqa: E731
        full = lambda n, v: torch.nn.Parameter(torch.full((n,), v, dtype=dtype, device="cuda"))  # noqa: E731
        fused = (heads + 2 * kv_heads) * head_dim
        self.qkv, self.out, self.up, self.down = weight(fused, width), weight(width, heads * head_dim), weight(hidden, width), weight(width, hidden)
        self.qkv_bias, self.out_bias, self.up_bias, self.down_bias = (full(n, 0.0) for n in (fused, width, hidden, width))
        self.norm_attention, self.norm_hidden, self.q_weight, self.k_weight = (full(n, 1.0) for n in (width, width, head_dim, head_dim))
        self.norm_attention_bias, self.norm_hidden_bias = full(width, 0.0), full(width, 0.0)

    def heads_of(self, x, tables, positions):
        """As DecoderLayer.heads_of."""
        qkv = linear(layer_norm(x, self.norm_attention, self.norm_attention_bias), self.qkv, self.qkv_bias).unflatten(-1, (-1, self.head_dim))
        q, k, v = qkv.split((self.heads, self.kv_heads, self.kv_heads), 2)
        q, k = head_norm_rope(q, k, self.q_weight, self.k_weight, *tables, positions)
        return q, k, v

    def finish(self, x, o, p, seed, offset):
        h = linear(o.flatten(2), self.out, self.out_bias)
        if p > 0:
            x = dropout(h, p, seed, offset, residual=x)
            y = layer_norm(x, self.norm_hidden, self.norm_hidden_bias)
        else:
            y, x = layer_norm(h, self.norm_hidden, self.norm_hidden_bias, residual=x)
        h = linear(y, self.up, self.up_bias, activation="gelu")
        if p > 0:
            return dropout(linear(h, self.down, self.down_bias), p, seed, offset + 1, residual=x)
        return linear(h, self.down, self.down_bias, residual=x)


class Cache(tuple):
    """(keys and values [layers, batch, tokens, 2, kv_heads, head_dim], how many there are of each sequence: int32 [batch]), both on the GPU."""

    most = 0     # as many as any sequence can have by what was appended: known here, where the numbers themselves are a copy away


class Decoder(torch.nn.Module):
    def __init__(self, rows: int, width: int = 256, layers: int = 2, heads: int = 4, kv_heads: int = 2, head_dim: int = 64, hidden: int = 512,
                 terms: int = 1, rank: int = 128, context: int = 512, p: float = 0.1, dtype: torch.dtype = torch.bfloat16, seed: int = 0, dense: bool = False):
        """``dense``: dense layers and layer norms in place of sketched ones (terms and rank are not looked at)."""
        super().__init__()
        g = torch.Generator().manual_seed(seed)
        self.table = torch.nn.Parameter((torch.randn(rows, width, generator=g) * width ** -0.5).to(dtype).cuda())
        make = (lambda s: DenseDecoderLayer(width, heads, kv_heads, head_dim, hidden, dtype, s)) if dense else \
            (lambda s: DecoderLayer(width, heads, kv_heads, head_dim, hidden, terms, rank, dtype, s))
        self.layers = torch.nn.ModuleList(make(seed + 1 + i) for i in range(layers))
        self.norm = torch.nn.Parameter(torch.ones(width, dtype=dtype, device="cuda"))
        self.tables, self.p, self.seed, self.scale = rotation_tables(context, head_dim), p, seed, width ** 0.5

    def logits(self, x):
        return F.rms_norm(x, x.shape[-1:], self.norm, 1e-6) @ self.table.t()

    def forward(self, ids, lengths=None, step: int = 0):
        """Logits [batch, tokens, rows]; ``lengths`` (int32 [batch]) of padded sequences, whose padding is an id outside the
        table.  ``step``: the training step, whose dropouts are its own."""
        if ids.shape[1] > len(self.tables[0]):
            raise ValueError(f"decoder: {ids.shape[1]} tokens, but positions for {len(self.tables[0])}")
        positions = torch.arange(ids.shape[1], device=ids.device).expand(ids.shape)
        p = self.p if self.training else 0.0
        x = embedding(ids, self.table, self.scale)
        for i, layer in enumerate(self.layers):
            o = attention(*layer.heads_of(x, self.tables, positions), lengths, lengths, causal=True)
            x = layer.finish(x, o, p, self.seed, 2 * (step * len(self.layers) + i))
        return self.logits(x)

    def cache(self, batch: int, tokens: int):
        """Empty room for ``tokens`` keys and values of each sequence, and how many there are of each."""
        layer = self.layers[0]
        kv = torch.zeros((len(self.layers), batch, tokens, 2, layer.kv_heads, layer.head_dim), dtype=self.table.dtype, device="cuda")
        return Cache((kv, torch.zeros(batch, dtype=torch.int32, device="cuda")))

    @torch.no_grad()
    def append(self, ids, cache):
        """Logits of ids [batch, n] behind what the cache holds of each sequence; their keys and values join it."""
        kv, lengths = cache
        n, room = ids.shape[1], min(kv.shape[2], len(self.tables[0]))
        most = cache.most if isinstance(cache, Cache) else room
        if most + n > room:
            most = int(lengths.max())           # (not known, or the program may have emptied sequences since)
        if most + n > room:
            raise ValueError(f"decoder: {n} tokens behind {most}, but room for {kv.shape[2]} and positions for {len(self.tables[0])}")
        if isinstance(cache, Cache):
            cache.most = most + n
        positions = lengths[:, None] + torch.arange(n, dtype=torch.int32, device=ids.device)
        # (inside the cache whatever the lengths are: a program that sets them itself must not write elsewhere)
        sequence, slots = torch.arange(len(ids), device=ids.device)[:, None], positions.clamp(0, kv.shape[2] - 1)
        lengths += n
        x = embedding(ids, self.table, self.scale)
        for i, layer in enumerate(self.layers):
            q, k, v = layer.heads_of(x, self.tables, positions)
            kv[i, sequence, slots, 0], kv[i, sequence, slots, 1] = k, v
            x = layer.finish(x, attention(q, kv[i, :, :, 0], kv[i, :, :, 1], k_lengths=lengths, causal=True), 0.0, 0, 0)
        return self.logits(x)


def repeating(batch: int, half: int, rows: int, generator):
    """Sequences whose second half is their first."""
    first = torch.randint(1, rows, (batch, half), generator=generator, device="cuda")
    return torch.cat((first, first), 1)


def train(model: Decoder, steps: int, batch: int = 32, half: int = 16, rate: float = 2e-3, report=lambda step, loss: None):
    """On what stands in the second half of each sequence (the first is anyone's guess)."""
    def loss_of(logits, ids):
        return F.cross_entropy(logits.float()[:, half - 1:].flatten(0, 1), ids[:, half:].flatten())

    _train(model, loss_of, steps, batch, half, rate, report)


def distill(model: Decoder, teacher: Decoder, steps: int, batch: int = 32, half: int = 16, rate: float = 2e-3, top: int = 8, temperature: float = 2.0,
            label_weight: float = 0.3, report=lambda step, loss: None):
    """As ``train``, against the ``top`` likeliest tokens of ``teacher`` beside the next ones."""
    teacher.eval()

    def loss_of(logits, ids):
        with torch.no_grad():
            values, places = teacher(ids[:, :-1])[:, half - 1:].topk(top, -1)
        return distillation_loss(logits[:, half - 1:], values.to(logits.dtype), places, ids[:, half:], temperature=temperature, label_weight=label_weight).mean()

    _train(model, loss_of, steps, batch, half, rate, report)


def _train(model, loss_of, steps, batch, half, rate, report):
    g = torch.Generator(device="cuda").manual_seed(1)
    weights = {p: p.detach().float() for p in model.parameters()}          # masters in fp32: bf16 ones would not see small steps
    optimizer = torch.optim.Adam(weights.values(), lr=rate)
    model.train()
    for step in range(steps):
        ids = repeating(batch, half, model.table.shape[0], g)
        loss = loss_of(model(ids[:, :-1], step=step), ids)
        model.zero_grad(set_to_none=True)
        loss.backward()
        for p, w in weights.items():
            w.grad = p.grad.float()
        optimizer.step()
        with torch.no_grad():
            for p, w in weights.items():
                p.copy_(w)
        report(step, loss)


@torch.no_grad()
def generate(model: Decoder, ids, n: int):
    """ids [batch, tokens] and the n likeliest tokens behind them, one at a time."""
    model.eval()
    cache = model.cache(len(ids), ids.shape[1] + n)
    logits = model.append(ids, cache)
    for _ in range(n):
        token = logits[:, -1:].argmax(-1)
        ids = torch.cat((ids, token), 1)
        logits = model.append(token, cache)
    return ids


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=200)
    ap.add_argument("--distill", action="store_true", help="train a dense model first, and a sketched one from it")
    args = ap.parse_args()
    steps = args.steps
    report = lambda step, loss: print(f"step {step}: loss {loss.item():.3f}", flush=True) if step % 20 == 0 or step == steps - 1 else None  # noqa: E731
    model = Decoder(rows=64, dense=args.distill)
    train(model, steps, report=report)
    if args.distill:
        teacher, model = model, Decoder(rows=64)
        distill(model, teacher, steps, report=report)
    ids = repeating(4, 16, 64, torch.Generator(device="cuda").manual_seed(2))
    right = (generate(model, ids[:, :17], 15)[:, 17:] == ids[:, 17:]).float().mean().item()
    print(f"continued as they began: {100 * right:.0f} % of the tokens")


if __name__ == "__main__":
    main()
