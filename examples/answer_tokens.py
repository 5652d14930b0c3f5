"""Which prompt tokens carry a language model's answer?

    python examples/answer_tokens.py [--tokens 96] [--samples 2000] [--layers 2]

A small decoder with random weights stands in for a trained one.  The prompt
is run through it once, its keys and values go into a paged cache, and the
token with the highest logit is the answer.  Then every prompt token but the
first four (the instruction, which all coalitions keep) is a player: a
coalition's new token attends over the one cached prompt through the
coalition's mask and over itself, in all layers, and the coalition's value is
the log probability of the answer.  The library's sampler and least squares
give the Shapley values.
"""
import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2401_04829_amd import answers  # noqa: E402


class Decoder:
    """A decoder of `layers` blocks (attention of `heads` heads over `kv_heads`
    with rotary positions, then a gated MLP), weights N(0, 1) / sqrt(width)."""

    def __init__(self, vocab=1000, width=256, heads=8, kv_heads=2, dim=32, layers=2, dtype=torch.bfloat16,
                 device="cuda", seed=0):
        gen = torch.Generator(device).manual_seed(seed)

        def weight(rows, cols):
            return (torch.randn((rows, cols), generator=gen, device=device) / math.sqrt(rows)).to(dtype)
        self.heads, self.kv_heads, self.dim, self.layers, self.dtype, self.device = (heads, kv_heads, dim, layers,
                                                                                    dtype, torch.device(device))
        self.embed = weight(vocab, width) * math.sqrt(vocab)
        self.blocks = [dict(qkv=weight(width, (heads + 2 * kv_heads) * dim), out=weight(heads * dim, width),
                            up=weight(width, 4 * width), down=weight(2 * width, width)) for _ in range(layers)]
        self.head = weight(width, vocab) * 3
        angle = torch.arange(4096, device=device)[:, None] * 10000.0 ** (
            -torch.arange(0, dim, 2, device=device, dtype=torch.float64) / dim)
        self.cos, self.sin = angle.cos().float(), angle.sin().float()

    @staticmethod
    def norm(x):
        y = x.float()
        return (y * torch.rsqrt(y.square().mean(-1, keepdim=True) + 1e-6)).to(x.dtype)

    def split(self, x, block):
        qkv = (self.norm(x) @ block["qkv"]).view(x.shape[0], -1, self.dim)
        return qkv.split([self.heads, self.kv_heads, self.kv_heads], 1)

    def mlp(self, x, attended, block):
        x = x + attended.flatten(1) @ block["out"]
        a, b = (self.norm(x) @ block["up"]).chunk(2, 1)
        return x + (torch.nn.functional.silu(a) * b) @ block["down"]

    def caches(self, pages, page):
        return [answers.PagedCache.empty(pages, page, self.kv_heads, self.dim, self.dtype, self.device)
                for _ in range(self.layers)]

    def prompt(self, tokens, caches, table):
        """Runs all but the last token through the model and caches their keys
        and values: token i attends over tokens 0 .. i, a group of its own."""
        n = tokens.numel() - 1
        index = torch.arange(n, dtype=torch.int32, device=self.device)
        rows = torch.zeros_like(index)
        x = self.embed[tokens[:n]]
        for block, cache in zip(self.blocks, caches):
            q, k, v = self.split(x, block)
            q = answers.append_tokens(cache, k, v, table, index, rows=rows, q=q, cos=self.cos, sin=self.sin)
            attended = answers.attend(cache, q, table.expand(n, -1).contiguous(), index + 1, max_length=n)
            x = self.mlp(x, attended, block)
        return n

    def answer_logits(self, token, position, masks, num_players, first_player, caches, table, own):
        """Logits behind `token`, once per coalition: its queries see the cached
        tokens that the coalition keeps and the token itself, whose keys and
        values (they differ from coalition to coalition) go to pages of its own."""
        k = masks.shape[0]
        zero = torch.zeros(k, dtype=torch.int32, device=self.device)
        one, place = zero + 1, zero + position
        x = self.embed[token].expand(k, -1).contiguous()
        for block, cache in zip(self.blocks, caches):
            q, key, v = self.split(x, block)
            q = answers.append_tokens(cache, key, v, own[:k], zero, positions=place, q=q, cos=self.cos, sin=self.sin)
            attended = answers.attend(cache, q, own[:k], one, max_length=1, shared_table=table,
                                      shared_lengths=torch.full((1,), position, dtype=torch.int32, device=self.device),
                                      max_shared=position, masks=masks, num_players=num_players,
                                      first_player=first_player)
            x = self.mlp(x, attended, block)
        return self.norm(x) @ self.head


def explain(model, tokens, instruction=4, samples=2000, seed=7, page=16, batch=4096):
    """Returns (explanation, answer, TokenLogprobs of the full prompt)."""
    n = tokens.numel() - 1
    pages = -(-n // page)
    table = torch.arange(pages, dtype=torch.int32, device=model.device)[None]
    own = (pages + torch.arange(batch, dtype=torch.int32, device=model.device))[:, None]
    caches = model.caches(pages + batch, page)
    model.prompt(tokens, caches, table)
    players = n - instruction

    def logits(masks):
        return model.answer_logits(tokens[n], n, masks, players, instruction, caches, table, own)
    full = answers.token_logprobs(logits(torch.full((1, -(-players // 64)), -1, dtype=torch.int64,
                                                    device=model.device)), top=5)
    answer = full.top_id[0, 0].long()

    def value(masks, _):
        return answers.token_logprobs(logits(masks), answer.expand(masks.shape[0]).contiguous()).logprob
    return answers.AnswerExplainer(value, model.device, batch).explain(players, samples, seed), answer, full


def main():
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--tokens", type=int, default=96)
    ap.add_argument("--samples", type=int, default=2000)
    ap.add_argument("--layers", type=int, default=2)
    args = ap.parse_args()
    model = Decoder(layers=args.layers)
    tokens = torch.randint(0, 1000, (args.tokens,), generator=torch.Generator("cuda").manual_seed(1), device="cuda")
    e, answer, full = explain(model, tokens, samples=args.samples)
    f0, f1 = e.f_empty_full.tolist()
    print(f"answer: token {int(answer)}, log probability {f1:.4f} ({f0:.4f} from the instruction alone), entropy "
          f"{float(full.entropy[0]):.3f}; alternatives "
          + ", ".join(f"{t} ({p:.2f})" for t, p in zip(full.top_id[0, 1:].tolist(), full.top_logprob[0, 1:].tolist())))
    print(f"sum of the Shapley values {float(e.phi.sum()):.4f}, f(all) - f(none) {f1 - f0:.4f}")
    for i in e.phi.abs().argsort(descending=True)[:8].tolist():
        print(f"  position {i + 4:4d}: token {int(tokens[i + 4]):4d}  phi {float(e.phi[i]):+.4f}")


if __name__ == "__main__":
    main()
