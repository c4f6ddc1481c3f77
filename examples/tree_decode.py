"""Tree-drafted decoding on a small hybrid stack, the five tree calls together.

A toy model with random weights (gated-delta-rule and softmax layers over one paged cache,
projections in PyTorch) decodes greedily.  Each round

  1. drafts a tree: the anchor, its three likeliest followers by a layer-free guess, and
     three followers of each of those (13 nodes),
  2. runs the stack over all nodes at once (flare_tree_linear_attn, flare_tree_softmax_attn),
  3. lets the target choose (flare_tree_verify),
  4. commits the accepted path (flare_tree_commit_state per linear layer, one
     flare_tree_append_kv for the caches of all softmax layers),

with no host synchronisation between rounds.  A prompt enters as a chain whose whole path is
committed, and ordinary decoding is a tree of one node: `--plain` decodes that way, and in
fp32 both give the same tokens.

    python examples/tree_decode.py [--requests 8] [--tokens 64] [--dtype f32] [--plain]
"""
from __future__ import annotations

import argparse
import math
import sys
import time
from pathlib import Path

import torch

sys.path.insert(0, str(Path(__file__).resolve().parents[1]))

from paper_2606_01774_gb300 import flare  # noqa: E402

TYPES = {"f32": (torch.float32, flare.FLARE_DT_F32), "bf16": (torch.bfloat16, flare.FLARE_DT_BF16)}


def _norm(x):
    return x * torch.rsqrt(x.square().mean(-1, keepdim=True) + 1e-6)


class HybridDecoder:
    """A stack of layers ("l" linear, "s" softmax) with the state of `requests` sequences."""

    def __init__(self, requests, max_nodes=16, max_tokens=512, layers="llsl", vocab=512, width=256,
                 dtype="f32", seed=0, device="cuda"):
        self.R, self.N, self.V = requests, max_nodes, vocab
        self.dt, code = TYPES[dtype]
        self.layers, self.device = layers, device
        Hk, Hv, d, Hq, Hkv, D, page = 2, 4, 64, 4, 2, 64, 16
        self.heads = Hk, Hv, d, Hq, Hkv, D
        g = torch.Generator(device=device)
        g.manual_seed(seed)

        def normal(*shape, scale=1.0):
            return torch.randn(shape, generator=g, device=device) * scale

        self.embed, self.head = normal(vocab, width), normal(width, vocab, scale=width ** -0.5)
        cols = {"l": 2 * Hk * d + Hv * d + 2 * Hv, "s": (Hq + 2 * Hkv) * D}
        self.w_in = [normal(width, cols[c], scale=width ** -0.5) for c in layers]
        self.w_out = [normal((Hv * d if c == "l" else Hq * D), width, scale=0.02) for c in layers]

        pages = -(-max_tokens // page)
        i32 = dict(dtype=torch.int32, device=device)
        self.page_table = torch.arange(requests * pages, **i32).reshape(requests, pages)
        self.prefix_len = torch.zeros(requests, **i32)
        self.slot = torch.arange(requests, **i32)
        self.state = [torch.zeros(requests, Hv, d, d, device=device) for c in layers if c == "l"]
        self.cache = [torch.zeros(2, requests * pages, Hkv, page, D, dtype=self.dt, device=device)
                      for c in layers if c == "s"]
        self.status = torch.zeros(1, **i32)
        self.lin = lambda n: flare.linear_desc(requests, n, Hk, Hv, d, d, requests, code,
                                               1 / math.sqrt(d))
        self.soft = lambda n: flare.softmax_desc(requests, n, Hq, Hkv, D, page, requests * pages,
                                                 pages, code, 1 / math.sqrt(D))
        self.verify_desc = lambda n: flare.tree_verify_desc(
            requests, n, vocab, flare.FLARE_DT_F32, flare.FLARE_VERIFY_GREEDY)
        self.work = torch.empty(max(
            max(flare.flare_tree_softmax_workspace_size(self.soft(n)),
                flare.flare_tree_verify_workspace_size(self.verify_desc(n)))
            for n in range(1, max_nodes + 1)), dtype=torch.uint8, device=device)
        self.path = torch.empty(requests, max_nodes, **i32)
        self.path_len, self.next_token = (torch.empty(requests, **i32) for _ in range(2))
        # the drafter: followers by the head on the bare embedding
        self.followers = (_norm(self.embed) @ self.head).topk(3, dim=1).indices.to(torch.int32)

    def forward(self, token, parent, node_len):
        """Logits [R, n, V] of every node; keeps what a commit of the round will need."""
        R, n = token.shape
        Hk, Hv, d, Hq, Hkv, D = self.heads
        x = self.embed[token.long()]
        self.kept, states, caches = [], iter(self.state), iter(self.cache)
        for c, w_in, w_out in zip(self.layers, self.w_in, self.w_out):
            y = _norm(x) @ w_in
            if c == "l":
                q, k, v, g, b = y.split([Hk * d, Hk * d, Hv * d, Hv, Hv], dim=-1)
                q, k = (torch.nn.functional.normalize(t.reshape(R, n, Hk, d), dim=-1)
                        .to(self.dt).contiguous() for t in (q, k))
                v = v.reshape(R, n, Hv, d).to(self.dt).contiguous()
                g = -torch.nn.functional.softplus(g - 2).contiguous()
                b = torch.sigmoid(b).contiguous()
                out = torch.empty_like(v)
                flare.check(flare.flare_tree_linear_attn(
                    self.lin(n), q, k, v, g, b, next(states), self.slot, parent, node_len, out,
                    self.status))
                self.kept.append((k, v, g, b))
            else:
                q, k, v = (t.reshape(R, n, -1, D).to(self.dt).contiguous()
                           for t in y.split([Hq * D, Hkv * D, Hkv * D], dim=-1))
                out, cache = torch.empty_like(q), next(caches)
                flare.check(flare.flare_tree_softmax_attn(
                    self.soft(n), q, k, v, cache[0], cache[1], self.page_table, self.prefix_len,
                    parent, node_len, out, None, self.work, self.work.numel(), self.status))
                self.kept.append((k, v))
            x = x + out.float().reshape(R, n, -1) @ w_out
        return (_norm(x) @ self.head).contiguous()

    def verify(self, logits, token, parent, node_len):
        """Accepted path, its length and the next token (in self.path, path_len, next_token)."""
        n = token.shape[1]
        path = self.path.view(-1)[:self.R * n].view(self.R, n)
        logp = torch.empty(self.R, n, device=self.device)
        flare.check(flare.flare_tree_verify(
            self.verify_desc(n), logits, None, token, parent, node_len, None, None, path,
            self.path_len, self.next_token, logp, self.work, self.work.numel(), self.status))
        return path, self.path_len, self.next_token

    def commit(self, path, path_len):
        """The accepted nodes into every layer's state or cache."""
        n, states = path.shape[1], iter(self.state)
        for c, kept in zip(self.layers, self.kept):
            if c == "l":
                flare.check(flare.flare_tree_commit_state(
                    self.lin(n), *kept, next(states), self.slot, self.slot, path, path_len,
                    self.status))
        soft = [kept for c, kept in zip(self.layers, self.kept) if c == "s"]
        if soft:
            flare.check(flare.flare_tree_append_kv(
                self.soft(n), [k for k, _ in soft], [v for _, v in soft],
                [c[0] for c in self.cache], [c[1] for c in self.cache], self.page_table,
                self.prefix_len, path, path_len, self.status))
        self.prefix_len += path_len

    def prompt(self, tokens):
        """Takes in all prompt tokens but the last, which is the first round's anchor."""
        n = tokens.shape[1] - 1
        for at in range(0, n, self.N):
            part = tokens[:, at:min(at + self.N, n)].contiguous()
            m = part.shape[1]
            line = torch.arange(m, dtype=torch.int32, device=self.device).repeat(self.R, 1)
            full = torch.full((self.R,), m, dtype=torch.int32, device=self.device)
            self.forward(part, line - 1, full)
            self.commit(line, full)
        return tokens[:, -1].contiguous()

    def draft(self, anchor, plain):
        """Tokens [R, n] and parents of a round's tree."""
        if plain:
            return anchor[:, None].contiguous(), [-1]
        one = self.followers[anchor.long()]
        two = self.followers[one.long()].reshape(self.R, 9)
        return (torch.cat([anchor[:, None], one, two], 1).contiguous(),
                [-1, 0, 0, 0, 1, 1, 1, 2, 2, 2, 3, 3, 3])

    def decode(self, tokens, rounds, plain=False):
        """Rounds of decoding; the new tokens of every request, and the mean accepted per round."""
        anchor = self.prompt(tokens)
        said = []
        for _ in range(rounds):
            token, tree = self.draft(anchor, plain)
            n = len(tree)
            parent = torch.tensor(tree, dtype=torch.int32, device=self.device).repeat(self.R, 1)
            node_len = torch.full((self.R,), n, dtype=torch.int32, device=self.device)
            logits = self.forward(token, parent, node_len)
            path, path_len, anchor = self.verify(logits, token, parent, node_len)
            self.commit(path, path_len)
            # the drafted tokens on the path, then the target's own
            drafted = token.gather(1, path.clamp(min=0).long())
            drafted = torch.where(path >= 0, drafted, -1)[:, 1:]
            anchor = anchor.clone()
            said.append(torch.cat([drafted, anchor[:, None]], 1))
        rc, bits = flare.flare_read_status(self.status)
        if rc != flare.FLARE_OK:
            raise RuntimeError(f"device status {bits:#x}")
        said = torch.cat(said, 1).cpu().tolist()
        new = [[t for t in line if t >= 0] for line in said]
        return new, sum(map(len, new)) / (len(new) * rounds)


def main():
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--requests", type=int, default=8)
    ap.add_argument("--tokens", type=int, default=64)
    ap.add_argument("--dtype", choices=sorted(TYPES), default="f32")
    ap.add_argument("--plain", action="store_true", help="one token a round")
    a = ap.parse_args()
    prompt = torch.randint(0, 512, (a.requests, 21), dtype=torch.int32, device="cuda",
                           generator=torch.Generator(device="cuda").manual_seed(1))
    model = HybridDecoder(a.requests, max_tokens=21 + 4 * a.tokens, dtype=a.dtype)
    start = time.perf_counter()
    new, rate = model.decode(prompt, a.tokens if a.plain else -(-a.tokens // 2), a.plain)
    print(f"{rate:.2f} tokens per round and request, {time.perf_counter() - start:.2f} s")
    for line in new[:4]:
        print(*line[:a.tokens])


if __name__ == "__main__":
    main()
