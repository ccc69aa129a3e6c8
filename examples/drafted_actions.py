"""Answers from the encoder's tokens: a small language backbone that takes a camera frame's tokens as its prompt and
decodes action tokens, one at a time or as trees of drafts that are verified in one pass.

    python examples/drafted_actions.py

Weights and frames are random, the drafter is a stand-in that guesses the next tokens right some of the time; what the
example shows is how the operators work together:

    ivit_step_plan       pages, slots, positions and tree masks of a step
    ivit_qk_norm_rope    queries and keys of a layer: view tokens with (time, height, width) positions go straight into
                         the cache, drafts' keys stay beside it
    ivit_tree_attention  the new rows over the cached tokens and over each other
    ivit_kv_write        keys and values of the accepted drafts of all layers into their slots

With greedy verification the trees give the same tokens as decoding one at a time, in fewer passes.

``sample`` does the same over a cache of 8 bits, with drafts that are drawn from a drafter's probabilities:

    ivit_tree_attention_quantised  the new rows over the cached tokens' codes and over each other
    ivit_tree_verify               which drafts are right, and the next token, from given random numbers
    ivit_kv_quantise               the accepted rows of all layers into their slots, in 8 bits
"""
from __future__ import annotations

import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.abspath(__file__)), ".."))

import paper_2607_12287_gb300 as ivit  # noqa: E402
from paper_2607_12287_gb300 import synth  # noqa: E402

PAGE, PAGES, TABLE = 16, 64, 32


def _i32(*values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


class Backbone:
    """A stack of attention layers over a paged cache, for one request."""

    def __init__(self, token_dim, seed=0, layers=2, dim=256, heads=8, kv_heads=2, head_dim=64, vocab=128):
        g = torch.Generator(device="cuda").manual_seed(seed)
        normal = lambda *shape: (torch.randn(shape, generator=g, device="cuda") * shape[-1] ** -0.5).bfloat16()
        self.layers, self.heads, self.kv, self.hd = layers, heads, kv_heads, head_dim
        self.project = normal(dim, token_dim)
        self.embed = torch.randn((vocab, dim), generator=g, device="cuda").bfloat16()
        self.w_out = torch.randn((vocab, dim), generator=g, device="cuda")
        self.w_qkv = [normal((heads + 2 * kv_heads) * head_dim, dim) for _ in range(layers)]
        self.w_o = [2 * normal(dim, heads * head_dim) for _ in range(layers)]
        self.norm = torch.ones(head_dim, dtype=torch.bfloat16, device="cuda")
        # pairs of a head: a fourth turns with time, the rest with height and width; text has one position for all
        half = head_dim // 2
        self.axis = _i32(*([0] * (half // 4) + [1] * (3 * half // 8) + [2] * (half - half // 4 - 3 * half // 8)))
        self.freq = (1000.0 ** (-torch.arange(half, device="cuda") / half)).float()
        self.rope = ivit.make_rope_config(heads, kv_heads, head_dim, n_axes=3)
        cache = lambda: torch.zeros((layers, PAGES, PAGE, kv_heads, head_dim), dtype=torch.bfloat16, device="cuda")
        self.k_cache, self.v_cache = cache(), cache()
        self.layout = ivit.make_cache_layout(self.k_cache[0])
        self.table = torch.full((1, TABLE), -1, dtype=torch.int32, device="cuda")
        self.ring, self.ring_at = torch.arange(PAGES, dtype=torch.int32, device="cuda"), _i32(0, PAGES)
        self.held, self.length, self.passes = 0, 0, 0

    def plan(self, new, parents=None):
        """Slots, positions and mask of ``new`` rows behind the cached tokens."""
        words = (new + 31) // 32 if parents is not None else 0
        cfg = ivit.make_plan_config(1, new, TABLE, PAGE, PAGES, words)
        rows = lambda *shape: torch.empty(shape, dtype=torch.int32, device="cuda")
        cu, slots, pos, mask, ring_at, status = rows(2), rows(new), rows(new), rows(new, max(words, 1)), rows(2), rows(1)
        ivit.ivit_step_plan(cfg, _i32(self.held), _i32(self.length), _i32(new), parents, self.ring, self.ring_at, self.table,
                            cu, None, slots, pos, mask if words else None, ring_at, status)
        if int(status):
            raise RuntimeError(f"the step was refused: {int(status)}")
        self.held, self.ring_at = self.length + new, ring_at
        return cu, slots, pos, mask if words else None

    def workspace(self, cfg):
        return ivit.ivit_tree_attention_workspace(cfg, self.layout)

    def attend(self, layer, cfg, q, k, v, cu, mask, out, ws):
        ivit.ivit_tree_attention(cfg, self.layout, q, k, v, self.k_cache[layer], self.v_cache[layer], self.table,
                                 _i32(self.length), cu, mask, out, None, ws)

    def forward(self, x, cu, positions, mask_mode, mask, slots=None):
        """Logits of new rows x, and their keys and values per layer; into the cache at once if they have ``slots``."""
        self.passes += 1
        n = x.shape[0]
        cfg = ivit.make_attention_config(1, self.heads, TABLE, n, mask_mode, 0 if mask is None else mask.shape[1], self.hd ** -0.5)
        ws = torch.empty(self.workspace(cfg), dtype=torch.uint8, device="cuda")
        keys, values = [], []
        for layer in range(self.layers):
            qkv = torch.nn.functional.rms_norm(x.float(), x.shape[-1:]).bfloat16() @ self.w_qkv[layer].T
            q, k, v = qkv.unflatten(1, (self.heads + 2 * self.kv, self.hd)).split([self.heads, self.kv, self.kv], dim=1)
            put = () if slots is None else (self.layout, self.k_cache[layer], self.v_cache[layer], slots)
            ivit.ivit_qk_norm_rope(self.rope, q, k, v if put else None, self.norm, self.norm, positions, self.freq, self.axis, q, k,
                                   *put)  # (in place, in the projection's output)
            out = torch.empty((n, self.heads, self.hd), dtype=torch.bfloat16, device="cuda")
            self.attend(layer, cfg, q, k, v, cu, mask, out, ws)
            x = x + out.flatten(1) @ self.w_o[layer].T
            keys.append(k)
            values.append(v)
        return x.float() @ self.w_out.T, torch.stack(keys), torch.stack(values)

    def prompt(self, tokens, grid_h, grid_w, time=0):
        """A view's tokens [n, token_dim]: every token sees all of them."""
        n = tokens.shape[0]
        cu, slots, _, _ = self.plan(n)
        i = torch.arange(n, device="cuda")
        positions = torch.stack([torch.full_like(i, time), i // grid_w, i % grid_w]).int()
        logits, _, _ = self.forward(tokens @ self.project.T, cu, positions, "all", None, slots)
        self.length += n
        return int(logits[-1].argmax())

    def step(self, tokens, parents):
        """One pass over a tree of drafted tokens (the first is the root, known to be right): the tokens that greedy
        decoding gives after it, found by following the drafts that are right."""
        cu, slots, positions, mask = self.plan(len(tokens), _i32(*parents))
        logits, k, v = self.forward(self.embed[torch.tensor(tokens, device="cuda")], cu, positions, "tree", mask)
        best = logits.argmax(1).tolist()
        path, said = [0], [best[0]]
        while True:
            right = [i for i, (t, p) in enumerate(zip(tokens, parents)) if p == path[-1] and t == said[-1]]
            if not right:
                break
            path.append(right[0])
            said.append(best[right[0]])
        ivit.ivit_kv_write(self.layout, k, v, _i32(*path), slots, self.k_cache, self.v_cache)
        self.length += len(path)
        return said


class QuantisedBackbone(Backbone):
    """The same over a cache of 8 bits, with a scale for each ``block`` tokens of a page and key head."""

    def __init__(self, *args, block=8, **kw):
        super().__init__(*args, **kw)
        shape = self.k_cache.shape
        self.k_cache, self.v_cache = (torch.zeros(shape, dtype=torch.float8_e4m3fn, device="cuda") for _ in range(2))
        self.k_scale, self.v_scale = (torch.zeros((*shape[:2], PAGE // block, self.kv), device="cuda") for _ in range(2))
        self.layout = ivit.make_quantised_layout(self.k_cache[0], block)

    def workspace(self, cfg):
        return ivit.ivit_tree_attention_quantised_workspace(cfg, self.layout)

    def attend(self, layer, cfg, q, k, v, cu, mask, out, ws):
        ivit.ivit_tree_attention_quantised(cfg, self.layout, q, k, v, self.k_cache[layer], self.v_cache[layer], self.k_scale[layer],
                                           self.v_scale[layer], self.table, _i32(self.length), cu, mask, out, None, ws)

    def write(self, k, v, rows, slots):
        ivit.ivit_kv_quantise(self.layout, k, v, rows, slots, self.k_cache, self.v_cache, self.k_scale, self.v_scale)

    def forward(self, x, cu, positions, mask_mode, mask, slots=None):
        logits, k, v = super().forward(x, cu, positions, mask_mode, mask)
        if slots is not None:  # a prompt's rows, all of them
            self.write(k, v, torch.arange(x.shape[0], dtype=torch.int32, device="cuda"), slots)
        return logits, k, v

    def sampled_step(self, tokens, parents, probs, temperature, generator):
        """One pass over a tree of drafts, of which those behind a node were drawn from its row of ``probs``: the tokens that
        follow the root, distributed as if the backbone had been sampled token by token."""
        n = len(tokens)
        parents = _i32(*parents)
        cu, slots, positions, mask = self.plan(n, parents)
        logits, k, v = self.forward(self.embed[tokens.long()], cu, positions, "tree", mask)
        vocab = logits.shape[1]
        uniform = torch.rand(n, generator=generator, device="cuda")
        noise = torch.empty((1, vocab), device="cuda").exponential_(generator=generator)
        path, accepted, after = (torch.empty(m, dtype=torch.int32, device="cuda") for m in (n, 1, 1))
        cfg = ivit.make_verify_config(1, vocab, n, "float32")
        ivit.ivit_tree_verify(cfg, logits, probs, tokens, parents, cu, torch.full((1,), temperature, device="cuda"), uniform, noise,
                              path, accepted, after)
        self.write(k, v, path, slots)  # (rows that were not accepted are -1 there)
        count = int(accepted)
        self.length += count
        return tokens[path[1:count].long()].tolist() + [int(after)]


def encode(seed=0):
    """Tokens of one camera frame, and their grid."""
    shape = synth.EncoderShape(112, 112, 14, 192, 2, 3, 520, synth.GELU_TANH)
    encoder = ivit.IncrementalViT(shape, synth.make_weights(shape, seed))
    frame = next(iter(synth.stream_random(shape, 1, 1, seed, change_p=0.2)))
    tokens = encoder.encode_full(torch.from_numpy(frame).cuda())[0].clone()
    encoder.close()
    return tokens, shape.grid_h, shape.grid_w


def decode(count=40, seed=0, drafts=4, right=0.8):
    """``count`` tokens one at a time and by trees of two candidates at each of ``drafts`` depths: both lists, and the
    passes that each took."""
    tokens, h, w = encode(seed)
    one = Backbone(tokens.shape[1], seed)
    said = [one.prompt(tokens, h, w)]
    while len(said) < count + drafts + 1:
        said += one.step(said[-1:], [-1])
    tree = Backbone(tokens.shape[1], seed)
    found = [tree.prompt(tokens, h, w)]
    r = np.random.default_rng(seed)
    while len(found) < count:
        nodes, parents, at = [found[-1]], [-1], 0
        for d in range(drafts):  # the drafter: the next token is among its two guesses some of the time
            guess = [int(t) for t in r.integers(0, 128, 2)]
            hit = int(r.integers(0, 2))
            if r.random() < right:
                guess[hit] = said[len(found) + d]
            nodes += guess
            parents += [at, at]
            at = len(nodes) - 2 + hit
        found += tree.step(nodes, parents)
    return said[:count], found[:count], one.passes, tree.passes


def sample(count=40, seed=0, drafts=3, temperature=0.7):
    """``count`` tokens over a cache of 8 bits, by trees of two candidates behind each of ``drafts`` nodes that a drafter, which knows
    the last token alone, draws from its probabilities: the tokens, and the passes that they took."""
    tokens, h, w = encode(seed)
    b = QuantisedBackbone(tokens.shape[1], seed)
    g = torch.Generator(device="cuda").manual_seed(seed)
    bigram = torch.softmax(b.embed.float() @ b.w_out.T / temperature, 1)
    said = [b.prompt(tokens, h, w)]
    while len(said) < count:
        nodes, parents = [said[-1]], [-1]
        for node in range(drafts):  # (breadth first: two behind the root, two behind the first of them, ...)
            nodes += torch.multinomial(bigram[nodes[node]], 2, replacement=True, generator=g).tolist()
            parents += [node, node]
        ids = _i32(*nodes)
        said += b.sampled_step(ids, parents, bigram[ids.long()].contiguous(), temperature, g)
    return said[:count], b.passes


if __name__ == "__main__":
    said, found, passes_one, passes_tree = decode()
    print("one at a time:", said)
    print("by trees:     ", found)
    print(f"{'the same' if said == found else 'DIFFERENT'}; {passes_one} passes against {passes_tree}")
    said, passes = sample()
    print("sampled, 8-bit cache:", said)
    print(f"{passes} passes")
