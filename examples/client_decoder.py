"""A small decoder whose every linear layer is delegated, from a prompt to generated tokens.

    python examples/client_decoder.py [--tokens 12] [--prompt 20] [--layers 2] [--temperature 0.8]

The client owns activations, cache, norms and the choice of tokens; the server owns the weights.  All that the
client does between two products runs in the library: integers go out, field elements come back, and no torch
operation lies between them but the lookup of the tokens' embeddings:

    pvmvmd_block_norm       residual stream -> integers of q, k, v's input
    [ q, k, v ]             pvmvmd_encode -> pvmvmd_server_mvm_grouped -> pvmvmd_decode_verify
    pvmvmd_kv_append        field elements -> rotated q, cache
    pvmvmd_paged_attention
    pvmvmd_glu              (without an activation) attention -> integers of o's input
    [ o ]
    pvmvmd_block_norm       residual added, normed -> integers of the feed-forward block's input
    [ gate and up ]         one matrix
    pvmvmd_glu              silu(gate) up -> integers of down's input
    [ down ]                ... and so on; behind the last layer
    [ vocabulary ]
    pvmvmd_sample           field elements -> tokens

Weights are synthetic; shapes are a small model's.
"""
import argparse
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
from client_attention import Delegated, pv, wl  # noqa: E402


class Decoder:
    """`layers` layers of `heads` query heads over `kv_heads` key heads of `dim`, and a feed-forward block of `inner`."""

    def __init__(self, layers=2, hidden=256, heads=4, kv_heads=2, dim=64, inner=704, vocabulary=1000, room=128, page=16, seed=0,
                 sampling=None):
        self.layers, self.hidden, self.heads, self.kv_heads, self.dim, self.inner = layers, hidden, heads, kv_heads, dim, inner
        rng = np.random.default_rng(seed)
        bf16 = lambda a: torch.from_numpy(a.astype(np.float32)).to(torch.bfloat16).cuda()  # noqa: E731
        shapes = {"q": (heads * dim, hidden), "k": (kv_heads * dim, hidden), "v": (kv_heads * dim, hidden),
                  "o": (hidden, heads * dim), "gate_up": (2 * inner, hidden), "down": (hidden, inner)}
        key = 100 * (seed + 1)
        self.W, self.mat, self.scale = {}, {}, {}
        names = [(l, n, s) for l in range(layers) for n, s in shapes.items()] + [(-1, "vocabulary", (vocabulary, hidden))]
        for i, (l, n, (m, K)) in enumerate(names):
            self.W[l, n] = wl.weights_gaussian(m, K, (seed, i))
            self.mat[l, n] = Delegated(self.W[l, n], key=key + i)
            self.scale[l, n] = 1.0 / (32.0 * K**0.5)  # a row of K weights of about 32: products of about the input's size
        self.norms = [pv.Norm("rms", bf16(1 + 0.1 * rng.standard_normal(hidden)), eps=1e-5) for _ in range(2 * layers + 1)]
        self.embedding = bf16(rng.standard_normal((vocabulary, hidden)))
        pages = -(-room // page)
        self.room, self.length = pages * page, 0
        new = lambda: torch.zeros(pages, page, kv_heads, dim, dtype=torch.bfloat16, device="cuda")  # noqa: E731
        self.pools = [pv.KvPool(new(), new()) for _ in range(layers)]
        self.table = torch.arange(pages, dtype=torch.int32, device="cuda")[None]
        self.lens = torch.zeros(1, dtype=torch.int32, device="cuda")
        self.rope = pv.pvmvmd_rope_table(dim, base=500000.0)
        self.sampling = sampling or pv.Sampling(0.8, 50, 0.95)
        self.random = np.random.default_rng(seed + 1)
        self.key = 1 << 40

    def _key(self):
        self.key += 1  # a key masks one call only
        return self.key

    def delegate(self, layer, names, x):
        """The products of a layer's matrices with integers x (T x K field elements), masked, verified and decrypted."""
        mats = [self.mat[layer, n] for n in names]
        masked = [pv.pvmvmd_encode(m.ctx, x, self._key()) for m in mats]
        Yh = [torch.empty((x.shape[0], m.W.shape[0]), dtype=torch.int32, device="cuda") for m in mats]
        pv.pvmvmd_server_mvm_grouped([(m.W, Xh, y) for m, (Xh, _), y in zip(mats, masked, Yh)])
        out = []
        for n, m, (Xh, st), y in zip(names, mats, masked, Yh):
            Y, accept = pv.pvmvmd_decode_verify(m.ctx, st, Xh, y, self._key())
            if int(accept.min()) != 1:
                raise RuntimeError(f"the server's product with {n} of layer {layer} was rejected")
            out.append(Y)
        return out

    def step(self, tokens, seen=None):
        """New tokens (int64, T) -> the next one, as a tensor.  seen: a list that takes what passes by, in order."""
        T = tokens.shape[0]
        if self.length + T > self.room:
            raise ValueError(f"{T} tokens behind {self.length} are more than the cache's {self.room} places")
        see = seen.append if seen is not None else lambda x: None
        self.lens += T
        batch = pv.KvBatch(self.table, self.lens, None if T == 1 else torch.tensor([0, T], dtype=torch.int32, device="cuda"),
                           max_new=T)
        positions = torch.arange(self.length, self.length + T, dtype=torch.int32, device="cuda")
        self.length += T
        ints = lambda width: torch.empty((T, width), dtype=torch.int32, device="cuda")  # noqa: E731
        steps = lambda: torch.empty(T, device="cuda")  # noqa: E731
        h = self.embedding[tokens].float()  # the residual stream, in 32 bits
        see(h.clone())
        y = None  # the last block's output
        for l in range(self.layers):
            x = ints(self.hidden)  # q, k and v share one scale, which the append takes: normed values have one size
            pv.pvmvmd_block_norm(y, h, residual_out=h if y is not None else False, pre=self.norms[2 * l], out=x, out_scale=32.0)
            q, k, v = self.delegate(l, ("q", "k", "v"), x)
            see((x, q, k, v, h.clone()))
            q = pv.pvmvmd_kv_append(self.pools[l], batch, k.view(T, self.kv_heads, self.dim), v.view(T, self.kv_heads, self.dim),
                                    positions, self.rope, q=q.view(T, self.heads, self.dim), scale=self.scale[l, "q"] / 32.0)
            attended = pv.pvmvmd_paged_attention(self.pools[l], batch, q).view(T, -1)
            x, step = ints(self.heads * self.dim), steps()
            pv.pvmvmd_glu(attended, act="none", out=x, out_token_scale=step)
            (o,) = self.delegate(l, ("o",), x)
            see((attended, x, step, o))
            x, y_step = ints(self.hidden), steps()
            pv.pvmvmd_block_norm(pv.Rows(o, self.scale[l, "o"], step), h, residual_out=h, pre=self.norms[2 * l + 1], out=x,
                                 out_token_scale=y_step)
            (gu,) = self.delegate(l, ("gate_up",), x)
            see((x, y_step, gu, h.clone()))
            x, step = ints(self.inner), steps()
            s = self.scale[l, "gate_up"]
            pv.pvmvmd_glu(pv.Rows(gu[:, :self.inner], s, y_step), pv.Rows(gu[:, self.inner:], s, y_step), out=x,
                          out_token_scale=step)
            (down,) = self.delegate(l, ("down",), x)
            see((x, step, down))
            y = pv.Rows(down, self.scale[l, "down"], step)
        # the last token alone goes on
        x, step = ints(self.hidden)[-1:], steps()[-1:]
        last = pv.Rows(y.data[-1:], y.scale, y.token_scale[-1:])
        pv.pvmvmd_block_norm(last, h[-1:], residual_out=h[-1:], pre=self.norms[-1], out=x, out_token_scale=step)
        (logits,) = self.delegate(-1, ("vocabulary",), x)
        word = torch.from_numpy(self.random.integers(0, 2**32, 1, dtype=np.uint32).view(np.int32)).cuda()
        logprob = torch.empty(1, device="cuda")
        token = pv.pvmvmd_sample(pv.Rows(logits, 2.0 * self.scale[-1, "vocabulary"], step), word, self.sampling, logprob=logprob)
        see((x, step, logits, word, token, logprob))
        return token


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--tokens", type=int, default=12)
    ap.add_argument("--prompt", type=int, default=20)
    ap.add_argument("--layers", type=int, default=2)
    ap.add_argument("--temperature", type=float, default=0.8)
    a = ap.parse_args()
    model = Decoder(layers=a.layers, sampling=pv.Sampling(a.temperature, 50, 0.95))
    prompt = torch.from_numpy(np.random.default_rng(3).integers(0, 1000, a.prompt)).cuda()
    token, out = model.step(prompt), []
    for _ in range(a.tokens):
        out.append(int(token))
        token = model.step(token.long())
    pv.pvmvmd_device_status()
    print(f"prompt of {a.prompt}, then {out}")


if __name__ == "__main__":
    main()
