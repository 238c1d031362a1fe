"""A client's attention block with its linear layers delegated, token by token.

    python examples/client_attention.py [--tokens 24] [--prompt 40] [--budget 48]

The client owns the activations and the cache; the server owns W_q, W_k, W_v and
W_o.  Each step of the loop is the paper's client loop for one attention block
(Sec. 7.2), for a prompt first and then one token at a time:

    pvmvmd_encode -> pvmvmd_server_mvm_grouped -> pvmvmd_decode_verify   q, k, v
    pvmvmd_kv_append                  field elements -> rotated q, cache
    pvmvmd_paged_attention            over the cache, weights accumulated
    pvmvmd_kv_evict                   once the cache is longer than its budget
    pvmvmd_encode -> pvmvmd_server_mvm -> pvmvmd_decode_verify           o

Weights and inputs are synthetic; shapes are a small model's.
"""
import argparse
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2609_10264_gb300 as pv  # noqa: E402
from paper_2609_10264_gb300 import workloads as wl  # noqa: E402

Q = pv.PVMVMD_Q


class Delegated:
    """One int8 weight matrix: the client's context, the server's copy."""

    def __init__(self, W, key):
        self.W = torch.from_numpy(W).cuda()
        self.ctx = pv.pvmvmd_preprocess(self.W, key=key)


def embed(x):
    """Integers -> field elements."""
    return torch.remainder(x.to(torch.int64), Q).to(torch.int32)


class AttentionBlock:
    """The client's side of one attention block: `heads` query heads over `kv_heads` key heads of `dim`."""

    def __init__(self, hidden=512, heads=8, kv_heads=2, dim=64, budget=48, recent=8, room=256, page=16, seed=0):
        self.hidden, self.heads, self.kv_heads, self.dim = hidden, heads, kv_heads, dim
        self.budget, self.recent, self.seed = budget, recent, seed
        shapes = {"q": heads * dim, "k": kv_heads * dim, "v": kv_heads * dim}
        self.W = {n: wl.weights_gaussian(m, hidden, (seed, i)) for i, (n, m) in enumerate(shapes.items())}
        self.W["o"] = wl.weights_gaussian(hidden, heads * dim, (seed, 3))
        self.mat = {n: Delegated(W, key=100 + i) for i, (n, W) in enumerate(self.W.items())}
        pages = -(-room // page)
        self.room = pages * page
        self.pool = pv.KvPool(torch.zeros(pages, page, kv_heads, dim, dtype=torch.bfloat16, device="cuda"),
                              torch.zeros(pages, page, kv_heads, dim, dtype=torch.bfloat16, device="cuda"),
                              torch.zeros(pages, kv_heads, page, device="cuda"))
        self.table = torch.arange(pages, dtype=torch.int32, device="cuda")[None]
        self.lens = torch.zeros(1, dtype=torch.int32, device="cuda")
        self.rope = pv.pvmvmd_rope_table(dim, base=500000.0)
        # an int8 activation of 64 is 1; a row of W has `hidden` entries of about 32: products back to about 1
        self.in_scale = 1.0 / (64 * 32 * hidden**0.5)
        self.out_scale = 64.0
        self.position, self.key, self.length = 0, 1 << 40, 0

    def _key(self):
        self.key += 1  # a key masks one call only
        return self.key

    def delegate(self, names, x_int):
        """The products of the matrices `names` with x_int (T x K integers), masked, verified and decrypted."""
        X = embed(x_int)
        masked = [pv.pvmvmd_encode(self.mat[n].ctx, X, self._key()) for n in names]
        Yh = [torch.empty((X.shape[0], self.mat[n].W.shape[0]), dtype=torch.int32, device="cuda") for n in names]
        pv.pvmvmd_server_mvm_grouped([(self.mat[n].W, m[0], y) for n, m, y in zip(names, masked, Yh)])
        out = []
        for n, (Xh, st), y in zip(names, masked, Yh):
            Y, accept = pv.pvmvmd_decode_verify(self.mat[n].ctx, st, Xh, y, self._key())
            if int(accept.min()) != 1:
                raise RuntimeError(f"the server's product with W_{n} was rejected")
            out.append(Y)
        return out

    def step(self, x_int):
        """T new tokens' int8 activations (T x hidden) -> (T x hidden field elements of W_o's product, q, attention)."""
        T = x_int.shape[0]
        if self.length + T > self.room:  # nothing outside the table is written or seen
            raise ValueError(f"{T} tokens behind {self.length} are more than the cache's {self.room} places")
        q, k, v = self.delegate(("q", "k", "v"), x_int)
        self.lens += T
        self.length += T
        cu = None if T == 1 else torch.tensor([0, T], dtype=torch.int32, device="cuda")
        batch = pv.KvBatch(self.table, self.lens, cu, max_new=T)
        positions = torch.arange(self.position, self.position + T, dtype=torch.int32, device="cuda")
        self.position += T
        q = pv.pvmvmd_kv_append(self.pool, batch, k.view(T, self.kv_heads, self.dim), v.view(T, self.kv_heads, self.dim),
                                positions, self.rope, q=q.view(T, self.heads, self.dim), scale=self.in_scale)
        out = pv.pvmvmd_paged_attention(self.pool, batch, q, accumulate=True)
        if self.length > self.budget + self.recent:  # now and then, not for every token
            pv.pvmvmd_kv_evict(self.pool, batch, self.budget, self.recent)
            self.length = self.budget
        o_int = (out.float() * self.out_scale).round_().clamp_(-1023, 1023).reshape(T, -1)
        return self.delegate(("o",), o_int)[0], q, out


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--tokens", type=int, default=24)
    ap.add_argument("--prompt", type=int, default=40)
    ap.add_argument("--budget", type=int, default=48)
    a = ap.parse_args()
    block = AttentionBlock(budget=a.budget)
    rng = np.random.default_rng(1)
    act = lambda n: torch.from_numpy(rng.integers(-127, 128, size=(n, block.hidden), dtype=np.int64)).cuda()  # noqa: E731
    y, _, _ = block.step(act(a.prompt))
    print(f"prompt of {a.prompt}: {int(block.lens)} tokens cached")
    for _ in range(a.tokens):
        y, _, _ = block.step(act(1))
    pv.pvmvmd_device_status()
    print(f"{a.tokens} more tokens: {int(block.lens)} cached, next position {block.position}; "
          f"last output {pv.as_u32(y)[0, :4].tolist()} ...")


if __name__ == "__main__":
    main()
