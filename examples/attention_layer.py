"""A compressed prompt through one attention layer: prefill, then decoding behind it.

The pass turns a synthetic prompt (workloads/) into macro-tokens and their
positions; a layer of random weights projects them to queries, keys and values
(plain matrix products), appends them to a paged cache (norm of queries and
keys, rotation by the macro-tokens' positions), attends over the prompt, and
then takes new tokens one by one, at the positions that follow the
uncompressed prompt.  The last decoded token is compared with the same token
taken through prefill.

    python examples/attention_layer.py [--workload tiny] [--steps 8]
"""
import argparse
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2607_19368_gb300 as sls  # noqa: E402
import workloads as WL  # noqa: E402

PAGE = 64


class Layer:
    """Random projections of one attention layer, its norms and rotation."""

    def __init__(self, d, q_heads, kv_heads, head_dim, seed=0):
        g = torch.Generator("cuda").manual_seed(seed)

        def weight(rows, cols):
            return (torch.randn(rows, cols, generator=g, device="cuda") * cols ** -0.5).bfloat16()

        self.heads = (q_heads, kv_heads, head_dim)
        self.qkv = weight((q_heads + 2 * kv_heads) * head_dim, d)
        self.out = weight(d, q_heads * head_dim)
        self.q_norm = torch.ones(head_dim, device="cuda").bfloat16()
        self.k_norm = torch.ones(head_dim, device="cuda").bfloat16()
        self.rope = sls.Rope.make(head_dim, base=1e6)

    def project(self, x):
        q, k, _ = self.heads
        y = torch.nn.functional.linear(x, self.qkv).view(x.shape[0], -1, self.heads[2])
        return y[:, :q], y[:, q:q + k], y[:, q + k:]


class Cache:
    """Pages of one sequence, handed out in order."""

    def __init__(self, layer, tokens):
        _, kv_heads, head_dim = layer.heads
        pages = -(-tokens // PAGE)
        shape = (pages, PAGE, kv_heads, head_dim)
        self.k = torch.empty(shape, dtype=torch.bfloat16, device="cuda")
        self.v = torch.empty(shape, dtype=torch.bfloat16, device="cuda")
        self.table = torch.arange(pages, dtype=torch.int32, device="cuda").view(1, pages)
        self.lens = torch.zeros(1, dtype=torch.int32, device="cuda")


def attend(layer, cache, x, positions):
    """One call of the layer on new tokens x (n x d) at `positions` (int32)."""
    n = x.shape[0]
    q, k, v = layer.project(x)
    cache.lens += n
    cu = torch.tensor([0, n], dtype=torch.int32, device="cuda")
    q = sls.qkv_append(q, k, v, cache.k, cache.v, cache.table, cache.lens,
                       cu_seqlens=cu, positions=positions, q_weight=layer.q_norm,
                       k_weight=layer.k_norm, rope=layer.rope)
    if n == 1:
        o = sls.attention_decode(q, cache.k, cache.v, cache.table, cache.lens)
    else:
        o = sls.attention_prefill(q, cache.k, cache.v, cache.table, cache.lens, cu)
    return torch.nn.functional.linear(o.view(n, -1), layer.out)


def run(workload="tiny", steps=8, q_heads=8, kv_heads=2, head_dim=64):
    w = WL.WORKLOADS[workload]
    prompt, prm = WL.make_prompt(w), WL.params_for(w)

    def put(a):
        t = torch.from_numpy(np.ascontiguousarray(a if w.dtype != "bf16" else a.view(np.int16)))
        return (t.view(torch.bfloat16) if w.dtype == "bf16" else t).cuda()

    cfg = sls.Config.make(rho=w.rho, D=w.D, r=w.r, bits=w.bits, preserve_last=w.preserve_last)
    Xt, pos, _, _, _ = sls.compress(put(prompt.X), cfg, put(prm.W), torch.from_numpy(prm.b).cuda(),
                                    torch.from_numpy(prm.R).cuda(), torch.from_numpy(prm.q1).cuda())
    M = Xt.shape[0]
    layer = Layer(w.d, q_heads, kv_heads, head_dim)
    # unit rows, as a norm in front of the layer leaves them
    x = torch.nn.functional.normalize(Xt, dim=1).mul(w.d ** 0.5).bfloat16()
    g = torch.Generator("cuda").manual_seed(1)
    new = torch.randn(steps, w.d, generator=g, device="cuda").bfloat16()
    at = torch.arange(w.N, w.N + steps, dtype=torch.int32, device="cuda")

    cache = Cache(layer, M + steps)
    first = attend(layer, cache, x, pos)
    for i in range(steps):
        last = attend(layer, cache, new[i:i + 1], at[i:i + 1])
    # the same tokens in one prefill
    again = Cache(layer, M + steps)
    whole = attend(layer, again, torch.cat([x, new]), torch.cat([pos, at]))
    torch.cuda.synchronize()
    far = [((a.float() - b.float()).norm() / b.float().norm()).item()
           for a, b in ((first, whole[:M]), (last[0], whole[-1]))]
    print(f"{w.N} tokens -> {M} macro-tokens at positions {int(pos[0])}..{int(pos[-1])}; "
          f"{steps} decoded; prefill against prefill {far[0]:.1e}, decode against prefill "
          f"{far[1]:.1e}")
    return M, far


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__,
                                 formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--workload", default="tiny", choices=sorted(WL.WORKLOADS))
    ap.add_argument("--steps", type=int, default=8)
    a = ap.parse_args()
    run(a.workload, a.steps)
