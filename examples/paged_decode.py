"""One layer of a looped model that goes on after its prompt, on a cache that holds 8 bits an element.

  prompt    in chunks: Q rotated, K and V appended (K rotated on the way), loop 1 = attention over the cache
  base      the prompt's rows read back as the cache holds them: what the sparse loops take as their loop-1 K and V
  loop 2    over the whole prompt (here: every token active) against that base, its residuals stored beside it
  decode    token by token: loop 1 dense over the cache, loop 2 sparse over the prompt's selected columns, which starts from
            loop 1's outputs and log-normalisers

Synthetic rows stand in for the projections.  `python examples/paged_decode.py` prints what came out; run() returns it.
"""
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import dataclasses

import torch

from paper_2609_29812_b200 import binding as B, pipeline as P, workloads


def run(prompt=1100, steps=3, heads=2, dim=128, chunk=400, columns=160, page=64, code=B.FL_INT8, seed=0):
    dev = "cuda:0"
    g = torch.Generator(device=dev)
    g.manual_seed(seed)
    rows = lambda n: torch.randn(n, 3, heads, dim, generator=g, device=dev).to(torch.bfloat16)     # Q | K | V of the stacked projection
    w = dataclasses.replace(workloads.config2(L=prompt, n_heads=heads), n_loops=2, q_block=256, col_budget=columns, changed_fracs=(0.3,))
    scale = w.sm_scale
    out = {"prompt_o": [], "prompt_lse": [], "decode": []}
    with B.Context(0) as ctx:
        rotary = P.RotaryTable(ctx, prompt + steps, dim, device=dev)
        cache = P.PagedCache(ctx, 1, heads, dim, prompt + steps, page=page, code=code, device=dev)

        # ---- prompt, loop 1 ------------------------------------------------------------------------------------
        qkv = rows(prompt)
        q = rotary.rotate(qkv[:, 0], None)
        for t in range(0, prompt, chunk):
            n = min(chunk, prompt - t)
            starts = cache.append(qkv[t:t + n, 1], qkv[t:t + n, 2], [n], rotary)
            o, lse = cache.attend(q[t:t + n], [n], scale, starts)
            out["prompt_o"].append(o)
            out["prompt_lse"].append(lse)
        k_base, v_base = cache.read(0)

        # ---- loop 2 of the prompt against the base that the cache holds ----------------------------------------
        st = P.LayerState(ctx, w, dev)
        st.dense_loop(q, k_base, v_base)
        st.select_columns_dense()
        every = torch.arange(prompt, dtype=torch.int32, device=dev)
        sel = P.TokenSelection(every, every.clone(), torch.zeros(prompt, device=dev), prompt)
        delta = lambda x: (x.float() + 0.05 * torch.randn(x.shape, generator=g, device=dev)).to(torch.bfloat16)
        q2, k2, v2 = delta(q), delta(k_base), delta(v_base)
        st.sparse_loop(2, q2, k2, v2, sel, indexed=True)

        # ---- decode --------------------------------------------------------------------------------------------
        for step in range(steps):
            x = rows(1)
            qn = rotary.rotate(x[:, 0], None, pos0=prompt + step)
            starts = cache.append(x[:, 1], x[:, 2], [1], rotary)
            o1, lse1 = cache.attend(qn, [1], scale, starts)
            q2 = delta(qn)
            # each head's subset: the columns of the prompt that loop 1 gives the most
            p = torch.einsum("qhd,khd->qhk", qn.float(), k_base.float())
            cols = p.topk(columns, -1).indices.sort(-1).values.to(torch.int32).contiguous()
            cnt = torch.full((1, heads), columns, dtype=torch.int32, device=dev)
            o2, lse2 = torch.empty_like(o1), torch.empty_like(lse1)
            B.fl_decode_attention(ctx, st.shape, 2, q2, qn, 1, st.store, cols, cnt, columns, lse1, lse2, o1, o2)
            out["decode"].append(dict(q=qn, q2=q2, o1=o1, lse1=lse1, cols=cols, o2=o2, lse2=lse2))
        st.check_status()
        cache.check_status()
        k_all, v_all = cache.read(0)
        out.update(k=k_all, v=v_all, q=q, k2=k2, v2=v2, sm_scale=scale, o_loop1=torch.cat(out.pop("prompt_o")), lse_loop1=torch.cat(out.pop("prompt_lse")))
        torch.cuda.synchronize()
    return out


if __name__ == "__main__":
    r = run()
    print(f"prompt: {r['o_loop1'].shape[0]} tokens, mean |o| {r['o_loop1'].float().abs().mean():.4f}")
    for i, d in enumerate(r["decode"]):
        print(f"token {i}: lse of loop 1 {d['lse1'].flatten().tolist()}, |o2 - o1| {(d['o2'].float() - d['o1'].float()).abs().mean():.4f}")
