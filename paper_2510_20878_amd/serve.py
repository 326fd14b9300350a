"""A small serving loop over one pool: questions to packed documents, answered token by token.

    python -m paper_2510_20878_amd.serve [--requests 8] [--steps 16] [--layers 4] [--check]

Every request retrieves some documents of the knowledge base (packed chunks in HBM: 16-bit, int8, int4) and asks a
question; its own tokens live in a paged cache.  Per step and layer: the new rows' keys and values go to their pages
(append_paged), their queries attend to the documents straight from the packed chunks (attend_chunks) and, merged with
that, to the request's own rows (attend_paged).  Between steps some requests end (their pages go back) and others take their place.  The
projections of a model are stood in for by random rows.  --check compares the last step with binary64 attention over documents and
own rows together."""
import argparse
import math
import time

import torch

from . import binding as B


def _documents(ctx, shape, n_docs, tokens, g):
    """The knowledge base: packed chunks 0 .. n_docs - 1 in HBM, hot ones in 16 bits."""
    L, H, D = shape
    precs = [(B.PREC_16, B.PREC_INT8, B.PREC_INT4)[min(2, i * 4 // n_docs)] for i in range(n_docs)]
    for prec in set(precs):
        slot = (ctx.chunk_bytes(prec, tokens) + 255) // 256 * 256
        ctx.register_slab(B.TIER_HBM, prec, torch.empty(slot * precs.count(prec), dtype=torch.uint8, device="cuda"))
    for i, prec in enumerate(precs):
        kv = torch.randn((L, 2, H, tokens, D), generator=g, device="cuda").bfloat16()
        ctx.pool_insert(i, prec, tokens, None, B.TIER_HBM)
        ctx.quantize_chunk(kv, tokens, prec, ctx.group_of(prec), ctx.pool_slot(i, B.TIER_HBM)[0])
        torch.cuda.synchronize()  # kv is reused
    ctx.rerank()


def _reference(ctx, shape, docs, pool, table, held, q, layer, tokens, P):
    """Binary64 attention of one request's new rows over its documents (as a load writes them) and its own rows."""
    L, H, D = shape
    cap = len(docs) * tokens
    cache = torch.empty((L, 2, H, cap, D), dtype=torch.bfloat16, device="cuda")
    ctx.load_chunks(docs, cache, cap)
    at = torch.arange(held, device="cuda")
    own = pool[table[at // P].long(), layer, :, :, at % P].permute(1, 2, 0, 3)
    k, v = torch.cat([cache[layer], own], 2).double()
    n, G = q.shape[0], q.shape[1] // H
    late = torch.arange(cap + held, device="cuda")[None] > torch.arange(cap + held - n, cap + held, device="cuda")[:, None]
    out = torch.empty(q.shape, dtype=torch.float64, device="cuda")
    for hq in range(q.shape[1]):
        s = (q[:, hq].double() @ k[hq // G].T.contiguous() * D ** -0.5).masked_fill(late, -math.inf)
        out[:, hq] = torch.softmax(s, -1) @ v[hq // G]
    return out


def serve(n_requests=8, n_steps=16, n_layers=4, kv_heads=8, q_heads=32, head_dim=128, doc_tokens=512, n_docs=32, per_request=4,
          question=(48, 17, 64, 33), answer=24, page_tokens=16, seed=0, check=False):
    """Runs the loop; returns (seconds a step that has rows, largest error of the last step over the size of its output; None without check, or if
    no request had rows in that step)."""
    shape = L, H, D = n_layers, kv_heads, head_dim
    P, scale = page_tokens, head_dim ** -0.5
    g = torch.Generator(device="cuda").manual_seed(seed)
    ctx = B.Context(L, H, D, doc_tokens, group_int8=128, group_int4=128)
    _documents(ctx, shape, n_docs, doc_tokens, g)

    i32 = dict(dtype=torch.int32, device="cuda")
    most = max(question) + answer
    n_table = -(-most // P)
    n_pages = n_requests * n_table
    n_rows = n_requests * max(question)
    pool = torch.zeros((n_pages, L, 2, H, P, D), dtype=torch.bfloat16, device="cuda")
    table = torch.full((n_requests, n_table), -1, **i32)
    held = torch.zeros(n_requests, **i32)
    tables = B.page_tables(table, held, torch.arange(n_pages, **i32), torch.full((1,), n_pages, **i32), P)
    cache = B.paged_cache(pool, table, P, n_pages, "page_major", L, H, D, n_table=n_table)
    plan = torch.empty(ctx.step_plan_bytes(n_requests, n_rows, q_heads), dtype=torch.uint8, device="cuda")
    starts, slots = torch.zeros(n_requests + 1, **i32), torch.zeros(n_rows, **i32)
    positions, refused = torch.zeros(n_rows, **i32), torch.zeros(n_requests, **i32)
    out = torch.zeros((L, n_rows, q_heads, D), dtype=torch.bfloat16, device="cuda")
    prior, prior_lse = torch.empty((n_rows, q_heads, D), device="cuda"), torch.empty((n_rows, q_heads), device="cuda")

    age = [-(i % 3) for i in range(n_requests)]  # steps that the request has seen; < 0: it has not come yet
    docs = [[(i * 7 + j) % n_docs for j in range(per_request)] for i in range(n_requests)]
    spent, worked, error = 0.0, 0, None
    for nth in range(n_steps):
        # what the scheduler decides, on the host: who brings a question, who decodes, who has ended
        new = [question[i % len(question)] if a == 0 else 1 if 0 < a < answer else 0 for i, a in enumerate(age)]
        n_new = torch.tensor(new, **i32)
        rows = max(sum(new), 1)
        # a plan is for its number of rows: decode alone and steps with questions are cut differently
        step = B.paged_step(starts, slots[:rows], q_heads, positions=positions, refused=refused, plan=plan)
        qkv = torch.randn((L, rows, (q_heads + 2 * H) * D), generator=g, device="cuda").bfloat16()
        q, k, v = (x.unflatten(-1, (-1, D)) for x in qkv.split([q_heads * D, H * D, H * D], -1))
        q = q.contiguous()
        first = [sum(new[:i]) for i in range(n_requests)]
        live = [i for i in range(n_requests) if new[i]]
        error = None
        if not live:  # one has ended and the next has not come yet
            age = [a + 1 for a in age]
            continue
        requests = [ctx.attend_id_lists([(docs[i], q[layer, first[i]:], prior[first[i]:], prior_lse[first[i]:], new[i]) for i in live])
                    for layer in range(L)]
        ws = torch.empty(max(ctx.attend_chunks_workspace_bytes(requests[0], q_heads), 16), dtype=torch.uint8, device="cuda")
        torch.cuda.synchronize()
        began = time.perf_counter()
        ctx.page_step(tables, n_new, step)
        for layer in range(L):
            ctx.append_paged(k[layer], v[layer], step, cache, layer)
            ctx.attend_chunks(requests[layer], layer, q_heads, scale, ws, count=layer == 0)
            ctx.attend_paged(q[layer], step, cache, layer, scale, out[layer], prior_out=prior, prior_lse=prior_lse)
        torch.cuda.synchronize()
        spent, worked = spent + time.perf_counter() - began, worked + 1
        assert not refused.any(), "the pool holds every request's longest conversation"
        if check and nth == n_steps - 1:
            error = 0.0
            for i in live:
                mine = slice(first[i], first[i] + new[i])
                want = _reference(ctx, shape, docs[i], pool, table[i], int(held[i]), q[L - 1, mine], L - 1, doc_tokens, P)
                error = max(error, float((out[L - 1, mine].double() - want).norm() / want.norm()))
        # requests that have answered give their pages back, and a new one with other documents takes the place
        ended = [i for i in range(n_requests) if age[i] == answer - 1]
        if ended:
            drop = torch.zeros(n_requests, **i32)
            drop[torch.tensor(ended, device="cuda")] = -most
            ctx.page_step(tables, drop, step)
            for i in ended:
                docs[i] = [(x + 3) % n_docs for x in docs[i]]
        age = [-1 if i in ended else a + 1 for i, a in enumerate(age)]
    torch.cuda.synchronize()
    ctx.destroy()
    return spent / max(worked, 1), error


def main(argv=None):
    p = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    p.add_argument("--requests", type=int, default=8)
    p.add_argument("--steps", type=int, default=16)
    p.add_argument("--layers", type=int, default=4)
    p.add_argument("--check", action="store_true")
    a = p.parse_args(argv)
    seconds, error = serve(a.requests, a.steps, a.layers, check=a.check)
    print(f"{a.steps} steps of {a.requests} requests, {a.layers} layers: {seconds * 1e6:.0f} us a step"
          + ("" if error is None else f"; last step's error against binary64 {error:.2g}"))


if __name__ == "__main__":
    main()
