"""One layer served from the paged 8-bit cache: a prompt is stored, evicted to a budget, compacted into fewer pages, forked
into branches, and every branch decodes on.

The layer is a stand-in (random projections of a random residual stream); everything around it is what a serving program
does with the library: store the prompt, keep what the eviction keeps, give the other pages back, then, per step, make
room, copy shared pages, store the new tokens and attend.

    python examples/serve_from_cache.py [prompt tokens] [budget] [branches] [steps]
"""
import os
import sys
import time

import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.abspath(__file__)), ".."))
from paper_2507_06517_amd import binding as sb  # noqa: E402

D, H, G, WINDOW, POOL, PAGE = 128, 8, 4, 32, 7, 64


class Layer:
    """Projections of a residual stream [tokens, D], brought to unit mean square, to queries, keys and values."""

    def __init__(self, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.wq, self.wk, self.wv = (torch.randn(D, n * D, generator=g, device="cuda").div_(D ** 0.5).half() for n in (H * G, H, H))
        self.wo = torch.randn(H * G * D, D, generator=g, device="cuda").div_((H * G * D) ** 0.5).half()

    def __call__(self, x):
        x = (x.float() * x.float().square().mean(-1, keepdim=True).rsqrt()).half()
        return (x @ self.wq).view(-1, H * G, D), (x @ self.wk).view(-1, H, D), (x @ self.wv).view(-1, H, D)


def ints(*v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def serve(prompt=4096, budget=1024, branches=4, steps=16, fmt="e4m3", seed=0):
    """Returns the branches' outputs [steps, branches, D], the pages in use after the prompt, after the eviction and at the end, and
    the seconds of the decode steps."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    layer = Layer(seed)
    n_prompt, n_kept = -(-prompt // PAGE), -(-budget // PAGE)
    width = max(n_prompt, -(-(budget + steps) // PAGE))
    n_pages = n_prompt + n_kept + branches * (1 + -(-steps // PAGE)) + 8
    cache = sb.new_cache(n_pages, H, PAGE, fmt, positions=True)
    refs = torch.zeros(n_pages, dtype=torch.int32, device="cuda")
    in_use = []

    # the prompt, stored whole (its own attention is the model's business)
    x = torch.randn(prompt, D, generator=g, device="cuda").half()
    q, k, v = layer(x)
    table = torch.full((1, width), -1, dtype=torch.int32, device="cuda")
    lens, _, status = sb.pages_reserve(refs, table, ints(0), ints(prompt), PAGE)
    assert status.tolist() == [0, 0]
    sb.cache_append(cache, table, ints(0), k, v, cu_new=ints(0, prompt), max_new=prompt)
    in_use.append(int((refs > 0).sum()))

    # what the eviction keeps goes into pages of its own, the prompt's pages are given back
    K, V = (t.view(1, prompt, H, D).transpose(1, 2) for t in (k, v))
    Qw = q[-WINDOW:].view(1, WINDOW, H * G, D).transpose(1, 2).contiguous()
    kept = sb.compress_deep(K, V, Qw, G, "f16", WINDOW, POOL, budget)[0]
    small = torch.full_like(table, -1)
    small_lens, _, status = sb.pages_reserve(refs, small, ints(0), ints(budget), PAGE)
    assert status.tolist() == [0, 0]
    sb.cache_compact(cache, table, lens, kept, small_lens, small)
    sb.pages_release(refs, table, lens, PAGE)
    in_use.append(int((refs > 0).sum()))

    # branches share the pages; the first token of each takes a copy of the last one, if that is half full
    table, lens = sb.pages_share(refs, small, small_lens, torch.zeros(branches, dtype=torch.int32, device="cuda"), PAGE)
    sb.pages_release(refs, small, small_lens, PAGE)
    one, cu = torch.ones(branches, dtype=torch.int32, device="cuda"), torch.arange(branches + 1, dtype=torch.int32, device="cuda")
    x = x[-1:] + 0.1 * torch.randn(branches, D, generator=g, device="cuda").half()
    outs = []
    torch.cuda.synchronize()
    begin = time.perf_counter()
    for step in range(steps):
        q, k, v = layer(x)
        at = torch.full((branches,), prompt + step, dtype=torch.int32, device="cuda")   # places in the text, not in the cache
        longer, copies, _ = sb.pages_reserve(refs, table, lens, one, PAGE)   # (the pool has pages for every step: no status to wait for)
        sb.cache_copy(cache, copies)
        sb.cache_append(cache, table, lens, k, v, cu_new=cu, max_new=1, positions=at)
        o = sb.cache_attend(cache, table, longer, q, G, cu_q=cu, max_q=1, q_pos=at)
        lens = longer
        x = x + o.view(branches, -1) @ layer.wo
        outs.append(x)
    torch.cuda.synchronize()
    seconds = time.perf_counter() - begin
    in_use.append(int((refs > 0).sum()))
    sb.pages_release(refs, table, lens, PAGE)
    assert int(refs.abs().sum()) == 0
    return torch.stack(outs), in_use, seconds


if __name__ == "__main__":
    arguments = [int(a) for a in sys.argv[1:]]
    serve(*arguments)                              # the first pass loads the kernels
    out, pages, seconds = serve(*arguments)
    print(f"pages in use: {pages[0]} for the prompt, {pages[1]} after the eviction, {pages[2]} with {out.shape[1]} branches; "
          f"{seconds / out.shape[0] * 1e6:.0f} us per step")
