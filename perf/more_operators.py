"""What differs from request to request in one batch of a target model, as cases that can be timed and compared.

Many requests share one target model and one pool of pages.  Each has a low-rank adapter of its own beside the shared
projections (`adapt`: a projection's result plus scale * B (A x), rows grouped by adapter); each samples with parameters of
its own from the logits of its row (`sample`: temperature, top-k, top-p and min-p, from a given uniform); and images of one
prompt share the prompt's pages until they write (`fork`: the pages are shared and the first pages to be written taken, the
part of a page that a request goes on in copied; `compact`: after requests have ended the pages in use move to the front of
the pool, tables rewritten).

Shapes are those of `synth.CONFIGS` (widths of 768, 1280 and 4096, slices of 16384 and 65536 entries, 36 layers of 20
heads of 64, 32 layers of 32 heads of 128, 120 condition rows) and generic ones.  Where `own` is false `run` computes in
elementary torch operations, in 32 bits, the sampling in 64 (its decisions are comparisons of neighbouring sums).
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda:0"
TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}


def listed():
    return [
        # One request, one token, the small model's width: all latency.
        dict(name="adapt-one", kind="adapt", n_seq=1, rows_lo=1, rows_hi=1, d_in=768, d_out=768, rank=8, n_adapters=4,
             without=0, x="bf16", out="bf16", base=True, scale=False),
        # A step of 16 requests, each the last token and five drafts; some requests have no adapter.
        dict(name="adapt-step", kind="adapt", n_seq=16, rows_lo=6, rows_hi=6, d_in=1280, d_out=3456, rank=16, n_adapters=8,
             without=3, x="bf16", out="bf16", base=True, scale=True),
        # Single tokens of many requests, as many adapters as a busy server holds, the large model's MLP.
        dict(name="adapt-many", kind="adapt", n_seq=200, rows_lo=1, rows_hi=1, d_in=4096, d_out=11008, rank=32, n_adapters=64,
             without=5, x="bf16", out="bf16", base=True, scale=True),
        # Pieces of four prompts of different requests, ragged.
        dict(name="adapt-prompt", kind="adapt", n_seq=4, rows_lo=700, rows_hi=1301, d_in=4096, d_out=4096, rank=16, n_adapters=8,
             without=0, x="bf16", out="bf16", base=True, scale=True),
        # A high rank, half precision in and 32 bits out, the adapter's part alone (added elsewhere).
        dict(name="adapt-rank", kind="adapt", n_seq=3, rows_lo=100, rows_hi=500, d_in=1280, d_out=1000, rank=128, n_adapters=3,
             without=0, x="fp16", out="fp32", base=False, scale=True),
        # One row over the image codes.
        dict(name="sample-one", kind="sample", rows=1, n=16384, x="fp32", top_k=1000, top_p=0.9, min_p=0.0, mixed=False),
        # A batch over the image codes, every request with parameters of its own.
        dict(name="sample-step", kind="sample", rows=96, n=16384, x="fp32", top_k=2000, top_p=0.95, min_p=0.02, mixed=True),
        # A batch over a whole vocabulary, cut by mass alone.
        dict(name="sample-vocab", kind="sample", rows=48, n=65536, x="fp32", top_k=0, top_p=0.9, min_p=0.0, mixed=False),
        # Few rows over a large vocabulary of odd size, logits of 16 bits.
        dict(name="sample-long", kind="sample", rows=4, n=200003, x="bf16", top_k=0, top_p=0.95, min_p=0.05, mixed=False),
        # One prompt of the small model, four images of it.
        dict(name="fork-one", kind="fork", prompts=1, images=4, layers=12, kv_heads=12, head_dim=64, page=16, cache="fp16",
             past_lo=120, past_hi=120, new_lo=6, new_hi=6),
        # Eight prompts, eight images of each, prompts that end inside a page.
        dict(name="fork-batch", kind="fork", prompts=8, images=8, layers=36, kv_heads=20, head_dim=64, page=16, cache="fp16",
             past_lo=100, past_hi=139, new_lo=1, new_hi=24),
        # A pool that ended requests have left in holes: the large model's pages.
        dict(name="compact-batch", kind="compact", n_seq=24, layers=32, kv_heads=32, head_dim=128, page=32, cache="bf16",
             past_lo=64, past_hi=300, moves=48),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["adapt", "adapt", "adapt", "sample", "sample", "fork", "compact"])
    if kind == "adapt":
        d_in = rng.choice([256, 768, 1280, 4096, 11008, 8 * _log(rng, 8, 640)])
        d_out = rng.choice([256, 768, 1280, 3456, 4096, 11008, 8 * _log(rng, 8, 640)])
        n_adapters = _log(rng, 1, 64)
        form = rng.choice(["one", "step", "step", "piece"])
        if form == "one":
            n_seq, lo, hi = _log(rng, 1, 256), 1, 1
        elif form == "step":
            n_seq, lo, hi = _log(rng, 1, 64), 0, rng.randint(2, 13)
        else:
            n_seq, lo, hi = rng.randint(1, 6), 1, _log(rng, 30, 600)
        return dict(kind=kind, n_seq=n_seq, rows_lo=lo, rows_hi=hi, d_in=d_in, d_out=d_out,
                    rank=rng.choice([8, 8, 16, 16, 16, 24, 32, 64, 128]), n_adapters=n_adapters, without=rng.choice([0, 0, 3, 10]),
                    x=rng.choice(["fp32", "bf16", "bf16", "fp16"]), out=rng.choice(["fp32", "bf16", "bf16", "fp16"]),
                    base=rng.random() < 0.7, scale=rng.random() < 0.7)
    if kind == "sample":
        n = rng.choice([4096, 8192, 16384, 65536, _log(rng, 300, 200000)])
        return dict(kind=kind, rows=_log(rng, 1, max(2, 3000000 // n if n > 12000 else 250)), n=n, x=rng.choice(["fp32", "fp32", "bf16", "fp16"]),
                    top_k=rng.choice([0, 0, 1000, _log(rng, 5, max(6, n // 2))]), top_p=rng.choice([1.0, 0.9, 0.95, round(rng.uniform(0.3, 0.99), 3)]),
                    min_p=rng.choice([0.0, 0.0, 0.05, round(rng.uniform(0.001, 0.2), 4)]), mixed=rng.random() < 0.4)
    kv_heads, head_dim = rng.choice([(20, 64), (32, 128), (8, 128), (4, 64), (2, 128), (1, 256), (12, 32), (3, 96), (6, 80)])
    c = dict(kind=kind, layers=_log(rng, 1, 32), kv_heads=kv_heads, head_dim=head_dim, page=rng.choice([8, 16, 24, 32, 64]),
             cache=rng.choice(["fp32", "bf16", "bf16", "fp16", "fp16"]))
    if kind == "fork":
        past = _log(rng, 1, 400)
        new = _log(rng, 1, 40)
        return dict(c, prompts=_log(rng, 1, 8), images=_log(rng, 1, 6), past_lo=rng.randint(0, past), past_hi=past,
                    new_lo=rng.randint(0, new), new_hi=new)
    past = _log(rng, 10, 250)
    return dict(c, n_seq=_log(rng, 2, 16), past_lo=rng.randint(1, past), past_hi=past, moves=rng.randint(0, 16))


# ------------------------------------------------------------------------------------------------------- inputs

def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _randn(g, *shape, dtype=torch.float32):
    return torch.randn(*shape, generator=g, device=DEV).to(dtype)


def _uniform(g, *shape):
    return torch.randint(0, 1 << 24, shape, generator=g, device=DEV).float() / float(1 << 24)


def _i32(a):
    return torch.tensor(np.asarray(a), dtype=torch.int32, device=DEV)


def _own_numbers(case):
    """Lengths are the case's own, so that inputs of another seed have the same shapes."""
    return np.random.RandomState(sum((i + 1) * v for i, v in enumerate(v for v in case.values() if type(v) is int)))


def _between(r, lo, hi, n):
    """n lengths from lo to hi, the upper bound among them."""
    a = r.randint(lo, hi + 1, n)
    a[r.randint(n)] = hi
    return a


def _rows_of(case):
    return _between(_own_numbers(case), case["rows_lo"], case["rows_hi"], case["n_seq"])


def _pool(g, *shape, dtype):
    """Keys or values of a pool, drawn in pieces."""
    out = torch.empty(*shape, dtype=dtype, device=DEV)
    flat = out.view(-1)
    step = 1 << 27
    for i in range(0, flat.numel(), step):
        m = min(step, flat.numel() - i)
        flat[i:i + m] = torch.randn(m, generator=g, device=DEV).to(dtype)
    return out


def prepare(case, seed):
    st = dict(case=dict(case))
    {"adapt": _prepare_adapt, "sample": _prepare_sample, "fork": _prepare_fork, "compact": _prepare_compact}[case["kind"]](st, case, _gen(seed), seed)
    return st


def _prepare_adapt(st, case, g, seed):
    r = np.random.RandomState((seed * 31 + 11) % (1 << 31))
    each = _rows_of(case)
    rows, x, out = int(each.sum()), TYPES[case["x"]], TYPES[case["out"]]
    adapter = r.randint(0, case["n_adapters"], case["n_seq"])
    if case["without"] and case["n_seq"] > 1:
        adapter[r.permutation(case["n_seq"])[::case["without"]]] = -1
    st.update(rows=rows, row_start=_i32(np.concatenate([[0], np.cumsum(each)])), adapter=_i32(adapter),
              x=_randn(g, rows, case["d_in"], dtype=x), base=_randn(g, rows, case["d_out"], dtype=out) if case["base"] else None,
              # as a trained adapter's: its part of the result is of the size of the projection's own, or below it
              a=(_randn(g, case["n_adapters"], case["rank"], case["d_in"]) * case["d_in"] ** -0.5).to(x),
              b=(_randn(g, case["n_adapters"], case["d_out"], case["rank"]) * case["rank"] ** -0.5).to(x),
              scale=0.25 + _uniform(g, case["n_adapters"]) if case["scale"] else None)
    if own:
        # which rows have which adapter is laid out once a step, for all projections of all layers
        import paper_2510_25739_amd as H
        st["plan"] = H.AdapterPlan(st["row_start"], st["adapter"], rows, case["n_adapters"])


def _prepare_sample(st, case, g, seed):
    rows, n = case["rows"], case["n"]
    # logits of a model that knows what it wants: a few entries far above a bulk
    z = _randn(g, rows, n) * 2.0 + 3.0 * (_uniform(g, rows, n) > 0.98)
    st.update(logits=z.to(TYPES[case["x"]]), u=_uniform(g, rows))
    if case["mixed"]:
        at = torch.arange(rows, device=DEV)
        st.update(temperature=torch.where(at % 7 == 3, torch.zeros(rows, device=DEV), 0.5 + _uniform(g, rows)),
                  top_k=torch.where(at % 3 == 1, torch.zeros_like(at), torch.randint(1, max(2, case["top_k"] or n), (rows,), generator=g, device=DEV)).int(),
                  top_p=torch.where(at % 4 == 2, torch.ones(rows, device=DEV), case["top_p"] - 0.2 * _uniform(g, rows)),
                  min_p=torch.where(at % 5 == 4, torch.zeros(rows, device=DEV), case["min_p"] * _uniform(g, rows)))
    else:
        st.update(temperature=torch.full((rows,), 0.8, device=DEV), top_k=torch.full((rows,), case["top_k"], dtype=torch.int32, device=DEV),
                  top_p=torch.full((rows,), case["top_p"], device=DEV), min_p=torch.full((rows,), case["min_p"], device=DEV))


def _pool_of(st, case, g, n_pages):
    shape = (case["layers"], n_pages, case["kv_heads"], case["page"], case["head_dim"])
    st.update(k_pool=_pool(g, *shape, dtype=TYPES[case["cache"]]), v_pool=_pool(g, *shape, dtype=TYPES[case["cache"]]))
    if own:
        import paper_2510_25739_amd as H
        st["cache"] = H.PagedCache(st["k_pool"], st["v_pool"], st["table"])


def _prepare_fork(st, case, g, seed):
    """Prompts in scattered pages of a pool, and as many free pages as their images may take."""
    r, own_r = np.random.RandomState((seed * 104729 + 7) % (1 << 31)), _own_numbers(case)
    n_p, n_i, page = case["prompts"], case["prompts"] * case["images"], case["page"]
    past = _between(own_r, case["past_lo"], case["past_hi"], n_p)
    new = _between(own_r, case["new_lo"], case["new_hi"], n_i)
    per = -(-past // page)
    cols = max(1, -(-(case["past_hi"] + case["new_hi"]) // page))
    n_pages = int(per.sum()) + n_i * (2 + case["new_hi"] // page) + 3
    order = r.permutation(n_pages)
    table, refs, at = np.full((n_p + n_i, cols), -1), np.zeros(n_pages), 0
    for s in range(n_p):
        table[s, :per[s]] = order[at:at + per[s]]
        at += per[s]
    refs[order[:at]] = 1
    st.update(table=_i32(table), refs=_i32(refs), n_past=_i32(np.concatenate([past, np.zeros(n_i, int)])),
              n_new=_i32(np.concatenate([np.full(n_p, -1), new])), src=_i32(np.arange(n_i) % n_p), dst=_i32(n_p + np.arange(n_i)))
    _pool_of(st, case, g, n_pages)


def _used_pages(case):
    """Pages of every sequence: its own, behind those that every four sequences share; how many the pool has in use."""
    past = _between(_own_numbers(case), case["past_lo"], case["past_hi"], case["n_seq"])
    per = -(-past // case["page"])
    shared = np.minimum(per, 2)
    first = np.arange(case["n_seq"]) % 4 == 0
    lead = np.maximum.accumulate(np.where(first, np.arange(case["n_seq"]), 0))
    shared = np.where(first, 0, np.minimum(shared, per[lead]))
    return per, lead, shared, int((per - shared).sum())


def _prepare_compact(st, case, g, seed):
    """A pool in which so many of the pages in use lie behind as many places as there are pages in use."""
    r = np.random.RandomState((seed * 104729 + 9) % (1 << 31))
    per, lead, shared, used = _used_pages(case)
    moves = min(case["moves"], used)
    n_pages = used + max(2 * moves, 8)
    at = r.permutation(np.concatenate([r.permutation(used)[:used - moves], used + r.permutation(n_pages - used)[:moves]]))
    table, refs, k = np.full((case["n_seq"], int(per.max())), -1), np.zeros(n_pages), 0
    for s in range(case["n_seq"]):
        table[s, :shared[s]] = table[lead[s], :shared[s]]
        table[s, shared[s]:per[s]] = at[k:k + per[s] - shared[s]]
        k += per[s] - shared[s]
        np.add.at(refs, table[s, :per[s]], 1)
    st.update(table=_i32(table), refs=_i32(refs))
    _pool_of(st, case, g, n_pages)


# ------------------------------------------------------------------------------------------------------- one pass

def run(st):
    kind = st["case"]["kind"]
    if own:
        return _OWN[kind](st)
    return _PLAIN[kind](st)


def _own_adapt(st):
    return st["plan"].apply(st["x"], st["a"], st["b"], base=st["base"], scale=st["scale"], dtype=TYPES[st["case"]["out"]])


def _own_sample(st):
    import paper_2510_25739_amd as H
    return H.sample_filtered(st["logits"], st["u"], temperature=st["temperature"], top_k=st["top_k"], top_p=st["top_p"], min_p=st["min_p"])


def _own_fork(st):
    # (images that an earlier pass left behind are given up: their rows of the table take the next ones)
    st["cache"].fork(st["refs"], st["n_past"], st["src"], st["dst"])
    short = st["cache"].take(st["refs"], st["n_past"], st["n_new"])
    return short, st["table"], st["refs"], st["n_past"], st["k_pool"], st["v_pool"]


def _own_compact(st):
    table, refs, used = st["cache"].compact(st["refs"])
    return table, refs, used, st["k_pool"], st["v_pool"]


_OWN = {"adapt": _own_adapt, "sample": _own_sample, "fork": _own_fork, "compact": _own_compact}


def _plain_adapt(st):
    # all adapters side by side: one product gives every row's A x of every adapter, of which its own is kept
    c = st["case"]
    n, rank = c["n_adapters"], c["rank"]
    seq = torch.searchsorted(st["row_start"], torch.arange(st["rows"], device=DEV), right=True) - 1
    mine = st["adapter"][seq]
    h = (st["x"].float() @ st["a"].float().view(n * rank, -1).t()).view(-1, n, rank)
    h = torch.where(mine[:, None, None] == torch.arange(n, device=DEV)[None, :, None], h, torch.zeros((), device=DEV))
    if st["scale"] is not None:
        h = h * st["scale"][None, :, None]
    y = h.view(-1, n * rank) @ st["b"].float().permute(0, 2, 1).reshape(n * rank, -1)
    if st["base"] is not None:
        y = y + st["base"].float()
    return y.to(TYPES[c["out"]])


def _plain_sample(st):
    n = st["logits"].shape[-1]
    at = torch.arange(n, device=DEV)
    greedy = (st["temperature"] <= 0)[:, None]
    z = st["logits"].float() * torch.where(greedy, torch.ones((), dtype=torch.float64, device=DEV), 1.0 / st["temperature"].double()[:, None]).float()
    ranked, index = torch.sort(z, dim=-1, descending=True, stable=True)
    w = torch.exp(ranked.double() - ranked[:, :1].double())
    k = torch.where(st["top_k"] < 1, n, st["top_k"].clamp(max=n))[:, None]
    keep = at < torch.where(greedy, 1, k)
    w = torch.where(keep, w, torch.zeros_like(w))
    sums = w.cumsum(-1)
    p = st["top_p"].double()[:, None]
    keep = keep & ((sums - w < p * sums[:, -1:]) | (p >= 1) | (at == 0)) & (w >= st["min_p"].double()[:, None])
    kept = torch.zeros_like(w).scatter_(-1, index, torch.where(keep, w, torch.zeros_like(w)))
    sums = kept.cumsum(-1)
    past = (sums > st["u"].double()[:, None] * sums[:, -1:]) & (kept > 0)
    first = torch.where(past, at, n).amin(-1)
    token = torch.where(first < n, first, torch.where(kept > 0, at, -1).amax(-1))
    return token.int(), (kept.gather(-1, token[:, None])[:, 0] / sums[:, -1]).float(), keep.sum(-1).int()


def _plain_fork(st):
    page, table, refs = st["case"]["page"], st["table"], st["refs"]
    src, dst = st["src"].long(), st["dst"].long()
    place = torch.arange(table.shape[1], device=DEV)

    def count(pages, where, by):
        refs.scatter_add_(0, torch.where(where, pages, 0).reshape(-1).long(), where.reshape(-1).int() * by)

    # what the images' rows held is given back, and the prompts' pages are theirs too
    held = table[dst]
    count(held, held >= 0, -1)
    given = torch.where(place < (st["n_past"][src][:, None] + page - 1) // page, table[src], -1)
    count(given, given >= 0, 1)
    table[dst] = given
    st["n_past"][dst] = st["n_past"][src]
    # the pages that are written next: those that are not there, and those that are somebody else's too
    past, new = st["n_past"][:, None], st["n_new"][:, None]
    write = (new > 0) & (place >= past // page) & (place < (past + new + page - 1) // page)
    shared = (table >= 0) & (refs[table.clamp(min=0).long()] > 1)
    lack = write & ((table < 0) | shared)
    free = torch.nonzero(refs == 0)[:, 0]
    wanted = lack.sum(-1)
    served = wanted.cumsum(0) <= free.numel()
    lack = lack & served[:, None]
    number = (lack.reshape(-1).cumsum(0) - 1).clamp(min=0).view(lack.shape)
    taken = torch.where(lack, free[number.clamp(max=max(free.numel() - 1, 0))].int() if free.numel() else table, table)
    # a page in whose middle a sequence goes on brings the entries before
    seq, at = torch.nonzero(lack & shared & (place == past // page) & (past % page > 0), as_tuple=True)
    if seq.numel():
        old, to = table[seq, at].long(), taken[seq, at].long()
        before = (torch.arange(page, device=DEV) < (st["n_past"][seq] % page)[:, None])[None, :, None, :, None]
        for pool in (st["k_pool"], st["v_pool"]):
            pool[:, to] = torch.where(before, pool[:, old], pool[:, to])
    count(table, lack & shared, -1)
    count(taken, lack, 1)
    table.copy_(taken)
    return torch.where(served, 0, wanted).int(), table, refs, st["n_past"], st["k_pool"], st["v_pool"]


def _plain_compact(st):
    refs, table = st["refs"], st["table"]
    page = torch.arange(refs.numel(), device=DEV)
    used = refs > 0
    n = used.sum()
    src, dst = torch.nonzero(used & (page >= n))[:, 0], torch.nonzero(~used & (page < n))[:, 0]
    for pool in (st["k_pool"], st["v_pool"]):
        pool[:, dst] = pool[:, src]
    to, new_refs = page.clone(), refs.clone()
    to[src] = dst
    new_refs[dst] = refs[src]
    new_refs[src] = 0
    there = (table >= 0) & used[table.clamp(min=0).long()]
    return torch.where(there, to[table.clamp(min=0).long()], -1).int(), new_refs, n.int().reshape(1), st["k_pool"], st["v_pool"]


_PLAIN = {"adapt": _plain_adapt, "sample": _plain_sample, "fork": _plain_fork, "compact": _plain_compact}


# ------------------------------------------------------------------------------------------------------- 64 bits

def exact(case, seed):
    st = prepare(case, seed)
    return {"adapt": _exact_adapt, "sample": _exact_sample, "fork": _exact_fork, "compact": _exact_compact}[case["kind"]](st)


def _exact_adapt(st):
    c = st["case"]
    y = st["base"].double() if st["base"] is not None else torch.zeros(st["rows"], c["d_out"], dtype=torch.float64, device=DEV)
    start, adapter = st["row_start"].tolist(), st["adapter"].tolist()
    for s, i in enumerate(adapter):
        if i < 0 or start[s] == start[s + 1]:
            continue
        rows = slice(start[s], start[s + 1])
        part = torch.mm(torch.mm(st["x"][rows].double(), st["a"][i].double().t().contiguous()), st["b"][i].double().t().contiguous())
        y[rows] += part * (float(st["scale"][i]) if st["scale"] is not None else 1.0)
    return y


def _exact_sample(st):
    logits = st["logits"].float().cpu().numpy()
    u, temp, top_k, top_p, min_p = (st[x].cpu().numpy() for x in ("u", "temperature", "top_k", "top_p", "min_p"))
    n = logits.shape[1]
    token, prob, kept = [], [], []
    for r in range(logits.shape[0]):
        if temp[r] <= 0:
            token.append(int(np.argmax(logits[r])))
            prob.append(1.0)
            kept.append(1)
            continue
        z = (logits[r] * (np.float32(1.0) / temp[r])).astype(np.float64)
        order = np.lexsort((np.arange(n), -z))
        if top_k[r] > 0:
            order = order[:top_k[r]]
        w = np.exp(z[order] - z[order[0]])
        m = order.size
        if top_p[r] < 1:
            m = max(1, int(np.searchsorted(np.concatenate([[0.0], np.cumsum(w)[:-1]]), float(top_p[r]) * w.sum(), side="left")))
        m = min(m, int((w >= float(min_p[r])).sum()))
        law = np.zeros(n)
        law[order[:m]] = w[:m]
        law /= law.sum()
        j = int(np.searchsorted(np.cumsum(law), float(u[r]), side="right"))
        j = j if j < n else int(np.flatnonzero(law)[-1])
        token.append(j)
        prob.append(law[j])
        kept.append(m)
    return torch.tensor(token, dtype=torch.int32), torch.tensor(prob, dtype=torch.float64), torch.tensor(kept, dtype=torch.int32)


MOST = 1 << 28      # values of a pool that are still compared in 64 bits


def _exact_fork(st):
    if st["k_pool"].numel() > MOST:
        return None
    page = st["case"]["page"]
    table, refs, past, new, src, dst = (st[x].tolist() for x in ("table", "refs", "n_past", "n_new", "src", "dst"))
    pools = [st["k_pool"].double(), st["v_pool"].double()]
    for a, b in zip(src, dst):
        table[b] = [p if i * page < past[a] else -1 for i, p in enumerate(table[a])]
        past[b] = past[a]
        for p in table[b]:
            if p >= 0:
                refs[p] += 1
    shared = [n > 1 for n in refs]
    free = [p for p, n in enumerate(refs) if n == 0]
    short, asked, room = [], 0, len(free)
    for s in range(len(table)):
        places = [i for i in range(past[s] // page, -(-(past[s] + new[s]) // page)) if table[s][i] < 0 or shared[table[s][i]]] if new[s] > 0 else []
        asked += len(places)
        short.append(len(places) if asked > room else 0)
        if short[-1]:
            continue
        for i in places:
            old, p = table[s][i], free.pop(0)
            n = past[s] - i * page
            if old >= 0:
                refs[old] -= 1
                if n > 0:
                    for pool in pools:
                        pool[:, p, :, :n] = pool[:, old, :, :n]
            refs[p] = 1
            table[s][i] = p
    return _i32(short), _i32(table), _i32(refs), _i32(past), pools[0], pools[1]


def _exact_compact(st):
    if st["k_pool"].numel() > MOST:
        return None
    table, refs = st["table"].tolist(), st["refs"].tolist()
    pools = [st["k_pool"].double(), st["v_pool"].double()]
    n = sum(1 for x in refs if x > 0)
    holes, to = [p for p in range(n) if refs[p] == 0], {}
    for p in range(n, len(refs)):
        if refs[p] > 0:
            q = to[p] = holes.pop(0)
            refs[q], refs[p] = refs[p], 0
            for pool in pools:
                pool[:, q] = pool[:, p]
    return _i32([[to.get(p, p) for p in row] for row in table]), _i32(refs), _i32([n]), pools[0], pools[1]


# ------------------------------------------------------------------------------------------------------- work

def work(case):
    kind = case["kind"]
    size = {"fp32": 4, "bf16": 2, "fp16": 2}
    if kind == "adapt":
        # rows in and out (and what they are added to), and the adapters that are in use: as many as there can be
        n = case["n_seq"]
        rows = int(_rows_of(case).sum())
        share = 1.0 - (-(-n // case["without"]) / n if case["without"] and n > 1 else 0.0)
        used = case["n_adapters"] * (1.0 - (1.0 - 1.0 / case["n_adapters"]) ** max(1.0, n * share))
        x, out = size[case["x"]], size[case["out"]]
        return {"bytes": int(rows * (case["d_in"] * x * share + case["d_out"] * out * (1 + case["base"])) + used * case["rank"] * (case["d_in"] + case["d_out"]) * x),
                "flops": int(2 * rows * share * case["rank"] * (case["d_in"] + case["d_out"]))}
    if kind == "sample":
        # the logits once, an exponential and a sum an entry
        return {"bytes": case["rows"] * case["n"] * size[case["x"]], "flops": case["rows"] * case["n"] * 4}
    entry = case["layers"] * 2 * case["kv_heads"] * case["head_dim"] * size[case["cache"]]
    if kind == "compact":
        return {"bytes": int(2 * min(case["moves"], _used_pages(case)[3]) * case["page"] * entry + 64), "flops": 0}
    # the entries of the pages in whose middle the images go on, read and written, and the tables
    r = _own_numbers(case)
    past = _between(r, case["past_lo"], case["past_hi"], case["prompts"])
    n = case["prompts"] * case["images"]
    new = _between(r, case["new_lo"], case["new_hi"], n)
    inside = (past % case["page"])[np.arange(n) % case["prompts"]] * (new > 0)
    return {"bytes": int(2 * inside.sum() * entry + 16 * n * -(-case["past_hi"] // case["page"])), "flops": 0}
