"""The operators over a paged cache, and the verification of drafted chains, as cases that can be timed and compared.

A step of a target model that serves many sequences from one pool of pages: the rows of the step - the last committed
token of each sequence and what was drafted behind it, or a piece of a prompt - get their queries and keys normalised and
rotated and their keys and values appended to the pages (`append`); their attention reads the pages (`attend`: causal
inside the step, or along a candidate tree); the drafts are verified against the target's rows (`verify`); after a tree
step the accepted path's entries are moved to their positions (`keep`).

Shapes are those of `synth.CONFIGS` (20 heads of 64; 32 heads of 128; slices of 16384 and 65536 entries; grids of 24 x 24
with 120 condition rows) and generic ones with shared key and value heads.  Where `own` is false `run` computes in
elementary torch operations, in 32 bits, the verification in 64 (its decisions are comparisons of neighbouring sums).
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda:0"
TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}


def listed():
    return [
        # One sequence, one token, the exact-parity type: all latency.
        dict(name="append-one", kind="append", n_seq=1, rows_lo=1, rows_hi=1, past_lo=300, past_hi=300, heads=4, kv_heads=4,
             head_dim=64, page=16, x="fp32", cache="fp32", norm=False, rot=64, halves=False),
        # Pieces of two prompts, queries and keys normalised per head, shared key and value heads.
        dict(name="append-prompt", kind="append", n_seq=2, rows_lo=2000, rows_hi=2048, past_lo=0, past_hi=2000, heads=32,
             kv_heads=8, head_dim=128, page=64, x="bf16", cache="bf16", norm=True, rot=128, halves=True),
        # One sequence in the middle of its image, one token.
        dict(name="attend-one", kind="attend", n_seq=1, rows_lo=1, rows_hi=1, past_lo=408, past_hi=408, heads=20, kv_heads=20,
             head_dim=64, page=16, cache="fp16", tree=False),
        # 16 sequences at different places of their images, each the last token and five drafts.
        dict(name="attend-step", kind="attend", n_seq=16, rows_lo=6, rows_hi=6, past_lo=120, past_hi=690, heads=20, kv_heads=20,
             head_dim=64, page=16, cache="fp16", tree=False),
        # Candidate trees (up to 13 nodes) over the large model's heads.
        dict(name="attend-tree", kind="attend", n_seq=8, rows_lo=7, rows_hi=13, past_lo=64, past_hi=1080, heads=32, kv_heads=32,
             head_dim=128, page=32, cache="bf16", tree=True),
        # Single tokens behind long histories, shared key and value heads.
        dict(name="attend-long", kind="attend", n_seq=4, rows_lo=1, rows_hi=1, past_lo=70001, past_hi=100000, heads=32, kv_heads=8,
             head_dim=128, page=64, cache="bf16", tree=False),
        # A piece of a prompt behind an earlier one: the contraction.
        dict(name="attend-prompt", kind="attend", n_seq=1, rows_lo=4001, rows_hi=4001, past_lo=2048, past_hi=2048, heads=32,
             kv_heads=8, head_dim=128, page=64, cache="bf16", tree=False),
        # The exact-parity type, ragged pieces.
        dict(name="attend-fp32", kind="attend", n_seq=3, rows_lo=1, rows_hi=65, past_lo=0, past_hi=500, heads=12, kv_heads=4,
             head_dim=64, page=24, cache="fp32", tree=False),
        # The accepted paths of one tree step, all layers: one sequence of the small model, and a batch of the large one.
        dict(name="keep-one", kind="keep", n_seq=1, layers=12, kv_heads=12, head_dim=64, page=16, cache="fp16", past_lo=200,
             past_hi=300, depth=2),
        dict(name="keep-batch", kind="keep", n_seq=16, layers=32, kv_heads=32, head_dim=128, page=32, cache="bf16", past_lo=64,
             past_hi=500, depth=4),
        # One sequence's five drafts over the image codes, and a batch's over a whole vocabulary.
        dict(name="verify-one", kind="verify", n_seq=1, k=5, n=16384, temperature=1.0, top_k=1000, ragged=False, proposals=True),
        dict(name="verify-batch", kind="verify", n_seq=48, k=4, n=65536, temperature=0.9, top_k=65536, ragged=True,
             proposals=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["append", "attend", "attend", "attend", "keep", "verify"])
    heads, kv_heads, head_dim = rng.choice([(20, 20, 64), (32, 32, 128), (32, 8, 128), (12, 4, 64), (16, 2, 128), (8, 1, 256),
                                            (12, 12, 32), (9, 3, 96), (6, 6, 80)])
    page = rng.choice([8, 16, 24, 32, 64, 128])
    cache = rng.choice(["fp32", "bf16", "bf16", "fp16", "fp16"])
    if kind == "append":
        n_seq = _log(rng, 1, 64)
        hi = _log(rng, 1, max(1, 4000 // n_seq))
        past = rng.randint(0, 1500)
        return dict(kind=kind, n_seq=n_seq, rows_lo=rng.randint(0 if n_seq > 1 else 1, hi), rows_hi=hi, past_lo=rng.randint(0, past), past_hi=past,
                    heads=heads, kv_heads=kv_heads, head_dim=head_dim, page=page, x=rng.choice(["fp32", "bf16", "fp16"]),
                    cache=cache, norm=rng.random() < 0.5, rot=rng.choice([0, head_dim, head_dim, head_dim // 2]),
                    halves=rng.random() < 0.5)
    if kind == "keep":
        return dict(kind=kind, n_seq=_log(rng, 1, 16), layers=_log(rng, 1, 32), kv_heads=kv_heads, head_dim=head_dim, page=page,
                    cache=cache, past_lo=0, past_hi=rng.randint(10, 400), depth=rng.randint(1, 6))
    if kind == "verify":
        n = rng.choice([8192, 16384, 65536, _log(rng, 500, 65536)])
        top_k = rng.choice([n, 1000, 2000, _log(rng, 20, 4000)])
        return dict(kind=kind, n_seq=_log(rng, 1, 48), k=rng.randint(1, 4), n=n, temperature=rng.choice([0.0, 0.7, 1.0, 1.0]),
                    top_k=min(top_k, n), ragged=rng.random() < 0.5, proposals=rng.random() < 0.8)
    form = rng.choice(["one", "step", "step", "tree", "long", "piece"])
    c = dict(kind=kind, heads=heads, kv_heads=kv_heads, head_dim=head_dim, page=page, cache=cache, tree=form == "tree")
    if form == "one":
        past = _log(rng, 1, 4000)
        return dict(c, n_seq=_log(rng, 1, 32), rows_lo=1, rows_hi=1, past_lo=rng.randint(0, past), past_hi=past)
    if form == "step":
        past, rows = _log(rng, 20, 3000), rng.randint(2, 9)
        return dict(c, n_seq=_log(rng, 1, 32), rows_lo=rng.randint(0, rows), rows_hi=rows, past_lo=rng.randint(0, past), past_hi=past)
    if form == "tree":
        past, rows = _log(rng, 20, 1500), rng.randint(4, 40)
        return dict(c, n_seq=_log(rng, 1, 8), rows_lo=rng.randint(1, rows), rows_hi=rows, past_lo=rng.randint(0, past), past_hi=past)
    if form == "long":
        past = _log(rng, 8000, 50000)
        return dict(c, n_seq=rng.randint(1, 3), rows_lo=1, rows_hi=rng.randint(1, 6), past_lo=past // 2, past_hi=past)
    hi = _log(rng, 30, 1200)
    past = rng.choice([0, rng.randint(1, 1500)])
    return dict(c, n_seq=rng.randint(1, 3), rows_lo=rng.randint(1, hi), rows_hi=hi, past_lo=past // 2, past_hi=past)


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
    return torch.tensor(a, dtype=torch.int32, device=DEV)


def _lengths(case):
    """Rows and committed entries of every sequence: the case's upper bounds among them, the rest between.  They are the
    case's own, so that inputs of another seed have the same shapes."""
    r = np.random.RandomState(sum((i + 1) * v for i, v in enumerate(v for v in case.values() if type(v) is int)))
    n = case["n_seq"]
    rows = r.randint(case["rows_lo"], case["rows_hi"] + 1, n) if "rows_lo" in case else np.ones(n, int)
    past = r.randint(case["past_lo"], case["past_hi"] + 1, n)
    if "rows_hi" in case:
        rows[r.randint(n)] = case["rows_hi"]
    past[r.randint(n)] = case["past_hi"]
    return [int(x) for x in rows], [int(x) for x in past]


def _pages(case, seed, need):
    """A table of pages scattered over a pool with some to spare."""
    r = np.random.RandomState((seed * 104729 + 7) % (1 << 31))
    per = [-(-n // case["page"]) for n in need]
    cols = max(1, max(per))
    total = sum(per) + 3
    order = r.permutation(total)
    table = np.zeros((case["n_seq"], cols), dtype=np.int32)
    at = 0
    for s, n in enumerate(per):
        table[s, :n] = order[at:at + n]
        at += n
    return total, torch.from_numpy(table).to(DEV)


def _pool(g, *shape, dtype):
    """Keys or values of a pool, drawn in pieces: a long history's pool in 32 bits would be twice its size."""
    out = torch.empty(*shape, dtype=dtype, device=DEV)
    flat = out.view(-1)
    step = 1 << 27
    for i in range(0, flat.numel(), step):
        m = min(step, flat.numel() - i)
        flat[i:i + m] = torch.randn(m, generator=g, device=DEV).to(dtype)
    return out


def _trees(rows, seed):
    """A random tree a sequence: every node's ancestors and itself as bits, parents before children."""
    r = np.random.RandomState((seed * 31 + 5) % (1 << 31))
    out = []
    for n in rows:
        mask = []
        for i in range(n):
            mask.append((mask[r.randint(max(0, i - 4), i)] if i else 0) | (1 << i))
        out += mask
    return torch.from_numpy(np.array(out, dtype=np.uint64).view(np.int64)).to(DEV)


def _rope(n_pos, rot, theta=10000.0):
    """cos and sin of position * theta^(-2 j / rot), [position][j][2]; the angles in 64 bits."""
    j = torch.arange(rot // 2, dtype=torch.float64, device=DEV)
    a = torch.arange(n_pos, dtype=torch.float64, device=DEV)[:, None] * theta ** (-2.0 * j / rot)
    return torch.stack([a.cos(), a.sin()], dim=-1).float().contiguous()


def prepare(case, seed):
    g = _gen(seed)
    st = dict(case=dict(case))
    kind = case["kind"]
    if kind == "verify":
        n_seq, k, n = case["n_seq"], case["k"], case["n"]
        # proposals of a draft model that knows the target roughly, and the drafts drawn from them
        p = _randn(g, n_seq, k + 1, n) * 2.0
        q = p[:, :k] + 0.5 * _randn(g, n_seq, k, n)
        t = case["temperature"] if case["temperature"] > 0 else 1e-3
        kept = torch.topk(q / t, min(case["top_k"], n), dim=-1)
        noise = -torch.log(-torch.log(_uniform(g, *kept.values.shape).clamp(1e-7, 1 - 1e-7)))
        draft = kept.indices.gather(-1, (kept.values + noise).argmax(-1, keepdim=True))[..., 0]
        st.update(p=p.reshape(n_seq * (k + 1), n).contiguous(), q=q.contiguous() if case["proposals"] else None, draft=draft.int().contiguous(),
                  u_acc=_uniform(g, n_seq, k), u_final=_uniform(g, n_seq),
                  n_draft=torch.randint(0, k + 1, (n_seq,), generator=g, device=DEV).int() if case["ragged"] else None)
        del p, q, kept, noise
    else:
        dt = TYPES[case["cache"]]
        rows, past = _lengths(case)
        hk, hd, page = case["kv_heads"], case["head_dim"], case["page"]
        if kind == "keep":
            # a tree deep and wide enough: an accepted path's nodes lie behind the entries that are kept, so that a second
            # pass moves the same keys and values again
            depth = case["depth"]
            r = np.random.RandomState((seed * 17 + 3) % (1 << 31))
            path = np.sort(depth + 1 + np.stack([r.choice(20, depth, replace=False) for _ in rows]), axis=1)
            keep = r.randint(0, depth + 1, len(rows))
            keep[0] = depth
            n_pages, table = _pages(case, seed, [p + depth + 22 for p in past])
            shape = (case["layers"], n_pages, hk, page, hd)
            st.update(path=_i32(path.tolist()), n_keep=_i32(keep.tolist()))
        else:
            n_pages, table = _pages(case, seed, [p + n for p, n in zip(past, rows)])
            shape = (1, n_pages, hk, page, hd)
            start = [0]
            for n in rows:
                start.append(start[-1] + n)
            st.update(rows=rows, past=past, total=start[-1], row_start=_i32(start), max_len=max(p + n for p, n in zip(past, rows)))
        st.update(k_pool=_pool(g, *shape, dtype=dt), v_pool=_pool(g, *shape, dtype=dt), table=table, n_past=_i32(past))
        if kind == "append":
            x = TYPES[case["x"]]
            # the columns of one projection, as a model's product leaves them
            qkv = _randn(g, st["total"], case["heads"] + 2 * hk, hd, dtype=x)
            st.update(q=qkv[:, :case["heads"]], k=qkv[:, case["heads"]:case["heads"] + hk], v=qkv[:, case["heads"] + hk:],
                      rot=_rope(st["max_len"], case["rot"]) if case["rot"] else None,
                      q_gain=1.0 + 0.2 * _randn(g, hd) if case["norm"] else None,
                      k_gain=1.0 + 0.2 * _randn(g, hd) if case["norm"] else None)
        if kind == "attend":
            st.update(q=_randn(g, st["total"], case["heads"], hd, dtype=dt), tree=_trees(rows, seed) if case["tree"] else None)
    if own:
        import paper_2510_25739_amd as H
        if kind != "verify":
            st["cache"] = H.PagedCache(st["k_pool"], st["v_pool"], st["table"])
    return st


# ------------------------------------------------------------------------------------------------------- one pass

def run(st):
    kind = st["case"]["kind"]
    if own:
        return _OWN[kind](st)
    return _PLAIN[kind](st)


def _own_append(st):
    c = st["case"]
    q = st["cache"].append(st["k"], st["v"], st["row_start"], st["n_past"], q=st["q"], rot=st["rot"], halves=c["halves"],
                           q_gain=st["q_gain"], k_gain=st["k_gain"], eps=1e-5)
    return q, st["k_pool"], st["v_pool"]


def _own_attend(st):
    return st["cache"].attend(st["q"], st["row_start"], st["n_past"], max_len=st["max_len"], tree=st["tree"])


def _own_keep(st):
    st["cache"].keep(st["n_past"], st["path"], st["n_keep"])
    return st["k_pool"], st["v_pool"]


def _own_verify(st):
    import paper_2510_25739_amd as H
    c = st["case"]
    return H.verify_chains(st["p"], st["q"], st["draft"], st["u_acc"], st["u_final"], c["temperature"], c["top_k"],
                           n_draft=st["n_draft"])


_OWN = {"append": _own_append, "attend": _own_attend, "keep": _own_keep, "verify": _own_verify}


def _normed(x, gain):
    x = x.float()
    if gain is None:
        return x
    return x * torch.rsqrt((x * x).mean(-1, keepdim=True) + 1e-5) * gain


def _rotated(x, cs, rot, halves):
    """x [rows, heads, head_dim], cs [rows, rot / 2, 2]"""
    if rot == 0:
        return x
    c, s = cs[:, None, :, 0], cs[:, None, :, 1]
    a, b = (x[..., :rot // 2], x[..., rot // 2:rot]) if halves else (x[..., 0:rot:2], x[..., 1:rot:2])
    y = [a * c - b * s, a * s + b * c]
    y = torch.cat(y, -1) if halves else torch.stack(y, -1).flatten(-2)
    return torch.cat([y, x[..., rot:]], -1)


def _plain_append(st):
    c, table, page = st["case"], st["table"], st["case"]["page"]
    at = torch.arange(st["total"], device=DEV)
    seq = torch.searchsorted(st["row_start"], at, right=True) - 1
    pos = (st["n_past"][seq] + at - st["row_start"][seq]).long()
    cs = st["rot"][pos] if c["rot"] else None
    dt = st["k_pool"].dtype
    q = _rotated(_normed(st["q"], st["q_gain"]), cs, c["rot"], c["halves"]).to(dt)
    k = _rotated(_normed(st["k"], st["k_gain"]), cs, c["rot"], c["halves"]).to(dt)
    pg = table[seq, pos // page].long()
    st["k_pool"][0][pg, :, pos % page] = k
    st["v_pool"][0][pg, :, pos % page] = st["v"].to(dt)
    return q, st["k_pool"], st["v_pool"]


def _plain_attend(st):
    # every sequence padded to the longest one's rows and to the table's width
    c = st["case"]
    hk, hd, group, n_seq, most = c["kv_heads"], c["head_dim"], c["heads"] // c["kv_heads"], c["n_seq"], max(st["rows"])
    at = torch.arange(st["total"], device=DEV)
    seq = torch.searchsorted(st["row_start"], at, right=True) - 1
    i = at - st["row_start"][seq]
    q = torch.zeros(n_seq, most, hk, group, hd, device=DEV)
    q[seq, i] = st["q"].float().view(-1, hk, group, hd)
    q = q.permute(0, 2, 3, 1, 4).reshape(n_seq, hk, group * most, hd)
    pages = st["table"].long()
    k = st["k_pool"][0][pages].float().permute(0, 2, 4, 1, 3).reshape(n_seq, hk, hd, -1)      # [sequence, head, feature, entry]
    z = (q @ k).view(n_seq, hk, group, most, -1) * (1.0 / math.sqrt(hd))
    del k
    j = torch.arange(z.shape[-1], device=DEV)
    past = st["n_past"][:, None, None]
    if st["tree"] is None:
        see = j <= past + torch.arange(most, device=DEV)[None, :, None]
    else:
        bits = torch.zeros(n_seq, most, dtype=torch.int64, device=DEV)
        bits[seq, i] = st["tree"]
        see = (j < past) | ((j < past + 64) & (((bits[..., None] >> (j - past).clamp(0, 63)) & 1) == 1))
    z = z.masked_fill_(~see[:, None, None], float("-inf"))
    m = z.amax(-1, keepdim=True)
    w = torch.exp_(z.sub_(torch.where(m == float("-inf"), torch.zeros_like(m), m)))
    total = w.sum(-1, keepdim=True)
    # entries behind a sequence's last one may hold anything: they are taken as zero, not weighted with it
    used = j[None, :] < st["n_past"][:, None] + (st["row_start"][1:] - st["row_start"][:-1])[:, None]
    v = st["v_pool"][0][pages].float().permute(0, 2, 1, 3, 4).reshape(n_seq, hk, -1, hd)
    v = torch.where(used[:, None, :, None], v, torch.zeros((), device=DEV))
    y = (w.view(n_seq, hk, group * most, -1) @ v).view(n_seq, hk, group, most, hd)
    y = y / torch.where(total > 0, total, torch.ones_like(total))
    return y.permute(0, 3, 1, 2, 4)[seq, i].reshape(st["q"].shape).to(st["q"].dtype)


def _plain_keep(st):
    page, depth = st["case"]["page"], st["case"]["depth"]
    step = torch.arange(1, depth + 1, device=DEV)[None, :]
    node = torch.where(step <= st["n_keep"][:, None], st["path"].long(), step)   # what is not kept stays where it is
    seq = torch.arange(st["table"].shape[0], device=DEV)[:, None].expand_as(node)
    src, dst = st["n_past"][:, None] + node, st["n_past"][:, None] + step
    ps, pd = st["table"][seq, src // page].long(), st["table"][seq, dst // page].long()
    st["k_pool"][:, pd, :, dst % page] = st["k_pool"][:, ps, :, src % page]
    st["v_pool"][:, pd, :, dst % page] = st["v_pool"][:, ps, :, src % page]
    return st["k_pool"], st["v_pool"]


def _warped(logits, temperature, top_k):
    """Probabilities of the last axis in 64 bits: temperature, the top_k largest (equal ones: lower index first)."""
    n = logits.shape[-1]
    if temperature == 0.0 or top_k == 1:
        top = logits.amax(-1, keepdim=True)
        first = torch.where(logits == top, torch.arange(n, device=DEV), n).amin(-1, keepdim=True)
        return (torch.arange(n, device=DEV) == first).double()
    z = logits * torch.tensor(1.0 / np.float32(temperature), dtype=torch.float32, device=DEV)
    w = torch.exp(z.double() - z.amax(-1, keepdim=True).double())
    if top_k < n:
        kept = torch.sort(z, dim=-1, descending=True, stable=True).indices[..., :top_k]
        w = w * torch.zeros_like(w).scatter_(-1, kept, 1.0)
    return w / w.sum(-1, keepdim=True)


def _plain_verify(st):
    c = st["case"]
    n_seq, k, n = c["n_seq"], c["k"], c["n"]
    drafts = st["n_draft"].long() if st["n_draft"] is not None else torch.full((n_seq,), k, device=DEV)
    draft = st["draft"].long()
    p = _warped(st["p"].view(n_seq, k + 1, n), c["temperature"], c["top_k"])
    if st["q"] is not None:
        q = _warped(st["q"], c["temperature"], c["top_k"])
    else:
        q = torch.zeros(n_seq, k, n, dtype=torch.float64, device=DEV).scatter_(-1, draft[..., None], 1.0)
    pd, qd = p[:, :k].gather(-1, draft[..., None])[..., 0], q.gather(-1, draft[..., None])[..., 0]
    ok = (st["u_acc"].double() * qd < pd) & (torch.arange(k, device=DEV) < drafts[:, None])
    a = ok.long().cumprod(-1).sum(-1)
    seq = torch.arange(n_seq, device=DEV)
    left = p[seq, a]
    over = (left - q[seq, a.clamp(max=k - 1)]).clamp(min=0.0)
    use = (a < drafts)[:, None] & (over.sum(-1, keepdim=True) > 0)
    left = torch.where(use, over, left)
    run_sum = left.cumsum(-1)
    past = run_sum > st["u_final"].double()[:, None] * left.sum(-1, keepdim=True)
    at = torch.arange(n, device=DEV)
    first = torch.where(past & (left > 0), at, n).amin(-1)
    last = torch.where(left > 0, at, -1).amax(-1)
    tok = torch.where(first < n, first, last)
    step = torch.arange(k + 1, device=DEV)[None, :]
    padded = torch.cat([draft, torch.zeros_like(draft[:, :1])], -1)
    out = torch.where(step < a[:, None], padded, torch.where(step == a[:, None], tok[:, None], -1))
    return a.int(), out.int()


_PLAIN = {"append": _plain_append, "attend": _plain_attend, "keep": _plain_keep, "verify": _plain_verify}


# ------------------------------------------------------------------------------------------------------- 64 bits

def exact(case, seed):
    st = prepare(case, seed)
    return {"append": _exact_append, "attend": _exact_attend, "keep": _exact_keep, "verify": _exact_verify}[case["kind"]](st)


def _entry(st, s, e):
    """Page and place of entry e of sequence s, on the host."""
    if "table_host" not in st:
        st["table_host"] = st["table"].cpu().numpy()
    return int(st["table_host"][s, e // st["case"]["page"]]), e % st["case"]["page"]


def _exact_append(st):
    c = st["case"]
    k_all, v_all = st["k_pool"].double(), st["v_pool"].double()
    q_all = torch.zeros(st["q"].shape, dtype=torch.float64, device=DEV)
    rot, half = c["rot"], c["rot"] // 2
    first = torch.arange(half, device=DEV) if c["halves"] else 2 * torch.arange(half, device=DEV)
    second = first + (half if c["halves"] else 1)

    def turned(x, gain, where):
        y = x.double()
        if gain is not None:
            y = y / (y.pow(2).sum(-1, keepdim=True) / c["head_dim"] + 1e-5).sqrt() * gain.double()
        if rot:
            z = torch.complex(y[..., first], y[..., second]) * torch.view_as_complex(st["rot"][where].double().contiguous())[:, None]
            y = y.clone()
            y[..., first], y[..., second] = z.real, z.imag
        return y

    r0 = 0
    for s, (n, past) in enumerate(zip(st["rows"], st["past"])):
        if n == 0:
            continue
        where = torch.arange(past, past + n, device=DEV)
        q_all[r0:r0 + n] = turned(st["q"][r0:r0 + n], st["q_gain"], where)
        k = turned(st["k"][r0:r0 + n], st["k_gain"], where)
        at = np.array([_entry(st, s, past + i) for i in range(n)])
        pg, slot = torch.from_numpy(at[:, 0]).to(DEV), torch.from_numpy(at[:, 1]).to(DEV)
        k_all[0, pg, :, slot] = k
        v_all[0, pg, :, slot] = st["v"][r0:r0 + n].double()
        r0 += n
    return q_all, k_all, v_all


def _exact_attend(st):
    c = st["case"]
    hd, group, page = c["head_dim"], c["heads"] // c["kv_heads"], c["page"]
    out = torch.zeros(st["q"].shape, dtype=torch.float64, device=DEV)
    trees = st["tree"].cpu().numpy().view(np.uint64) if st["tree"] is not None else None
    r0 = 0
    for s, (n, past) in enumerate(zip(st["rows"], st["past"])):
        if n == 0:
            continue
        length = past + n
        bias = torch.zeros(n, length, dtype=torch.float64, device=DEV)
        if trees is None:
            bias += torch.full_like(bias, float("-inf")).triu(past + 1)
        else:
            hidden = np.zeros((n, n), dtype=bool)
            for i in range(n):
                for j in range(n):
                    hidden[i, j] = not (int(trees[r0 + i]) >> j) & 1
            bias[:, past:][torch.from_numpy(hidden).to(DEV)] = float("-inf")
        pages = st["table"][s, :-(-length // page)].long()
        for h in range(c["heads"]):
            k = st["k_pool"][0, pages, h // group].flatten(0, 1)[:length].double()
            v = st["v_pool"][0, pages, h // group].flatten(0, 1)[:length].double()
            z = torch.matmul(st["q"][r0:r0 + n, h].double(), k.t().contiguous()) / math.sqrt(hd) + bias
            out[r0:r0 + n, h] = torch.matmul(torch.softmax(z, -1), v)
        r0 += n
    return out


def _exact_keep(st):
    k, v = st["k_pool"].double(), st["v_pool"].double()
    path, keep, past = (st[x].cpu().numpy() for x in ("path", "n_keep", "n_past"))
    for s in range(len(keep)):
        for j in range(int(keep[s])):
            (ps, es), (pd, ed) = _entry(st, s, int(past[s] + path[s, j])), _entry(st, s, int(past[s]) + j + 1)
            for pool in (k, v):
                pool[:, pd, :, ed] = pool[:, ps, :, es]
    return k, v


def _host_probs(row, temperature, top_k):
    row = row.astype(np.float32)
    if temperature == 0.0 or top_k == 1:
        w = np.zeros(row.size)
        w[int(row.argmax())] = 1.0
        return w
    z = row * np.float32(np.float32(1.0) / np.float32(temperature))
    w = np.exp(z.astype(np.float64) - float(z.max()))
    if top_k < row.size:
        keep = np.lexsort((np.arange(row.size), -z))[:top_k]
        mask = np.zeros(row.size)
        mask[keep] = 1.0
        w = w * mask
    return w / w.sum()


def _exact_verify(st):
    c = st["case"]
    n_seq, k, n, t, top = c["n_seq"], c["k"], c["n"], c["temperature"], c["top_k"]
    p_rows, draft, ua, uf = (st[x].cpu().numpy() for x in ("p", "draft", "u_acc", "u_final"))
    q_rows = st["q"].cpu().numpy() if st["q"] is not None else None
    drafts = st["n_draft"].cpu().numpy() if st["n_draft"] is not None else np.full(n_seq, k)
    count, toks = np.zeros(n_seq, np.int32), np.full((n_seq, k + 1), -1, np.int32)
    for s in range(n_seq):
        law = None
        a = 0
        while a < int(drafts[s]):
            d = int(draft[s, a])
            p = _host_probs(p_rows[s * (k + 1) + a], t, top)
            if q_rows is not None:
                q = _host_probs(q_rows[s, a], t, top)
            else:
                q = np.zeros(n)
                q[d] = 1.0
            if float(ua[s, a]) * q[d] < p[d]:
                toks[s, a] = d
                a += 1
                continue
            rest = np.maximum(p - q, 0.0)
            law = rest if rest.sum() > 0 else p
            break
        if law is None:
            law = _host_probs(p_rows[s * (k + 1) + a], t, top)
        sums = np.cumsum(law)
        j = int(np.searchsorted(sums, float(uf[s]) * law.sum(), side="right"))
        toks[s, a] = j if j < n else int(np.flatnonzero(law > 0)[-1])
        count[s] = a
    return torch.from_numpy(count), torch.from_numpy(toks)


# ------------------------------------------------------------------------------------------------------- work

def work(case):
    kind = case["kind"]
    if kind == "verify":
        # the drafted rows of the target and of the proposals once, an exponential and a sum an entry
        k = case["k"] / 2 if case["ragged"] else case["k"]
        rows = int(case["n_seq"] * (2 * k + 1 if case["proposals"] else k + 1))
        return {"bytes": rows * case["n"] * 4, "flops": rows * case["n"] * 4}
    size = 4 if case["cache"] == "fp32" else 2
    hk, hd = case["kv_heads"], case["head_dim"]
    if kind == "keep":
        mean = case["n_seq"] * (case["depth"] + 1) / 2
        return {"bytes": int(mean * case["layers"] * 2 * hk * hd * size * 2), "flops": 0}
    rows = case["n_seq"] * (case["rows_lo"] + case["rows_hi"]) / 2
    past = (case["past_lo"] + case["past_hi"]) / 2
    each = rows / case["n_seq"]
    if kind == "append":
        x = 4 if case["x"] == "fp32" else 2
        heads = case["heads"] + 2 * hk
        return {"bytes": int(rows * (heads * hd * (x + size) + case["rot"] * 4)),
                "flops": int(rows * (case["heads"] + hk) * hd * (3 * bool(case["rot"]) + 4 * case["norm"]))}
    seen = past + each if case["tree"] else past + (each + 1) / 2
    return {"bytes": int(2 * rows * case["heads"] * hd * size + case["n_seq"] * (past + each) * 2 * hk * hd * size),
            "flops": int(4 * rows * case["heads"] * hd * seen)}
