"""The calls over a paged cache as they are used together: a small decoder that serves ragged sequences from one pool -
prompts in one ragged pass, chains drafted and verified, a tree step whose accepted path is moved into place -, against the
same decoder run densely in float64 on every sequence alone; and the same step captured into a graph and on a stream of its own."""
import numpy as np
import pytest

from test_gpu_chains import chain, compare, dev
from test_gpu_paged import DEV, attention_reference, check_attention, Setup, weight_step

pytestmark = pytest.mark.gpu

LAYERS, HEADS, KV, HD, VOCAB, PAGE = 2, 4, 2, 64, 300, 6
D = HEADS * HD


@pytest.fixture(scope="module")
def H():
    import torch
    import paper_2510_25739_amd as H
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    return H


class Decoder:
    def __init__(self, seed):
        import torch
        g = torch.Generator().manual_seed(seed)
        r = lambda *s, std=1.0: torch.randn(*s, generator=g) * std
        self.E = r(VOCAB, D)
        self.qkv = [r(D, (HEADS + 2 * KV) * HD, std=D ** -0.5) for _ in range(LAYERS)]
        self.o = [r(D, D, std=D ** -0.5) for _ in range(LAYERS)]
        self.gain = 1 + 0.2 * r(2, HD)
        self.W = r(D, VOCAB, std=2 * D ** -0.5)

    def paged(self, H, cache, rot, tokens, row_start, n_past, tree=None, pos=None):
        x = self.E.to(DEV)[tokens.long()]
        gain = self.gain.to(DEV)
        for l in range(LAYERS):
            h = (x @ self.qkv[l].to(DEV)).view(-1, HEADS + 2 * KV, HD)
            q = cache.append(h[:, HEADS:HEADS + KV], h[:, HEADS + KV:], row_start, n_past, q=h[:, :HEADS], rot=rot, halves=True, pos=pos,
                             q_gain=gain[0].contiguous(), k_gain=gain[1].contiguous(), layer=l)
            x = x + cache.attend(q, row_start, n_past, tree=tree, layer=l).view(-1, D) @ self.o[l].to(DEV)
        return (x @ self.W.to(DEV)).contiguous()

    def dense(self, tokens):
        """Logits of every position of one sequence, float64."""
        import torch
        x = self.E.double()[torch.tensor(tokens)]
        n = len(tokens)
        j = torch.arange(HD // 2, dtype=torch.float64)
        a = torch.arange(n, dtype=torch.float64)[:, None] * 10000.0 ** (-2 * j / HD)
        c, s = a.cos()[:, None], a.sin()[:, None]

        def turned(v, gain):
            v = v / torch.sqrt((v * v).mean(-1, keepdim=True) + 1e-5) * gain.double()
            u, w = v[..., :HD // 2], v[..., HD // 2:]
            return torch.cat([u * c - w * s, u * s + w * c], -1)

        for l in range(LAYERS):
            h = (x @ self.qkv[l].double()).view(n, HEADS + 2 * KV, HD)
            q, k, v = turned(h[:, :HEADS], self.gain[0]), turned(h[:, HEADS:HEADS + KV], self.gain[1]), h[:, HEADS + KV:]
            k, v = (t.repeat_interleave(HEADS // KV, 1).transpose(0, 1) for t in (k, v))
            z = q.transpose(0, 1) @ k.transpose(1, 2) / HD ** 0.5 + torch.full((n, n), float("-inf"), dtype=torch.float64).triu(1)
            x = x + (torch.softmax(z, -1) @ v).transpose(0, 1).reshape(n, D) @ self.o[l].double()
        return x @ self.W.double()


# fp32 products of 256 and 300 terms and an fp32 table through two layers: each is off by about 256 * 2^-24 = 1.5e-5 of its
# terms' absolute sum, itself some ten times the result; four such products in a row
LOGIT_TOL = 1e-3


def close(got, want):
    err = float((got.double().cpu() - want).abs().max()) / float(want.abs().max())
    print(f"largest logit error {err:.1e} of the largest logit")
    assert err < LOGIT_TOL


def test_prompts_chains_and_a_tree(H):
    import torch
    rng = np.random.RandomState(1)
    m = Decoder(0)
    prompts = [list(rng.randint(0, VOCAB, n)) for n in (7, 1, 25)]
    n_seq, cols, k = 3, 12, 3
    pool = torch.full((2, LAYERS, n_seq * cols + 5, KV, PAGE, HD), float("nan"), device=DEV)
    table = torch.from_numpy(rng.permutation(n_seq * cols + 5)[:n_seq * cols].reshape(n_seq, cols).astype(np.int32)).to(DEV)
    cache = H.PagedCache(pool[0], pool[1], table)
    rot = H.rotary_table(cols * PAGE, HD)
    i32 = lambda a: torch.tensor(a, dtype=torch.int32, device=DEV)

    start = np.concatenate([[0], np.cumsum([len(p) for p in prompts])])
    lg = m.paged(H, cache, rot, i32(sum(prompts, [])), i32(start.tolist()), i32([0] * n_seq))
    for s, p in enumerate(prompts):
        close(lg[start[s]:start[s + 1]], m.dense(p))
    last = start[1:] - 1
    count, toks = H.verify_chains(lg, None, torch.zeros((n_seq, 0), dtype=torch.int32, device=DEV), torch.zeros((n_seq, 0), device=DEV),
                                  dev(rng.rand(n_seq).astype(np.float32)), 1.0, 50, p_start=i32(last.tolist()))
    seqs = [list(p) for p in prompts]
    new = toks[:, 0].tolist()

    for step in range(4):
        # chains: sequence 1 sits the second step out
        live = [not (step == 1 and s == 1) for s in range(n_seq)]
        rows = [k + 1 if ok else 0 for ok in live]
        start = np.concatenate([[0], np.cumsum(rows)])
        q = torch.randn(n_seq, k, VOCAB, device=DEV) * 2
        draft = q.argmax(-1).int()
        tokens = [t for s in range(n_seq) if live[s] for t in [new[s]] + draft[s].tolist()]
        past = [len(x) for x in seqs]
        lg = m.paged(H, cache, rot, i32(tokens), i32(start.tolist()), i32(past))
        ua, uf = rng.rand(n_seq, k).astype(np.float32) ** 2, rng.rand(n_seq).astype(np.float32)
        count, toks = H.verify_chains(lg, q, draft, dev(ua), dev(uf), 1.0, 200, n_draft=i32([k if ok else -1 for ok in live]),
                                      p_start=i32(start[:-1].tolist()))
        host, qh, dh = lg.cpu().numpy(), q.cpu().numpy(), draft.cpu().numpy()
        want = [chain(host[start[s]:start[s + 1]], qh[s], dh[s], ua[s], uf[s], 1.0, 200) if live[s] else (-1, []) for s in range(n_seq)]
        compare(count, toks, want, k)
        for s in range(n_seq):
            if live[s]:
                close(lg[start[s]:start[s + 1]], m.dense(seqs[s] + [new[s]] + dh[s].tolist())[-(k + 1):])
                seqs[s] += [new[s]] + want[s][1][:-1]
                new[s] = want[s][1][-1]

    # a tree step: 1 + 2 + 4 nodes a sequence, a path accepted by hand, then a chain on top of what was kept
    parent, depth, _, anc = H.tree_layout((2, 2))
    nodes = rng.randint(0, VOCAB, (n_seq, 7))
    nodes[:, 0] = new
    past = [len(x) for x in seqs]
    pos = np.concatenate([[p + d for d in depth] for p in past])
    lg = m.paged(H, cache, rot, i32(nodes.reshape(-1).tolist()), i32([0, 7, 14, 21]), i32(past),
                 tree=torch.from_numpy(np.tile(anc, n_seq).view(np.int64)).to(DEV), pos=i32(pos.tolist()))
    paths = [[2, 6], [1, 3], [2, 5]]
    for s in range(n_seq):
        for node in range(7):
            line, at = [], node
            while at >= 0:
                line.insert(0, int(nodes[s, at]))
                at = int(parent[at])
            close(lg[7 * s + node:7 * s + node + 1], m.dense(seqs[s] + line)[-1:])
    keep = [2, 1, 2]
    cache.keep(i32(past), i32(paths), i32(keep))
    for s in range(n_seq):
        seqs[s] += [int(nodes[s, 0])] + [int(nodes[s, x]) for x in paths[s][:keep[s]]]
    tokens = [5, 6, 7]
    lg = m.paged(H, cache, rot, i32(tokens), i32([0, 1, 2, 3]), i32([len(x) for x in seqs]))
    for s in range(n_seq):
        close(lg[s:s + 1], m.dense(seqs[s] + [tokens[s]])[-1:])


def test_a_captured_step_replays(H):
    # append, a split attention, keep and verification in one graph; between replays lengths, pages and rows change and the same
    # calls run eagerly
    import torch
    su = Setup(H, 4, "bf16", 2, 128, 16, [5, 5], [1400, 900], spare=2, extra=40)
    su.k.copy_(su.randn(*su.k.shape))
    su.v.copy_(su.randn(*su.v.shape))
    n = 20000
    state = dict(q=su.randn(10, 8, 128).to(DEV), k=su.randn(10, 2, 128).to(DEV), p=torch.randn(10, n, device=DEV), z=torch.randn(2, 4, n, device=DEV),
                 d=torch.randint(0, n, (2, 4), device=DEV).int(), ua=torch.rand(2, 4, device=DEV), uf=torch.rand(2, device=DEV),
                 path=torch.tensor([[2, 4], [1, 3]], dtype=torch.int32, device=DEV), keep=torch.tensor([2, 1], dtype=torch.int32, device=DEV))
    rot = H.rotary_table(2000, 128)

    def step(cache, x):
        q = cache.append(x["k"], x["k"], su.row_start, su.n_past, q=x["q"], rot=rot)
        o = cache.attend(q, su.row_start, su.n_past)
        cache.keep(su.n_past, x["path"], x["keep"])
        return o, *H.verify_chains(x["p"], x["z"], x["d"], x["ua"], x["uf"], 1.0, n)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(su.cache, state)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step(su.cache, state)
    twin_k, twin_v = su.k.clone(), su.v.clone()
    twin = H.PagedCache(twin_k, twin_v, su.table)
    for turn in range(4):
        su.n_past.copy_(torch.tensor([1400 - 300 * turn, 900 + 5 * turn]))
        for key in ("q", "k", "p", "z", "ua", "uf"):
            state[key].copy_(torch.rand_like(state[key].float()) if key[0] == "u" else torch.randn_like(state[key].float()))
        su.table.copy_(su.table.roll(1, dims=0) if turn == 2 else su.table)
        twin_k.copy_(su.k)
        twin_v.copy_(su.v)
        graph.replay()
        torch.cuda.synchronize()
        eager = step(twin, state)
        torch.cuda.synchronize()
        for a, b in zip(out, eager):
            assert torch.equal(a, b)
        assert torch.equal(su.k, twin_k) and torch.equal(su.v, twin_v)


def test_two_streams_at_once(H):
    # the same cache read by two streams, each with its own rows and results
    import torch
    su = Setup(H, 6, "fp16", 4, 64, 16, [6, 6], [1500, 700])
    su.fill()
    qs = [su.randn(12, 8, 64) for _ in range(2)]
    wants = [attention_reference(su, q, lambda s, i, e: e <= su.past[s] + i, 0.125) for q in qs]
    on = [q.to(DEV) for q in qs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    outs = [None, None]
    for turn in range(3):
        for i, st in enumerate(streams):
            with torch.cuda.stream(st):
                outs[i] = su.cache.attend(on[i], su.row_start, su.n_past)
    torch.cuda.synchronize()
    for i in range(2):
        check_attention(su, outs[i], wants[i], "fp16", weight_step("fp16"))
