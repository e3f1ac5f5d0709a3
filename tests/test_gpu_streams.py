"""The target pass in a process that uses several streams: the round of workgroups over the XCDs starts elsewhere on each hardware queue,
and a stream, the default one too, may be on another queue from launch to launch."""
import numpy as np
import pytest

import synth

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def H():
    import paper_2510_25739_amd as H
    return H


def steps(H, s, blob, cond, stream=None, between=lambda: None):
    hk = H.Hawk(H.HawkConfig.from_shape(s), stream=stream)
    hk.load(blob)
    hk.prefill(cond, None, s.grid_h, s.grid_w, 0.0, s.top_k, 1.0, [0.25])
    u = np.full((1, s.k), 0.5, np.float32)
    got = []
    for _ in range(4):
        between()
        hk.draft(s.k, u)
        between()
        na, toks = hk.verify(s.k, u, [0.5])
        got.append((int(na[0]), toks.tolist()))
    assert hk.last_path() == 1
    got.append(hk.grid().tolist())
    hk.close()
    return got


def test_the_pass_runs_on_every_queue(H):
    import torch
    s = synth.CONFIGS[1].replace(n_layers=2, n_cond=24, grid_h=6, grid_w=8)
    blob, cond = synth.make_weights(s, seed=0), synth.make_cond(s, seed=2)
    want = steps(H, s, blob, cond)
    streams = [torch.cuda.Stream() for _ in range(6)]
    x = torch.ones(1000, device="cuda:0")
    torch.cuda.synchronize()

    def others():
        for st in streams:
            with torch.cuda.stream(st):
                x * 2
            torch.cuda.synchronize()

    assert steps(H, s, blob, cond, between=others) == want
    for st in streams:
        assert steps(H, s, blob, cond, stream=st) == want
        assert steps(H, s, blob, cond) == want
