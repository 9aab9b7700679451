"""Two batches' serving steps on two streams at once leave the bits that each leaves alone.  Needs an MI355X: ``-m gpu``."""
import os

import pytest
import torch

from paper_2604_24013_amd import binding as cf
from tests.test_gpu_window_decoder_run import DEV, SCALE, Server, _i32

pytestmark = pytest.mark.gpu
STEPS = [[[1400, 5, 700], [300, 1, 400], [1, 700, 1], [1, 1, 1], [2, 1, 0], [600, 1, 1]],       # new tokens of each server's places
         [[9, 1300, 800], [1, 1, 900], [1, 1, 1], [800, 0, 1], [1, 1, 1], [1, 500, 300]]]
ROWS = 2304


def _server(i):
    return Server(40 + i, 3, 8, 1, 16, ("bf16", "e4m3")[i], 600, 4, pages=500, width=192, rows=ROWS)


def _inputs(i):
    """What comes from outside, for each step: lengths, pages that have left a window, rows."""
    g, held, steps = torch.Generator(device=DEV), [0, 0, 0], []
    g.manual_seed(50 + i)
    for new in STEPS[i]:
        steps.append(dict(held=_i32(held), new_tokens=_i32(new), back_from=_i32([1] * 3), back_to=_i32([(h + 1 - 600) // 16 for h in held]),
                          x=torch.randn(ROWS, 10, 128, generator=g, device=DEV).bfloat16()))
        held = [h + n for h, n in zip(held, new)]
    return steps


def _enqueue(server, steps, new, stream):
    """All steps on the stream, with nothing waited for; what each of them leaves."""
    left = []
    with torch.cuda.stream(stream):
        for s, n in zip(steps, new):
            for name in ("held", "new_tokens", "back_from", "back_to"):
                server.t[name].copy_(s[name])
            server.x.copy_(s["x"])
            server.out.fill_(-7), server.lse.fill_(-7)
            server.step(max(n), stream)
            left.append([server.out.clone(), server.lse.clone(), server.q.clone()] + [server.t[k].clone() for k in sorted(server.t)])
        left.append([t.clone() for t in server.pool + server.exps])
    return left


def test_steps_of_two_batches_at_once():
    assert torch.cuda.is_available() and os.path.exists(cf.LIB_PATH)
    streams, spaces = [torch.cuda.Stream() for _ in range(2)], [torch.empty(128 << 20, dtype=torch.uint8, device=DEV) for _ in range(2)]
    inputs = [_inputs(i) for i in range(2)]
    for i in range(2):                                                       # (chunks whose walks are cut)
        s, paged = _server(i), cf.paged_desc(3, 8, ROWS, max(STEPS[i][0]), 192 * 16, 192, SCALE)
        assert 0 < cf.attn_paged_window_workspace_bytes(s.desc, paged, cf.window(600, 4)) <= spaces[i].numel()
    for st, ws in zip(streams, spaces):
        cf.set_workspace(ws, 0, st)
    try:
        torch.cuda.synchronize()
        alone = []
        for i in range(2):
            s = _server(i)
            torch.cuda.synchronize()
            alone.append(_enqueue(s, inputs[i], STEPS[i], streams[i]))
            torch.cuda.synchronize()
            assert int(s.t["free_left"]) >= 0 and bool(torch.isfinite(alone[i][0][0][:sum(STEPS[i][0])].float()).all())
        for _ in range(3):
            servers = [_server(i) for i in range(2)]
            torch.cuda.synchronize()
            together = [_enqueue(s, inputs[i], STEPS[i], streams[i]) for i, s in enumerate(servers)]
            torch.cuda.synchronize()
            for a, b in zip(alone, together):
                for x, y in zip(a, b):
                    assert all(torch.equal(t.view(torch.uint8), u.view(torch.uint8)) for t, u in zip(x, y))
    finally:
        for st in streams:
            cf.set_workspace(None, 0, st)
