"""es_route where its kernels' shared memory grows, and calls of different sizes at once. The definition:
project_reference.py."""
import os
import subprocess
import sys
import textwrap
import threading

import pytest
import torch

import project_reference as R
from test_gpu_project import pj  # noqa: F401

pytestmark = pytest.mark.gpu


class Routed:
    def __init__(self, pj, scores, top, normalise=True):  # noqa: F811
        self.pj, self.scores, self.top, self.normalise = pj, scores.cuda(), top, normalise
        tokens, count = scores.shape
        self.chosen, self.places = (torch.empty(tokens, top, dtype=torch.int32, device="cuda") for _ in range(2))
        self.weights = torch.empty(tokens, top, device="cuda")
        self.start = torch.empty(count + 1, dtype=torch.int32, device="cuda")
        self.rows = torch.full((tokens * top,), -7, dtype=torch.int32, device="cuda")
        self.space = torch.empty(pj.es_route_workspace(tokens, count, top), dtype=torch.uint8, device="cuda")

    def run(self):
        self.pj.es_route(self.scores, self.chosen, self.weights, self.start, self.rows, self.places, self.space,
                         normalise=self.normalise)

    def check(self):
        chosen, weights, start, rows, places = R.route(self.scores.cpu(), self.top, self.normalise)
        assert self.chosen.tolist() == chosen and self.start.tolist() == start and self.places.tolist() == places
        assert self.rows.tolist()[:len(rows)] == rows
        want = torch.tensor(weights, dtype=torch.float64)
        off = (2.0 ** -20 + self.scores.shape[1] * 2.0 ** -23) * want + 1e-44
        assert ((self.weights.double().cpu() - want).abs() <= off).all()


ALONE = """
    import sys
    sys.path[:0] = [{root!r}, {tests!r}]
    import torch
    from paper_2608_17310_gb300 import project as pj
    from test_gpu_route_ranges import Routed
    for count in {counts}:
        for dtype in (torch.bfloat16, torch.float32):
            r = Routed(pj, torch.randn({tokens}, count, generator=torch.Generator().manual_seed(count)).to(dtype), 6)
            r.run()
            r.check()
    print("fine")
"""


def alone(text, **kw):
    """A program of its own, in which no earlier call has set anything."""
    from conftest import ROOT
    text = textwrap.dedent(text).format(root=ROOT, tests=os.path.join(ROOT, "tests"), **kw)
    done = subprocess.run([sys.executable, "-c", text], capture_output=True, text=True, timeout=300, cwd=ROOT)
    assert done.returncode == 0 and done.stdout.endswith("fine\n"), done.stderr[-2000:]


@pytest.mark.parametrize("tokens,counts", [(7, [384]), (256, [383, 384, 385]), (300, [384, 1024, 384])])
def test_counts_around_the_default_shared_memory(pj, tokens, counts):  # noqa: F811
    """384 experts' counters by 32 warps are just the 48 KB that a block has without asking for more, and the block has others."""
    alone(ALONE, counts=counts, tokens=tokens)


def test_calls_of_different_sizes_from_two_threads(pj):  # noqa: F811
    """What a launch may use of shared memory is a property of the kernel in the whole process: no call takes it
    from another."""
    calls = [Routed(pj, torch.randn(tokens, count, generator=torch.Generator().manual_seed(count)), 3)
             for count, tokens in ((1024, 200), (400, 200), (1024, 400), (400, 400))]
    torch.cuda.synchronize()
    failed = []

    def loop(mine):
        try:
            with torch.cuda.stream(torch.cuda.Stream()):
                for _ in range(2000):
                    mine.run()
                torch.cuda.current_stream().synchronize()
        except Exception as e:
            failed.append(e)

    threads = [threading.Thread(target=loop, args=(c,)) for c in calls]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not failed, failed
    for c in calls:
        c.check()


@pytest.mark.parametrize("count", [2, 31, 64, 100, 200, 700])
@pytest.mark.parametrize("tokens", [5, 400])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_zeros_of_both_signs_are_equal_scores(pj, count, tokens, dtype):  # noqa: F811
    """In one lane's scores and across lanes, as the largest scores and among others."""
    g = torch.Generator().manual_seed(count + tokens)
    scores = torch.randn(tokens, count, generator=g)
    zero = torch.rand(tokens, count, generator=g) < 0.6
    scores = torch.where(zero, torch.where(torch.rand(tokens, count, generator=g) < 0.5, 0.0, -0.0), scores)
    scores[::2] = torch.where(zero[::2], scores[::2], -scores[::2].abs())  # zeros are the largest
    scores[0] = -0.0
    scores[0, count - 1] = 0.0
    r = Routed(pj, scores.to(dtype), min(4, count))
    r.run()
    r.check()
