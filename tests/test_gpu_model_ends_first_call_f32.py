"""The f32 kernels of the cross entropy, those of numbers in three parts among them, recorded into a HIP graph by the first call that a process makes of them."""
import os
import subprocess
import sys

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.gpu
def test_first_calls_are_recorded():
    """A process of its own, because the other tests have made eager calls in this one."""
    r = subprocess.run([sys.executable, "-u", os.path.abspath(__file__)], cwd=ROOT, stdout=subprocess.PIPE, stderr=subprocess.STDOUT,
                       timeout=100, text=True)
    assert r.returncode == 0 and r.stdout.rstrip().endswith("every first call was recorded"), r.stdout[-4000:]


def calls(kt, normal, gen):
    """(name, input that replays change, outputs, call): few tokens, tiles of 64 and 128, three parts in one piece of the vocabulary and in several."""
    dev = "cuda"
    g = gen(1)
    empty = lambda *s: torch.empty(*s, device=dev)  # noqa: E731
    for tokens, vocab, width in ((20, 500, 136), (300, 700, 136), (1500, 2100, 100), (1500, 6200, 130), (20000, 4099, 136), (20000, 6657, 40)):
        x, w = normal(g, tokens, width, scale=0.3), normal(g, vocab, width, scale=0.1)
        t = torch.randint(-1, vocab, (tokens,), generator=g, device=dev)
        dloss, one = torch.rand(tokens, generator=g, device=dev), torch.ones(tokens, device=dev)
        loss, lse, dx, dw = empty(tokens), empty(tokens), empty(tokens, width), empty(vocab, width)
        yield "linear_xent_bwd of %d x %d" % (tokens, vocab), dloss, (dx, dw), lambda x=x, w=w, t=t, d=dloss, l=one, dx=dx, dw=dw: kt.kt_linear_xent_bwd(d, x, w, t, l, dx, dw)
        yield "linear_xent_fwd of %d x %d" % (tokens, vocab), x, (loss, lse), lambda x=x, w=w, t=t, a=loss, b=lse: kt.kt_linear_xent_fwd(x, w, t, a, b)


def main():
    sys.path[:0] = [ROOT, os.path.join(ROOT, "tests")]
    import paper_2505_10183_amd as kt
    from ops_util import gen, normal
    for name, given, out, call in calls(kt, normal, gen):
        torch.cuda.synchronize()
        print(name)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            call()
        for _ in range(3):
            given.mul_(1.25)
            for t in out:
                t.zero_()
            graph.replay()
            torch.cuda.synchronize()
            got = [t.clone() for t in out]
            for t in out:
                t.zero_()
            call()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(got, out)) and any(bool(t.any()) for t in got), name
    print("every first call was recorded")


if __name__ == "__main__":
    main()
