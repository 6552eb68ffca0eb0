"""Operators recorded into a HIP graph by the first call that a process makes of them: no eager call before it."""
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
    """(name, input that replays change, outputs, call) of every operator, and of the weight gradient with tiles of every size."""
    bf16, dev = torch.bfloat16, "cuda"
    g = gen(1)
    empty = lambda *s, dtype=bf16: torch.empty(*s, dtype=dtype, device=dev)  # noqa: E731

    def checkpoint(rows, cols):
        q, e = kt.kt_act8_shapes(rows, cols)
        return (torch.randint(-127, 128, q, generator=g, device=dev, dtype=torch.int8),
                torch.randint(118, 123, e, generator=g, device=dev, dtype=torch.uint8))

    x, gamma, dgamma = normal(g, 300, 2048, dtype=bf16), normal(g, 2048, dtype=bf16), empty(2048)
    y, mean, rstd = empty(300, 2048), empty(300, dtype=torch.float32), empty(300, dtype=torch.float32)
    yield "layernorm_fwd", x, (y, mean, rstd), lambda: kt.kt_layernorm_fwd(x, gamma, gamma, 1e-5, y, mean, rstd)
    dx, dy, one = empty(300, 2048), normal(g, 300, 2048, dtype=bf16), torch.ones(300, device=dev)
    yield "layernorm_bwd", dy, (dx, dgamma), lambda: kt.kt_layernorm_bwd(dy, x, gamma, one, one, dx, dgamma)
    q8, e8 = checkpoint(300, 2048)
    yield "act8_save", x, (q8, e8), lambda: kt.kt_act8_save(x, q8, e8)
    e2 = torch.randint(118, 123, e8.shape, generator=g, device=dev, dtype=torch.uint8)
    yield "act8_restore", e2, (y,), lambda: kt.kt_act8_restore(q8, e2, y)
    for tokens, out, inn in ((1111, 96, 130), (300, 1792, 1800), (1111, 3600, 3700)):
        d, w, (q, e) = normal(g, tokens, out, dtype=bf16), empty(out, inn), checkpoint(tokens, inn)
        yield "weight_grad of %d x %d" % (out, inn), d, (w,), lambda d=d, w=w, q=q, e=e: kt.kt_act8_weight_grad(d, q, e, w)
    q, k, v, do = (normal(g, 2, 200, 2, 128, dtype=bf16) for _ in range(4))
    o, lse, back = empty(2, 200, 2, 128), empty(2, 2, 200, dtype=torch.float32), [empty(2, 200, 2, 128) for _ in range(3)]
    yield "attention_fwd", q, (o, lse), lambda: kt.kt_attention_fwd(q, k, v, o, lse, causal=True)
    yield "attention_bwd", do, back, lambda: kt.kt_attention_bwd(do, q, k, v, o, lse, *back, causal=True)


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
            if given.dtype == torch.uint8:
                given.add_(1)
            else:
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
