"""Calls that are recorded in torch's inference mode and outside of it on one handle, replayed among eager ones of both."""
import pytest
import torch

from paper_2309_06973_amd.q8 import Q8

pytestmark = pytest.mark.gpu
DEV = "cuda"


def test_recorded_in_one_mode_and_another():
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        ops = Q8()
        x = torch.randn(3, 50001, generator=torch.Generator().manual_seed(1)).to(DEV)
        grads = [torch.randn(40000, generator=torch.Generator().manual_seed(2)).to(DEV), torch.ones(7, device=DEV)]
        answer = lambda: ops.log_probs(x, entropy=True, top=5)
        with torch.inference_mode():
            answer()
        ops.grad_norm(grads)
        torch.cuda.synchronize()
        graphs = []
        for mode in (True, False, True, False):
            g = torch.cuda.CUDAGraph()
            # inside of the recording: torch's own state of a recording belongs to the mode that the first one began in
            with torch.cuda.graph(g, stream=stream), torch.inference_mode(mode):
                r, n = answer(), ops.grad_norm(grads)
            graphs.append((g, r, n))
        for i in range(3):
            x.copy_(torch.randn(3, 50001, generator=torch.Generator().manual_seed(10 + i)))
            graphs.reverse()
            for j, (g, r, n) in enumerate(graphs):
                grads[0].mul_(1.25)
                with torch.inference_mode(j % 2 == 0):
                    want, norm = answer(), ops.grad_norm(grads)
                g.replay()
                torch.cuda.synchronize()
                assert torch.equal(n, norm)
                assert all(torch.equal(p, q) for p, q in zip(r, want) if p is not None)
        torch.cuda.synchronize()
        ops.close()
