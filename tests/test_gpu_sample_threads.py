"""Draws by host threads of their own at once: rows of lengths that take unlike amounts of shared memory, each on its own stream
with its own workspace, give what they give alone, and no call is refused.  The threads call the library itself, with arguments made
beforehand, so that several of them are inside it at a time."""
import ctypes
import threading

import pytest
import torch

import paper_2512_06547_b200 as a3po

pytestmark = pytest.mark.gpu
DEV = "cuda"


class Draw:
    def __init__(self, n, v, td, seed):
        gen = torch.Generator(device=DEV).manual_seed(seed)
        self.logits = (torch.randn(n, v, generator=gen, device=DEV) * 2).to(td)
        self.u = torch.rand(n, generator=gen, device=DEV)
        self.k = torch.full((n,), 40, dtype=torch.int32, device=DEV)
        self.ws = a3po.new_workspace(a3po.a3po_sample_workspace_bytes(n, v), DEV)
        self.token = torch.empty(n, dtype=torch.int32, device=DEV)
        self.logp = torch.empty(n, device=DEV)

        self.stream = torch.cuda.Stream()
        at = lambda t: ctypes.c_void_p(t.data_ptr())
        self.args = [at(self.logits), v, None, n, v, a3po.A3PO_F32 if td == torch.float32 else a3po.A3PO_BF16, None, at(self.k), None,
                     None, at(self.u), at(self.token), at(self.logp), None, None, at(self.ws), self.ws.numel(),
                     ctypes.c_void_p(self.stream.cuda_stream)]


@pytest.mark.parametrize("td", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("sizes", [((2, 151936), (2, 4096)), ((300, 4000), (300, 300)), ((1, 300000), (8, 20000))])
def test_threads(td, sizes):
    draws = [Draw(n, v, td, 1 + i) for i, (n, v) in enumerate(sizes * 4)]
    call = a3po.load_library().a3po_sample
    alone = []
    torch.cuda.synchronize()
    for d in draws:
        assert call(*d.args) == 0
        torch.cuda.synchronize()
        alone.append((d.token.clone(), d.logp.clone()))
    refused, start = [0] * len(draws), threading.Barrier(len(draws))

    def work(i):
        args = draws[i].args
        start.wait()
        for _ in range(1500):
            if call(*args) != 0:
                refused[i] += 1

    threads = [threading.Thread(target=work, args=(i,)) for i in range(len(draws))]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert refused == [0] * len(draws)
    for d, (token, logp) in zip(draws, alone):
        assert torch.equal(d.token, token) and torch.equal(d.logp, logp)
