"""The operators of a training step together: tokens are looked up, a layer with 8-bit weights is applied, the layer's and the
table's gradients are added up over micro-batches in one flat bucket per worker, and the workers' buckets are exchanged.  Every
stage is compared with 64 bits on what the stage before it left."""
import numpy as np
import pytest
import torch

import paper_2407_01378_amd as thc
from gpu_util import check_against_oracle, run_path_fused
from oracle import embed as E
from oracle import fp8 as O

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _u8(n, fill=0xAB):
    return torch.full((n,), fill, dtype=torch.uint8, device=DEV)


def _codes(rows, cols):
    return _u8(rows * thc.thc_fp8_row_bytes(cols)), _u8(thc.thc_fp8_scale_bytes(rows, cols))


class Worker:
    """A table, weights in both forms and one flat fp32 bucket for their gradients."""

    def __init__(self, vocab, dim, out, count, seed):
        self.vocab, self.dim, self.out, self.count = vocab, dim, out, count
        self.table = torch.randn(vocab, dim, generator=_gen(1), device=DEV).bfloat16()
        self.w = torch.randn(out, dim, generator=_gen(2), device=DEV) / dim ** 0.5
        self.wq, self.wtq = _codes(out, dim), _codes(dim, out)
        thc.thc_fp8_quantize(self.w, thc.THC_E4M3, *self.wq, *self.wtq, True)
        self.bucket = torch.empty(vocab * dim + out * dim, device=DEV)
        self.dtable = self.bucket[:vocab * dim].view(vocab, dim)
        self.dw = self.bucket[vocab * dim:].view(out, dim)
        self.tokens = torch.zeros(count, dtype=torch.int64, device=DEV)
        self.target = torch.randn(count, out, generator=_gen(50 + seed), device=DEV)
        self.x = torch.empty(count, dim, dtype=torch.bfloat16, device=DEV)
        self.y, self.dy = torch.empty(count, out, device=DEV), torch.empty(count, out, device=DEV)
        self.dx = torch.empty(count, dim, device=DEV)
        self.xq, self.xtq, self.dyq, self.dytq = _codes(count, dim), _codes(dim, count), _codes(count, out), _codes(out, count)
        self.ws = _u8(max(thc.thc_fp8_linear_workspace_bytes(count, out, dim), thc.thc_fp8_matmul_workspace_bytes(out, dim, count),
                          thc.thc_fp8_matmul_workspace_bytes(count, dim, out), thc.thc_embed_backward_workspace_bytes(count, vocab, dim)))

    def step(self):
        thc.thc_embed_forward(self.table, self.tokens, 0.5, self.x)
        thc.thc_fp8_linear(self.x, thc.THC_E4M3, *self.wq, thc.THC_E4M3, self.y, self.ws)
        torch.sub(self.y, self.target, out=self.dy)
        thc.thc_fp8_quantize(self.x, thc.THC_E4M3, None, None, *self.xtq)
        thc.thc_fp8_quantize(self.dy, thc.THC_E5M2, *self.dyq, *self.dytq)
        thc.thc_fp8_matmul(*self.dytq, thc.THC_E5M2, *self.xtq, thc.THC_E4M3, self.count, self.dw, self.ws, True)
        thc.thc_fp8_matmul(*self.dyq, thc.THC_E5M2, *self.wtq, thc.THC_E4M3, self.out, self.dx, self.ws)
        thc.thc_embed_backward(self.dx, self.tokens, 0.5, self.dtable, self.ws, True)


def _values(x, fmt, tile=False):
    x64 = x.double().cpu().numpy()
    return O.values(*O.quantize(np.ascontiguousarray(x64), fmt, tile), fmt, x64.shape[1])


def _near(got, want, size, terms):
    """Each of `terms` additions off by at most 2^-23 of a partial sum, none of which exceeds the sum of magnitudes."""
    err = np.abs(got.double().cpu().numpy() - want)
    assert (err <= size * terms * 2.0 ** -23 + 1e-38).all(), float((err / (size + 1e-38)).max())


@pytest.mark.parametrize("vocab,dim,out,count", [(300, 320, 200, 160), (77, 130, 264, 1), (1000, 96, 130, 700)])
def test_steps_of_three_workers(vocab, dim, out, count):
    workers = [Worker(vocab, dim, out, count, i) for i in range(3)]
    rng = np.random.default_rng(count)
    w64 = _values(workers[0].w, "e4m3", True)
    wt64 = _values(workers[0].w.t().contiguous(), "e4m3", True)
    assert np.array_equal(wt64, w64.T)
    for worker in workers:
        worker.bucket.zero_()
        dw = np.zeros((2, out, dim))        # the gradient and the sum of magnitudes
        dt = np.zeros((2, vocab, dim))
        for _ in range(2):
            tokens = rng.integers(-1, vocab, count)
            worker.tokens.copy_(torch.tensor(tokens))
            worker.step()
            x = torch.tensor(E.forward(worker.table.double().cpu().numpy(), tokens, 0.5))
            assert torch.equal(worker.x.cpu(), x.float().bfloat16())
            x64 = _values(worker.x, "e4m3")
            _near(worker.y, x64 @ w64.T, np.abs(x64) @ np.abs(w64.T), dim)
            xt64, dy64, dyt64 = (_values(v, f) for v, f in ((worker.x.t(), "e4m3"), (worker.dy, "e5m2"), (worker.dy.t(), "e5m2")))
            _near(worker.dx, dy64 @ w64, np.abs(dy64) @ np.abs(w64), out)
            dw += dyt64 @ xt64.T, np.abs(dyt64) @ np.abs(xt64.T)
            d, size, _ = E.backward(worker.dx.double().cpu().numpy(), tokens, 0.5, vocab)
            dt += d, size
        _near(worker.dw, dw[0], dw[1], count + 2)              # (and the additions to what was there)
        _near(worker.dtable, dt[0], dt[1], count + 4)
    # the exchange
    buckets = [worker.bucket for worker in workers]
    check_against_oracle(buckets, run_path_fused(buckets, 10, 5, 4), 10, 5, 4)


def test_a_step_captured_and_replayed():
    """On one workspace and bucket for two graphs, with eager steps between the replays."""
    workers = [Worker(500, 136, 264, count, i) for i, count in enumerate((48, 300))]
    workers[0].ws = workers[1].ws
    graphs = []
    for worker in workers:
        worker.step()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            worker.step()
        graphs.append(graph)
    for i in range(4):
        eager = []
        for worker in workers:
            worker.tokens.copy_(torch.randint(-1, 500, (worker.count,), generator=_gen(i), device=DEV))
            worker.bucket.fill_(0.25 * i)
            worker.step()
            torch.cuda.synchronize()
            eager.append((worker.y.clone(), worker.bucket.clone()))
            worker.bucket.fill_(0.25 * i)
            worker.y.zero_()
            worker.ws.random_(0, 256)
        torch.cuda.synchronize()
        for graph in graphs if i % 2 else graphs[::-1]:
            graph.replay()
        torch.cuda.synchronize()
        for worker, (y, bucket) in zip(workers, eager):
            assert torch.equal(worker.y, y) and torch.equal(worker.bucket, bucket)


def test_workers_on_streams_of_their_own():
    """Steps on two streams at once, each with its own memory, give what they give one after the other."""
    workers = [Worker(400, 256, 130, 200, i) for i in range(2)]
    alone = []
    for i, worker in enumerate(workers):
        worker.tokens.copy_(torch.randint(0, 400, (200,), generator=_gen(i), device=DEV))
        worker.bucket.zero_()
        worker.step()
        torch.cuda.synchronize()
        alone.append(worker.bucket.clone())
    streams = [torch.cuda.Stream() for _ in workers]
    for _ in range(3):
        for worker in workers:
            worker.bucket.zero_()
        torch.cuda.synchronize()
        for worker, stream in zip(workers, streams):
            with torch.cuda.stream(stream):
                worker.step()
        torch.cuda.synchronize()
        assert all(torch.equal(worker.bucket, a) for worker, a in zip(workers, alone))
