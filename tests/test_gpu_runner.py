"""The cache classes on other streams than the current one, and under capture."""
import numpy as np
import pytest
import torch

from oracle import evict as OE
from paper_2601_21927_amd import sonic
from paper_2601_21927_amd.runner import bf16_to_device
from tests import gpu_helpers as H
from tests.test_gpu_q4 import EPS, Cache, i32, normal_bits

pytestmark = pytest.mark.gpu

BUSY = 20_000_000   # cycles of a waiting kernel, some ten milliseconds


@pytest.mark.parametrize("q4", [True, False])
def test_eviction_on_another_stream_while_the_current_one_allocates(q4):
    H.need_gpu()
    rng = np.random.default_rng(31 + q4)
    c = Cache(rng, [700, 30, 3000, 90], 2, 2, 128, q4)
    want = [OE.kept_rows(c.weight[o:o + n], 8, 5, 100) for o, n in zip(c.off, c.lens)]
    before = [x.clone() for x in (c.dev.k, c.dev.v, c.dev.row_weight)]
    lim = [i32([x] * 4) for x in (8, 5, 100)]
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(BUSY)
    assert c.dev.evict(*lim, c.status, stream=side) == sonic.OK
    size = sonic.cache_evict_workspace_bytes(4, int(c.cap.max()))
    held = [torch.full((size,), 0x7F, dtype=torch.uint8, device="cuda") for _ in range(20)]
    torch.cuda.synchronize()
    assert int(c.status.item()) == 0 and all(int(x[0]) == 0x7F for x in held)
    assert c.dev.length.tolist() == [len(w) for w in want]
    for old, x in zip(before, (c.dev.k, c.dev.v, c.dev.row_weight)):
        for o, kept in zip(c.off, want):
            assert torch.equal(x[o:o + len(kept)], old[o + torch.from_numpy(kept).cuda()])


@pytest.mark.parametrize("q4,weighted", [(True, True), (True, False), (False, True), (False, False)])
def test_a_first_step_on_another_stream_while_the_current_one_is_busy(q4, weighted):
    """The workspace's zeros are written where the step waits for them, and a replaced workspace is not handed out."""
    H.need_gpu()
    rng = np.random.default_rng(33 + q4)
    c = Cache(rng, [700, 30, 3000], 4, 2, 64, q4)
    side = torch.cuda.Stream()
    dirt = [torch.full((1 << 22,), 0xFF, dtype=torch.uint8, device="cuda") for _ in range(4)]
    del dirt          # what the allocator hands out next is not zero
    torch.cuda.synchronize()
    torch.cuda._sleep(BUSY)
    for bound in (c.max_ctx, 9000):
        q, k, v = (normal_bits(rng, 3, h, 64) for h in (8, 2, 2))
        with torch.cuda.stream(side):
            args = [bf16_to_device(x) for x in (q, k, v)] + [torch.zeros((3, 8, 64), device="cuda"), c.status, bound]
        if q4:
            st = c.dev.decode(*args, weighted=weighted, stream=side)
        else:
            st = (c.dev.decode_weighted if weighted else c.dev.decode)(*args, stream=side)
        assert st == sonic.OK
        held = [torch.full((1 << 20,), 0x7F, dtype=torch.uint8, device="cuda") for _ in range(8)]
        side.synchronize()
        with torch.cuda.stream(side):
            if q4 or weighted:
                c.check(q, k, v, args[3].cpu().numpy(), weighted=weighted)
            else:
                for b in range(3):
                    H.assert_close(args[3][b].cpu().numpy(), c.expect(b, q, k, v)[0], f"request {b}")
                    c.lens[b] += 1
        del held
    torch.cuda.synchronize()


@pytest.mark.parametrize("q4", [True, False])
def test_a_step_captured_before_any_eager_one(q4):
    """What a capture makes is not taken for zeroed by eager steps, nor by another graph."""
    H.need_gpu()
    rng = np.random.default_rng(35 + q4)
    c = Cache(rng, [700, 30, 3000], 40, 2, 64, q4)
    q, k, v = (bf16_to_device(normal_bits(rng, 3, h, 64)) for h in (8, 2, 2))
    out, start, w0 = torch.zeros((3, 8, 64), device="cuda"), c.dev.length.clone(), c.dev.row_weight.clone()

    def steps():
        torch.add(start, 0, out=c.dev.length)
        torch.add(w0, 0, out=c.dev.row_weight)
        for _ in range(2):
            args = (q, k, v, out, c.status, c.max_ctx)
            assert (c.dev.decode(*args, weighted=True) if q4 else c.dev.decode_weighted(*args)) == sonic.OK

    def result():
        torch.cuda.synchronize()
        got = [x.clone() for x in (out, c.dev.row_weight, c.dev.length)]
        out.zero_()
        return got

    dirt = [torch.full((1 << 22,), 0xFF, dtype=torch.uint8, device="cuda") for _ in range(4)]
    del dirt
    torch.cuda.synchronize()
    graphs = [torch.cuda.CUDAGraph() for _ in range(2)]
    for g in graphs:
        with torch.cuda.graph(g):
            steps()
    steps()
    want = result()
    assert want[2].tolist() == [702, 32, 3002] and torch.isfinite(want[0]).all() and want[0].any()
    for g in graphs[::-1] * 2:
        g.replay()
        assert all(torch.equal(x, y) for x, y in zip(result(), want))
        steps()
        assert all(torch.equal(x, y) for x, y in zip(result(), want))


def test_weights_are_not_made_under_capture():
    H.need_gpu()
    rng = np.random.default_rng(37)
    c = Cache(rng, [20, 30], 4, 2, 64, False)
    q, k, v = (bf16_to_device(normal_bits(rng, 2, h, 64)) for h in (8, 2, 2))
    out = torch.zeros((2, 8, 64), device="cuda")
    c.dev.row_weight = None
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        g = torch.cuda.CUDAGraph()
        g.capture_begin()
        try:
            with pytest.raises(RuntimeError, match="row_weight"):
                c.dev.decode_weighted(q, k, v, out, c.status, c.max_ctx)
            out.add_(1.0)
        finally:
            g.capture_end()
    torch.cuda.synchronize()
    assert c.dev.row_weight is None
    assert c.dev.decode_weighted(q, k, v, out, c.status, c.max_ctx) == sonic.OK
    assert c.dev.length.tolist() == [21, 31] and bool((c.dev.row_weight > 0).any())


@pytest.mark.parametrize("q4", [True, False])
def test_two_caches_on_two_streams_at_once(q4):
    H.need_gpu()
    rng = np.random.default_rng(39 + q4)
    caches = [Cache(rng, lens, 8, 2, 64, q4) for lens in ([700, 30, 3000], [5, 4000, 60])]
    side = [torch.cuda.Stream() for _ in caches]
    inputs = [[[normal_bits(rng, 3, h, 64) for h in (8, 2, 2)] for _ in range(6)] for _ in caches]
    dev = [[[bf16_to_device(x) for x in step] for step in steps] for steps in inputs]
    outs = [[torch.zeros((3, 8, 64), device="cuda") for _ in range(6)] for _ in caches]
    torch.cuda.synchronize()
    for t in range(6):
        for c, s, d, o in zip(caches, side, dev, outs):
            args = (*d[t], o[t], c.status, c.max_ctx)
            assert (c.dev.decode(*args, weighted=True, stream=s) if q4 else c.dev.decode_weighted(*args, stream=s)) == sonic.OK
    torch.cuda.synchronize()
    for c, steps, o in zip(caches, inputs, outs):
        got = c.dev.row_weight.cpu().numpy()
        full = c.weight.astype(np.float64)
        for t, (q, k, v) in enumerate(steps):
            for b in range(3):
                want, w = c.expect(b, q, k, v)
                rows = slice(int(c.off[b]), int(c.off[b]) + len(w))
                full[rows.stop - 1] = 0.0
                full[rows] += w
                assert np.all(np.abs(o[t][b].cpu().numpy() - want) <= 2 * EPS * np.abs(c.values[1][rows]).max())
                c.lens[b] += 1
        # six weights, each within 2 EPS of itself, and a rounding for each sum
        assert np.all(np.abs(got - full) <= 2 * EPS * (full - np.where(full == c.weight, full, 0)) + 6 * 2.0 ** -24 * full)
        assert np.array_equal(c.dev.length.cpu().numpy(), c.lens)
