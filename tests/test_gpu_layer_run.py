"""A memory-attention layer as a tracker with hypotheses runs it: heads turned by frame, row and column, keys
committed, the readout over the shared prefix, the norm and gate behind it, the scored readout of a second
block, and again.  Every call against 64 bits on what it was given; captured and replayed."""
import pytest
import torch

from test_gpu_layer import angles, block_ref, check, check_rope, frequencies, rope_ref
from test_gpu_long_bank import DT, Built, bits, gen
from test_gpu_more_readouts import frames_of, reference, scored_rows, shared_rows

pytestmark = pytest.mark.gpu


class Held:
    """A pipeline's bank as the references read it."""
    places = Built.places

    def __init__(self, rs3, pipe):
        self.rs3, self.bank = rs3, pipe.bank


def workload(synth, dtype, H, d, per, window, frames):
    return synth.Workload("layer", 90, 12, 13, H, d, dtype, 2, per, frames, 0.1, 0.4, 1, window, 3)


@pytest.mark.parametrize("dtype,H,d", [("bf16", 2, 64), ("bf16", 1, 256), ("f32", 2, 32)])
def test_frames_of_a_layer_with_hypotheses(dtype, H, d):
    from paper_2608_22526_gb300 import rs3, synth
    from paper_2608_22526_gb300.pipeline import Pipeline
    G, per, m, n, D = 2, 3, 12, 13, H * d
    mn, U, dt = m * n, G * per, DT[dtype]
    g = gen(d)

    def rand(*shape, scale=1.0):
        return (torch.randn(shape, generator=g, device="cuda") * scale).to(dt)

    track = Pipeline(workload(synth, dtype, H, d, 1, -1, 6), ring_cap=6 * mn)
    hyp = Pipeline(workload(synth, dtype, H, d, per, 2, 6))
    prefix_unit = torch.tensor([0, 0, -1, 1, 1, 1], dtype=torch.int32, device="cuda")
    hyp.share(track, prefix_unit)
    F = hyp.bank.max_frames
    bias = torch.randn((H, F + 2), generator=g, device="cuda")
    keep = torch.ones((U, F + 2), dtype=torch.uint8, device="cuda")
    keep[1, 0] = keep[4, F] = 0
    hyp.use_scores(15.0, bias, keep)
    pairs = (d // 8, d // 8, d // 8)
    spec = rs3.rope_spec(2 * sum(pairs), pairs, "halves", factor=4.0, context=64.0)
    freq = frequencies(pairs, 10000.0, 4.0, 64.0, 32.0, 1.0)
    cell = torch.arange(mn, device="cuda")

    def positions(units, t):
        return torch.stack([torch.full_like(cell, t), cell // n, cell % n], -1).to(torch.int32)[None].repeat(units, 1, 1).contiguous()

    def masks(units, seed):
        return (torch.rand((units, mn), generator=gen(seed), device="cuda") < 0.35).to(torch.uint8)

    def put(pipe, t, cond):                                # a frame's keys turned and committed
        k, v, mask, pos = rand(pipe.w.U, mn, D), rand(pipe.w.U, mn, D), masks(pipe.w.U, t), positions(pipe.w.U, t)
        turned = torch.zeros_like(k)
        pipe.rotate(None, None, None, k, turned, pos, spec, k_keep=mask)
        on = mask.view(-1) != 0
        ang = angles(pos, pairs, freq)[on]
        check_rope(turned.view(-1, D)[on], *rope_ref(k.view(-1, D)[on], H, d, spec.rot, "halves", ang), dtype, ang)
        pipe.commit(turned, v, mask, cond)

    for t in range(5):
        put(track, t, int(t == 0))
    track.set_pointers(rand(G, 3, D), rand(G, 3, D))
    put(hyp, 5, 1)
    hyp.set_pointers(rand(U, 3, D), rand(U, 3, D))
    w = [1 + 0.2 * torch.randn(s, generator=g, device="cuda") for s in ((D,), (U, D), (D,))]
    norms = dict(post="rms", post_weight=w[0], gate=w[1], alpha=0.9, pre="layer", pre_weight=w[2], eps=1e-5)
    x, z, q = rand(U, mn, D), rand(G, mn, D, scale=1.3), torch.zeros((G, mn, D), dtype=dt, device="cuda")
    a, h = (torch.zeros((U, mn, D), dtype=dt, device="cuda") for _ in range(2))
    prev = masks(U, 50)
    pos = positions(G, 0)

    def block(read):                                       # one block: attention, then the residual stream and the next input
        read(q, None, a)
        before = x.clone()
        hyp.norm_residual(a, x, x, h, **norms)
        return before

    for t in range(6, 9):
        pos.copy_(positions(G, t))
        z.copy_(rand(G, mn, D, scale=1.3))
        put(hyp, t, 0)
        hyp.select(z, prev)
        hyp.rotate(z, q, pos, None, None, None, spec)
        ang = angles(pos, pairs, freq)
        check_rope(q.view(-1, D), *rope_ref(z.view(-1, D), H, d, spec.rot, "halves", ang), dtype, ang)
        counts, idx = hyp.count.tolist(), hyp.idx
        assert min(counts) > 0
        for read, rows, cap, of in ((hyp.readout_shared, shared_rows(Held(rs3, hyp), Held(rs3, track), prefix_unit), 0.0, None),
                                    (hyp.readout_scored, scored_rows(Held(rs3, hyp), keep), 15.0, lambda u, i: bias[i])):
            before = block(read)
            want, tol = reference(dtype, H, d, q, idx, counts, hyp.unit_group, None, d ** -0.5, None, a.shape, rows, cap, of)
            assert ((a.double() - want).abs() <= tol).all()
            for u in range(U):
                cells = idx[u, :counts[u]].long()
                vx, vh = block_ref(a[u, cells], before[u, cells], ("rms", w[0], None), ("layer", w[2], None), w[1][u], 0.9, 1e-5)
                check(x[u, cells], *vx, dtype)
                check(h[u, cells], *vh, dtype)
                rest = torch.ones(mn, dtype=torch.bool, device="cuda")
                rest[cells] = False
                assert torch.equal(bits(x[u, rest]), bits(before[u, rest]))
        assert hyp.status_code() == 0 and track.status_code() == 0

    # the same frame captured: replayed on other queries, and again as it was
    x0 = x.clone()

    def frame():
        hyp.rotate(z, q, pos, None, None, None, spec)
        block(hyp.readout_shared)
        block(hyp.readout_scored)

    frame()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        frame()
    z.mul_(0.5)
    x.copy_(x0)
    graph.replay()
    torch.cuda.synchronize()
    got = [v.clone() for v in (q, a, x, h)]
    x.copy_(x0)
    for v in (q, a):
        v.zero_()
    frame()
    torch.cuda.synchronize()
    assert all(torch.equal(bits(i), bits(j)) for i, j in zip(got, (q, a, x, h)))
    assert hyp.status_code() == 0


def test_frames_command_with_scores():
    from paper_2608_22526_gb300 import run_frames
    pipe = run_frames.run("sam2_1obj", 4, False, 50.0, 0.5)
    assert pipe.status_code() == 0 and int(pipe.count.min()) > 0
