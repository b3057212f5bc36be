"""Calls of the orthogonalised updates that the documentation allows, beside
those of test_gpu_ortho.py (GPU): handles of default precision in the outer
step, calls after a failed one, and layouts beyond a launch."""
import pytest
import torch

from ortho_reference import layout
from paper_2412_07210_amd.outer import EDIT_EINVAL
from paper_2412_07210_amd import ONE_PASS, EditOuter, EditOuterError, OrthoConfig, Orthogonalizer, OuterConfig

pytestmark = pytest.mark.gpu

DEV = torch.device("cuda:0")


def _randn(n, seed, std=1.0):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    return torch.empty(n, device=DEV).normal_(0.0, std, generator=gen)


def _ortho(numel, matrices, **more):
    return Orthogonalizer(OrthoConfig(numel, matrices, scale="rms", **more), DEV)


SHAPES = [[(128, 100), (60, 60)], [(200, 300), (90, 70)]]


def _outer_step(numel, ortho, seed=1):
    """theta, momentum and replicas behind one outer step with `ortho`."""
    cfg = OuterConfig(2, [numel], "bf16", outer_lr=2e-3)
    theta, b = _randn(numel, seed, 0.02), _randn(numel, seed + 1, 1e-3)
    reps = [(theta + _randn(numel, seed + 2 + j, 1e-3)).to(torch.bfloat16) for j in range(2)]
    with EditOuter(cfg, DEV) as h:
        h.step_layer_ortho(0, ortho, theta, b, reps)
        torch.cuda.synchronize()
    return [theta, b, *reps]


@pytest.mark.parametrize("shapes", SHAPES, ids=["one block", "tiles"])
def test_outer_step_takes_full_unless_told(shapes):
    """theta is fp32: a handle that no precision was named for steps it with
    FULL whatever its dtype; a named precision holds."""
    numel, mats = layout(shapes, tail=9)
    with _ortho(numel, mats, dtype="f32", precision="full") as full, _ortho(numel, mats, dtype="f32", precision="fast") as fast:
        want_full, want_fast = _outer_step(numel, full), _outer_step(numel, fast)
    assert not torch.equal(want_full[0], want_fast[0])
    for dtype, precision, want in (("bf16", None, want_full), ("f32", None, want_full), ("bf16", "full", want_full),
                                   ("bf16", "fast", want_fast)):
        with _ortho(numel, mats, dtype=dtype, precision=precision) as o:
            for _ in range(2):
                got = _outer_step(numel, o)
                assert all(torch.equal(x, y) for x, y in zip(got, want)), f"{dtype} {precision}"


def test_default_handle_serves_both_steps():
    """One bf16 handle as a worker's and as the outer step's: its own calls keep FAST's results."""
    numel, mats = layout(SHAPES[1], tail=9)
    x = _randn(numel, 30).to(torch.bfloat16)
    with _ortho(numel, mats, precision="fast") as named, _ortho(numel, mats) as o, \
            _ortho(numel, mats, dtype="f32") as full:
        want, steps = named.orthogonalize(x), _outer_step(numel, full)
        for _ in range(2):
            assert torch.equal(o.orthogonalize(x), want)
            assert all(torch.equal(p, q) for p, q in zip(_outer_step(numel, o), steps))


def test_default_handle_in_a_graph():
    """The first outer step with a handle of default precision makes a workspace:
    refused in a capture, which stays usable; a later one is captured and replayed."""
    numel, mats = layout(SHAPES[1], tail=9)
    cfg = OuterConfig(2, [numel], "bf16", outer_lr=2e-3)
    theta, b = _randn(numel, 1, 0.02), _randn(numel, 2, 1e-3)
    reps = [(theta + _randn(numel, 3 + j, 1e-3)).to(torch.bfloat16) for j in range(2)]
    fixed = [theta, b, *reps]
    eager = [t.clone() for t in fixed]
    mark = torch.zeros(4, device=DEV)
    with EditOuter(cfg, DEV) as h, EditOuter(cfg, DEV) as h2, _ortho(numel, mats) as o, _ortho(numel, mats, dtype="f32") as full:
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=torch.cuda.Stream(DEV)):
            mark.add_(1.0)
            with pytest.raises(EditOuterError, match="before the capture"):
                h.step_layer_ortho(0, o, theta, b, reps)
        graph.replay()
        torch.cuda.synchronize()
        assert mark.tolist() == [1.0] * 4
        assert all(torch.equal(x, y) for x, y in zip(fixed, eager))
        h.step_layer_ortho(0, o, theta, b, reps)
        h2.step_layer_ortho(0, full, eager[0], eager[1], eager[2:])
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=torch.cuda.Stream(DEV)):
            h.step_layer_ortho(0, o, theta, b, reps)
        for replay in range(3):
            for j, r in enumerate(reps):
                r.add_(_randn(numel, 50 + 2 * replay + j, 1e-3).to(r.dtype))
            for src, dst in zip(fixed, eager):
                dst.copy_(src)
            h2.step_layer_ortho(0, full, eager[0], eager[1], eager[2:])
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(x, y) for x, y in zip(fixed, eager)), f"replay {replay}"


def test_calls_after_a_failed_init():
    """A workspace that does not fit is refused, and that is all: later calls are as before."""
    numel, mats = layout(SHAPES[1])
    x = _randn(numel, 31).to(torch.bfloat16)
    with _ortho(numel, mats) as o:
        want = o.orthogonalize(x)
        for make in (lambda: _ortho(2 ** 42, mats),  # 16 TiB
                     lambda: EditOuter(OuterConfig(2, [2 ** 38] * 4000, "bf16", flags=ONE_PASS), DEV)):
            with pytest.raises(EditOuterError, match="out of memory"):
                make()
            assert torch.equal(o.orthogonalize(x), want)
            assert float(torch.ones(8, device=DEV).sum()) == 8.0


def test_layouts_beyond_a_launch_are_refused():
    """More tiles than a launch takes are refused at init, not in the middle of a step."""
    long = 2 ** 24
    with pytest.raises(EditOuterError, match="too many") as e:
        _ortho(32 * long, [(k * long, long, 1) for k in range(32)])
    assert e.value.status == EDIT_EINVAL


@pytest.mark.skipif(torch.cuda.device_count() < 2, reason="needs two devices")
def test_destroy_beside_another_current_device():
    """The workspace is released behind its own device's work, and the current device stays."""
    numel, mats = layout([(2000, 2000)])
    x = _randn(numel, 32).to(torch.bfloat16)
    with _ortho(numel, mats) as o:
        want = o.orthogonalize(x)
    out = torch.empty_like(x)
    o = _ortho(numel, mats)
    with torch.cuda.device(1):
        o.orthogonalize(x, out)
        o._lib.edit_ortho_destroy(o._h)
        o._h = None
        assert torch.cuda.current_device() == 1
    torch.cuda.synchronize(DEV)
    assert torch.equal(out, want)
