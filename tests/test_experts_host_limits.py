"""What the operators of a Dense Part made of experts check on the host before anything runs, where lists and devices go wrong."""
import itertools
import random

import pytest
import torch

from paper_1806_03925_amd import binding as b, experts


@pytest.mark.parametrize("src,dst,shared", [
    ([(0, 8), (8, 8)], [(0, 8), (8, 8)], False),            # in place, neighbours
    ([(0, 8), (0, 8)], [(0, 8), (0, 8)], True),             # a tensor twice, in place
    ([(0, 8), (0, 8)], [(64, 8), (72, 8)], False),          # a tensor twice, scaled into two others
    ([(0, 8), (16, 8)], [(64, 8), (64, 8)], True),          # two results in one place
    ([(0, 8), (16, 8)], [(64, 8), (71, 8)], True),
    ([(0, 8), (16, 8)], [(16, 8), (0, 8)], True),           # in one another's place
    ([(0, 8), (16, 8)], [(64, 8), (0, 8)], True),           # one result in another's source
    ([(0, 8)], [(4, 8)], True),                             # shifted against its own source
    ([(0, 0), (0, 8), (4, 0)], [(0, 0), (0, 8), (4, 0)], False),   # tensors without elements are nowhere
    ([], [], False)])
def test_memory_that_gradients_share(src, dst, shared):
    assert experts._share_memory(src, dst) is shared


def test_memory_that_gradients_share_against_every_pair():
    rng = random.Random(5)
    seen = set()
    for _ in range(3000):
        n = rng.randint(1, 5)
        size = [rng.randint(0, 4) for _ in range(n)]
        src = [(rng.randint(0, 30), s) for s in size]
        dst = [a if rng.random() < 0.6 else (rng.randint(0, 60), a[1]) for a in src]
        meet = lambda a, b: set(range(a[0], sum(a))) & set(range(b[0], sum(b)))
        want = any(meet(a, b) for a, b in itertools.combinations(dst, 2))
        want = want or any(meet(s, d) and not (i == j and s == d) for i, s in enumerate(src) for j, d in enumerate(dst))
        assert experts._share_memory(src, dst) is bool(want), (src, dst)
        seen.add(bool(want))
    assert seen == {True, False}


# ---- tensors of several GPUs: stand-ins without memory that say which GPU they are on -----------------------------------------
PLACES = itertools.count(1 << 20, 1 << 16)


class OnGpu(torch.Tensor):
    gpu = 0
    is_cuda = True
    device = property(lambda t: torch.device("cuda", t.gpu))
    get_device = lambda t: t.gpu
    data_ptr = lambda t: t.at


def on(gpu, *shape, dtype=torch.bfloat16):
    t = torch.empty(shape, dtype=dtype, device="meta").as_subclass(OnGpu)
    t.gpu, t.at = gpu, next(PLACES)
    return t


class NothingRuns:
    def __getattr__(self, name):
        raise AssertionError(f"{name} was called")


def expert_weights(gpu, kind=experts.ExpertWeights):
    w = object.__new__(kind)
    w.experts, w.N, w.K, w.dtype, w.code, w.gpu = 2, 72, 64, torch.bfloat16, b.GEAR_BF16, gpu
    w.address = w.forward = w.transposed = w.p_scale = w.p_status = 1 << 20
    return w


def rows8(gpu, dim=64):
    return experts.Rows8(on(gpu, 4, 128, dtype=torch.uint8), on(gpu, 4, 4, dtype=torch.uint8), dim)


F32, I32 = torch.float32, torch.int32
MOVED = {   # call -> its tensors: each of them on the other GPU once, all others on this one
    "rmsnorm": (dict(x=lambda d: on(d, 4, 64), gain=lambda d: on(d, 64, dtype=F32), residual=lambda d: on(d, 4, 64), sum=lambda d: on(d, 4, 64),
                     y=lambda d: on(d, 4, 64), rows8=rows8),
                lambda x, gain, residual, sum, y, rows8: experts.gear_rmsnorm(x, gain, 1e-6, residual, True, True, experts.NormOutput(sum, y, rows8))),
    "backward": (dict(h=lambda d: on(d, 4, 64), gain=lambda d: on(d, 64, dtype=F32), dy=lambda d: on(d, 4, 64), dsum=lambda d: on(d, 4, 64),
                      dx=lambda d: on(d, 4, 64), dgain=lambda d: on(d, 64, dtype=F32)),
                 lambda h, gain, dy, dsum, dx, dgain: experts.gear_rmsnorm_backward(h, gain, dy, 1e-6, dsum, dx, dgain)),
    "rows8": (dict(x=lambda d: on(d, 4, 64), out=rows8), lambda x, out: experts.gear_rows8(x, out)),
    "matmul8": (dict(r=rows8, w=lambda d: expert_weights(d, experts.Weights8), off=lambda d: on(d, 3, dtype=I32), out=lambda d: on(d, 4, 72),
                     status=lambda d: on(d, 1, dtype=I32)),
                lambda r, w, off, out, status: experts.gear_matmul8(r, w, off, out, status=status)),
    "matmul": (dict(x=lambda d: on(d, 4, 64), w=expert_weights, off=lambda d: on(d, 3, dtype=I32), out=lambda d: on(d, 4, 72),
                    status=lambda d: on(d, 1, dtype=I32)),
               lambda x, w, off, out, status: experts.gear_expert_matmul(x, w, off, out, status=status)),
    "dgrad": (dict(dy=lambda d: on(d, 4, 72), w=expert_weights, off=lambda d: on(d, 3, dtype=I32), out=lambda d: on(d, 4, 64),
                   status=lambda d: on(d, 1, dtype=I32)),
              lambda dy, w, off, out, status: experts.gear_expert_dgrad(dy, w, off, out, status=status)),
    "wgrad": (dict(dy=lambda d: on(d, 4, 72), x=lambda d: on(d, 4, 64), off=lambda d: on(d, 3, dtype=I32), dw=lambda d: on(d, 2, 72, 64, dtype=F32),
                   status=lambda d: on(d, 1, dtype=I32)),
              lambda dy, x, off, dw, status: experts.gear_expert_wgrad(dy, x, off, dw, status)),
    "update": (dict(w=lambda d: on(d, 2, 72, 64), weights=expert_weights), lambda w, weights: weights.update(w)),
    "list": (dict(g=lambda d: on(d, 8), h=lambda d: on(d, 8), o=lambda d: on(d, 8), p=lambda d: on(d, 8)),
             lambda g, h, o, p: experts.GradList([g, h], [o, p])),
}


@pytest.mark.parametrize("call,moved", [(c, m) for c, (tensors, _) in MOVED.items() for m in tensors])
def test_tensors_of_several_gpus_are_refused(monkeypatch, call, moved):
    monkeypatch.setattr(experts, "lib", NothingRuns())
    monkeypatch.setattr(experts, "_current_gpu", lambda: 0, raising=False)
    tensors, run = MOVED[call]
    with pytest.raises(b.GearError) as e:
        run(**{name: make(int(name == moved)) for name, make in tensors.items()})
    assert e.value.code == b.GEAR_ERR_INVALID


@pytest.mark.parametrize("call", MOVED)
def test_tensors_of_a_gpu_that_is_not_the_current_one_are_refused(monkeypatch, call):
    """Kernels are launched on the current GPU: neither its streams nor its memory are those of the tensors."""
    monkeypatch.setattr(experts, "lib", NothingRuns())
    monkeypatch.setattr(experts, "_current_gpu", lambda: 0, raising=False)
    tensors, run = MOVED[call]
    with pytest.raises(b.GearError) as e:
        run(**{name: make(1) for name, make in tensors.items()})
    assert e.value.code == b.GEAR_ERR_INVALID


@pytest.mark.parametrize("call", MOVED)
def test_tensors_of_one_gpu_are_taken(monkeypatch, call):
    """The stand-ins above are refused for where they are and nothing else."""
    monkeypatch.setattr(experts, "lib", NothingRuns())
    monkeypatch.setattr(experts, "_current_gpu", lambda: 0, raising=False)
    tensors, run = MOVED[call]
    with pytest.raises(AssertionError, match="was called"):
        run(**{name: make(0) for name, make in tensors.items()})


@pytest.mark.parametrize("call", [
    lambda: experts.gear_expert_wgrad(on(0, 4, 72), on(0, 4, 64), on(0, 0, dtype=I32)),             # no offset at all
    lambda: experts.gear_expert_wgrad(on(0, 4, 72), on(0, 4, 64), on(0, 1, dtype=I32)),             # of no expert
    lambda: experts.gear_expert_wgrad(on(0), on(0, 4, 64)),
    lambda: experts.gear_expert_wgrad(on(0, 4, 72), on(0)),
    lambda: experts.gear_expert_matmul(on(0), expert_weights(0), on(0, 3, dtype=I32)),
    lambda: experts.gear_expert_dgrad(on(0), expert_weights(0), on(0, 3, dtype=I32)),
    lambda: experts.gear_rmsnorm(on(0), on(0, 64, dtype=F32), 1e-6),
    lambda: experts.gear_rmsnorm_backward(on(0), on(0, 64, dtype=F32), on(0), 1e-6),
    lambda: experts.gear_rows8(on(0)),
    lambda: experts.gear_weights8(on(0)),
    lambda: experts.Rows8(on(0, dtype=torch.uint8), on(0, dtype=torch.uint8), 64)])
def test_tensors_without_dimensions_and_lists_without_entries(monkeypatch, call):
    monkeypatch.setattr(experts, "lib", NothingRuns())
    monkeypatch.setattr(experts, "_current_gpu", lambda: 0)
    with pytest.raises(b.GearError) as e:
        call()
    assert e.value.code == b.GEAR_ERR_INVALID


def test_a_first_report_is_not_made_while_a_graph_is_captured(monkeypatch):
    """The word would belong to the graph, and be cleared by its replays: a call that needs it says so, one with a status of its own does not
    need it, nor one without offsets."""
    monkeypatch.setattr(experts, "lib", NothingRuns())
    monkeypatch.setattr(experts, "_current_gpu", lambda: 0)
    monkeypatch.setattr(experts, "_words", {})
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: True)
    x, dy, off, status = on(0, 4, 64), on(0, 4, 72), on(0, 3, dtype=I32), on(0, 1, dtype=I32)
    out, dw, weights = on(0, 4, 72), on(0, 2, 72, 64, dtype=F32), expert_weights(0)
    for call in (lambda: experts.gear_expert_matmul(x, weights, off, out), lambda: experts.gear_expert_wgrad(dy, x, off, dw)):
        with pytest.raises(b.GearError) as e:
            call()
        assert e.value.code == b.GEAR_ERR_INVALID
    weights.experts = 1
    for call in (lambda: experts.gear_expert_matmul(x, weights, None, out), lambda: experts.gear_expert_wgrad(dy, x, off, dw, status)):
        with pytest.raises(AssertionError, match="was called"):
            call()
    weights.experts = 2
    with pytest.raises(AssertionError, match="was called"):
        experts.gear_expert_matmul(x, weights, off, out, status=status)
