"""AdamW on the GPU as programs meet it: parameters whose gradients come and go, states, autograd, refused handles."""
import io

import pytest

torch = pytest.importorskip("torch")

from lm_check import within  # noqa: E402
from paper_2310_12298_amd import lm  # noqa: E402
from paper_2310_12298_amd.optim import AdamWOptimizer  # noqa: E402
from test_gpu_lm_adamw import BF16, F32, HP, flat, formula, tensors  # noqa: E402

pytestmark = pytest.mark.gpu

SIZES = [300, 5, 1000, 257, 64]
# Which tensors have a gradient at each step: the second's come late, the third's every other time, the fourth's once.
GIVEN = [(0, 4), (0, 2, 4), (0, 4), (0, 1, 2, 4), (0, 1, 4), (), (0, 1, 2, 3, 4), (1, 3)]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("bits", [32, 8])
def test_each_parameter_counts_its_own_steps(bits, dtype):
    params = tensors(SIZES, dtype)
    opt, taken = lm.AdamW(params, bits=bits, seed=3), [0] * len(SIZES)
    for k, given in enumerate(GIVEN):
        grads = [g if i in given else None for i, g in enumerate(tensors(SIZES, dtype, seed=k + 1, scale=0.1))]
        old = [p.clone() for p in params]
        p, g = flat(opt, params), flat(opt, [torch.zeros_like(q) if x is None else x for q, x in zip(params, grads)])
        m, v = (x.double().cpu() for x in opt.moment_values())
        opt.step(grads, **HP)
        after = [x.double().cpu() for x in opt.moment_values()]
        for i, b in enumerate(opt.blocks[:-1]):
            s = slice(b * lm.BLOCK, b * lm.BLOCK + SIZES[i])
            if i in given:
                taken[i] += 1
                p1, _, _, _, _, size = formula(p[s], g[s], m[s], v[s], taken[i], **HP)
                within(params[i], p1, size, 24, f"step {k}, parameter {i}")
            else:
                assert torch.equal(params[i], old[i])
                assert torch.equal(after[0][s], m[s]) and torch.equal(after[1][s], v[s])
        assert opt.steps == taken and opt.t == max(taken)


def test_optimizer_agrees_with_torch_where_gradients_come_late():
    def make():
        torch.manual_seed(1)
        return [torch.nn.Parameter(torch.randn(n, device="cuda")) for n in SIZES]
    a, b = make(), make()
    opt = AdamWOptimizer([{"params": a[:3]}, {"params": a[3:]}], lr=1e-2, weight_decay=0.1, max_norm=1.0)
    ref = torch.optim.AdamW([{"params": b[:3]}, {"params": b[3:]}], lr=1e-2, weight_decay=0.1)
    for k, given in enumerate(GIVEN):
        for i, (p, q) in enumerate(zip(a, b)):
            gen = torch.Generator(device="cuda").manual_seed(10 * k + i)
            p.grad = torch.randn(p.shape, generator=gen, device="cuda") if i in given else None
            q.grad = None if p.grad is None else p.grad.clone()
        opt.step()
        torch.nn.utils.clip_grad_norm_(b, 1.0)
        ref.step()
        for p, q in zip(a, b):
            assert torch.allclose(p, q, rtol=1e-5, atol=1e-6)


@pytest.mark.parametrize("bits", [32, 8])
def test_counts_of_steps_are_part_of_the_state(bits):
    params = tensors(SIZES, F32)
    opt = lm.AdamW(params, bits=bits, seed=3)

    def step(o, k, given):
        o.step([g if i in given else None for i, g in enumerate(tensors(SIZES, F32, seed=k))], **HP)
    step(opt, 1, (0, 1))
    step(opt, 2, (0, 4))
    buf = io.BytesIO()
    torch.save(opt.state_dict(), buf)
    buf.seek(0)
    twin = lm.AdamW([p.clone() for p in params], bits=bits)
    twin.load_state_dict(torch.load(buf, weights_only=True))
    assert twin.steps == [2, 1, 0, 0, 1] and twin.t == 2
    for o in (opt, twin):
        step(o, 3, (0, 1, 2, 3, 4))
    for x, y in zip(opt.params, twin.params):
        assert torch.equal(x, y)
    old = opt.state_dict()
    del old["steps"]                                          # a state that holds one count for all
    twin.load_state_dict(old)
    assert twin.steps == [3] * 5
    short = opt.state_dict()
    short["steps"] = short["steps"][:4]
    with pytest.raises(ValueError):
        twin.load_state_dict(short)


def test_a_step_without_any_gradient_checks_and_changes_nothing():
    params = tensors(SIZES, F32)
    opt, old = lm.AdamW(params), [p.clone() for p in params]
    opt.step([None] * len(SIZES), **HP)
    with pytest.raises(lm.JorgeError):
        opt.step([None] * len(SIZES), lr=-1.0)
    assert opt.t == 0 and all(torch.equal(x, y) for x, y in zip(params, old))


@pytest.mark.parametrize("optimizer", [False, True])
def test_a_step_between_forward_and_backward_is_noticed(optimizer):
    w, u = (torch.nn.Parameter(torch.randn(8, 8, device="cuda")) for _ in range(2))
    x = torch.randn(8, 8, device="cuda", requires_grad=True)
    opt = AdamWOptimizer([w, u]) if optimizer else lm.AdamW([w, u])
    loss, other = (x @ w).square().sum(), (x @ u).square().sum()
    w.grad, before = torch.ones_like(w), (w._version, u._version)
    opt.step()
    assert w._version > before[0] and u._version == before[1]
    other.backward()                                          # u had no gradient and stands as it was
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        loss.backward()


def test_parameters_made_in_inference_mode_are_stepped():
    with torch.inference_mode():
        p = torch.ones(300, device="cuda")
    opt = lm.AdamW([p])
    opt.step([torch.ones(300, device="cuda")], lr=0.5, weight_decay=0.0)
    assert bool((p == 0.5).all())


@pytest.mark.parametrize("bits", [32, 8])
def test_a_captured_step_warns_and_repeats_its_own_step(bits):
    g = tensors([700], F32, seed=1)
    a, b = (lm.AdamW(tensors([700], F32), bits=bits) for _ in range(2))
    for o in (a, b):
        o.step(g, **HP)
    graph = torch.cuda.CUDAGraph()
    with pytest.warns(UserWarning, match="every replay"):
        with torch.cuda.graph(graph):
            a.step(g, **HP)
    for _ in range(4):
        graph.replay()
        b.t = 1
        b.step(g, **HP)
        torch.cuda.synchronize()
        assert torch.equal(a.params[0], b.params[0])
        assert all(torch.equal(x, y) for x, y in zip(a.moments.values(), b.moments.values()))


def test_8_bit_moments_past_two_to_the_31_elements_are_read_and_written():
    """More blocks than a launch takes (2^24) too: 2^24 + 70 of them, and the values around every boundary."""
    blocks = (1 << 24) + 70
    n, last = blocks * lm.BLOCK, lm.BLOCK * 200
    opt = lm.AdamW([torch.empty(n, dtype=BF16, device="cuda")], bits=8)
    g = torch.Generator(device="cuda").manual_seed(0)
    for k in opt.moments:
        code = opt.moments[k]
        code[-last:] = torch.randint(1, 200, (min(last, code.numel()),), generator=g, device="cuda").to(torch.uint8)[
            :code[-last:].numel()]
    few = lm.AdamW([torch.empty(last, dtype=BF16, device="cuda")], bits=8, moments={
        k: x[-(last if x.numel() == n else 200):].clone() for k, x in opt.moments.items()})
    for x, y in zip(opt.moment_values(BF16), few.moment_values(BF16)):
        assert torch.equal(x[-last:], y) and not bool(x[:-last].view(torch.int32).any())
    del x, y
    values = [x.clone() for x in few.moment_values()]
    values[0] *= -1
    wide = torch.zeros(n, device="cuda")
    both = []
    for v in values:
        wide[-last:] = v
        both.append(wide.clone() if not both else wide)
    opt.set_moment_values(*both)
    few.set_moment_values(*values)
    for k, x in opt.moments.items():
        end = last if x.numel() == n else 200
        assert torch.equal(x[-end:], few.moments[k])
    del wide, both
    assert all(torch.equal(x[-last:], y) for x, y in zip(opt.moment_values(BF16), few.moment_values(BF16)))


@pytest.mark.parametrize("bits", [32, 8])
def test_moment_values_stay_as_they_were_read(bits):
    opt = lm.AdamW(tensors(SIZES, F32), bits=bits)
    opt.step(tensors(SIZES, F32, seed=1), **HP)
    read = opt.moment_values()
    kept = [x.clone() for x in read]
    opt.step(tensors(SIZES, F32, seed=2), **HP)
    assert all(torch.equal(x, y) for x, y in zip(read, kept))
    assert not torch.equal(opt.moment_values()[0], kept[0])


def test_a_refused_state_changes_nothing():
    opt = lm.AdamW(tensors(SIZES, F32), bits=8, seed=4)
    opt.step(tensors(SIZES, F32, seed=1), **HP)
    good = opt.state_dict()
    twin = lm.AdamW(tensors(SIZES, F32), bits=8)
    for change in ({"t": None}, {"t": -1}, {"seed": None}, {"seed": 1 << 32}, {"exp_avg_sq": None}, {"steps": [1] * 4},
                   {"steps": [1, 1, 1, 1, -1]}, {"exp_avg_scale": good["exp_avg_scale"][1:]}, {"bits": 32}):
        bad = {k: v for k, v in {**good, **change}.items() if v is not None}
        with pytest.raises(ValueError):
            twin.load_state_dict(bad)
        assert twin.t == 0 and twin.seed == 0 and not any(bool(x.any()) for x in twin.moments.values())
    twin.load_state_dict(good)
    assert twin.t == 1 and twin.seed == 4 and all(torch.equal(opt.moments[k], x) for k, x in twin.moments.items())
    twin.load_state_dict({k: v.long() if torch.is_tensor(v) else v for k, v in good.items()})   # the same bytes
    assert all(torch.equal(opt.moments[k], x) for k, x in twin.moments.items())


def test_a_state_that_one_group_refuses_changes_no_group():
    def make(sizes):
        ps = [torch.nn.Parameter(p) for p in tensors(sizes, F32)]
        return AdamWOptimizer([{"params": ps[:1]}, {"params": ps[1:], "lr": 0.5}], lr=0.25)
    a, b = make([30, 600]), make([30, 300])
    for g in a.param_groups:
        g["lr"] = 0.125
        for p in g["params"]:
            p.grad = torch.ones_like(p)
    a.step()
    with pytest.raises(ValueError):
        b.load_state_dict(a.state_dict())
    assert [g["lr"] for g in b.param_groups] == [0.25, 0.5]
    assert all(h.t == 0 and not any(bool(x.any()) for x in h.moments.values()) for h in b._handles)


def test_parameters_that_share_memory_are_refused():
    hold = tensors([1000], F32)[0]
    for params in ([hold, hold], [hold[:600], hold[599:]], [hold[10:20], hold.view(10, 100)]):
        with pytest.raises(ValueError, match="share memory"):
            lm.AdamW(params)
    lm.AdamW([hold[600:], hold[:0], hold[:600], hold[600:600]])
    q = torch.nn.Parameter(tensors([8], F32)[0])
    with pytest.warns(UserWarning), pytest.raises(ValueError, match="share memory"):
        AdamWOptimizer([q, q])


@pytest.mark.parametrize("bits", [32, 8])
def test_refused_moment_values_change_nothing(bits):
    opt = lm.AdamW(tensors(SIZES, F32), bits=bits)
    n = opt.moments["exp_avg"].numel()
    ones = torch.ones(n, device="cuda")
    for bad in (ones[1:], ones.bfloat16(), ones.cpu(), None):
        with pytest.raises(ValueError):
            opt.set_moment_values(ones, bad)
        assert not any(bool(x.any()) for x in opt.moments.values())
    opt.set_moment_values(ones, ones)
    assert all(torch.equal(x, ones) for x in opt.moment_values())
