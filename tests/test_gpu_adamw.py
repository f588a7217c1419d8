"""GPU parity of qlora_adamw_step and qlora_grad_norm against the oracle (oracle/adamw.py).

Tolerances.  States of 32 bits: a moment is two products and a sum, each rounded (u = 2^-24), on a gradient that was
rounded once or twice before: |error| <= 4 u (|b m| + |c g|), and 5 u v for the second.  Weights: the update lr m / (sqrt v + eps)
carries a dozen roundings and two hardware approximations of one unit (2^-23): within 32 u of its size, plus one rounding
of the decay and one of the sum (2 u |w|), plus half a unit of a 16-bit weight.  States of 8 bits are compared with
the same arithmetic done in fp32 and the documented rounding: equal codes, save where the hardware's square root (one unit
in 2^23 off) carries a value over the step that the 20 random bits define: 2^-23 of the value is at most 2^-23 * 16 * 2^20 =
2 of those steps in the coarsest place, so about 2 in 2^20 codes of sqrt(v) differ; 8 + n / 2^17 are allowed."""
import numpy as np
import pytest

import oracle
from oracle import adamw as ref
from paper_2306_08162_amd import binding as ql
from paper_2306_08162_amd import workloads as wl
from parity import announce, small_inputs

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
HALF_ULP = {"f16": 2.0 ** -11, "bf16": 2.0 ** -8, "f32": 2.0 ** -24}
SIZES = (1, 3, 4, 255, 256, 257, 1023, 4095, 4096, 4097, 12289, 33000, 2)


def _torch(dtype):
    import torch
    return {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32, "u8": torch.uint8}[dtype]


class _Set:
    """Tensors of all sizes in one allocation a kind, 64 entries of 77 behind each."""

    def __init__(self, seed, sizes=SIZES, param="f16", grad="f32", bits=32, master=False, spread=1e-3):
        import torch
        self.sizes, self.param, self.grad, self.bits, self.has_master = sizes, param, grad, bits, master
        self.seed, self.spread = seed, spread
        self.at, total = [], 0
        for n in sizes:
            self.at.append(total)
            total += (n + 255) // 256 * 256 + 256
        self.total = total
        full = lambda dtype, fill=77: torch.full((total,), fill, dtype=_torch(dtype), device="cuda:0")
        state = "u8" if bits == 8 else "f32"
        self.buf = {"param": full(param), "grad": full(grad), "exp_avg": full(state), "exp_avg_sq": full(state)}
        if master:
            self.buf["master"] = full("f32")
        if bits == 8:
            for n in ("avg_scale", "avg_sq_scale"):
                self.buf[n] = torch.full((total // 256,), 77.0, device="cuda:0")
        self.lr_scale = [1.0, 4.0, 0.0, 0.5][:]
        self.decay = [0.0, 0.1, 0.01]
        for i in range(len(sizes)):
            w = wl.normal(seed + 10 * i, sizes[i])
            self.put("param", i, w)
            if master:
                self.put("master", i, w)
            for n in ("exp_avg", "exp_avg_sq", "avg_scale", "avg_sq_scale"):
                if n in self.buf:
                    self.put(n, i, np.zeros(self.length(n, i)))
        self.gradient(0)
        self.start = {n: b.clone() for n, b in self.buf.items()}

    def length(self, name, i):
        return -(-self.sizes[i] // 256) if name.endswith("scale") else self.sizes[i]

    def view(self, name, i):
        at = self.at[i] // (256 if name.endswith("scale") else 1)
        return self.buf[name][at:at + self.length(name, i)]

    def put(self, name, i, values):
        import torch
        self.view(name, i).copy_(torch.from_numpy(np.ascontiguousarray(values)).to("cuda:0"))

    def get(self, name, i):
        return self.view(name, i).double().cpu().numpy() if not (self.bits == 8 and name in ("exp_avg", "exp_avg_sq")) \
            else self.view(name, i).cpu().numpy()

    def gradient(self, t):
        for i, n in enumerate(self.sizes):
            g = wl.normal(self.seed + 1000 * (t + 1) + i, n) * self.spread * 10.0 ** (i % 4 - 2)
            self.put("grad", i, g)

    def hyper(self, i):
        return self.lr_scale[i % 4], self.decay[i % 3]

    def optimizer(self, **kw):
        from paper_2306_08162_amd.device import AdapterOptimizer, OptimTensor
        ts = []
        for i in range(len(self.sizes)):
            part = lambda n: self.view(n, i) if n in self.buf else None
            ts.append(OptimTensor(part("param"), part("grad"), part("master"), part("exp_avg"), part("exp_avg_sq"),
                                  part("avg_scale"), part("avg_sq_scale"), *self.hyper(i)))
        return AdapterOptimizer(ts, **kw)

    def untouched_between(self):
        """What lies behind each tensor still holds 77."""
        for name, b in self.buf.items():
            unit = 256 if name.endswith("scale") else 1
            inside = np.zeros(len(b), bool)
            for i in range(len(self.sizes)):
                inside[self.at[i] // unit:self.at[i] // unit + self.length(name, i)] = True
            rest = b.double().cpu().numpy()[~inside]
            assert (rest == 77).all(), f"{name}: entries behind a tensor were written"


def _norm(s, scale):
    return np.sqrt(sum(float((s.get("grad", i) ** 2).sum()) for i in range(len(s.sizes)))) * scale


KINDS = [  # param, grad, bits, master, guarded
    ("f16", "f32", 32, False, False), ("bf16", "f32", 32, False, True), ("f32", "f32", 32, False, True),
    ("f16", "f32", 32, True, True), ("bf16", "bf16", 32, True, False), ("f16", "f16", 32, False, False),
    ("f32", "f16", 32, False, True), ("f32", "bf16", 32, False, False),
]


@pytest.mark.parametrize("param,grad,bits,master,guarded", KINDS)
def test_three_steps_with_states_of_32_bits(param, grad, bits, master, guarded):
    announce(f"adamw param={param} grad={grad} master={master} guarded={guarded}")
    s = _Set(7, param=param, grad=grad, master=master)
    lr, eps, scale, b1, b2 = 1e-2, 1e-8, 0.25, 0.9, 0.98
    max_norm = 0.6 * _norm(s, scale) if guarded else 0.0
    opt = s.optimizer(lr=lr, betas=(b1, b2), eps=eps, max_grad_norm=max_norm, grad_scale=scale)
    for t in range(1, 4):
        s.gradient(t)
        norm = _norm(s, scale)
        before = [{n: s.get(n, i) for n in s.buf} for i in range(len(s.sizes))]
        opt.step()
        clip = min(1.0, max_norm / norm) if guarded else 1.0
        if guarded:
            assert abs(float(opt.last_grad_norm) - norm) <= 2 * U * norm
        for i, old in enumerate(before):
            ratio, wd = s.hyper(i)
            g = old["grad"] * scale * clip
            w0 = old["master" if master else "param"]
            w, m, v = ref.step(w0, old["exp_avg"], old["exp_avg_sq"], g, lr=lr * ratio, beta1=b1, beta2=b2, eps=eps,
                               weight_decay=wd, t=t)
            assert np.all(np.abs(s.get("exp_avg", i) - m) <= 4 * U * (np.abs(b1 * old["exp_avg"]) + np.abs(g)) + 1e-38)
            assert np.all(np.abs(s.get("exp_avg_sq", i) - v) <= 6 * U * v + 1e-38)
            update = np.abs(w - w0 * (1 - lr * ratio * wd))
            # the moments' own errors enter the update relative to what they were summed from
            spread = lr * ratio / (1 - b1 ** t) * (np.abs(b1 * old["exp_avg"]) + np.abs((1 - b1) * g)) / (
                np.sqrt(v / (1 - b2 ** t)) + eps)
            bound = 32 * U * (update + spread) + 3 * U * np.abs(w0)
            if master:
                assert np.all(np.abs(s.get("master", i) - w) <= bound)
            half = HALF_ULP[param] * np.abs(w) + 2.0 ** -25
            assert np.all(np.abs(s.get("param", i) - w) <= bound * 1.01 + half)
    assert int(opt.steps_taken) == 3 and int(opt.steps_skipped) == 0
    s.untouched_between()


@pytest.mark.parametrize("param,grad,master,guarded", [("bf16", "f32", False, True), ("f16", "f32", True, False),
                                                       ("f32", "f32", False, False), ("bf16", "bf16", True, True)])
def test_four_steps_with_states_of_8_bits(param, grad, master, guarded):
    announce(f"adamw 8 bits param={param} grad={grad} master={master} guarded={guarded}")
    s = _Set(11, param=param, grad=grad, master=master, bits=8)
    lr, eps, scale, b1, b2, seed = 1e-2, 1e-8, 0.5, 0.9, 0.999, 1234
    max_norm = 1e3 if guarded else 0.0                              # guarded, and never clipped
    opt = s.optimizer(lr=lr, betas=(b1, b2), eps=eps, max_grad_norm=max_norm, grad_scale=scale, seed=seed)
    first = np.cumsum([0] + [-(-n // 256) for n in s.sizes])
    codes_off = 0
    for t in range(1, 5):
        s.gradient(t)
        before = [{n: s.get(n, i) for n in s.buf} for i in range(len(s.sizes))]
        opt.step()
        for i, old in enumerate(before):
            ratio, wd = s.hyper(i)
            f = np.float32
            g = old["grad"].astype(f) * f(scale)
            m0 = ref.decode(old["exp_avg"], old["avg_scale"]).astype(f)
            u0 = ref.decode(old["exp_avg_sq"], old["avg_sq_scale"]).astype(f)
            m, v = ref.moments_f32(m0, u0 * u0, g, b1, b2)
            words = ref.random_words(seed, t, int(first[i]), s.sizes[i])
            mc, uc, ms, us = ref.states8(m, v, words)
            np.testing.assert_array_equal(s.get("avg_scale", i), ms)
            np.testing.assert_array_equal(s.get("avg_sq_scale", i), us)
            np.testing.assert_array_equal(s.get("exp_avg", i), mc)
            off = s.get("exp_avg_sq", i).astype(int) - uc
            assert np.all(np.abs(off) <= 1)
            codes_off += int((off != 0).sum())
            w0 = old["master" if master else "param"]
            w, _, _ = ref.step(w0, m0, u0.astype(float) ** 2, g, lr=lr * ratio, beta1=b1, beta2=b2, eps=eps, weight_decay=wd, t=t)
            spread = lr * ratio / (1 - b1 ** t) * (np.abs(b1 * m0) + np.abs((1 - b1) * g)) / (
                np.sqrt(v.astype(float) / (1 - b2 ** t)) + eps)
            bound = 64 * U * spread + 3 * U * np.abs(w0) + HALF_ULP[param] * np.abs(w) * 1.01 + 2.0 ** -25
            assert np.all(np.abs(s.get("param", i) - w) <= bound)
    assert codes_off <= 8 + 4 * sum(s.sizes) / 2 ** 17
    s.untouched_between()


def test_small_second_moments_decay():
    """No gradient for 300 steps, beta2 = 0.99: sqrt(v) has to fall to 0.99^150 of its start on average.  Rounded to the
    nearest code it would not move at all (a step takes off half a percent, two codes are six percent apart)."""
    import torch
    announce("adamw 8 bits, decay of the second moment")
    n, steps = 64 * 256, 300
    s = _Set(3, sizes=(n,), bits=8, spread=1.0)
    s.put("grad", 0, np.full(n, 2.0))
    opt = s.optimizer(lr=0.0, betas=(0.9, 0.99), seed=5)
    opt.step()
    root = ref.decode(s.get("exp_avg_sq", 0), s.get("avg_sq_scale", 0))
    start = root.mean()
    s.put("grad", 0, np.zeros(n))
    for _ in range(steps):
        opt.step()
    root = ref.decode(s.get("exp_avg_sq", 0), s.get("avg_sq_scale", 0))
    # Each rounding keeps the mean of sqrt(v); one weight's relative variance grows by at most (1/8)^2 / 4 a step in units of
    # the value, but only with the probability that a step of half a percent moves a code: 0.005 / (1/16..1/8) of that,
    # so after 300 steps its spread is below sqrt(300 * 0.005 * 0.125) = 0.43, the mean's over 16384 weights 0.0034: six of those
    assert abs(root.mean() / (start * 0.99 ** (steps / 2)) - 1) <= 6 * 0.0034
    assert (s.get("exp_avg_sq", 0) > 0).all()


def test_zero_and_tiny_second_moments():
    """A block of zeros keeps zeros and a scale of 0; in a block of one large and many tiny gradients every code of a second
    moment above zero stays above zero, and no update is larger than the ratio of the moments allows."""
    announce("adamw 8 bits, zeros and tiny moments")
    n = 768
    s = _Set(4, sizes=(n,), param="f32", bits=8)
    g = np.zeros(n)
    g[256:512] = 1e-9
    g[300] = 1.0
    s.put("grad", 0, g)
    s.put("param", 0, np.zeros(n))
    opt = s.optimizer(lr=1.0, seed=9)
    for _ in range(30):
        opt.step()
        s.put("grad", 0, g * 0)
    codes, scale = s.get("exp_avg_sq", 0), s.get("avg_sq_scale", 0)
    assert (codes[:256] == 0).all() and (codes[512:] == 0).all() and scale[0] == scale[2] == 0
    assert (codes[256:512] > 0).all()
    w = s.get("param", 0)
    assert (w[:256] == 0).all() and np.isfinite(w).all()
    # Of exact moments |m| / sqrt v <= (1 - b1) / sqrt((1 - b2) (1 - b1^2 / b2)) = 7.28, and the bias corrections,
    # sqrt(1 - b2^t) / (1 - b1^t) <= 0.32 (t = 1), leave less of it.  Of the tiny weights both codes are at most the lowest but
    # one here: m <= 2^-9 of a scale of 2^-12, sqrt v >= 2^-9 of 2^-13, a ratio of 2.  30 steps of at most 7.3 are more than either.
    assert np.abs(w).max() < 30 * 7.3


@pytest.mark.parametrize("bits", [8, 32])
@pytest.mark.parametrize("bad", [np.inf, -np.inf, np.nan])
def test_steps_on_gradients_that_overflowed_are_not_taken(bits, bad):
    import torch
    announce(f"adamw skipped step bits={bits} {bad}")
    s = _Set(21, bits=bits, master=True)
    opt = s.optimizer(lr=1e-2, max_grad_norm=np.inf, seed=3)
    s.gradient(1)
    opt.step()
    kept = {n: b.clone() for n, b in s.buf.items()}
    s.view("grad", 9)[4095] = bad
    opt.step()
    assert not np.isfinite(float(opt.last_grad_norm)) and int(opt.steps_taken) == 1 and int(opt.steps_skipped) == 1
    for n, b in s.buf.items():
        if n != "grad":
            assert torch.equal(b, kept[n]), n
    # the next step is the second one, as if nothing had been in between
    s.gradient(2)
    opt.step()
    once = {n: b.clone() for n, b in s.buf.items()}
    for n, b in s.buf.items():
        b.copy_(s.start[n])
    fresh = s.optimizer(lr=1e-2, max_grad_norm=np.inf, seed=3)
    for t in (1, 2):
        s.gradient(t)
        fresh.step()
    for n, b in s.buf.items():
        assert torch.equal(b, once[n]), n
    assert int(opt.steps_taken) == 2


@pytest.mark.parametrize("bits", [8, 32])
def test_gradients_whose_squares_leave_fp32(bits):
    """A gradient of 1e20: without clipping the step is not taken, clipped to a norm of 1 it is."""
    import torch
    announce(f"adamw large gradients bits={bits}")
    s = _Set(23, sizes=(600, 300), param="f32", bits=bits)
    s.view("grad", 0)[300] = 1e20
    kept = {n: b.clone() for n, b in s.buf.items()}
    opt = s.optimizer(lr=1e-2, max_grad_norm=np.inf)
    opt.step()
    assert (int(opt.steps_taken), int(opt.steps_skipped)) == (0, 1) and abs(float(opt.last_grad_norm) / 1e20 - 1) < 1e-6
    assert all(torch.equal(b, kept[n]) for n, b in s.buf.items())
    opt = s.optimizer(lr=1e-2, max_grad_norm=1.0)
    opt.step()
    assert (int(opt.steps_taken), int(opt.steps_skipped)) == (1, 0)
    for n in ("param", "exp_avg_sq"):
        assert all(np.isfinite(s.get(n, i)).all() for i in range(2)), n
    # g = 1: the first step is lr (1 - b) / sqrt(1 - b2) / (its bias correction) = lr, after the weight's own decay (0.0)
    assert abs(s.get("param", 0)[300] - (kept["param"][s.at[0] + 300].item() - 1e-2)) <= 64 * U


def test_unguarded_steps_keep_the_damage_where_it_is():
    announce("adamw unguarded, not finite")
    for bits in (32, 8):
        s = _Set(22, sizes=(1000, 700), bits=bits, param="f32")
        s.view("grad", 0)[300] = float("inf")
        s.view("grad", 0)[700] = float("nan")
        s.optimizer(lr=1e-2).step()
        w = s.get("param", 0)
        assert np.isnan(w[300]) and np.isnan(w[700]) and np.isfinite(np.delete(w, [300, 700])).all()
        assert np.isfinite(s.get("param", 1)).all()
        if bits == 8:
            assert list(np.isnan(s.get("avg_scale", 0))) == [False, True, True, False]
            assert list(np.isnan(s.get("avg_sq_scale", 0))) == [False, True, True, False]
            assert np.isfinite(s.get("avg_scale", 1)).all()


@pytest.mark.parametrize("grad", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("size", [1e-3, 1e30, 1e-30])
def test_norm(grad, size):
    import torch
    from paper_2306_08162_amd.device import AdapterOptimizer, OptimTensor
    if grad == "f16" and size != 1e-3:
        pytest.skip("outside the type")
    announce(f"grad norm {grad} {size}")
    s = _Set(31, sizes=SIZES + (0, 100003), grad=grad, spread=size)
    opt = AdapterOptimizer([OptimTensor(None, s.view("grad", i)) for i in range(len(s.sizes))], lr=0.0)
    out = torch.full((1,), 5.0, device="cuda:0")
    for scale in (1.0, 2.0 ** -14, -0.37):
        opt.grad_norm(out, scale)
        # summed in 64 bits (relative 2^-40 at most), the factor as fp32, the result rounded once
        assert abs(float(out) - _norm(s, abs(float(np.float32(scale))))) <= 1.01 * U * float(out)
    s.view("grad", 5)[7] = float("nan")
    opt.grad_norm(out)
    assert np.isnan(float(out))


@pytest.mark.parametrize("bits", [8, 32])
def test_smallest_eps_without_a_gradient(bits):
    announce(f"adamw eps 2^-126 bits={bits}")
    s = _Set(34, param="f32", bits=bits)
    for i in range(len(s.sizes)):
        s.put("grad", i, np.zeros(s.sizes[i]))
    before = [s.get("param", i) for i in range(len(s.sizes))]
    s.optimizer(lr=1.0, eps=2.0 ** -126).step()
    for i, w in enumerate(before):
        ratio, wd = s.hyper(i)
        assert np.all(np.abs(s.get("param", i) - w * (1 - ratio * wd)) <= 3 * U * np.abs(w))


def test_no_gradient_at_all():
    announce("adamw zero gradients, clipped")
    s = _Set(33, param="f32")
    for i in range(len(s.sizes)):
        s.put("grad", i, np.zeros(s.sizes[i]))
    opt = s.optimizer(lr=1e-2, max_grad_norm=1.0)
    before = [s.get("param", i) for i in range(len(s.sizes))]
    opt.step()
    assert float(opt.last_grad_norm) == 0 and int(opt.steps_taken) == 1
    for i, w in enumerate(before):
        ratio, wd = s.hyper(i)
        assert np.all(np.abs(s.get("param", i) - w * (1 - 1e-2 * ratio * wd)) <= 3 * U * np.abs(w))


@pytest.mark.parametrize("bits", [8, 32])
def test_five_hundred_tensors_twice_give_the_same_bits(bits):
    import torch
    announce(f"adamw 500 tensors bits={bits}")
    sizes = tuple(1 + (i * 7919) % 3000 for i in range(500))
    runs = []
    for _ in range(2):
        s = _Set(41, sizes=sizes, bits=bits, param="bf16")
        opt = s.optimizer(lr=1e-2, max_grad_norm=0.5, seed=8)
        for t in range(3):
            s.view("grad", t).mul_(2)
            opt.step()
        runs.append({n: b.clone() for n, b in s.buf.items()} | {"norm": opt.last_grad_norm.clone()})
        s.untouched_between()
    for n in runs[0]:
        assert torch.equal(runs[0][n], runs[1][n]), n


@pytest.mark.parametrize("bits", [8, 32])
def test_graph_replays_match_eager(bits):
    """A captured step is replayed with new gradients and a new rate each time; the step count lives on the device."""
    import torch
    announce(f"adamw graph bits={bits}")
    eager, captured = (_Set(51, bits=bits, master=True, param="bf16") for _ in range(2))
    kw = dict(lr=1e-2, max_grad_norm=0.02, seed=6)
    a, b = eager.optimizer(**kw), captured.optimizer(**kw)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        b.step()
    for rep in range(6):
        for s, opt in ((eager, a), (captured, b)):
            s.gradient(rep)
            if rep == 3:
                s.view("grad", 4)[0] = float("inf")
            opt.lr.fill_(1e-2 / (1 + rep))
        a.step()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for n in eager.buf:
            assert torch.equal(eager.buf[n], captured.buf[n]), f"replay {rep}: {n}"
        assert torch.equal(a.control, b.control)
    assert int(b.steps_taken) == 5 and int(b.steps_skipped) == 1


@pytest.mark.parametrize("bits", [8, 32])
def test_small_and_large_plans_take_the_same_step(bits):
    """Without clipping: 128 chunks of a plan are one launch, 129 are two; the tensors of both and the control block agree."""
    import torch
    announce(f"adamw 128 and 129 chunks bits={bits}")
    sizes = (2048 * 120 + 7, 300, 2048 * 5 + 1)
    one, two = _Set(71, sizes=sizes, param="bf16", bits=bits), _Set(71, sizes=sizes + (5,), param="bf16", bits=bits)
    kw = dict(lr=1e-2, betas=(0.9, 0.99), seed=5)
    a, b = one.optimizer(**kw), two.optimizer(**kw)
    assert [ql.qlora_optim_plan_bytes([o._describe(t) for t in o.tensors]) for o in (a, b)] == [64 + 80 * 128, 64 + 80 * 129]
    for t in range(5):
        for s, o in ((one, a), (two, b)):
            s.gradient(t)
            o.step()
        assert torch.equal(a.control, b.control), t
        for n in one.buf:
            for i in range(len(sizes)):
                assert torch.equal(one.view(n, i), two.view(n, i)), (t, n, i)
    assert int(a.steps_taken) == 5
    one.untouched_between()
    two.untouched_between()


@pytest.mark.parametrize("bits", [8, 32])
def test_graph_replays_of_a_small_step_match_eager(bits):
    import torch
    announce(f"adamw graph of one launch bits={bits}")
    eager, captured = (_Set(52, bits=bits, param="f16") for _ in range(2))
    a, b = eager.optimizer(lr=1e-2, seed=6), captured.optimizer(lr=1e-2, seed=6)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        b.step()
        b.step()
    for t in range(6):
        for s, o in ((eager, a), (captured, b)):
            s.gradient(t)
            o.lr.fill_(1e-2 / (t + 1))
        a.step()
        a.step()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(a.control, b.control), t
        for n in eager.buf:
            assert torch.equal(eager.buf[n], captured.buf[n]), (t, n)
    assert int(b.steps_taken) == 12


def test_step_on_another_stream_and_refused_tensors():
    import torch
    from paper_2306_08162_amd.device import AdapterOptimizer, OptimTensor
    announce("adamw other stream, refusals")
    one, two = (_Set(61) for _ in range(2))
    one.optimizer(lr=1e-2, max_grad_norm=1.0).step()
    opt = two.optimizer(lr=1e-2, max_grad_norm=1.0)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    opt.step(stream=side)
    side.synchronize()
    assert torch.equal(one.buf["param"], two.buf["param"]) and torch.equal(one.buf["exp_avg_sq"], two.buf["exp_avg_sq"])
    t = lambda n, dtype=torch.float32: torch.zeros(n, dtype=dtype, device="cuda:0")
    for bad in (OptimTensor(t(8), t(9)), OptimTensor(t(8), t(8), exp_avg=t(8, torch.float16)), OptimTensor(t(8), t(8).cpu()),
                OptimTensor(t(8), t(8), exp_avg=t(7)), OptimTensor(t(8, torch.int16), t(8), param_dtype=ql.QLORA_F32),
                OptimTensor(t(512), t(512), state_bits=8, avg_scale=t(1)), OptimTensor(t(16)[::2], t(8))):
        with pytest.raises(ValueError):
            AdapterOptimizer([OptimTensor(t(4), t(4)), bad], lr=1e-3)
    with pytest.raises(ValueError):
        AdapterOptimizer([], lr=1e-3)
    with pytest.raises(ql.QLoraError):
        AdapterOptimizer([OptimTensor(t(8), t(8))], lr=1e-3, betas=(1.0, 0.9))
    w = t(64)
    with pytest.raises(ql.QLoraError):                              # the same weights twice
        AdapterOptimizer([OptimTensor(w, t(64)), OptimTensor(w, t(64))], lr=1e-3)


def test_states_it_allocates_are_ready_on_any_stream():
    """400 MB of states are cleared on the current stream; a step on another one right after finds zeros."""
    import torch
    from paper_2306_08162_amd.device import AdapterOptimizer, OptimTensor
    announce("adamw own states, other stream")
    n = 50_000_000
    dirty = [torch.full((n,), float("nan"), device="cuda:0") for _ in range(2)]   # what the allocator hands out again
    torch.cuda.synchronize()
    w, g, side = torch.zeros(n, device="cuda:0"), torch.ones(n, device="cuda:0"), torch.cuda.Stream()
    torch.cuda.synchronize()
    del dirty
    AdapterOptimizer([OptimTensor(w, g)], lr=0.5).step(stream=side)
    side.synchronize()
    # the first step is lr g / (|g| + eps): within the dozen roundings and two approximations of 32 u
    assert float((w + 0.5).abs().max()) <= 0.5 * 32 * U + 1e-8


def test_tensors_of_unknown_contents_and_norms_elsewhere_are_refused():
    import torch
    from paper_2306_08162_amd.device import AdapterOptimizer, OptimTensor
    announce("adamw refusals of types")
    t = lambda n, dtype=torch.float32: torch.zeros(n, dtype=dtype, device="cuda:0")
    for bad in (OptimTensor(t(8, torch.int16), t(8)), OptimTensor(t(8), t(8, torch.float64))):
        with pytest.raises(ValueError):
            AdapterOptimizer([bad], lr=1e-3)
    opt = AdapterOptimizer([OptimTensor(t(8), t(8))], lr=1e-3)
    for out in (t(1, torch.float64), t(0), t(1).cpu()):
        with pytest.raises(ValueError):
            opt.grad_norm(out)


def test_adapters_learn_from_token_scores():
    """The calls of a training step in a row: a quantized head with adapters makes logits, the tokens are scored, the gradient
    of their log probabilities goes back through the layer into dA and dB, and the optimizer moves A and B; every
    number on the way is held against the oracle on the values that the library itself handed on."""
    import torch
    from oracle import scoring
    from paper_2306_08162_amd.device import AdapterOptimizer, DeviceLayer, OptimTensor
    announce("token logprobs -> linear backward -> adamw")
    M, V = 48, 264
    inp = small_inputs(71, M, 256, V, 4, 64, 8, "bf16")
    layer = DeviceLayer(inp)
    c = layer.cfg
    tokens_h = (wl.splitmix64(72, 0, M) % np.uint64(V)).astype(np.int64)
    tokens = torch.from_numpy(tokens_h.astype(np.int32)).to("cuda:0")
    logprob, stats = torch.empty(M, device="cuda:0"), torch.empty((M, 4), device="cuda:0")
    g = torch.full((M,), -64.0 / M, device="cuda:0")                # the mean of -log p, under a loss scale of 64
    A, B = (torch.zeros_like(t).copy_(t) for t in (layer.A, layer.B))
    layer.A, layer.B = A, B
    opt = AdapterOptimizer([OptimTensor(A, layer.dA, param_dtype=ql.QLORA_BF16, state_bits=8, master=A.view(torch.bfloat16).float()),
                            OptimTensor(B, layer.dB, param_dtype=ql.QLORA_BF16, master=B.view(torch.bfloat16).float())],
                           lr=1e-2, max_grad_norm=1.0, grad_scale=1 / 64, seed=1)
    mA, mB = opt.tensors[0].master.view_as(A), opt.tensors[1].master.view_as(B)
    old = [(mA.double().cpu().numpy(), np.zeros(A.shape), np.zeros(A.shape)),
           (mB.double().cpu().numpy(), np.zeros(B.shape), np.zeros(B.shape))]
    for t in range(1, 4):
        layer.forward()
        ql.qlora_token_logprobs(layer.y, V, tokens, logprob, None, None, None, 0, stats, M, V, ql.QLORA_BF16, None)
        ql.qlora_token_logprobs_bwd(layer.y, V, tokens, stats, g, None, layer.dy, V, M, V, ql.QLORA_BF16)
        layer.backward()
        torch.cuda.synchronize()
        z = oracle.widen(layer.host_y(), "bf16")
        lp = scoring.score(z, tokens_h, 0)[0]
        np.testing.assert_allclose(logprob.cpu().numpy(), lp, atol=1e-5 * (1 + np.abs(lp).max()))
        dz = scoring.score_gradient(z, tokens_h, np.full(M, -64.0 / M), None)
        assert np.linalg.norm(oracle.widen(_host16(layer.dy), "bf16") - dz) <= 5e-3 * np.linalg.norm(dz)
        lo = oracle.LayerOracle(inp.codes, inp.scales, inp.zeros, _host16(A), _host16(B), bits=c.bits,
                                group_size=c.group_size, alpha=c.alpha, dtype=c.dtype)
        want = lo.backward_adapters(_host16(layer.dy), inp.x)
        grads = [layer.host_dA().astype(float), layer.host_dB().astype(float)]
        for got, w in zip(grads, want):
            assert np.linalg.norm(got - w) <= 5e-3 * np.linalg.norm(w)
        norm = np.sqrt(sum((a ** 2).sum() for a in grads)) / 64
        opt.step()
        assert abs(float(opt.last_grad_norm) - norm) <= 1e-6 * norm
        for i, (param, master) in enumerate(((A, mA), (B, mB))):
            w, m, v = old[i]
            if i == 0 and t > 1:                                    # the 8-bit states as they were stored
                m = ref.decode(stored[0], stored[1]).reshape(w.shape)
                v = ref.decode(stored[2], stored[3]).reshape(w.shape) ** 2
            w, m, v = ref.step(w, m, v, grads[i] / 64 * min(1.0, 1.0 / norm), lr=1e-2, beta1=0.9, beta2=0.999, eps=1e-8,
                               weight_decay=0.0, t=t)
            got = master.double().cpu().numpy()
            np.testing.assert_allclose(got, w, atol=1e-2 * 1e-4 + 4 * U * np.abs(w).max())
            assert np.array_equal(param.view(torch.bfloat16).float().cpu().numpy(), master.bfloat16().float().cpu().numpy())
            old[i] = (got, m, v)
        o = opt.tensors[0]
        stored = [x.cpu().numpy() for x in (o.exp_avg, o.avg_scale, o.exp_avg_sq, o.avg_sq_scale)]
    assert int(opt.steps_taken) == 3


def _host16(t):
    return t.cpu().numpy().view(np.uint16)


def test_tensor_of_more_than_two_to_the_31_weights():
    """Offsets that pass 32 bits: bf16 weights and gradients with 8-bit states, gradients at both ends and at 2^31."""
    import torch
    from paper_2306_08162_amd.device import AdapterOptimizer, OptimTensor
    announce("adamw, one tensor of 2^31 + 5001 weights")
    n = 2 ** 31 + 5001
    new = lambda size, t: torch.zeros(size, dtype=t, device="cuda:0")
    w, g = new(n, torch.bfloat16), new(n, torch.bfloat16)
    places = [slice(0, 300), slice(2 ** 31 - 5, 2 ** 31 + 7), slice(n - 300, n)]
    for s in places:
        g[s] = 0.5
    opt = AdapterOptimizer([OptimTensor(w, g, state_bits=8)], lr=1e-2, max_grad_norm=1e3)
    opt.step()
    count = sum(s.stop - s.start for s in places)
    assert abs(float(opt.last_grad_norm) - 0.5 * np.sqrt(count)) <= 2 * U * 0.5 * np.sqrt(count)
    for s in places:                     # a first step moves each weight by lr against its gradient
        assert (w[s].float() + 1e-2).abs().max() <= 1e-2 * 2 ** -8
    moved = 0
    for at in range(0, n, 2 ** 28):      # ... and no other weight
        moved += int((w[at:at + 2 ** 28] != 0).sum())
    assert moved == count
    assert int((opt.tensors[0].exp_avg[n - 300:] != 0).sum()) == 300 and int((opt.tensors[0].exp_avg_sq[:300] != 0).sum()) == 300


def test_a_norm_and_a_step_share_no_scratch(monkeypatch):
    """A norm for a log line may run beside a step on another stream: the partial sums of the two lie apart."""
    import torch
    from paper_2306_08162_amd.device import AdapterOptimizer, OptimTensor
    announce("adamw scratch of norm and step")
    t = lambda n: torch.zeros(n, device="cuda:0")
    opt = AdapterOptimizer([OptimTensor(t(8), t(8))], lr=1e-3, max_grad_norm=1.0)
    seen = {}
    monkeypatch.setattr(ql, "qlora_adamw_step", lambda *a, **kw: seen.__setitem__("step", a[-2:]))
    monkeypatch.setattr(ql, "qlora_grad_norm", lambda *a, **kw: seen.__setitem__("norm", a[-2:]))
    opt.step()
    opt.grad_norm(t(1))
    (a, na), (b, nb) = seen["step"], seen["norm"]
    need = ql.qlora_optim_workspace_bytes()
    assert min(na, nb) >= need and (a + need <= b or b + need <= a)


def test_norms_beside_steps_on_another_stream():
    import torch
    announce("adamw norm on one stream, steps on another")
    alone, both = (_Set(91, sizes=(300000, 70001, 5), param="bf16") for _ in range(2))
    kw = dict(lr=1e-2, max_grad_norm=0.05, seed=2)
    a, b = alone.optimizer(**kw), both.optimizer(**kw)
    outs = [torch.zeros(1, device="cuda:0") for _ in range(20)]
    torch.cuda.synchronize()
    one, two = torch.cuda.Stream(), torch.cuda.Stream()
    for out in outs:
        a.step()
        b.step(stream=one)
        b.grad_norm(out, 0.5, stream=two)
    torch.cuda.synchronize()
    assert torch.equal(a.control, b.control)
    for n in alone.buf:
        assert torch.equal(alone.buf[n], both.buf[n]), n
    norm = _norm(alone, 0.5)
    assert all(abs(float(out) - norm) <= 1.01 * U * norm for out in outs)


@pytest.mark.parametrize("bits", [8, 32])
def test_second_moments_below_the_normal_numbers(bits):
    """Gradients of 1.5e-19 to 3e-19: v lies below 2^-126, its root does not, and with a tiny eps the update is lr as for
    any other gradient."""
    announce(f"adamw tiny second moments bits={bits}")
    sizes = (1000, 4097)
    s = _Set(81, sizes=sizes, param="f32", bits=bits)
    lr, eps, b1, b2, seed = 1e-2, 1e-30, 0.9, 0.98, 17
    opt = s.optimizer(lr=lr, betas=(b1, b2), eps=eps, seed=seed)
    first, codes_off = [0, 4], 0
    for t in range(1, 4):
        for i, n in enumerate(sizes):
            x = wl.normal(900 + 10 * t + i, n)
            s.put("grad", i, np.sign(x) * (1.5e-19 + 1.5e-19 * (np.abs(x) % 1.0)))
        before = [{n: s.get(n, i) for n in s.buf} for i in range(len(sizes))]
        opt.step()
        for i, old in enumerate(before):
            ratio, wd = s.hyper(i)
            f = np.float32
            g = old["grad"].astype(f)
            if bits == 8:
                m0 = ref.decode(old["exp_avg"], old["avg_scale"]).astype(f)
                u0 = ref.decode(old["exp_avg_sq"], old["avg_sq_scale"]).astype(f)
                v0 = u0 * u0
                m, v = ref.moments_f32(m0, v0, g, b1, b2)
                mc, uc, ms, us = ref.states8(m, v, ref.random_words(seed, t, first[i], sizes[i]))
                np.testing.assert_array_equal(s.get("avg_scale", i), ms)
                np.testing.assert_array_equal(s.get("avg_sq_scale", i), us)
                np.testing.assert_array_equal(s.get("exp_avg", i), mc)
                off = s.get("exp_avg_sq", i).astype(int) - uc
                assert np.all(np.abs(off) <= 1)
                codes_off += int((off != 0).sum())
            else:
                m0, v0 = old["exp_avg"], old["exp_avg_sq"]
            w, m, v = ref.step(old["param"], m0, v0, g, lr=lr * ratio, beta1=b1, beta2=b2, eps=eps, weight_decay=wd, t=t)
            # Below 2^-126 a product is off by half a unit of 2^-149: v by two of them and by that of u0 u0 (8 bits)
            v_off = 2.0 ** -149 * 1.5 + 6 * U * v
            assert v.max() < 2.0 ** -126 and v.min() > 2.0 ** -132
            if bits == 32:
                assert np.all(np.abs(s.get("exp_avg_sq", i) - v) <= v_off)
            # ... the root by half of that relative to v; the rest as for ordinary gradients
            spread = lr * ratio / (1 - b1 ** t) * (np.abs(b1 * m0) + np.abs((1 - b1) * g)) / (np.sqrt(v / (1 - b2 ** t)) + eps)
            bound = (64 * U + 0.51 * v_off / v) * spread + 3 * U * np.abs(old["param"])
            assert np.all(np.abs(s.get("param", i) - w) <= bound)
    assert codes_off <= 8 + 3 * sum(sizes) / 2 ** 17
    s.untouched_between()
