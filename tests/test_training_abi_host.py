"""Host-only checks of the calls of scoring and training: every refusal comes before anything could reach a device, and
the plan's layout is what the kernels are handed."""
import ctypes
import struct

import pytest

from paper_2306_08162_amd import binding as ql

FAKE, ODD = 0x10000, 0x10008        # never dereferenced: validation fails first
E = {n: i for i, n in enumerate(ql.STATUS_NAMES)}


def _score(z=FAKE, stride=64, tok=FAKE, lp=FAKE, ent=FAKE, at=FAKE, alp=FAKE, k=5, stats=FAKE, M=4, V=64, dtype=0, ws=FAKE,
           wsb=1 << 30):
    return ql.qlora_token_logprobs(z, stride, tok, lp, ent, at, alp, k, stats, M, V, dtype, ws, wsb, stream=0, check=False)


@pytest.mark.parametrize("change,status", [
    (dict(M=0), "SHAPE"), (dict(V=0), "SHAPE"), (dict(M=-1), "SHAPE"), (dict(M=1 << 22), "SHAPE"),
    (dict(M=1 << 20, V=1 << 15, stride=1 << 15), "SHAPE"), (dict(dtype=3), "DTYPE"), (dict(dtype=-1), "DTYPE"),
    (dict(stride=63), "VALUE"), (dict(stride=-64), "VALUE"), (dict(stride=1 << 40), "VALUE"), (dict(stride=1 << 62), "VALUE"),
    (dict(k=-1), "VALUE"), (dict(k=65), "VALUE"),
    (dict(z=None), "NULL"), (dict(tok=None), "NULL"), (dict(at=None), "NULL"), (dict(alp=None), "NULL"),
    (dict(lp=None, ent=None, stats=None, k=0), "NULL"),
    (dict(z=0x10001), "ALIGN"), (dict(z=0x10002, dtype=2), "ALIGN"), (dict(stats=ODD), "ALIGN"), (dict(ws=ODD), "ALIGN"),
    (dict(tok=0x10002), "ALIGN"), (dict(V=(1 << 28) + 1, M=1, stride=1 << 29), "SHAPE"),
    (dict(lp=0x10002), "ALIGN"), (dict(ent=0x10001), "ALIGN"), (dict(at=0x10002), "ALIGN"), (dict(alp=0x10002), "ALIGN"),
    (dict(V=1 << 20, stride=1 << 20, ws=None), "WORKSPACE"), (dict(V=1 << 20, stride=1 << 20, wsb=64), "WORKSPACE"),
])
def test_token_logprobs_refusals(change, status):
    assert _score(**change) == E["QLORA_E_" + status]


def test_token_logprobs_workspace():
    size = ql.qlora_token_logprobs_workspace_bytes
    assert size(0, 100, 0, 0) == size(4, 0, 0, 0) == size(4, 100, 65, 0) == size(4, 100, 0, 3) == 0
    assert size(2048, 32000, 20, 0) == 0                            # whole rows: none
    assert size(3, 1 << 20, 20, 0) >= 3 * 32 * (16 + 8 * 20)        # a MiB-token row is 32 segments at least


@pytest.mark.parametrize("change,status", [
    (dict(M=0), "SHAPE"), (dict(V=0), "SHAPE"), (dict(dtype=3), "DTYPE"), (dict(stride=63), "VALUE"), (dict(ds=63), "VALUE"),
    (dict(z=None), "NULL"), (dict(stats=None), "NULL"), (dict(dz=None), "NULL"), (dict(g=None, h=None), "NULL"),
    (dict(tok=None), "NULL"), (dict(z=0x10001), "ALIGN"), (dict(dz=0x20001), "ALIGN"), (dict(stats=ODD), "ALIGN"),
    (dict(dz=0x20002, dtype=2), "ALIGN"),
    (dict(g=0x10002), "ALIGN"), (dict(h=0x10002), "ALIGN"), (dict(tok=0x10002), "ALIGN"), (dict(dz=FAKE, ds=65), "VALUE"),
])
def test_token_logprobs_bwd_refusals(change, status):
    a = dict(z=FAKE, stride=64, tok=FAKE, stats=FAKE, g=FAKE, h=FAKE, dz=0x20000, ds=64, M=4, V=64, dtype=0) | change
    assert ql.qlora_token_logprobs_bwd(a["z"], a["stride"], a["tok"], a["stats"], a["g"], a["h"], a["dz"], a["ds"], a["M"],
                                       a["V"], a["dtype"], stream=0, check=False) == E["QLORA_E_" + status]


def _tensor(at=0x100000, n=1000, **over):
    """Buffers 1 MiB apart from one another."""
    names = ("param", "grad", "master", "exp_avg", "exp_avg_sq", "avg_scale", "avg_sq_scale")
    t = ql.OptimTensorStruct(**{name: at + (i << 20) for i, name in enumerate(names)}, numel=n, lr_scale=1.0,
                             weight_decay=0.0, param_dtype=0, grad_dtype=2, state_bits=8)
    for k, v in over.items():
        setattr(t, k, v)
    return t


@pytest.mark.parametrize("change,status", [
    (dict(numel=-1), "SHAPE"), (dict(numel=(1 << 36) + 1), "SHAPE"), (dict(numel=0), "SHAPE"), (dict(grad=None), "NULL"),
    (dict(exp_avg=None), "NULL"), (dict(exp_avg_sq=None), "NULL"), (dict(avg_scale=None), "NULL"),
    (dict(avg_sq_scale=None), "NULL"), (dict(param_dtype=3), "DTYPE"), (dict(grad_dtype=-1), "DTYPE"),
    (dict(param_dtype=2), "DTYPE"), (dict(state_bits=16), "BITS"), (dict(param=0x100008), "ALIGN"),
    (dict(grad=0x200004), "ALIGN"), (dict(master=0x300008), "ALIGN"), (dict(exp_avg=0x400001), "ALIGN"),
    (dict(avg_scale=0x600002), "ALIGN"), (dict(lr_scale=-1.0), "VALUE"), (dict(lr_scale=float("nan")), "VALUE"),
    (dict(weight_decay=float("inf")), "VALUE"), (dict(weight_decay=-0.1), "VALUE"),
    (dict(exp_avg=0x500000 + 992), "PLAN"), (dict(param=0x200000 + 3984), "PLAN"), (dict(master=0x100000), "PLAN"),
])
def test_plan_refusals(change, status):
    assert ql.qlora_optim_plan([_tensor(**change)], check=False)[1] == E["QLORA_E_" + status]


def test_plan_refuses_a_tensor_twice_and_takes_shared_gradients():
    a, b = _tensor(), _tensor(at=0x100000)
    assert ql.qlora_optim_plan([a, b], check=False)[1] == E["QLORA_E_PLAN"]
    b = _tensor(at=0x4000000, grad=0x200000)                        # one gradient for two tensors: only read
    assert ql.qlora_optim_plan([a, b], check=False)[1] == 0
    b = _tensor(at=0x4000000, param=0x200000)                       # ... but not a gradient that another tensor's step overwrites
    assert ql.qlora_optim_plan([a, b], check=False)[1] == E["QLORA_E_PLAN"]


def test_plan_layout():
    tensors = [_tensor(at=0x10000000 * (i + 1), n=n, lr_scale=2.0 + i) for i, n in enumerate((1, 4096, 0, 4097, 300))]
    plan, st = ql.qlora_optim_plan(tensors, check=False)
    assert st == 0
    assert ql.qlora_optim_plan_bytes(tensors) == 64 + 80 * 7 == len(plan.raw)
    magic, nbytes, weights, count, chunks, steppable = struct.unpack_from("<QQQIII", plan.raw)
    assert (nbytes, weights, count, chunks, steppable) == (len(plan.raw), 1 + 4096 + 4097 + 300, 5, 7, 1)
    got = [struct.unpack_from("<7QIIffBBBB", plan.raw, 64 + 80 * c) for c in range(7)]
    # (tensor, first weight, weights, place in the plan): tensors begin at whole blocks of 256
    for rec, (i, begin, n, place) in zip(got, [(0, 0, 1, 0), (1, 0, 2048, 256), (1, 2048, 2048, 2304), (3, 0, 2048, 4352),
                                               (3, 2048, 2048, 6400), (3, 4096, 1, 8448), (4, 0, 300, 8704)]):
        t = tensors[i]
        assert rec[7:10] == (n, place, 2.0 + i) and rec[11:14] == (0, 2, 8)
        assert rec[:7] == (t.param + 2 * begin, t.grad + 4 * begin, t.master + 4 * begin, t.exp_avg + begin,
                           t.exp_avg_sq + begin, t.avg_scale + begin // 64, t.avg_sq_scale + begin // 64)


def test_plan_bytes_of_nothing():
    assert ql.qlora_optim_plan_bytes([]) == 0
    assert ql.qlora_optim_plan_bytes([_tensor(n=0)]) == 0
    lib = ql.load()
    t = _tensor()
    buf = ctypes.create_string_buffer(4096)
    need = ql.qlora_optim_plan_bytes([t])
    assert lib.qlora_optim_plan(1, ctypes.byref(t), buf, need - 1) == E["QLORA_E_WORKSPACE"]
    assert lib.qlora_optim_plan(1, ctypes.byref(t), None, need) == E["QLORA_E_NULL"]
    assert lib.qlora_optim_plan(1, None, buf, need) == E["QLORA_E_NULL"]
    assert lib.qlora_optim_plan(0, ctypes.byref(t), buf, need) == E["QLORA_E_SHAPE"]


@pytest.mark.parametrize("change,status", [
    (dict(plan=None), "NULL"), (dict(device=None), "NULL"), (dict(control=None), "NULL"), (dict(device=ODD), "ALIGN"),
    (dict(control=ODD), "ALIGN"), (dict(ws=ODD), "ALIGN"), (dict(ws=None), "WORKSPACE"), (dict(wsb=100), "WORKSPACE"),
    (dict(beta1=1.0), "VALUE"), (dict(beta1=-0.1), "VALUE"), (dict(beta2=float("nan")), "VALUE"), (dict(eps=-1.0), "VALUE"),
    (dict(eps=float("inf")), "VALUE"), (dict(clip=-1.0), "VALUE"), (dict(clip=float("nan")), "VALUE"),
])
def test_step_refusals(change, status):
    a = dict(plan=ql.qlora_optim_plan([_tensor()]), device=FAKE, control=FAKE, beta1=0.9, beta2=0.999, eps=1e-8, clip=1.0,
             ws=FAKE, wsb=1 << 20) | change
    assert ql.qlora_adamw_step(a["plan"], a["device"], a["control"], a["beta1"], a["beta2"], a["eps"], a["clip"], a["ws"],
                               a["wsb"], stream=0, check=False) == E["QLORA_E_" + status]


@pytest.mark.parametrize("eps", [0.0, 1e-45, 2.0 ** -127, 1e39, float("nan")])
def test_step_refuses_an_eps_that_fp32_does_not_hold(eps):
    """With none (or one that the division flushes) a weight without a gradient, as A's are while B is 0, would become NaN."""
    plan = ql.qlora_optim_plan([_tensor()])
    assert ql.qlora_adamw_step(plan, FAKE, FAKE, 0.9, 0.999, eps, 0.0, None, stream=0, check=False) == E["QLORA_E_VALUE"]


def test_step_refuses_other_plans():
    step = lambda plan: ql.qlora_adamw_step(plan, FAKE, FAKE, 0.9, 0.999, 1e-8, 0.0, None, stream=0, check=False)
    assert step(ctypes.create_string_buffer(4096)) == E["QLORA_E_PLAN"]
    gradients_only = ql.qlora_optim_plan([_tensor(), _tensor(at=0x4000000, param=None)])
    assert step(gradients_only) == E["QLORA_E_PLAN"]
    norm = lambda **kw: ql.qlora_grad_norm(*(kw | {}).values(), stream=0, check=False)
    base = dict(plan=gradients_only, device=FAKE, scale=1.0, norm=FAKE, ws=FAKE, wsb=1 << 20)
    for change, status in ((dict(plan=ctypes.create_string_buffer(64)), "PLAN"), (dict(norm=None), "NULL"),
                           (dict(norm=0x10002), "ALIGN"), (dict(ws=None), "WORKSPACE"), (dict(wsb=8), "WORKSPACE"),
                           (dict(device=None), "NULL")):
        assert norm(**(base | change)) == E["QLORA_E_" + status], change


def test_control_block():
    c = ql.qlora_optim_control_init(1e-3, 0.5, 77, 3, 0.9, 0.99)
    assert (c.lr, c.grad_scale, c.seed, c.step, c.skipped) == (pytest.approx(1e-3), 0.5, 77, 3, 0)
    assert c.beta1_power == pytest.approx(0.729) and c.beta2_power == pytest.approx(0.99 ** 3)
    assert ctypes.sizeof(c) == 64
    for bad in ((1e-3, 1.0, 0, -1, 0.9, 0.99), (1e-3, 1.0, 0, 0, 1.0, 0.99), (1e-3, 1.0, 0, 0, 0.9, -0.5)):
        assert ql.qlora_optim_control_init(*bad, check=False)[1] == E["QLORA_E_VALUE"]


def test_new_status_strings():
    texts = [ql.status_string(i) for i in range(len(ql.STATUS_NAMES))]
    assert len(set(texts)) == len(texts) and "unknown status" not in texts


def test_optimizer_refuses_tensors_in_host_memory():
    import torch
    from paper_2306_08162_amd.device import AdapterOptimizer, OptimTensor
    with pytest.raises(ValueError):
        AdapterOptimizer([OptimTensor(torch.zeros(8), torch.zeros(8))], lr=1e-3)


@pytest.mark.parametrize("V,dtype", [(100000, 0), (128259, 1), (65537, 0), (40000, 2), (50257, 2), (1 << 20, 0), (32000, 0)])
def test_token_logprobs_workspace_of_a_batch_serves_its_smaller_ones(V, dtype):
    """Never less for more rows or alternatives, none for one number of rows and some for another."""
    sizes = [[ql.qlora_token_logprobs_workspace_bytes(M, V, k, dtype) for M in range(1, 700)] for k in (0, 5, 64)]
    for row in sizes:
        assert all(a <= b for a, b in zip(row, row[1:])) and len({n == 0 for n in row}) == 1
    assert all(a <= b <= c for a, b, c in zip(*sizes))


def _tensors(M=4, V=64, k=5):
    import torch
    f32 = lambda *shape: torch.zeros(shape)
    return dict(z=torch.zeros((M, V), dtype=torch.float16), tok=torch.zeros(M, dtype=torch.int32), lp=f32(M), ent=f32(M),
                at=torch.zeros((M, k), dtype=torch.int32), alp=f32(M, k), stats=f32(M, 4), ws=torch.zeros(64, dtype=torch.uint8))


@pytest.mark.parametrize("name,dtype", [("tok", "int64"), ("lp", "float16"), ("ent", "float64"), ("at", "int64"), ("alp", "bfloat16"),
                                        ("stats", "float16"), ("z", "bfloat16"), ("z", "float32"), ("z", "uint8"), ("z", "int32")])
def test_token_logprobs_refuses_tensors_of_other_types(name, dtype):
    import torch
    t = _tensors()
    t[name] = t[name].to(getattr(torch, dtype))
    with pytest.raises(ValueError, match="holds torch." + dtype):
        _score(**{name: t[name]})


@pytest.mark.parametrize("name", ["tok", "lp", "ent", "at", "alp", "stats", "z"])
def test_token_logprobs_refuses_tensors_that_are_too_short(name):
    t = _tensors()
    short = t[name].flatten()[1:].clone()
    with pytest.raises(ValueError, match="entries|ends before"):
        _score(**{name: short})
    with pytest.raises(ValueError, match="current GPU"):            # one entry further back in memory that is long enough
        _score(**{name: t[name].flatten()[:-1]})


def test_token_logprobs_refuses_rows_that_pass_the_end():
    import torch
    t = _tensors()
    with pytest.raises(ValueError, match="ends before"):
        _score(z=t["z"], stride=65)
    wide = torch.zeros((4, 70), dtype=torch.float16)[:, :64]        # ... and takes a slice, 16-bit patterns as integers
    for z in (wide, wide.view(torch.int16)):
        with pytest.raises(ValueError, match="current GPU"):
            _score(z=z, stride=70)
    with pytest.raises(ValueError, match="a row must be contiguous"):
        _score(z=torch.zeros((64, 4), dtype=torch.float16).T)


@pytest.mark.parametrize("keep", ["z", "tok", "lp", "ent", "at", "alp", "stats", "ws"])
def test_token_logprobs_refuses_tensors_in_host_memory(keep):
    with pytest.raises(ValueError, match="current GPU"):
        _score(**{keep: _tensors()[keep]})


def test_token_logprobs_ignores_what_is_not_asked_for():
    """Tokens beside no logprob, alternatives beside a count of 0: not looked at, so the refusal is that of the workspace."""
    import torch
    wrong = torch.zeros(1, dtype=torch.int64)
    a = dict(V=1 << 20, stride=1 << 20, ws=None)
    assert _score(tok=wrong, lp=None, **a) == E["QLORA_E_WORKSPACE"]
    assert _score(at=wrong, alp=wrong, k=0, **a) == E["QLORA_E_WORKSPACE"]


@pytest.mark.parametrize("name,dtype", [("tok", "int64"), ("stats", "float64"), ("g", "float16"), ("h", "float64"), ("z", "float32"),
                                        ("dz", "bfloat16")])
def test_token_logprobs_bwd_refuses_tensors_that_do_not_fit(name, dtype):
    import torch
    M, V = 4, 64
    t = dict(z=torch.zeros((M, V), dtype=torch.float16), tok=torch.zeros(M, dtype=torch.int32), stats=torch.zeros((M, 4)),
             g=torch.zeros(M), h=torch.zeros(M), dz=torch.zeros((M, V), dtype=torch.float16))
    fake = dict(z=FAKE, tok=FAKE, stats=FAKE, g=FAKE, h=FAKE, dz=0x20000)
    call = lambda a: ql.qlora_token_logprobs_bwd(a["z"], V, a["tok"], a["stats"], a["g"], a["h"], a["dz"], V, M, V, ql.QLORA_F16,
                                                 stream=0, check=False)
    with pytest.raises(ValueError, match="holds torch." + dtype):
        call(fake | {name: t[name].to(getattr(torch, dtype))})
    with pytest.raises(ValueError, match="entries|ends before"):
        call(fake | {name: t[name].flatten()[1:].clone()})
    with pytest.raises(ValueError, match="current GPU"):
        call(fake | {name: t[name]})
