"""GPU parity of qlora_token_logprobs and its gradient against the fp64 oracle (oracle/scoring.py).

Tolerances, by counting roundings (u = 2^-24).  A weight exp(z - m) carries one rounding of the difference, one of the
product with log2 e (both relative to its exponent x, so |x| u each in the weight) and one unit of the hardware's exp2; a sum
of a row passes at most 64 + 8 + 6 + 8 additions in a segment and 6 + a few more across segments.  So ln S is off
by at most (100 + 2 E|x|) u, with E|x| <= H + ln S under the softmax, the difference z - m by u |z - m|, and
    |logprob|: C u (1 + |z - m| + ln S),  |entropy|: C u (1 + H + ln S)  with C = 128
covers them.  A gradient entry p (g + h (log p + H)) adds the relative error of p, (2 |x| + 100) u, and one rounding to the
output type (half a unit in the last place, or half the smallest subnormal of fp16)."""
import numpy as np
import pytest

import oracle
from oracle import scoring
from paper_2306_08162_amd import binding as ql
from paper_2306_08162_amd import workloads as wl
from parity import announce

pytestmark = pytest.mark.gpu

C, U = 128.0, 2.0 ** -24
FLAG = {"f16": ql.QLORA_F16, "bf16": ql.QLORA_BF16, "f32": ql.QLORA_F32}
HALF_ULP = {"f16": 2.0 ** -11, "bf16": 2.0 ** -8, "f32": 2.0 ** -24}
TINY = {"f16": 2.0 ** -25, "bf16": 2.0 ** -126, "f32": 2.0 ** -126}


def _torch(dtype):
    import torch
    return {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}[dtype]


def _logits(seed, M, V, dtype, spread=2.5):
    """fp64 values that `dtype` holds exactly."""
    z = wl.normal(seed, M * V).reshape(M, V) * spread
    z[np.arange(M), (wl.splitmix64(seed + 1, 0, M) % np.uint64(V)).astype(np.int64)] += 12.0 * (np.arange(M) % 2)
    return _rounded(z, dtype)


def _rounded(z, dtype):
    import torch
    return torch.from_numpy(np.ascontiguousarray(z)).to(_torch(dtype)).double().numpy()


def _upload(z, dtype, pad, fill=0.0):
    import torch
    M, V = z.shape
    full = torch.full((M, V + pad), fill, dtype=_torch(dtype), device="cuda:0")
    full[:, :V] = torch.from_numpy(np.ascontiguousarray(z)).to("cuda:0").to(_torch(dtype))
    return full


class _Call:
    """Buffers of one problem, outputs filled with what no call writes."""

    def __init__(self, z, tokens, dtype, k, pad=0, stats=True):
        import torch
        self.z, self.tokens_h, self.dtype, self.k, self.pad = z, np.asarray(tokens), dtype, k, pad
        M, V = self.shape = z.shape
        dev = "cuda:0"
        self.logits = _upload(z, dtype, pad, 77.0)
        self.tokens = torch.from_numpy(self.tokens_h.astype(np.int32)).to(dev)
        new = lambda shape, t=torch.float32: torch.full(shape, 99, dtype=t, device=dev)
        self.logprob, self.entropy, self.stats = new((M,)), new((M,)), new((M, 4)) if stats else None
        self.alt = new((M, k), torch.int32) if k else None
        self.alt_lp = new((M, k)) if k else None
        nbytes = ql.qlora_token_logprobs_workspace_bytes(M, V, k, FLAG[dtype])
        self.ws = torch.full((max(nbytes, 16),), 0xFF, dtype=torch.uint8, device=dev)

    def forward(self, stream=None):
        M, V = self.shape
        ql.qlora_token_logprobs(self.logits, V + self.pad, self.tokens, self.logprob, self.entropy, self.alt, self.alt_lp,
                                self.k, self.stats, M, V, FLAG[self.dtype], self.ws, stream=stream)

    def check(self):
        M, V = self.shape
        lp, H, alt, alt_lp = scoring.score(self.z, self.tokens_h, self.k)
        got = {n: getattr(self, n).double().cpu().numpy() for n in ("logprob", "entropy")}
        with np.errstate(invalid="ignore"):
            full = scoring.log_probabilities(self.z)
            ls = np.nan_to_num(-(full.max(axis=1)), nan=0.0, posinf=0.0)           # ln S = -(log p of the largest)
            given = (self.tokens_h >= 0) & (self.tokens_h < V)
            d = np.abs(lp) + ls
            self._near(got["logprob"], lp, C * U * (1 + np.nan_to_num(d, nan=0, posinf=0)))
            self._near(got["entropy"], H, C * U * (1 + np.nan_to_num(H) + ls))
            if self.k:
                np.testing.assert_array_equal(self.alt.cpu().numpy(), alt)
                far = np.nan_to_num(np.abs(alt_lp), nan=0, posinf=0) + ls[:, None]
                self._near(self.alt_lp.double().cpu().numpy(), alt_lp, C * U * (1 + far))
        return given

    @staticmethod
    def _near(got, want, bound):
        np.testing.assert_array_equal(np.isnan(got), np.isnan(want))
        inf = np.isinf(want)
        np.testing.assert_array_equal(got[inf], want[inf])
        ok = np.isfinite(want)
        assert np.all(np.isfinite(got[ok])), "a finite value is expected"
        worst = np.max(np.abs(got[ok] - want[ok]) / np.broadcast_to(bound, want.shape)[ok]) if ok.any() else 0.0
        assert worst <= 1.0, f"{worst:.3g} times the bound"

    def backward(self, g, h, d_pad=0, into=None, stride=None, stream=None):
        import torch
        M, V = self.shape
        up = lambda a: None if a is None else torch.from_numpy(np.asarray(a, np.float32)).to("cuda:0")
        self.g, self.h = up(g), up(h)
        self.dlogits = torch.full((M, V + d_pad), 55, dtype=_torch(self.dtype), device="cuda:0") if into is None else into
        ql.qlora_token_logprobs_bwd(self.logits, V + self.pad, self.tokens, self.stats, self.g, self.h, self.dlogits,
                                    stride or self.dlogits.shape[1], M, V, FLAG[self.dtype], stream=stream)

    def check_gradient(self):
        M, V = self.shape
        g = None if self.g is None else self.g.double().cpu().numpy()
        h = None if self.h is None else self.h.double().cpu().numpy()
        want = scoring.score_gradient(self.z, self.tokens_h, g, h)
        got = self.dlogits[:, :V].double().cpu().numpy()
        with np.errstate(invalid="ignore"):
            lp = scoring.log_probabilities(self.z)
            p = np.nan_to_num(np.exp(lp))
            alp = np.nan_to_num(np.abs(lp), posinf=0, neginf=0)
            H = (p * alp).sum(axis=1, keepdims=True)
            ls = np.nan_to_num(-(lp.max(axis=1, keepdims=True)), nan=0, posinf=0)
            zero = np.zeros((M, 1))
            ga, ha = (zero if a is None else np.abs(a)[:, None] for a in (g, h))
            slope = p * (ga + ha * (alp + H))
            bound = C * U * (slope * (1 + alp + ls) + p * (ga + ha * (1 + H + ls)) + ga * (want != 0) * U)
            bound += HALF_ULP[self.dtype] * 1.01 * np.nan_to_num(np.abs(want)) + TINY[self.dtype] * (1 + ga + ha)
        self._near(got, want, bound)
        if self.dlogits.shape[1] > V:
            assert (self.dlogits[:, V:].float() == 55).all(), "entries behind the row were written"


def _tokens(seed, M, V):
    t = (wl.splitmix64(seed, 0, M) % np.uint64(V)).astype(np.int64)
    t[M // 3::7] = -1
    return t


# V around every boundary: pieces of 8 (4 in fp32), 64 lanes, a workgroup's 64 KB, segments; V < k; rows at any alignment
SHAPES = [
    (3, 1, "f16", 5, 0), (2, 2, "f32", 1, 1), (3, 7, "bf16", 8, 1), (2, 8, "f16", 8, 3), (3, 9, "f32", 20, 0),
    (4, 64, "bf16", 64, 0), (3, 65, "f16", 33, 7), (2, 511, "f32", 20, 2), (3, 513, "bf16", 5, 0), (2, 1025, "f16", 64, 5),
    (2, 4096, "f16", 20, 0), (3, 4097, "f32", 5, 3), (2, 8200, "bf16", 40, 1), (5, 32000, "f16", 5, 0),
    (2, 32003, "bf16", 20, 61), (2, 32768, "f16", 64, 0), (2, 32769, "f16", 20, 0), (3, 16384, "f32", 20, 0),
    (2, 16385, "f32", 64, 0), (2, 50257, "f32", 8, 1), (2, 128259, "bf16", 20, 61), (1, 400001, "f16", 16, 0),
    (70, 999, "f16", 3, 0), (33, 32000, "f32", 20, 0),
    # more rows than compute units: other workgroups (64 to 512 threads), rows in one piece and in segments
    (300, 400, "f16", 5, 0), (1100, 3001, "bf16", 64, 1), (2100, 5000, "f16", 2, 0), (260, 31999, "f16", 20, 0),
    (258, 40001, "bf16", 33, 3), (90, 128259, "bf16", 20, 61), (130, 40000, "f32", 5, 0),
]


@pytest.mark.parametrize("M,V,dtype,k,pad", SHAPES)
def test_scores_and_gradient(M, V, dtype, k, pad):
    announce(f"token logprobs M={M} V={V} {dtype} k={k} pad={pad}")
    c = _Call(_logits(V + M, M, V, dtype), _tokens(V, M, V), dtype, k, pad)
    c.forward()
    c.check()
    g, h = wl.normal(V + 5, M) * 3.0, wl.normal(V + 6, M)
    for gg, hh in ((g, h), (g, None), (None, h)):
        c.backward(gg, hh, d_pad=pad % 5)
        c.check_gradient()


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("V,times", [(100, 1), (5000, 1), (40000, 1), (5000, 30), (20000, 30)])
def test_masks(V, times, dtype):
    """Rows that mask all, all but one, all but a few, by -inf and by the type's lowest number; a masked target."""
    announce(f"token logprobs masks V={V} {dtype}, {times} times")
    import torch
    low = torch.finfo(_torch(dtype)).min
    M = 10
    z = _logits(V, M, V, dtype)
    few = (wl.splitmix64(V + 9, 0, 6) % np.uint64(V)).astype(np.int64)
    for row, fill in ((1, -np.inf), (2, -np.inf), (3, low), (4, low), (5, -np.inf), (6, low)):
        keep = z[row].copy()
        z[row] = fill
        if row in (2, 4):
            z[row, few[0]] = keep[few[0]]
        if row in (5, 6):
            z[row, few] = keep[few]
    z[7, V // 2:] = -np.inf                      # half a row, and a target in it
    z[8, ::3] = low
    tokens = _tokens(V + 1, M, V)
    tokens[:9] = [V, 0, few[0], 1, few[0], few[1], few[2], V - 1, 3]
    z, tokens, M = np.tile(z, (times, 1)), np.tile(tokens, times), M * times
    for k in (8, 20, 64):
        c = _Call(z, tokens, dtype, k)
        c.forward()
        c.check()
    c.backward(np.linspace(-2, 2, M), np.linspace(1, -1, M))
    c.check_gradient()


@pytest.mark.parametrize("dtype", ["f16", "f32"])
@pytest.mark.parametrize("kind", ["rising", "falling", "constant", "two_values", "hot_run", "integers", "zeros_of_both_signs"])
@pytest.mark.parametrize("times", [1, 131])
def test_alternatives_of_rows_in_order(kind, dtype, times):
    """Rows that defeat the first threshold: more entries above it than fit, and ties that go to the lower index."""
    announce(f"token logprobs alternatives {kind} {dtype}")
    M, V = 2, 20000
    i = np.arange(V)
    row = {"rising": i / 4096.0, "falling": -i / 4096.0, "constant": np.full(V, 1.5), "two_values": np.where(i % 7001 == 5, 2.0, 1.0),
           "hot_run": np.where((i > 3000) & (i < 9000), 5.0 + (i % 997) / 512.0, -3.0),
           "integers": (i * 7919 % 23).astype(float), "zeros_of_both_signs": np.where(i % 2 == 0, -0.0, 0.0)}[kind]
    z = np.tile(_rounded(np.stack([row, row[::-1]]), dtype), (times, 1))
    for k in (1, 5, 8, 33, 64) if times == 1 else (1, 20, 64):
        c = _Call(z, [3, V - 2] * times, dtype, k)
        c.forward()
        c.check()


@pytest.mark.parametrize("V", [50, 3000, 70000])
def test_not_finite_rows(V):
    """A NaN or plus infinity poisons its row and no other; rows whose gradients are 0 are zeros all the same."""
    announce(f"token logprobs not finite V={V}")
    z = _logits(3, 6, V, "f32")
    z[1, V - 1] = np.nan
    z[2, V // 2] = np.inf
    z[4] = np.nan
    z[5, 0], z[5, V - 1] = -np.inf, np.inf
    c = _Call(z, [1, 2, V - 1, 0, 5, V - 1], "f32", 5)
    c.forward()
    c.check()
    c.backward([1, 0, 2, 3, 0, 1], None)
    got = c.dlogits.cpu().numpy()
    assert (got[1] == 0).all() and (got[4] == 0).all()
    assert np.isnan(got[2]).all() and np.isnan(got[5]).all()
    want = scoring.score_gradient(z[[0, 3]], c.tokens_h[[0, 3]], np.array([1.0, 3.0]), None)
    np.testing.assert_allclose(got[[0, 3]], want, rtol=1e-4, atol=1e-6)


@pytest.mark.parametrize("dtype", ["f16", "f32"])
def test_nan_in_a_masked_stretch_of_a_long_row(dtype):
    """A row of several segments; one of them holds masked tokens and a single NaN: all that the row writes is NaN."""
    announce(f"token logprobs NaN among masks {dtype}")
    V = 140000
    z = _logits(4, 3, V, dtype)
    z[1, :30000] = -np.inf
    z[1, 7] = np.nan
    c = _Call(z, [40000, 40000, 5], dtype, 3)
    c.forward()
    c.check()
    stats = c.stats.cpu().numpy()
    assert np.isnan(stats[1]).all() and np.isfinite(stats[[0, 2]]).all()
    c.backward([1, 1, 1], None)
    got = c.dlogits.float().cpu().numpy()
    assert np.isnan(got[1]).all() and np.isfinite(got[[0, 2]]).all()


def test_almost_certain_tokens_keep_their_digits():
    """log p = -s of a dominant token: relative accuracy where 1 + s would round s away."""
    announce("token logprobs almost certain")
    V = 32000
    z = np.zeros((4, V))
    for row, top in enumerate((20.0, 25.0, 30.0, 40.0)):
        z[row, 100 * row] = top
    c = _Call(z, [0, 100, 200, 300], "f32", 1)
    c.forward()
    lp, H, _, _ = scoring.score(z, c.tokens_h, 0)
    # every weight is off by the same (2 * 40 * 1.45 + 2) u at most, the sum by 100 u, the entropy's factor by a few more
    np.testing.assert_allclose(c.logprob.cpu().numpy(), lp, rtol=300 * U)
    np.testing.assert_allclose(c.alt_lp.cpu().numpy()[:, 0], lp, rtol=300 * U)
    np.testing.assert_allclose(c.entropy.cpu().numpy(), H, rtol=300 * U)


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("M", [5, 300])
def test_outputs_are_optional(M, dtype):
    """Each output alone has the bits that it has beside the others."""
    import torch
    announce(f"token logprobs optional outputs M={M} {dtype}")
    V, k = 30000, 7
    z, tokens = _logits(8, M, V, dtype), _tokens(8, M, V)
    full = _Call(z, tokens, dtype, k)
    full.forward()
    names = ("logprob", "entropy", "alt", "stats")
    for only in names:
        c = _Call(z, tokens, dtype, k if only == "alt" else 0)
        for n in ("logprob", "entropy", "stats"):
            if n != only:
                setattr(c, n, None)
        if only != "logprob":
            c.tokens = None
        c.forward()
        assert torch.equal(getattr(c, only), getattr(full, only))
        if only == "alt":
            assert torch.equal(c.alt_lp, full.alt_lp)


@pytest.mark.parametrize("dtype,offset", [("f16", 1), ("f16", 5), ("bf16", 3), ("f32", 1), ("f32", 3)])
def test_slices_of_larger_tensors(dtype, offset):
    """The last position of every sequence of a batch with an odd vocabulary: rows begin at any element, S V apart."""
    import torch
    announce(f"token logprobs slices {dtype} {offset}")
    batch, S, V, k = 5, 3, 3001, 9
    whole = _logits(60, batch * S, V, dtype)
    store = torch.zeros(batch * S * V + offset, dtype=_torch(dtype), device="cuda:0")
    store[offset:] = _upload(whole, dtype, 0).view(-1)
    z = whole.reshape(batch, S, V)[:, -1]
    c = _Call(z, _tokens(61, batch, V), dtype, k)
    c.logits, c.pad = store[offset:].view(batch, S, V)[:, -1], (S - 1) * V
    c.forward()
    c.check()
    d = torch.full((batch * S * V + offset,), 55, dtype=_torch(dtype), device="cuda:0")
    c.backward(np.linspace(-1, 2, batch), np.ones(batch), into=d[offset:].view(batch, S, V)[:, -1], stride=S * V)
    c.check_gradient()
    others = d[offset:].view(batch, S, V)[:, :-1].float()
    assert (others == 55).all() and (d[:offset].float() == 55).all()


def test_entropy_gradient_without_tokens():
    announce("token logprobs, entropy alone")
    c = _Call(_logits(80, 4, 1000, "f16"), [-1] * 4, "f16", 0)
    c.forward()
    c.tokens = None
    c.backward(None, [1.0, 0.0, -2.0, 0.5])
    c.check_gradient()


@pytest.mark.parametrize("dtype", ["f16", "f32"])
def test_gradient_replaces_the_logits(dtype):
    import torch
    announce(f"token logprobs gradient in place {dtype}")
    M, V = 4, 5003
    c = _Call(_logits(12, M, V, dtype), _tokens(12, M, V), dtype, 0, pad=2)
    c.forward()
    g, h = np.linspace(1, 2, M), np.linspace(-1, 1, M)
    c.backward(g, h)
    apart = c.dlogits.clone()
    c.backward(g, h, into=c.logits)
    assert torch.equal(apart, c.logits[:, :V]) and (c.logits[:, V:].float() == 77).all()


def test_results_repeat_and_follow_the_stream():
    import torch
    announce("token logprobs repeat, other stream")
    M, V = 9, 50257
    c = _Call(_logits(20, M, V, "f16"), _tokens(20, M, V), "f16", 20)
    c.forward()
    c.backward(np.ones(M), np.ones(M))
    first = [t.clone() for t in (c.logprob, c.entropy, c.alt, c.alt_lp, c.stats, c.dlogits)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for t in (c.logprob, c.entropy, c.alt, c.alt_lp, c.stats, c.dlogits):
        t.fill_(3)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        c.ws.fill_(0x7F)
        c.forward()
        c.backward(np.ones(M), np.ones(M))
    side.synchronize()
    for a, b in zip(first, (c.logprob, c.entropy, c.alt, c.alt_lp, c.stats, c.dlogits)):
        assert torch.equal(a, b)


def test_graph_replays_match_eager():
    import torch
    announce("token logprobs graph")
    M, V = 6, 70001
    c = _Call(_logits(30, M, V, "bf16"), _tokens(30, M, V), "bf16", 9)
    others = [_upload(_logits(31 + i, M, V, "bf16"), "bf16", 0) for i in range(3)]
    g = torch.ones(M, device="cuda:0")
    d = torch.empty_like(c.logits)
    flag = FLAG["bf16"]

    def run():
        c.forward()
        ql.qlora_token_logprobs_bwd(c.logits, V, c.tokens, c.stats, g, g, d, V, M, V, flag)

    outs = lambda: [t.clone() for t in (c.logprob, c.entropy, c.alt, c.alt_lp, c.stats, d)]
    eager = []
    for z in others:
        c.logits.copy_(z)
        run()
        eager.append(outs())
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        run()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    for rep in range(6):
        c.logits.copy_(others[rep % 3])
        for t in (c.logprob, c.entropy, c.alt, c.alt_lp, c.stats, d):
            t.fill_(5)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(eager[rep % 3], outs()):
            assert torch.equal(a, b), f"replay {rep}"


@pytest.mark.parametrize("kind", ["normal", "rising", "constant"])
@pytest.mark.parametrize("M,dtype", [(1, "f32"), (2, "f16")])
def test_rows_of_many_segments(M, dtype, kind):
    """1.5 million tokens: more segments than a wave has lanes, and lists of 64 alternatives of each to be joined."""
    announce(f"token logprobs {M} x 1500001 {dtype} {kind}")
    V = 1500001
    i = np.arange(V)
    z = {"normal": lambda: _logits(9, M, V, dtype), "rising": lambda: np.tile(_rounded(i / 2.0 ** 17, dtype), (M, 1)),
         "constant": lambda: np.full((M, V), -2.5)}[kind]()
    c = _Call(z, np.array([V - 1, 7])[:M], dtype, 64)
    c.forward()
    c.check()
    c.backward(np.ones(M), np.ones(M))
    c.check_gradient()


def test_longest_row():
    """2^28 tokens.  All logits are 0 but 20 in places from the first to the last; the sums are then known."""
    import torch
    announce("token logprobs 1 x 2^28 f16")
    V, k = 1 << 28, 21
    z = torch.zeros((1, V), dtype=torch.float16, device="cuda:0")
    at = [int(p) for p in np.linspace(0, V - 1, 20)]
    high = 12.0 + np.arange(20) / 4.0
    z[0, torch.tensor(at, device="cuda:0")] = torch.from_numpy(high).half().cuda()
    dev = lambda shape, t=torch.float32: torch.full(shape, 9, dtype=t, device="cuda:0")
    lp, H, st, alt, alp, token = dev((1,)), dev((1,)), dev((1, 4)), dev((1, k), torch.int32), dev((1, k)), dev((1,), torch.int32)
    token.fill_(V - 1)
    ws = torch.empty(ql.qlora_token_logprobs_workspace_bytes(1, V, k, ql.QLORA_F16), dtype=torch.uint8, device="cuda:0")
    ql.qlora_token_logprobs(z, V, token, lp, H, alt, alp, k, st, 1, V, ql.QLORA_F16, ws)
    total = np.exp(high).sum() + (V - 20)
    want = np.concatenate([high[::-1], [0.0]]) - np.log(total)
    entropy = np.log(total) - (np.exp(high) * high).sum() / total
    ls = np.log(total) - high[-1]
    assert alt[0].tolist() == at[::-1] + [1]
    # a lane adds up to 64 equal weights, 2^12 segments are joined by 64 additions a lane: the module's C covers both
    assert np.all(np.abs(alp[0].cpu().numpy() - want) <= C * U * (1 + np.abs(want) + ls))
    assert abs(float(lp) - want[0]) <= C * U * (1 + abs(want[0]) + ls)
    assert abs(float(H) - entropy) <= C * U * (1 + entropy + ls)
    g = torch.ones(1, device="cuda:0")
    ql.qlora_token_logprobs_bwd(z, V, token, st, g, None, z, V, 1, V, ql.QLORA_F16)
    p = np.exp(want)
    got = z[0, torch.tensor(at[::-1], device="cuda:0")].double().cpu().numpy()
    exact = np.eye(20)[0] - p[:20]
    off = C * U * p[:20] * (1 + np.abs(want[:20]) + ls)
    assert np.all(np.abs(got - exact) <= off + HALF_ULP["f16"] * 1.01 * np.abs(exact) + TINY["f16"] * 1.01)
    rest = z[0].count_nonzero().item()                      # the others' -p = 1 / total is below fp16's smallest number
    assert rest == 20 and p[20] < TINY["f16"]


def test_two_calls_at_once():
    """Two streams, each with its own workspace and outputs, find what one does."""
    import torch
    announce("token logprobs two streams")
    calls = [_Call(_logits(40 + i, 12, 90001, "f16"), _tokens(40 + i, 12, 90001), "f16", 20) for i in range(2)]
    outs = lambda c: [t.clone() for t in (c.logprob, c.entropy, c.alt, c.alt_lp, c.stats)]
    for c in calls:
        c.forward()
    first = [outs(c) for c in calls]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in calls]
    for _ in range(20):
        for c, s in zip(calls, streams):
            c.forward(stream=s)
    torch.cuda.synchronize()
    for c, was in zip(calls, first):
        assert all(torch.equal(a, b) for a, b in zip(was, outs(c)))


def test_logits_beyond_four_gigabytes():
    """Offsets that pass 32 bits, of elements and of bytes: sampled rows of 70000 x 32000, scored and differentiated in place."""
    import torch
    announce("token logprobs 70000 x 32000 f16")
    M, V, k = 70000, 32000, 3
    dev = "cuda:0"
    z = torch.empty((M, V), dtype=torch.float16, device=dev)
    part = torch.randn((1000, V), device=dev, generator=torch.Generator(device=dev).manual_seed(5)).mul_(2.5).half()
    for at in range(0, M, 1000):
        z[at:at + 1000] = part.roll(at // 1000 * 37, 1)
    tokens = (torch.arange(M, device=dev) * 7919 % V).int()
    new = lambda *s, t=torch.float32: torch.empty(s, dtype=t, device=dev)
    lp, H, st, alt, alp, g = new(M), new(M), new(M, 4), new(M, k, t=torch.int32), new(M, k), torch.ones(M, device=dev)
    rows = np.array([0, 1, 33554, 33555, 67107, 67109, 67110, M - 2, M - 1])
    zs = z[torch.from_numpy(rows).to(dev)].double().cpu().numpy()
    ql.qlora_token_logprobs(z, V, tokens, lp, H, alt, alp, k, st, M, V, ql.QLORA_F16, None)
    ql.qlora_token_logprobs_bwd(z, V, tokens, st, g, None, z, V, M, V, ql.QLORA_F16)
    at = torch.from_numpy(rows).to(dev)
    ts = tokens[at].cpu().numpy()
    wl_, wH, walt, walp = scoring.score(zs, ts, k)
    np.testing.assert_allclose(lp[at].cpu().numpy(), wl_, atol=C * U * 40)
    np.testing.assert_allclose(H[at].cpu().numpy(), wH, atol=C * U * 40)
    np.testing.assert_array_equal(alt[at].cpu().numpy(), walt)
    dz = scoring.score_gradient(zs, ts, np.ones(len(rows)), None)
    np.testing.assert_allclose(z[at].double().cpu().numpy(), dz, rtol=2 * HALF_ULP["f16"], atol=TINY["f16"] * 1.01)


LARGE = (-1e10, -1e11, -1e12, -1e15, -1e18, -1e30, -1e31, -1e32)        # numbers that programs mask with


def _check_both(z, tokens, dtype, k):
    """Scores and gradient against the oracle; nothing of a finite row may be anything but finite."""
    c = _Call(z, tokens, dtype, k)
    c.forward()
    c.check()
    assert np.isfinite(c.logprob.cpu().numpy()).all() and np.isfinite(c.stats.cpu().numpy()).all()
    M = len(z)
    c.backward(np.linspace(-2, 2, M), np.linspace(1, -1, M))
    c.check_gradient()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V,times", [(100, 1), (1000, 40), (40000, 1), (5000, 30)])
def test_rows_of_one_large_number(V, times, dtype):
    """Every token masked by the same finite number: a uniform distribution over all of them."""
    announce(f"token logprobs rows of one large number V={V} {dtype}, {times} times")
    z = _rounded(np.tile(np.repeat(np.array(LARGE)[:, None], V, axis=1), (times, 1)), dtype)
    _check_both(z, _tokens(V, *z.shape), dtype, 5)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V,times", [(1000, 1), (33000, 1), (140003, 1), (140003, 4)])
def test_ordinary_rows_masked_by_large_numbers(V, times, dtype):
    """Ordinary logits beside large finite masks.  Rows of 140003 tokens are taken in segments, of which some hold the mask and nothing
    else: at the row's head, at its tail, all but one, and all but one token."""
    announce(f"token logprobs masked by large numbers V={V} {dtype}, {times} times")
    rows = []
    for i, low in enumerate(LARGE):
        head, tail, middle, one = _logits(V + 7 * i, 4, V, dtype)
        head[:V // 2] = low
        tail[V - V // 3:] = low
        middle[:V // 3], middle[V // 3 + 50:] = low, low
        kept = one[V - 1]
        one[:] = low
        one[V - 1] = kept
        rows += [head, tail, middle, one]
    z = _rounded(np.tile(np.stack(rows), (times, 1)), dtype)
    M = len(z)
    tokens = np.tile([V - 1, 3, V // 3 + 7, V - 1], M // 4)
    tokens[4::9] = 0                             # a masked target
    _check_both(z, tokens, dtype, 20)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V", [900, 140003])
def test_rows_with_a_large_maximum(V, dtype):
    """One token far above all others, two of them at the maximum, and a neighbour one step of the type below it."""
    import torch
    announce(f"token logprobs large maxima V={V} {dtype}")
    tops = _rounded(np.array([[1e9, 5e9, 1e10, 3e12, 1e20, 1e31, 3e38]]), dtype)[0]
    M = len(tops)
    z = np.tile(_logits(V, M, V, dtype), (3, 1))
    for i, top in enumerate(tops):
        below = torch.nextafter(torch.tensor(top, dtype=_torch(dtype)), torch.tensor(0.0, dtype=_torch(dtype))).item()
        z[i, V // 2] = top
        z[M + i, [5, V - 2]] = top
        z[2 * M + i, [7, V - 3]] = top, below
    _check_both(z, np.tile([V // 2, 5, V - 3], (M, 1)).T.ravel(), dtype, 3)


def test_workspace_of_a_batch_serves_a_smaller_one():
    """64 rows are taken in more segments than 100 are; what lies behind the larger batch's workspace stays as it was."""
    import torch
    announce("token logprobs workspace of 100 rows, 64 rows")
    V, k = 100000, 20
    need = ql.qlora_token_logprobs_workspace_bytes(100, V, k, ql.QLORA_F16)
    c = _Call(_logits(70, 64, V, "f16"), _tokens(70, 64, V), "f16", k)
    store = torch.full((need + 4096,), 0xA5, dtype=torch.uint8, device="cuda:0")
    c.ws = store[:need]
    c.forward()
    c.check()
    assert (store[need:] == 0xA5).all()


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
def test_gradients_of_almost_certain_tokens_keep_their_digits(dtype):
    """g (1 - p) of a dominant token, where p rounds to 1; and that of a token which another one dominates."""
    announce(f"token logprobs gradient, almost certain {dtype}")
    V = 32000
    z = np.zeros((5, V))
    for row, top in enumerate((20.0, 25.0, 30.0, 40.0, 30.0)):
        z[row, 100 * row] = top
    c = _Call(z, [0, 100, 200, 300, 401], dtype, 0)
    c.forward()
    g = np.array([1024.0, -1024.0, 4096.0, 2.0 ** 30, 3.0])
    c.backward(g, None)
    at = (np.arange(5), c.tokens_h)
    want = -g * np.expm1(scoring.score(z, c.tokens_h, 0)[0])           # (1 - p in 64 bits is off by 2^-54: half a step of fp16 at 40)
    got = c.dlogits.double().cpu().numpy()[at]
    # log p is off by 300 u (see the test of the scores), a difference carries that over with a factor of at most 1, and expm1
    # and the product add a few more
    bound = (310 * U + HALF_ULP[dtype]) * 1.01 * np.abs(want) + TINY[dtype]
    assert np.all(np.abs(got - want) <= bound), np.abs(got - want) / bound
