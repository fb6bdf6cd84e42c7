"""dcd_sample against the definition in 64 bits: tokens and kept counts exactly, probabilities
to 2^-23 (one rounding to fp32, 2^-24, and as much again for the fixed-point total), the
log-probability to one rounding of its value plus 1e-9.
"""
import numpy as np
import pytest
import torch

import proposal_oracle as oracle
from paper_2608_12913_amd import dcd

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def uniforms(R, seed):
    return (np.random.RandomState(seed).randint(0, 2 ** 23, R) + 0.5) * 2.0 ** -23


class Call:
    """One call's buffers; logits [R, V] (float32 values) laid out with `stride` and `offset` elements."""

    def __init__(self, z, u, dtype="f32", stride=0, offset=0, want=True, **rules):
        self.R, self.V = z.shape
        self.dtype, self.stride = dtype, stride or self.V
        flat = torch.full((self.R * self.stride + offset,), float("nan"), dtype=TYPES[dtype], device=DEV)
        self.z = flat[offset:].view(self.R, self.stride)
        self.z[:, :self.V] = torch.from_numpy(np.asarray(z, np.float32)).to(DEV)
        self.u = torch.from_numpy(np.asarray(u, np.float32)).to(DEV)
        self.rules = {n: None if v is None else torch.from_numpy(np.asarray(v)).to(DEV) for n, v in rules.items()}
        i32 = dict(dtype=torch.int32, device=DEV)
        self.tokens, self.kept = torch.full((self.R,), -9, **i32), torch.full((self.R,), -9, **i32)
        self.logprob = torch.full((self.R,), 9.0, device=DEV)
        self.probs = torch.full((self.R, self.V), 9.0, device=DEV)
        self.problem = dcd.make_sample_problem(self.R, self.V, dtype, stride)
        self.bytes = dcd.sample_workspace_bytes(self.problem)
        self.ws = torch.full((self.bytes,), 255, dtype=torch.uint8, device=DEV)
        r = self.rules
        self.ins = dcd.make_sample_inputs(self.z, self.u, r.get("temperature"), r.get("top_k"), r.get("top_p"),
                                          r.get("min_p"))
        self.outs = (dcd.make_sample_outputs(self.tokens, self.probs, self.logprob, self.kept) if want
                     else dcd.make_sample_outputs(self.tokens))

    def run(self, stream=None):
        dcd.sample(self.problem, self.ins, self.outs, self.ws, self.bytes, stream or torch.cuda.current_stream())
        return self

    def results(self):
        torch.cuda.synchronize()
        return [t.cpu().numpy() for t in (self.tokens, self.kept, self.probs, self.logprob)]

    def check(self, rows=None):
        tokens, kept, probs, logprob = self.results()
        z = self.z[:, :self.V].double().cpu().numpy()
        u = self.u.cpu().numpy().astype(np.float64)
        rule = {n: None if v is None else v.cpu().numpy() for n, v in self.rules.items()}
        one = lambda n, r, d: d if rule.get(n) is None else rule[n][r].item()  # noqa: E731
        for r in rows if rows is not None else range(self.R):
            t, n, p, lp = oracle.sample_row(z[r], u[r], one("temperature", r, 1.0), one("top_k", r, 0),
                                            one("top_p", r, 1.0), one("min_p", r, 0.0))
            assert (tokens[r], kept[r]) == (t, n), (r, tokens[r], t, kept[r], n)
            assert np.array_equal(probs[r] > 0, p > 2.0 ** -150) or np.array_equal((probs[r] > 0)[p > 1e-37], (p > 0)[p > 1e-37])
            assert (np.abs(probs[r] - p) <= 2.0 ** -23 * p + 2.0 ** -149).all(), r
            assert np.array_equal(np.isnan(logprob[r]), np.isnan(lp))
            assert not abs(logprob[r] - lp) > 2.0 ** -24 * abs(lp) + 1e-9, (r, logprob[r], lp)


def logits(R, V, seed, spread=3.0):
    rng = np.random.RandomState(seed)
    return rng.randn(R, V).astype(np.float32) * np.float32(spread) - np.log(np.arange(1, V + 1)).astype(np.float32)


def mixed(R, seed):
    rng = np.random.RandomState(seed)
    i = np.arange(R)
    return dict(temperature=np.where(i % 7 == 3, 0, rng.uniform(0.5, 1.6, R)).astype(np.float32),
                top_k=np.where(i % 3 == 0, 0, rng.randint(1, 200, R)).astype(np.int32),
                top_p=np.where(i % 5 == 0, 1, rng.uniform(0.3, 0.99, R)).astype(np.float32),
                min_p=np.where(i % 2 == 0, 0, rng.uniform(0, 0.3, R)).astype(np.float32))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [1, 2, 5, 63, 64, 65, 255, 1000, 1031, 4096, 4097, 8193, 32003, 50001])
def test_vocabularies(V, dtype):
    Call(logits(24, V, V), uniforms(24, V), dtype, **mixed(24, V)).run().check()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("R", [1, 3, 300])
def test_full_vocabulary(R, dtype):
    Call(logits(R, 128256, R), uniforms(R, R), dtype, **mixed(R, R)).run().check(range(0, R, max(1, R // 20)))


@pytest.mark.parametrize("name, value", [
    ("temperature", [0.0, 1e-30, 1e-3, 0.3, 1.0, 4.0, 1e4, 1e30]), ("top_k", [-5, 0, 1, 2, 40, 900, 1999, 2000, 5000]),
    ("top_p", [0.0, 1e-7, 0.1, 0.5, 0.9, 0.999, 0.9999999, 1.0]), ("min_p", [0.0, 1e-30, 1e-3, 0.1, 0.5, 0.999, 1.0])])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_one_rule_alone(name, value, dtype):
    value = np.repeat(np.array(value, np.int32 if name == "top_k" else np.float32), 3)
    for V in (2000, 20011):
        Call(logits(len(value), V, 3), uniforms(len(value), 4), dtype, **{name: value}).run().check()


@pytest.mark.parametrize("T", [1e-20, 1e-3, 50.0, 1e6, 1e30])
def test_top_p_and_min_p_at_extreme_temperatures(T):
    """Weights that all but vanish beside the largest, or all but equal it."""
    for V in (3001, 40000):
        R = 8
        p, m = np.array([0.3, 0.9, 1, 1] * 2, np.float32), np.array([0, 0, 0.2, 0.99999] * 2, np.float32)
        z = logits(R, V, 5, 2.0)
        z[4:] *= 1e-30
        Call(z, uniforms(R, 3), temperature=np.full(R, T, np.float32), top_p=p, min_p=m).run().check()


@pytest.mark.parametrize("V", [9000, 128256])
def test_top_p_with_min_p_and_deep_rows(V):
    """Where one of the two rules cuts far above the other, and nuclei of many tokens."""
    R = 24
    p = np.array([0.2, 0.6, 0.9, 0.99, 0.9999, 1.0] * 4, np.float32)
    m = np.repeat(np.array([1e-9, 1e-4, 0.02, 0.7], np.float32), 6)
    Call(logits(R, V, 6, 2.5), uniforms(R, 7), top_p=p, min_p=m).run().check()
    Call(logits(R, V, 6, 1.0), uniforms(R, 7), "bf16", top_p=p).run().check()


@pytest.mark.parametrize("V", [3001, 40000])
@pytest.mark.parametrize("spread", [0.0, 0.01, 0.3, 1.0])
def test_flat_rows(V, spread):
    """Nuclei of thousands of tokens, and rows of equal logits (ties cut by id)."""
    R = 12
    z = np.random.RandomState(1).randn(R, V).astype(np.float32) * np.float32(spread)
    top_p = np.array([0.1, 0.5, 0.75, 0.9, 0.99, 1.0] * 2, np.float32)
    top_k = np.array([0] * 6 + [V // 3, 700, 0, V - 1, 5, 2500], np.int32)
    Call(z, uniforms(R, 2), top_p=top_p, top_k=top_k).run().check()


@pytest.mark.parametrize("V", [3, 701, 9001, 20003])
def test_more_rows_than_compute_units(V):
    """Deep, flat, mixed and masked rows by the hundred (a row has fewer threads there)."""
    R = 300
    z = logits(R, V, 15, 2.0)
    z[5::7] *= 0.02
    z[3::11, ::2] = -np.inf
    z[4::50] = -np.inf
    rules = mixed(R, 16)
    rules["top_k"][::9] = V // 2
    rules["top_p"][1::8], rules["top_k"][1::8], rules["min_p"][1::8] = 0.97, 0, 0
    Call(z, uniforms(R, 17), **rules).run().check(range(0, R, 3))
    Call(z, uniforms(R, 18), top_p=np.linspace(0, 1, R).astype(np.float32)).run().check(range(1, R, 3))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [700, 20003])
def test_masks_and_values_at_the_ends(V, dtype):
    lowest = torch.finfo(TYPES[dtype]).min
    rng = np.random.RandomState(0)
    z = logits(20, V, 8, 2.0)
    z[0, :] = -np.inf                           # nothing left
    z[1, :] = -np.inf
    z[1, V // 2] = -3.0                         # one token left
    z[2, :] = lowest                            # a flat row of the lowest value
    z[3, 10:] = lowest
    z[4, 7] = np.nan
    z[5, V - 1] = np.inf
    z[6, rng.rand(V) < 0.9] = -np.inf
    z[7, :] = 0.0
    z[7, ::2] = -0.0                            # equal logits
    z[8, V - 1] = 80.0                          # all of the weight in the last token
    z[9, 0] = 300.0
    z[10, :] = np.float32(3e38)
    z[10, 5] = np.float32(-3e38)
    z[11, 1:] = -np.inf
    z[12, :-1] = -np.inf
    z[13, 20:] = np.float32(1e-40)              # subnormal logits
    top_k = np.full(20, 50, np.int32)
    for k in (None, top_k):
        for p in (None, np.full(20, 0.9, np.float32)):
            for m in (None, np.full(20, 0.25, np.float32)):
                Call(z, uniforms(20, 5), dtype, top_k=k, top_p=p, min_p=m).run().check()


def test_rules_outside_their_range_leave_the_row_without_a_token():
    nan, inf = np.nan, np.inf
    T = np.array([1, -1, nan, inf, 1, 1, 1, 1, 1, 1, 1, 1], np.float32)
    p = np.array([1, 1, 1, 1, -0.1, 1.1, nan, 1, 1, 1, 1, 0.5], np.float32)
    m = np.array([0, 0, 0, 0, 0, 0, 0, -0.1, 1.5, nan, 0, 0], np.float32)
    u = np.full(12, 0.5)
    u[10] = 1.0
    for V in (500, 20000):
        c = Call(logits(12, V, 2), u, temperature=T, top_p=p, min_p=m).run()
        c.check()
        assert c.results()[0].tolist()[1:11] == [-1] * 10 and c.results()[0][0] >= 0 and c.results()[0][11] >= 0


@pytest.mark.parametrize("V", [2, 700, 9001, 40000])
@pytest.mark.parametrize("bits", [0x7fffffff, -1, 0x7f800001])
def test_every_kind_of_nan_leaves_the_row_without_a_token(V, bits):
    """NaN of any payload and sign, with rules of each kind and without."""
    z = logits(8, V, 19)
    z.view(np.int32)[::2, V // 2] = np.int32(bits)
    off = dict(top_k=np.zeros(8, np.int32), top_p=np.ones(8, np.float32), min_p=np.zeros(8, np.float32))
    for name, value in (("top_k", 5), ("top_p", 0.7), ("min_p", 0.1), ("top_p", 1.0)):
        rules = {n: a.copy() for n, a in off.items()}
        rules[name][:] = value
        Call(z, uniforms(8, 20), **rules).run().check()


@pytest.mark.parametrize("V", [900, 30011])
def test_first_and_last_uniforms(V):
    z = logits(8, V, 11, 1.0)
    z[4:, 0] = z[4:, V - 1] = -np.inf
    u = np.array([0.0, 1 - 2.0 ** -24, 0.0, 1 - 2.0 ** -24] * 2)
    k = np.array([0, 0, 30, 30] * 2, np.int32)
    Call(z, u, top_k=k).run().check()


@pytest.mark.parametrize("V", [(1 << 20) - 3, 1 << 20, (1 << 20) + 5])
def test_the_longest_rows(V):
    """Either side of the longest vocabulary that is read in slices."""
    R = 9
    z = np.random.RandomState(2).randn(R, V).astype(np.float32) * 4
    rules = mixed(R, 5)
    rules["temperature"][0], rules["top_k"][0], rules["top_p"][0], rules["min_p"][0] = 1, 0, 1, 0
    rules["top_k"][4] = 3000
    Call(z, uniforms(R, 6), **rules).run().check()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_rows_past_32_bits(dtype):
    """The third row starts 2^31 elements behind the first."""
    Call(logits(3, 5003, 21), uniforms(3, 21), dtype, 1 << 30, **mixed(3, 22)).run().check()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V, stride, offset", [(1000, 1003, 0), (1000, 1024, 1), (20001, 20008, 3), (20001, 20001, 1)])
def test_strides_and_alignment(V, stride, offset, dtype):
    """Rows that start anywhere; what lies between them (NaN here) is not read."""
    Call(logits(9, V, 1), uniforms(9, 1), dtype, stride, offset, **mixed(9, 4)).run().check()


def test_optional_outputs():
    a = Call(logits(16, 20000, 5), uniforms(16, 5), **mixed(16, 5)).run()
    b = Call(logits(16, 20000, 5), uniforms(16, 5), want=False, **mixed(16, 5)).run()
    assert np.array_equal(a.results()[0], b.results()[0])
    assert (b.results()[1] == -9).all() and (b.results()[2] == 9).all()


def test_draws_follow_the_distribution():
    """Over a midpoint grid of uniforms the frequencies are the probabilities."""
    V, R = 40, 4000
    z = np.repeat(logits(1, V, 3, 1.0), R, axis=0)
    c = Call(z, (np.arange(R) + 0.5) / R, top_k=np.full(R, 20, np.int32), top_p=np.full(R, 0.9, np.float32)).run()
    tokens, _, probs, _ = c.results()
    freq = np.bincount(tokens, minlength=V) / R
    assert np.abs(freq - probs[0]).max() <= 1.0 / R + 1e-6


@pytest.mark.parametrize("R, V", [(1, 128256), (40, 20011), (200, 1500)])
def test_repeats_streams_and_graphs(R, V):
    """Bit-identical repeats; two calls at once on two streams; a captured call replayed with
    new inputs, with eager calls in between."""
    c = Call(logits(R, V, 1), uniforms(R, 1), **mixed(R, 1)).run()
    first = c.results()
    for _ in range(3):
        assert all(np.array_equal(x, y, equal_nan=True) for x, y in zip(first, c.run().results()))
    d = Call(logits(R, V, 2), uniforms(R, 2), **mixed(R, 2))
    torch.cuda.synchronize()
    s, t = torch.cuda.Stream(), torch.cuda.Stream()
    for _ in range(3):
        c.run(s)
        d.run(t)
    assert all(np.array_equal(x, y, equal_nan=True) for x, y in zip(first, c.results()))
    d.check(range(min(R, 5)))
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        c.run(torch.cuda.current_stream())
    for seed in (3, 4, 5):
        c.z[:, :V] = torch.from_numpy(logits(R, V, seed)).to(DEV)
        c.u.copy_(torch.from_numpy(uniforms(R, seed).astype(np.float32)))
        g.replay()
        torch.cuda.synchronize()
        replayed = c.results()
        c.check(range(min(R, 3)))
        assert all(np.array_equal(x, y, equal_nan=True) for x, y in zip(replayed, c.run().results()))
