"""The 8-bit proposal path as a proposer runs it: codes of the hidden states, logits, sampling, and the
proposals' own probabilities into dcd_verify_sample, without the host in between."""
import numpy as np
import pytest
import torch

import oracle
import proposal_oracle
from paper_2608_12913_amd import dcd, synth
from paper_2608_12913_amd.runner import DeviceProblem, DraftHead
from tests import parity

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _rules(rows, seed):
    """One value per row of each rule, every rule off for some rows."""
    rng = np.random.default_rng(seed)
    i = np.arange(rows)
    return dict(temperature=np.where(i % 5 == 4, 0, rng.uniform(0.6, 1.3, rows)).astype(np.float32),
                top_k=np.where(i % 2 == 0, 0, rng.integers(1, 60, rows)).astype(np.int32),
                top_p=np.where(i % 3 == 0, 1, rng.uniform(0.5, 0.99, rows)).astype(np.float32),
                min_p=np.where(i % 4 == 1, 0.02, 0).astype(np.float32))


def _check_step(head, h, u, rules, g):
    """One step's outputs: codes exactly; logits to d fp32 sums' and products' roundings, 2^-24 of the
    magnitudes' sum each, and one rounding to the logits' type; the draws from the logits that the
    kernels made exactly."""
    rows = len(h)
    q, s = proposal_oracle.quantize(h, 1)
    assert np.array_equal(head.h[:rows].cpu().numpy(), q) and np.array_equal(head.h_scale[:rows].cpu().numpy(), s)
    bias = None if head.bias is None else head.bias.double().cpu().numpy()
    z, mag = proposal_oracle.logits(q, s, head.w.cpu().numpy(), head.w_scale.cpu().numpy(), bias)
    got = head.logits[:rows].double().cpu().numpy()
    per = 2.0 ** -8 if head.logits_dtype == "bf16" else 2.0 ** -24
    room = head.d * 2.0 ** -24 * mag + per * np.abs(z) + 2.0 ** -20
    assert (np.abs(got - z) <= room).all(), np.abs(got - z).max()
    for r in range(rows):
        t, n, p, lp = proposal_oracle.sample_row(got[r], float(u[r]), *(rules[k][r].item() for k in
                                                 ("temperature", "top_k", "top_p", "min_p")))
        assert (g["tokens"][r], g["kept"][r]) == (t, n), r
        assert (np.abs(g["probs"][r] - p) <= 2.0 ** -23 * p + 2.0 ** -149).all()


@pytest.mark.parametrize("logits_dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows, V, d, dtype, with_bias", [(1, 4099, 256, "f32", True), (24, 2000, 400, "bf16", False),
                                                          (64, 1111, 128, "bf16", True)])
def test_steps(rows, V, d, dtype, with_bias, logits_dtype):
    rng = np.random.default_rng(rows)
    t = torch.bfloat16 if dtype == "bf16" else torch.float32
    w = (torch.from_numpy(rng.standard_normal((V, d)).astype(np.float32)) * 3 / d ** 0.5).to(t)
    head = DraftHead(w, rng.standard_normal(V).astype(np.float32) if with_bias else None, max_rows=rows + 3,
                     logits_dtype=logits_dtype, device=DEV)
    q, s = proposal_oracle.quantize(w.double().numpy(), 128)
    assert np.array_equal(head.w.cpu().numpy(), q) and np.array_equal(head.w_scale.cpu().numpy(), s)
    for step in range(2):
        h = torch.from_numpy(rng.standard_normal((rows, d)).astype(np.float32)).to(t)
        u, rules = rng.random(rows).astype(np.float32), _rules(rows, step)
        _check_step(head, h.double().numpy(), u, rules, head.propose(h, u, **rules))


def test_drafts_feed_sampled_verification():
    """A chain's nodes are drawn from an 8-bit copy of the expert head, their tokens and distributions
    left where dcd_verify_sample reads them; the verification against its oracle on those."""
    rng = np.random.default_rng(72)
    case = synth.make_case("s8_chain16x8", 72, B=4, N=8, V=2000, dp=256, dq=128, theta=0.1)
    B, N, V, R = case.B, case.N, case.V, case.R
    head = DraftHead(case.wp, case.bias, max_rows=R, device=DEV)
    # row b * N + i proposes node i: the hidden state of its parent (the roots': of themselves)
    parent = np.maximum(np.asarray(case.parents).reshape(B, N), 0) + np.arange(B)[:, None] * N
    h = torch.from_numpy(oracle.as_f32(case.hp)[parent.reshape(-1)]).to(DEV)
    u = torch.from_numpy(rng.random(R).astype(np.float32)).to(DEV)
    rules = {n: torch.from_numpy(a).to(DEV) for n, a in _rules(R, 3).items()}
    dev = DeviceProblem.from_case(case, np.zeros((B, N), np.int32), draft_probs=np.zeros((R, V), np.float32))
    kept = torch.empty(R, dtype=torch.int32, device=DEV)
    head.launch(h, u, dev.tokens, dev.draft_probs, kept=kept, **rules)
    v = dev.run("sample")
    tokens, probs = dev.tokens.cpu().numpy(), dev.draft_probs.cpu().numpy()
    host = {n: a.cpu().numpy() for n, a in rules.items()}
    _check_step(head, h.double().cpu().numpy(), u.cpu().numpy(), host,
                dict(tokens=tokens.reshape(-1), kept=kept.cpu().numpy(), probs=probs))
    o = oracle.verify("sample", B, N, case.hp, case.hq, case.wp, case.wq, case.bias, case.bias, case.parents, tokens,
                      theta=case.theta, s=case.s, temperature=case.T, draft_probs=probs, u_acc=case.u_acc,
                      u_res=case.u_res)
    lp = oracle.eval_rows(case.hp, case.hq, case.wp, case.wq, case.bias, case.bias, theta=case.theta, s=case.s,
                          temperature=case.T, want_lpcd=True)["lpcd"]
    report = {}
    amb = parity.compare_rows(v, o, np.arange(R), report)
    parity.compare_nodes(v, o, case.parents, amb, report)
    boundary = o["row_gap"] <= parity.BOUNDARY_GATE
    parity.measure_target_error(dev.propose(case.u_res)["probs"], lp, boundary, report)
    parity.compare_sample(v, o, lp, probs, case.parents, tokens, case.u_acc, case.u_res, boundary, report)
    parity.check_gates(report)


def test_step_and_verification_in_one_graph():
    """Proposals and their verification captured together and replayed on new inputs, with eager steps
    of another problem on a second stream in between: the same results as eager calls, bit by bit."""
    case = synth.make_case("s8_chain16x8", 73, B=3, N=8, V=3001, dp=256, dq=128, theta=0.1)
    R, V = case.R, case.V
    head = DraftHead(case.wp, case.bias, max_rows=R, device=DEV)
    other = DraftHead(case.wp, None, max_rows=70, logits_dtype="bf16", device=DEV)
    dev = DeviceProblem.from_case(case, np.zeros((case.B, case.N), np.int32), draft_probs=np.zeros((R, V), np.float32))
    rules = {n: torch.from_numpy(a).to(DEV) for n, a in _rules(R, 4).items()}
    rng = np.random.default_rng(74)
    inputs = [(torch.from_numpy(rng.standard_normal((R, 256)).astype(np.float32)).to(DEV),
               torch.from_numpy(rng.random(R).astype(np.float32)).to(DEV)) for _ in range(3)]
    h, u = (t.clone() for t in inputs[0])

    def step():
        head.launch(h, u, dev.tokens, dev.draft_probs, **rules)
        dev.launch("sample")

    def results():
        torch.cuda.synchronize()
        return [t.clone() for t in (dev.tokens, dev.draft_probs, dev.accept_len, dev.accept_path, dev.next_token, dev.status)]

    eager = []
    for a, b in inputs:
        h.copy_(a)
        u.copy_(b)
        step()
        eager.append(results())
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    oh = torch.from_numpy(rng.standard_normal((70, 256)).astype(np.float32)).to(DEV)
    ou, ot = torch.full((70,), 0.5, device=DEV), torch.empty(70, dtype=torch.int32, device=DEV)
    torch.cuda.synchronize()
    for _ in range(2):
        for (a, b), want in zip(inputs, eager):
            h.copy_(a)
            u.copy_(b)
            graph.replay()
            with torch.cuda.stream(side):
                other.launch(oh, ou, ot)
            for x, y in zip(results(), want):
                assert torch.equal(x, y)


def test_refusals():
    head = DraftHead(torch.randn(500, 64), max_rows=4, device=DEV)
    h, u = torch.randn(3, 64, device=DEV), torch.full((3,), 0.25, device=DEV)
    tokens = torch.full((3,), -7, dtype=torch.int32, device=DEV)
    one = torch.ones(3, device=DEV)
    bad = [dict(h=torch.randn(5, 64, device=DEV), u=torch.rand(5, device=DEV), tokens=torch.zeros(5, dtype=torch.int32, device=DEV)),
           dict(h=torch.randn(3, 48, device=DEV)), dict(h=torch.randn(64, 3, device=DEV).t()), dict(h=h.half()), dict(h=h.cpu()),
           dict(u=u.double()), dict(u=u[:2]), dict(tokens=tokens.long()), dict(top_k=one), dict(temperature=one.double()),
           dict(probs=torch.zeros(3, 499, device=DEV)), dict(kept=one)]
    for kw in bad:
        with pytest.raises(ValueError):
            head.launch(**{**dict(h=h, u=u, tokens=tokens), **kw})
    with pytest.raises(dcd.DcdError):
        DraftHead(torch.randn(500, 40), max_rows=4, device=DEV)
    with pytest.raises(ValueError):
        DraftHead(torch.randn(500, 64).half(), max_rows=4, device=DEV)
    with pytest.raises(ValueError):
        DraftHead(torch.randn(500, 64), torch.zeros(499), max_rows=4, device=DEV)
    head.launch(h[:0], u[:0], tokens[:0])
    torch.cuda.synchronize()
    assert (tokens == -7).all()
