"""Refusals of the 8-bit proposal path's entry points: every one is decided on the host,
before anything is launched."""
import ctypes

import numpy as np
import pytest

import proposal_oracle as oracle
from paper_2608_12913_amd import dcd

buf = (ctypes.c_char * 8192)()
A = (ctypes.addressof(buf) + 255) // 256 * 256  # never dereferenced


def _code(call, *a, **kw):
    with pytest.raises(dcd.DcdError) as e:
        call(*a, **kw)
    return e.value.code


def test_struct_layouts_match_the_header(tmp_path):
    import os
    import subprocess
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    structs = {"dcd_fp8_problem": dcd.Fp8Problem, "dcd_fp8_inputs": dcd.Fp8Inputs,
               "dcd_sample_problem": dcd.SampleProblem, "dcd_sample_inputs": dcd.SampleInputs,
               "dcd_sample_outputs": dcd.SampleOutputs}
    lines = ["#include <stdio.h>", "#include <stddef.h>", '#include "dcd.h"', "int main(void) {"]
    for cname, py in structs.items():
        lines.append(f'printf("{cname} size %zu\\n", sizeof({cname}));')
        lines += [f'printf("{cname} {f} %zu\\n", offsetof({cname}, {f}));' for f, _ in py._fields_]
    src, exe = tmp_path / "layout.c", tmp_path / "layout"
    src.write_text("\n".join(lines + ["return 0;", "}"]) + "\n")
    subprocess.check_call(["gcc", "-std=c11", "-I", os.path.join(root, "include"), str(src), "-o", str(exe)])
    got = {tuple(l.split()[:2]): int(l.split()[2])
           for l in subprocess.check_output([str(exe)], text=True).splitlines()}
    for cname, py in structs.items():
        assert got[(cname, "size")] == ctypes.sizeof(py)
        for f, _ in py._fields_:
            assert got[(cname, f)] == getattr(py, f).offset, (cname, f)


@pytest.mark.parametrize("kw, code", [
    (dict(rows=-1), dcd.DCD_ERR_SHAPE), (dict(cols=0), dcd.DCD_ERR_SHAPE), (dict(rows=1 << 31), dcd.DCD_ERR_SHAPE),
    (dict(cols=(1 << 20) + 16), dcd.DCD_ERR_SHAPE), (dict(rows=1 << 30, cols=256), dcd.DCD_ERR_SHAPE),
    (dict(rows=1 << 28, cols=4096, block_rows=128), dcd.DCD_ERR_SHAPE), (dict(dtype=5), dcd.DCD_ERR_PARAM),
    (dict(block_rows=64), dcd.DCD_ERR_PARAM), (dict(cols=200), dcd.DCD_ERR_ALIGN), (dict(x=None), dcd.DCD_ERR_NULL),
    (dict(q=None), dcd.DCD_ERR_NULL), (dict(scale=None), dcd.DCD_ERR_NULL), (dict(x=A + 8), dcd.DCD_ERR_ALIGN),
    (dict(q=A + 4), dcd.DCD_ERR_ALIGN), (dict(scale=A + 2), dcd.DCD_ERR_ALIGN)])
def test_quantize_refusals(kw, code):
    a = dict(x=A, q=A, scale=A, rows=8, cols=256)
    a.update(kw)
    assert _code(dcd.quantize_fp8, **a) == code


def test_nothing_to_do():
    """No rows: no pointer is looked at and nothing is launched."""
    dcd.quantize_fp8(None, None, None, rows=0, cols=256)
    dcd.logits_fp8(dcd.make_fp8_problem(0, 100, 64), dcd.make_fp8_inputs(None, None, None, None), None)
    dcd.sample(dcd.make_sample_problem(0, 100), dcd.make_sample_inputs(None, None), dcd.make_sample_outputs(None),
               None, 0)


@pytest.mark.parametrize("prob, ins, out, code", [
    (dict(rows=-1), {}, A, dcd.DCD_ERR_SHAPE), (dict(vocab=0), {}, A, dcd.DCD_ERR_SHAPE),
    (dict(hidden=0), {}, A, dcd.DCD_ERR_SHAPE), (dict(rows=(1 << 24) + 1), {}, A, dcd.DCD_ERR_SHAPE),
    (dict(vocab=(1 << 30) + 1), {}, A, dcd.DCD_ERR_SHAPE), (dict(hidden=(1 << 20) + 16), {}, A, dcd.DCD_ERR_SHAPE),
    (dict(stride=99), {}, A, dcd.DCD_ERR_SHAPE), (dict(stride=-1), {}, A, dcd.DCD_ERR_SHAPE),
    (dict(dtype=2), {}, A, dcd.DCD_ERR_PARAM), (dict(hidden=72), {}, A, dcd.DCD_ERR_ALIGN),
    ({}, dict(h=None), A, dcd.DCD_ERR_NULL), ({}, dict(h_scale=None), A, dcd.DCD_ERR_NULL),
    ({}, dict(w=None), A, dcd.DCD_ERR_NULL), ({}, dict(w_scale=None), A, dcd.DCD_ERR_NULL),
    ({}, {}, None, dcd.DCD_ERR_NULL), ({}, dict(h=A + 8), A, dcd.DCD_ERR_ALIGN),
    ({}, dict(w=A + 8), A, dcd.DCD_ERR_ALIGN), ({}, dict(bias=A + 2), A, dcd.DCD_ERR_ALIGN),
    ({}, dict(h_scale=A + 1), A, dcd.DCD_ERR_ALIGN), ({}, {}, A + 2, dcd.DCD_ERR_ALIGN),
    (dict(dtype="bf16"), {}, A + 1, dcd.DCD_ERR_ALIGN)])
def test_logits_refusals(prob, ins, out, code):
    p = dict(rows=4, vocab=100, hidden=64)
    p.update(prob)
    i = dict(h=A, h_scale=A, w=A, w_scale=A, bias=A)
    i.update(ins)
    assert _code(dcd.logits_fp8, dcd.make_fp8_problem(**p), dcd.make_fp8_inputs(**i), out) == code


@pytest.mark.parametrize("prob, ins, outs, ws, code", [
    (dict(rows=-1), {}, {}, A, dcd.DCD_ERR_SHAPE), (dict(vocab=0), {}, {}, A, dcd.DCD_ERR_SHAPE),
    (dict(rows=(1 << 24) + 1), {}, {}, A, dcd.DCD_ERR_SHAPE), (dict(stride=99), {}, {}, A, dcd.DCD_ERR_SHAPE),
    (dict(vocab=(1 << 30) + 1), {}, {}, A, dcd.DCD_ERR_SHAPE), (dict(dtype=9), {}, {}, A, dcd.DCD_ERR_PARAM),
    ({}, dict(logits=None), {}, A, dcd.DCD_ERR_NULL), ({}, dict(u=None), {}, A, dcd.DCD_ERR_NULL),
    ({}, {}, dict(tokens=None), A, dcd.DCD_ERR_NULL), ({}, dict(logits=A + 2), {}, A, dcd.DCD_ERR_ALIGN),
    (dict(dtype="bf16"), dict(logits=A + 1), {}, A, dcd.DCD_ERR_ALIGN),
    ({}, dict(u=A + 2), {}, A, dcd.DCD_ERR_ALIGN), ({}, dict(top_k=A + 2), {}, A, dcd.DCD_ERR_ALIGN),
    ({}, {}, dict(probs=A + 2), A, dcd.DCD_ERR_ALIGN), ({}, {}, dict(kept=A + 1), A, dcd.DCD_ERR_ALIGN),
    ({}, {}, {}, None, dcd.DCD_ERR_WORKSPACE), ({}, {}, {}, A + 16, dcd.DCD_ERR_WORKSPACE)])
def test_sample_refusals(prob, ins, outs, ws, code):
    p = dict(rows=4, vocab=100)
    p.update(prob)
    i = dict(logits=A, u=A, temperature=A, top_k=A, top_p=A, min_p=A)
    i.update(ins)
    o = dict(tokens=A, probs=A, logprob=A, kept=A)
    o.update(outs)
    problem = dcd.make_sample_problem(**p)
    need = dcd.sample_workspace_bytes(problem)
    bad_problem = bool(prob) and "dtype" not in prob or prob.get("dtype") == 9
    assert (need == 0) == bool(bad_problem)
    assert _code(dcd.sample, problem, dcd.make_sample_inputs(**i), dcd.make_sample_outputs(**o), ws,
                 max(need, 1)) == code


def test_sample_workspace_too_small():
    p = dcd.make_sample_problem(4, 1000)
    need = dcd.sample_workspace_bytes(p)
    assert need > 0
    assert _code(dcd.sample, p, dcd.make_sample_inputs(A, A), dcd.make_sample_outputs(A), A,
                 need - 1) == dcd.DCD_ERR_WORKSPACE


# the oracle itself, on worked examples

def test_oracle_codes():
    v = oracle.e4m3_values()
    assert v[0] == 0 and v[1] == 2.0 ** -9 and v[8] == 2.0 ** -6 and v[126] == 448 and v[0x38] == 1.0
    import torch
    t = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(oracle.decode(np.arange(256, dtype=np.uint8)), t, equal_nan=True)
    # 448 / 448 = 1: codes are the values themselves; 17 lies between 16 and 18 (even: 16), 19 goes to 20
    x = np.zeros((1, 128))
    x[0, :5] = [448, 17, 19, -21, 2.0 ** -10]
    q, s = oracle.quantize(x, 1)
    assert s[0, 0] == 1 and oracle.decode(q)[0, :5].tolist() == [448, 16, 20, -20, 0]


def test_oracle_sample_by_hand():
    """Probabilities 0.5, 0.25, 0.125, 0.125 in the order of ids 2, 0, 1, 3."""
    z = np.log(np.array([0.25, 0.125, 0.5, 0.125]))
    t, n, p, lp = oracle.sample_row(z, 0.0)
    assert (t, n) == (0, 4) and np.allclose(p, [0.25, 0.125, 0.5, 0.125]) and np.isclose(lp, np.log(0.25))
    assert oracle.sample_row(z, 0.26)[0] == 1 and oracle.sample_row(z, 0.38)[0] == 2
    assert oracle.sample_row(z, 0.9, k=2)[:2] == (2, 2)
    assert oracle.sample_row(z, 0.2, k=3)[:2] == (0, 3)  # ids 1 and 3 tie: the lower one stays
    assert oracle.sample_row(z, 0.5, p=0.6)[:2] == (2, 2)
    assert oracle.sample_row(z, 0.5, m=0.3)[:2] == (2, 2)
    assert oracle.sample_row(z, 0.9, T=0.0)[:2] == (2, 1)
    assert oracle.sample_row(np.full(3, -np.inf), 0.5)[:2] == (-1, 0)
