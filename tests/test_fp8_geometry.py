"""The CPU model of the many-row 8-bit logits kernel (test_fp8_addresses) has the kernel's own sizes and
index arithmetic: those of csrc/logits_fp8_geo.h, which the kernels include, compiled for the host."""
import ctypes
import os
import subprocess

import numpy as np
import pytest

import test_fp8_addresses as model

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LANE = range(64)


@pytest.fixture(scope="module")
def geo(tmp_path_factory):
    so = str(tmp_path_factory.mktemp("geo") / "geo.so")
    subprocess.check_call(["g++", "-O1", "-std=c++17", "-Wall", "-Werror", "-shared", "-fPIC",
                           "-I", os.path.join(ROOT, "paper_2608_12913_amd", "csrc"),
                           os.path.join(ROOT, "tests", "native", "fp8_geo_capi.cpp"), "-o", so])
    return ctypes.CDLL(so)


def _tile(geo, rb):
    out = (ctypes.c_int * 13)()
    geo.geo_tile(rb, out)
    return dict(zip("TR HSTAGE NW NH WAHEAD HAHEAD SROWS SSTAGE SAT BAT LDS HL HALF".split(), out))


def test_sizes(geo):
    out = (ctypes.c_int * 8)()
    geo.geo_constants(out)
    assert list(out) == [128, 2048, model.TT, 4, 64, model.TT * 128, model.WL, model.SB]


@pytest.mark.parametrize("rb", [4, 6])
def test_rings_and_lds(geo, rb):
    t = _tile(geo, rb)
    assert (t["NW"], t["NH"]) == (model.NW, model.NH)
    assert (t["WAHEAD"], t["HAHEAD"]) == (model.NW - 1, model.NH - 2)
    assert t["TR"] == 32 * rb and t["HL"] == rb // 2 and t["HALF"] == 8 * rb and t["SROWS"] == 8 * rb
    assert t["HSTAGE"] == 2 * 16 * (rb // 2) * 128
    assert t["SAT"] == model.NW * model.TT * 128 + model.NH * t["HSTAGE"]
    assert t["SSTAGE"] == (32 * rb + 64 - 8 * rb) * model.SB * 4
    assert t["BAT"] == t["SAT"] + 2 * t["SSTAGE"] and t["LDS"] == t["BAT"] + model.TT * 4 <= model.CUS_LDS
    rows = sorted(geo.geo_first_row(rb, wv) + 8 * q + geo.geo_half_row(l) + par * t["HALF"]
                  for wv in range(4) for q in range(t["HL"]) for l in LANE[::8] for par in range(2))
    assert rows == list(range(t["TR"]))
    assert [geo.geo_first_row(rb, wv) for wv in range(4)] == [wv // 2 * 16 * rb + wv % 2 * 8 * (rb // 2) for wv in range(4)]


def test_tokens_and_lanes(geo):
    assert [geo.geo_token_of(r) for r in range(64)] == model.token_of(np.arange(64)).tolist()
    for l in LANE:
        assert (geo.geo_half_row(l), geo.geo_half_column(l)) == (l // 8, (l % 8 ^ l // 8) * 16)
        n, g = l % 16, l // 16
        assert geo.geo_piece_at(l) == n * 128 + (g ^ n % 8) * 16


@pytest.mark.parametrize("K", [16, 112, 128, 400, 2000, 4096, 1 << 20])
def test_columns(geo, K):
    last = -(-K // 128) - 1
    for block in {0, last // 2, last}:
        for l in LANE:
            col = geo.geo_half_column(l)
            at = geo.geo_load_column(block, col, K)
            assert at == min(block * 128 + col, K - 16) and 0 <= at <= K - 16


@pytest.mark.parametrize("nb", list(range(1, 40)) + [64, 128, 8192])
def test_walk(geo, nb):
    for tile in list(range(min(2 * nb, 64))) + [500, 1 << 22]:
        start = geo.geo_walk_start(tile, 1, nb)
        assert start == (tile * model.SB % nb if nb % model.SB == 0 else 0)
        assert geo.geo_walk_start(tile, 2, nb) == 0
        for b in list(range(min(nb, 64))) + list(range(nb, nb + model.NW + model.NH)):
            assert geo.geo_walk_block(b, nb, start) == model._block(b, nb, start)
