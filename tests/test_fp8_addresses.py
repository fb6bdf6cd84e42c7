"""CPU model of the many-row 8-bit logits kernel (csrc/logits_fp8_tile.hip: the walk along K, Loader,
the swizzled reads, token_of and the rings): every block is multiplied once with its own scales, loads
stay inside their rows and fill a stage, each read finds the columns that the swizzle put there, the staged
logits belong to their tokens, and no stage is read before it is waited for or filled while a wave may
still read it."""
import numpy as np
import pytest

SB, NW, NH, WL, TT, CUS_LDS = 4, 2, 5, 8, 256, 160 * 1024
LANE = np.arange(64)


def token_of(r):
    return r // 32 * 32 + r % 16 // 4 * 8 + r // 16 % 2 * 4 + r % 4


def _block(b, nb, start):
    b = min(b, nb - 1) + start
    return b if b < nb else b - nb


@pytest.mark.parametrize("nb", list(range(1, 40)) + [64, 128])
def test_walk_along_k(nb):
    for tile in range(2 * nb):
        start = tile * SB % nb if nb % SB == 0 else 0
        walk = [_block(b, nb, start) for b in range(nb)]
        assert sorted(walk) == list(range(nb))
        assert all(0 <= _block(b, nb, start) < nb for b in range(nb, nb + NW + NH))
        for b in range(0, nb, SB):  # scales are loaded SB blocks at a time, from the first one's
            for j in range(min(SB, nb - b)):
                assert walk[b + j] == walk[b] + j


@pytest.mark.parametrize("K", [16, 112, 128, 400, 2000, 4096])
def test_loads_and_reads_of_weights(K):
    for block in range(-(-K // 128)):
        lds = np.full((64, 8, 2), -1)  # row of a stage, 16-byte slot: (token, column)
        for q in range(WL):
            token = token_of(LANE // 8) + token_of(8 * q) - token_of(0)
            col = (LANE % 8 ^ LANE // 8) * 16
            at = np.minimum(block * 128 + col, K - 16)
            assert (token < 64).all() and (at >= 0).all() and (at + 16 <= K).all()
            byte = q * 1024 + LANE * 16
            lds[byte // 128, byte % 128 // 16] = np.stack([token, col], 1)
        assert (lds >= 0).all() and len(set(lds[:, 0, 0])) == 64
        for v in range(4):
            n, g = LANE % 16, LANE // 16
            at = v * 2048 + n * 128 + (g ^ n % 8) * 16
            for add, want in ((0, 16 * g), (64, 64 + 16 * g)):
                token, col = lds[(at ^ add) // 128, (at ^ add) % 128 // 16].T
                assert (token == token_of(16 * v + n)).all() and (col == want).all()


def test_tokens_of_the_results():
    assert sorted(token_of(np.arange(64))) == list(range(64))
    for i in range(2):
        for g in range(4):
            for j in range(4):
                assert token_of(16 * 2 * i + 4 * g + j) == 32 * i + 8 * g + j
                assert token_of(16 * (2 * i + 1) + 4 * g + j) == 32 * i + 8 * g + 4 + j


@pytest.mark.parametrize("rb", [4, 6, 8])
def test_lds(rb):
    hstage, rows = 2 * 16 * (rb // 2) * 128, 32 * rb
    scales_at = NW * TT * 128 + NH * hstage
    sstage = (rows + 64 - 8 * rb) * SB * 4
    assert max(wv * 8 * rb + 64 for wv in range(4)) * SB * 4 <= sstage
    bias_at = scales_at + 2 * sstage
    assert bias_at + TT * 4 <= CUS_LDS and rows * (512 + 16) <= bias_at
    assert scales_at % 128 == 0 and hstage % 128 == 0
    # a loading wave's hidden states: its rows of either half of the stage, every row once
    got = sorted(wv // 2 * 16 * rb + wv % 2 * 8 * (rb // 2) + 8 * q + lane // 8 + par * 16 * (rb // 2)
                 for wv in range(4) for q in range(rb // 2) for lane in range(0, 64, 8) for par in range(2))
    assert got == list(range(rows))


@pytest.mark.parametrize("nb", range(1, 24))
def test_rings(nb):
    """Slots: waves G = 0 read stage q in slot 2 q and multiply in 2 q + 1, waves G = 1 one slot later.
    landed[s]: the slot at whose end stage s was waited for by the wave that asked for it."""
    weights, rows = {c: -1 for c in range(NW)}, {q: -1 for q in range(NH)}
    asked_w, asked_h = list(range(NW)), list(range(NH))
    read_w, read_h = {}, {}
    done_w, done_h = NW, NH
    for slot in range(4 * nb + 1):
        if slot < 4 * nb:
            q = slot // 2
            if slot % 2 == 0:
                assert rows[q] < slot
                read_h.setdefault(q, []).append(slot)
                if q % 2 == 0:
                    assert weights[q // 2] < slot
                    read_w.setdefault(q // 2, []).append(slot)
                else:  # block q // 2 + NW is asked for, into the stage of block q // 2
                    assert len(read_w[q // 2]) == 2 and max(read_w[q // 2]) < slot
            elif q % 2 == 1:
                asked_w.append(q // 2 + NW)
                for c in asked_w[done_w:len(asked_w) - (NW - 1)]:
                    weights[c] = slot
                done_w = max(done_w, len(asked_w) - (NW - 1))
        if slot % 2 == 1:
            q = (slot - 1) // 2
            assert rows[q] < slot
            read_h[q].append(slot)
            if q % 2 == 0:
                assert weights[q // 2] < slot
                read_w[q // 2].append(slot)
            for h in asked_h[done_h:len(asked_h) - (NH - 2)]:
                rows[h] = slot
            done_h = max(done_h, len(asked_h) - (NH - 2))
        elif slot >= 2:
            q = (slot - 2) // 2
            assert len(read_h[q]) == 2 and max(read_h[q]) < slot  # stage q + NH goes where q was
            asked_h.append(q + NH)
