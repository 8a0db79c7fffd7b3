"""The waits of the 4-bit kernels' DMA rings on the CPU, as late as they allow: what is read has landed, what is
overwritten has been read, the DMA instructions cover a block and stay inside its rows.

Few rows: a ring of NS blocks of 64 keys for each wave, PB instructions to a block.  Many rows: three raw slots of a
wave, three instructions to a stage (two halves of 16 keys, their scales)."""
import os
import re

import pytest

from test_paged_ring_waits import CSRC, landed


def few_rows(k, mine, slack=0):
    """Reads of a block that had not landed or was not the slot's, with waits that leave `slack` pieces more; the first
    block is waited for as the others are, with the ring's blocks under way."""
    NS, PB = k["NS"], k["PB"]
    bad, flight, asked = 0, [], {}
    for b in range(NS if mine else 0):
        asked[b % NS] = b
        flight += [b] * PB
    for b in range(mine):
        flight = landed(flight, min((NS - 1) * PB + slack, len(flight)))
        bad += asked[b % NS] != b or b in flight
        asked[b % NS] = b + NS  # behind the reads of block b
        flight += [b + NS] * PB
    return bad

def constant(name, const, **known):
    with open(os.path.join(CSRC, name)) as f:
        text = f.read()
    expr = re.search(rf"\b{const} = ([^;,]+)[;,]", text)[1]
    expr = re.sub(r"(\S+) \? (\S.*) : (.+)", r"((\2) if \1 else (\3))", expr).replace("/", "//")
    return eval(expr, {}, known)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("BIG", [False, True])
def test_few_rows(D, BIG):
    k = {"D": D, "BIG": BIG, "NW": 8, "kUnit": 64, "kE2m1Block": 32}
    for c in ("RING", "ROWB", "KB", "TENSOR", "SLOT", "NS", "CPK", "QB", "SPK", "SC", "PT", "PB", "EXPS"):
        k[c] = constant("kernel_paged_few4.h", c, **k)
    lanes, kpi = 64, 1024 // k["ROWB"]
    assert k["NS"] == {64: 4, 128: 2}[D] and k["PB"] == 2 * k["PT"] + 1 and k["PT"] * kpi == 64
    # the instructions make the block, one of SC / 16 lanes its scales
    assert 2 * k["PT"] * 16 * lanes == k["SLOT"] == 64 * 2 * D // 2 and k["SC"] == 64 * 2 * D // 32 and k["SC"] // 16 <= 64
    # (with the queries of three or four tiles)
    assert 48 * 2 * 128 + 8 * (k["RING"] + k["NS"] * k["SC"] + k["EXPS"]) <= 160 * 1024 - 8 * 128  # with m_s and l_s
    # an instruction's lanes cover its rows, each chunk once, where the reads look for it (at D = 64 over small pages
    # two quarters of 16 keys, each on its page: here as if they followed each other)
    kswz = lambda key: key >> 4 & (3 if D == 128 else 1)
    vswz = lambda key: key >> 2 & 3 if D == 128 else key >> 3 & 1
    for i in range(k["PT"]):
        for swz, flip, period in ((kswz, kswz(kpi * i), 64), (vswz, 0, 16)):
            offs = []
            for lane in range(lanes):
                ikey = lane // k["CPK"] % kpi
                off = (ikey * k["ROWB"] + 16 * ((lane % k["CPK"]) ^ swz(ikey % period))) ^ (16 * flip)
                offs.append(off)
                key = kpi * i + 16 * lane // k["ROWB"]  # where the lane's bytes land
                assert off // k["ROWB"] == key - kpi * i and off % k["ROWB"] // 16 == (16 * lane % k["ROWB"] // 16) ^ swz(key % period)
            assert sorted(offs) == list(range(0, 16 * lanes, 16))
    assert not any(few_rows(k, mine) for mine in range(12))
    assert any(few_rows(k, mine, 1) for mine in range(12))  # the model sees a wait that is one piece short


@pytest.mark.parametrize("D", [64, 128])
def test_many_rows(D):
    rows4 = constant("kernel_paged_rows.h", "ROWS4", D=D)
    under_way = constant("kernel_paged_rows.h", "UNDER_WAY", Q4=True, FLIGHT=None)
    assert rows4 + 32 * D // 32 <= 32 * D and under_way == 6  # rows and scales in a raw slot; two stages
    for slack, good in ((0, True), (1, False)):
        bad = 0
        for nst in range(14):
            raw, flight = {st % 3: st for st in range(3)}, []
            for st in range(2):  # turned, then the raw slot asked for again
                raw[(st + 3) % 3] = st + 3
                flight += [st + 3] * 3
            for st in range(nst):
                flight = landed(flight, min(under_way + slack, len(flight)))
                bad += raw[(st + 2) % 3] != st + 2 or (st + 2) in flight
                raw[(st + 5) % 3] = st + 5
                flight += [st + 5] * 3
        assert (bad == 0) == good


@pytest.mark.parametrize("D", [64, 128])
def test_the_turned_rows(D):
    """Every 16-byte chunk of 32 bfloat16 rows is written once, from the word that holds its eight elements, with its scale."""
    c4, turns = D // 32, 16 * D // 1024
    kswz = (lambda key: key & 15) if D == 128 else (lambda key: key >> 1 & 7)
    vswz = (lambda key: (6 * (key & 1)) ^ (12 * (key >> 1 & 1))) if D == 128 else (lambda key: 4 * (key >> 1 & 1))
    for swz in (kswz, vswz):
        seen = {}
        for lane in range(64):
            key0, ch0 = lane // c4, 4 * (lane % c4)
            to = key0 * 2 * D + 16 * (ch0 ^ swz(key0))
            for i in range(turns):
                for j in range(4):
                    at = (to ^ (16 * j)) + i * (64 // c4) * 2 * D
                    key, ch = at // (2 * D), (at % (2 * D)) // 16
                    raw = 16 * lane + 1024 * i + 4 * j      # byte of the raw slot: row, then element pairs
                    assert at not in seen
                    seen[at] = (raw // (D // 2), raw % (D // 2) // 4, 64 * i + lane)
                    assert seen[at] == (key, ch ^ swz(key), key * c4 + (ch ^ swz(key)) // 4)
        assert len(seen) == 32 * D // 8
