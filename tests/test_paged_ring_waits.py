"""The waits of the paged kernels' DMA rings on the CPU, as late as they allow (see test_ring_waits.py): what is read has
landed, and what is overwritten has been read.

Few rows: a ring of NS blocks for each wave; the block read is waited for with NS - 1 blocks under way, then block
b + NS is asked for.  Many rows over 8-bit pages: three raw slots of a wave; behind the barrier of stage st the raw
stage st + 2 is turned into the bfloat16 ring of three slots, and then stage st + 5 asked for.
"""
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2607_02963_amd", "csrc")


def constants(name, **known):
    """The integer constants of a kernel, in order, with the template's arguments known."""
    with open(os.path.join(CSRC, name)) as f:
        text = f.read()
    env = {"kFewWaves": int(re.search(r"constexpr int kFewWaves = (\d+)", text)[1]) if "kFewWaves = " in text else 0, **known}
    for decl in re.findall(r"^    constexpr int ([^;]+);", text, re.M):
        for part in re.split(r",\s*(?=\w+ = )", decl):
            left, right = part.split(" = ", 1)
            right = re.sub(r"(\w+) \? ([^:?]+) : (.+)", r"((\2) if \1 else (\3))", re.sub(r"\(FP8 \? 1 : 0\)", "int(FP8)", right))
            right = right.replace("C::NSTAGE", "4").replace("/", "//")
            try:
                env[left] = eval(right, {}, env)
            except NameError:
                pass  # of another kernel's types
    return env


def landed(flight, left):
    """The pieces of a list, oldest first, that may still be under way when a wait leaves `left` of them."""
    return flight[len(flight) - left:] if left else []


def few_rows(k, mine, slack=0):
    """Reads of a block that had not landed or was not the slot's, with waits that leave `slack` pieces more."""
    NS, PB = k["NS"], k["PB"]
    bad, flight = 0, []  # the initial wait is for everything
    asked = {b % NS: b for b in range(NS)} if mine else {}
    for b in range(mine):
        flight = landed(flight, min((NS - 1) * PB + slack, len(flight)))
        bad += asked[b % NS] != b or b in flight
        asked[b % NS] = b + NS  # behind the reads of block b
        flight += [b + NS] * PB
    return bad


def many_rows(k, FP8, nst, slack=0):
    """The same, and slots that were overwritten before all had consumed them."""
    AHEAD, FLIGHT, NB, NRAW, PPW = (k[x] for x in ("AHEAD", "FLIGHT", "NB", "NRAW", "PPW"))
    pieces = PPW + (1 if FP8 else 0)  # a stage's, the scales with them
    bad, flight, ring, raw = 0, [], {st: st for st in range(2 if FP8 else 3)}, {st: st for st in range(3)}
    if FP8:
        for st in range(2):  # turned, then the raw slot asked for again
            raw[(st + 3) % NRAW] = st + 3
            flight += [st + 3] * pieces
    for st in range(nst):
        bad += ring[st % NB] != st  # the stage's first half may be read in front of the barrier
        flight = landed(flight, min(FLIGHT + slack, len(flight)))
        into = st + 2 if FP8 else st + AHEAD
        bad += ring.get(into % NB) not in (None, st - 1)  # consumed by all behind this barrier
        if FP8:
            bad += raw[into % NRAW] != into or into in flight
            raw[(st + AHEAD) % NRAW] = st + AHEAD
        else:
            bad += st + 1 in flight
        ring[into % NB] = into
        flight += [st + AHEAD] * pieces
        bad += ring[(st + 1) % NB] != st + 1
    return bad


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("FP8", [False, True])
@pytest.mark.parametrize("HW", [1, 2])
def test_few_rows(D, FP8, HW):
    k = constants("kernel_paged_few.h", D=D, FP8=FP8, HW=HW, NT=1)
    assert (k["NS"], k["PB"]) == {(64, False): (2, 8), (64, True): (4, 5), (128, False): (1, 16), (128, True): (2, 9)}[D, FP8]
    assert not any(few_rows(k, mine) for mine in range(12))
    assert any(few_rows(k, mine, 1) for mine in range(12))  # the model sees a wait that is one piece short


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("FP8", [False, True])
def test_many_rows(D, FP8):
    k = constants("kernel_paged_rows.h", D=D, FP8=FP8, NT=1)
    assert k["FLIGHT"] < 64 and k["PPW"] == 32 * D * (1 if FP8 else 2) // 1024  # 32 keys in pieces of 1 KB
    assert not any(many_rows(k, FP8, nst) for nst in range(14))
    assert any(many_rows(k, FP8, nst, 1) for nst in range(14))
