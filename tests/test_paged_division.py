"""The division of a paged attention call's work (csrc/paged_common.h) on the CPU, 64 lanes of a wave in step.

Lengths within the contract: every pair's units are taken once, and the finish pass's note names the slots that its
states lie in.  Lengths outside it: what a work-group takes lies inside the arrays all the same, also where the units of
all pairs together pass 32 bits.
"""
import os
import shutil
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2607_02963_amd", "csrc")

# What paged_common.h takes from the device: one fiber per lane, and an operation across lanes passes the turn round
# the ring of fibers once.  Two buffers: a lane may be an operation ahead of the others.
WAVE = r"""
#pragma once
#include <algorithm>
#include <cstdint>
#include <cstdio>
#include <cstdlib>
#include <functional>
#include <vector>
#include <ucontext.h>
#define __device__
using std::max;
using std::min;
struct int4 { int x, y, z, w; };
inline int4 make_int4(int x, int y, int z, int w) { return {x, y, z, w}; }
struct Wave {
    ucontext_t main, lane[64];
    std::vector<char> stacks = std::vector<char>(64 << 16);
    int at = 0, live = 0, turn[64];
    uint32_t val[2][64];
    std::function<void()> body;
};
inline Wave W;
inline void wave_step()
{
    const int me = W.at;
    W.at = (me + 1) % 64;
    swapcontext(&W.lane[me], &W.lane[W.at]);
}
inline const uint32_t* wave_all(uint32_t x)
{
    const int me = W.at, b = W.turn[me]++ & 1;
    W.val[b][me] = x;
    wave_step();
    return W.val[b];
}
inline void wave_entry()
{
    W.body();
    const int me = W.at;
    W.at = me + 1;
    if (me < 63) setcontext(&W.lane[me + 1]);
    setcontext(&W.main);  // every lane has left after the same operation
}
inline void wave_run(std::function<void()> f)
{
    W.body = f;
    for (int i = 0; i < 64; ++i) {
        W.turn[i] = 0;
        getcontext(&W.lane[i]);
        W.lane[i].uc_stack.ss_sp = &W.stacks[(size_t)i << 16];
        W.lane[i].uc_stack.ss_size = 1 << 16;
        W.lane[i].uc_link = nullptr;
        makecontext(&W.lane[i], wave_entry, 0);
    }
    W.at = 0;
    swapcontext(&W.main, &W.lane[0]);
}
inline uint32_t __builtin_amdgcn_mbcnt_lo(uint32_t, uint32_t) { return 0; }
inline uint32_t __builtin_amdgcn_mbcnt_hi(uint32_t, uint32_t) { return (uint32_t)W.at; }
template <typename T> T __shfl_up(T x, int off)
{
    const int me = W.at;
    const uint32_t* v = wave_all((uint32_t)x);
    return me >= off ? (T)v[me - off] : x;
}
inline int __builtin_amdgcn_readlane(int x, int i) { return (int)wave_all((uint32_t)x)[i]; }
inline uint64_t __ballot(bool p)
{
    const uint32_t* v = wave_all(p);
    uint64_t b = 0;
    for (int i = 0; i < 64; ++i) b |= (uint64_t)v[i] << i;
    return b;
}
inline uint32_t __builtin_elementwise_add_sat(uint32_t x, uint32_t y) { return x + y < x ? ~0u : x + y; }
inline float __uint_as_float(uint32_t x) { return __builtin_bit_cast(float, x); }
typedef void* hipStream_t;
namespace pdec { constexpr int kUnit = 64; }
"""

MAIN = r"""
#include "paged_common.h"
#include <cstring>
#include <map>
#include <random>
using namespace pdec;

#define CHECK(c) do { if (!(c)) { std::printf("failed: %s (line %d)\n", #c, __LINE__); std::exit(1); } } while (0)

struct Call {
    PagedArgs a;
    std::vector<int32_t> cu, lens;
    std::vector<int4> cut;
    Call(int S, int T, int G, int H_kv, int rows, int max_chunk, int max_len, int causal, int workers, int pad, int least)
        : cu(S + 1, 0), lens(S, 0)
    {
        std::memset(&a, 0, sizeof(a));
        a.num_seqs = S, a.num_tokens = T, a.G = G, a.H_kv = H_kv, a.H_q = G * H_kv, a.rows = rows, a.heads = 1;
        a.max_chunk = max_chunk, a.max_len = max_len, a.causal = causal, a.workers = workers, a.pad = pad, a.least = least;
        a.rows_from = 0, a.rows_to = INT32_MAX;
        a.groups = ((int64_t)max_chunk * G + rows - 1) / rows;
        a.by_pair = (int64_t)S * a.groups * H_kv <= workers;
        a.blocks = workers;
        cut.assign(workers, {-9, -9, -9, -9});
        a.cu_tokens = cu.data(), a.seq_lens = lens.data(), a.cut = cut.data();
    }
    // f(work-group, part) for every part, in a work-group's order
    template <typename F> void parts(F f, const std::vector<int>& which = {})
    {
        auto one = [&](int w) {
            std::vector<PagedPart> got;
            wave_run([&] {
                PagedRun run;
                PagedPart part;
                const int me = paged_lane();
                if (!paged_begin(a, w, run, me == 0)) return;
                for (int64_t n = 0; paged_next(a, run, part); ++n) {
                    CHECK(n <= (int64_t)a.num_seqs * a.groups * a.H_kv);
                    if (me == 0) {
                        paged_note(a, run, part);
                        got.push_back(part);
                    }
                }
            });
            for (auto& p : got) f(w, p);
        };
        if (which.empty()) for (int w = 0; w < a.workers; ++w) one(w);
        else for (int w : which) one(w);
    }
    void inside(const PagedPart& p) const
    {
        CHECK(p.head >= 0 && p.head < a.H_kv && p.s >= 0 && p.s < a.num_seqs && p.group >= 0 && p.group < a.groups);
        const PagedSeq x = paged_seq(a, p.s);
        CHECK(x.t0 == p.seq.t0 && x.n == p.seq.n && x.L == p.seq.L);
        CHECK(p.u0 >= 0 && p.u0 < p.u1 && p.u1 <= paged_units_of(a, x, p.group));
        CHECK(p.slot >= 0 && p.slot < 2 * a.workers);
    }
};

// Every unit once, and the notes name the slots of a cut pair's states in order.
void covers(Call& c)
{
    const PagedArgs& a = c.a;
    struct Piece { int w, u0, u1, slot; };
    std::map<long, std::vector<Piece>> by;
    const long J = (long)a.num_seqs * a.groups;
    c.parts([&](int w, const PagedPart& p) {
        c.inside(p);
        by[p.head * J + (long)p.s * a.groups + p.group].push_back({w, p.u0, p.u1, p.whole ? -1 : p.slot});
    });
    std::map<long, int4> notes;
    for (int i = 0; i < a.workers; ++i) {
        const int4 n = c.cut[i];
        if (a.by_pair && (i >= J * a.H_kv || paged_units(a, i % J) == 0)) continue;
        CHECK(n.x != -9);
        if (n.x >= 0) CHECK(notes.emplace(n.w * J + n.z, n).second);
    }
    for (long k = 0; k < J * a.H_kv; ++k) {
        const int units = paged_units(a, k % J);
        auto& v = by[k];
        int u = 0;
        for (auto& x : v) {
            CHECK(x.u0 == u);
            u = x.u1;
        }
        CHECK(u == units);
        if (v.size() <= 1) {
            CHECK(notes.count(k) == 0 && (v.empty() || v[0].slot == -1));
            continue;
        }
        CHECK(notes.count(k) == 1);
        const int4 n = notes[k];
        CHECK(n.y - n.x + 1 == (int)v.size());
        for (int i = 0; i < (int)v.size(); ++i) CHECK(v[i].w == n.x + i && v[i].slot == 2 * (n.x + i) + (i == 0 ? 1 : 0));
    }
}

int main(int argc, char** v)
{
    std::mt19937 rng(atoi(v[2]));
    auto in = [&](int lo, int hi) { return lo + (int)(rng() % (unsigned)(hi - lo + 1)); };
    if (!strcmp(v[1], "batches")) {
        for (int i = 0; i < 12; ++i) {
            const bool many = i % 3 == 2;
            const int S = many ? in(17, 400) : in(1, 60), most = many ? in(100, 900) : in(1, 200);
            const int rows = 16 << in(0, 4), G = in(1, 8), H_kv = in(1, 4), max_len = in(300, 5000);
            std::vector<int> n(S);
            int T = 0;
            for (int& x : n) T += x = in(0, 3) ? in(0, 2) : in(0, most);
            if (T == 0) T = n[0] = 1;
            Call c(S, T + in(0, 5), G, H_kv, rows, *std::max_element(n.begin(), n.end()), max_len, in(0, 1), 8 * in(1, 20), in(0, 6), in(1, 4));
            for (int s = 0; s < S; ++s) c.cu[s + 1] = c.cu[s] + n[s], c.lens[s] = in(0, max_len);
            covers(c);
        }
    } else if (!strcmp(v[1], "junk")) {  // any lengths at all
        for (int i = 0; i < 12; ++i) {
            const int S = in(1, 300), T = in(1, 3000), rows = 16 << in(0, 4), G = in(1, 8), H_kv = in(1, 4);
            Call c(S, T, G, H_kv, rows, in(1, T), in(300, 5000), in(0, 1), 8 * in(1, 12), in(0, 6), in(1, 4));
            auto any = [&] { const int k = in(0, 5); return k == 0 ? INT32_MIN : k == 1 ? INT32_MAX : k == 2 ? -in(0, 9) : in(0, 2 * T); };
            for (int& x : c.cu) x = any();
            for (int& x : c.lens) x = any();
            c.parts([&](int, const PagedPart& p) { c.inside(p); });
        }
    } else {
        // Every second of S sequences has all of the call's tokens: the units of a head are
        // 2^19 (u + pad) in all for S = 128, so u is chosen for what 32 bits leave of them, and of 8 heads' of them.
        const int T = 1 << 18, G = 8, rows = 256, H_kv = atoi(v[3]), pad = 6, groups = T / rows * G;
        for (int64_t total : {(int64_t)1 << 30, ((int64_t)1 << 31) - (1 << 19), (int64_t)1 << 31, ((int64_t)1 << 32) - ((int64_t)600 << 19),
                              (int64_t)1 << 32, ((int64_t)1 << 32) + (1 << 28), ((int64_t)3 << 31) + (1 << 30), ((int64_t)1 << 33) - (1 << 19)}) {
            const int u = (int)(total / 64 / groups) - pad;
            Call c(128, T, G, H_kv, rows, T, u * 64, 0, 256, pad, 4);
            if (((int64_t)T * G / rows + 128) * H_kv * (u + pad + 1) > INT32_MAX / 2) continue;  // refused on the host
            for (int s = 0; s < 128; ++s) c.cu[s + 1] = s % 2 ? 0 : T, c.lens[s] = u * 64;
            c.parts([&](int, const PagedPart& p) { c.inside(p); }, {0, 1, 100, 255});
        }
    }
    std::printf("ok\n");
}
"""


@pytest.fixture(scope="module")
def program(tmp_path_factory):
    if shutil.which("g++") is None:
        pytest.skip("g++ not found")
    d = tmp_path_factory.mktemp("division")
    shutil.copy(os.path.join(CSRC, "paged_common.h"), d)
    (d / "pdec_common.h").write_text(WAVE)
    (d / "main.cpp").write_text(MAIN)
    exe = str(d / "division")
    subprocess.run(["g++", "-std=c++17", "-O1", "-g", "-fwrapv", "-Wno-attributes", str(d / "main.cpp"), "-o", exe], check=True)
    return exe


def _run(*cmd):
    r = subprocess.run(cmd, capture_output=True, text=True, timeout=240)
    assert r.returncode == 0 and "ok" in r.stdout, (r.returncode, r.stdout, r.stderr[-500:])


@pytest.mark.parametrize("seed", range(4))
def test_every_unit_is_taken_once_and_the_notes_name_its_states(program, seed):
    _run(program, "batches", str(seed))


@pytest.mark.parametrize("seed", range(4))
def test_lengths_outside_the_contract(program, seed):
    _run(program, "junk", str(seed))


@pytest.mark.parametrize("H_kv", [1, 2, 8])
def test_lengths_whose_units_pass_32_bits(program, H_kv):
    _run(program, "past32", "0", str(H_kv))
