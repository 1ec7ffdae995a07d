"""How the products of the feed-forward block are divided among workgroups (csrc/hdt_ffn_plan.h, compiled for the host): every tile and every part of k has one
owner, every part a place of its own in the workspace; and the sizes of tests/ffn_cases.py meet the forms they say."""
import os
import shutil
import subprocess

import pytest

import ffn_cases

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
pytestmark = pytest.mark.skipif(shutil.which("g++") is None, reason="no host compiler")


def program(tmp_path, text):
    src, exe = tmp_path / "plan.cpp", tmp_path / "plan"
    src.write_text(text)
    subprocess.run(["g++", "-std=c++17", "-O1", "-I", os.path.join(ROOT, "include"), "-I", os.path.join(ROOT, "paper_2407_08330_amd", "csrc"), str(src), "-o", str(exe)],
                   check=True)
    return str(exe)


WALK = r"""
#include <cmath>
#include <cstdio>
#include <map>
#include <random>
#include <vector>
#include "hdt_ffn_plan.h"
using namespace hdt_ffn;

// the parts that k_ffn_tile's workgroups write, and those that k_ffn_join adds up
static int check(const Plan &p, int bk, size_t tile_bytes, int k, int ranges, bool divisible)
{
    const int k_tiles = ranges * ((k + bk - 1) / bk);
    if (p.direct == p.tiles) return p.parts_bytes != 0 || p.piece_items + p.sharers != 0;
    const unsigned cut = p.tiles - p.direct;
    int bad = !divisible || p.direct > p.tiles || p.piece_items % 8 || p.sharers % 8 || p.per < 1;
    struct Part { unsigned tile; int t0, t1; };
    std::map<size_t, Part> parts;
    auto add = [&](size_t slot, unsigned tile, int t0, int t1) {
        bad += t0 < 0 || t0 >= t1 || t1 > k_tiles || t1 - t0 == k_tiles || tile >= cut || (slot + 1) * tile_bytes > p.parts_bytes;
        bad += !parts.insert({slot, {tile, t0, t1}}).second;
    };
    for (unsigned item = 0; item < p.piece_items; item++) {
        const unsigned piece = item / cut, tile = item - piece * cut;
        if (piece < (unsigned)p.pieces) add(item, tile, piece * p.per, std::min((int)(piece + 1) * p.per, k_tiles));
    }
    for (unsigned me = 0; me < p.sharers; me++) {
        int64_t at = (int64_t)me * p.per;
        const int64_t end = std::min(at + p.per, (int64_t)cut * p.rest);
        while (at < end) {
            const int64_t tile = at / p.rest;
            const int t0 = (int)(at - tile * p.rest), t1 = (int)std::min((int64_t)p.rest, t0 + (end - at)), from = p.pieces * p.per;
            add((size_t)p.pieces * cut + me + tile, (unsigned)tile, from + t0, from + t1);
            at += t1 - t0;
        }
    }
    for (unsigned tile = 0; tile < cut; tile++) {
        const int64_t first = (int64_t)tile * p.rest / p.per, last = p.rest ? ((int64_t)(tile + 1) * p.rest - 1) / p.per : first - 1;
        const int n = p.pieces + (int)(last - first + 1);
        int next = 0;
        bad += n < 2;
        for (int s = 0; s < n; s++) {
            const size_t slot = s < p.pieces ? (size_t)s * cut + tile : (size_t)p.pieces * cut + (size_t)(first + s - p.pieces) + tile;
            const auto it = parts.find(slot);
            if (it == parts.end() || it->second.tile != tile || it->second.t0 != next) { bad++; continue; }
            next = it->second.t1;
            parts.erase(it);
        }
        bad += next != k_tiles;
    }
    return bad + !parts.empty();
}

int main()
{
    std::mt19937 gen(3);
    std::uniform_real_distribution<double> u(0, 1);
    auto size = [&](double most) { return (int)std::exp(u(gen) * std::log(most)); };
    int bad = 0, cut = 0, shared = 0;
    for (int i = 0; i < 20000; i++) {
        const Sizes s = {size(70000.), size(6000.), size(12000.), HDT_BF16};
        const struct { Plan p; int k, ranges; bool divisible; } of[] = {{s.plan_gate(), s.width, 1, false}, {s.plan_down(), s.inner, 1, true}, {s.plan_dgate(), s.width, 1, false},
                                                                        {s.plan_dx(), s.inner, 2, true}, {s.plan_weights(), (int)s.rows, 1, true}};
        for (const auto &c : of) {
            const size_t tile = c.p.shape ? Small::BM * Small::BN * 4 : Large::BM * Large::BN * 4;
            const int b = check(c.p, c.p.shape ? Small::BK : Large::BK, tile, c.k, c.ranges, c.divisible);
            if (b) std::printf("%lld x %d x %d: %d faults\n", (long long)s.rows, s.width, s.inner, b);
            bad += b;
            cut += c.p.direct < c.p.tiles;
            shared += c.p.sharers > 0;
        }
    }
    return bad != 0 || cut < 1000 || shared < 100;
}
"""


def test_every_part_of_a_tile_has_one_owner_and_a_place(tmp_path):
    run = subprocess.run([program(tmp_path, WALK)], stdout=subprocess.PIPE, text=True)
    assert run.returncode == 0, run.stdout[-2000:]


FORMS = r"""
#include <cstdio>
#include <string>
#include "hdt_ffn_plan.h"
using namespace hdt_ffn;

static std::string form(const Plan &p)
{
    return std::string(p.shape ? "S" : "L") + (p.direct ? "D" : "") + (p.tiles > p.direct ? "P" : "") + (p.sharers ? "R" : "");
}
static std::string plain(int64_t tiles) { return std::to_string((int)plain_form(tiles)); }

int main()
{
    int bf16, width, inner;
    long long rows;
    while (std::scanf("%d %lld %d %d", &bf16, &rows, &width, &inner) == 4) {
        const Sizes s = {rows, width, inner, bf16 ? HDT_BF16 : HDT_F32};
        const int m = (int)rows;
        const std::string gate = !bf16 ? plain(plain_tiles({m, inner})) : s.few() ? "few" : form(s.plan_gate());
        const std::string down = !bf16 ? plain(plain_tiles({m, width})) : s.few() ? "few" : form(s.plan_down());
        const std::string dgate = !bf16 ? plain(plain_tiles({m, inner})) : form(s.plan_dgate());
        const std::string dx = !bf16 ? plain(plain_tiles({m, width})) : form(s.plan_dx());
        const std::string weights = !bf16 ? plain(2 * plain_tiles({inner, width}) + plain_tiles({width, inner})) : form(s.plan_weights());
        std::printf("%s %s %s %s %s\n", gate.c_str(), down.c_str(), dgate.c_str(), dx.c_str(), weights.c_str());
    }
}
"""


def test_the_tested_sizes_meet_every_form(tmp_path):
    """A change of the rule that moves a size to another form has to find another size for the form that is left."""
    cases = [(1, *c) for c in ffn_cases.BF16] + [(0, *c) for c in ffn_cases.F32]
    run = subprocess.run([program(tmp_path, FORMS)], input="".join(f"{b} {r} {w} {n}\n" for b, r, w, n, _ in cases), stdout=subprocess.PIPE, text=True, check=True)
    assert run.stdout.splitlines() == [c[-1] for c in cases]
    met = {(product, form, width % 8 == 0 and inner % 8 == 0)
           for _, width, inner, forms in ffn_cases.BF16 for product, form in zip(ffn_cases.PRODUCTS, forms.split())}
    cuts = {"LD", "LP", "LDP", "LPR", "LDPR", "SD", "SP", "SDP", "SPR", "SDPR"}
    want = {"gate": {"few", "LD", "SD"}, "dgate": {"LD", "SD"}, "down": {"few"} | cuts - {"LDPR"}, "dx": cuts, "weights": cuts}  # (no size has been found whose down is LDPR)
    assert met >= {(product, form, even) for product, forms in want.items() for form in forms for even in (True, False)}
    met = {(product, form) for *_, forms in ffn_cases.F32 for product, form in zip(ffn_cases.PRODUCTS, forms.split())}
    assert met == {(product, form) for product in ffn_cases.PRODUCTS for form in "012"}
