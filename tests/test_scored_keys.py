"""Routing by scores, rows of up to 256 experts: what sixteen lanes keep of a row's keys while its best experts are chosen (csrc/scored_keys.h), on the
CPU. A driver makes the keys as the kernel does and goes through the rounds lane by lane; every expert that is asked about has to be one of the row."""
import math
import os
import shutil
import subprocess

import numpy as np
import pytest
import torch

from oracle import map_oracle as mo

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

#: a line of sizes, one of biases, then rows: float32 numbers as the whole numbers of their bits
SOURCE = r"""
#include <cmath>
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <vector>
#include "scored_keys.h"
using namespace nomad_router;

static int experts, groups, top_groups, k, softmax, biased, narrow, epc;
static float number() {
    unsigned bits;
    float v;
    if (std::scanf("%u", &bits) != 1) std::exit(2);
    std::memcpy(&v, &bits, 4);
    return v;
}

template <int CAP, int K>
static void row(const std::vector<float>& raw, const std::vector<float>& bias) {
    constexpr int lanes = 16, bits = CAP == 8 ? 7 : 8;
    constexpr uint32_t mask = (1u << bits) - 1u;
    int teams = 1;
    while (teams < groups && teams < lanes) teams *= 2;
    const int team = lanes / teams, size = experts / groups;
    float low = 0.f, high = 0.f;
    if (biased) {
        low = INFINITY;
        high = -INFINITY;
        for (float b : bias) { low = std::fmin(low, b); high = std::fmax(high, b); }
    }
    const float steps = (float)((1ull << (32 - bits)) - 64) / (1.f + (high - low)), slack = 0x1p-21f * (std::fmax(std::fabs(low), std::fabs(high)) + 1.f);
    std::vector<float> c(experts);
    float top = -INFINITY, sum = 0.f, near = 0x1p-21f;
    if (biased && softmax) {
        for (float v : raw) top = std::fmax(top, v);
        for (int e = 0; e < experts; ++e) sum += c[e] = raw[e] > -INFINITY ? std::exp(raw[e] - top) : 0.f;
        near = 1.f / sum * ((float)CAP + 32.f) * 0x1p-23f;
        for (float& v : c) v *= 1.f / sum;
    } else {
        for (int e = 0; e < experts; ++e) c[e] = 1.f / (1.f + std::exp(-raw[e]));
    }
    // open groups, by their best (in 64 bits)
    std::vector<double> score(groups, -INFINITY);
    for (int e = 0; e < experts; ++e)
        if (raw[e] > -INFINITY) {
            double v = raw[e];
            if (biased) {
                double all = 0.0;
                if (softmax) for (float x : raw) all += x > -INFINITY ? std::exp((double)x - top) : 0.0;
                v = (softmax ? std::exp((double)raw[e] - top) / all : 1.0 / (1.0 + std::exp(-(double)raw[e]))) + (double)bias[e];
            }
            if (v > score[e / size]) score[e / size] = v;
        }
    std::vector<bool> open(groups);
    for (int g = 0; g < groups; ++g) {
        int ahead = 0;
        for (int h = 0; h < groups; ++h) ahead += score[h] > score[g] || (score[h] == score[g] && h < g);
        open[g] = score[g] > -INFINITY && ahead < top_groups;
    }
    Kept<CAP, K> kept[lanes];
    for (int lane = 0; lane < lanes; ++lane) {
        const int group = lane / team, from = lane % team * epc;
        uint32_t key[CAP];
        for (int i = 0; i < CAP; ++i) {
            const int at = from + i / epc * (team * epc) + i % epc, e = group * size + at;
            key[i] = 0;
            if (group >= groups || at >= size || !(raw[e] > -INFINITY)) continue;
            if (biased) {
                key[i] = (uint32_t)std::fma(c[e], steps, (bias[e] - low) * steps + 1.f) << bits | (mask - (uint32_t)e);
            } else {
                uint32_t u;
                const float v = raw[e] + 0.f;
                std::memcpy(&u, &v, 4);
                u = u & 0x80000000u ? ~u : u | 0x80000000u;
                key[i] = (u & ~mask) | (mask - (uint32_t)e);
            }
        }
        kept[lane].keep(key, group < groups && open[group]);
    }
    const uint32_t apart = biased ? (uint32_t)std::fmin((near + slack) * steps, 1e9f) + 2u : 0u;
    int astray = 0;
    const auto same = [&](uint32_t a, uint32_t b) {
        const uint32_t ea = mask - (a & mask), eb = mask - (b & mask);
        if (ea >= (uint32_t)experts || eb >= (uint32_t)experts) { ++astray; return false; }
        return raw[ea] == raw[eb] && (!biased || bias[ea] == bias[eb]);
    };
    const bool exact = !biased && narrow;
    bool sure = true;
    int chosen[K];
    uint32_t last = 0, before = 0;
    for (int j = 0; j < k; ++j) {
        uint32_t best = 0;
        for (int lane = 0; lane < lanes; ++lane) best = kept[lane].list[0] > best ? kept[lane].list[0] : best;
        for (int lane = 0; lane < lanes; ++lane) kept[lane].give(best);
        chosen[j] = best ? (int)(mask - (best & mask)) : -1;
        if (chosen[j] >= experts) ++astray;
        if (!exact && best && before && (before >> bits) - (best >> bits) <= apart && !same(before, best)) sure = false;
        before = best;
        if (j == k - 1) last = best;
    }
    if (!exact)
        for (int lane = 0; lane < lanes; ++lane)
            if (kept[lane].unsure(last, apart, bits, same)) sure = false;
    std::printf("%d %d", (int)sure, astray);
    for (int j = 0; j < k; ++j) std::printf(" %d", chosen[j]);
    std::printf("\n");
}

int main() {
    int rows;
    while (std::scanf("%d %d %d %d %d %d %d %d %d", &rows, &experts, &groups, &top_groups, &k, &softmax, &biased, &narrow, &epc) == 9) {
        std::vector<float> bias(experts), raw(experts);
        for (float& b : bias) b = number();
        int teams = 1;
        while (teams < groups && teams < 16) teams *= 2;
        const int each = 16 / teams * epc, held = (experts / groups + each - 1) / each * epc;
        for (int i = 0; i < rows; ++i) {
            for (float& v : raw) v = number();
            if (held > 16) return 3;
            if (held <= 8 && k <= 2) row<8, 2>(raw, bias);
            else if (held <= 8) row<8, 8>(raw, bias);
            else if (k <= 2) row<16, 2>(raw, bias);
            else row<16, 8>(raw, bias);
        }
    }
    return 0;
}
"""


@pytest.fixture(scope="module")
def choose(tmp_path_factory):
    """What the lanes choose of rows (float32 numbers of `dtype`): experts, whether they are sure of them, how often something that is no expert was asked about."""
    if not shutil.which("g++"):
        pytest.skip("no C++ compiler")
    at = tmp_path_factory.mktemp("keys")
    (at / "keys.cpp").write_text(SOURCE)
    exe = str(at / "keys")
    subprocess.run(["g++", "-O2", "-std=c++17", "-ffp-contract=off", "-Wno-unknown-pragmas", "-I" + os.path.join(ROOT, "paper_2505_15511_amd", "csrc"), str(at / "keys.cpp"), "-o", exe], check=True)

    def run(rows, k, dtype=torch.float32, score="sigmoid", bias=None, groups=1, top_groups=1):
        rows = np.ascontiguousarray(rows, np.float32)
        n, experts = rows.shape
        vec = 4 if dtype == torch.float32 else 8
        epc = vec if experts // groups % vec == 0 else 1
        told = np.zeros(experts, np.float32) if bias is None else np.ascontiguousarray(bias, np.float32)
        text = f"{n} {experts} {groups} {top_groups} {k} {int(score == 'softmax')} {int(bias is not None)} {int(dtype != torch.float32)} {epc}\n"
        text += "\n".join(" ".join(map(str, line.view(np.uint32).tolist())) for line in (told, *rows)) + "\n"
        said = np.array([line.split() for line in subprocess.run([exe], input=text, capture_output=True, text=True, check=True).stdout.splitlines()], dtype=np.int64)
        return said[:, 2:], said[:, 0].astype(bool), said[:, 1]
    return run


def of(dtype, rows):
    return torch.from_numpy(np.ascontiguousarray(rows, np.float32)).to(dtype).float().numpy()


def peaked(rng, n, experts, spread, low):
    """Rows whose scores are all but zero for most experts."""
    return spread * rng.normal(size=(n, experts)) + low


@pytest.mark.parametrize("experts", [8, 50, 64, 100, 128, 160, 200, 256])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
def test_only_experts_of_the_row_are_asked_about(choose, experts, dtype):
    rng = np.random.default_rng(experts)
    zero, some = np.zeros(experts, np.float32), (1e-3 * rng.integers(0, 3, experts)).astype(np.float32)
    for score, spread, low in (("softmax", 6.0, 0.0), ("softmax", 30.0, 0.0), ("sigmoid", 1.0, -18.0), ("sigmoid", 0.0, -200.0), ("sigmoid", 5.0, 0.0)):
        for k in (1, 2, 3, 8):
            rows = of(dtype, peaked(rng, 30, experts, spread, low))
            rows[::5, 1:] = -math.inf                                     # fewer than are asked for
            rows[1] = -math.inf
            for bias in (zero, some, None):
                _, _, astray = choose(rows, k, dtype, score, bias)
                assert not astray.any(), (score, spread, low, k)
                if experts % 4 == 0:
                    assert not choose(rows, k, dtype, score, bias, groups=4, top_groups=min(4, 4 * k // experts + 1))[2].any()


def right(rows, k, score="sigmoid", bias=None, groups=1, top_groups=1):
    return mo.route_scored(rows, k, score=score, bias=bias, groups=groups, top_groups=top_groups)[0]


def test_what_a_lane_lets_go_may_be_the_best(choose):
    """As many equal logits in one lane as it keeps, and one more in it that is larger by less than a key holds."""
    def row(experts, equal, value, at, larger, rest):
        x = np.full((1, experts), rest, np.float32)
        x[0, :equal], x[0, at] = value, larger
        return x
    up = np.nextafter(np.float32(6.0), np.float32(7.0))
    for x, k, dtype, biased, want in ((row(128, 4, 1.0, 64, 1 + 2.0 ** -18, 0.0), 1, torch.float32, False, [64]), (row(128, 4, 1.0, 64, 1 + 2.0 ** -18, 0.0), 2, torch.float32, False, [64, 0]),
                                      (row(64, 4, 20.0, 4, 21.0, 0.0), 2, torch.bfloat16, True, [4, 0]), (row(128, 4, 6.0, 64, up, 0.0), 1, torch.float32, True, [64]),
                                      (row(256, 4, 1.0, 128, 1 + 2.0 ** -18, 0.0), 3, torch.float32, False, [128, 0, 1])):
        if k == 3:
            x[0, [64, 65, 66, 67]] = 1.0                                  # eight in all
        bias = np.zeros(x.shape[1], np.float32) if biased else None
        assert right(x, k, bias=bias).tolist() == [want]
        said, sure, _ = choose(x, k, dtype, bias=bias)
        assert not sure[0] or said.tolist() == [want], (k, dtype, said)


@pytest.mark.parametrize("experts", [50, 64, 128, 200, 256])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("score", ["sigmoid", "softmax"])
def test_lanes_that_are_sure_are_right(choose, experts, dtype, score):
    """Rows that repeat one logit, some of them moved by a few units; others saturated or all but zero."""
    rng = np.random.default_rng(experts)
    zero, two, some = (np.asarray(b, np.float32) for b in (np.zeros(experts), 0.25 * (np.arange(experts) % 2), 0.02 * rng.normal(size=experts)))
    kinds = []
    for value in (1.0, 6.0, 17.0, -9.0):
        x = np.full((20, experts), value, np.float32)
        moved = rng.random(x.shape) < np.array([0.02, 0.1, 0.5, 1.0])[rng.integers(0, 4, 20)][:, None]
        x = np.where(moved, x.view(np.int32) + rng.integers(-200, 201, x.shape), x.view(np.int32)).astype(np.int32).view(np.float32)
        kinds.append(np.where(rng.random(x.shape) < np.array([0.0, 0.5, 0.9])[rng.integers(0, 3, 20)][:, None], value - 5.0, x).astype(np.float32))
    kinds += [rng.integers(-3, 4, (20, experts)) * 7.0, peaked(rng, 20, experts, 6.0, 0.0), peaked(rng, 20, experts, 1.0, 30.0)]
    rows = of(dtype, np.concatenate(kinds))
    rows[::9, experts // 3:] = -math.inf
    for bias in (None, zero, two, some):
        for groups, top in ((1, 1), (4, 2), (2, 1)) if experts % 4 == 0 else ((1, 1),):
            want = right(rows, 8, score, bias, groups, top)
            for k in (1, 2, 3, 8):
                said, sure, _ = choose(rows, k, dtype, score, bias, groups, top)
                assert np.array_equal(said[sure], want[sure, :k]), (k, groups)


@pytest.mark.parametrize("experts,groups,top,k", [(256, 1, 1, 2), (256, 8, 4, 8), (256, 16, 1, 8), (50, 5, 2, 3), (128, 1, 1, 1)])
def test_lanes_are_sure_of_ordinary_rows(choose, experts, groups, top, k):
    """Two sums of some hundred in a range of about two are closer than 10^-5 in one of a hundred rows at most; also where one lane has all that is chosen."""
    rng = np.random.default_rng(experts + k)
    rows, bias = rng.normal(size=(400, experts)).astype(np.float32), (0.1 * rng.normal(size=experts)).astype(np.float32)
    said, sure, _ = choose(rows, k, bias=bias, groups=groups, top_groups=top)
    assert sure.mean() > 0.95 and np.array_equal(said[sure], right(rows, k, bias=bias, groups=groups, top_groups=top)[sure])
