"""Which kernel computes a router's logits, and what its work buffer holds, for devices of any number of compute units."""
import os
import subprocess

import pytest

from paper_2304_09049_amd import binding as dg
from paper_2304_09049_amd.build import CSRC

PROGRAM = """
#include <stdio.h>
#include "dg_route_rule.h"
int main()
{
    long long T, E, K, units;
    while (scanf("%lld %lld %lld %lld", &T, &E, &K, &units) == 4)
        printf("%d %zu\\n", (int)dg_route_form(T, E, K, units), dg_route_work_bytes(T, E));
    return 0;
}
"""
ONE, FOUR, TILES16, PARTS16, TILES32 = range(5)


@pytest.fixture(scope="module")
def rule(tmp_path_factory):
    at = tmp_path_factory.mktemp("rule")
    (at / "rule.cpp").write_text(PROGRAM)
    subprocess.run(["g++", "-std=c++17", "-Wall", "-Werror", "-I", CSRC, str(at / "rule.cpp"), "-o", str(at / "rule")], check=True)

    def ask(calls):
        out = subprocess.run([str(at / "rule")], input="\n".join(" ".join(map(str, c)) for c in calls), capture_output=True, text=True, check=True).stdout
        return [tuple(map(int, line.split())) for line in out.splitlines()]
    return ask


def test_a_form_and_the_buffer_that_it_writes(rule):
    """Parts leave four sums in binary64 for each token and expert, all others a logit: on a device of few units too, where tiles of 32 x 32 suffice as well."""
    calls = [(T, E, K, units) for E in (1, 2, 8, 16, 17, 60, 64, 128, 257, 1024) for K in (64, 1023, 1024, 4096) for units in (1, 16, 32, 48, 64, 128, 256, 304)
             for T in (1, 2, 3, 16, 40, 63, 100, 161, 512, 768, 769, 1000, 2560, 2900, 3100, 8192, 100000)]
    forms = set()
    for (T, E, K, units), (form, size) in zip(calls, rule(calls)):
        assert size >= T * E * (32 if form == PARTS16 else 4), (T, E, K, units)
        tiles = -(-T // 16) * -(-E // 16)
        assert form == (ONE if T == 1 else FOUR if T * E <= 2560 else form)
        assert (form == PARTS16) == (T > 1 and T * E > 2560 and tiles <= 192 and K >= 1024), (T, E, K, units)       # (whatever the device)
        forms.add(form)
    assert forms == {ONE, FOUR, TILES16, PARTS16, TILES32}


def test_the_measured_sides(rule):
    """256 compute units."""
    assert [f for f, _ in rule([(T, E, K, 256) for T, E, K in ((1, 64, 4096), (37, 60, 1444), (1024, 64, 1352), (512, 16, 5120), (8192, 128, 2048), (2048, 128, 2048))])] == \
        [ONE, FOUR, TILES16, PARTS16, TILES32, TILES16]


def test_what_a_device_of_few_units_would_take_by_both_rules(rule):
    """2560 tokens to 16 experts: 160 tiles of 16 x 16, and 80 of 32 x 32 for 32 units."""
    assert [f for f, _ in rule([(2560, 16, 1024, u) for u in (32, 40, 256)])] == [PARTS16] * 3


@pytest.mark.parametrize("E", [1, 2, 7, 8, 16, 17, 33, 60, 64, 128, 200, 256, 1000, 1024])
def test_a_buffer_for_more_tokens_suffices_for_fewer(E):
    """A program makes it once, for its largest batch."""
    sizes = [dg.dg_route_tokens_work_bytes(T, E) for T in range(1, 10000)]
    assert all(a <= b for a, b in zip(sizes, sizes[1:]))
    assert sizes[-1] <= max(4 * E * 9999, 32 * 192 * 256)


def test_every_form_fits_a_buffer_for_more_tokens(rule):
    calls = [(T, E, 4096, 256) for E in (1, 8, 60, 64, 100, 1024) for T in range(1, 4000, 7)]
    for (T, E, _, _), (form, _) in zip(calls, rule(calls)):
        for more in (0, 1, 100, 5000):
            assert dg.dg_route_tokens_work_bytes(T + more, E) >= T * E * (32 if form == PARTS16 else 4), (T, E, more)
