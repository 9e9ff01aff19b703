"""The rules that choose a kernel for the products grouped by expert (csrc/moe_grouped_pick.h, compiled for the host): the GPU tests'
cases are on the kernels that they are there for, and together on all of them."""
import random

import pytest

import sched_host
from operator_plans import CASES, PLANS

PROGRAM = r"""
#include "moe_grouped_pick.h"
#include <cstdio>
#include <cstring>
int main() {
    char kind[8];
    int rows, E, K, N;
    while (scanf("%7s %d %d %d %d", kind, &rows, &E, &K, &N) == 5) {
        const bool mx = !strcmp(kind, "mx");
        const GroupedPlan p = !strcmp(kind, "dw") ? grouped_weights_plan(rows, E, K, N) : grouped_rows_plan(rows, E, mx ? K / 2 : K * 2, N, !strcmp(kind, "fwd"), mx);
        printf("%d %d %d\n", p.bm, p.splits, (int)p.tail);
    }
}
"""


@pytest.fixture(scope="module")
def plans(tmp_path_factory):
    exe = sched_host.compile_host(PROGRAM, str(tmp_path_factory.mktemp("plans")))

    def of(calls):
        lines = sched_host.run(exe, "\n".join(" ".join(map(str, c)) for c in calls)).splitlines()
        assert len(lines) == len(calls)
        return [(int(bm), int(splits), tail == "1") for bm, splits, tail in map(str.split, lines)]
    return of


def test_every_case_runs_on_the_kernel_it_is_there_for(plans):
    got = plans([(kind, sum(rows) + more, len(rows), K, N) for kind, rows, more, K, N, _ in CASES])
    wrong = [(c, p) for c, p in zip(CASES, got) if (p[0], p[1] > 1, p[2]) != c[5]]
    assert not wrong
    assert {(c[0], *c[5]) for c in CASES} == PLANS


def test_there_are_no_other_plans(plans):
    rng, calls = random.Random(5), []
    for kind in ("fwd", "dx", "mx", "dw"):
        for _ in range(10000):
            unit = 32 if kind == "mx" else 8
            calls.append((kind, int(2 ** rng.uniform(0, 17)), rng.choice([1, 2, 4, 8, 32, 128, 256]), unit * int(2 ** rng.uniform(0, 12)), 8 * int(2 ** rng.uniform(0, 12))))
    assert {(c[0], p[0], p[1] > 1, p[2]) for c, p in zip(calls, plans(calls))} == PLANS
