"""Numbers of workgroups and places on the host.  latent_write: a launch of more than 2^22 workgroups is
rounded up to whole rows of the grid, and those past the last one have nothing to do.  latent_evict: a
budget may be any positive int32."""
import os
import shutil
import subprocess

import pytest

from paper_2607_17154_amd import build as b

SOURCE = r"""
#include <cstdio>
#include <cstdlib>

#include "grid.hpp"
#include "write_blocks.hpp"
using namespace ordermoe;

// T n_q head_dim rank rot queries absorb -> workgroups of each kind and of the launch, those of the launch that do something
int main(int, char** v) {
    int64_t x[7];
    for (int i = 0; i < 7; ++i) x[i] = atoll(v[i + 1]);
    const WriteBlocks n = write_blocks(x[0], (int)x[1], (int)x[2], (int)x[3], (int)x[4], x[5] != 0, x[6] != 0);
    const int64_t all = n.absorb + n.rows + n.copies + n.turns;
    const dim3 grid = grid_of(all);
    const int64_t launched = (int64_t)grid.x * grid.y;
    int64_t did[5] = {}, last[5] = {};
    for (int64_t i = 0; i < launched; ++i) {
        int64_t at = i;
        const int k = n.kind(at);
        if (k != WriteBlocks::NONE && at != did[k]) return 1;        // numbered one after the other
        ++did[k];
        last[k] = at;
    }
    printf("%lld %lld %lld %lld %lld %lld %lld %lld %lld\n", (long long)n.absorb, (long long)n.rows, (long long)n.copies, (long long)n.turns,
           (long long)launched, (long long)did[0], (long long)did[1], (long long)did[2], (long long)did[3]);
    return 0;
}
"""


def _program(d, source):
    if not shutil.which(b.HIPCC):
        pytest.skip("no hipcc")
    src, exe = d / "host.hip", d / "host"
    src.write_text(source)
    # (-fwrapv: a count that outgrows its type is seen, not optimised away)
    subprocess.run([b.HIPCC] + b.FLAGS + ["-fwrapv", "-I", b.CSRC, str(src), "-o", str(exe)], check=True, capture_output=True)

    def run(*args):
        r = subprocess.run([str(exe)] + [str(int(a)) for a in args], capture_output=True, text=True, timeout=100)
        assert r.returncode == 0, r.stdout + r.stderr
        return [int(x) for x in r.stdout.split()]
    return run


@pytest.fixture(scope="module")
def blocks(tmp_path_factory):
    return _program(tmp_path_factory.mktemp("blocks"), SOURCE)


@pytest.mark.parametrize("T,n_q,D,R,rot,queries,absorb", [
    (1, 1, 64, 128, 32, 1, 1), (7, 32, 128, 512, 64, 1, 0), (16001, 32, 128, 512, 64, 1, 0), (130, 4, 128, 128, 32, 0, 0),
    (1 << 24, 1, 64, 128, 32, 0, 0), ((1 << 24) + 4, 1, 64, 128, 32, 0, 0), ((1 << 24) + 1, 127, 128, 512, 64, 0, 1),
    ((1 << 26) + 3, 16, 128, 128, 64, 0, 0), ((1 << 23) + 5, 2, 64, 128, 32, 1, 1), ((1 << 24) + 9, 3, 128, 256, 64, 1, 0),
])
def test_every_workgroup_of_a_write_has_its_own_work_or_none(blocks, T, n_q, D, R, rot, queries, absorb):
    n_absorb, n_rows, n_copies, n_turns, launched, *did = blocks(T, n_q, D, R, rot, queries, absorb)
    assert launched >= n_absorb + n_rows + n_copies + n_turns and did == [n_absorb, n_rows, n_copies, n_turns]
    heads = T * n_q if queries else 0
    assert n_rows == -(-T // 4) and n_turns == -(-heads // (256 // (rot // 16) * 2))
    assert n_absorb == (-(-T // 64) * n_q * (R // 64) if queries and absorb else 0)
    assert n_copies == (0 if absorb else -(-heads // (256 // (D // 8) * 4)))


STRIDES = r"""
#include <cstdio>
#include <cstdlib>

#include "grid.hpp"

// first n step -> how many numbers, and the last one
int main(int, char** v) {
    int64_t count = 0, last = -1;
    ordermoe::every(atoi(v[1]), atoi(v[2]), atoi(v[3]), [&](int i) {
        if (i <= last) exit(1);
        ++count;
        last = i;
    });
    printf("%lld %lld\n", (long long)count, (long long)last);
    return 0;
}
"""


@pytest.fixture(scope="module")
def strides(tmp_path_factory):
    return _program(tmp_path_factory.mktemp("strides"), STRIDES)


@pytest.mark.parametrize("n", [1, 511, 512, 513, 5000, (1 << 30) + 1, (1 << 31) - 1024, (1 << 31) - 513, (1 << 31) - 2, (1 << 31) - 1])
@pytest.mark.parametrize("step", [512, 1024])
def test_a_thread_s_places_of_any_budget(strides, n, step):
    for first in (0, 1, step - 1):
        want = range(first, n, step)
        assert strides(first, n, step) == [len(want), want[-1] if len(want) else -1]
