"""dps_sum_compact where memory runs out: whichever allocation fails, the call changes
nothing.  Host only: the manager's source is built into a program of its own, in which the
n-th allocation of a call fails."""
import os
import subprocess

from paper_2609_34380_amd import dps

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(dps.__file__)))

PROGRAM = r"""
#include <stdio.h>
#include <stdlib.h>

#include <new>
#include <vector>

#include "dps.h"

static long long left = -1;  // allocations until one fails; -1: none does
static long long failed = 0;

void *operator new(size_t n)
{
    if (left == 0) {
        ++failed;
        throw std::bad_alloc();
    }
    if (left > 0)
        --left;
    void *p = malloc(n ? n : 1);
    if (!p)
        throw std::bad_alloc();
    return p;
}
void operator delete(void *p) noexcept { free(p); }
void operator delete(void *p, size_t) noexcept { free(p); }

#include "dps_sum.cpp"

// Six units of eight blocks: 1, 2, 3, 6, 7 and 8 of them held.
static dps_sum *made()
{
    dps_sum *s = nullptr;
    const int64_t keep[6] = {3, 7, 1, 8, 2, 6};
    int64_t all[48], gone[48], n = 0;
    if (dps_sum_create(6, 8, 2, &s) || dps_sum_alloc(s, 48, all))
        abort();
    for (int u = 0; u < 6; ++u)
        for (int64_t i = keep[u]; i < 8; ++i)
            gone[n++] = u * 8 + (i + u) % 8;
    if (dps_sum_free(s, gone, n, nullptr))
        abort();
    return s;
}

int main()
{
    int64_t src[64], dst[64], n = 0, want_src[64], want_dst[64], want = 0;
    dps_sum *s = made();
    if (dps_sum_compact(s, 64, want_src, want_dst, &want) || want == 0)
        return 1;
    dps_sum_destroy(s);
    int steps = 0;
    for (;; ++steps) {
        s = made();
        failed = 0;
        left = steps;
        n = -1;
        const dps_status status = dps_sum_compact(s, 64, src, dst, &n);
        left = -1;
        if (status == DPS_OK && failed == 0)
            break;
        if (status != DPS_OK) {
            if (n != 0)
                return printf("allocation %d: n is %lld\n", steps, (long long)n), 2;
            if (dps_sum_compact(s, 64, src, dst, &n) != DPS_OK)
                return printf("allocation %d: then refused\n", steps), 3;
        }
        if (n != want)
            return printf("allocation %d: %lld moves, not %lld\n", steps, (long long)n,
                          (long long)want), 4;
        for (int64_t i = 0; i < n; ++i)
            if (src[i] != want_src[i] || dst[i] != want_dst[i])
                return printf("allocation %d: move %lld differs\n", steps, (long long)i), 5;
        if (dps_sum_free(s, src, n, nullptr) != DPS_OK)
            return printf("allocation %d: src is not held\n", steps), 6;
        dps_sum_destroy(s);
    }
    printf("%d allocations\n", steps);
    return steps > 0 ? 0 : 7;
}
"""


def test_no_allocation_fails_half_way(tmp_path):
    source, program = tmp_path / "compact.cpp", tmp_path / "compact"
    source.write_text(PROGRAM)
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-I", os.path.join(ROOT, "include"), "-I",
                    os.path.join(ROOT, "paper_2609_34380_amd", "csrc"), str(source), "-o", str(program),
                    "-pthread"], check=True)
    r = subprocess.run([str(program)], capture_output=True, text=True, timeout=60)
    assert r.returncode == 0, r.stdout + r.stderr
