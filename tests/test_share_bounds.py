"""What the threads of a workgroup take of many things, on the host (share_bounds.cpp, compiled
with the kernels' own share.h): every place once and in order, up to the largest numbers that
the entry points take, where 32-bit counters pass their range."""
import os
import subprocess

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
INT_MAX = (1 << 31) - 1


@pytest.fixture(scope="module")
def program(tmp_path_factory):
    from paper_2608_24411_amd import build
    env = {k: v for k, v in os.environ.items() if k != "LD_PRELOAD"}     # (a sanitizer's runtime)
    exe = str(tmp_path_factory.mktemp("share") / "bounds")
    subprocess.run([build.HIPCC, "--offload-host-only", "-x", "hip", "-std=c++17", "-O1", "-w", "-I",
                    os.path.join(build.HERE, "csrc"), os.path.join(HERE, "share_bounds.cpp"), "-o", exe], check=True, env=env)
    return exe


def counts(program, cases):
    r = subprocess.run([program] + cases, capture_output=True, text=True, timeout=60)
    assert r.returncode == 0, r.stdout[-300:]
    return dict(line.split() for line in r.stdout.split("\n") if line)


def test_entries_of_block_tables(program):
    """The page check of a paged reorder: rows of a block table from none to 2^31 - 1 entries,
    among them those whose number over all beams is 2^32 (0 in 32 bits: no page looked at) and
    those within a step of it (a counter that goes round)."""
    sizes = [(0, 4), (1, 1), (1, 64), (7, 64), (255, 3), (256, 5), (257, 2), (1000, 64),
             (1 << 26, 64), ((1 << 26) + 1, 64), (INT_MAX, 2), (INT_MAX, 3), (1 << 30, 4)]
    for used, rows in sizes:
        threads = range(256) if used < 2000 else (0, 255)
        cases = ["entries:%d:%d:%d:256" % (used, rows, t) for t in threads]
        got = counts(program, cases)
        assert [int(got[c]) for c in cases] == [max(0, -(-(used * rows - t) // 256)) for t in threads], (used, rows)


def test_pages_of_a_plan(program):
    """The pages of a step's requests, which may be 2^31 - 1 (that many rows in pages of one
    position): with 256 or 1024 threads the last counter is INT_MAX + 1 or more."""
    for n in (0, 1, 255, 256, 1023, 1024, 1025, 5000, INT_MAX - 1024, INT_MAX - 255, INT_MAX):
        for step in (256, 1024):
            threads = range(step) if n <= 5000 else (0, step - 2, step - 1)
            cases = ["of:%d:%d:%d" % (n, t, step) for t in threads]
            got = counts(program, cases)
            assert [int(got[c]) for c in cases] == [max(0, -(-(n - t) // step)) for t in threads], n


def test_padding_of_a_path(program):
    """What lies behind a path, which begins anywhere, in rows of up to 2^31 - 1 entries."""
    for n, on, step in ((10, 3, 256), (600, 66, 256), (INT_MAX, 3, 256), (INT_MAX, 8192, 1024), (INT_MAX - 700, 0, 1024)):
        threads = range(step) if n <= 5000 else (0, step - 1)
        cases = ["of:%d:%d:%d" % (n, on + t, step) for t in threads]
        got = counts(program, cases)
        assert [int(got[c]) for c in cases] == [max(0, -(-(n - on - t) // step)) for t in threads], n


def test_tiles_of_requests(program):
    """The tiles of a plan's requests, as many as an int32 counts."""
    for n in (0, 1, 1023, 1024, 1025, 3000, INT_MAX - 1024, INT_MAX - 1023, INT_MAX - 1022, INT_MAX):
        case = "blocks:%d:1024" % n
        assert int(counts(program, [case])[case]) == -(-n // 1024)
