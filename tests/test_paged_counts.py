"""Calls over as many requests, tokens and entries of lists as an int counts: the steps of the kernels' loops end behind the
last one (no GPU needed: the arrays of such a call take 8 GB each)."""
import ctypes
import os
import re
import subprocess

import pytest

import paper_2205_11622_gb300 as slnr
from test_paged_abi import UNSUPPORTED, WORKSPACE, cache, opts, pages, rows

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2205_11622_gb300", "csrc")
MOST = 2 ** 31 - 1
SOURCES = sorted(f for f in os.listdir(CSRC) if re.match(r"page[ds_4]?.*\.cuh?$", f))

WALK = """
#include "range.h"
// How often requests [r, end) are looked at, by lanes of `each` neighbours, `step` at a time; -1: one outside of them
extern "C" long long walk(int r, int step, int each, int end) {
  long long seen = 0;
  for (int r0 = r; r0 < end; r0 = slnr::step_end(r0, step, end))
    for (int lane = 0; lane < step / each; ++lane)
      for (int i = 0; i < each; ++i)
        if (slnr::inside(r0, each * lane + i, end)) {
          if (slnr::item(r0, each * lane + i) >= (unsigned)end) return -1;
          ++seen;
        }
  return seen;
}
"""


def code(name):
    with open(os.path.join(CSRC, name)) as f:
        return re.sub(r"//[^\n]*", "", f.read())


@pytest.fixture(scope="module")
def walk(tmp_path_factory):
    d = tmp_path_factory.mktemp("walk")
    (d / "walk.cpp").write_text(WALK)
    so = str(d / "walk.so")
    subprocess.run(["g++", "-std=c++17", "-O2", "-Wall", "-Werror", "-shared", "-fPIC", "-I", CSRC, str(d / "walk.cpp"),
                    "-o", so], check=True)
    f = ctypes.CDLL(so).walk
    f.restype = ctypes.c_longlong
    return f


@pytest.mark.parametrize("step,each", [(32, 1), (128, 4), (1024, 1)])
@pytest.mark.parametrize("nreq", [0, 1, 127, 128, 5000, MOST - 1000, MOST - 1, MOST])
def test_requests_are_looked_at_once(walk, step, each, nreq):
    first = max(0, nreq - 3 * step - 1)
    assert walk(first, step, each, nreq) == nreq - first


def test_loops_over_requests_use_those_steps():
    """A counter of requests that is an int is stepped by step_end and compared by inside: its sum with a step, or with a lane,
    passes the largest int before it passes nreq."""
    assert {"pages.cu", "paged4_rows.cu", "paged_chunk.cu", "paged_tile.cuh", "page_sets.cu"} <= set(SOURCES)
    loops = 0
    for name in SOURCES:
        text = code(name)
        for m in re.finditer(r"for \(\s*(?P<type>\w+) (?P<i>\w+) = [^;]*; (?P=i) < (?:\w+\.)?nreq; (?P<step>[^{;]*)\)", text):
            loops += 1
            assert m["type"] == "int64_t" or m["step"].startswith(m["i"] + " = step_end("), f"{name}: {m[0]}"
        assert not re.search(r"\b(?:r0|r|i)\b \+ [^;=]*< (?:\w+\.)?nreq", text), name
    assert loops >= 8


def test_requests_that_end_are_counted_in_64_bits():
    """page_free takes as many entries of drop as an int counts, 16384 a step: up to 2^31 - 1 of the same few requests."""
    text = code("page_sets.cu")
    loops = re.findall(r"for \((\w+) \w+ = [^;]*; \w+ < ndrop;", text)
    assert loops and set(loops) == {"int64_t"}


def test_tokens_of_tables_are_counted_from_a_blocks_first():
    """page_tables takes as many tokens as an int counts: a block's loops count from its own first one, so that no sum with a
    step passes the largest int."""
    text, loops = code("pages.cu"), 0
    text = text[text.index("k_page_tables(int nreq"):text.index("k_page_append(")]
    for m in re.finditer(r"for \(int (\w+) = ([^;]*); ([^;]*); \1 \+= kTablesThreads\)", text):
        loops += 1
        assert m[2] == "tid" and not re.search(r"< (t1|hi|ntok)$", m[3]), m[0]
    assert loops == 2


def test_page_append_refuses_more_tokens_than_its_steps_count():
    """A block steps by up to 1024 tokens, as an int."""
    slnr.build()
    lib, p = slnr.lib(), ctypes.byref
    k = rows(tok=128)
    for ntok, status in ((2 ** 31 - 2 ** 16, WORKSPACE), (2 ** 31 - 2 ** 16 + 1, UNSUPPORTED), (MOST, UNSUPPORTED)):
        step = pages(ntok=ntok, max_q=1)
        assert lib.slnr_page_append(p(cache()), p(step), p(k), p(k), p(opts(validate=1))) == status, slnr.last_error()
