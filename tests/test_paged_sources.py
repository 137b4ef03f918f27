"""What the sources of the paged-cache kernels have to keep to, where no run can show it (no GPU needed)."""
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2205_11622_gb300", "csrc")


def code(name):
    with open(os.path.join(CSRC, name)) as f:
        return re.sub(r"//[^\n]*", "", f.read())


def test_no_read_only_load_of_what_an_earlier_launch_of_the_call_writes():
    """Kernels of a call start before the one ahead of them has ended and read the plan that it writes.  A read-only
    (non-coherent) load wants data that nothing writes while the kernel runs, and may be moved ahead of the wait."""
    for name in ("paged_chunk.cu", "paged_attn.cu", "paged_tile.cuh", "paged.cuh"):
        text = code(name)
        assert not re.search(r"__ldg\s*\(\s*(\([^()]*\)\s*)?&?a\.plan\b", text), name
        assert "ld.global.nc" not in text, name
        assert not re.search(r"const\s+\w+\s*\*\s*__restrict__[^;]*a\.plan", text), name


def test_costs_of_items_are_summed_in_64_bits():
    """An item's cost is a few units and one or two for each 128 keys.  The sum of a step of 1024 items passes the largest
    int where they have 2^27 keys each, and a wrapped sum would be an index of the shares; such a call takes ten seconds of
    a GPU, so no run shows it."""
    plan = code("paged_chunk.cu")
    plan = plan[plan.index("k_paged_plan(AttnArgs a"):plan.index("read_row")]
    cost = plan[plan.index("kItemCost") - 200:]
    assert 1024 * (6 + 2 * (2 ** 27 // 128)) > 2 ** 31
    assert re.search(r"(int64_t|long long) mine = 0, total;", cost)
    assert re.search(r"(int64_t|long long) sum = block_sum\(mine, total, \w+\)", cost)
    assert re.search(r"__shared__ (int64_t|long long) s_cost\[32\]", plan)


def test_no_lane_runs_on_beside_a_run_of_products():
    """The warp's other lanes wait behind each run that an elected lane issues."""
    text = code("paged_chunk.cu")
    text = text[text.index("const uint32_t id_s ="):text.index("regs_up<kSoftRegs>();")]
    runs = list(re.finditer(r"^( *)if \((ok && )?tc::elect_one\(\)\) ?(\{.*?^\1\}|[^\n]*;)\n\s*(\S[^\n]*)", text, re.M | re.S))
    assert len(runs) == text.count("elect_one") == 7
    for run in runs:
        assert run.group(4).startswith("__syncwarp();"), run.group(0)
