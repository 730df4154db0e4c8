"""What the kernels' texts must keep that no run can show: orderings whose loss would corrupt results only now and then."""
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2510_05186_amd", "csrc")


def test_no_counted_wait_stands_behind_the_epilogue_s_requests():
    """gemm_bf16.hip, direct_tile: a wait for all but the newest n memory operations tells tile loads from other loads by their
    number, which holds only where every load is written in assembly.  The loads that the epilogue requests are the
    compiler's, to merge and to move: ahead of them nothing may be in flight, and behind them no wait may count."""
    text = open(os.path.join(CSRC, "gemm_bf16.hip")).read()
    body = text[text.index("void direct_tile("):]
    body = body[:body.index("\n}\n")]
    requests = [m.start() for m in re.finditer(r"old_value\(reinterpret_cast|reinterpret_cast<const bf16x4_t\*>\(R \+", body)]
    assert len(requests) == 2
    waits = [(m.start(), int(m.group(1))) for m in re.finditer(r"(?:OPTSTAGE_TILE_SYNC\(|vmcnt\()(\d+)\)", body)]
    ahead = [n for at, n in waits if at < min(requests)]
    behind = [n for at, n in waits if at > min(requests)]
    assert ahead[-1] == 0 and not any(behind), (ahead, behind)
    # and no tile load is written between that wait and the end
    last_wait = max(at for at, _ in waits if at < min(requests))
    assert not re.search(r"trip\([^)]*, true, (?:true|false)\)|issue_one\(", body[last_wait:])


def test_every_function_of_the_8_bit_keeping_has_a_caller():
    text = open(os.path.join(CSRC, "keep8.h")).read()
    everything = "\n".join(open(os.path.join(CSRC, f)).read() for f in sorted(os.listdir(CSRC)))
    names = set(re.findall(r"__forceinline__ [\w:<> ]*?[ >](\w+)\(", text))
    assert {"keep_values", "keep_chunk", "lanes_sum"} <= names
    assert not [n for n in names if len(re.findall(rf"\b{n}\b", everything)) < 2]


def test_the_library_holds_the_norm_kernels_that_a_call_can_reach():
    """Rows of bf16 have at most 1024 chunks of 16 bytes, 8 waves; 16 waves are for fp32."""
    from paper_2510_05186_amd import binding
    held = open(binding.LIB_PATH, "rb").read()
    for kernel in (b"norm_fwd_pack8_kernelI", b"norm_bwd8_kernelI"):
        for layer_norm in b"01":
            form = lambda t, waves: kernel + t + b"Lb%cELi%dE" % (layer_norm, waves)  # noqa: B023, E731
            assert form(b"DF16b", 8) in held and form(b"f", 16) in held and form(b"DF16b", 16) not in held
