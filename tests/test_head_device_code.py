"""CPU: the written-out direct loads of the output head's contractions as compiled: the rule that test_device_code.py states for the others."""
import re

import test_device_code as others

KERNEL = re.compile(r"[0-9a-f]+ <.*sdp_head_gemm_kernelI(?:Li\d+E){6}Li(\d)EE.*>:")


def test_written_out_loads_meet_their_hazards(tmp_path):
    n, bad = 0, []
    for lines in others.gfx950_code(tmp_path):
        lines = [line.split("//")[0].strip() for line in lines]
        written_out = False
        for i, line in enumerate(lines):
            if line.endswith(">:"):
                k = KERNEL.match(line)
                written_out = bool(k) and k[1] != "0"
            m = others.LOAD.match(line)
            if m and written_out:
                n += 1
                if not lines[i - 1].startswith(f"s_mov_b64 {m[1]}, ") or not lines[i - 2].startswith("s_mov_b32 m0, "):
                    bad.append(lines[max(0, i - 6): i + 1])
    assert n > 0
    assert not bad, "\n\n".join("\n".join(b) for b in bad[:3]) + f"\n{len(bad)} of {n} loads"
