"""The matrix-core decode over the 8-bit cache counts its vector-memory operations by hand: between the first load-to-LDS copy and
the last product of a kernel nothing else may load from memory (no spilled register, no ordinary load), or a wait ends early
and a block is computed from rows that have not arrived. Read from the code that the compiler makes (no GPU: a run shows it
only now and then)."""
import os
import re
import subprocess

from paper_2506_11104_amd import build as hip_build


def test_nothing_but_copies_loads_between_the_first_copy_and_the_last_product(tmp_path):
    out = tmp_path / "dam_decode_quant.s"
    src = os.path.join(hip_build.CSRC, "dam_decode_quant.hip")
    subprocess.run(["hipcc", "--cuda-device-only", "-S", src, "-o", str(out)] + hip_build.FLAGS, check=True, capture_output=True, timeout=300)
    text = out.read_text()
    kernels = dict(re.findall(r"\n(_ZN\S*k_decode_quant_group\S*):(.*?)\n\.Lfunc_end", text, re.S))
    assert len(kernels) == 32, sorted(kernels)                # 2 types, 2 formats, 2 head sizes, lists and plans, narrow and wide
    for name, code in kernels.items():
        ops = re.findall(r"^\s+([a-z]\w+)", code, re.M)
        first = next(i for i, o in enumerate(ops) if o.startswith("global_load_lds"))
        last = max(i for i, o in enumerate(ops) if o.startswith("v_mfma"))
        assert ops.count("s_barrier") >= 2 and last > first
        loads = [o for o in ops[first:last] if re.match(r"(global|flat|scratch|buffer)_", o) and not o.startswith("global_load_lds")]
        assert not loads, (name, loads)
    spills = re.findall(r"\.name: +(\S*k_decode_quant\S*)\n(?:.*\n)*?.*\.private_segment_fixed_size: +(\d+)", text)
    assert len(spills) == 48 and all(n == "0" for _, n in spills), spills
