"""What the compiler makes of the paged cache's kernels, read from the assembly that it writes for them: no GPU is needed."""

import re

import pytest

from test_kernel_resources import _assembly


@pytest.fixture(scope="module")
def assembly(tmp_path_factory):
    return {s: _assembly(s, tmp_path_factory.mktemp(s)) for s in ("paged.hip", "paged_decode.hip", "paged_select.hip")}


def _kernels(text):
    return {name: {k: int(v) for k, v in re.findall(r"\.amdhsa_(\w+) (\d+)\n", body)}
            for name, body in re.findall(r"\.amdhsa_kernel (\S+)\n(.*?)\.end_amdhsa_kernel", text, re.S)}


def test_no_kernel_spills(assembly):
    kernels = {n: k for text in assembly.values() for n, k in _kernels(text).items()}
    assert len(kernels) == (2 + 8) + (48 + 2) + (3 * (4 + 5) + 4)
    assert not any(k["private_segment_fixed_size"] for k in kernels.values())


def test_as_many_workgroups_reside_as_the_shared_runs_are_cut_for(assembly):
    # 512 registers per lane and SIMD, given out by the eight; a workgroup has a wavefront on each (the same rule as in the source)
    seen = 0
    for name, k in _kernels(assembly["paged_decode.hip"]).items():
        m = re.search(r"decode_paged_kernelILb([01])ELi(\d+)ELi(\d+)ELb([01])E", name)
        if not m:
            continue
        bf16, dim, shared = m[1] == "1", 16 * int(m[2]), m[4] == "1"
        assert int(m[3]) == (32 if bf16 and dim <= (128 if shared else 64) else 16)
        resident = 512 // -(-k["next_free_vgpr"] // 8 * 8)
        planned = 3 if dim <= 64 or (bf16 and dim <= 128 and not shared) else 2 if bf16 or dim <= 160 else 1
        assert resident >= planned, (name, k["next_free_vgpr"])
        seen += 1
    assert seen == 48


def _registers(operand):
    return {int(a) for a in re.findall(r"\bv(\d+)\b", operand)} | {r for a, b in re.findall(r"\bv\[(\d+):(\d+)\]", operand) for r in range(int(a), int(b) + 1)}


@pytest.mark.parametrize("source,kernel,least", [("paged_decode.hip", "decode_paged_kernel", 1000), ("paged_select.hip", "page_scores_kernel", 1000)])
def test_matrix_results_are_waited_for_on_every_path(assembly, source, kernel, least):
    # An instruction of another kind that touches a product's result has to come as many wait states behind it as the compiler leaves
    # between them within a block: 8 behind the bf16 products, 10 behind the fp32 ones, 6 behind the small fp64 ones.  Where a branch came between, it was found to
    # leave fewer, down to 1, and old values were read.
    states_behind = {"v_mfma_f32_16x16x32_bf16": 8, "v_mfma_f32_16x16x16_bf16": 8, "v_mfma_f32_16x16x4_f32": 10, "v_mfma_f64_4x4x4_4b_f64": 6}
    products = 0
    for name, body in re.findall(rf"^(\S*{kernel}\S*):.*?\n(.*?)^\.Lfunc_end", assembly[source], re.S | re.M):
        code, labels = [], {}
        for line in body.split("\n"):
            label = re.match(r"(\.LBB\w+):", line)
            if label:
                labels[label[1]] = len(code)
            op = re.match(r"\t([a-z]\w+)(?:\s+(.*))?$", line.split(";")[0].rstrip())
            if op:
                code.append((op[1], op[2] or ""))

        def following(i):
            op, arg = code[i]
            if op == "s_endpgm":
                return []
            if op == "s_branch":
                return [labels[arg]]
            return [i + 1] + ([labels[arg]] if op.startswith("s_cbranch") else [])

        for i, (op, arg) in enumerate(code):
            if not op.startswith("v_mfma"):
                continue
            products += 1
            result, need = _registers(arg.split(",")[0]), states_behind[op]
            ways, seen = [(j, 0) for j in following(i)], {}
            while ways:
                j, states = ways.pop()
                if states >= need or seen.get(j, need) <= states:
                    continue
                seen[j] = states
                o, x = code[j]
                if o.startswith("v_mfma"):                     # products wait for products by rules of their own
                    if _registers(x.split(",")[0]) >= result:
                        continue                               # the later one's result from here on
                else:
                    assert not (result & _registers(x)), f"{name}: {o} {x} {states} states behind {op} {arg}"
                ways += [(n, states + (int(x) + 1 if o == "s_nop" else 1)) for n in following(j)]
    assert products > least


def test_as_many_workgroups_of_the_scores_reside_as_the_source_says(assembly):
    # by registers as above, and by 160 KB of LDS; three, but for more than eight heads of the widest rows
    seen = {}
    for name, k in _kernels(assembly["paged_select.hip"]).items():
        m = re.search(r"page_scores_kernelILb([01])ELi(\d+)ELi(\d+)ELi(\d+)E", name)
        if m:
            lds = k["group_segment_fixed_size"]
            seen[m.groups()] = min(512 // -(-k["next_free_vgpr"] // 8 * 8), 160 * 1024 // lds if lds else 8)
    two = {("1", "16", "2", "4"), ("0", "16", "4", "4")}
    assert len(seen) == 27 and two < set(seen)
    assert all(n == 2 if i in two else n >= 3 for i, n in seen.items()), seen
