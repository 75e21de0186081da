"""What no run can show without a fault, read from the kernels' sources."""
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2607_15810_b200", "csrc")


def test_kernels_that_abandon_a_wait_let_their_copies_land():
    """Every kernel that loads behind bounded mbarrier waits ends with settle_if_abandoned, which keeps its shared memory until what is in
    flight has landed: beside the freeing of tensor memory behind the last barrier, in a CTA pair in front of that barrier."""
    single = r"\n  if \(warp == [\w:]+\) tmem_dealloc<\w+>\([^)]*\);\n  if \((?:CG == 1 && )?warp == 0\) settle_if_abandoned\(abort_flag\);"
    pair = r"__syncthreads\(\);\n  if \((?:CG == 2 && )?warp == 0\) settle_if_abandoned\(abort_flag\);\n  (?:if \(CG == 2\) )?cluster_sync_all\(\);"
    for name, singles, pairs in (("gemm.cu", 1, 1), ("gemm_swapped.cu", 1, 0), ("gemm_dense.cu", 1, 0), ("gemm_bf16.cu", 1, 1), ("fp8.cu", 1, 0)):
        with open(os.path.join(CSRC, name)) as f:
            text = re.sub(r"[ ]*//[^\n]*", "", f.read())
        assert len(re.findall(single, text)) == singles, name
        assert len(re.findall(pair, text)) == pairs, name
        assert len(re.findall(r"tmem_dealloc<", text)) == max(singles, singles + pairs - (1 if name == "gemm.cu" else 0)), name


def _functions(text):
    """name -> body of the functions and kernels that a source defines, the bodies of one name joined."""
    def closing(at, pair):
        depth = 1
        while depth and at < len(text):
            depth += {pair[0]: 1, pair[1]: -1}.get(text[at], 0)
            at += 1
        return at
    out = {}
    for m in re.finditer(r"\b(?!if\b|for\b|while\b|switch\b|__)(\w+)\(", text):
        brace = re.compile(r"\s*\{").match(text, closing(m.end(), "()"))
        if brace:
            out[m.group(1)] = out.get(m.group(1), "") + text[brace.end():closing(brace.end(), "{}")]
    return out


def test_kernels_that_may_start_early_wait_for_the_one_in_front():
    """A launch through launch_kernel or launch_cluster(s) lets the kernel start while its predecessor still runs: every kernel launched so waits
    for it (griddepcontrol.wait), itself or in a function that it calls.  Without that it may read what is not written yet and write
    what is still read, and what comes behind it no longer waits for what was in front."""
    texts = {}
    for name in os.listdir(CSRC):
        if name.endswith((".cu", ".cuh")):
            with open(os.path.join(CSRC, name)) as f:
                texts[name] = re.sub(r"//[^\n]*", "", f.read())
    bodies = {}
    for text in texts.values():
        for name, body in _functions(text).items():
            bodies[name] = bodies.get(name, "") + body
    launched = set()
    for text in texts.values():
        alias = re.findall(r"constexpr auto (\w+) = (\w+)<", text)
        for k in re.findall(r"\blaunch_(?:kernel|clusters?)\(\s*(\w+)", text):
            launched |= {kernel for name, kernel in alias if name == k} or {k}
    launched -= {"void", "kernel"}                           # the launchers themselves
    assert len(launched) >= 25 and {"fp8_quantize_weight_kernel", "gemm_kernel", "route_experts_kernel", "front_small_kernel"} <= launched
    waits = lambda body: "pdl_sync()" in body or "griddepcontrol.wait" in body
    for k in sorted(launched):
        assert k in bodies, k
        called = set(re.findall(r"\b(\w+)(?:<[^;(]*>)?\(", bodies[k])) & set(bodies)
        assert waits(bodies[k]) or any(waits(bodies[c]) for c in called - {k}), k
