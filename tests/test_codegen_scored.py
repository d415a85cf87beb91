"""What the compiled prefill kernels with other scores look like (no GPU needed): the waits
for a step's gathers are counted by hand, as in the plain kernel, so nothing else may load
while gathers are in flight, the heads' slopes and the cap's constants included."""
import re

from tests.test_codegen import _functions, disassembly  # noqa: F401

KERNEL = "scored_prompt_kernel"


def test_only_gathers_load_inside_the_pipeline(disassembly):  # noqa: F811
    fns = _functions(disassembly, KERNEL)
    # three kinds of scores, by group size, block-offset form and kind of step
    assert len(fns) == 3 * 4 * 4, sorted(fns)
    for name, ins in fns.items():
        vmem = [i for i in ins if re.match(r"(global|buffer|flat|scratch)_", i)]
        gathers = [i for i, x in enumerate(vmem) if x == "global_load_lds_dwordx4"]
        assert len(gathers) >= 8, name
        assert vmem[:gathers[0]] == ["global_load_dwordx4"] * 8, name     # the Q^T operand
        assert gathers == list(range(gathers[0], gathers[-1] + 1)), name
        assert not [i for i in vmem if i.startswith("scratch_")], name
        assert any(i.startswith("s_load_dword") for i in ins), name       # scalar table reads


def test_m0_is_saved_and_restored(disassembly):  # noqa: F811
    """Each pair of gathers sits in one block that saves M0 and restores it."""
    for name, ins in _functions(disassembly, KERNEL, operands=True).items():
        gathers = [i for i, (mn, _) in enumerate(ins) if mn == "global_load_lds_dwordx4"]
        assert gathers and len(gathers) % 2 == 0, name
        for a, b in zip(gathers[0::2], gathers[1::2]):
            assert b == a + 3, (name, a, b)
            saved = ins[a - 3][1].split(",")[0]
            assert ins[a - 3] == ("s_mov_b32", f"{saved},m0"), (name, ins[a - 3])
            assert ins[b + 1] == ("s_mov_b32", f"m0,{saved}"), (name, ins[b + 1])


def test_no_kernel_has_private_memory(disassembly):  # noqa: F811
    """No call allocates: a kernel with private memory has the runtime set up scratch for the
    queue on its first launch, and each of its wavefronts writes and reads it."""
    notes = disassembly[1]
    names = re.findall(r"\.symbol:\s+(\S+)", notes)
    private = [int(x) for x in re.findall(r"\.private_segment_fixed_size:\s+(\d+)", notes)]
    assert len(names) == len(private) >= 300, (len(names), len(private))
    assert sum("qkv_append_kernel" in n for n in names) == 24
    assert not re.findall(r"\.uses_dynamic_stack:\s+true", notes)
    bad = [(n, b) for n, b in zip(names, private) if b]
    assert not bad, bad
