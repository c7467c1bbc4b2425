"""The attention kernels' loads to LDS keep the distances that inline assembly
has to keep by itself: five states between a scalar register that the vector
unit wrote and the load that reads it, one behind M0."""

from test_kernel_code_cpu import kernels  # noqa: F401


def test_states_before_loads_to_lds(kernels):  # noqa: F811
    seen = 0
    for name, ins in kernels.items():
        if "attend" not in name:
            continue
        for i, load in enumerate(ins):
            if not (load.startswith("buffer_load") and load.endswith("lds")):
                continue
            seen += 1
            assert ins[i - 2].startswith("s_mov_b32 m0,"), (name, ins[i - 3:i + 1])
            nop = ins[i - 1].split()
            assert nop[0] == "s_nop" and int(nop[1], 0) >= 4, (name, ins[i - 3:i + 1])
    assert seen > 100
