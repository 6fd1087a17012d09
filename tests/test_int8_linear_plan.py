"""Which kernels the 8-bit product launches, by size (no GPU: the runtime is the recording stand-in)."""
import pytest

import paper_2601_19675_amd as ptq
from launch_recorder import PTR, record


def launched(t, m, n, odt=1):
    args = [PTR, n, PTR, t, PTR, n, PTR, m, n, PTR, PTR, odt, m, PTR, 1 << 40, 0]
    (rc, launches), = record([("ptq_int8_linear", args)])
    assert rc == 0
    return [(k["kernel"], k["grid"]) for k in launches]


@pytest.mark.parametrize("t,m,n,kernel,blocks,summed", [
    (1, 4096, 4096, "skinny_kernelILi1ELi1E", 256, False), (17, 100, 64, "skinny_kernelILi1ELi2E", 7, False),
    (64, 1024, 4096, "skinny_kernelILi1ELi4E", 64, False),
    (64, 4096, 4096, "tile_kernelILi1ELi1ELi2E", 64, False),        # tokens enough for tiles, if not for all of one
    (512, 4096, 4096, "tile_kernelILi1ELi1ELi2E", 256, False),      # 64 x 128 tiles: one to a compute unit
    (65, 70, 11008, "tile_kernelILin1ELi1ELi2E", 30, True),          # few of them: k in splits
    (1024, 4096, 4096, "tile_kernelILi1ELi2ELi2E", 256, False),
    (8192, 11008, 4096, "tile_kernelILi1ELi4ELi4E", 1376, False),
])
def test_forms(t, m, n, kernel, blocks, summed):
    got = launched(t, m, n)
    assert kernel in got[0][0] and got[0][1][0] == blocks
    assert len(got) == (2 if summed else 1) and (not summed or "split_sum_kernel" in got[1][0])
    # the workspace holds every split's sums, and only splits have one
    need = ptq.ptq_workspace_bytes(ptq.OP_INT8_LINEAR, m, n, t)
    assert (need > 0) == summed
    if summed:
        assert need == blocks * 64 * 128 * 4


def test_every_form_is_reached():
    calls = []
    for t in (65, 150, 333, 700, 2000):
        for m in (64, 1000, 4096, 11008):
            for n in (512, 4096, 11008):
                calls.append(("ptq_int8_linear", [PTR, n, PTR, t, PTR, n, PTR, m, n, PTR, PTR, 1, m, PTR, 1 << 40, 0]))
    seen = {launches[0]["kernel"].split("tile_kernelI")[1].split("EEEv")[0] for _, launches in record(calls)}
    assert seen == {"Li1ELi4ELi4ELi2", "Li1ELi2ELi2ELi4", "Li1ELi1ELi2ELi4", "Lin1ELi1ELi2ELi4"}
