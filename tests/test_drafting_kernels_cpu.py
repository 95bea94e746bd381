"""What the compiler makes of the drafting operators' kernels, checked on the gfx950
assembly: things that no result shows, or only now and then."""

import re

import pytest

from tests.test_kernel_schedule_cpu import assembly, kernels, reads_at_barriers

SOURCES = ("w4_pack.hip", "w4_gemm.hip", "beam_search.hip", "reorder.hip")


@pytest.fixture(scope="module", params=SOURCES)
def compiled(request, tmp_path_factory):
    return request.param, assembly(request.param, str(tmp_path_factory.mktemp("asm")))


def test_no_registers_in_memory(compiled):
    """Spills cost the products of few rows a tenth of their time."""
    _, text = compiled
    sizes = re.findall(r"\.private_segment_fixed_size:\s*(\d+)", text)
    assert len(sizes) == len(kernels(text)) > 0
    assert set(sizes) == {"0"}


def test_no_64_bit_scalar_literals(compiled):
    """s_mov_b64 takes 32 bits of a literal; this compiler gives it more of a double."""
    _, text = compiled
    literals = [int(x, 16) for x in re.findall(r"s_mov_b64 s\[\d+:\d+\], 0x([0-9a-f]+)", text)]
    assert all(x < 1 << 32 for x in literals)


def test_wait_state_between_m0_and_lds_loads(compiled):
    _, text = compiled
    for body in kernels(text).values():
        for n, line in enumerate(body):
            if line.startswith("global_load_lds"):
                assert body[n - 1].startswith("s_nop") and "m0" in body[n - 2]


@pytest.mark.parametrize("compiled", ["w4_gemm.hip"], indirect=True)
def test_lds_reads_are_complete_at_barriers(compiled):
    """A tile's place is refilled by direct loads behind the barrier."""
    found = kernels(compiled[1])
    tiles = [body for k, body in found.items() if "w4_tile_kernel" in k]
    assert len(tiles) == 12
    for body in tiles:
        assert reads_at_barriers(body) and max(reads_at_barriers(body)) == 0
