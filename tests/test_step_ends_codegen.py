"""Generated gfx950 code of the embedding rows, the clipping and the update (no GPU needed: hipcc cross-compiles): no spill code,
rows in 16-byte accesses at whatever address, and lanes read only from registers that all lanes have written."""
import re
from concurrent.futures import ThreadPoolExecutor

import pytest

from test_kernel_codegen import _device_asm, _functions, _meta


@pytest.fixture(scope="module")
def asm():
    with ThreadPoolExecutor(max_workers=2) as ex:
        return dict(zip(("embed", "update"), ex.map(_device_asm, ("embed.hip", "update.hip"))))


@pytest.mark.parametrize("source,kernels", [("embed", 8), ("update", 7)])
def test_no_spills(asm, source, kernels):
    names = [n for n, _ in _functions(asm[source], "_ZN4alch")]
    assert len(names) >= kernels
    for n in names:
        assert _meta(asm[source], n, "vgpr_spill_count") == 0 and _meta(asm[source], n, "private_segment_fixed_size") == 0, n


def test_rows_of_any_width_move_16_bytes(asm):
    """Rows need not begin at a multiple of 16 bytes: the loads of the sums are whole for both types, a tail of a row aside."""
    bodies = [b for n, b in _functions(asm["embed"], "_ZN4alch12k_embed_sums") if "Li1E" not in n]
    assert len(bodies) == 4  # two types, accumulating or not
    for body in bodies:
        assert body.count("global_load_dwordx4") >= 16 and "global_load_ushort" not in body


def test_lanes_are_read_from_registers_that_all_lanes_have_written(asm):
    """A lane is read whether a branch has switched it off or not.  Keys and tokens of a part come by a load: nothing chooses between two
    of them in a register, in a branch perhaps, before a lane is read."""
    for name, body in _functions(asm["embed"], "_ZN4alch12k_embed_sums"):
        code = [l.strip() for l in body.split("\n") if re.match(r"\s+[a-z]", l)]
        reads = [i for i, l in enumerate(code) if l.startswith("v_readlane_b32")]
        assert len(reads) >= 16, name
        for i in reads:
            src = re.match(r"v_readlane_b32 \w+, (v\d+)", code[i]).group(1)
            writer = next(l for l in reversed(code[:i]) if re.match(r"\S+ %s\b(?!:)" % src, l) and not l.startswith(("v_cmp", "global_store")))
            # (or by v_writelane: scalars that were put aside)
            assert writer.startswith(("global_load_dword ", "v_writelane_b32")), (name, writer, code[i])
