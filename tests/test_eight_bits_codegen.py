"""Generated gfx950 code of the records in 8 bits, the policy loss and the update with 8-bit moments (no GPU needed: hipcc cross-compiles): no
spill code, registers for as many wavefronts as the kernels count on, and a row's loads that nothing waits for before its own turn."""
import re
from concurrent.futures import ThreadPoolExecutor

import pytest

from test_kernel_codegen import _device_asm, _functions, _meta

SOURCES = ("record8", "policy", "update8")


@pytest.fixture(scope="module")
def asm():
    with ThreadPoolExecutor(max_workers=3) as ex:
        return dict(zip(SOURCES, ex.map(_device_asm, (s + ".hip" for s in SOURCES))))


@pytest.mark.parametrize("source,kernels", [("record8", 8), ("policy", 25), ("update8", 8)])
def test_no_spills(asm, source, kernels):
    names = [n for n, _ in _functions(asm[source], "_ZN4alch")]
    assert len(names) >= kernels
    for n in names:
        assert _meta(asm[source], n, "vgpr_spill_count") == 0 and _meta(asm[source], n, "private_segment_fixed_size") == 0, n


def test_rows_that_are_held_leave_room_for_more_wavefronts(asm):
    """512 registers a lane of a SIMD: 80 for six wavefronts, 128 for four (one work-group of 1024 threads)."""
    held = [n for n, _ in _functions(asm["policy"], "_ZN4alch13k_policy_held")]
    assert len(held) == 14
    for n in held:
        pieces = int(re.search(r"Li\d+ELi(\d+)ELi\d+E", n).group(1))
        assert _meta(asm["policy"], n, "vgpr_count") <= (80 if pieces <= 8 else 128), n


def test_the_next_row_is_not_waited_for_before_this_one_is_done(asm):
    """From the first load of the next row into LDS to the last store of this one: loads, 16 of them in pieces, may all be on their way."""
    bodies = list(_functions(asm["policy"], "_ZN4alch13k_policy_stay"))
    assert len(bodies) == 2
    for n, body in bodies:
        assert _meta(asm["policy"], n, "vgpr_count") <= 128, n
        code = [l.strip() for l in body.split("\n") if re.match(r"\s+[a-z]", l)]
        loads = [i for i, l in enumerate(code) if re.match(r"buffer_load_dwordx4 .* lds$", l)]
        assert len(loads) == 27  # 9 before the loop, 9 in each of its branches
        loop = code[loads[9]:]
        assert sum(l.startswith("buffer_store_dwordx4") for l in loop) >= 31
        last = max(i for i, l in enumerate(loop) if l.startswith("s_waitcnt vmcnt"))  # behind the loop
        waits = [int(m.group(1)) for l in loop[:last] for m in [re.match(r"s_waitcnt vmcnt\((\d+)\)", l)] if m]
        assert all(w >= 16 for w in waits), (n, waits)


def test_pieces_move_whole(asm):
    """bf16 rows of whole pieces: 16 bytes read, 8 of codes written; and the reverse."""
    for name in ("_ZN4alch11k_gather_q8", "_ZN4alch8k_expand"):
        for n, body in _functions(asm["record8"], name):
            wide, narrow = ("global_load_dwordx4", "global_store_dwordx2") if "gather" in n else ("global_store_dwordx4", "global_load_dwordx2")
            assert body.count(wide) >= 4 and body.count(narrow) >= 4, n
