"""Static checks on the gfx950 code of the operators around the attention (CPU: hipcc cross-compiles):
no spills or scratch, the wait states of tests/test_wait_states.py, and in the gradients' loops over
tiles no vector-memory instruction other than the tile copies, whose arrival they wait for."""

import re

import pytest

from test_wait_states import listing, too_soon

SOURCES = ["norm_rope.hip", "select.hip", "decode.hip", "attn_bwd.hip"]


@pytest.fixture(scope="module")
def texts(tmp_path_factory):
    return {s: listing(s, tmp_path_factory.mktemp("isa")) for s in SOURCES}


@pytest.mark.parametrize("source", SOURCES)
def test_wait_states(source, texts):
    found = too_soon(texts[source])
    assert not found, "%d pairs, the first: %s" % (len(found), found[:3])


@pytest.mark.parametrize("source", SOURCES)
def test_no_spills_or_scratch(source, texts):
    kernels = texts[source].split("  - .agpr_count")[1:]
    assert kernels
    for block in kernels:
        name = re.search(r"\.name:\s+(\S+)", block).group(1)
        assert int(re.search(r"\.vgpr_spill_count:\s+(\d+)", block).group(1)) == 0, name
        assert int(re.search(r"\.private_segment_fixed_size:\s+(\d+)", block).group(1)) == 0, name


def test_only_tile_copies_inside_the_gradients_loops(texts):
    seen = 0
    for m in re.finditer(r"^(_ZN2sa\S+10bwd_kernel\S+):.*?^\.Lfunc_end", texts["attn_bwd.hip"],
                         re.M | re.S):
        lines = m.group(0).split("\n")
        starts = [i for i, l in enumerate(lines) if re.match(r"^(\.LBB|; %bb)", l)] + [len(lines)]
        loops = 0
        for i, j in zip(starts, starts[1:]):
            # a block's comments say whether it is part of a loop; tile loops have matrix products
            head = lines[i:i + 3]
            if not any("Loop" in l for l in head if l.startswith((".LBB", "; %bb")) or ";" in l[:45]):
                continue
            loops += any("v_mfma" in l for l in lines[i:j])
            used = {l.split()[0] for l in lines[i:j] if re.match(r"^\s+(global_|buffer_|scratch_|flat_)", l)}
            assert used <= {"global_load_lds_dwordx4", "global_load_lds_dword"}, (m.group(1), used)
        assert loops, m.group(1)
        seen += 1
    assert seen == 12  # both in one of either block size, each alone of either, two head dims
