"""The division of a batch's keys among the workgroups of chunk_attn, and what they leave for the join, gone
through on the host by chunk_plan.cpp with the kernels' own arithmetic (these run without a GPU)."""
import os
import subprocess

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    from paper_2502_20766_amd import _build
    try:
        hipcc = _build._hipcc()
    except RuntimeError:
        pytest.skip("hipcc is not available")
    exe = str(tmp_path_factory.mktemp("plan") / "chunk_plan")
    r = subprocess.run([hipcc, "-x", "hip", "--offload-host-only", "-O2", "-std=c++17", "-Wall",
                        os.path.join(HERE, "chunk_plan.cpp"), "-o", exe], capture_output=True, text=True)
    assert r.returncode == 0, r.stdout + r.stderr

    def run(*args):
        r = subprocess.run([exe, *map(str, args)], capture_output=True, text=True, timeout=100)
        assert r.returncode == 0, r.stdout + r.stderr
        return [int(x) for x in r.stdout.split()]
    return run


def test_every_record_has_one_writer(plan):
    """All workgroup counts, widths and numbers of parts: each row tile of a part has one workgroup, and
    each record, also of a number that no part has."""
    assert plan("places") == [sum(wgs // w for wgs in (256, 512, 768) for w in range(1, 17))]


@pytest.mark.parametrize("seed", range(6))
def test_drawn_batches(plan, seed):
    """Each key tile of a row tile in one piece, each record written once, numbers of pieces and first
    parts as the pieces are; with sequences without tokens that have many rows."""
    cut, joined, dealt, few = plan("batches", seed, 3000)
    assert cut > 2900 and joined > 10000
    assert dealt > 300 and few > 5       # more records than the clusters that are dealt out over the XCDs


@pytest.mark.parametrize("batch", [
    (256, 256, 3, 16, 2, "-1:995", "-1:995", "1207:1"), (128, 768, 5, 16, 2, "1479:39", "-1:3037"),
    (128, 768, 9, 16, 2, "1241:41", "0:3078"), (256, 256, 3, 4, 2, "1151:1", "-1:5538", "0:2462")])
def test_more_segments_than_parts(plan, batch):
    """Idle sequences of many rows beside one that is cut: a record for every part, of which there are few,
    and a width that leaves workgroups of every XCD over."""
    cut, joined, dealt, few = plan("batch", *batch)
    assert cut == dealt == few == 1 and joined > 0
