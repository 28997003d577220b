"""The bench's traffic of a step comes from counters of the step kernel's
current sources: an entry of other sources would leave it unknown."""
import bench


def test_counters_are_of_the_current_sources():
    entry = bench.STEP_TRAFFIC.get(bench.step_source_hash())
    assert entry is not None, "read the counters again (profiles/step_serve64_hbm_bytes.md) and enter them in bench.py"
    # serve64: 64 requests, 16 and 4 heads, d = f = 128, blocks of 32: what a step cannot do without, and little more
    need = bench.step_bytes(64, 16, 4, 128, 32, 128)
    assert need <= entry["read"] + entry["written"] <= 1.1 * need
