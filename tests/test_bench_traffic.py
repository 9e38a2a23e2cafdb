"""Which sources the bench line's captured traffic depends on."""
import os

import bench


def test_traffic_depends_on_the_layers_sources():
    names = [os.path.basename(f) for f in bench.kernel_sources()]
    assert {"noble_api.cu", "tc_group.cuh", "tc_pair.cuh", "tc_cosnet.cuh", "simt.cuh", "sm100_ptx.cuh", "host.cuh"} <= set(names)
    assert not [n for n in names if n.startswith(("attn", "rope"))], names
