"""CPU: the eviction's workspace holds the lists of moving rows where a launch of their own reads them, and nothing where the unit's workgroup moves its rows."""
import ctypes as C

import paper_2510_18716_amd as ssd
from paper_2510_18716_amd.binding import make_paged_config

FAKE = 1 << 24


def _evict(cfg, ws, size, table=FAKE):
    return ssd.lib.ssd_paged_evict(C.byref(cfg), FAKE, FAKE, table, FAKE, FAKE, FAKE, 1, 2, FAKE, FAKE, FAKE, FAKE, FAKE + 64, 0, ws, size, None)


def test_lists_that_nobody_reads_take_no_memory():
    many = make_paged_config(128, 32, 32, 128, "bf16", 16, 9000, 512)           # 4096 units of up to 8192 rows
    assert ssd.ssd_paged_evict_workspace_bytes(many) == 0 and ssd.ssd_last_error() == ""
    few = make_paged_config(8, 8, 8, 128, "bf16", 16, 9000, 512)                # 64 of them: two lists of half as many places and a count
    need = ssd.ssd_paged_evict_workspace_bytes(few)
    assert 64 * 4 * (8192 + 1) <= need <= 64 * 4 * (8192 + 4)
    long = make_paged_config(128, 32, 32, 128, "bf16", 64, 9000, 512)           # up to 32768 rows: in slices
    assert ssd.ssd_paged_evict_workspace_bytes(long) > 4096 * 4 * 32768
    for cfg in (few, long):
        size = ssd.ssd_paged_evict_workspace_bytes(cfg)
        for ws, given in ((None, size), (FAKE + 128, size), (FAKE, size - 1)):
            assert _evict(cfg, ws, given) == ssd.SSD_ERR_INVALID_ARG and "workspace" in ssd.ssd_last_error()
    # without one the call goes on to its other checks
    assert _evict(many, None, 0, table=None) == ssd.SSD_ERR_INVALID_ARG and "workspace" not in ssd.ssd_last_error()
