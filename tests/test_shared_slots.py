"""Groups of unknown sizes in one launch: where each workgroup finds its group and row tile (no GPU needed)."""
from tests.test_abi_host import build_and_run_host_check


def test_every_row_tile_is_found_once(tmp_path):
    """However the requests are dealt to the groups, one of thousands among them, no workgroup has more than one row tile."""
    res = build_and_run_host_check(tmp_path, "shared_slots_check")
    assert res.returncode == 0 and "slot checks OK" in res.stdout, res.stdout + res.stderr
