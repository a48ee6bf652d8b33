"""Attention behind shared prefixes, replayed without a GPU: where the workgroups of one launch find their groups and row tiles, and what the
workgroups of a cut call leave behind and the join finds."""
from tests.test_abi_host import build_and_run_host_check


def test_every_row_tile_is_found_once(tmp_path):
    """However the requests are dealt to the groups, one of thousands among them, no workgroup has more than one row tile."""
    res = build_and_run_host_check(tmp_path, "shared_slots_check")
    assert res.returncode == 0 and "slot checks OK" in res.stdout, res.stdout + res.stderr


def test_every_part_is_joined_once(tmp_path):
    res = build_and_run_host_check(tmp_path, "shared_replay_check")
    assert res.returncode == 0 and "replay checks OK" in res.stdout, res.stdout + res.stderr
