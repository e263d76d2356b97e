"""What goes wrong on the way of the fine-tuning operators has to be seen: waits that run out, copies of an optimiser or a
layer, settings that change between steps.  No GPU needed."""
import pytest


@pytest.mark.parametrize("turns", [1, 3, 15])
def test_a_wait_that_runs_out_in_any_turn_is_reported(gf, turns):
    """Also in the last one, after which the blocks do not meet."""
    for turn in range(turns):
        assert not gf.gf_selftest_end_of_turn(turn, turns, ok=False, met=True), turn
        assert gf.gf_selftest_end_of_turn(turn, turns, ok=True, met=True), turn
    for turn in range(turns - 1):
        assert not gf.gf_selftest_end_of_turn(turn, turns, ok=True, met=False), turn


def test_the_warp_wait_checks_its_arguments(gf):
    for bad in (0, -1, 10 ** 8 + 1):
        with pytest.raises(gf.GfError) as e:
            gf.gf_selftest_warp_wait(0x1000, bad, 0)
        assert e.value.status == gf.GF_ERR_BAD_DESC
    with pytest.raises(gf.GfError) as e:
        gf.gf_selftest_warp_wait(None, 1000, 0)
    assert e.value.status == gf.GF_ERR_NULL
