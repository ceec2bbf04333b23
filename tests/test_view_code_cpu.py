"""The many-rows kernel over a window, and with partial sums as results, in the code that the compiler makes of it: the checks of test_stream_code_cpu.py, whose fast
loop these variants share."""
import re

import pytest

import test_stream_code_cpu as base

KERNELS = [(d, p, mode) for d in (64, 128) for p in (32, 64, 128) for mode in (1, 2)]


@pytest.fixture(scope="module")
def listing(tmp_path_factory):
    return base._compile("k_cache_attn_view", tmp_path_factory.mktemp("view"))


@pytest.fixture(params=KERNELS, ids=lambda k: "d%d-P%d-mode%d" % k)
def one(request, listing):
    """(The listing of one kernel, d, p) as the functions of the other file find it."""
    d, p, mode = request.param
    return re.search(r"^_ZN\S*17k_cache_attn_tileILi%dELi%dELi%dE\S*:.*?^\.Lfunc_end" % (d, p, mode), listing, re.S | re.M).group(0), d, p


@pytest.mark.parametrize("check", [base.test_the_fast_loop_keeps_everything_in_registers, base.test_no_operand_is_used_while_its_load_is_under_way,
                                   base.test_writes_of_a_stage_are_done_before_its_barrier, base.test_room_between_a_matrix_instruction_and_its_readers],
                         ids=["registers", "loads", "stages", "room"])
def test_fast_loop(one, check):
    check(*one)


@pytest.mark.parametrize("check", [base.test_no_move_of_a_value_runs_with_half_of_the_lanes, base.test_no_tuple_is_filled_with_one_of_its_elements], ids=["moves", "tuples"])
def test_moves(check, tmp_path):
    check("k_cache_attn_view", tmp_path)
