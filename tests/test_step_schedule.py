"""The static checks of direct-to-LDS loads (tests/test_kernel_schedule.py) on the attention over listed blocks."""
import test_kernel_schedule as T


def test_lds_loads_read_no_freshly_vector_written_scalar():
    T.test_lds_loads_read_no_freshly_vector_written_scalar("block_attn.hip")


def test_compiler_keeps_nothing_in_m0():
    T.test_compiler_keeps_nothing_in_m0("block_attn.hip")
