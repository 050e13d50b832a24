"""The paged attention kernels' LDS ring: no wave passes a barrier with an LDS
read of its own in flight (from the assembly, on the CPU)."""
import tests.test_lds_order as lds


def test_no_lds_read_in_flight_at_a_barrier(tmp_path):
    lds.test_no_lds_read_in_flight_at_a_barrier("paged_attn.hip", tmp_path)
