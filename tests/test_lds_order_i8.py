"""Order of LDS reads and refills in the 8-bit products' tile kernels (CPU only), as in test_lds_order."""
import pytest

from test_lds_order import _kernels, longest_flight


def test_no_lds_read_is_in_flight_across_two_barriers(tmp_path):
    bodies = _kernels(tmp_path, "gateup_i8.hip")
    names = [n for n in bodies if "gateup_kernelILi256E" in n or "gateup_kernelILi128E" in n]
    assert len(names) == 4
    for n in names:
        assert sum(l.startswith("s_barrier") for l in bodies[n]) >= 4 and \
            sum(l.startswith("ds_read") for l in bodies[n]) >= 16, n
        worst, where = longest_flight(bodies[n])
        assert worst <= 1, f"{n}: an LDS read in flight across {worst} barriers ({where})"


def test_tiles_of_128_rows_and_columns(tmp_path):
    """Their ring buffers are refilled right behind the barrier that ends the slot of the reads."""
    bodies = _kernels(tmp_path, "gateup_i8.hip")
    names = [n for n in bodies if "gateup_i8_mid_kernel" in n]
    assert len(names) == 1
    body = bodies[names[0]]
    assert sum(l.startswith("s_barrier") for l in body) >= 4 and sum(l.startswith("ds_read") for l in body) >= 16
    worst, where = longest_flight(body)
    assert worst <= 0, f"an LDS read in flight across {worst} barriers ({where})"
