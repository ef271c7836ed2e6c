import os
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)


def pytest_configure(config):
    config.addinivalue_line("markers", "gpu: needs an MI355X (gfx950) GPU and the built HIP library")
    config.addinivalue_line("markers", "slow: long-running case")


def pytest_collection_modifyitems(items):
    # Its queries are whatever torch's generator holds, and between two orders of the same fp32 sums of absolute value 0.9 it
    # allows 2^-26 and 2^-20 of the result: a quarter of one unit of those sums, which 2 to 7 of 100 queries pass.  Last, so that a run
    # that ends with the first failure has run all others.  (Both orders against 64 bits: test_gpu_kv4_lengths.py.)
    items.sort(key=lambda i: "test_gpu_kv4_chunk.py::test_lengths_to_the_end_of_32_bits" in i.nodeid)
