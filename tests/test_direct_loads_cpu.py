"""Where the loads of the matrix products' operands read, at the sizes at which
addresses pass 31 and 32 bits: issued on the host, nothing is read (no GPU
needed)."""
import os
import subprocess

from paper_2607_13511_amd import build

HERE = os.path.dirname(os.path.abspath(__file__))


def test_no_load_outside_an_operand(tmp_path):
    """Operands by columns, 64 rows a step of up to 2^25 entries each, and by rows, of which the loop asks for more than
    there are."""
    exe = str(tmp_path / "direct_loads")
    subprocess.run([build.HIPCC, "-std=c++17", "-O1", "-x", "hip", "--offload-host-only", f"-I{build.INCLUDE}", f"-I{build.CSRC}",
                    os.path.join(HERE, "direct_loads.hip"), "-o", exe], check=True, capture_output=True)
    got = subprocess.run([exe], capture_output=True, text=True, timeout=100)
    assert got.returncode == 0, got.stdout[-2000:]
