"""CPU-side check of where the attention tiles' loads go."""
import os
import subprocess

from paper_2607_02097_amd import build as B


def test_direct_tiles_load_whole_rows_and_nothing_else():
    """Tiles that go from memory straight to LDS, every thread's loads
    enumerated while the header is compiled for the host: none passes the end
    of its row (which may be the end of the tensor's memory)."""
    here = os.path.dirname(os.path.abspath(__file__))
    r = subprocess.run([B.hipcc(), "-x", "hip", "--offload-host-only", "-fsyntax-only", "--offload-arch=" + B.ARCH,
                        "-std=c++20", "-fconstexpr-steps=100000000", "-I" + B.INCLUDE, "-I" + B.CSRC,
                        os.path.join(here, "attention_places.hip")], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
