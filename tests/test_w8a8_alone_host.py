"""Host-only: a program of W8A8 linears loads libw8a8 and nothing else of this project."""
import subprocess
import sys

from paper_2505_22179_amd import binding as B

ALONE = f"""
import ctypes
L = ctypes.CDLL({B.LIB_W8A8_PATH!r})
assert not any("libw4a16" in ln for ln in open("/proc/self/maps"))
L.w4a16_strerror.restype = ctypes.c_char_p
print([L.w4a16_strerror(c).decode() for c in range(-7, 1)])
f = L.w4a16_workspace_init
f.argtypes = [ctypes.c_void_p, ctypes.c_size_t, ctypes.c_void_p]
print([f(None, 1 << 20, None), f(0x1010, 1 << 20, None), f(0x1000, 16383, None)])
"""


def test_the_library_prepares_its_workspaces_and_names_its_errors_by_itself():
    out = subprocess.run([sys.executable, "-c", ALONE], capture_output=True, text=True)
    assert out.returncode == 0, out.stderr
    texts, codes = out.stdout.splitlines()
    assert texts == str([B.strerror(c) for c in range(-7, 1)])
    init = B.load().w4a16_workspace_init
    assert codes == str([init(None, 1 << 20, None), init(0x1010, 1 << 20, None), init(0x1000, 16383, None)])
