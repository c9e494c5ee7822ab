"""The extension calls an entry point through a type of as many arguments as it has; other numbers of them it leaves to ctypes."""
import ctypes

import pytest

from paper_2108_13191_amd import binding

if binding._fastcall is None:
    pytest.skip("no extension", allow_module_level=True)


def test_each_number_of_arguments():
    known = {len(letters) for name, letters in binding._OPS.items() if name != "rms_norm"}
    for n in range(0, 21):
        seen = []
        f = ctypes.CFUNCTYPE(ctypes.c_int, *[ctypes.c_int64] * n)(lambda *a: (seen.append(a), 5)[1])
        args = [(i + 1) * 0x100000001 for i in range(n)]
        rc = binding._fastcall.words(ctypes.cast(f, ctypes.c_void_p).value, "i" * n, *args)
        if n in known:
            assert rc == 5 and seen == [tuple(args)]
        else:
            assert rc is NotImplemented and not seen
