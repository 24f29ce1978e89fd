"""Child of test_step_launch_forms.py: as block_launch_worker.py, for the
operators of fsdp_step.h.  ``step_launch_worker.py STUB LIB`` reads a JSON list
of calls (function, struct fields in order) on stdin and prints each launch's
mangled name, threads along x and workgroups along y, and the names of all
kernels of LIB.  Every address is made up: nothing is read or written."""

import ctypes
import json
import os
import sys

KINDS = {"p": ctypes.c_void_p, "q": ctypes.c_int64, "i": ctypes.c_int32, "f": ctypes.c_float}


def main():
    stub = ctypes.CDLL(sys.argv[1], mode=ctypes.RTLD_GLOBAL)
    stub.stub_kernel.restype = stub.stub_launch.restype = ctypes.c_char_p
    stub.stub_threads.restype = ctypes.c_uint64
    stub.stub_grid_y.restype = ctypes.c_uint32
    block = ctypes.CDLL(os.path.join(os.path.dirname(sys.argv[2]), "libfsdp_block.so"))
    others = stub.stub_kernels()                 # of the library that LIB links
    block.fsdp_block_last_error.restype = ctypes.c_char_p
    lib = ctypes.CDLL(sys.argv[2])
    launched = []
    for name, fields in json.load(sys.stdin):
        args = type("Args", (ctypes.Structure,), {"_fields_": [(f, KINDS[k]) for f, k, _ in fields]})(*[v for _, _, v in fields])
        stub.stub_reset()
        if hasattr(lib, name + "_workspace"):
            need = ctypes.c_int64(-1)
            status = getattr(lib, name + "_workspace")(ctypes.byref(args), ctypes.byref(need))
            assert status == 0 and need.value >= 0, (name, fields, block.fsdp_block_last_error())
            assert stub.stub_launches() == 0
            if need.value:                       # too small a workspace is refused, and nothing launched
                assert getattr(lib, name)(ctypes.byref(args), ctypes.c_void_p(1 << 46), ctypes.c_int64(need.value - 1), None) == 1
                assert stub.stub_launches() == 0
            status = getattr(lib, name)(ctypes.byref(args), ctypes.c_void_p(1 << 46), need, None)
        else:
            status = getattr(lib, name)(ctypes.byref(args), None)
        assert status == 0, (name, fields, block.fsdp_block_last_error())
        launched.append([(stub.stub_launch(k).decode(), stub.stub_threads(k), stub.stub_grid_y(k))
                         for k in range(stub.stub_launches())])
    print(json.dumps({"launched": launched, "kernels": [stub.stub_kernel(k).decode() for k in range(others, stub.stub_kernels())]}))


main()
