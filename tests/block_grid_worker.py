"""Child of test_block_grids.py: calls of the block operators against
tests/hip_grid_stub.c.  ``block_grid_worker.py STUB LIB`` reads a JSON list of
calls (function, struct fields in order) on stdin and prints each launch's
mangled name, threads along x and workgroups along y.  Every address is made up:
nothing is read or written."""

import ctypes
import json
import sys

KINDS = {"p": ctypes.c_void_p, "q": ctypes.c_int64, "i": ctypes.c_int32, "f": ctypes.c_float}


def main():
    stub = ctypes.CDLL(sys.argv[1], mode=ctypes.RTLD_GLOBAL)
    lib = ctypes.CDLL(sys.argv[2])
    stub.stub_launch.restype = lib.fsdp_block_last_error.restype = ctypes.c_char_p
    stub.stub_threads.restype = ctypes.c_uint64
    stub.stub_grid_y.restype = ctypes.c_uint32
    launched = []
    for name, fields in json.load(sys.stdin):
        args = type("Args", (ctypes.Structure,), {"_fields_": [(f, KINDS[k]) for f, k, _ in fields]})(*[v for _, _, v in fields])
        stub.stub_reset()
        if name in ("fsdp_block_norm_grad", "fsdp_block_linear", "fsdp_block_linear_grad"):
            need = ctypes.c_int64(-1)
            status = getattr(lib, name + "_workspace")(ctypes.byref(args), ctypes.byref(need))
            assert status == 0, (name, fields, lib.fsdp_block_last_error())
            status = getattr(lib, name)(ctypes.byref(args), ctypes.c_void_p(1 << 46), need, None)
        else:
            status = getattr(lib, name)(ctypes.byref(args), None)
        assert status == 0, (name, fields, lib.fsdp_block_last_error())
        launched.append([(stub.stub_launch(k).decode(), stub.stub_threads(k), stub.stub_grid_y(k))
                         for k in range(stub.stub_launches())])
    print(json.dumps(launched))


main()
