"""A process that uses more than one GPU, worked out without one: kernels with more than 64 KB of dynamic LDS are declared on each GPU that launches them."""
import json
import os
import subprocess
import sys
import textwrap

from tests.test_launches import PRELUDE, ROOT


def test_lds_is_declared_on_every_gpu(tmp_path):
    from paper_2003_00822_amd import build
    build.ensure(verbose=False)
    libs = []
    for name in ("mock_devices", "mock_hip"):
        libs.append(str(tmp_path / ("lib%s.so" % name)))
        subprocess.check_call(["g++", "-O1", "-std=c++17", "-shared", "-fPIC", "-pthread", "-o", libs[-1], os.path.join(ROOT, "tests", name + ".cpp")])
    code = "import ctypes, sys\ndevices = ctypes.CDLL(sys.argv[3], mode=ctypes.RTLD_GLOBAL)\n" + PRELUDE + textwrap.dedent("""
        class Adapters(ctypes.Structure):
            _fields_ = [(n, ctypes.c_int32) for n in ("count", "rank", "type", "reserved")] + [(n, ctypes.c_void_p) for n in ("A", "B", "scale")]
        ref, out = ctypes.byref, []
        a = Adapters(3, 16, 1, 0, 0x1000, 0x1000, None)
        shapes = [(1024, 1024), (8192, 8192), (2048, 512), (400, 8300), (200, 30000), (200, 12000), (200, 16384), (200, 7000)]
        for dev in (0, 1, 0, 1):
            devices.devices_use(dev)
            for rows, cols in shapes:
                for layout in (BITS, GATES, PAIRS):
                    for bits in (4, 8):
                        d = desc(rows, cols, bits, layout)
                        for n in (1, 3, 24, 56, 300, 1500):
                            assert L.pb_matmul(F, F, ref(d), bits, F, n, F, WORK, None) == 0
                            assert L.pb_matmul_grad(F, F, ref(d), bits, F, n, F, WORK, None) == 0
                            assert L.pb_gated_linear(F, F, ref(d), bits, F, n, None, 1, F, None, WORK, None) == 0
                            assert L.pb_gated_linear_grad(F, F, ref(d), bits, F, F, n, 1, F, F, WORK, None) == 0
                            assert L.pb_matmul_adapters(F, F, ref(d), bits, F, n, ref(a), F, None, F, WORK, None) == 0
                            assert L.pb_matmul_adapters_grad(F, F, ref(d), bits, F, F, n, ref(a), F, F, F, F, WORK, None) == 0
            out.append((devices.devices_launches(), devices.devices_undeclared()))
        print(json.dumps(out))
    """)
    r = subprocess.run([sys.executable, "-c", code, libs[1], build.LIB, libs[0]], stdout=subprocess.PIPE, check=True, timeout=300)
    seen = json.loads(r.stdout)
    assert seen[0][0] > 1000
    assert [undeclared for _, undeclared in seen] == [0, 0, 0, 0], seen
