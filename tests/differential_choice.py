"""Which kernels differential attention launches, seen without a GPU (see kernel_choice)."""
import ctypes
import os
import pickle
import subprocess
import sys
import types

import kernel_choice


def pair_launches(cases):
    """Per case (kernel_choice.case) the kernels of one call, each (name, template arguments, (grid x, y, z, threads of a block))."""
    done = subprocess.run([sys.executable, os.path.abspath(__file__), kernel_choice._fake()], input=pickle.dumps(cases),
                          stdout=subprocess.PIPE, check=True)
    return pickle.loads(done.stdout)


def _main():
    cases = pickle.loads(sys.stdin.buffer.read())
    fake = ctypes.CDLL(sys.argv[1], mode=ctypes.RTLD_GLOBAL)    # ahead of the runtime that the library is linked to
    fake.fake_launches.restype = ctypes.c_char_p
    sys.modules["torch"] = None                                 # the binding does without it
    pkg = types.ModuleType("codec_binding")
    pkg.__path__ = [kernel_choice.PKG]
    sys.modules["codec_binding"] = pkg
    from codec_binding import binding as B
    out = []
    for c in cases:
        o = dict(dict(num_slots=0, split_align=0, max_rows=0, share=1, cost_table=None, fixed_slices=0, schedule=0, extensions=0, fused=0), **c["opts"])
        st, plan = B.codec_plan_create(*c["tree"], *c["head"], o["num_slots"], o["split_align"], o["max_rows"], o["share"], o["cost_table"],
                                       o["fixed_slices"], o["schedule"], o["extensions"], o["fused"], *(c["masks"] or (None, None)))
        assert st == B.CODEC_OK, st
        assert B.codec_plan_upload(plan, 4096, B.codec_plan_device_bytes(plan), 0) == B.CODEC_OK
        ws = B.codec_plan_workspace_bytes(plan)
        fake.fake_launches()
        config = B.codec_differential(1 << 20, 0, 0, 0, B.CODEC_DTYPE_FP32, None, 0.0, 1.0)
        st = B.codec_differential_attention(plan, config, 1 << 40, 1 << 41, 1 << 42, B.codec_kv_layout(*c["pool"]), 1 << 43, 1 << 44, ws)
        assert st == B.CODEC_OK, st
        out.append(kernel_choice._parse(fake.fake_launches()))
        B.codec_plan_destroy(plan)
    sys.stdout.buffer.write(pickle.dumps(out))


if __name__ == "__main__":
    _main()
