"""The built library's code objects, read on the host: the scratch memory of
the linear, norm and clipping kernels is what their comments say -- none, but
for the few values that some norm kernels spill."""
import re

from test_kernel_resources import _kernels

BF16, F32 = "DF16b", "f"
# bytes a lane, at most: norm_fwd<type, values, threads>, norm_bwd<type, values, threads, whole gates>
SPILLS = {("fwd", BF16, 16, 512, 0): 36, ("bwd", BF16, 8, 512, 0): 12, ("bwd", F32, 8, 512, 0): 20,
          ("bwd", BF16, 8, 64, 1): 28, ("bwd", BF16, 8, 128, 1): 44, ("bwd", BF16, 8, 256, 1): 60, ("bwd", BF16, 8, 512, 1): 76,
          ("bwd", F32, 8, 256, 1): 44, ("bwd", F32, 8, 512, 1): 68}


def test_scratch():
    norms, others = 0, 0
    for k in _kernels():
        name, scratch = k[".name"], k[".private_segment_fixed_size"]
        m = re.search(r"norm_(fwd|bwd)_kernelI(DF16b|f)Li(\d+)ELi(\d+)E(?:Lb([01])E)?", name)
        if m:
            norms += 1
            key = (m[1], m[2], int(m[3]), int(m[4]), int(m[5] or 0))
            assert scratch <= SPILLS.get(key, 0), (name, scratch)
        elif re.search(r"linear_kernel|lin_join|norm_join|clip_norm|clip_scale", name):
            others += 1
            assert scratch == 0, name
    assert norms == 30 and others > 60
