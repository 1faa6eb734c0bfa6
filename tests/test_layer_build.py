"""Build facts that the layer products rely on, from the compiler's own report."""
import os
import re
import subprocess
import tempfile

from paper_2009_09271_b200 import build as scbuild


def test_register_split_fits_the_launch():
    """The 256-wide weight-gradient builds hand registers from four warps to eight; what they ask for must be within what the
    launch holds (384 threads at the reported count), or they would wait for ever."""
    text = open(os.path.join(scbuild.CSRC, "sc_product.cuh")).read()
    low, high = (int(re.search(rf"setmaxnreg\.{d}\.sync\.aligned\.u32 (\d+)", text).group(1)) for d in ("dec", "inc"))
    least = int(re.search(r"TC_LEAST_REGS = (\d+)", text).group(1))
    assert 128 * low + 256 * high <= 384 * least
    with tempfile.TemporaryDirectory() as tmp:
        res = subprocess.run([scbuild._nvcc()] + scbuild.NVCC_FLAGS + ["-Xptxas", "-v", "-c", "-o", os.path.join(tmp, "o.o"),
                              os.path.join(scbuild.CSRC, "sc_layer.cu")], capture_output=True, text=True)
    assert res.returncode == 0
    regs = {m.group(1): int(m.group(2)) for m in
            re.finditer(r"Compiling entry function '(\S*product_kernel\S*Li2ELi256E\S*)'.*?Used (\d+) registers", res.stderr + res.stdout, re.S)}
    assert len(regs) == 2 and all(n >= least for n in regs.values()), regs
