"""The microscaled product's loads end inside their arrays (CPU: the kernels' assembly, compiled here).

K may end inside a step, and rows and columns inside a tile: what lies behind is kept out by the buffer's size alone.  The
hardware compares a raw buffer load's vector offset with that size; the compiler's contract leaves the scalar offset out of the
comparison, so a load with one may read behind the array as far as the scalar offset reaches."""
import os
import re
import subprocess

from paper_2609_24433_amd import build

LOAD = re.compile(r"\bbuffer_load_\S+ .*s\[\d+:\d+\], (\S+) offen")


def test_no_scalar_offset_that_the_range_check_leaves_out(tmp_path):
    name = "fq_mx_gemm.hip"
    out = tmp_path / "product.s"
    subprocess.run([build._hipcc(), *build.COMMON_FLAGS, *build.EXTRA_FLAGS.get(name, []), "-x", "hip", "--cuda-device-only", "-S",
                    os.path.join(build.CSRC, name), "-o", str(out)], check=True, capture_output=True, timeout=300)
    kernel, seen, bad = None, {}, []
    for line in out.read_text().splitlines():
        if line.startswith("_Z") and line.split(":")[0].find("kernel") > 0:
            kernel = line.split(":")[0]
        if "buffer_load" in line:
            m = LOAD.search(line)
            assert m, line  # every form that the kernels use is one that is checked here
            seen[kernel] = seen.get(kernel, 0) + 1
            if m.group(1) != "0":
                bad.append((kernel, line.strip()))
    kinds = ("mx_gemm_stream_kernel", "mx_token_kernel", "mx_gemm_tile_kernel")
    assert all(any(kind in k for k in seen) for kind in kinds), seen
    assert not bad, (len(bad), bad[:4])
