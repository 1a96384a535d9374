"""The rules by which the experts' products are cut, as the host's code in csrc/ has them: a small program of that code, compiled for the host alone."""
import functools
import os
import subprocess
import tempfile

from paper_2605_22428_amd import build

HIPCC = build._hipcc()


@functools.lru_cache(None)
def values(includes, expressions):
    """What C++ expressions over the sources' rules come to, as whole numbers.  includes: files of csrc/."""
    source = "".join('#include "%s"\n' % f for f in includes) + "#include <cstdio>\nint main() {\n%s}\n" % "".join('    printf("%%lld\\n", (long long)(%s));\n' % e for e in expressions)
    with tempfile.TemporaryDirectory() as at:
        path = os.path.join(at, "rules.hip")
        with open(path, "w") as f:
            f.write(source)
        subprocess.run([HIPCC, "--offload-host-only", "-std=c++17", "-O1", "-w", "-I", os.path.join(build.ROOT, "include"), "-I", build.CSRC, path, "-o", path + ".out"], check=True)
        return tuple(int(v) for v in subprocess.run([path + ".out"], check=True, capture_output=True, text=True).stdout.split())
