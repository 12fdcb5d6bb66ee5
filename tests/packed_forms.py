"""Which form the library's rule gives to a product, from its header, on the CPU."""
from __future__ import annotations

import os
import re
import subprocess

HEADER = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2312_11514_amd", "csrc", "lif_packed_form.h")


def forms(folder, products):
    """[(rows, n_in, n_out, group, fp32 rows)]: the names of their forms."""
    source, program = os.path.join(str(folder), "forms.cpp"), os.path.join(str(folder), "forms")
    calls = "".join("    std::printf(\"%%d \", (int)lif::packed_form(%d, %d, %d, %s, %d));\n" % ((n_out + 15) // 16, (n_in + 127) // 128, rows, str(f32).lower(), group)
                    for rows, n_in, n_out, group, f32 in products)
    with open(source, "w") as f:
        f.write('#include <cstdio>\n#include "%s"\nint main() {\n%s}\n' % (HEADER, calls))
    subprocess.run(["g++", "-std=c++17", "-o", program, source], check=True)
    with open(HEADER) as f:
        names = re.findall(r"\w+", re.search(r"enum class PackedForm \{(.*?)\}", f.read(), re.S)[1])
    return [names[int(i)] for i in subprocess.run([program], capture_output=True, text=True, check=True).stdout.split()]


def few(name):
    return name.startswith("few")
