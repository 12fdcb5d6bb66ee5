"""Which form the library's rule gives to a product, from its header, on the CPU."""
from __future__ import annotations

import os
import re
import subprocess

HEADER = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2312_11514_amd", "csrc", "lif_packed_form.h")


def form_names():
    with open(HEADER) as f:
        return re.findall(r"\w+", re.search(r"enum class PackedForm \{(.*?)\}", f.read(), re.S)[1])


def forms(folder, products):
    """[(rows, n_in, n_out, group, fp32 rows)]: the names of their forms."""
    source, program = os.path.join(str(folder), "forms.cpp"), os.path.join(str(folder), "forms")
    with open(source, "w") as f:
        f.write('#include <cstdio>\n#include "%s"\nint main() {\n    int rows, in, out, group, f32;\n'
                '    while (std::scanf("%%d %%d %%d %%d %%d", &rows, &in, &out, &group, &f32) == 5)\n'
                '        std::printf("%%d ", (int)lif::packed_form((out + 15) / 16, (in + 127) / 128, rows, f32 != 0, group));\n}\n' % HEADER)
    subprocess.run(["g++", "-std=c++17", "-o", program, source], check=True)
    text = "".join("%d %d %d %d %d\n" % p for p in products)
    names = form_names()
    return [names[int(i)] for i in subprocess.run([program], input=text, capture_output=True, text=True, check=True).stdout.split()]


def few(name):
    return name.startswith("few")
