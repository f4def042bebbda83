"""Compiles a kernel's source for the host (see host_cuda.h): copies of the sources without their PTX, then g++."""
import glob
import os
import re
import subprocess

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
UNDEFINED = ["-fsanitize=integer-divide-by-zero,signed-integer-overflow,shift,bounds", "-fno-sanitize-recover=all"]   # end the process


def without_ptx(text):
    out, at = [], 0
    for m in re.finditer(r"\basm\b(\s+volatile)?\s*\(", text):
        if m.start() < at:
            continue
        end, depth, quoted = m.end(), 1, False
        while depth:
            c = text[end]
            if c == '"' and text[end - 1] != "\\":
                quoted = not quoted
            elif not quoted:
                depth += (c == "(") - (c == ")")
            end += 1
        out += [text[at:m.start()], "(void)0"]
        at = end
    return "".join(out) + text[at:]


def build(folder, main):
    """The program of `main` (which includes host_cuda.h and csrc's files by name), built in `folder`."""
    csrc, include = os.path.join(folder, "package", "csrc"), os.path.join(folder, "include")
    os.makedirs(csrc), os.makedirs(include)
    for src in glob.glob(os.path.join(ROOT, "paper_2602_08686_b200", "csrc", "*.cu*")):
        with open(src) as f, open(os.path.join(csrc, os.path.basename(src)), "w") as g:
            g.write(without_ptx(f.read()))
    with open(os.path.join(ROOT, "include", "ckv.h")) as f, open(os.path.join(include, "ckv.h"), "w") as g:
        g.write(f.read())
    src, exe = os.path.join(folder, "main.cpp"), os.path.join(folder, "main")
    with open(src, "w") as f:
        f.write(main)
    cuda = os.path.join(os.path.dirname(os.path.dirname(os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc"))), "include")
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-w", *UNDEFINED, "-I", HERE, "-I", csrc, "-I", cuda, src, "-o", exe])
    return exe
