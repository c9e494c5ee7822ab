"""Shapes that reach each kernel form of the row operators of include/gemm_layer.h, rows of whole chunks of 8 and others, and the rules between the forms as the sources have
them.  Shared by the CPU test, which reads the rules and counts what is reached, and the GPU tests, which run the shapes."""
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2108_13191_amd", "csrc")
CUS = 256

# M, N
NORM = [(65, 24), (65, 61), (33, 128), (33, 100), (17, 256), (17, 130), (9, 512), (9, 300), (9, 1024), (9, 777), (9, 2048), (9, 2047), (600, 4000), (600, 3001), (600, 8192), (600, 8191), (16, 8192), (16, 4001),
        (9, 16384), (9, 9001), (2, 16400), (2, 20001)]
# ... of gradients row by row: three rows and more one after another in each of a workgroup's places
GRAD = [(33000, 64), (33000, 61), (16500, 104), (16500, 100), (8300, 256), (8300, 203), (8300, 512), (8300, 300), (4200, 1024), (4200, 777), (2100, 1504), (2100, 1501), (1100, 4000), (1100, 4001), (800, 8192), (800, 8191), (2050, 8200)]
GRAD_ONLY_IN_PLACE = [(600, 16384), (600, 9001)]
GRAD_FEW = [(130, 64), (130, 61), (300, 256), (300, 203), (100, 512), (100, 300), (513, 1024), (513, 777), (700, 2048), (700, 1501), (500, 4000), (500, 4001), (700, 8192), (700, 8191), (1500, 9000), (1500, 8201), (2050, 8201), (300, 16384)]
# T, choices, N
COMBINE = [(9, 3, 64), (9, 3, 61), (9, 3, 128), (9, 3, 100), (9, 5, 256), (9, 5, 203), (9, 3, 1024), (9, 3, 777)]
COMBINE_GRAD = [(40, 3, 64), (40, 3, 61), (40, 3, 128), (40, 3, 100), (40, 5, 256), (40, 5, 203), (40, 3, 512), (40, 3, 300), (40, 3, 1024), (40, 3, 777), (600, 3, 2048), (600, 3, 2047), (700, 3, 4000), (700, 3, 3999),
                (600, 2, 8192), (600, 2, 8191), (300, 3, 4096), (300, 3, 2001), (300, 2, 8192), (300, 5, 5001), (4, 2, 8200), (4, 2, 17001)]


def source(name):
    return open(os.path.join(CSRC, name)).read()


def function(text, start, end="\n}"):
    at = text.index(start)
    return text[at:text.index(end, at)]


def rule(body):
    """[(condition or None, form)] of a function of lines `if (..) return launch_x<T, ..>(..);`, or of such calls parted by ? and :, in their order."""
    found = []
    for line in body.splitlines():
        m = re.match(r"\s*(?:else )?(?:if \((.*?)\) )?(?:(?:return|rc =) )?(.*)", line)
        parts = re.split(r" [?:] ", m[2])
        if not re.search(r"\w+<T\b[^>]*>", parts[-1]):
            continue
        for choice, call in [*zip(parts[:-1:2], parts[1::2]), (None, parts[-1])]:
            conditions = [c for c in (m[1], choice) if c]
            found.append((" && ".join(f"({c})" for c in conditions) or None, re.search(r"\w+<T\b[^>]*>", call).group(0)))
    return found


def form(found, **sizes):
    for condition, name in found:
        if condition is None or eval(re.sub(r"\ba\.", "", condition).replace("chip().cus", str(CUS)).replace("&&", "and").replace("||", "or"), {}, sizes):
            return name
    raise AssertionError(f"nothing for {sizes}")
