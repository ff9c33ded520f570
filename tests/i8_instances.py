"""The instances of the 8-bit product's kernels: those that the sources compile, and products that take each."""
import os
import re

from paper_2505_05286_amd import build, hxf

from . import i8_util as U

EPILOGUES = {"bf16": hxf.EPI_BF16, "resid": hxf.EPI_RESID, "swiglu": hxf.EPI_SWIGLU, "f32": hxf.EPI_F32}


def instance(m, n, k, epi):
    """(kernel, row tiles, column tiles, wavefronts, read once) of a product with n output columns; the kernel: K shared out in
    a workgroup ("thin") or whole, of an epilogue each, or K cut, with or without a gate."""
    tm, nw, wv, once, pieces, _, thin = hxf.op_gemm_i8_plan(m, 2 * n if epi == "swiglu" else n, k, EPILOGUES[epi])
    if thin:
        return "thin " + epi, tm, nw, wv, 0
    return ("cut swiglu" if epi == "swiglu" else "cut") if pieces > 1 else epi, tm, nw, wv, once


def compiled():
    """Every instance that the launch tables of the sources name."""
    def table(name, macro):
        with open(os.path.join(build.CSRC, "kernels", name)) as f:
            return [tuple(map(int, t)) for t in re.findall(macro + r"\((\d+), (\d+), (\d+), (\d+)\)", f.read())]
    wide = [(tm, nw, wv, int(cache == 2)) for tm, nw, wv, cache in table("gemm_i8.hpp", "HXF_I8")]
    thin = [(tm, nw, wv, 0) for tm, nw, _, wv in table("gemm_i8_thin.hip", "HXF_THIN")]
    return {(kernel, *t) for kernel in (*EPILOGUES, "cut", "cut swiglu") for t in wide} | \
           {("thin " + epi, *t) for epi in EPILOGUES for t in thin}


# (rows, output columns, K, epilogue): products that take the instances which no epilogue of i8_util.PLANS takes
MORE = [(1, 4421, 24592, "swiglu"), (18, 8266, 8716, "swiglu"), (66, 2706, 7248, "swiglu"), (33, 16482, 31, "swiglu"),
        (389, 775, 16942, "swiglu"), (197, 4129, 14672, "swiglu"), (325, 1402, 15919, "swiglu"), (65, 24591, 102, "swiglu"),
        (257, 4107, 15270, "swiglu"), (194, 2230, 18640, "swiglu"), (296, 4225, 16519, "swiglu"), (9549, 129, 500, "swiglu"),
        (98, 16235, 575, "swiglu"), (97, 24757, 584, "swiglu"), (354, 4145, 17897, "swiglu"), (11051, 130, 229, "swiglu"),
        (428, 2749, 29459, "swiglu"), (12290, 129, 69, "swiglu"), (145, 81967, 190, "resid"), (129, 32482, 871, "swiglu"),
        (14340, 129, 183, "swiglu"), (15177, 129, 336, "swiglu"), (182, 2183, 16027, "swiglu"), (357, 2210, 23075, "swiglu"),
        (161, 131325, 96, "resid"), (161, 32533, 1088, "swiglu"), (581, 1603, 23650, "swiglu"), (419, 2213, 30418, "swiglu"),
        (195, 65345, 2126, "resid"), (193, 31902, 1459, "swiglu"), (1014, 1027, 38439, "swiglu"), (226, 64181, 3005, "resid"),
        (225, 32363, 1946, "swiglu"), (225, 92097, 52, "f32"), (226, 5447, 18423, "swiglu"),
        # and projections of 4096 to 8192 wide layers in batches of decoding sequences, logits among them
        (40, 28672, 8192, "swiglu"), (70, 28672, 8192, "swiglu"), (100, 27648, 5120, "swiglu"), (150, 28672, 8192, "swiglu"),
        (250, 28672, 8192, "swiglu"), (80, 14336, 4096, "swiglu"), (130, 14336, 4096, "swiglu"), (250, 128256, 4096, "f32"),
        (440, 5120, 27648, "resid"), (82, 8192, 28672, "resid")]


def products():
    """Every product of the two lists."""
    return [(m, n, k, epi) for m, n, k in U.PLANS for epi in EPILOGUES] + MORE
