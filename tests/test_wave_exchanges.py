"""Lanes of one wave that exchange through LDS without a block's barrier: the source has to ask for the order of its stores and reads, which nothing
else keeps the compiler from changing.  (Results of a build do not show it: they are right until a build happens to move one.)"""
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2501_19324_amd", "csrc")


def test_few_row_products_order_their_exchange():
    text = re.sub(r"//.*", "", open(os.path.join(CSRC, "w4.h")).read())
    kernel = text[text.index("void w4_few_kernel("):text.index("void w4_many_kernel(")]
    work = kernel[kernel.index("auto work ="):]
    work = work[:work.index("};")]
    put, read = work.index("w4_put("), work.index("= stage[")
    assert put < read and "wave_order()" in work[:put] and "wave_order()" in work[put:read]


def test_the_order_is_of_the_whole_wave():
    text = open(os.path.join(CSRC, "q4.h")).read()
    body = text[text.index("void wave_order()"):]
    body = body[:body.index("\n}")]
    assert "__ATOMIC_ACQ_REL" in body and "wavefront" in body and "__builtin_amdgcn_wave_barrier" in body
