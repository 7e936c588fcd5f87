"""Row strides in index arithmetic, read from the source: a stride is an int that a caller may choose up to 2^31 - 1, so a
product with one has to be taken in 64 bits."""
import glob
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2509_10918_b200", "csrc")
FILES = sorted(glob.glob(os.path.join(CSRC, "*.cu")) + glob.glob(os.path.join(CSRC, "*.cuh")))
STRIDE = r"(?:\w+\.)?ld[a-z]\b"


def narrow_products(src):
    """Statements that multiply by a row stride with neither factor cast to 64 bits."""
    src = re.sub(r"//[^\n]*", "", src)
    for m in re.finditer(rf"\* *{STRIDE}(?! *%)|{STRIDE} *\* *[\w(]", src):
        # from the beginning of the sum, argument or operand that the product is part of
        before = re.split(r"[;,{{?:=]|\+=| \+ ", src[max(0, m.start() - 60): m.start()])
        text = src[max(0, m.start() - 60): m.end()]
        if not re.search(r"\((?:size_t|uint64_t|long long)\)", before[-1] + m.group()) and not re.search(r"\((?:size_t|uint64_t|long long)\)\([^;{}]*\) \* *" + STRIDE + "$", text):
            yield re.sub(r"\s+", " ", text).strip()


def test_a_narrow_product_is_seen():
    assert list(narrow_products("for (j = 0; j < 8; ++j, w_at += 8 * o.ldw) w[j] = 0;"))
    assert list(narrow_products("x = p + o.lda * row;")) and list(narrow_products("f((n0 + g) * o.ldw + k);"))
    assert not list(narrow_products("w_at += (size_t)8 * o.ldw; x = (const T*)a + (size_t)(m0 + row) * o.lda + k; s = {(uint64_t)o.lda * (f8 ? 1 : 2)};"))


@pytest.mark.parametrize("path", FILES, ids=[os.path.basename(f) for f in FILES])
def test_products_with_strides_are_64_bits_wide(path):
    assert list(narrow_products(open(path).read())) == []
