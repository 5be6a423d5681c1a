"""The language-model loss's matrix products are written in assembly, so what the
hardware does not wait for by itself is kept apart by the kernel: looked at here in
the compiled kernels.  Between the first and the last product the sums do not move
(they are read and written by products alone); no instruction of the vector unit
writes a product's operands shortly before it; the sums are zeroed well before the
first product and read well after the last."""
import os
import re
import subprocess

import pytest

from paper_2607_20357_amd import build


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    """{name: instructions in order} of the product kernels, built as the library builds them."""
    if not os.path.exists(build.HIPCC):
        pytest.skip("no hipcc")
    asm = str(tmp_path_factory.mktemp("asm") / "lm_gemm.s")
    flags = [f for f in build.COMMON if f != "-fPIC"]
    subprocess.run([build.HIPCC] + flags + ["--cuda-device-only", "-S", "-x", "hip",
                                            os.path.join(build.CSRC, "lm_gemm.hip"), "-o", asm],
                   check=True, capture_output=True)
    text = open(asm).read()
    out = {}
    for name in re.findall(r"^(_Z\w*lm_product_kernel\w*):", text, re.M):
        body = re.search(rf"^{name}:.*?^\.Lfunc_end", text, re.S | re.M).group(0)
        lines = (l.split(";")[0].strip() for l in body.split("\n"))
        out[name] = [l for l in lines if l and not l.endswith(":") and not l.startswith(".")]
    return out


def _registers(word):
    """v[4:7] -> {("v", 4), ...}"""
    m = re.fullmatch(r"([va])\[(\d+):(\d+)\]", word) or re.fullmatch(r"([va])(\d+)", word)
    if not m:
        return set()
    first = int(m.group(2))
    last = int(m.group(3)) if m.lastindex == 3 else first
    return {(m.group(1), i) for i in range(first, last + 1)}


def _operands(line):
    return [w.strip() for w in line.split(None, 1)[1].split(",")] if " " in line or "\t" in line else []


def test_products_are_kept_apart(kernels):
    assert len(kernels) == 10          # logits and grad_w of large and small tiles, grad_x; two types
    for name, code in kernels.items():
        products = [i for i, l in enumerate(code) if l.startswith("v_mfma")]
        side = 4 if "ELi64E" in name else 8
        assert len(products) == 2 * side * side, name
        for i in products:
            d, a, b, c = _operands(code[i])
            assert d == c and d.startswith("a"), (name, code[i])
            sources = _registers(a) | _registers(b)
            for l in code[i - 3:i]:
                if l.startswith("v_") and not l.startswith("v_mfma"):
                    assert not sources & _registers(_operands(l)[0]), (name, l, code[i])
        inside = code[products[0]:products[-1]]
        assert not any("accvgpr" in l or l.startswith("scratch") for l in inside), name
        # what goes to and from the sums outside: two s_nop 15 at least between it and the products
        before = max(i for i, l in enumerate(code[:products[0]]) if "accvgpr_write" in l)
        assert sum(l == "s_nop 15" for l in code[before:products[0]]) >= 2, name
        after = next(i for i in range(products[-1], len(code)) if "accvgpr" in code[i])
        assert sum(l == "s_nop 15" for l in code[products[-1]:after]) >= 2, name
