"""What the inline assembly of the kernels says to the compiler, read from the sources."""
import glob
import os
import re

import paper_2509_22418_amd as pp

CSRC = os.path.join(os.path.dirname(pp.lib_path()), "csrc")


def statements():
    for path in sorted(glob.glob(os.path.join(CSRC, "*.hip")) + glob.glob(os.path.join(CSRC, "*.h"))):
        text = open(path).read()
        for m in re.finditer(r"\basm\s+volatile\s*\(", text):
            depth, quoted, i = 1, False, m.end()
            while depth:          # to the closing parenthesis outside of strings
                c = text[i]
                quoted ^= c == '"' and text[i - 1] != "\\"
                depth += 0 if quoted else (c == "(") - (c == ")")
                i += 1
            yield f"{os.path.basename(path)}:{text.count(chr(10), 0, m.start()) + 1}", text[m.end():i - 1]


def clobbers(body):
    """The strings behind the third colon outside of strings and parentheses (`::` is two of them)."""
    depth, quoted, colons = 0, False, []
    for i, c in enumerate(body):
        quoted ^= c == '"' and body[i - 1] != "\\"
        if not quoted:
            depth += (c == "(") - (c == ")")
            if c == ":" and not depth:
                colons.append(i)
    return re.findall(r'"([^"]*)"', body[colons[2]:]) if len(colons) > 2 else []


def test_assembly_that_sets_m0_says_so():
    """The compiler sets m0 for its own loads into LDS and may expect it to hold what it put there."""
    writes = [(at, body) for at, body in statements() if re.search(r"\bs_\w+ m0,", body)]
    assert writes
    for at, body in writes:
        assert "m0" in clobbers(body), at
