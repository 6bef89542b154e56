"""How much dynamic shared memory a kernel may be launched with is a state of the kernel in its context, not of a launch: a call that sets what
it needs itself lowers it for a launch of another host thread that has just set more.  So what a kernel is allowed is the same for every
call."""
import re

from test_launch_rule import SOURCES, code


def arguments(text, call):
    """The argument lists of `call`<..>( .. ) in the text."""
    for m in re.finditer(r"\b%s<[^;()]*>\s*\(" % call, text):
        i, depth = m.end(), 1
        while depth:
            depth += {"(": 1, ")": -1}.get(text[i], 0)
            i += 1
        yield text[m.end():i - 1]


def constant(expression):
    """Made of constants of the library and sizes of types; neither a variable nor a call."""
    return not re.sub(r"\bsizeof\(\w+\)|\(int\)|\b[A-Z][A-Z0-9_]*\b|\b\d+\b|[\s*+]", "", expression)


def test_what_a_kernel_is_allowed_is_a_constant():
    found = 0
    for f in SOURCES:
        for a in arguments(code(f), "allow_smem"):
            assert constant(a), (f, a)
            found += 1
        for a in re.findall(r"cudaFuncAttributeMaxDynamicSharedMemorySize,([^;]*)\)\);", code(f)):
            assert constant(a) or (f, a.strip()) == ("common.cuh", "(int)bytes"), (f, a)   # allow_smem() itself
            found += 1
    assert found >= 14
    assert constant("SEL_CACHE * sizeof(uint32_t)") and not constant("bytes(2)") and not constant("n * 4")
