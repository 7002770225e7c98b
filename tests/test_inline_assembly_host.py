"""Inline assembly of the kernels says which special registers it writes (the text of the sources; no GPU needed)."""
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2203_04071_amd", "csrc")


def statements(text):
    """The asm statements of a source, with macros that stand for pieces of assembly put in."""
    macros = dict(re.findall(r'^[ \t]*#define[ \t]+(\w+)[ \t]+("(?:[^\n]|\\\n)*)$', text, re.M))
    for m in re.finditer(r"\basm(?:\s+volatile)?\s*\(", text):
        depth, at = 1, m.end()
        while depth:                                # (parentheses inside strings pair up in this code)
            depth += {"(": 1, ")": -1}.get(text[at], 0)
            at += 1
        body = text[m.end():at - 1]
        for name, value in macros.items():
            body = re.sub(r"\b%s\b" % name, lambda _: value, body)
        yield text.count("\n", 0, m.start()) + 1, body


def undeclared(text):
    return [line for line, body in statements(text) if re.search(r"\bs_mov_b32 m0\b", body) and '"m0"' not in body]


def test_every_statement_that_writes_m0_says_so():
    seen, bad = 0, []
    for name in sorted(os.listdir(CSRC)):
        with open(os.path.join(CSRC, name)) as f:
            text = f.read()
        seen += sum("m0" in body for _, body in statements(text))
        bad += [(name, line) for line in undeclared(text)]
    assert seen >= 8 and not bad, bad


def test_the_reader_itself():
    op = '#define OP "s_mov_b32 m0, %[to]\\n\\t" \n'
    assert undeclared('asm volatile("s_mov_b32 m0, %0" : : "s"(f(x)) : "memory");') == [1]
    assert undeclared('asm volatile("s_mov_b32 m0, %0" : : "s"(f(x)) : "memory", "m0");') == []
    assert undeclared(op + 'asm volatile("s_nop 0\\n\\t" OP : : [to] "s"(x) : "memory");') == [2]
    assert undeclared(op + 'asm(OP : : [to] "s"(x) : "m0", "scc");') == []
