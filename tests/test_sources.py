"""The C++ sources as text: what a compiler that sees one of them at a time does not check."""

import os
import re

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2609_21827_amd", "csrc")


def _types(text):
    """Names of the structs and classes that a source gives a body outside of functions, other
    types and anonymous namespaces; specialisations with their arguments."""
    text = re.sub(r"//[^\n]*|/\*.*?\*/", " ", text, flags=re.S)
    text = re.sub(r'"(\\.|[^"\\\n])*"|\'(\\.|[^\'\\\n])+\'', " 0 ", text)
    text = re.sub(r"^[ \t]*#(\\\n|[^\n])*", " ", text, flags=re.M)
    names, inside, head = [], [], ""
    for part in re.split(r"([{};])", text):
        if part == "{":
            space = re.search(r"\b(?:namespace\b\s*(\w*)|extern\s+0)\s*$", head.rstrip())
            kind = None if space is None else space.group(1)
            body = re.search(r"\b(?:struct|class)\s+(?:alignas\s*\([^)]*\)\s*)?(\w+\s*(?:<[^;{}()=]*>)?)"
                             r"\s*(?:final\s*)?(?::[^:].*)?$", head.strip(), flags=re.S)
            if body and all(inside):
                names.append(re.sub(r"\s+", "", body.group(1)))
            inside.append(kind or ("extern" if space is not None and "namespace" not in space.group(0)
                                   else ""))
            head = ""
        elif part == "}":
            inside.pop()
            head = ""
        elif part == ";":
            head = ""
        else:
            head += part
    assert not inside
    return names


def test_the_reading_of_types():
    assert _types("namespace a { struct X { int y; struct Z { }; }; template <int N> struct Y<N, 2> : X {};"
                  "namespace { struct W {}; } void f() { struct V {}; } struct U; extern const U u; }"
                  "typedef struct t { int a; } t; struct X* g(struct X x) { return 0; }") == \
        ["X", "Y<N,2>", "t"]


def test_no_type_has_two_bodies():
    """A type of more than one source, anonymous namespaces aside, stands in a header they
    share: two bodies of a name make the program's meaning undefined, and nothing says so."""
    where = {}
    for name in sorted(os.listdir(CSRC)):
        if name.endswith((".h", ".hip", ".cpp")):
            with open(os.path.join(CSRC, name)) as f:
                for t in _types(f.read()):
                    where.setdefault(t, []).append(name)
    assert len(where) > 10
    assert not {t: files for t, files in where.items() if len(files) > 1}
