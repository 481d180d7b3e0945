"""Types of the library's sources: one definition a name, in whichever files it is seen."""
import os
import re
from collections import defaultdict

from paper_2111_06483_amd import build


def types_outside_unnamed_namespaces(text):
    """Names of the classes that a source defines in named namespaces, by its braces."""
    text = re.sub(r"//[^\n]*|/\*.*?\*/", "", text, flags=re.S)
    text = re.sub(r"(?m)^[ \t]*#(?:\\\n|[^\n])*", "", text)
    text = re.sub(r'"(?:\\.|[^"\\])*"|\'(?:\\.|[^\'\\])\'', "0", text)
    names, open_, start = [], [], 0
    for k, c in enumerate(text):
        if c == ";":
            start = k + 1
        elif c == "{":
            head = text[start:k].strip()
            if re.search(r"\bnamespace$", head):
                open_.append("unnamed")
            elif re.search(r"\bnamespace\s+\w+$", head):
                open_.append("named")
            else:
                m = re.search(r"\b(?:struct|class|union)\s+(?:__attribute__\s*\(\(.*?\)\)\s*)?(\w+(?:<[^{;]*>)?)\s*(?::[^{;]*)?$", head)
                if m and all(o == "named" for o in open_):
                    names.append(m.group(1))
                open_.append("body")
            start = k + 1
        elif c == "}":
            open_.pop()
            start = k + 1
    assert not open_
    return names


def test_the_reading_of_sources():
    text = """namespace sar { struct A { struct Inner { int x; }; };  // struct Comment {
    namespace { struct Hidden { }; } template <typename T> struct B; template <> struct B<int> : A { }; int f(struct A a) { struct Local { }; return 0; } }"""
    assert types_outside_unnamed_namespaces(text) == ["A", "B<int>"]


def test_a_type_is_defined_once():
    """Two classes of one name in one namespace of one library: the linker may take either's members for both."""
    where = defaultdict(list)
    for name in sorted(os.listdir(build.CSRC)):
        if name in build.BENCH_SOURCES or not name.endswith((".h", ".hip")):
            continue
        with open(os.path.join(build.CSRC, name)) as f:
            for t in types_outside_unnamed_namespaces(f.read()):
                where[t].append(name)
    assert "Types" in where and "Block" in where
    assert {t: files for t, files in where.items() if len(files) > 1} == {}
