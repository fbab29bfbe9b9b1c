"""The examples of README.md (CPU): they are Python, and a rotation takes both results of
rope_frequencies, the frequencies and the factor of the turned part.  (Queries and keys turned without
the factor have scores that are too small by its square.)"""
import ast
import os
import re

README = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "README.md")


def _statements():
    with open(README) as f:
        blocks = re.findall(r"^```python\n(.*?)^```", f.read(), re.S | re.M)
    assert len(blocks) >= 4
    return [s for b in blocks for s in ast.parse(b).body]


def test_rotations_take_the_frequencies_and_their_factor():
    made, calls = {}, 0                 # name -> which result of which call of rope_frequencies it is
    for number, s in enumerate(_statements()):
        for call in (n for n in ast.walk(s) if isinstance(n, ast.Call)):
            name = call.func.attr if isinstance(call.func, ast.Attribute) else ""
            if name in ("rope", "rope_bwd", "mala_rope", "paged_rope_write", "mala_paged_rope_write"):
                calls += 1
                given = [a.id for a in call.args if isinstance(a, ast.Name)]
                freqs = [made[a] for a in given if made.get(a, ("", 0))[0] == "frequencies"]
                factor = [k.value.id for k in call.keywords if k.arg == "scale" and isinstance(k.value, ast.Name)]
                assert len(freqs) == 1 and len(factor) == 1, ast.unparse(call)
                assert made.get(factor[0]) == ("factor", freqs[0][1]), ast.unparse(call)
        if isinstance(s, ast.Assign):
            names = [n.id for t in s.targets for n in ast.walk(t) if isinstance(n, ast.Name)]
            for n in names:
                made.pop(n, None)
            if isinstance(s.value, ast.Call) and ast.unparse(s.value.func) == "mala.rope_frequencies":
                made[names[0]], made[names[1]] = ("frequencies", number), ("factor", number)
    assert calls >= 2
