"""No test hides another: a second function of a name would replace the first, which is then never collected."""
import ast
import glob
import os
from collections import Counter

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))


@pytest.mark.parametrize("path", sorted(glob.glob(os.path.join(HERE, "*.py"))), ids=os.path.basename)
def test_every_name_once(path):
    with open(path) as f:
        tree = ast.parse(f.read())
    for scope in [tree] + [n for n in ast.walk(tree) if isinstance(n, ast.ClassDef)]:
        names = Counter(n.name for n in scope.body if isinstance(n, (ast.FunctionDef, ast.ClassDef)))
        assert not [name for name, k in names.items() if k > 1]
