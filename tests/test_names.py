"""No test hides another: in one module a second definition of a name replaces the
first, which then never runs."""
import ast
import glob
import os

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))


@pytest.mark.parametrize("path", sorted(glob.glob(os.path.join(HERE, "*.py"))), ids=os.path.basename)
def test_defined_once(path):
    with open(path) as f:
        tree = ast.parse(f.read())
    scopes = [tree] + [n for n in tree.body if isinstance(n, ast.ClassDef)]
    for scope in scopes:
        names = [n.name for n in scope.body if isinstance(n, (ast.FunctionDef, ast.AsyncFunctionDef, ast.ClassDef))]
        twice = {n for n in names if names.count(n) > 1}
        assert not twice, twice
