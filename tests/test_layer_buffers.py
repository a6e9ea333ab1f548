"""What a layer allocates it uses: every attribute that __init__ sets is read somewhere in the class (or handed on by it)."""
import ast
import inspect

import pytest

from paper_2203_05705_b200.delta import DeltaLayer
from paper_2203_05705_b200.glr import GlrLayer
from paper_2203_05705_b200.lm import TokenEnds


def _self_attributes(tree, kind):
    return {n.attr for n in ast.walk(tree) if isinstance(n, ast.Attribute) and isinstance(n.value, ast.Name) and n.value.id == "self" and isinstance(n.ctx, kind)}


@pytest.mark.parametrize("layer", [DeltaLayer, GlrLayer, TokenEnds])
def test_every_buffer_is_read(layer):
    tree = ast.parse(inspect.getsource(layer))
    init = next(f for f in tree.body[0].body if isinstance(f, ast.FunctionDef) and f.name == "__init__")
    assert _self_attributes(init, ast.Store) <= _self_attributes(tree, ast.Load)
