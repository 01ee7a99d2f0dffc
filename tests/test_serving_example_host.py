"""What the example server refuses before it asks for a GPU."""
import importlib.util
import os
import types

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_contexts_that_are_cut_need_exact_layers():
    spec = importlib.util.spec_from_file_location("serve_example", os.path.join(ROOT, "examples", "serve.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    with pytest.raises(ValueError, match="approximated"):
        module.Server(types.SimpleNamespace(approximated={3}, layers=[None] * 4), keep=256)
