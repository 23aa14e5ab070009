"""Calls of the operators beside the plan that are easy to get wrong around the kernels: how names, gradients, layouts and sizes are taken and refused."""
import subprocess
import sys

import pytest

torch = pytest.importorskip("torch")

import paper_2506_06095_amd as smha  # noqa: E402


def test_a_name_is_looked_up_once():
    """In a fresh process: the package resolves an operator's name at its first use and then holds it."""
    code = ("import paper_2506_06095_amd as smha\n"
            "names = sorted(smha._OPERATORS)\n"
            "assert not any(n in vars(smha) for n in names)\n"
            "first = [getattr(smha, n) for n in names]\n"
            "assert all(vars(smha).get(n) is f for n, f in zip(names, first))\n"
            "try:\n    smha.no_such_operator\nexcept AttributeError:\n    pass\nelse:\n    raise SystemExit('found')\n")
    subprocess.run([sys.executable, "-c", code], check=True, cwd=smha.__path__[0] + "/..")
