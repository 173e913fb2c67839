"""Importing the package loads nothing, neither the library nor torch (no GPU needed)."""
import os
import subprocess
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

OPERATORS = ["Routing", "State8", "adamw_state", "adamw_state_values", "adamw_step", "combine", "combine_gradient", "grouped_product",
             "grouped_weight_gradient", "route", "route_gradient"]


def _run(code):
    return subprocess.run([sys.executable, "-c", code], cwd=ROOT, capture_output=True, text=True, timeout=300)


def test_the_package_comes_without_torch():
    run = _run("import sys; sys.modules['torch'] = None\n"          # (an import of it would fail)
               "import paper_2505_15511_amd as nomad\n"
               "assert nomad.NomadConfig and nomad.knn_in_clusters and nomad.binding._lib is None\n"
               f"assert set({OPERATORS!r}) <= set(dir(nomad)) and set({OPERATORS!r}) <= set(nomad.__all__)\n"
               "assert not hasattr(nomad, 'no_such_name')")
    assert run.returncode == 0, run.stderr


def test_their_module_comes_when_asked_for():
    run = _run("import paper_2505_15511_amd as nomad\nassert 'operators' in dir(nomad) and nomad.operators.route is nomad.route\n"
               "import paper_2505_15511_amd.operators as again\nassert again is nomad.operators")
    assert run.returncode == 0, run.stderr


def test_operators_come_when_asked_for():
    run = _run(f"import paper_2505_15511_amd as nomad\nnames = {OPERATORS!r}\n"
               "from paper_2505_15511_amd import operators, route\n"
               "assert route is operators.route and all(getattr(nomad, n) is getattr(operators, n) for n in names)\n"
               "space = {}\nexec('from paper_2505_15511_amd import *', space)\n"
               "assert all(n in space for n in names + ['Nomad', 'pca_init'])")
    assert run.returncode == 0, run.stderr
