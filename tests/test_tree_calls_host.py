"""Calls of the operators for several new tokens that are easy to forget, on the host: nothing here launches a kernel."""

import os
import shutil
import subprocess

import numpy as np
import pytest

from oracle import tree as oracle

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2609_38095_amd", "csrc")


def sanitized(tmp_path, name, *sources):
    """Builds tests/helpers/<name>.cpp with host sources under ASan and UBSan, and runs it."""
    cxx = shutil.which("g++")
    if cxx is None:
        pytest.skip("no g++")
    exe = str(tmp_path / name)
    cmd = [cxx, "-std=c++17", "-O1", "-g", "-fno-omit-frame-pointer", "-fsanitize=address,undefined", "-fno-sanitize-recover=all",
           "-Wall", "-Wextra", "-Werror", "-I", os.path.join(ROOT, "include"), "-I", CSRC,
           os.path.join(ROOT, "tests", "helpers", name + ".cpp"), *[os.path.join(CSRC, s) for s in sources], "-o", exe]
    r = subprocess.run(cmd, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    r = subprocess.run([exe], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and name + " ok" in r.stdout, r.stdout + r.stderr


def test_checks(tmp_path):
    sanitized(tmp_path, "tree_calls_check", "zo_checks.cpp")


def test_deal(tmp_path):
    """The split of the tree attention's work over its workgroups, for random batches in every form's sizes."""
    sanitized(tmp_path, "tree_deal_check")


def test_a_walked_path_moves_once():
    """Moved twice, a path takes rows from where the first pass has put others: so a tensor that is listed twice may not."""
    cache, table, path = np.arange(4.0).reshape(1, 1, 4, 1), np.array([[0]]), np.array([[0, 2, 3]])
    once = oracle.keep(cache, table, [0], path)
    assert once.ravel().tolist() == [0, 2, 3, 3]
    assert oracle.keep(once, table, [0], path).ravel().tolist() == [0, 3, 3, 3]
