"""The rule that gives a product of 8-bit rows its tile, against measured calls in all three tiles, and the strips of a launch (host
code; nothing is launched)."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def rule(tmp_path_factory):
    if shutil.which("g++") is None:
        pytest.skip("no host C++ compiler")
    exe = str(tmp_path_factory.mktemp("rule") / "product_rule")
    r = subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Wextra", "-Werror", "-I", os.path.join(ROOT, "paper_2605_28396_amd", "csrc"),
                        os.path.join(ROOT, "tests", "product_rule_main.cpp"), "-o", exe], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0, r.stderr

    def ask(calls):
        text = "".join("%d %d %d %d\n" % c for c in calls)
        out = subprocess.run([exe], input=text, capture_output=True, text=True, timeout=120, check=True).stdout
        return [[float(x) for x in line.split()] for line in out.splitlines()]
    return ask


def _measured():
    calls = []
    for line in open(os.path.join(ROOT, "profiles", "token_scoring_tiles.txt")):
        if not line.startswith("#"):
            f = line.split()
            calls.append((tuple(int(x) for x in f[:4]), [float(x) for x in f[4:7]], f[7:] == ["check"]))
    return calls


def test_the_rule_takes_the_fast_tile(rule):
    calls = _measured()
    assert len(calls) > 300
    lost, off = {False: [], True: []}, {False: [], True: []}
    for (_, us, check), got in zip(calls, rule([c for c, _, _ in calls])):
        lost[check].append(us[int(got[0])] / min(us) - 1)
        off[check] += [got[1 + 3 * i] / us[i] - 1 for i in range(3)]
    # what the comment beside the rule says of it
    assert max(lost[False]) <= 0.04 and sum(lost[False]) / len(lost[False]) <= 0.0015
    assert sorted(lost[True])[-3] <= 0.04 and max(lost[True]) <= 0.11
    for check, rms, most in ((False, 0.09, 0.49), (True, 0.11, 0.32)):
        assert (sum(x * x for x in off[check]) / len(off[check])) ** 0.5 <= rms and max(abs(x) for x in off[check]) <= most


def test_launches_hold(rule):
    """Calls of the most rows: fewer than 2^32 threads, whatever the tile."""
    calls = [(T, V, 128, 2) for T in (2 ** 24 - 1, 2 ** 24 - 65, 15796645, 15349619, 5219489, 7067305, 65537) for V in (1, 300, 8579, 8841, 19363, 26249, 2 ** 28)]
    for call, got in zip(calls, rule(calls)):
        assert all(got[3 + 3 * i] == 1 and got[2 + 3 * i] >= 1 for i in range(3)), call
