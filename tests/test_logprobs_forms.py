"""The forms of short rows of logits go by a rule on their length, read from the source on the CPU: every number of units that the
next one doubles has a form with one element more a lane, none of them alone."""
import os
import re

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SOURCE = open(os.path.join(ROOT, "paper_2609_30846_gb300", "csrc", "ip_logprobs.cu")).read()


def forms():
    """[(longest row, units, elements more)] of the warp's forms, in the source's order."""
    hold = lambda units: 32 * units * 8 - 8
    assert "return threads * units * 8 - (on16 ? 0 : 8);" in SOURCE
    found = re.findall(r"if \(prm\.V <= hold\(32, (\d+)\)( \+ 32)?\) return launch<T, 32, (\d+), (\d+), ipl::WHOLE>", SOURCE)
    assert len(found) == SOURCE.count("launch<T, 32,")
    return [(hold(int(h)) + (32 if more else 0), int(u), int(s)) for h, more, u, s in found]


def test_one_rule_for_every_number_of_units():
    f = forms()
    assert [n for n, _, _ in f] == sorted(n for n, _, _ in f)
    units = sorted({u for _, u, _ in f})
    assert units == [1, 2, 4, 8] and {u for _, u, s in f if s == 0} == set(units)
    assert {u for _, u, s in f if s} == {u for u in units if 2 * u in units}


def test_every_form_holds_its_longest_row():
    # a row starts up to seven elements behind 16 bytes; the elements more lie behind the units
    for longest, units, more in forms():
        for shift in range(8):
            assert longest + shift <= 32 * (units * 8 + more)
