"""The scaled product's pipeline of copies, conversion and MMA, as a model of its barriers on
the CPU: a wait on a parity alone must never let a role at a stage that is not there.

An mbarrier wait names the parity of a phase, so it is also satisfied two phases early.  The
model runs the roles of one CTA in random order, with copies that land in any order, and takes
the numbers of slots and groups and the order of the converters' waits from the source."""
import os
import random
import re

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SOURCE = open(os.path.join(ROOT, "paper_2609_30846_gb300", "csrc", "ip_scaled_kernels.cuh")).read()


def constant(pattern):
    return [int(x) for x in re.search(pattern, SOURCE).groups()]


RS_32, RS_WIDE = constant(r"constexpr int RS = BN == 32 \? (\d+) : (\d+);")
FS, = constant(r"constexpr int FS = (\d+);")
GROUPS, = constant(r"CONV_GROUPS = (\d+);")


def converter_waits():
    """The barriers that a converter waits on for a stage, in the source's order."""
    at = SOURCE.index("if (turn == grp)")
    body = SOURCE[at:SOURCE.index("mbar_arrive(raw_empty(rs))", at)]
    names = re.findall(r"wait_or_dead<\w+>\((\w+)\(", body)
    assert sorted(names) == ["f16_empty", "raw_full"]
    return names


class Bar:
    def __init__(self):
        self.done = 0           # completed phases

    def passes(self, parity):
        return (self.done & 1) != parity


class Cta:
    """One CTA's pipeline; a step of a role is one item of its generator."""

    def __init__(self, rs, fs, groups, stages, waits, rng):
        self.rng, self.stages, self.waits, self.groups = rng, stages, waits, groups
        self.rs, self.fs = rs, fs
        self.raw_full, self.raw_empty = [Bar() for _ in range(rs)], [Bar() for _ in range(rs)]
        self.f16_full, self.f16_empty = [Bar() for _ in range(fs)], [Bar() for _ in range(fs)]
        self.raw, self.f16 = [None] * rs, [None] * fs      # stage that a slot holds, None while written
        self.flying, self.mmas, self.finished = [], [], 0

    def fetch(self):
        for i in range(self.stages):
            s = i % self.rs
            while not self.raw_empty[s].passes((i // self.rs & 1) ^ 1):
                yield
            self.raw[s] = None
            self.flying.append(i)
            yield

    def land(self):
        while True:
            if self.flying:
                i = self.flying.pop(self.rng.randrange(len(self.flying)))
                self.raw[i % self.rs] = i
                self.raw_full[i % self.rs].done += 1
            yield

    def convert(self, group):
        for i in range(group, self.stages, self.groups):
            r, f = i % self.rs, i % self.fs
            for name in self.waits:
                if name == "raw_full":
                    while not self.raw_full[r].passes(i // self.rs & 1):
                        yield
                    assert self.raw[r] == i, f"stage {i} read from a slot that holds {self.raw[r]}"
                else:
                    while not self.f16_empty[f].passes((i // self.fs & 1) ^ 1):
                        yield
                    assert self.finished >= i - self.fs + 1, f"stage {i} over an operand in use"
                yield
            assert self.raw[r] == i
            self.f16[f] = i
            yield
            self.f16_full[f].done += 1
            self.raw_empty[r].done += 1

    def issue(self):
        for i in range(self.stages):
            while not self.f16_full[i % self.fs].passes(i // self.fs & 1):
                yield
            assert self.f16[i % self.fs] == i
            self.mmas.append(i)
            yield

    def multiply(self):
        while True:
            if self.mmas:
                i = self.mmas.pop(0)      # in order
                assert self.f16[i % self.fs] == i
                self.finished = i + 1
                self.f16_empty[i % self.fs].done += 1
            yield

    def run(self):
        roles = [self.fetch(), self.land(), self.issue(), self.multiply()] + [
            self.convert(g) for g in range(self.groups)]
        weights = [self.rng.choice((1, 3, 30)) for _ in roles]
        for _ in range(200000):
            if self.finished == self.stages:
                return
            k = self.rng.choices(range(len(roles)), weights)[0]
            try:
                next(roles[k])
            except StopIteration:
                weights[k] = 0
        raise AssertionError("the pipeline stands still")


def hazards(rs, fs, groups, waits, runs=80):
    n = 0
    for seed in range(runs):
        try:
            Cta(rs, fs, groups, 3 * rs * groups, waits, random.Random(seed)).run()
        except AssertionError:
            n += 1
    return n


@pytest.mark.parametrize("rs", sorted({RS_32, RS_WIDE}))
def test_no_role_reads_a_stage_that_is_not_there(rs):
    assert hazards(rs, FS, GROUPS, converter_waits()) == 0


def test_the_model_sees_waits_that_are_ambiguous():
    # five raw slots: the one of a group's next stage was another group's before, so its copy may
    # still be on its way when the raw barrier is asked first; the fp16 barrier first rules it out
    assert hazards(5, 4, 4, ["raw_full", "f16_empty"]) > 0
    assert hazards(5, 4, 4, ["f16_empty", "raw_full"]) == 0
    assert hazards(8, 4, 4, ["raw_full", "f16_empty"]) == 0      # the group's own before
    assert hazards(3, 4, 4, ["f16_empty", "raw_full"]) > 0       # fewer raw slots than fp16 slots
