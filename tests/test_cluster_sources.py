"""A rule of the sources, no GPU: where a kernel touches another block's shared memory, all blocks of the cluster have met before the first such
access (a block that has not started has no shared memory yet) and meet after the last one (nor has one that has left)."""

import os
import re

import pytest

from paper_2604_13634_b200 import build

CSRC = os.path.join(os.path.dirname(os.path.abspath(build.__file__)), "csrc")
FILES = sorted(f for f in os.listdir(CSRC) if f.endswith(".cuh"))

MEETS = r"\bcluster_(?:meet|wait|sync_all)\("
REMOTE = r"mapa\.|(?:ld|st|red)\.(?:async\.)?shared::cluster|multicast::cluster"


def code_of(name):
    with open(os.path.join(CSRC, name)) as f:
        return re.sub(r"//[^\n]*|__launch_bounds__\([^()]*(?:<[^<>]*>)?[^()]*\)", "", f.read())


def bodies(code):
    """(is a kernel, name, body) of every function; bodies end at the first closing brace in the first column."""
    for m in re.finditer(r"^(?:template[^\n]*\n)?((?:__global__|__device__|static|inline)[^;{]*?)(\w+)\([^;{}]*\)\s*\{", code, re.M):
        end = code.find("\n}", m.end())
        one_line = code[m.end():code.find("\n", m.end())]
        yield "__global__" in m.group(1), m.group(2), one_line if one_line.rstrip().endswith("}") else code[m.end():end]


def remote_functions():
    """Device functions that reach into another block, by themselves or through others."""
    found = [(name, body) for f in FILES for kernel, name, body in bodies(code_of(f)) if not kernel]
    names = {name for name, body in found if re.search(REMOTE, body)}
    while True:
        more = {name for name, body in found if any(re.search(rf"\b{n}\(", body) for n in names)}
        if more <= names:
            return names
        names |= more


def breaks_the_rule(body, names):
    uses = [m.start() for m in re.finditer("|".join([REMOTE] + [rf"\b{n}\(" for n in sorted(names)]), body)]
    if not uses:
        return None
    meets = [m.start() for m in re.finditer(MEETS, body)]
    return not any(m < uses[0] for m in meets) or not any(m > uses[-1] for m in meets)


def kernels(name):
    return [(n, breaks_the_rule(body, remote_functions())) for kernel, n, body in bodies(code_of(name)) if kernel]


def test_the_rule_sees_what_it_is_about():
    names = remote_functions()
    assert {"in_block", "st_cluster"} <= names and "cluster_meet" not in names and "tma_load_page" not in names
    assert breaks_the_rule("int x = 1;", names) is None
    assert breaks_the_rule("cluster_arrive(); st_cluster(a, 1); cluster_meet();", names) is True
    assert breaks_the_rule("cluster_meet(); st_cluster(a, 1);", names) is True
    assert breaks_the_rule("cluster_arrive(); cluster_wait(); st_cluster(a, 1); cluster_meet();", names) is False
    seen = {n for f in FILES for n, broken in kernels(f) if broken is not None}
    assert seen == {"verify_tree_kernel", "evict_pick_kernel", "mass_kernel", "lmhead_stats_pair_kernel"}


@pytest.mark.parametrize("name", FILES)
def test_blocks_meet_around_their_accesses(name):
    assert not [n for n, broken in kernels(name) if broken]
