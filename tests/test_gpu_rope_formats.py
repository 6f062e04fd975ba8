"""Appends with positions and drafted trees in every family of kernels: the ones that
the formats of test_gpu_append.py do not reach among them.

Appends: every head size with every pair of code widths, per-channel keys, plain
affine groups, and the rest (symmetric, rotated, fp16 metadata or a window); as single
tokens, parts of blocks, and calls whose workgroups take several heads.  Trees: every
head size and key group, with two more pairs of widths than the workloads have, fp16
metadata, rotation and fp16 tokens.
"""
import pytest

import oracle
from paper_2609_04263_amd import configs

import test_gpu_append
import test_gpu_rope as rope
import test_gpu_tree as trees

pytestmark = pytest.mark.gpu

WIDTHS = [(2, 2), (2, 4), (4, 2), (4, 4), (8, 8)]


def appended(kind, D, kb, vb):
    if kind == "per_channel":
        f = configs.make_format(kb, vb, k_axis=1, k_group=32, v_group=64, residual=64, flush=32)
    elif kind == "plain":
        f = configs.make_format(kb, vb, k_group=D // 2, v_group=32)
    elif kb == vb:
        f = configs.make_format(kb, vb, k_mode=1, v_mode=1, k_group=D, v_group=D // 2, rotate=D, meta_fp16=1)
    else:
        f = configs.make_format(kb, vb, k_mode=1, k_group=32, v_group=64, residual=32, flush=32)
    assert oracle.check_format(f, D) == 0
    return f, D


@pytest.fixture
def named(monkeypatch):
    """A name for a format, as the cases of the other modules have."""
    def name(fmt, D):
        monkeypatch.setitem(test_gpu_append.CASES, "more", (fmt, D))
        return "more"
    return name


@pytest.mark.parametrize("kb,vb", WIDTHS)
@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("kind", ["per_channel", "plain", "other"])
def test_appends(named, kind, D, kb, vb):
    name = named(*appended(kind, D, kb, vb))
    rope.append_case(name, 2, 3, [0, 1, 2, 31, 64, 100, 131, 200, 233], seed=141)
    rope.append_case(name, 2, 2, [0, 70, 71, 150], seed=142, rot=D // 2 + 16, norm=1, kind="mixed", H_q=4)
    rope.append_case(name, 1, 2, [0, 33, 34, 170], seed=143, interleaved=True, norm=1, kind="far")
    rope.append_case(name, 3, 2, [0, 1, 6, 140, 141, 165], seed=145, drafts=13, kind="mixed")


@pytest.mark.parametrize("kb,vb", WIDTHS)
@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("kind", ["per_channel", "plain", "other"])
def test_several_heads_of_a_workgroup(named, kind, D, kb, vb):
    rope.test_append_several_heads_of_a_workgroup(named(*appended(kind, D, kb, vb)), 8, 9, 1030, 1)


def drafted(D, kg, option):
    """Formats of tree kernels with key groups of 32 kg (0: per-channel keys)."""
    axis = dict(k_axis=1, k_group=32, residual=32, flush=32) if kg == 0 else dict(k_group=32 * kg)
    f = {"k2v4": lambda: configs.make_format(2, 4, v_group=32, **axis),
         "k4v2_sym_rot_meta16": lambda: configs.make_format(4, 2, k_mode=1, v_mode=1, v_group=D, rotate=D, meta_fp16=1, **axis),
         "k8v8_meta16": lambda: configs.make_format(8, 8, v_group=64, meta_fp16=1, **axis),
         "k4v4_rot_sink": lambda: configs.make_format(4, 4, v_group=64, rotate=D, sink=32, **axis)}[option]()
    assert oracle.check_format(f, D) == 0
    return f, D


FAMILIES = [(D, kg) for D in (64, 128, 256) for kg in (0, 1, 2, 4, 8) if 32 * kg <= D]


@pytest.mark.parametrize("option", ["k2v4", "k4v2_sym_rot_meta16", "k8v8_meta16", "k4v4_rot_sink"])
@pytest.mark.parametrize("D,kg", FAMILIES)
def test_trees(named, D, kg, option):
    name = named(*drafted(D, kg, option))
    for C, n_s in ((1, 1), (8, 165), (37, 70)):
        trees.run(name, [0, 1, 3], 290, n_s, C, seed=200 + C)
