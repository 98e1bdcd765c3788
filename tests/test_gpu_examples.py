"""The examples, at a small size."""

import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _load(name):
    spec = importlib.util.spec_from_file_location(name, os.path.join(ROOT, "examples", name + ".py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def test_on_policy_distillation_learns():
    kl, off = _load("on_policy_distillation").train(steps=30, vocab=200, batch=32, length=16, k=20)
    assert kl[-1] < 0.5 * kl[0]     # the student comes nearer to its teacher
    assert off < 4e-6               # what the draw records is what the loss computes
