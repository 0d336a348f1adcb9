"""The rule of test_kernel_protocols.py in the functions that kernels are made of: whether a thread arrives at a barrier of many,
the cluster's and the arrivals without a wait included, must not depend on how a bounded wait of its own ended."""
import glob
import os
import re

import pytest

import test_kernel_protocols as protocols

SOURCES = sorted(os.path.basename(p) for p in glob.glob(os.path.join(protocols.CSRC, "*.cu*")))
BARRIER = re.compile(r"\b(named_barrier_sync|named_barrier_arrive|__syncthreads\w*|cluster_arrive|cluster_wait)\s*\(")


def functions(path):
    """[(name, body without comments)] of a source file's device functions."""
    with open(path) as f:
        text = f.read()
    text = re.sub(r"//[^\n]*", "", re.sub(r"/\*.*?\*/", "", text, flags=re.S))
    found = []
    for m in re.finditer(r"__device__\b[^;{}()]*?\b(\w+)\s*\(", text):
        at, depth = m.end(), 1
        while depth:                                          # (behind the parameters)
            depth += {"(": 1, ")": -1}.get(text[at], 0)
            at += 1
        rest = re.match(r"\s*(?:const\s*)?\{", text[at:])
        if not rest:
            continue                                          # (a declaration, a constructor's list)
        at += rest.end()
        depth, end = 1, at
        while depth:
            depth += {"{": 1, "}": -1}.get(text[end], 0)
            end += 1
        found.append((m.group(1), text[at:end - 1]))
    return found


@pytest.mark.parametrize("source", SOURCES)
def test_no_barrier_of_a_function_stands_behind_one_threads_wait(source, monkeypatch):
    monkeypatch.setattr(protocols, "BARRIER", BARRIER)
    for name, body in functions(os.path.join(protocols.CSRC, source)):
        assert not protocols.barriers_behind_a_wait("{" + body + "}"), name      # (so that a return leaves something)


def test_the_functions_are_found():
    names = [n for n, _ in functions(os.path.join(protocols.CSRC, "tree_tc.cu"))]
    for n in ("cache_part", "umma_load", "umma_logits", "umma_sums", "umma_softmax", "tree_part"):
        assert n in names
    body = dict(functions(os.path.join(protocols.CSRC, "tree_tc.cu")))["umma_softmax"]
    assert len(re.findall(protocols.WAIT, body)) >= 4 and len(BARRIER.findall(body)) >= 4
    assert "join_rows_of" in [n for n, _ in functions(os.path.join(protocols.CSRC, "tree_common.cuh"))]


def test_arrivals_count(monkeypatch):
    ok = "bool ok = wait_all(&a, 0, f); "
    monkeypatch.setattr(protocols, "BARRIER", BARRIER)
    assert protocols.barriers_behind_a_wait(ok + "if (ok) tc::named_barrier_arrive(5, 192);")
    assert protocols.barriers_behind_a_wait("{" + ok + "if (!ok) return; tree::cluster_arrive(); }")
    assert not protocols.barriers_behind_a_wait(ok + "if (ok) x(); cluster_arrive();")


def arrivals_in_spite_of_a_wait(body):
    """The arrivals on an mbarrier that a thread makes behind a bounded wait, however that ended: neither their statement nor a
    block around it asks for the outcome, and no way out that does lies before them.  Arrivals without the waits between
    them run ahead of what they stand for: a ring's place passes for free while a copy into it is in flight, and the barrier of
    that copy is armed a second time.  (Those on places, which are named empty or free; a barrier of one phase has nothing to
    run ahead of.)"""
    wait = protocols.WAIT
    outcomes = set(re.findall(r"(\w+)\s*=[^=;{}]*" + wait, body))
    while outcomes:
        more = set(re.findall(r"(\w+)\s*=[^=;{}]*\b(?:%s)\b" % "|".join(outcomes), body))
        if more <= outcomes:
            break
        outcomes |= more
    decided = re.compile(wait + "".join(r"|\b%s\b" % n for n in sorted(outcomes)))
    found, stack, start, i, waited = [], [False], 0, 0, False
    while i < len(body):
        if body[i] == "(":
            depth = 1
            while depth:
                i += 1
                depth += {"(": 1, ")": -1}.get(body[i], 0)
        if body[i] in "{;}":
            words = body[start:i]
            asks = bool(re.search(r"\b(if|while|for)\s*\(|&&", words)) and bool(decided.search(words))
            if re.search(r"\bmbar_arrive\s*\([^;]*(?:empty|\bfree)\b", words) and waited and not asks and not any(stack):
                found.append(" ".join(words.split()))
            waited |= bool(re.search(wait, words))
            if asks and re.search(r"\b(break|continue|return)\b", words):
                stack[-1] = True                              # (the rest of this block)
            if body[i] == "{":
                stack.append(asks)
            elif body[i] == "}" and len(stack) > 1:
                stack.pop()
            start = i + 1
        i += 1
    return found


@pytest.mark.parametrize("source", SOURCES)
def test_who_has_given_up_announces_nothing(source):
    path = os.path.join(protocols.CSRC, source)
    for name, body in protocols.kernels(path) + functions(path):
        assert not arrivals_in_spite_of_a_wait(body), name


def test_the_rule_on_arrivals_finds_what_it_is_for():
    assert arrivals_in_spite_of_a_wait("ok = ok && wait_all(&f, 0, a); x(); mbar_arrive(&empty);")
    assert arrivals_in_spite_of_a_wait("for (;;) { if (n) { ok = wait_all(&f, 0, a) && ok; mbar_arrive(&empty); } }")
    assert not arrivals_in_spite_of_a_wait("ok = ok && wait_all(&f, 0, a); if (ok) mbar_arrive(&empty);")
    assert not arrivals_in_spite_of_a_wait("ok = ok && wait_all(&f, 0, a); if (ok) { x(); mbar_arrive(&empty); }")
    assert not arrivals_in_spite_of_a_wait("for (;;) { if (!wait_all(&f, 0, a)) break; mbar_arrive(&empty); }")
    assert not arrivals_in_spite_of_a_wait("mbar_arrive(&empty); ok = wait_all(&f, 0, a);")


def test_who_waits_for_a_copy_of_v_follows_every_one():
    """The wait for a phase of a barrier takes the phase before the last for the one to come.  So it is for warps that wait for
    every tile of a ring, one after the other: one that takes every second tile of V, say, and only looks at the last one's
    barrier, may be as far ahead of the copies as the logits let it be.  (K's it may look at: its place is filled again only
    behind its own arrival, and the logits that it has waited for are behind the copy.)"""
    waits = [(n, b) for n, b in functions(os.path.join(protocols.CSRC, "tree_tc.cu")) if re.search(r"full\[1\]", b)]
    assert [n for n, _ in waits] == ["umma_sums"]
    assert re.search(r"for \(int t = 0; ok && t < tiles; \+\+t\)", waits[0][1])
