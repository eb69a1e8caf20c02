"""Copies into LDS that the 128-row kernel of the 8-bit cache issues by hand: none may be under way when a wave ends, since the memory
that they write is reused by the merge before that and by other workgroups after it.  Followed through the kernels' instructions."""
import os
import re
import subprocess

from paper_2404_12457_amd import build


def _kernels(text):
    name, body = None, []
    for line in text.splitlines():
        line = line.split(";")[0].strip()
        start = re.match(r"(_Z\w+):$", line)
        if start:
            name, body = start[1], []
        elif line.startswith(".Lfunc_end"):
            if name:
                yield name, body
            name = None
        elif name and line:
            body.append(line)


def _copies_at_the_end(body):
    """Copies that some path through the instructions leaves without a wait for all of them between copy and end."""
    at = {line[:-1]: i for i, line in enumerate(body) if line.endswith(":")}
    seen, todo, left = [set() for _ in body], [(0, None)], []
    while todo:
        i, copy = todo.pop()
        while copy not in seen[i]:
            seen[i].add(copy)
            line = body[i]
            if line.startswith("global_load_lds"):
                copy = line.split()[0]
            elif line.startswith("s_waitcnt") and "vmcnt(0)" in line:
                copy = None
            elif line.startswith("s_endpgm"):
                left += [copy] if copy else []
                break
            jump = re.match(r"s_(c?)branch\S*\s+(\S+)", line)
            if jump and jump[1]:
                todo.append((at[jump[2]], copy))
            i = at[jump[2]] if jump and not jump[1] else i + 1
    return left


def test_the_walk_finds_a_copy_that_nothing_waits_for():
    loop = ["global_load_lds_dword v[0:1], off", ".L0:", "s_waitcnt vmcnt(0) lgkmcnt(0)", "s_barrier"]
    assert not _copies_at_the_end([*loop, "s_cbranch_scc1 .L0", "s_endpgm"])
    assert _copies_at_the_end([*loop, "global_load_lds_dword v[0:1], off", "s_cbranch_scc1 .L0", "s_waitcnt vmcnt(1)", "s_endpgm"]) == ["global_load_lds_dword"]
    assert not _copies_at_the_end([*loop, "global_load_lds_dword v[0:1], off", "s_branch .L0", "s_endpgm"])


def test_no_copy_into_lds_outlives_the_key_loop(tmp_path):
    out = str(tmp_path / "kv8_attn.s")
    subprocess.run(["hipcc", *build.FLAGS, "--offload-device-only", "-S", os.path.join(build.CSRC, "kv8_attn.hip"), "-o", out], check=True, capture_output=True)
    kernels = {n: b for n, b in _kernels(open(out).read()) if any(x.startswith("global_load_lds") for x in b)}
    assert len(kernels) == 8  # head_dim, wave groups, request list
    assert {n: _copies_at_the_end(b) for n, b in kernels.items()} == {n: [] for n in kernels}
