"""Rules that every kernel keeps and no run can show reliably, checked on the sources."""
import glob
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2607_14695_b200", "csrc")


def _kernels():
    """(file: name, parameters, body) of every __global__ function; comments taken out."""
    out = []
    for path in sorted(glob.glob(os.path.join(CSRC, "*.cu")) + glob.glob(os.path.join(CSRC, "*.cuh"))):
        text = re.sub(r"//[^\n]*|/\*.*?\*/", "", open(path).read(), flags=re.S)
        for m in re.finditer(r"__global__\s+void\s+(?:__\w+__\((?:[^()]|\([^()]*\))*\)\s*)*(\w+)\s*\(([^{]*?)\)\s*\{", text):
            depth, i = 1, m.end()
            while depth:
                depth += {"{": 1, "}": -1}.get(text[i], 0)
                i += 1
            out.append((f"{os.path.basename(path)}: {m.group(1)}", m.group(2), text[m.end():i]))
    return out


KERNELS = _kernels()


def test_kernels_are_found():
    names = {n.split(": ")[1] for n, _, _ in KERNELS}
    assert {"chain_attn_kernel", "attn_pair_kernel", "chain_gemm_kernel", "chain_in_kernel", "tile_gemm_kernel", "attn_tc2_kernel", "gate_kernel",
            "flow_step_kernel", "init_static_kernel", "linear_half_kernel", "linear_res_tc_kernel"} <= names


def test_attention_kernels_are_the_ones_a_call_can_reach():
    """(Clusters of four with 128 rows per CTA were left with groups of 128 heads of 256 inside a step, which refuses more than 12288 / 256 heads.)"""
    assert {n.split(": ")[1] for n, _, _ in KERNELS if re.search(r"(attn|attention)_?\w*kernel", n)} == {
        "attn_merge_kernel", "attn_pair_kernel", "attn_simt_kernel", "attn_tc2_kernel", "attn_tc_kernel", "chain_attn_kernel"}


@pytest.mark.parametrize("kernel", [k for k in KERNELS if "tmem_alloc" in k[2]], ids=lambda k: k[0])
def test_tensor_memory_is_taken_before_dependents_are_released(kernel):
    """A dependent grid may move in as soon as it is released. If it takes tensor memory that this grid has yet to take, the two wait
    for one another."""
    _, _, body = kernel
    assert body.index("tmem_alloc") < body.index("griddepcontrol.launch_dependents")


@pytest.mark.parametrize("kernel", [k for k in KERNELS if re.search(r"griddepcontrol\.wait|wait_then_release", k[2])], ids=lambda k: k[0])
def test_inputs_read_behind_the_wait_may_not_be_taken_for_constants(kernel):
    """A programmatically launched grid may run beside the one that writes its inputs. A const __restrict__ parameter promises that
    nobody writes it while the kernel runs, so its loads could be moved ahead of the wait. (The weights of the plain gate kernels, which
    wait_prior marks, are read ahead of it on purpose: the launch in front of them writes none.)"""
    _, params, _ = kernel
    bad = re.findall(r"const [^,]*__restrict__ (\w+)", params)
    assert not [b for b in bad if not ("wait_prior" in params and b in ("W", "bias"))], bad


PROJECTIONS = [k for k in KERNELS if k[0].split(":")[0] in ("tile_gemm.cu", "linear_half.cu", "linear_tc.cu", "qkv_tc.cu", "chain_gemm.cu", "gate_tc.cu") and "commit" in k[2]]


@pytest.mark.parametrize("kernel", PROJECTIONS, ids=lambda k: k[0])
def test_sums_are_announced_only_when_complete(kernel):
    """After a wait that ran out a contraction is not complete. The warps that read the accumulator (in a pair those of the other CTA, which sees nothing
    of the failed wait) may take it for complete only by the barrier that the last commit arrives on: no commit, no result but NaN."""
    commits = re.findall(r"([^;{}]*)\bumma2?_commit\w*\(bar\w*(?:\((?:S::)?(\w+))?", kernel[2])
    last = [before for before, name in commits if name.endswith("_ACC") or not name]
    assert last and all(re.search(r"if \(ok\)\s*$", b) for b in last), last


@pytest.mark.parametrize("kernel", PROJECTIONS, ids=lambda k: k[0])
def test_a_tile_of_a_failed_wait_is_written_as_nan(kernel):
    """A store that is left out keeps what the last call wrote: the result is written whatever the waits said, and is NaN where one ran out."""
    _, _, body = kernel
    assert "0x7fc00000" in body
    assert not re.search(r"if \([^()]*\bok && (?:m0|dst)|if \(!ok \|\| f >=", body)


def test_a_reported_wait_names_its_kernel():
    """The status word holds a number for every wait: kernels count theirs from bases of their own, far enough apart."""
    header = open(os.path.join(CSRC, "reflex_internal.cuh")).read()
    sites = {n: int(v) for n, v in re.findall(r"(kSite\w+) = (\d+)", header)}
    used = {}
    for name, _, body in KERNELS:
        assert len(re.findall(r"atomicCAS\((?:p\.)?status,", body)) == len(re.findall(r"atomicCAS\((?:p\.)?status, 0u, status_word\(kSite", body)), name
        for base in set(re.findall(r"status_word\((kSite\w+)", body)):
            last = max([int(c) for c in re.findall(r"\bwait(?:_slow|_cl)?\([^;]*?, (\d+)u?\)", body)] + [int(c) for c in re.findall(base + r" \+ (\d+)u", body)] + [0])
            used[base] = (name, last)
    assert len(used) == len({n for n, _ in used.values()}) == 12, used       # one base a kernel, no two kernels on one
    bases = sorted(sites[b] for b in used) + [sites["kSiteEnd"]]
    for base, (name, last) in used.items():
        assert sites[base] + last < min(b for b in bases if b > sites[base]), name


# ---- the exchange of a row's threads in page_chunk_kernel ----

def _body(name):
    return next(body for n, _, body in KERNELS if n.endswith(": " + name))


def test_a_reference_is_not_written_where_the_row_s_other_thread_reads_it():
    """Behind the barrier of a tile both threads of a row read the reference that the other softmax group has left, and one of them writes the group's own: nothing orders
    the two, so they may not be one place."""
    body = _body("page_chunk_kernel")
    written = re.findall(r"\bref\[([^;=]+?)\] = ", body)
    read = re.findall(r"[:(,=] ref\[([^;=]+?)\][;,)]", body)
    assert written == ["group * 128 + row"] and read == ["(group ^ 1) * 128 + row"], (written, read)


def test_maxima_of_a_group_s_next_tile_go_to_another_place():
    """The maxima of a tile are read behind its barrier, and the next tile's are written with no barrier between. Tiles of a group are two apart where there are two groups."""
    body = _body("page_chunk_kernel")
    place = re.search(r"const int meet = \(\((.*?)\) \* 128 \+ row\) \* 2;", body)
    assert place and not re.search(r"maxima\[(?!meet \+ half\])|maxima \+ (?!meet\))", body), place
    for groups in (1, 2):
        at = [eval(place.group(1).replace("NG", str(groups)), {"gi": gi}) for gi in range(16)]
        assert all(a != b for a, b in zip(at, at[groups:])) and max(at) < 2 * groups          # a group's tile and its next one
        for gi in range(14):                                                                   # and no group writes where the other one reads
            assert groups == 1 or at[gi] not in (at[gi + 1], at[gi + 2])


def test_a_unit_without_tiles_leaves_no_sums():
    """A softmax group that is ahead does not meet the other one at a unit without tiles. What it wrote there would be in the place of a unit that the other group may
    not have finished."""
    assert re.findall(r"([^;{}]*)\bsums\[[^;=]*\] = ", _body("page_chunk_kernel"))[0].strip() == "if (n > 0)"


def test_32_byte_stores_to_the_caller_s_rows_look_at_their_address():
    """Outputs are promised 16-byte alignment. A store of 32 bytes faults on any other multiple of 16: of the paged prefix, those that do not go to the workspace come behind a
    look at the address."""
    text = open(os.path.join(CSRC, "page_rows.cu")).read()
    stores = re.findall(r"([^\n;{}]*)\bptx::st_global_v8\(", text)
    assert stores and all(s.strip() == "if (sectors)" for s in stores), stores
    assert re.search(r"const bool sectors = \(\(reinterpret_cast<uintptr_t>\(k_out\) \| reinterpret_cast<uintptr_t>\(v_out\)\) & 31u\) == 0;", text)


def test_a_reported_wait_of_the_pages_names_its_kernel():
    """Their waits are reported through report_page_wait, with numbers from a base of the kernel's own; the table gives every base's kernel, in order."""
    sites = {n: int(v) for n, v in re.findall(r"(kSite\w+) = (\d+)", open(os.path.join(CSRC, "reflex_internal.cuh")).read())}
    used = {}
    for name, _, body in KERNELS:
        calls = re.findall(r"report_page_wait\([^,]*, (\w+) \+ (\w+)\)", body)
        assert len(calls) == body.count("report_page_wait("), name
        if calls:
            assert len({b for b, _ in calls}) == 1, calls
            codes = [int(c) for c in re.findall(r"\bwait\([^;]*?, (\d+)\)", body)] + [int(c[:-1]) for _, c in calls if c != "code"]
            used[calls[0][0]] = (name.split(": ")[1], max(codes))
    assert {n for n, _ in used.values()} == {"page_chunk_kernel", "page_token_kernel"} and len(used) == 2, used
    table = re.findall(r'\{(kSite\w+), "(\w+)"\}', open(os.path.join(CSRC, "reflex_api.cu")).read())
    ends = [sites[e] for e, _ in table]
    assert ends == sorted(ends) and table[-1][0] == "kSiteEnd"
    for base, (name, last) in used.items():
        for site in (sites[base] + 1, sites[base] + last):
            assert next(n for e, n in table if site < sites[e]) == name


def test_every_call_on_pages_looks_at_the_device():
    """The pages' calls are refused while another device is current: with another device's NULL stream the status word would be read ahead of the kernels that
    write it. (reflex_pages_destroy touches host memory alone.)"""
    text = re.sub(r"//[^\n]*|/\*.*?\*/", "", open(os.path.join(CSRC, "pages_api.cu")).read(), flags=re.S)
    calls = re.findall(r"\nint (reflex_pages_\w+)\(reflex_pages_t \*p\b[^{]*\{(.*?)\n\}\n", text, flags=re.S)
    assert {n for n, _ in calls} == {"reflex_pages_destroy", "reflex_pages_check_status", "reflex_pages_write", "reflex_pages_read", "reflex_pages_attention"}
    assert "return check_device(p);" in re.search(r"int check_call\(.*?\n\}\n", text, flags=re.S).group(0)
    for name, body in calls:
        assert name == "reflex_pages_destroy" or re.search(r"(?:const int|int) rc = check_(?:call|device)\(p", body), name


def test_kernels_of_the_paged_prefix_are_the_ones_a_call_can_reach():
    assert {n for n, _, _ in KERNELS if re.match(r"(page\w*|rotary)\.cuh?: ", n)} == {
        "rotary.cu: rotary_axes_kernel", "page_rows.cu: page_write_kernel", "page_rows.cu: page_read_kernel", "page_plain.cu: page_plain_kernel",
        "page_token.cu: page_token_kernel", "page_chunk.cu: page_chunk_kernel", "page_chunk.cu: page_widen_kernel", "page_merge.cu: page_merge_kernel"}
    for name, launcher in (("rotary_axes", "launch_rotary_axes"), ("page_write", "launch_page_write"), ("page_read", "launch_page_read"), ("page_plain", "launch_page_plain"),
                           ("page_token", "launch_page_token"), ("page_chunk", "launch_page_chunk"), ("page_widen", "launch_page_widen"), ("page_merge", "launch_page_merge")):
        assert f" = {launcher}(" in open(os.path.join(CSRC, "pages_api.cu")).read(), name


def test_the_issuer_of_both_products_does_not_wait_for_keys_ahead_of_a_product_that_is_due():
    """The producer of keys lists units as far as the list has room, and an entry is free once its unit's last P V is done. A warp that issues both products and waited for the next tile's
    keys with that P V still to be issued would wait for itself, through units without tiles that fill the list."""
    body = _body("page_chunk_kernel")
    both = body[body.index("bool ok = true, end = false"):body.index("float *maxima")]
    assert "wait(L::KFULL" not in both and "if (!keys_or_due()) break;" in both
    assert "if (q > v && all(mbar_test_wait(due, v_bph))) return false;" in both
