"""What the sources have to keep to so that kernels launched with programmatic stream serialization, each of which may
start while its predecessor runs, stay ordered like a plain stream (the rules stand in tik_ptx.cuh)."""
import glob
import os
import re

from paper_2609_35140_b200 import build


def _sources():
    for path in sorted(glob.glob(os.path.join(build.CSRC, "*.cu*"))):
        text = re.sub(r"//[^\n]*", "", open(path).read())
        yield os.path.basename(path), re.sub(r"/\*.*?\*/", "", text, flags=re.S)


def test_no_load_that_may_move_above_the_wait():
    """__restrict__ and read-only loads tell the compiler that an input does not change while the kernel lives."""
    for name, text in _sources():
        assert not re.search(r"__restrict__|\b__ldg\b|ld\.global\.nc", text), name


def _kernels():
    for name, text in _sources():
        for body in text.split("__global__")[1:]:
            head = re.search(r"\b(\w+_kernel)\s*\(", body)
            if head:
                yield name + ": " + head.group(1), body


def test_dependents_are_released_after_the_wait_and_the_tensor_memory():
    """A dependent CTA on the same SM may allocate tensor memory before it waits: were it released while a CTA of this
    grid has yet to allocate, the two could wait for each other for ever."""
    seen = set()
    for name, body in _kernels():
        releases = [m.start() for m in re.finditer(r"\bpdl_launch_dependents\(\)", body)]
        allocs = [m.start() for m in re.finditer(r"\btmem_alloc(?:_pair)?\(", body)]
        assert releases and "pdl_wait()" in body, name
        assert body.index("pdl_wait()") < releases[0], name
        if allocs:
            assert max(allocs) < body.index("__syncthreads()", max(allocs)) < releases[0], name
            seen.add(name.split(": ")[1])
    assert seen == {"attn_kernel", "attn_persist_kernel", "attn_bwd_kernel", "decode2_kernel", "decode_cluster_kernel",
                    "linear_kernel", "linear_unit_kernel", "linear_narrow_kernel", "logprob_kernel"}


def _function(text, name):
    """The body of a kernel, without what follows it in the file."""
    at = text.index("{", re.search(r"\b%s\s*\(const EmbedParams" % name, text).start())
    depth = 0
    for i in range(at, len(text)):
        depth += {"{": 1, "}": -1}.get(text[i], 0)
        if depth == 0:
            return text[at:i + 1]


def test_what_starts_beside_the_sort_of_a_table_gradient():
    """embed_sum_kernel reads the ids and writes the table before it waits.  That is in order because whatever can come right before it
    releases it behind its own wait (so everything older has completed), and writes neither."""
    text = dict(_sources())["tik_embed.cu"]
    last = ("embed_rank_kernel", "embed_sort_kernel", "embed_wide_record_kernel")
    for name in last:
        body = _function(text, name)
        wait = body.index("pdl_wait()")
        assert body.count("pdl_wait()") == body.count("pdl_launch_dependents()") == 1 and wait < body.index("pdl_launch_dependents()"), name
        # both on every thread's way: in the kernel's outermost block, behind no return
        assert body[:wait].count("{") - body[:wait].count("}") == 1 and "return" not in body[:wait], name
        assert not re.search(r"\bp\.(ids|order|place|keys|tickets|counts|dev_status|part)\b", body[:wait]), name
        assert "d_table" not in body and not re.search(r"\bp\.ids\[[^\]]*\]\s*=[^=]", body), name
    # of the kernels of a call, one of those is the last before the sums; without tokens, when none is, the sums wait first
    launch = text[text.index("cudaError_t launch_embed_bwd("):]
    launched = re.findall(r"launch_pdl\((\w+)|return p\.fp32 \? \(p\.accumulate \? (launch_embed_sums)", launch)
    order = [a or b for a, b in launched]
    assert order == ["embed_wide_count_kernel", "embed_wide_move_kernel", "embed_wide_record_kernel", "kern", "embed_rank_kernel", "launch_embed_sums"]
    assert set(re.findall(r"auto kern = ([^;]*);", launch)[0].replace("<", " ").split()) & {"embed_sort_kernel"}
    sums = _function(text, "embed_sum_kernel")
    assert sums.index("if (p.T == 0) pdl_wait();") < min(m.start() for m in re.finditer(r"emb_fill_words|emb_store|p\.ids", sums))
