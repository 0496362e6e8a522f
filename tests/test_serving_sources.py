"""Properties of the serving kernels' sources that no run can show reliably: checked on the text."""
import re

from tests.test_kernel_sources import _sources


def _kernel(text, name):
    return re.search(r"\b%s\(const __grid_constant__.*?\n\}\n" % name, text, re.S).group(0)


def test_serving_kernels_wait_for_what_is_before_them():
    # all of them are launched as programmatic dependents: nothing is read from global memory ahead of the wait, and every kernel waits,
    # so that completion stays transitive along the stream
    sources = dict(_sources())
    for name, kernels in (("kernels_paging.cuh", ("page_tables", "rope_store_rows")), ("attention_causal.cuh", ("causal_attention_rows",)),
                          ("attention_causal_few.cuh", ("causal_attention_few", "causal_few_join")),
                          ("attention_causal_tcgen05.cuh", ("causal_attention_tcgen05", "causal_join"))):
        for kernel in kernels:
            head, _, rest = _kernel(sources[name], kernel).partition("ptx::pdl_wait();")
            assert rest, kernel
            assert not re.search(r"\bp\.(c\.)?\w+\[|\*p\.|causal_(cu|ctx|request|divide)\(|tma_load", head), kernel
    assert len(re.findall(r"\blaunch\(k::", sources["serving.cu"])) >= 9 and "<<<" not in sources["serving.cu"]


def test_each_producer_has_a_ring_of_its_own():
    # two producers of one ring could be two phases of a barrier apart, where parities look alike.  In the few-row kernel both fill the stages of one ring,
    # but each waits for every phase of the stage's one barrier in turn, on a full barrier of its own
    sources = dict(_sources())
    text = sources["attention_causal_tcgen05.cuh"]
    assert re.search(r"full = is_k \? k_full : v_full;\s*uint64_t\* free_ = is_k \? k_free : v_free;\s*uint8_t\* ring = is_k \? sK : sV;\s*const int stages = is_k \? KS : VS;", text)
    assert text.count("mbar_wait_warp(&free_[stage], (use - 1) & 1, dead)") == 1
    text = sources["attention_causal_few.cuh"]
    assert re.search(r"full = is_k \? k_full : v_full;\s*uint8_t\* ring = is_k \? sK : sV;", text)
    assert text.count("if (use > 0) ptx::mbar_wait_warp(&freed[stage], (use - 1) & 1, dead);") == 1


def test_registers_are_shared_out_of_what_the_cta_has():
    sources = dict(_sources())
    text = sources["attention_causal_tcgen05.cuh"]
    assert "static_assert(2 * CTC_REGS_SOFTMAX + CTC_REGS_OTHERS == 3 * CTC_REGS" in text and "CTC_THREADS = 384" in text
    assert re.search(r"at\.numRegs != regs\) e = cudaErrorInvalidKernelImage", sources["serving.cu"])
    assert "CtcShape<DP>::SMEM, k::CTC_REGS, done)" in sources["serving.cu"]


def test_scores_are_overwritten_only_behind_their_product():
    # P lies over S: the order of two MMAs on different accumulators is not documented, so S is issued behind the commit of the product before
    text = dict(_sources())["attention_causal_tcgen05.cuh"]
    issue = text[text.index("auto issue_s ="):text.index("auto issue_o =")]
    assert issue.index("mbar_wait_lanes(&o_full[t], (n - 1) & 1, dead)") < issue.index("ptx::mma_bf16(one")
