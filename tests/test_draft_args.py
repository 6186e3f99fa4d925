"""What the entry points of drafted decoding refuse, before anything reaches a device (host only)."""
import pytest

from paper_2505_10951_amd import sgc

E, S, T, U = sgc.SGC_EINVAL, sgc.SGC_ESHAPE, sgc.SGC_ESTATE, sgc.SGC_EUNSUPPORTED


def _plan(suffix=(4, 4), prefix=(32, 48), **kw):
    args = dict(n_q_heads=8, n_kv_heads=2, head_dim=128, n_layers=2, io_dtype="bf16", rope_base=10000.0)
    params = sgc.make_params(**{**args, **kw})
    ctx = sgc.sgc_ctx_create(params)
    nbytes = sgc.sgc_cache_pool_bytes(params, 64)
    cache = sgc.sgc_cache_create(ctx, 0x7F0000000000, nbytes, len(prefix))          # (never dereferenced)
    for c, p in enumerate(prefix):
        sgc.sgc_cache_alloc_cluster(ctx, cache, c, p)
    plan = sgc.sgc_assign_clusters(ctx, cache, [i % len(prefix) for i in range(len(suffix))], list(suffix), len(prefix))[3]
    return ctx, cache, plan


def _refused(fn, status):
    with pytest.raises(sgc.SgcError) as e:
        fn()
    assert e.value.status == status, str(e.value)


def test_draft_entry_points():
    ctx, cache, plan = _plan()
    step = lambda *a: sgc.sgc_draft_step_batched(ctx, cache, plan, *a)
    _refused(lambda: step(0, 256, None, 512, 768, 1024, 1280), T)                  # not enabled
    for cap, rows in ((8, 0), (8, 17), (3, 4), (0, 1), (5000, 4), (1100, 4)):
        _refused(lambda: sgc.sgc_plan_enable_drafts(ctx, plan, cap, rows), E)
    _refused(lambda: step(0, 256, None, 512, 768, 1024, 1280), T)                  # still not
    sgc.sgc_plan_enable_drafts(ctx, plan, 32, 5)
    _refused(lambda: step(2, 256, None, 512, 768, 1024, 1280), E)                  # layer range
    _refused(lambda: step(-1, 256, None, 512, 768, 1024, 1280), E)
    _refused(lambda: step(0, 256, None, 512, 768, 1024, 1280), T)                  # no suffix prefill has run
    _refused(lambda: sgc.sgc_draft_step_batched(ctx, None, plan, 0, 256, None, 512, 768, 1024, 1280), E)
    _refused(lambda: sgc.sgc_draft_step_batched(ctx, cache, None, 0, 256, None, 512, 768, 1024, 1280), E)
    other, other_cache, other_plan = _plan()
    _refused(lambda: sgc.sgc_draft_step_batched(ctx, cache, other_plan, 0, 256, None, 512, 768, 1024, 1280), E)
    _refused(lambda: sgc.sgc_plan_enable_drafts(ctx, None, 32, 5), E)
    for x in ((ctx, cache, plan), (other, other_cache, other_plan)):
        sgc.sgc_plan_destroy(x[2])
        sgc.sgc_cache_destroy(x[1])
        sgc.sgc_ctx_destroy(x[0])


@pytest.mark.parametrize("kw", [dict(head_dim=64), dict(io_dtype="f32"), dict(kernel=sgc.SGC_KERNEL_GENERIC)])
def test_drafts_need_the_matrix_core_path(kw):
    ctx, cache, plan = _plan(**kw)
    _refused(lambda: sgc.sgc_plan_enable_drafts(ctx, plan, 32, 5), U)
    sgc.sgc_plan_destroy(plan)
    sgc.sgc_cache_destroy(cache)
    sgc.sgc_ctx_destroy(ctx)


def test_drafts_fit_the_own_keys():
    ctx, cache, plan = _plan(suffix=(1000, 4))
    _refused(lambda: sgc.sgc_plan_enable_drafts(ctx, plan, 25, 5), E)              # 1025 own keys
    sgc.sgc_plan_enable_drafts(ctx, plan, 24, 5)
    sgc.sgc_plan_destroy(plan)
    sgc.sgc_cache_destroy(cache)
    sgc.sgc_ctx_destroy(ctx)


def test_token_probs():
    ok = dict(n_rows=2000, vocab=100, dev_logits=256, logits_dtype=sgc.SGC_F32, logits_stride=100, temperature=1.0, dev_probs=512, probs_stride=100)
    few = dict(ok, n_rows=2, vocab=100000, logits_stride=100000, probs_stride=100000)
    need = sgc.sgc_token_probs_workspace(2, 100000)
    assert need > 0 and sgc.sgc_token_probs_workspace(2000, 100) == 0
    assert sgc.sgc_token_probs_workspace(0, 100) == 0 and sgc.sgc_token_probs_workspace(-1, 100) == 0 and sgc.sgc_token_probs_workspace(5, 0) == 0
    for kw, status in ((dict(ok, n_rows=-1), E), (dict(ok, n_rows=1 << 31), E), (dict(ok, vocab=0), E), (dict(ok, logits_dtype=sgc.SGC_FP8_E4M3), U),
                       (dict(ok, temperature=-1.0), E), (dict(ok, temperature=float("nan")), E), (dict(ok, temperature=float("inf")), E),
                       (dict(ok, logits_stride=99), S), (dict(ok, probs_stride=99), S), (dict(ok, dev_logits=None), E), (dict(ok, dev_probs=None), E),
                       (dict(ok, dev_logits=258), E), (dict(ok, dev_probs=514), E), (few, E), (dict(few, dev_workspace=1024, workspace_bytes=need - 1), E),
                       (dict(few, dev_workspace=1028, workspace_bytes=need), E), (dict(ok, dev_logits=257, logits_dtype=sgc.SGC_BF16), E)):
        _refused(lambda: sgc.sgc_token_probs(None, **kw), status)
    sgc.sgc_token_probs(None, **dict(ok, n_rows=0, dev_logits=None, dev_probs=None))            # nothing to do


def test_verify_drafts():
    ok = dict(n_queries=3, max_rows=4, vocab=100, dev_target=256, target_stride=100, dev_draft=None, draft_stride=0, dev_tokens=512, dev_rows=None,
              dev_uniform=768, dev_out_tokens=1024, dev_accepted=1280)
    for kw, status in ((dict(ok, n_queries=-1), E), (dict(ok, max_rows=0), E), (dict(ok, max_rows=17), E), (dict(ok, vocab=0), E),
                       (dict(ok, target_stride=99), S), (dict(ok, dev_draft=256, draft_stride=99), S), (dict(ok, dev_target=None), E),
                       (dict(ok, dev_tokens=None), E), (dict(ok, dev_uniform=None), E), (dict(ok, dev_out_tokens=None), E),
                       (dict(ok, dev_accepted=None), E), (dict(ok, dev_target=258), E), (dict(ok, dev_tokens=513), E), (dict(ok, dev_done=514), E)):
        _refused(lambda: sgc.sgc_verify_drafts(None, **kw), status)
    sgc.sgc_verify_drafts(None, **dict(ok, n_queries=0))


def test_project_fp8():
    need = sgc.sgc_project_fp8_workspace(3, 40, 256)
    assert need > 0 and sgc.sgc_project_fp8_workspace(0, 40, 256) == 0 and sgc.sgc_project_fp8_workspace(3, -1, 256) == 0
    ok = dict(dev_x=256, x_dtype=sgc.SGC_BF16, x_stride=256, n_rows=3, dev_codes=512, dev_exponents=768, n_features=40, d_model=256, dev_y=1024,
              y_dtype=sgc.SGC_BF16, y_stride=40, dev_workspace=2048, workspace_bytes=need)
    for kw, status in ((dict(ok, x_dtype=sgc.SGC_FP8_E4M3), U), (dict(ok, y_dtype=7), U), (dict(ok, n_features=0), E), (dict(ok, d_model=0), E),
                       (dict(ok, d_model=250, x_stride=256), E), (dict(ok, n_rows=-1), E), (dict(ok, x_stride=255), S), (dict(ok, y_stride=39), S),
                       (dict(ok, x_stride=257), E), (dict(ok, dev_x=None), E), (dict(ok, dev_codes=None), E), (dict(ok, dev_exponents=None), E),
                       (dict(ok, dev_y=None), E), (dict(ok, dev_x=264), E), (dict(ok, dev_codes=520), E), (dict(ok, dev_y=1025), E),
                       (dict(ok, dev_workspace=None), E), (dict(ok, workspace_bytes=need - 1), E), (dict(ok, dev_workspace=2056), E)):
        _refused(lambda: sgc.sgc_project_fp8(None, **kw), status)
    sgc.sgc_project_fp8(None, **dict(ok, n_rows=0, dev_x=None))
    w = dict(dev_w=256, w_dtype=sgc.SGC_BF16, n_features=40, d_model=256, dev_codes=512, dev_exponents=768)
    for kw, status in ((dict(w, w_dtype=sgc.SGC_FP8_E4M3), U), (dict(w, n_features=0), E), (dict(w, d_model=8), E), (dict(w, dev_w=None), E),
                       (dict(w, dev_codes=None), E), (dict(w, dev_exponents=None), E), (dict(w, dev_w=260), E)):
        _refused(lambda: sgc.sgc_quantise_weight_fp8(None, **kw), status)
