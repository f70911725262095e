"""MI355X-native Group Shifted Window Attention (GSWA) layer, forward and backward.

``paper_2409_06206_amd.gswa`` is the thin binding over the C-ABI HIP library; ``astl`` (whole layers and
sequences of them), ``lnorm`` (LayerNorm of rows), ``relpos`` (relative position bias by buckets) and ``adamw``
(AdamW over many tensors) bind the rest of it, and ``runner`` owns buffers around them;
``paper_2409_06206_amd.synth`` draws the seeded synthetic inputs.  Importing the
package loads nothing; the HIP library is loaded on the first call and its
absence is an error, never a fallback.
"""
